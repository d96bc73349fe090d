"""Every kernel of the sequence operators on another stream, in a replayed graph, again on the same inputs, and
with the others at the same time on streams of their own: the same bits each time.  The losses' values do not
depend on whether a gradient is asked for."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def simx():
    from paper_2607_05272_gb300 import build as B
    B.build()
    from paper_2607_05272_gb300 import simx
    return simx


def _ws(size):
    return torch.empty(size, dtype=torch.uint8, device="cuda")


def _gen(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s: torch.randn(s, generator=g, device="cuda")


def _token(simx, n, V, dtype="f32", want=True):
    r = _gen(n + V)
    logits = (2 * r(n, V)).to(DT[dtype])
    action = (r(n).abs() * 1e6).long() % V
    lp = logits.float().log_softmax(1).gather(1, action[:, None])[:, 0]
    kw = dict(logp_old=lp + 0.1 * r(n), logp_ref=lp + 0.2 * r(n), weight=(r(n) > -1.0).float() / n)
    adv, ws = r(n), _ws(simx.token_loss_grad_workspace_size(n))
    out = dict(stats=torch.empty(5, device="cuda"), logp=torch.empty(n, device="cuda"),
               entropy=torch.empty(n, device="cuda"), grad=torch.empty_like(logits) if want else None)
    stats = out["stats"]
    rest = {k: v for k, v in out.items() if k != "stats"}
    return [v for v in out.values() if v is not None], lambda s=None: simx.token_loss_grad(
        logits, action, adv, stats, ws, c_kl=0.1, c_entropy=0.02, temperature=0.8, stream=s, **kw, **rest)


def _pref(simx, lengths, V, dtype="f32", want=True):
    n, pairs = sum(lengths), len(lengths) // 2
    r = _gen(n + V + 1)
    logits, token = (2 * r(n, V)).to(DT[dtype]), (r(n).abs() * 1e6).long() % V
    start = torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)])).cuda()
    kw = dict(logp_ref=r(n) - 5.0, mask=(r(n) > -0.5).to(torch.uint8), weight=r(pairs).abs())
    ws = _ws(simx.preference_loss_grad_workspace_size(n, pairs))
    stats, grad = torch.empty(3, device="cuda"), torch.empty_like(logits) if want else None
    ratio, margin = torch.empty(2 * pairs, device="cuda"), torch.empty(pairs, device="cuda")
    return [v for v in (stats, ratio, margin, grad) if v is not None], lambda s=None: simx.preference_loss_grad(
        logits, token, start, stats, ws, grad=grad, ratio=ratio, margin=margin, label_smoothing=0.1, stream=s, **kw)


def _scan(simx, B, T, C, dtype="f32"):
    r = _gen(B + T + C)
    x, gate, dh = (v.to(DT[dtype]) for v in (r(B, T, C), 1.5 * r(B, T, C) + 2.0, r(B, T, C)))
    bias, h0, dh_last, done = r(C), r(B, C), r(B, C), (r(B, T) > 2.5).to(torch.uint8)
    h, dx, dg = (torch.empty_like(x) for _ in range(3))
    last, d0, db = torch.empty_like(h0), torch.empty_like(h0), torch.empty_like(bias)
    ws = _ws(simx.gated_scan_workspace_size(B, T, C))

    def run(s=None):
        simx.gated_scan(x, gate, h, bias=bias, h0=h0, done=done, h_last=last, stream=s)
        simx.gated_scan_grad(x, gate, h, dh, dx, dg, ws, bias=bias, h0=h0, done=done, dh_last=dh_last, dbias=db,
                             dh0=d0, stream=s)
    return [h, dx, dg, last, d0, db], run


def _norm(simx, n, W, dtype="f32"):
    r = _gen(n + W)
    x, res, dy, dz = (r(n, W).to(DT[dtype]) for _ in range(4))
    gain, kw = r(W), dict(p=0.2, seed=11, step=3)
    z, y, dx, dr = (torch.empty_like(x) for _ in range(4))
    rstd, dgain = torch.empty(n, device="cuda"), torch.empty(W, device="cuda")
    ws = _ws(simx.dropout_add_norm_grad_workspace_size(n, W))

    def run(s=None):
        simx.dropout_add_norm(x, gain, y, residual=res, z=z, rstd=rstd, stream=s, **kw)
        simx.dropout_add_norm_grad(z, gain, rstd, dy, dx, ws, dz=dz, dresidual=dr, dgain=dgain, stream=s, **kw)
    return [z, y, rstd, dx, dr, dgain], run


CALLS = {
    "token lanes": lambda s: _token(s, 3000, 48),
    "token one warp": lambda s: _token(s, 500, 400, "bf16"),
    "token streamed": lambda s: _token(s, 400, 5003, "bf16"),
    "token clusters": lambda s: _token(s, 6, 70000, "bf16"),
    "preference": lambda s: _pref(s, [30, 20, 0, 17, 25, 25], 4099),
    "preference bf16": lambda s: _pref(s, [9, 12], 40001, "bf16"),
    "scan columns": lambda s: _scan(s, 300, 3, 64),
    "scan tiles": lambda s: _scan(s, 700, 40, 64),
    "scan narrow": lambda s: _scan(s, 6, 700, 5, "bf16"),
    "scan clusters": lambda s: _scan(s, 1, 6000, 64, "bf16"),
    "scan clusters of elements": lambda s: _scan(s, 1, 5000, 67, "bf16"),
    "norm rows of a warp": lambda s: _norm(s, 3000, 64),
    "norm aligned": lambda s: _norm(s, 900, 2048, "bf16"),
    "norm off the grid": lambda s: _norm(s, 900, 2047, "bf16"),
}


def _forget(outs):
    for o in outs:
        o.zero_()


@pytest.mark.parametrize("name", list(CALLS))
def test_other_stream_graph_and_again(simx, name):
    outs, run = CALLS[name](simx)
    run()
    torch.cuda.synchronize()
    ref = [o.clone() for o in outs]
    assert all(torch.isfinite(o).all() for o in ref) and any(o.any() for o in ref)
    _forget(outs)
    run()
    assert all(torch.equal(a, b) for a, b in zip(outs, ref))
    _forget(outs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    run(side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="relaxed"):
        run()
    for _ in range(2):
        _forget(outs)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, ref))


def test_all_at_once(simx):
    """Every call on a stream of its own, with a workspace of its own, over and over."""
    made = [f(simx) for f in CALLS.values()]
    for _, run in made:
        run()
    torch.cuda.synchronize()
    ref = [[o.clone() for o in outs] for outs, _ in made]
    for outs, _ in made:
        _forget(outs)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in made]
    for _ in range(8):
        for (_, run), s in zip(made, streams):
            run(s.cuda_stream)
    torch.cuda.synchronize()
    for name, (outs, _), want in zip(CALLS, made, ref):
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,V", [(9, 7), (70, 48), (70, 300), (40, 700), (40, 5000), (5, 40000), (5, 131072), (24, 70001)])
def test_token_values_alone(simx, n, V, dtype):
    (stats, lp, H, _), run = _token(simx, n, V, dtype)
    values, alone = _token(simx, n, V, dtype, want=False)
    run()
    alone()
    torch.cuda.synchronize()
    assert torch.isfinite(stats).all() and all(torch.equal(a, b) for a, b in zip((stats, lp, H), values))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5, 300, 5000, 70001])
def test_preference_values_alone(simx, V, dtype):
    (*ref, _), run = _pref(simx, [4, 7, 0, 3], V, dtype)
    values, alone = _pref(simx, [4, 7, 0, 3], V, dtype, want=False)
    run()
    alone()
    torch.cuda.synchronize()
    assert torch.isfinite(ref[0]).all() and all(torch.equal(a, b) for a, b in zip(ref, values))
