"""The token loss and the preference loss against their 64-bit definitions (oracle/seq.py).

Tolerances.  In fp32, with |x - m| / T at most 40 here: the exponent's argument carries two
roundings of a number up to 58 (5e-6 of e^x at most), ex2 and the sums about 1e-6 more, so a
probability is off by at most 1e-5 of itself, a log probability by 1e-5 (1 + |lp|), and a ratio by
as much of itself.  The oracle's `scale` is the sum of the absolute terms that each gradient adds,
with the factor 1 + |lp| where a ratio enters; gradients and statistics are held to 2e-5 of it, and a
bf16 output to half a unit in its last place (8 significant bits: at most 2^-8 of itself) on top.
"""
import math

import numpy as np
import pytest

from oracle import seq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TOL = 2e-5
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def simx():
    from paper_2607_05272_gb300 import build as B
    B.build()
    from paper_2607_05272_gb300 import simx
    return simx


def _dev(a, dtype=torch.float32):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def _rows(values, dtype, ld, offset):
    """values [n, V] on the device as rows of stride ld that start `offset` elements in."""
    n, V = values.shape
    buf = torch.full((offset + n * ld + 8,), float("nan"), dtype=DT[dtype], device="cuda")
    view = buf[offset:offset + n * ld].view(n, ld)[:, :V] if n else buf[:0].view(0, V)
    view.copy_(torch.from_numpy(values).to(DT[dtype]))
    return view


def _f64(t):
    return t.detach().double().cpu().numpy()


def _close(got, ref, scale, dtype="f32"):
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    bad = ~(np.abs(got - ref) <= TOL * scale + half * np.abs(ref) + 1e-37)
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4], np.broadcast_to(scale, got.shape)[bad][:4])


def _token(simx, x, action, ld=None, offset=0, dtype="f32", inplace=False, want=True, **kw):
    n, V = x.shape
    logits = _rows(x, dtype, ld or V, offset)
    grad = (logits if inplace else _rows(np.full((n, V), 7.0), dtype, ld or V, offset)) if want else None
    ws = torch.empty(simx.token_loss_grad_workspace_size(n), dtype=torch.uint8, device="cuda")
    stats = torch.empty(5, device="cuda")
    lp, H = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    exact = _f64(logits)
    simx.token_loss_grad(logits, _dev(action, torch.int64), kw.pop("adv", None), stats, ws,
                         grad=grad, logp=lp, entropy=H, **kw)
    torch.cuda.synchronize()
    return exact, None if grad is None else _f64(grad), _f64(stats), _f64(lp), _f64(H)


def _inputs(n, V, seed, masked=0.3):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, V)) * 2
    action = rng.integers(0, V, n)
    lp = np.take_along_axis(seq.log_softmax(x), action[:, None], 1)[:, 0]
    old = lp + rng.standard_normal(n) * 0.25
    # off the clip edges, where the loss has a kink (bf16 logits move lp, so by a wide margin)
    w = rng.random(n) * (rng.random(n) >= masked)
    return (x, action, dict(adv=rng.standard_normal(n), logp_old=old,
                            logp_ref=lp + rng.standard_normal(n) * 0.2, weight=w))


def _check_token(simx, n, V, dtype, seed, ld=None, offset=0, inplace=False, **par):
    x, action, kw = _inputs(n, V, seed)
    x = _f64(torch.from_numpy(x).to(DT[dtype]))
    par = dict(dict(clip_low=0.2, clip_high=0.3, c_kl=0.1, c_entropy=0.02, temperature=1.0), **par)
    # ratios within 1e-3 of a clip edge are moved off it
    lp = np.take_along_axis(seq.log_softmax(x, par["temperature"]), action[:, None], 1)[:, 0]
    d = lp - kw["logp_old"]
    for e in (math.log1p(-par["clip_low"]), math.log1p(par["clip_high"])):
        d = np.where(np.abs(d - e) < 1e-3, e + 1e-3, d)
    kw["logp_old"] = lp - d
    k32 = {k: v.astype(np.float32).astype(np.float64) for k, v in kw.items()}
    exact, grad, stats, glp, H = _token(simx, x, action, ld, offset, dtype, inplace,
                                        **{k: _dev(v) for k, v in kw.items()}, **par)
    ref = seq.token_loss(exact, action, **k32, **par)
    _close(grad, ref["grad"], ref["scale"], dtype)
    _close(stats, ref["stats"], ref["stats_scale"])
    _close(glp, ref["logp"], 1 + np.abs(ref["logp"]))
    _close(H, ref["entropy"], 1 + np.abs(ref["entropy"]))
    assert not grad[kw["weight"] == 0].any()


VOCABS = [1, 2, 3, 31, 32, 33, 48, 64, 65, 127, 129, 255, 256, 257, 511, 700, 1000, 1023, 1024, 1025,
          2047, 2049, 4095, 4096, 4099, 8191, 8193, 12289, 16383, 16384, 16385]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", VOCABS)
def test_token_vocabularies(simx, V, dtype):
    _check_token(simx, 9, V, dtype, V)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [32768, 50001, 65537, 131071, 131072, 262144, 270001])
def test_token_large_vocabularies(simx, V, dtype):
    _check_token(simx, 3, V, dtype, V)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,ld,offset", [(48, 51, 1), (48, 56, 8), (333, 333, 3), (1000, 1024, 0), (4099, 4101, 5),
                                         (20001, 20003, 1), (70000, 70008, 8)])
def test_token_strides_and_alignment(simx, V, ld, offset, dtype):
    _check_token(simx, 5, V, dtype, V + ld, ld=ld, offset=offset, temperature=0.7)


@pytest.mark.parametrize("V", [40, 3000, 40000, 270001])
def test_token_gradient_in_place(simx, V):
    _check_token(simx, 6, V, "f32", V, inplace=True)
    _check_token(simx, 6, V, "bf16", V, inplace=True, c_entropy=0.0)


@pytest.mark.parametrize("V", [40, 3000, 40000])
def test_token_gradient_of_other_alignment(simx, V):
    """Logits and gradient rows that start at different places within 16 bytes."""
    x, action, kw = _inputs(5, V, V)
    for dtype in ("f32", "bf16"):
        logits = _rows(x, dtype, V, 0)
        grad = _rows(np.zeros((5, V)), dtype, V + 1, 1)
        ws = torch.empty(simx.token_loss_grad_workspace_size(5), dtype=torch.uint8, device="cuda")
        stats = torch.empty(5, device="cuda")
        simx.token_loss_grad(logits, _dev(action, torch.int64), _dev(kw["adv"]), stats, ws, grad=grad)
        torch.cuda.synchronize()
        ref = seq.token_loss(_f64(logits), action, kw["adv"].astype(np.float32).astype(np.float64))
        _close(_f64(grad), ref["grad"], ref["scale"], dtype)


@pytest.mark.parametrize("n,V", [(1, 48), (1, 5000), (1, 100000), (20000, 5), (3000, 100), (5000, 1500), (700, 20000)])
def test_token_row_counts(simx, n, V):
    """From one row to more rows than blocks: the loss and a few rows against the definition."""
    g = torch.Generator(device="cuda").manual_seed(n)
    logits = torch.randn((n, V), generator=g, device="cuda") * 2
    action = torch.randint(0, V, (n,), generator=g, device="cuda")
    adv = torch.randn(n, generator=g, device="cuda")
    ws = torch.empty(simx.token_loss_grad_workspace_size(n), dtype=torch.uint8, device="cuda")
    stats, grad = torch.empty(5, device="cuda"), torch.empty_like(logits)
    simx.token_loss_grad(logits, action, adv, stats, ws, grad=grad, c_entropy=0.01)
    lp = logits.double().log_softmax(1)
    ent = -(lp.exp() * lp).sum(1)
    pol = -adv.double().mean().item()  # on-policy: rho = 1
    assert abs(stats[1].item() - pol) <= TOL * adv.double().abs().mean().item() * 1.0 + 1e-12
    assert abs(stats[3].item() - ent.mean().item()) <= TOL * (1 + ent.mean().item())
    rows = np.unique(np.linspace(0, n - 1, 7).astype(int))
    r = torch.from_numpy(rows).cuda()
    ref = seq.token_loss(_f64(logits[r]), action[r].cpu().numpy(), _f64(adv[r]), weight=np.full(len(rows), 1.0 / n),
                         c_entropy=0.01)
    _close(_f64(grad[r]), ref["grad"], ref["scale"])


def test_token_optional_terms(simx):
    x, action, kw = _inputs(7, 90, 1)
    x = x.astype(np.float32).astype(np.float64)
    adv = kw["adv"].astype(np.float32).astype(np.float64)
    for par in (dict(), dict(c_entropy=0.5), dict(adv=adv), dict(adv=adv, c_kl=2.0)):
        dev = {k: _dev(v) if k == "adv" else v for k, v in par.items()}
        exact, grad, stats, lp, H = _token(simx, x, action, **dev)
        ref = seq.token_loss(exact, action, **par)
        _close(grad, ref["grad"], ref["scale"] + 1e-9)
        _close(stats, ref["stats"], ref["stats_scale"] + 1e-9)
    # without a gradient the values are the same
    _, none, s2, lp2, H2 = _token(simx, x, action, want=False, **dev)
    assert none is None and np.array_equal(s2, stats) and np.array_equal(lp2, lp) and np.array_equal(H2, H)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [50, 700, 5000, 40000])
def test_token_extreme_logits(simx, V, dtype):
    low = torch.finfo(DT[dtype]).min
    rng = np.random.default_rng(V)
    x = rng.standard_normal((6, V))
    x[0, 1:] = -np.inf                    # one token left: probability 1
    x[1, ::2] = low                       # masked with the lowest value
    x[2, :] = low                         # nothing but the lowest value: uniform
    x[3, ::3] = -np.inf
    x[4, :V // 2] = 3e38                  # the difference to the others overflows
    x[4, V // 2:] = -3e38
    action = np.array([0, 1, 3, 1, 2, V - 1])
    adv = np.ones(6)
    exact, grad, stats, lp, H = _token(simx, x, action, dtype=dtype, adv=_dev(adv), c_entropy=0.1, temperature=0.5)
    x = np.clip(exact, -1e30, 1e30)       # the same probabilities, within what 64-bit exp takes
    x[2], x[4] = 0.0, np.where(np.arange(V) < V // 2, 0.0, -np.inf)
    with np.errstate(over="ignore"):
        ref = seq.token_loss(x, action, adv, c_entropy=0.1, temperature=0.5)
    _close(grad, ref["grad"], ref["scale"], dtype)
    _close(lp, ref["logp"], 1 + np.abs(ref["logp"]))
    _close(H, ref["entropy"], 1 + np.abs(ref["entropy"]))
    _close(stats, ref["stats"], ref["stats_scale"])


@pytest.mark.parametrize("V", [50, 700, 5000, 40000])
def test_token_rows_without_weight_are_not_read(simx, V):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, V))
    x[0], x[2], x[4, 3] = np.nan, -np.inf, np.inf
    action = np.array([-100, 3, 10 ** 12, 4, V])
    w = np.array([0.0, 0.7, 0.0, 0.0, 0.0])
    _, grad, stats, lp, H = _token(simx, x, action, adv=_dev(np.ones(5)), weight=_dev(w), c_entropy=0.1)
    ref = seq.token_loss(x[1:2].astype(np.float32).astype(np.float64), action[1:2], np.ones(1),
                         weight=w[1:2].astype(np.float32).astype(np.float64), c_entropy=0.1)
    assert not grad[[0, 2, 3, 4]].any() and not lp[[0, 2, 3, 4]].any() and not H[[0, 2, 3, 4]].any()
    _close(grad[1:2], ref["grad"], ref["scale"])
    _close(stats, ref["stats"], ref["stats_scale"])
    _, grad, stats, _, _ = _token(simx, x, action, adv=_dev(np.ones(5)), weight=_dev(np.zeros(5)))
    assert not grad.any() and not stats.any()


@pytest.mark.parametrize("V", [50, 700, 5000, 40000])
def test_token_bad_rows_give_nan(simx, V):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, V))
    x[0, 1], x[1, V - 1] = np.nan, np.inf
    x[2] = -np.inf
    action = np.array([2, 2, 2, V, -1])
    _, grad, stats, lp, _ = _token(simx, x, action, adv=_dev(np.ones(5)))
    assert np.isnan(grad).all() and np.isnan(stats[0]) and np.isnan(lp).all()


def test_token_loss_is_the_same_bits_every_run(simx):
    for V in (48, 5000, 60000):
        x, action, kw = _inputs(400 if V < 60000 else 40, V, 9)
        dev = {k: _dev(v) for k, v in kw.items()}
        a = _token(simx, x, action, **dev, c_kl=0.1)
        b = _token(simx, x, action, **dev, c_kl=0.1)
        assert all(np.array_equal(p, q) for p, q in zip(a, b))


def test_token_loss_moves_as_its_gradient_says(simx):
    """The loss along a direction, by differences: L changes by step * <grad, v> up to the second
    order (step^2, curvature of order |v|^2) and the fp32 rounding of L."""
    x, action, kw = _inputs(32, 200, 5, masked=0.0)
    kw["weight"] = np.full(32, 1 / 32)
    kw["logp_old"] = np.take_along_axis(seq.log_softmax(x), action[:, None], 1)[:, 0]  # ratios of 1
    v = np.random.default_rng(2).standard_normal(x.shape)
    dev = {k: _dev(t) for k, t in kw.items()}
    par = dict(clip_low=10.0, clip_high=10.0, c_kl=0.1, c_entropy=0.05)
    step = 1e-3
    _, grad, _, _, _ = _token(simx, x, action, **dev, **par)
    up = _token(simx, x + step * v, action, **dev, **par)[2][0]
    down = _token(simx, x - step * v, action, **dev, **par)[2][0]
    slope = (grad * v).sum()
    # L is about 0.3: fp32 rounding of both sides over 2 step; third-order term step^2
    assert abs((up - down) / (2 * step) - slope) <= 4 * 6e-8 / step + 100 * step ** 2 * (1 + abs(slope))


def test_token_empty(simx):
    _, grad, stats, _, _ = _token(simx, np.zeros((0, 17)), np.zeros(0, np.int64))
    assert not stats.any()


def test_token_on_another_stream_and_in_a_graph(simx):
    x, action, kw = _inputs(64, 3000, 8)
    logits, act, adv = _rows(x, "f32", 3000, 0), _dev(action, torch.int64), _dev(kw["adv"])
    ws = torch.empty(simx.token_loss_grad_workspace_size(64), dtype=torch.uint8, device="cuda")
    ref_s, ref_g = torch.empty(5, device="cuda"), torch.empty_like(logits)
    simx.token_loss_grad(logits, act, adv, ref_s, ws, grad=ref_g)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    s2, g2 = torch.empty(5, device="cuda"), torch.empty_like(logits)
    side.wait_stream(torch.cuda.current_stream())
    simx.token_loss_grad(logits, act, adv, s2, ws, grad=g2, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(s2, ref_s) and torch.equal(g2, ref_g)
    s3, g3 = torch.empty(5, device="cuda"), torch.empty_like(logits)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="relaxed"):
        simx.token_loss_grad(logits, act, adv, s3, ws, grad=g3)
    for _ in range(2):
        s3.zero_()
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(s3, ref_s) and torch.equal(g3, ref_g)


def _pref_case(lengths, V, seed, dtype, extra=0, mask_share=0.3):
    rng = np.random.default_rng(seed)
    start = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64) + (2 if extra else 0)
    n = int(start[-1]) + extra
    x = _f64(torch.from_numpy(rng.standard_normal((n, V)) * 2).to(DT[dtype]))
    token = rng.integers(0, V, n)
    lp = np.take_along_axis(seq.log_softmax(x), token[:, None], 1)[:, 0] if n else np.zeros(0)
    f = lambda v: v.astype(np.float32).astype(np.float64)  # noqa: E731
    return x, token, start, dict(logp_ref=f(lp + rng.standard_normal(n) * 0.3),
                                 mask=(rng.random(n) >= mask_share).astype(np.uint8),
                                 weight=f(rng.random(len(lengths) // 2) + 0.1))


def _pref(simx, x, token, start, kw, par, dtype, ld=None, offset=0, inplace=False):
    n, V = x.shape
    pairs = len(start) // 2
    logits = _rows(x, dtype, ld or V, offset)
    grad = logits if inplace else _rows(np.full((n, V), 7.0), dtype, ld or V, offset)
    ws = torch.empty(simx.preference_loss_grad_workspace_size(n, pairs), dtype=torch.uint8, device="cuda")
    ws.fill_(0xFF)
    stats, ratio, margin = torch.empty(3, device="cuda"), torch.empty(2 * pairs, device="cuda"), torch.empty(pairs, device="cuda")
    dev = {k: _dev(v, torch.uint8 if k == "mask" else torch.float32) for k, v in kw.items()}
    simx.preference_loss_grad(logits, _dev(token, torch.int64), _dev(start, torch.int64), stats, ws,
                              grad=grad, ratio=ratio, margin=margin, **dev, **par)
    torch.cuda.synchronize()
    return _f64(grad), _f64(stats), _f64(ratio), _f64(margin)


def _check_pref(simx, lengths, V, dtype, seed, extra=0, par=None, drop=(), **kw2):
    x, token, start, kw = _pref_case(lengths, V, seed, dtype, extra)
    for k in drop:
        kw[k] = None
    par = dict(dict(beta=0.2, label_smoothing=0.1, temperature=1.0), **(par or {}))
    grad, stats, ratio, margin = _pref(simx, x, token, start, kw, par, dtype, **kw2)
    ref = seq.preference_loss(x, token, start, beta=float(np.float32(par["beta"])),
                              smoothing=float(np.float32(par["label_smoothing"])), temperature=par["temperature"], **kw)
    _close(ratio, ref["ratio"], ref["ratio_scale"])
    _close(margin, ref["margin"], ref["margin_scale"])
    _close(stats, ref["stats"], ref["stats_scale"])
    _close(grad, ref["grad"], ref["scale"], dtype)
    return grad


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 33, 48, 200, 257, 1000, 1025, 4099, 16384, 16385, 50001, 131072, 270001])
def test_preference_vocabularies(simx, V, dtype):
    lengths = [3, 2, 1, 4] if V > 20000 else [3, 9, 0, 1, 5, 0, 17, 2]
    _check_pref(simx, lengths, V, dtype, V)


def test_preference_layouts(simx):
    for dtype in ("f32", "bf16"):
        _check_pref(simx, [3, 9, 4, 1], 333, dtype, 1, ld=335, offset=3)
        _check_pref(simx, [3, 9, 4, 1], 6000, dtype, 2, inplace=True)
        grad = _check_pref(simx, [3, 9, 4, 1], 48, dtype, 3, extra=5, inplace=True)
        assert not grad[:2].any() and not grad[-5:].any()  # rows of no sequence


@pytest.mark.parametrize("drop", [("mask",), ("logp_ref",), ("weight",), ("mask", "logp_ref", "weight")])
def test_preference_optional_arguments(simx, drop):
    _check_pref(simx, [5, 2, 3, 7], 70, "f32", 11, drop=drop, par=dict(label_smoothing=0.0, temperature=0.7))


def test_preference_many_pairs_and_long_sequences(simx):
    rng = np.random.default_rng(3)
    _check_pref(simx, list(rng.integers(0, 4, 2 * 300)), 9, "f32", 5)
    _check_pref(simx, [1500, 700, 300, 2000], 17, "f32", 6)


def test_preference_all_masked_and_empty(simx):
    x, token, start, kw = _pref_case([4, 4, 3, 5], 60, 7, "f32")
    kw["mask"][:] = 0
    x[:] = np.nan                                              # nothing is read
    token[:] = -1
    grad, stats, ratio, margin = _pref(simx, x, token, start, kw, dict(beta=0.3), "f32")
    assert not grad.any() and not ratio.any() and not margin.any()
    assert abs(stats[0] - math.log(2) * kw["weight"].sum()) <= 1e-6 * kw["weight"].sum()
    grad, stats, _, _ = _pref(simx, np.ones((3, 60)), np.zeros(3, np.int64), np.zeros(1, np.int64), {}, {}, "f32")
    assert not grad.any() and not stats.any()                  # no pairs
    _, stats, ratio, _ = _pref(simx, np.ones((0, 60)), np.zeros(0, np.int64), np.zeros(3, np.int64), {}, {}, "f32")
    assert abs(stats[0] - math.log(2)) <= 1e-6 and not ratio.any()  # no rows


def test_preference_bad_token_gives_nan_in_its_pair_only(simx):
    x, token, start, kw = _pref_case([4, 4, 3, 5], 60, 7, "f32")
    kw["mask"][:] = 1
    token[5] = 60
    grad, stats, ratio, margin = _pref(simx, x, token, start, kw, {}, "f32")
    assert np.isnan(grad[:8]).all() and np.isfinite(grad[8:]).all()
    assert np.isnan(stats[0]) and np.isnan(margin[0]) and np.isfinite(margin[1])


def test_preference_starts_outside_the_rows_are_taken_as_the_bounds(simx):
    x, token, _, kw = _pref_case([4, 4], 30, 7, "f32")
    a = _pref(simx, x, token, np.array([0, 4, 8]), kw, {}, "f32")
    b = _pref(simx, x, token, np.array([-5, 4, 10 ** 14]), kw, {}, "f32")
    assert all(np.array_equal(p, q) for p, q in zip(a, b))


def test_refusals(simx):
    x = torch.zeros((4, 10), device="cuda")
    act, adv, st = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(5, device="cuda")
    ws = torch.empty(simx.token_loss_grad_workspace_size(4), dtype=torch.uint8, device="cuda")

    def refused(f, *a, **kw):
        with pytest.raises(simx.SimxError) as e:
            f(*a, **kw)
        assert e.value.status == simx.EINVAL

    t = simx.token_loss_grad
    refused(t, x.half(), act, adv, st, ws)
    refused(t, x.cpu(), act, adv, st, ws)
    refused(t, x[0], act, adv, st, ws)
    refused(t, x.t(), act, adv, st, ws)
    refused(t, x, act.int(), adv, st, ws)
    refused(t, x, act[:3], adv, st, ws)
    refused(t, x, act, adv.double(), st, ws)
    refused(t, x, act, adv, st[:4], ws)
    refused(t, x, act, adv, st, ws[:16])
    refused(t, x, act, adv, st, None)
    refused(t, x, act, adv, st, ws, grad=x.bfloat16())
    refused(t, x, act, adv, st, ws, temperature=0.0)
    refused(t, x, act, adv, st, ws, temperature=float("nan"))
    refused(t, x, act, adv, st, ws, clip_low=-0.1)
    refused(t, x, act, adv, st, ws, c_kl=float("inf"))
    tok = torch.zeros(4, dtype=torch.int64, device="cuda")
    start = torch.tensor([0, 2, 4], device="cuda")
    ws2 = torch.empty(simx.preference_loss_grad_workspace_size(4, 1), dtype=torch.uint8, device="cuda")
    p = simx.preference_loss_grad
    refused(p, x, tok, start[:2], st[:3], ws2)
    refused(p, x, tok, start.int(), st[:3], ws2)
    refused(p, x, tok, start, st, ws2)
    refused(p, x, tok, start, st[:3], ws2[:8])
    refused(p, x, tok, start, st[:3], ws2, label_smoothing=1.5)
    refused(p, x, tok, start, st[:3], ws2, beta=float("nan"))
    refused(p, x, tok, start, st[:3], ws2, mask=torch.ones(4, device="cuda"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,V,ld", [(20, 70001, 70001), (20, 131072, 131072), (40, 33000, 33003)])
def test_token_rows_enough_to_stream(simx, n, V, ld, dtype):
    """Large vocabularies with more rows than go to clusters."""
    _check_token(simx, n, V, dtype, n + V, ld=ld)


@pytest.mark.parametrize("V", [70001, 131072])
def test_token_streamed_rows_at_the_edges(simx, V):
    """Masked, extreme, weightless and bad rows among streamed ones."""
    rng = np.random.default_rng(V)
    n, low = 24, float(np.finfo(np.float32).min)
    x = rng.standard_normal((n, V)) * 2
    x[0, 1:], x[1, ::2], x[2], x[3, ::3] = -np.inf, low, low, -np.inf
    x[4], x[5, 7], x[6] = np.nan, np.inf, -np.inf
    action = rng.integers(0, V, n)
    action[:4] = [0, 1, 3, 1]
    action[7] = -1
    w = np.full(n, 0.25)
    w[4:8] = 0.0
    exact, grad, stats, lp, H = _token(simx, x, action, adv=_dev(np.ones(n)), weight=_dev(w), c_entropy=0.1, temperature=0.5)
    z = np.clip(exact, -1e30, 1e30)
    z[2], z[4:8] = 0.0, 0.0
    action[4:8] = 0
    with np.errstate(over="ignore"):
        ref = seq.token_loss(z, action, np.ones(n), weight=w, c_entropy=0.1, temperature=0.5)
    _close(grad, ref["grad"], ref["scale"])
    _close(lp, ref["logp"], 1 + np.abs(ref["logp"]))
    _close(stats, ref["stats"], ref["stats_scale"])
    w[4:8] = 0.25
    action[7] = -1
    _, grad, stats, lp, _ = _token(simx, x, action, adv=_dev(np.ones(n)), weight=_dev(w))
    assert np.isnan(grad[4:8]).all() and np.isfinite(np.delete(grad, range(4, 8), 0)).all() and np.isnan(stats[0])


def test_preference_long_rows_extremes(simx):
    """-inf and lowest-value masks among the logits, temperature off 1, rows that are their own pair."""
    x, token, start, kw = _pref_case([2, 3, 1, 2], 40003, 19, "f32")
    kw["mask"][:] = 1
    keep = x[np.arange(len(token)), token].copy()
    x[:, ::3], x[1:4, 1::3] = -np.inf, -3e38
    x[np.arange(len(token)), token] = keep
    grad, stats, ratio, margin = _pref(simx, x, token, start, kw, dict(beta=0.2, temperature=0.8), "f32")
    z = np.maximum(_f64(torch.from_numpy(x).float()), -1e30)
    ref = seq.preference_loss(z, token, start, beta=float(np.float32(0.2)), temperature=float(np.float32(0.8)), **kw)
    _close(ratio, ref["ratio"], ref["ratio_scale"])
    _close(stats, ref["stats"], ref["stats_scale"])
    _close(grad, ref["grad"], ref["scale"])


@pytest.mark.parametrize("V", [50, 700, 5000, 131072])
def test_token_ratios_beyond_fp32(simx, V):
    """exp(lp - logp_old) and exp(logp_ref - lp) overflow fp32: an advantage of zero, a ratio that is clipped and a
    KL term of coefficient zero take nothing from them; only the KL itself is infinite."""
    x, action, kw = _inputs(3, V, V, masked=0.0)
    x = _f64(torch.from_numpy(x).float())
    f = lambda v: v.astype(np.float32).astype(np.float64)  # noqa: E731
    lp = np.take_along_axis(seq.log_softmax(x), action[:, None], 1)[:, 0]
    kw = dict(adv=np.array([0.0, 1.5, -0.5]), logp_old=f(lp - np.array([95.0, 95.0, 0.1])),
              logp_ref=f(lp + np.array([95.0, 0.1, 0.2])), weight=np.array([0.5, 0.25, 0.25]))
    par = dict(clip_low=0.2, clip_high=0.3, c_kl=0.0, c_entropy=0.02)
    _, grad, stats, glp, H = _token(simx, x, action, **{k: _dev(v) for k, v in kw.items()}, **par)
    ref = seq.token_loss(x, action, **kw, **par)
    # a clipped ratio adds nothing to the gradient and its bound to the loss, whatever the ratio
    size = seq.token_loss(x, action, **dict(kw, adv=np.array([0.0, 0.0, -0.5])), **par)
    _close(grad, ref["grad"], size["scale"])
    keep = [0, 1, 3, 4]
    _close(stats[keep], ref["stats"][keep], (size["stats_scale"] + 0.25 * 1.3 * 1.5)[keep])
    assert stats[2] == np.inf


@pytest.mark.parametrize("V", [60, 5000, 70000])
def test_preference_pairs_without_weight_count_for_nothing(simx, V):
    x, token, start, kw = _pref_case([4, 4, 3, 5], V, 7, "f32")
    kw["mask"][:] = 1
    kw["weight"][0] = 0.0
    ref = seq.preference_loss(x, token, start, beta=float(np.float32(0.1)), **kw)
    x[:3] = np.nan
    token[5] = -1
    grad, stats, ratio, margin = _pref(simx, x, token, start, kw, dict(beta=0.1), "f32")
    assert not grad[:8].any() and np.isnan(margin[0]) and np.isnan(ratio[:2]).all()
    _close(grad[8:], ref["grad"][8:], ref["scale"][8:])
    _close(stats, ref["stats"], ref["stats_scale"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [50, 300, 700, 5000, 40000, 70000])
def test_token_of_probability_zero(simx, V, dtype):
    """Actions whose logit is -inf: a ratio of 0 to an old policy takes nothing, on-policy and under a KL term
    the loss has no gradient there; no logit of -inf ever gets a finite one but 0."""
    rng = np.random.default_rng(V)
    x = rng.standard_normal((4, V))
    x[:, 3::5] = -np.inf
    action, adv = np.array([3, 3, 3, 0]), np.array([1.0, -1.0, 0.0, 0.5])
    par = dict(clip_low=0.2, clip_high=0.3, c_entropy=0.1)
    old = np.full(4, -2.0)
    exact, grad, stats, lp, H = _token(simx, x, action, dtype=dtype, adv=_dev(adv), logp_old=_dev(old), **par)
    fine = seq.token_loss(exact[3:], action[3:], adv[3:], old[3:], weight=np.full(1, 0.25), **par)
    rest = seq.token_loss(exact[:3], np.zeros(3, int), weight=np.full(3, 0.25), **par)  # their entropy alone
    assert np.isneginf(lp[:3]).all()
    _close(H[:3], rest["entropy"], 1 + rest["entropy"])
    _close(grad, np.concatenate([rest["grad"], fine["grad"]]), np.concatenate([rest["scale"], fine["scale"]]), dtype)
    assert not grad[:, 3::5].any()
    # min(0, 0.8) for the first, -0.8 clipped for the second
    _close(stats[1], fine["stats"][1] + 0.25 * 0.8, fine["stats_scale"][1] + 0.25)
    _close(stats[4], fine["stats"][4] + 0.25, fine["stats_scale"][4] + 0.25)
    _, grad, stats, _, _ = _token(simx, x, action, dtype=dtype, adv=_dev(adv), **par)
    fine = seq.token_loss(exact[3:], action[3:], adv[3:], weight=np.full(1, 0.25), **par)
    assert np.isnan(grad[:2]).all() and abs(stats[1] + 0.125) <= TOL
    _close(grad[2:], np.concatenate([rest["grad"][2:], fine["grad"]]), np.concatenate([rest["scale"][2:], fine["scale"]]), dtype)
    for c_kl in (0.0, 0.1):
        _, grad, stats, _, _ = _token(simx, x, action, dtype=dtype, adv=_dev(adv), logp_old=_dev(old), logp_ref=_dev(old),
                                      c_kl=c_kl, **par)
        assert np.isposinf(stats[2]) and np.isfinite(grad[3]).all()
        assert np.isnan(grad[:3]).all() if c_kl else np.isfinite(grad).all()
        assert np.isposinf(stats[0]) if c_kl else np.isfinite(stats[0])


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("V", [60, 5000, 70000])
def test_preference_token_of_probability_zero(simx, V, inplace):
    """In a preferred sequence the loss is infinite and only that row has no gradient; in the other one the pair is
    settled and takes nothing."""
    x, token, start, kw = _pref_case([3, 2, 2, 3], V, 7, "f32")
    kw["mask"][:] = 1
    x[1, token[1]] = x[8, token[8]] = -np.inf
    grad, stats, ratio, margin = _pref(simx, x, token, start, kw, dict(beta=0.2), "f32", inplace=inplace)
    assert np.isneginf(ratio[[0, 3]]).all() and np.isneginf(margin[0]) and np.isposinf(margin[1])
    assert np.isposinf(stats[0]) and np.isnan(grad[1]).all() and not grad[5:].any()
    c = -kw["weight"][0] * np.float64(np.float32(0.2))
    for i in (0, 2, 3, 4):
        p = np.exp(seq.log_softmax(x[i:i + 1])[0])
        hot = np.arange(V) == token[i]
        _close(grad[i], (c if i < 3 else -c) * (hot - p), abs(c) * (hot + p))
