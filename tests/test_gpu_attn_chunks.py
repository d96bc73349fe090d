"""Linear attention by chunks on the tensor cores: what only that form can get wrong."""
import numpy as np
import pytest

from oracle import attn
from tests.test_gpu_attn import _close, _state

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def simx():
    from paper_2607_05272_gb300 import build as B
    B.build()
    from paper_2607_05272_gb300 import simx
    return simx


def _ws(size):
    return torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")


def _f64(t):
    return t.detach().double().cpu().numpy()


def _call(simx, q, k, v, ld, s0=None, done=None, scale=None, ws=None, o=None, last=None):
    B, T, H, dk = q.shape
    Hk, dv = v.shape[2:]
    o = torch.empty((B, T, H, dv), dtype=q.dtype, device="cuda") if o is None else o
    last = torch.empty((B, H, dk, dv), device="cuda") if last is None else last
    ws = _ws(simx.decay_attention_workspace_size(B, T, H, Hk, dk, dv)) if ws is None else ws
    simx.decay_attention(q, k, v, o, ld, ws, scale=scale, s0=s0, done=done, s_last=last)
    return o, last


def _call_grad(simx, q, k, v, go, ld, s0=None, done=None, ds_last=None, scale=None, ws=None, g=None):
    B, T, H, dk = q.shape
    Hk, dv = v.shape[2:]
    g = [torch.empty_like(x) for x in (q, k, v)] + [torch.empty((B, H, dk, dv), device="cuda")] if g is None else g
    ws = _ws(simx.decay_attention_grad_workspace_size(B, T, H, Hk, dk, dv)) if ws is None else ws
    simx.decay_attention_grad(q, k, v, go, *g[:3], ld, ws, scale=scale, s0=s0, done=done, ds_last=ds_last, ds0=g[3])
    return g


@pytest.mark.parametrize("B,T,H,D", [(20, 256, 8, 128), (10, 500, 4, 128), (40, 384, 8, 64), (64, 260, 8, 32), (1, 3000, 4, 64), (19, 300, 8, 128)])
def test_rows_leave_whole_while_memory_is_busy(simx, B, T, H, D):
    """o leaves by the copy engine, the next chunk's o is written where it was: the same bits where other streams
    hold the copies up."""
    gen = torch.Generator(device="cuda").manual_seed(D)
    q, k, v, go = (torch.randn((B, T, H, D), generator=gen, device="cuda").bfloat16() for _ in range(4))
    ld = -torch.rand(H, generator=gen, device="cuda") * 0.1
    ref = [x.clone() for x in (*_call(simx, q, k, v, ld), *_call_grad(simx, q, k, v, go, ld))]
    o, last, g = torch.empty_like(q), torch.empty_like(ref[1]), [torch.empty_like(x) for x in ref[2:]]
    wf = _ws(simx.decay_attention_workspace_size(B, T, H, H, D, D))
    wb = _ws(simx.decay_attention_grad_workspace_size(B, T, H, H, D, D))
    big = [torch.zeros(1 << 28, device="cuda") for _ in range(4)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, x, y in zip(streams, big[::2], big[1::2]):
            with torch.cuda.stream(s):
                for _ in range(4):
                    y.copy_(x, non_blocking=True)
        for _ in range(4):
            for x in (o, last, *g):
                x.zero_()
            _call(simx, q, k, v, ld, ws=wf, o=o, last=last)
            _call_grad(simx, q, k, v, go, ld, ws=wb, g=g)
            assert all(torch.equal(a, b) for a, b in zip((o, last, *g), ref))
        torch.cuda.synchronize()


@pytest.mark.parametrize("D", [24, 64, 128])
def test_states_of_a_gradient_keep_their_digits(simx, D):
    """grad_q where what the steps add to the state cancels: steps 40, 140 and 200 leave some 2^-18 of what each
    added.  Tolerance, of the sum of absolute terms: a power of the decay is off by 2^-22, twice; products and sums in
    fp32 by 2^-24, four of them; three parts added up by 2^-23 each, cut off: (4 + 2 + 3) 2^-23 < 2^-19.  On the result
    itself 2^-16 for the state as an operand and 2^-8 for its rounding to bf16."""
    B, T, H = 4, 300, 8
    r = np.random.default_rng(D)
    ld = -np.exp(r.uniform(np.log(1e-3), np.log(2e-2), H)).astype(np.float32)
    lam = np.exp(ld.astype(np.float64))[None, :, None]
    bf = lambda x: torch.from_numpy(x).bfloat16()  # noqa: E731
    v, k = torch.zeros(B, T, H, D), torch.zeros(B, T, H, D)
    k[:, [40, 140, 200]] = bf(r.standard_normal((B, 1, H, D))).float()
    v[:, 40] = bf(r.standard_normal((B, H, D))).float()
    left, at = v[:, 40].double().numpy(), 40
    for t in (140, 200):
        left, at = left * lam ** (t - at), t
        v[:, t] = bf(-left).float()
        left = left + v[:, t].double().numpy()
    go = torch.zeros(B, T, H, D)
    rows = np.arange(256, T)
    go[:, rows, :, rows % D] = 1.0
    q, k, v, go = (x.cuda().bfloat16() for x in (torch.zeros(B, T, H, D), k, v, go))
    g = _call_grad(simx, q, k, v, go, torch.from_numpy(ld).cuda(), scale=1.0)
    ref = attn.decay_attention_grad(_f64(q), _f64(k), _f64(v), _f64(go), ld.astype(np.float64), 1.0)
    got, want, size = _f64(g[0]), ref["grad_q"], ref["grad_q_size"]
    assert (np.abs(want).sum() < 2.0 ** -15 * size.sum()) and want[:, rows].any()
    assert (np.abs(got - want) <= 2.0 ** -19 * size + (2.0 ** -8 + 2.0 ** -16) * np.abs(want)).all()


@pytest.mark.parametrize("D", [32, 64, 128])
def test_a_state_as_an_operand(simx, D):
    """q S where rows of the state cancel.  Both parts are rounded: the first leaves at most 2^-8 of a power of two
    below the number, the second half a step of that, 2^-17; sums add 2^-23 each, cut off, eight of them at most; past the
    first chunk the state was multiplied by a power of the decay, 2^-22; another one and the rounding to bf16 are 2^-20 and
    2^-8 of the result itself."""
    B, T, H = 2, 200, 4
    r = np.random.default_rng(D + 1)
    s0 = r.standard_normal((B, H, D, D)).astype(np.float32)
    s0[:, :, 1::2] = s0[:, :, ::2] * (1 + 2.0 ** -12 * r.standard_normal((B, H, D // 2, D))).astype(np.float32)
    ld = np.float32([-1e-3, -1e-4, 0.0, -3e-3])
    q = np.zeros((B, T, H, D), np.float32)
    x = 2 * (np.arange(T) % (D // 2))
    q[:, np.arange(T), :, x], q[:, np.arange(T), :, x + 1] = 1.0, -1.0
    q = torch.from_numpy(q).cuda().bfloat16()
    zero = torch.zeros_like(q)
    o, last = _call(simx, q, zero, zero, torch.from_numpy(ld).cuda(), s0=torch.from_numpy(s0).cuda(), scale=1.0)
    ref = attn.decay_attention(_f64(q), _f64(zero), _f64(zero), ld.astype(np.float64), 1.0, s0.astype(np.float64))
    err = (2.0 ** -17 + 8 * 2.0 ** -23 + 2.0 ** -22) * ref["o_size"] + (2.0 ** -8 + 2.0 ** -20) * np.abs(ref["o"])
    assert (np.abs(_f64(o) - ref["o"]) <= err).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,at", [(5, 2), (9, 3), (150, 60), (300, 127), (300, 128), (300, 250)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_no_memory_links_no_step(simx, T, at, bad, dtype):
    """Decays that are 0 in fp32: a step that is not finite reaches itself alone, forward and backward, whatever its
    place in a chunk; neither do s0 and other steps."""
    B, H, D = 2, 5, 24
    gen = torch.Generator(device="cuda").manual_seed(T)
    clean = [torch.randn((B, T, H, D), generator=gen, device="cuda").to(dtype) for _ in range(4)]
    ld = torch.tensor([-float("inf"), -200.0, -110.0, -1e30, -0.1], device="cuda")
    s0 = torch.randn((B, H, D, D), generator=gen, device="cuda")
    ref = [*_call(simx, *clean[:3], ld, s0=s0), *_call_grad(simx, *clean, ld, s0=s0)]
    assert all(torch.isfinite(x).all() for x in ref)
    for i in range(4):
        t = [x.clone() for x in clean]
        t[i][0, at, :4, 3] = bad
        got = [*_call(simx, *t[:3], ld, s0=s0), *_call_grad(simx, *t, ld, s0=s0)]
        hit = torch.zeros((B, T, H), dtype=torch.bool, device="cuda")
        hit[0, at, :4] = True
        for n, (x, y) in enumerate(zip(got, ref)):
            assert torch.equal(x, y) if n in (1, 5) else torch.equal(x[~hit], y[~hit])  # the states, all of them
        o, gq, gk, gv = got[0][hit], *(x[hit] for x in got[2:5])
        assert not torch.isfinite(o).all() or i == 3
        assert not (torch.isfinite(gq).all() and torch.isfinite(gk).all() and torch.isfinite(gv).all())


@pytest.mark.parametrize("D", [32, 128])
@pytest.mark.parametrize("small", ["v", "go"])
def test_large_scores(simx, D, small):
    """Queries and keys whose products come near to the largest that the chunks take (|v grad_o| in the same way), with
    values as small: test_gpu_attn's bounds."""
    B, T, H = 2, 300, 2
    gen = torch.Generator(device="cuda").manual_seed(D)
    q, k, v, go = (torch.randn((B, T, H, D), generator=gen, device="cuda") for _ in range(4))
    # the sum over a head's elements: below 128 * 5 * 5 * 2^110 < 2^123
    if small == "v":
        q, k, v, go = q * 2.0 ** 55, k * 2.0 ** 55, v * 2.0 ** -80, go * 2.0 ** -30
    else:
        q, k, v, go = q * 2.0 ** -70, k * 2.0 ** -40, v * 2.0 ** 50, go * 2.0 ** 60
    q, k, v, go = (x.bfloat16() for x in (q, k, v, go))
    ld = torch.tensor([-0.01, -0.3], device="cuda")
    done = (torch.rand((B, T), generator=gen, device="cuda") < 0.01).to(torch.uint8)
    o, last = _call(simx, q, k, v, ld, done=done)
    g = _call_grad(simx, q, k, v, go, ld, done=done)
    sc, d = np.float64(np.float32(D ** -0.5)), done.cpu().numpy()
    ref = attn.decay_attention(_f64(q), _f64(k), _f64(v), _f64(ld), sc, None, d)
    _close(_f64(o), ref["o"], ref["o_size"], "bf16", T, "o")
    _state(_f64(last), ref["s_last"], ref["s_last_size"], T, "s_last")
    ref = attn.decay_attention_grad(_f64(q), _f64(k), _f64(v), _f64(go), _f64(ld), sc, None, d)
    for n, x in zip(("grad_q", "grad_k", "grad_v"), g):
        _close(_f64(x), ref[n], ref[n + "_size"], "bf16", T, n)
    _state(_f64(g[3]), ref["ds0"], ref["ds0_size"], T, "ds0")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,T,D", [(400, 40000, 16), (160, 20000, 128), (1, 300000, 64), (3, 60001, 32)])
def test_long_memories(simx, H, T, D, dtype):
    """A state over hundreds of chunks of steps that add nothing: lambda^T s0 (backward lambda^T ds_last), cut into
    segments or not.  Each of at most 2400 multiplications rounds every element by 2^-24 of its own, 3e-8 in the
    mean square, which is 3e-8 * 49 / 16 < 1e-7 of the mean over a state's 256 elements or more; a power of the decay,
    three times at most, 2^-22 each: below 1e-6.  A factor that is always rounded the same way would add up to 3e-8
    for each chunk.  In fp32 and one piece the state is multiplied every fourth step, by as little as 1 - 4e-7: a product
    s - s 7 2^-24 is rounded to a few whole steps of s, by the same part of a step for as long as s stays near where it is, so that
    these roundings do not cancel, and all T / 4 of 2^-24 count."""
    gen = torch.Generator(device="cuda").manual_seed(T)
    zero = torch.zeros((1, 1, 1, D), dtype=dtype, device="cuda").expand(1, T, H, D)
    ld = -torch.exp(torch.linspace(np.log(1e-7), np.log(8.0 / T), H, device="cuda"))
    s0 = torch.rand((1, H, D, D), generator=gen, device="cuda") + 0.5
    last = torch.empty_like(s0)
    want, tol = torch.exp(T * ld.double()), T / 4 * 2.0 ** -24 if dtype == torch.float32 and H >= 152 else 1e-6
    o = torch.empty((1, T, H, D), dtype=dtype, device="cuda")
    simx.decay_attention(zero, zero, zero, o, ld, _ws(simx.decay_attention_workspace_size(1, T, H, H, D, D)), s0=s0, s_last=last)

    def off(x):
        return ((x.double() / (s0.double() * want[None, :, None, None]) - 1).mean((0, 2, 3))).abs().max().item()
    assert not o.any() and off(last) <= tol
    del o
    if H * T * D > 1 << 28:
        return
    last.zero_()
    g = [torch.empty((1, T, H, D), dtype=dtype, device="cuda") for _ in range(3)]
    simx.decay_attention_grad(zero, zero, zero, zero, *g, ld, _ws(simx.decay_attention_grad_workspace_size(1, T, H, H, D, D)), ds_last=s0, ds0=last)
    assert off(last) <= tol
