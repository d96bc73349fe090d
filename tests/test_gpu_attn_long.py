"""Linear attention over long sequences and with heads of up to 64 elements that blocks share, against the 64-bit
definition run on the device; the tolerances are those of test_gpu_attn."""
import numpy as np
import pytest

from oracle import attn
from tests.test_gpu_attn import _close, _f64, _state

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
BLOCKS = 304  # that run at a time, dimensions up to 64


@pytest.fixture(scope="module")
def simx():
    from paper_2607_05272_gb300 import build as B
    B.build()
    from paper_2607_05272_gb300 import simx
    return simx


def _forward64(q, k, v, ld, scale, s0, done):
    """oracle.attn.decay_attention, on the device."""
    H = q.shape[2]
    k, v = (x.repeat_interleave(H // x.shape[2], 2) for x in (k, v))
    q, k, v, s = (x.double() for x in (q, k, v, s0))
    lam, live = ld.double().exp()[None, :, None, None], (done == 0).double()[:, :, None, None, None]
    e, o, size = s.abs(), torch.empty_like(v), torch.empty_like(v)
    for t in range(q.shape[1]):
        kv = k[:, t, :, :, None] * v[:, t, :, None, :]
        s, e = torch.addcmul(kv, lam, s), torch.addcmul(kv.abs(), lam, e)
        o[:, t], size[:, t] = (scale * (q[:, t, :, None] @ s))[:, :, 0], (abs(scale) * (q[:, t, :, None].abs() @ e))[:, :, 0]
        s, e = s * live[:, t], e * live[:, t]
    return {"o": o, "o_size": size, "s_last": s, "s_last_size": e}


def _backward64(q, k, v, go, ld, scale, s0, done, ds_last):
    """oracle.attn.decay_attention_grad, on the device."""
    H, Hk = q.shape[2], k.shape[2]
    kk, vv = (x.double().repeat_interleave(H // Hk, 2) for x in (k, v))
    q, go, s, r = (x.double() for x in (q, go, s0, ds_last))
    lam, live = ld.double().exp()[None, :, None, None], (done == 0).double()[:, :, None, None, None]
    out = {n + m: torch.empty(x.shape, dtype=torch.float64, device="cuda") for n, x in (("grad_q", q), ("grad_k", kk), ("grad_v", vv))
           for m in ("", "_size")}

    def put(name, t, a, b):
        out[name][:, t], out[name + "_size"][:, t] = a, b
    e = s.abs()
    for t in range(q.shape[1]):
        kv = kk[:, t, :, :, None] * vv[:, t, :, None, :]
        s, e = torch.addcmul(kv, lam, s), torch.addcmul(kv.abs(), lam, e)
        put("grad_q", t, scale * (s @ go[:, t, :, :, None])[..., 0], abs(scale) * (e @ go[:, t, :, :, None].abs())[..., 0])
        s, e = s * live[:, t], e * live[:, t]
    e = r.abs()
    for t in range(q.shape[1] - 1, -1, -1):
        qo = scale * q[:, t, :, :, None] * go[:, t, :, None, :]
        r, e = torch.addcmul(qo, live[:, t], r), torch.addcmul(qo.abs(), live[:, t], e)
        put("grad_k", t, (r @ vv[:, t, :, :, None])[..., 0], (e @ vv[:, t, :, :, None].abs())[..., 0])
        put("grad_v", t, (kk[:, t, :, None] @ r)[:, :, 0], (kk[:, t, :, None].abs() @ e)[:, :, 0])
        r, e = lam * r, lam * e
    for n in ("grad_k", "grad_v", "grad_k_size", "grad_v_size"):
        out[n] = out[n].unflatten(2, (Hk, H // Hk)).sum(3)
    return {**out, "ds0": r, "ds0_size": e}


def _inputs(B, T, H, Hk, dk, dv, done, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    t = [r(B, T, h, d).to(dtype) for h, d in ((H, dk), (Hk, dk), (Hk, dv), (H, dv))]
    ld = torch.log1p(-torch.exp2(-(torch.rand(H, generator=gen, device="cuda") * 9 + 1)))
    return (*t, ld, r(B, H, dk, dv), (torch.rand((B, T), generator=gen, device="cuda") < done).to(torch.uint8), r(B, H, dk, dv))


def _check_forward(simx, B, T, H, Hk, dk, dv, done, dtype="bf16"):
    q, k, v, _, ld, s0, dn, _ = _inputs(B, T, H, Hk, dk, dv, done, torch.bfloat16 if dtype == "bf16" else torch.float32, T + H)
    o, last = torch.empty((B, T, H, dv), dtype=q.dtype, device="cuda"), torch.empty_like(s0)
    ws = torch.empty(max(16, simx.decay_attention_workspace_size(B, T, H, Hk, dk, dv)), dtype=torch.uint8, device="cuda")
    simx.decay_attention(q, k, v, o, ld, ws, s0=s0, done=dn, s_last=last)
    ref = {n: x.cpu().numpy() for n, x in _forward64(q, k, v, ld, float(np.float32(dk ** -0.5)), s0, dn).items()}
    _close(_f64(o), ref["o"], ref["o_size"], dtype, T, "o")
    _state(_f64(last), ref["s_last"], ref["s_last_size"], T, "s_last")


def _check_backward(simx, B, T, H, Hk, dk, dv, done, dtype="bf16"):
    q, k, v, go, ld, s0, dn, dl = _inputs(B, T, H, Hk, dk, dv, done, torch.bfloat16 if dtype == "bf16" else torch.float32, T + H)
    g, d0 = [torch.empty_like(x) for x in (q, k, v)], torch.empty_like(s0)
    ws = torch.empty(simx.decay_attention_grad_workspace_size(B, T, H, Hk, dk, dv), dtype=torch.uint8, device="cuda")
    simx.decay_attention_grad(q, k, v, go, *g, ld, ws, s0=s0, done=dn, ds_last=dl, ds0=d0)
    ref = {n: x.cpu().numpy() for n, x in _backward64(q, k, v, go, ld, float(np.float32(dk ** -0.5)), s0, dn, dl).items()}
    for n, x in zip(("grad_q", "grad_k", "grad_v"), g):
        _close(_f64(x), ref[n], ref[n + "_size"], dtype, T, n)
    _state(_f64(d0), ref["ds0"], ref["ds0_size"], T, "ds0")


def test_the_definition_on_the_device():
    q, k, v, go, ld, s0, dn, dl = _inputs(2, 20, 4, 2, 5, 3, 0.2, torch.float32, 1)
    a = [_f64(x) for x in (q, k, v, ld)]
    pairs = [(_forward64(q, k, v, ld, 0.3, s0, dn), attn.decay_attention(*a, 0.3, _f64(s0), dn.cpu().numpy())),
             (_backward64(q, k, v, go, ld, 0.3, s0, dn, dl),
              attn.decay_attention_grad(*a[:3], _f64(go), a[3], 0.3, _f64(s0), dn.cpu().numpy(), _f64(dl)))]
    for got, want in pairs:
        assert set(got) == set(want)
        for n in want:
            assert np.abs(_f64(got[n]) - want[n]).max() <= 1e-13 * (1 + np.abs(want[n]).max()), n


@pytest.mark.parametrize("B,T,H,Hk,dk,dv", [(38, 2100, 8, 8, 64, 64), (57, 2049, 8, 2, 40, 64), (19, 2305, 16, 4, 32, 32), (56, 2200, 8, 8, 24, 17)])
@pytest.mark.parametrize("done", [0.0, 0.002])
def test_heads_that_blocks_share(simx, B, T, H, Hk, dk, dv, done):
    """As many heads as blocks run at a time, up to half as many again: a workspace that nothing else would need."""
    assert BLOCKS <= B * H <= 1.5 * BLOCKS
    assert simx.decay_attention_workspace_size(B, T, H, Hk, dk, dv) >= BLOCKS * 512 * (64 if max(dk, dv) > 32 else 32)
    _check_forward(simx, B, T, H, Hk, dk, dv, done)


@pytest.mark.parametrize("B,T,H,dk,dv", [(17, 2100, 6, 64, 16), (19, 2049, 8, 10, 50), (13, 2305, 8, 32, 8), (15, 2178, 10, 8, 30)])
@pytest.mark.parametrize("done", [0.0, 0.002])
def test_gradients_of_heads_that_blocks_share(simx, B, T, H, dk, dv, done):
    assert BLOCKS <= 3 * B * H <= 1.5 * BLOCKS
    share = BLOCKS * 512 * (64 if max(dk, dv) > 32 else 32)
    assert simx.decay_attention_grad_workspace_size(B, T, H, H, dk, dv) >= share > 3 * B * H * 3 * (dk * dv + 1) * 4  # more than segments take
    _check_backward(simx, B, T, H, H, dk, dv, done)


def test_gradients_of_shared_heads_that_blocks_share(simx):
    _check_backward(simx, 17, 2100, 8, 2, 64, 64, 0.001)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_sequences(simx, dtype):
    _check_forward(simx, 1, 60001, 16, 4, 64, 64, 1 / 2048, dtype)
    _check_backward(simx, 1, 10011, 4, 1, 64, 64, 1 / 2048, dtype)
