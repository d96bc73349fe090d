"""Linear attention by chunks on the tensor cores: what only that form can get wrong."""
import numpy as np
import pytest

from oracle import attn

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
