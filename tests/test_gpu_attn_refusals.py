"""Linear attention through the binding: calls that are refused, as the library's own error and before any launch."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def simx():
    from paper_2607_05272_gb300 import build as B
    B.build()
    from paper_2607_05272_gb300 import simx
    return simx


def _refused(simx, f):
    before = simx.lib().simx_launches()
    with pytest.raises(simx.SimxError) as e:
        f()
    assert e.value.status == simx.EINVAL and simx.lib().simx_launches() == before


@pytest.mark.parametrize("dk,dv", [(0, 8), (8, 0), (129, 8)])
def test_head_sizes(simx, dk, dv):
    q, v, ld = torch.zeros(2, 4, 3, dk, device="cuda"), torch.zeros(2, 4, 3, dv, device="cuda"), torch.zeros(3, device="cuda")
    _refused(simx, lambda: simx.decay_attention(q, q.clone(), v, v.clone(), ld))
    _refused(simx, lambda: simx.decay_attention_grad(q, q.clone(), v, v.clone(), q.clone(), q.clone(), v.clone(), ld, None))


def test_outputs_in_place_of_inputs(simx):
    x = [torch.randn(2, 4, 3, 8, device="cuda") for _ in range(7)]
    ld, s = -torch.ones(3, device="cuda"), torch.randn(2, 3, 8, 8, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    for i in range(3):
        _refused(simx, lambda: simx.decay_attention(*x[:3], x[i], ld))
    for i in range(4, 7):
        for j in range(i):
            _refused(simx, lambda: simx.decay_attention_grad(*x[:i], x[j], *x[i + 1:], ld, ws))
    _refused(simx, lambda: simx.decay_attention_grad(*x, ld, ws, s0=s, ds0=s))
    _refused(simx, lambda: simx.decay_attention_grad(*x, ld, ws, ds_last=s, ds0=s))
    # parts of one buffer lie apart, and a state goes on in place
    p = torch.randn(2, 4, 9, 8, device="cuda")
    g = torch.empty_like(p)
    simx.decay_attention(p[:, :, :3], p[:, :, 3:6], p[:, :, 6:], x[0], ld, ws, s0=s, s_last=s)
    simx.decay_attention_grad(p[:, :, :3], p[:, :, 3:6], p[:, :, 6:], x[0], g[:, :, :3], g[:, :, 3:6], g[:, :, 6:], ld, ws, s0=s,
                              ds0=torch.empty_like(s))
    torch.cuda.synchronize()
    assert torch.isfinite(g).all()
