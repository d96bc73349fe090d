"""Linear attention at the C ABI, without a GPU: outputs that share memory with what the call still reads."""
import ctypes as C

import pytest

from paper_2607_05272_gb300 import build as B
from paper_2607_05272_gb300 import simx
from tests.test_seq_abi import FAKE, _refused

H = simx.Heads
STEP = 1 << 20  # between tensors that lie apart


@pytest.fixture(scope="module")
def lib():
    B.build()
    return simx.lib()


def _attention(**kw):
    x = [H(FAKE + i * STEP, 1024, 128, 32) for i in range(8)]  # 8 steps of 4 heads of 32
    d = dict(batch=2, len=8, heads=4, kv_heads=4, dk=32, dv=32, dtype=0, scale=0.5, q=x[0], k=x[1], v=x[2], o=x[3], log_decay=FAKE,
             grad_o=x[4], grad_q=x[5], grad_k=x[6], grad_v=x[7])
    d.update(kw)
    return simx.Attention(**d)


def _why(lib, call, a, ws=None):
    status = call(C.byref(a), ws, 0, None)
    assert status == simx.EINVAL
    return lib.simx_last_error().decode()


def _forward(lib, **kw):
    return _why(lib, lib.simx_decay_attention, _attention(**kw))


def _backward(lib, **kw):
    return _why(lib, lib.simx_decay_attention_grad, _attention(**kw))


def _at(i, off=0, strides=(1024, 128, 32)):
    return H(FAKE + i * STEP + off, *strides)


@pytest.mark.parametrize("name,i", [("q", 0), ("k", 1), ("v", 2)])
@pytest.mark.parametrize("off", [0, 4, 124, 512, 4 * 1024 + 128])
def test_outputs_on_inputs(lib, name, i, off):
    """At the same address, and a few elements, a head, a step or a sequence on."""
    assert _forward(lib, o=_at(i, off)) == "o overlaps %s" % name
    for g in ("grad_q", "grad_k", "grad_v"):
        assert _backward(lib, **{g: _at(i, off)}) == "%s overlaps %s" % (g, name)
        assert _backward(lib, **{g: _at(4, off)}) == "%s overlaps grad_o" % g
    assert _forward(lib, o=_at(i, 0, (4096, 512, 128))) == "o overlaps %s" % name  # other strides


@pytest.mark.parametrize("one,two", [("grad_k", "grad_q"), ("grad_v", "grad_q"), ("grad_v", "grad_k")])
def test_gradients_on_one_another(lib, one, two):
    assert _backward(lib, **{one: _at(9), two: _at(9)}) == "%s overlaps %s" % (one, two)
    assert _backward(lib, **{one: _at(9), two: _at(9, -128)}) == "%s overlaps %s" % (one, two)


def test_states(lib):
    s = 4 * 2 * 4 * 32 * 32
    for off in (-s + 4, -4, 4, s - 4):
        assert _forward(lib, s0=FAKE, s_last=FAKE + off) == "s_last overlaps s0"
    for off in (-s + 4, -4, 0, 4, s - 4):
        assert _backward(lib, ds_last=FAKE, ds0=FAKE + off) == "ds0 overlaps ds_last"
        assert _backward(lib, s0=FAKE, ds0=FAKE + off) == "ds0 overlaps s0"


def test_what_lies_apart_is_not_refused(lib):
    """Parts of a packed projection, time-major views, states beside one another and in place: the call is refused for
    its workspace alone, behind all these checks."""
    n = 1 << 15  # long enough to be cut into segments
    packed = [H(FAKE + 4 * i * 32, n * 3 * 32, 3 * 32, 32) for i in range(3)]
    grads = [H(FAKE + (1 << 30) + 4 * i * 32, n * 3 * 32, 3 * 32, 32) for i in range(3)]
    o = H(FAKE + (1 << 31), n * 32, 32, 32)
    s = 4 * 32 * 32
    one = dict(batch=1, len=n, heads=1, kv_heads=1, q=packed[0], k=packed[1], v=packed[2], o=o, grad_o=o, grad_q=grads[0], grad_k=grads[1],
               grad_v=grads[2])
    for kw in (dict(s0=FAKE, s_last=FAKE), dict(s0=FAKE, s_last=FAKE + s), dict(s0=FAKE + s, s_last=FAKE)):
        assert "workspace" in _forward(lib, **one, **kw)
    for kw in (dict(s0=FAKE, ds0=FAKE + s), dict(ds_last=FAKE + s, ds0=FAKE), dict(s0=FAKE, ds_last=FAKE)):
        assert "workspace" in _backward(lib, **one, **kw)
    # inputs may be the same
    assert "workspace" in _forward(lib, **{**one, "k": packed[0], "v": packed[0]})
    # heads of several tensors side by side in each step
    q, k, v, out = (H(FAKE + 4 * off, n * 512, 512, 32) for off in (0, 128, 192, 256))
    kw = dict(batch=1, len=n, heads=4, kv_heads=2, q=q, k=k, v=v, o=out)
    assert "workspace" in _forward(lib, **kw)
    assert _forward(lib, **{**kw, "o": H(FAKE + 4 * 160, n * 512, 512, 32)}) == "o overlaps k"
    # time-major, and zero strides of inputs
    q, out = H(FAKE, 32, 64, 32), H(FAKE + 4 * 64 * n, 32, 64, 32)
    kw = dict(batch=2, len=n, heads=1, kv_heads=1, q=q, k=H(FAKE, 0, 64, 0), v=q, o=out)
    assert "workspace" in _forward(lib, **kw)


def test_axes_of_one(lib):
    """The stride of an axis that is one long says nothing, whatever it is."""
    n = 1 << 15
    for sb in (0, 32, 500, 1 << 30):
        for sh in (0, 7, 900, 1 << 30):
            q, k, v = (H(FAKE + i * (1 << 30), sb, 96, sh) for i in range(3))
            for off in (0, 96, 9600, 96 * (n - 1) + 31, -96 * (n - 1) - 31):
                kw = dict(batch=1, len=n, heads=1, kv_heads=1, q=q, k=k, v=v)
                assert _forward(lib, **kw, o=H(k.p + 4 * off, sb, 96, sh)) == "o overlaps k"
            for off in (32, 64, 96 * n, -96 * n):
                assert "workspace" in _forward(lib, **kw, o=H(k.p + 4 * off, sb, 96, sh))


def test_no_steps(lib):
    """Tensors of no elements share none."""
    x = H(FAKE, 0, 0, 0)
    a = _attention(len=0, q=x, k=x, v=x, grad_o=x, grad_q=x, grad_k=x, grad_v=x)
    assert lib.simx_decay_attention_grad(C.byref(a), None, 0, None) == simx.OK
    _refused(lib, lib.simx_decay_attention_grad(C.byref(_attention(len=0, ds_last=FAKE, ds0=FAKE)), FAKE, 1 << 40, None))
