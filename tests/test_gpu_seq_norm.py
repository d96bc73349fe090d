"""Dropout + residual + root-mean-square norm, forward and backward, against the 64-bit definition
(oracle/seq.py).

Tolerances.  z has one rounding of the product and sum: 2^-22 of |residual| + |x scale|.  The mean
square, rstd and y add a handful of roundings and a sum of at most 16384 terms in parts: 5e-6 of
their terms.  The backward pass adds one more such sum: 1e-5 of the absolute terms, dgain 1e-5 of the
sum of the absolute terms.  bf16 outputs: half a unit in the last place (8 significant bits: 2^-8) on top.  The mask is
exact: a dropped element's dx is zero and its z is the residual's bits.
"""
import numpy as np
import pytest

from oracle import seq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


@pytest.fixture(scope="module")
def simx():
    from paper_2607_05272_gb300 import build as B
    B.build()
    from paper_2607_05272_gb300 import simx
    return simx


def _f64(t):
    return t.detach().double().cpu().numpy()


def _close(got, ref, err, dtype="f32"):
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    bad = ~(np.abs(got - ref) <= err + half * np.abs(ref) + 1e-37)
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4])


def _rows(values, dtype, pad, offset):
    n, W = values.shape
    buf = torch.full((offset + n * (W + pad) + 8,), float("nan"), dtype=DT[dtype], device="cuda")
    v = buf[offset:offset + n * (W + pad)].view(n, W + pad)[:, :W]
    v.copy_(torch.from_numpy(values).to(DT[dtype]))
    return v


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _check(simx, n, W, dtype="f32", p=0.0, pad=0, offset=0, residual=True, dz=True, row_base=0, seed=(7 << 40) + 3,
           step=11, odd=False):
    """odd: every tensor at an alignment of its own."""
    rng = np.random.default_rng(n + W)
    k = iter(range(100))
    mk = lambda v=None: _rows(rng.standard_normal((n, W)) if v is None else v, dtype, pad + (next(k) if odd else 0),  # noqa: E731
                              offset + (next(k) if odd else 0))
    gain = (1 + 0.3 * rng.standard_normal(W)).astype(np.float32)
    x, res = mk(), mk() if residual else None
    z, y, rstd = mk(), mk(), torch.empty(n, device="cuda")
    simx.dropout_add_norm(x, _dev(gain), y, residual=res, z=z, rstd=rstd, p=p, eps=EPS, seed=seed, step=step,
                          row_base=row_base)
    torch.cuda.synchronize()
    keep, scale = seq.keep_mask(n, W, p, seed, step, row_base)
    g64 = gain.astype(np.float64)
    ref = seq.dropout_add_norm(_f64(x), g64, _f64(res) if residual else None, keep, scale, np.float64(np.float32(EPS)))
    _close(_f64(z), ref["z"], 2.0 ** -22 * ref["z_scale"], dtype)
    _close(_f64(rstd), ref["rstd"], 5e-6 * ref["rstd"])
    r = ref["rstd"][:, None]
    _close(_f64(y), ref["y"], np.abs(g64) * r * (2.0 ** -22 * ref["z_scale"] + 5e-6 * np.abs(ref["z"])), dtype)
    if residual:
        assert torch.equal(z[_dev(~keep)], res[_dev(~keep)])
    # backward
    dy, dzt, dx, dr = mk(), mk() if dz else None, mk(), mk()
    dgain = torch.full((W,), float("nan"), device="cuda")
    ws = torch.empty(simx.dropout_add_norm_grad_workspace_size(n, W), dtype=torch.uint8, device="cuda")
    ws.fill_(0xFF)
    simx.dropout_add_norm_grad(z, _dev(gain), rstd, dy, dx, ws, dz=dzt, dresidual=dr, dgain=dgain, p=p, seed=seed,
                               step=step, row_base=row_base)
    torch.cuda.synchronize()
    ref = seq.dropout_add_norm_grad(_f64(z), g64, _f64(rstd), _f64(dy), _f64(dzt) if dz else None, keep, scale)
    _close(_f64(dr), ref["dresidual"], 1e-5 * ref["scale"], dtype)
    _close(_f64(dx), ref["dx"], 1e-5 * ref["scale"] * scale, dtype)
    _close(_f64(dgain), ref["dgain"], 1e-5 * ref["dgain_scale"])
    assert not dx[_dev(~keep)].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("W", [1, 2, 3, 7, 8, 9, 15, 16, 17, 31, 33, 64, 100, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1000, 1023, 1024,
                               1025, 2047, 2048, 2049, 4096, 4097])
def test_widths(simx, W, dtype):
    _check(simx, 5, W, dtype, p=0.0)
    _check(simx, 5, W, dtype, p=0.3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("W", [5000, 8191, 8192, 8200, 12345, 16383, 16384])
def test_wide_rows(simx, W, dtype):
    _check(simx, 3, W, dtype, p=0.1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("W,pad,offset", [(64, 8, 0), (64, 1, 0), (64, 0, 3), (1000, 3, 1), (1024, 8, 8), (2047, 1, 0), (5003, 2, 1)])
def test_strides_and_alignment(simx, W, pad, offset, dtype):
    _check(simx, 7, W, dtype, p=0.2, pad=pad, offset=offset)
    _check(simx, 7, W, dtype, p=0.2, pad=pad, offset=offset, odd=True)
    _check(simx, 7, W, dtype, pad=pad, offset=offset, odd=True)


@pytest.mark.parametrize("n", [1, 2, 63, 700])
def test_row_counts(simx, n):
    _check(simx, n, 48, p=0.5)
    _check(simx, n, 515, "bf16", p=0.1)


def test_many_rows(simx):
    """More rows than any grid: every row against torch in 64 bits."""
    n, W = 100000, 96
    g = torch.Generator(device="cuda").manual_seed(1)
    x, res, dy = (torch.randn((n, W), generator=g, device="cuda") for _ in range(3))
    gain = torch.rand(W, generator=g, device="cuda") + 0.5
    z, y, rstd, dx, dr, dgain = torch.empty_like(x), torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty_like(x), \
        torch.empty_like(x), torch.empty(W, device="cuda")
    simx.dropout_add_norm(x, gain, y, residual=res, z=z, rstd=rstd)
    ws = torch.empty(simx.dropout_add_norm_grad_workspace_size(n, W), dtype=torch.uint8, device="cuda")
    simx.dropout_add_norm_grad(z, gain, rstd, dy, dx, ws, dresidual=dr, dgain=dgain)
    z64 = x.double() + res.double()
    r = (z64.square().mean(1, keepdim=True) + 1e-6).rsqrt()
    assert ((y.double() - z64 * r * gain).abs() <= 1e-5 * (z64.abs() * r * gain) + 1e-5).all()
    zh, gg = z.double() * rstd.double()[:, None], dy.double() * gain
    d = rstd.double()[:, None] * (gg - zh * (gg * zh).mean(1, keepdim=True))
    assert (dr.double() - d).abs().max().item() <= 1e-5 * 10 and torch.equal(dx, dr)
    t = dy.double() * zh
    assert ((dgain.double() - t.sum(0)).abs() <= 1e-5 * t.abs().sum(0)).all()


@pytest.mark.parametrize("W", [48, 515, 3000])
def test_optional_arguments(simx, W):
    _check(simx, 4, W, residual=False, p=0.25)
    _check(simx, 4, W, dz=False, p=0.25)
    n = 4
    x, dy = torch.randn((2, n, W), device="cuda")
    gain = torch.ones(W, device="cuda")
    y, y2, z, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty(n, device="cuda")
    simx.dropout_add_norm(x, gain, y)                       # a plain norm: neither z nor rstd kept
    simx.dropout_add_norm(x, gain, y2, z=z, rstd=rstd)
    assert torch.equal(y, y2) and torch.equal(z, x)
    ws = torch.empty(simx.dropout_add_norm_grad_workspace_size(n, W), dtype=torch.uint8, device="cuda")
    a, b, c = torch.empty_like(x), torch.empty_like(x), torch.empty(W, device="cuda")
    simx.dropout_add_norm_grad(z, gain, rstd, dy, a, ws, dgain=c)
    simx.dropout_add_norm_grad(z, gain, rstd, dy, None, None, dresidual=b)
    d = torch.empty(W, device="cuda")
    simx.dropout_add_norm_grad(z, gain, rstd, dy, None, ws, dgain=d)
    assert torch.equal(a, b) and torch.equal(c, d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("W", [48, 515, 1024, 3000, 9000])
def test_in_place(simx, W, dtype):
    n = 6
    mk = lambda: torch.randn((n, W), device="cuda").to(DT[dtype])  # noqa: E731
    x, res, dy, dz = mk(), mk(), mk(), mk()
    gain = torch.rand(W, device="cuda") + 0.5
    kw = dict(p=0.2, seed=5, step=6)
    z, y, rstd = mk(), mk(), torch.empty(n, device="cuda")
    simx.dropout_add_norm(x, gain, y, residual=res, z=z, rstd=rstd, **kw)
    for zi, yi in (("residual", "x"), ("x", None)):
        b = {"x": x.clone(), "residual": res.clone()}
        z2, y2 = b[zi], b[yi] if yi else mk()
        simx.dropout_add_norm(b["x"], gain, y2, residual=b["residual"], z=z2, **kw)
        assert torch.equal(z2, z) and torch.equal(y2, y)
    ws = torch.empty(simx.dropout_add_norm_grad_workspace_size(n, W), dtype=torch.uint8, device="cuda")
    dx, dr = mk(), mk()
    simx.dropout_add_norm_grad(z, gain, rstd, dy, dx, ws, dz=dz, dresidual=dr, **kw)
    for swap in (False, True):
        a, b = dy.clone(), dz.clone()
        ox, orr = (b, a) if swap else (a, b)
        simx.dropout_add_norm_grad(z, gain, rstd, a, ox, ws, dz=b, dresidual=orr, **kw)
        assert torch.equal(ox, dx) and torch.equal(orr, dr)


def test_rows_keep_their_mask_in_chunks_and_other_layouts(simx):
    n, W = 20, 200
    x = torch.randn((n, W), device="cuda")
    gain = torch.ones(W, device="cuda")
    z, y = torch.empty_like(x), torch.empty_like(x)
    kw = dict(p=0.5, seed=1 << 63, step=(1 << 32) - 1)
    simx.dropout_add_norm(x, gain, y, z=z, row_base=100, **kw)
    wide = torch.zeros((n, 333), device="cuda")
    for a, b in ((0, 7), (7, 20)):
        simx.dropout_add_norm(x[a:b], gain, wide[a:b, 3:3 + W], row_base=100 + a, **kw)
    assert torch.equal(wide[:, 3:3 + W], y)
    other = torch.empty_like(x)
    simx.dropout_add_norm(x, gain, y, z=other, row_base=101, **kw)
    assert not torch.equal(other, z) and torch.equal((other[:-1] != 0) , (torch.where(z[1:] != 0, 1, 0) != 0))
    _check(simx, 3, 40, p=0.4, row_base=(1 << 32) - 3)


def test_what_is_dropped_counts_as_zero(simx):
    n, W, p = 4, 300, 0.5
    keep, _ = seq.keep_mask(n, W, p, 3, 4)
    x = np.where(keep, 1.0, np.where(np.arange(W) % 2, np.inf, np.nan)).astype(np.float32)
    y, z = torch.empty((n, W), device="cuda"), torch.empty((n, W), device="cuda")
    simx.dropout_add_norm(_dev(x), torch.ones(W, device="cuda"), y, z=z, p=p, seed=3, step=4)
    assert torch.isfinite(y).all() and torch.isfinite(z).all() and not z[_dev(~keep)].any()


def test_rows_of_zeros(simx):
    for W in (40, 2000):
        x = torch.zeros((3, W), device="cuda")
        y, rstd = torch.ones_like(x), torch.empty(3, device="cuda")
        simx.dropout_add_norm(x, torch.ones(W, device="cuda"), y, rstd=rstd, eps=1e-4)
        assert not y.any() and (rstd - 100).abs().max().item() <= 1e-3


def test_empty(simx):
    e, gain = torch.empty((0, 40), device="cuda"), torch.ones(40, device="cuda")
    d = torch.ones(40, device="cuda")
    simx.dropout_add_norm(e, gain, e, rstd=e[:, 0].clone())
    simx.dropout_add_norm_grad(e, gain, torch.empty(0, device="cuda"), e, None,
                               torch.empty(1 << 12, dtype=torch.uint8, device="cuda"), dgain=d)
    torch.cuda.synchronize()
    assert not d.any()


def test_gradient_by_differences(simx):
    """<y, dy> + <z, dz> along a direction of x; sums of 3000 fp32 terms, each rounded to 1e-6."""
    n, W, p = 6, 500, 0.2
    rng = np.random.default_rng(2)
    x, v, dy, dz = rng.standard_normal((4, n, W))
    gain = _dev((1 + 0.2 * rng.standard_normal(W)).astype(np.float32))
    f = lambda a: _dev(a.astype(np.float32))  # noqa: E731
    kw = dict(p=p, seed=9, step=1)

    def value(s):
        y, z, rstd = torch.empty((n, W), device="cuda"), torch.empty((n, W), device="cuda"), torch.empty(n, device="cuda")
        simx.dropout_add_norm(f(x + s * v), gain, y, z=z, rstd=rstd, **kw)
        return (_f64(y) * dy).sum() + (_f64(z) * dz).sum(), z, rstd

    _, z, rstd = value(0.0)
    dx = torch.empty((n, W), device="cuda")
    ws = torch.empty(simx.dropout_add_norm_grad_workspace_size(n, W), dtype=torch.uint8, device="cuda")
    simx.dropout_add_norm_grad(z, gain, rstd, f(dy), dx, ws, dz=f(dz), **kw)
    step = 1e-2
    slope = (_f64(dx) * v).sum()
    diff = (value(step)[0] - value(-step)[0]) / (2 * step)
    assert abs(diff - slope) <= 3000 * 1e-6 / step + 50 * step ** 2 * (1 + abs(slope))


def test_refusals(simx):
    x, gain = torch.zeros((4, 10), device="cuda"), torch.ones(10, device="cuda")
    o, r = torch.empty_like, torch.ones(4, device="cuda")
    ws = torch.empty(simx.dropout_add_norm_grad_workspace_size(4, 10), dtype=torch.uint8, device="cuda")

    def refused(f, *a, **kw):
        with pytest.raises(simx.SimxError) as e:
            f(*a, **kw)
        assert e.value.status == simx.EINVAL

    f, g = simx.dropout_add_norm, simx.dropout_add_norm_grad
    refused(f, x.half(), gain, o(x).half())
    refused(f, x.cpu(), gain.cpu(), o(x).cpu())
    refused(f, x, gain[:9], o(x))
    refused(f, x, gain.double(), o(x))
    refused(f, x, None, o(x))
    refused(f, x, gain, None)
    refused(f, x, gain, o(x), residual=x[:3])
    refused(f, x, gain, o(x), residual=x[:1].expand(4, 10))
    for p in (-0.1, 1.0, 0.99999999, float("nan")):
        refused(f, x, gain, o(x), p=p)
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        refused(f, x, gain, o(x), eps=eps)
    refused(f, x, gain, o(x), seed=-1)
    refused(f, x, gain, o(x), step=1 << 32)
    refused(f, x, gain, o(x), row_base=(1 << 32) - 3)
    w = torch.zeros((1, 16385), device="cuda")
    refused(f, w, torch.ones(16385, device="cuda"), o(w))
    refused(g, x, gain, None, x, o(x), ws)
    refused(g, x, gain, r, None, o(x), ws)
    refused(g, x, gain, r, x, o(x), ws[:8], dgain=gain.clone())
    refused(g, x, gain, r, x, o(x), None, dgain=gain.clone())


@pytest.mark.parametrize("W", [40, 16384])
def test_gain_gradient_of_no_rows_with_the_workspace_asked_for(simx, W):
    """The size function asks for 0 bytes, so the workspace may be an empty tensor or None."""
    e, gain, r = torch.empty((0, W), device="cuda"), torch.ones(W, device="cuda"), torch.empty(0, device="cuda")
    size = simx.dropout_add_norm_grad_workspace_size(0, W)
    for ws in (torch.empty(size, dtype=torch.uint8, device="cuda"), None):
        d = torch.ones(W, device="cuda")
        simx.dropout_add_norm_grad(e, gain, r, e, None, ws, dgain=d)
        torch.cuda.synchronize()
        assert not d.any()
