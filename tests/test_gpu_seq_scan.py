"""The gated scan and its backward pass against their 64-bit definitions (oracle/seq.py).

Tolerances.  sigmoid(-z) is off by at most 7e-7 of itself and each step rounds once, so step t adds
at most 1e-6 (|s_t| + |x_t|) to the error that a_t carries on; the oracle's `err` is that recurrence
for a unit of relative error.  Combining chunks of steps rounds as often again: fp32 results are held
to 2e-6 err, backward ones (dx and dgate multiply by b and a b (s - x), each with its own error) to
4e-6 of theirs, dbias to 2e-5 of the sum of the absolute terms (a running sum of up to a few hundred
fp32 terms per partial), and bf16 outputs to half a unit in the last place (8 significant bits: 2^-8) on top.
"""
import numpy as np
import pytest

from oracle import seq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


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
    bad = ~(np.abs(got - ref) <= err + half * np.abs(ref) + 1e-36)
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4], err[bad][:4])


def _tensor(shape, dtype, layout, fill=None, offset=0):
    """[B, T, C] on the device in a layout, with NaN around it."""
    B, T, C = shape
    n = {"batch": B * T * C, "padded": B * (T * (C + 3) + 5), "packed": B * T * 2 * C, "time": T * B * C}[layout]
    buf = torch.full((offset + n,), float("nan"), dtype=DT[dtype], device="cuda")[offset:]
    if layout == "batch":
        v = buf.view(B, T, C)
    elif layout == "padded":
        v = buf.view(B, T * (C + 3) + 5)[:, :T * (C + 3)].reshape(B, T, C + 3)[:, :, :C] if B * T == 0 else \
            torch.as_strided(buf, (B, T, C), (T * (C + 3) + 5, C + 3, 1), buf.storage_offset())
    elif layout == "packed":
        v = buf.view(B, T, 2 * C)[:, :, C:]
    else:
        v = buf.view(T, B, C).transpose(0, 1)
    if fill is not None:
        v.copy_(torch.from_numpy(fill).to(DT[dtype]))
    return v


def _case(B, T, C, seed, done, long_memory=False):
    rng = np.random.default_rng(seed)
    f = lambda v: v.astype(np.float32)  # noqa: E731
    x, gate = rng.standard_normal((B, T, C)), rng.standard_normal((B, T, C)) * 1.5 + (9.0 if long_memory else 2.0)
    dn = (rng.random((B, T)) < done).astype(np.uint8) if done else None
    return dict(x=x, gate=gate, bias=f(rng.standard_normal(C) * 0.5), h0=f(rng.standard_normal((B, C))), done=dn,
                dh=rng.standard_normal((B, T, C)), dh_last=f(rng.standard_normal((B, C))))


def _done(dn, layout):
    if dn is None:
        return None
    t = torch.from_numpy(dn).cuda()
    return t.t().contiguous().t() if layout == "time" else t


def _dev(a):
    return None if a is None else torch.from_numpy(a).cuda()


def _check(simx, B, T, C, dtype="f32", layout="batch", done=0.0, seed=0, offset=0, drop=(), long_memory=False):
    c = _case(B, T, C, seed + B + T + C, done, long_memory)
    for k in drop:
        c[k] = None
    x, gate, h = (_tensor((B, T, C), dtype, layout, v, offset) for v in (c["x"], c["gate"], None))
    dn, bias, h0 = _done(c["done"], layout), _dev(c["bias"]), _dev(c["h0"])
    last = torch.full((B, C), float("nan"), device="cuda")
    ws = torch.empty(max(16, simx.gated_scan_workspace_size(B, T, C)), dtype=torch.uint8, device="cuda")
    ws.fill_(0xFF)
    simx.gated_scan(x, gate, h, ws, bias=bias, h0=h0, done=dn, h_last=last)
    torch.cuda.synchronize()
    d = lambda k: None if c[k] is None else c[k].astype(np.float64)  # noqa: E731
    ref = seq.gated_scan(_f64(x), _f64(gate), d("bias"), d("h0"), c["done"])
    _close(_f64(h), ref["h"], 2e-6 * ref["err"], dtype)
    _close(_f64(last), ref["h_last"], 2e-6 * ref["err_last"])
    # backward
    dh, dx, dg = (_tensor((B, T, C), dtype, layout, v, offset) for v in (c["dh"], None, None))
    db, d0 = torch.full((C,), float("nan"), device="cuda"), torch.full((B, C), float("nan"), device="cuda")
    simx.gated_scan_grad(x, gate, h, dh, dx, dg, ws, bias=bias, h0=h0, done=dn, dh_last=_dev(c["dh_last"]),
                         dbias=db, dh0=d0)
    torch.cuda.synchronize()
    ref = seq.gated_scan_grad(_f64(x), _f64(gate), _f64(h), _f64(dh), d("bias"), d("h0"), c["done"], d("dh_last"))
    _close(_f64(dx), ref["dx"], 4e-6 * ref["err_dx"], dtype)
    _close(_f64(dg), ref["dgate"], 4e-6 * ref["err_dgate"], dtype)
    _close(_f64(d0), ref["dh0"], 4e-6 * ref["err_dh0"])
    _close(_f64(db), ref["dbias"], 2e-5 * ref["err_dbias"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 7, 8, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 255, 257, 300, 1000])
def test_lengths(simx, T, dtype):
    _check(simx, 2, T, 64, dtype, done=0.05)
    _check(simx, 3, T, 5, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [1, 2, 3, 4, 7, 8, 9, 16, 31, 32, 33, 40, 63, 64, 65, 100, 128, 200, 256, 264])
def test_channels(simx, C, dtype):
    _check(simx, 2, 150, C, dtype, done=0.05)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["batch", "padded", "packed", "time"])
@pytest.mark.parametrize("C,offset", [(64, 0), (24, 0), (17, 0), (64, 1), (32, 4)])
def test_layouts_and_alignment(simx, layout, C, offset, dtype):
    _check(simx, 3, 70, C, dtype, layout, done=0.1, offset=offset)
    _check(simx, 5, 1, C, dtype, layout, done=0.5, offset=offset)


@pytest.mark.parametrize("B,T,C", [(1, 5000, 16), (1, 20000, 3), (2, 9000, 64), (1, 4097, 130), (40, 700, 8)])
def test_long_sequences(simx, B, T, C):
    _check(simx, B, T, C, done=0.002)
    _check(simx, B, T, C, "bf16", "time")


@pytest.mark.parametrize("B,C", [(700, 64), (5000, 8), (300, 257), (1, 4096)])
def test_many_columns(simx, B, C):
    for T in (1, 6, 40):
        _check(simx, B, T, C, done=0.1)
    _check(simx, B, 1, C, "bf16")


def test_long_memories_stay_exact(simx):
    """Gates around 9: a within 1e-4 of 1, where a recurrence on a rounded a loses three digits."""
    _check(simx, 1, 6000, 32, long_memory=True)
    _check(simx, 2, 3000, 5, long_memory=True)


@pytest.mark.parametrize("drop", [("bias",), ("h0",), ("dh_last",), ("bias", "h0", "dh_last")])
def test_optional_arguments(simx, drop):
    for T in (1, 100):
        _check(simx, 3, T, 24, drop=drop, done=0.1)


def test_every_step_ends_an_episode(simx):
    _check(simx, 2, 50, 32, done=1.1)
    _check(simx, 2, 50, 5, done=1.1)


def test_what_an_episode_left_behind_is_dropped(simx):
    """States of inf and NaN before an episode's end do not reach the next one."""
    for T, C in ((40, 64), (40, 5), (300, 64), (6, 64)):
        c = _case(2, T, C, 3, 0.0)
        cut = T // 2
        dn = np.zeros((2, T), np.uint8)
        dn[:, cut - 1] = 1
        bad, good = c["x"].copy(), c["x"].copy()
        bad[:, cut - 2], bad[0, cut - 3] = np.inf, np.nan
        out = []
        for x in (bad, good):
            xt, gt, h = (_tensor((2, T, C), "f32", "batch", v) for v in (x, c["gate"], None))
            last = torch.empty((2, C), device="cuda")
            simx.gated_scan(xt, gt, h, torch.empty(max(16, simx.gated_scan_workspace_size(2, T, C)), dtype=torch.uint8, device="cuda"),
                            h0=_dev(c["h0"]), done=_done(dn, "batch"), h_last=last)
            torch.cuda.synchronize()
            out.append((h, last))
        (hb, lb), (hgood, lg) = out
        assert torch.equal(hb[:, cut:], hgood[:, cut:]) and torch.equal(lb, lg)
        assert torch.isfinite(hb[:, cut:]).all()


def test_gradients_stop_at_an_episode_end(simx):
    for T, C in ((40, 64), (40, 5), (300, 64), (6, 64)):
        c = _case(2, T, C, 3, 0.0)
        cut = T // 2
        dn = np.zeros((2, T), np.uint8)
        dn[:, cut - 1] = 1
        res = []
        for poison in (False, True):
            dh = c["dh"].copy()
            hv = c["x"].copy()  # any saved h will do
            if poison:
                dh[:, cut + 1] = np.nan
                dh[0, cut + 2] = np.inf
                hv[:, cut - 1] = np.nan  # the dropped state
            t = [_tensor((2, T, C), "f32", "batch", v) for v in (c["x"], c["gate"], hv, dh, None, None)]
            d0 = torch.empty((2, C), device="cuda")
            ws = torch.empty(max(16, simx.gated_scan_workspace_size(2, T, C)), dtype=torch.uint8, device="cuda")
            simx.gated_scan_grad(*t, ws, h0=_dev(c["h0"]), done=_done(dn, "batch"), dh0=d0)
            torch.cuda.synchronize()
            res.append((t[4][:, :cut].clone(), t[5][:, :cut].clone(), d0))
        assert all(torch.equal(a, b) for a, b in zip(*res))
        assert all(torch.isfinite(a).all() for a in res[1])


def test_state_in_place_and_chunked_calls(simx):
    """len = 1 calls with the state updated in place give the long call's bits within tolerance."""
    B, T, C = 4, 37, 48
    c = _case(B, T, C, 11, 0.1)
    x, gate, h = (_tensor((B, T, C), "f32", "time", v) for v in (c["x"], c["gate"], None))
    dn, state = _done(c["done"], "time"), _dev(c["h0"]).clone()
    ref = seq.gated_scan(_f64(x), _f64(gate), c["bias"].astype(np.float64), c["h0"].astype(np.float64), c["done"])
    for t in range(T):
        simx.gated_scan(x[:, t:t + 1], gate[:, t:t + 1], h[:, t:t + 1], bias=_dev(c["bias"]), h0=state,
                        done=dn[:, t:t + 1], h_last=state)
    torch.cuda.synchronize()
    _close(_f64(h), ref["h"], 2e-6 * ref["err"])
    _close(_f64(state), ref["h_last"], 2e-6 * ref["err_last"])


def test_long_call_with_the_state_in_place(simx):
    for B, T, C in ((2, 3000, 64), (1, 3000, 5), (300, 30, 64)):
        c = _case(B, T, C, 12, 0.0)
        x, gate, h = (_tensor((B, T, C), "f32", "batch", v) for v in (c["x"], c["gate"], None))
        ws = torch.empty(max(16, simx.gated_scan_workspace_size(B, T, C)), dtype=torch.uint8, device="cuda")
        state, last = _dev(c["h0"]).clone(), torch.empty((B, C), device="cuda")
        simx.gated_scan(x, gate, h, ws, h0=_dev(c["h0"]), h_last=last)
        simx.gated_scan(x, gate, h, ws, h0=state, h_last=state)
        torch.cuda.synchronize()
        assert torch.equal(state, last)


def test_empty_problems(simx):
    h0 = torch.randn((2, 3), device="cuda")
    last, d0, db = torch.zeros((2, 3), device="cuda"), torch.zeros((2, 3), device="cuda"), torch.ones(3, device="cuda")
    ws = torch.empty(1 << 12, dtype=torch.uint8, device="cuda")
    e = [torch.empty((2, 0, 3), device="cuda") for _ in range(6)]
    simx.gated_scan(e[0], e[1], e[2], ws, h0=h0, h_last=last)
    simx.gated_scan_grad(*e, ws, dh_last=h0, dbias=db, dh0=d0)
    torch.cuda.synchronize()
    assert torch.equal(last, h0) and torch.equal(d0, h0) and not db.any()
    for shape in ((0, 4, 3), (2, 4, 0)):
        e = [torch.empty(shape, device="cuda") for _ in range(6)]
        simx.gated_scan(e[0], e[1], e[2], ws)
        simx.gated_scan_grad(*e, ws)


def test_extreme_gates(simx):
    """Gates of +-inf and +-1e4: the state held, or replaced, exactly."""
    B, T, C = 1, 20, 8
    x, h0 = np.random.default_rng(1).standard_normal((B, T, C)), np.ones((B, C), np.float32)
    for v, keeps in ((np.inf, True), (1e4, True), (-np.inf, False), (-1e4, False)):
        xt, gt, h = (_tensor((B, T, C), "f32", "batch", a) for a in (x, np.full((B, T, C), v), None))
        simx.gated_scan(xt, gt, h, h0=_dev(h0))
        torch.cuda.synchronize()
        if keeps:
            assert (h == 1).all()
        else:
            assert (h - xt).abs().max().item() <= 2 * 2.0 ** -23 * 4  # one rounding of x - s, one of the sum


def test_same_bits_every_run(simx):
    for B, T, C in ((1, 5000, 64), (1, 5000, 5), (64, 200, 64)):
        c = _case(B, T, C, 5, 0.01)
        t = [_tensor((B, T, C), "f32", "batch", v) for v in (c["x"], c["gate"], c["x"], c["dh"], None, None)]
        ws = torch.empty(max(16, simx.gated_scan_workspace_size(B, T, C)), dtype=torch.uint8, device="cuda")
        out = []
        for _ in range(2):
            db, h = torch.empty(C, device="cuda"), torch.empty((B, T, C), device="cuda")
            simx.gated_scan(t[0], t[1], h, ws)
            simx.gated_scan_grad(*t, ws, dbias=db)
            torch.cuda.synchronize()
            out.append([h, t[4].clone(), t[5].clone(), db])
        assert all(torch.equal(a, b) for a, b in zip(*out))


def test_gradient_by_differences(simx):
    """<h, dh> along a direction of x and gate; fp32 sums of 500 terms of order 1 round to 1e-5."""
    B, T, C = 2, 30, 8
    c = _case(B, T, C, 21, 0.1)
    rng = np.random.default_rng(9)
    vx, vg = rng.standard_normal((2, B, T, C))
    dn = _done(c["done"], "batch")

    def value(s):
        x, gate, h = (_tensor((B, T, C), "f32", "batch", v) for v in (c["x"] + s * vx, c["gate"] + s * vg, None))
        simx.gated_scan(x, gate, h, done=dn)
        torch.cuda.synchronize()
        return (_f64(h) * c["dh"].astype(np.float32)).sum(), x, gate, h

    _, x, gate, h = value(0.0)
    dh, dx, dg = (_tensor((B, T, C), "f32", "batch", v) for v in (c["dh"], None, None))
    ws = torch.empty(max(16, simx.gated_scan_workspace_size(B, T, C)), dtype=torch.uint8, device="cuda")
    simx.gated_scan_grad(x, gate, h, dh, dx, dg, ws, done=dn)
    torch.cuda.synchronize()
    step = 1e-2
    slope = (_f64(dx) * vx).sum() + (_f64(dg) * vg).sum()
    diff = (value(step)[0] - value(-step)[0]) / (2 * step)
    # rounding 480 terms * 1e-6 / step, and the third-order term
    assert abs(diff - slope) <= 480 * 1e-6 / step + 50 * step ** 2 * (1 + abs(slope))


def test_refusals(simx):
    x = torch.zeros((2, 4, 6), device="cuda")
    ws = torch.empty(1 << 12, dtype=torch.uint8, device="cuda")

    def refused(f, *a, **kw):
        with pytest.raises(simx.SimxError) as e:
            f(*a, **kw)
        assert e.value.status == simx.EINVAL

    s, g = simx.gated_scan, simx.gated_scan_grad
    o = torch.empty_like
    refused(s, x.half(), x.half(), o(x).half())
    refused(s, x.cpu(), x.cpu(), o(x).cpu())
    refused(s, x[0], x[0], o(x[0]))
    refused(s, x, x[:, :3], o(x))
    refused(s, x, x.bfloat16(), o(x))
    refused(s, x, x, None)
    refused(s, x, x, torch.zeros((2, 1, 6), device="cuda").expand(2, 4, 6))     # an output over itself
    refused(s, x.transpose(1, 2), x.transpose(1, 2), o(x).transpose(1, 2))      # no unit stride
    refused(s, x, x, o(x), bias=torch.zeros(5, device="cuda"))
    refused(s, x, x, o(x), h0=torch.zeros((2, 6), device="cuda", dtype=torch.bfloat16))
    refused(s, x, x, o(x), done=torch.zeros((2, 4), device="cuda"))
    refused(g, x, x, x, x, o(x), o(x), None, dbias=torch.zeros(6, device="cuda"))
    refused(g, x, x, x, x, None, o(x), ws)
    refused(g, x, x, x, x, o(x), o(x)[:, :, :5], ws)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [64, 66, 67, 130, 131])
@pytest.mark.parametrize("layout", ["batch", "padded", "packed"])
def test_clusters_of_every_access(simx, layout, C, dtype):
    """Few columns and many steps: blocks of a cluster share them, whatever the channels' alignment."""
    _check(simx, 1, 4500, C, dtype, layout, done=0.003)
    _check(simx, 2, 1100, C, dtype, layout, offset=1)


def test_clusters_with_the_state_in_place_and_ends_everywhere(simx):
    for C in (64, 66, 67):
        _check(simx, 1, 3000, C, "bf16", done=1.1)
        c = _case(1, 5000, C, 31, 0.01)
        x, gate, h = (_tensor((1, 5000, C), "bf16", "batch", v) for v in (c["x"], c["gate"], None))
        state, last, dn = _dev(c["h0"]).clone(), torch.empty((1, C), device="cuda"), _done(c["done"], "batch")
        simx.gated_scan(x, gate, h, h0=_dev(c["h0"]), done=dn, h_last=last)
        simx.gated_scan(x, gate, h, h0=state, done=dn, h_last=state)
        torch.cuda.synchronize()
        assert torch.equal(state, last)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [64, 66, 67])
def test_clusters_say_nan_where_a_post_never_comes(simx, C, dtype, monkeypatch):
    """SIMX_WITHHOLD_COPIES keeps the last block of each cluster from posting, so the bounded waits (about a second)
    run out: what depends on a state from another block is NaN, the rest is what it was."""
    T = 5000
    c = _case(1, T, C, 41, 0.004)
    c["done"][0, :8] = c["done"][0, -8:] = 0
    x, gate, dh = (_tensor((1, T, C), dtype, "batch", c[k]) for k in ("x", "gate", "dh"))
    dn, h0 = _done(c["done"], "batch"), _dev(c["h0"])
    ws = torch.empty(simx.gated_scan_workspace_size(1, T, C), dtype=torch.uint8, device="cuda")

    def call(saved=None):
        h, dx, dg = (_tensor((1, T, C), dtype, "batch") for _ in range(3))
        last, d0, db = torch.zeros((1, C), device="cuda"), torch.zeros((1, C), device="cuda"), torch.zeros(C, device="cuda")
        simx.gated_scan(x, gate, h, h0=h0, done=dn, h_last=last)
        simx.gated_scan_grad(x, gate, h if saved is None else saved, dh, dx, dg, ws, h0=h0, done=dn, dbias=db, dh0=d0)
        torch.cuda.synchronize()
        return h, dx, dg, last, d0, db

    good = call()
    monkeypatch.setenv("SIMX_WITHHOLD_COPIES", "1")
    bad = call(good[0])
    monkeypatch.delenv("SIMX_WITHHOLD_COPIES")
    assert all(torch.equal(a, b) for a, b in zip(good, call()))
    h, dx, dg, last, d0, db = bad
    assert torch.isnan(h[:, 0]).all() and torch.isnan(dx[:, -1]).all() and torch.isnan(dg[:, -1]).all()
    assert torch.isnan(last).all() and torch.isnan(d0).all() and torch.isnan(db).all()
    for a, b in zip(good[:3], bad[:3]):
        there = ~torch.isnan(b)
        assert there.any() and torch.equal(a[there], b[there])


@pytest.mark.parametrize("dtype,B,cluster", [("f32", 48, 4), ("f32", 30, 8), ("bf16", 48, 8)])
def test_clusters_by_the_blocks_that_fit(simx, dtype, B, cluster):
    """One wave of blocks, where they fit: fp32 gradients in clusters of 8 two to an SM, the others three.  Every
    block leaves a row of partial sums of dbias in the workspace."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    if sms != 152:
        pytest.skip("sizes for 152 SMs")
    T, C = 2048, 64
    t = [_tensor((B, T, C), dtype, "batch", np.ones((B, T, C))) for _ in range(6)]
    size = simx.gated_scan_workspace_size(B, T, C)
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    simx.gated_scan_grad(*t, ws, dbias=torch.empty(C, device="cuda"))
    torch.cuda.synchronize()
    written = ~torch.isnan(ws.view(torch.float32)).view(-1, C)
    assert written[:B * cluster].all() and not written[B * cluster:].any()
