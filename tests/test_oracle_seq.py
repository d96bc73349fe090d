"""The 64-bit definitions of the sequence-policy operators: gradients against central differences,
and the dropout mask against the published Philox4x32-10 vectors.

A central difference with step e of a smooth function has the error O(e^2) + O(eps / e): with
e = 1e-5 about 1e-10 each way at values of order 1, so the gradients are held to 1e-7.
"""
import numpy as np
import pytest

from oracle import seq

STEP, TOL = 1e-5, 1e-7


def _differences(f, x):
    g = np.zeros_like(x)
    it = np.nditer(x, flags=["multi_index"])
    for _ in it:
        k = it.multi_index
        keep = x[k]
        x[k] = keep + STEP
        up = f()
        x[k] = keep - STEP
        down = f()
        x[k] = keep
        g[k] = (up - down) / (2 * STEP)
    return g


@pytest.mark.parametrize("kl,ent,temp,old", [(0.0, 0.0, 1.0, True), (0.3, 0.2, 0.7, True),
                                             (0.1, 0.05, 1.5, False)])
def test_token_loss_gradient(kl, ent, temp, old):
    rng = np.random.default_rng(3)
    n, V = 6, 7
    x = rng.standard_normal((n, V))
    act = rng.integers(0, V, n)
    lp = np.take_along_axis(seq.log_softmax(x, temp), act[:, None], 1)[:, 0]
    # on-policy, the ratio's gradient is that of log pi: the ratio to a frozen copy of itself
    kw = dict(adv=rng.standard_normal(n), logp_old=lp + (rng.standard_normal(n) * 0.4 if old else 0),
              logp_ref=lp + 0.3 * rng.standard_normal(n), weight=rng.random(n) * (rng.random(n) < 0.8),
              c_kl=kl, c_entropy=ent, temperature=temp)
    g = seq.token_loss(x, act, **kw)["grad"]
    d = _differences(lambda: seq.token_loss(x, act, **kw)["stats"][0], x)
    assert np.abs(g - d).max() <= TOL
    if not old:
        kw["logp_old"] = None
        assert np.abs(seq.token_loss(x, act, **kw)["grad"] - g).max() <= 1e-12


@pytest.mark.parametrize("eps,temp", [(0.0, 1.0), (0.2, 0.8)])
def test_preference_loss_gradient(eps, temp):
    rng = np.random.default_rng(4)
    start = np.array([0, 3, 3, 4, 6])
    x = rng.standard_normal((7, 5))  # the last row belongs to no sequence
    kw = dict(token=rng.integers(0, 5, 7), start=start, logp_ref=rng.standard_normal(7),
              mask=np.array([1, 0, 1, 1, 1, 1, 1]), weight=np.array([0.3, 0.9]), beta=0.5,
              smoothing=eps, temperature=temp)
    g = seq.preference_loss(x, **kw)["grad"]
    d = _differences(lambda: seq.preference_loss(x, **kw)["stats"][0], x)
    assert np.abs(g - d).max() <= TOL
    assert not g[6].any() and not g[1].any()


@pytest.mark.parametrize("done", [False, True])
def test_gated_scan_gradients(done):
    rng = np.random.default_rng(5)
    B, T, C = 2, 6, 3
    x, gate = rng.standard_normal((2, B, T, C))
    bias, h0 = rng.standard_normal(C), rng.standard_normal((B, C))
    dn = (rng.random((B, T)) < 0.3).astype(np.uint8) if done else None
    dh, dl = rng.standard_normal((B, T, C)), rng.standard_normal((B, C))

    def loss():
        o = seq.gated_scan(x, gate, bias, h0, dn)
        return (o["h"] * dh).sum() + (o["h_last"] * dl).sum()

    h = seq.gated_scan(x, gate, bias, h0, dn)["h"]
    g = seq.gated_scan_grad(x, gate, h, dh, bias, h0, dn, dl)
    for name, v in (("dx", x), ("dgate", gate), ("dbias", bias), ("dh0", h0)):
        assert np.abs(g[name] - _differences(loss, v)).max() <= TOL, name


@pytest.mark.parametrize("p", [0.0, 0.4])
def test_dropout_add_norm_gradients(p):
    rng = np.random.default_rng(6)
    n, W = 3, 11
    x, res, dy, dz = rng.standard_normal((4, n, W))
    gain = 1 + 0.3 * rng.standard_normal(W)
    keep, scale = seq.keep_mask(n, W, p, 99, 7)

    def loss():
        o = seq.dropout_add_norm(x, gain, res, keep, scale)
        return (o["y"] * dy).sum() + (o["z"] * dz).sum()

    o = seq.dropout_add_norm(x, gain, res, keep, scale)
    g = seq.dropout_add_norm_grad(o["z"], gain, o["rstd"], dy, dz, keep, scale)
    for name, v in (("dx", x), ("dresidual", res), ("dgain", gain)):
        assert np.abs(g[name] - _differences(loss, v)).max() <= TOL, name


def test_mask_fields_are_the_published_generator():
    # Philox4x32-10's known answers (Salmon et al.)
    assert seq.philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    f = 0xFFFFFFFF
    assert seq.philox((f, f, f, f), (f, f)) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def test_mask_keeps_its_share_and_moves_with_the_rows():
    keep, scale = seq.keep_mask(64, 96, 0.25, 5, 3)
    assert abs(keep.mean() - 0.75) < 5 * np.sqrt(0.25 * 0.75 / keep.size)
    assert abs(scale - 4 / 3) < 1e-4
    assert np.array_equal(seq.keep_mask(10, 96, 0.25, 5, 3, row_base=20)[0], keep[20:30])
    assert not np.array_equal(seq.keep_mask(64, 96, 0.25, 5, 4)[0], keep)
