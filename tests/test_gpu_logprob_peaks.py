"""Log probabilities and entropies of rows with a peak late in the row: differences of numbers that are near one
another if the sums' reference is far below the peak.  Tolerances as in test_gpu_logprobs: there all of a term's
roundings count with y = (x - max) / T; a reference at most 2^8 below its thread's largest term adds 2^-24 of
8 log 2 = 5.6 twice, in the exponential's argument and where the sums move, 7e-7 together."""
import numpy as np
import pytest

from tests.test_gpu_logprobs import BOTH, _check, _rows, _run, simx  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@BOTH
@pytest.mark.parametrize("V,n", [(40, 12), (3000, 12), (9000, 3000), (50000, 12), (50000, 400), (131072, 6)])
@pytest.mark.parametrize("temperature", [0.7, 0.8, 1.0, 3.0])
def test_peaks(simx, V, n, temperature, dtype):  # noqa: F811
    """One token 2 to 60 nats above the rest, at the end of its row or anywhere: constant rows and random ones."""
    r = np.random.default_rng(V + n)
    x = r.standard_normal((n, V)) * np.where(np.arange(n) % 2, 0.5, 0.0)[:, None]
    gaps = np.linspace(2, 60, n) * temperature
    at = np.where(np.arange(n) % 3 == 0, V - 1, r.integers(0, V, n))
    x[np.arange(n), at] += gaps
    _check(simx, x, dtype, top=3, temperature=temperature)
    logits = _rows(x, dtype, 0, 0)
    lp, H, tl, ti = _run(simx, logits, torch.from_numpy(at).cuda(), 3, temperature)
    assert (lp <= 0).all() and (tl <= 0).all() and (H >= 0).all()
    want = (logits.double() / float(np.float32(temperature))).log_softmax(1).cpu().numpy()[np.arange(n), at]
    assert (np.abs(lp.double().cpu().numpy() - want) <= 2e-6 * (1 + np.abs(want))).all()


@pytest.mark.parametrize("temperature", [0.7, 1.0])
def test_steps_up(simx, temperature):  # noqa: F811
    """Rows that rise in steps of 1 to 30 nats, so that references lag by every distance."""
    V = 50000
    x = np.stack([np.floor(np.linspace(0, 9.99, V)) * s for s in (1.0, 3.0, 5.0, 5.5, 6.0, 11.0, 20.0, 30.0)]) * temperature
    for rows in (x, np.repeat(x, 60, 0)):
        _check(simx, rows, "f32", top=2, temperature=temperature)
