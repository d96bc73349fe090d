"""The sequence policy: its operators together against one network in torch's 64-bit autograd, its
single-token form against its sequence form, and a short training run.

The network is evaluated in fp32 with fp32 matrix products (width 64), so its values and gradients are
off by some 1e-6 of their terms per layer; they are held to 1e-4 of the gradient's norm per parameter.
"""
import numpy as np
import pytest

from oracle import seq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2607_05272_gb300 import build as B
    B.build()
    torch.backends.cuda.matmul.allow_tf32 = False
    from paper_2607_05272_gb300 import seqpolicy
    return seqpolicy


def _network(pol, b, p, step):
    """(parameters, logits [H * E, A]) in 64 bits with autograd."""
    w = {k: v.detach().double().cpu().requires_grad_() for k, v in pol.w.items()}
    obs, done, s = b["obs"].double().cpu(), b["done"].cpu(), b["state"].double().cpu()
    hh, e, d = obs.shape
    n, c = hh * e, pol.C
    keep = []
    for q in (2 * step, 2 * step + 1):
        k, scale = seq.keep_mask(n, c, p, pol.seed, q)
        keep.append(torch.from_numpy(k * scale))

    def norm(z, gain):
        return z * (z.square().mean(1, keepdim=True) + 1e-6).rsqrt() * gain
    z1 = (obs.reshape(n, d) @ w["w_in"].t()) * keep[0]
    pr = (norm(z1, w["gain1"]) @ w["w_p"].t()).view(hh, e, 2 * c)
    hs = []
    for t in range(hh):
        a = torch.sigmoid(pr[t, :, c:] + w["bias"])
        h = a * s + (1 - a) * pr[t, :, :c]
        hs.append(h)
        s = h * (done[t, :, None] == 0)
    z2 = z1 + (torch.stack(hs).reshape(n, c) @ w["w_o"].t()) * keep[1]
    return w, norm(z2, w["gain2"]) @ w["w_h"].t()


def _batch(pol, hh, e, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    return dict(obs=r(hh, e, pol.D), action=torch.randint(0, pol.A, (hh, e), generator=g, device="cuda"),
                logp=-2.0 + 0.2 * r(hh, e), reward=r(hh, e), state=r(e, pol.C),
                done=(torch.rand((hh, e), generator=g, device="cuda") < 0.1).to(torch.uint8))


def _compare(pol, w):
    for k, g in pol.g.items():
        ref = w[k].grad.numpy()
        assert np.linalg.norm(g.cpu().numpy() - ref) <= 1e-4 * np.linalg.norm(ref) + 1e-9, k


def _frozen(pol, monkeypatch):
    monkeypatch.setattr(pol, "_adam", lambda lr: None)


@pytest.mark.parametrize("width,p", [(64, 0.25), (20, 0.0), (33, 0.1)])
def test_policy_update_gradient(sp, monkeypatch, width, p):
    hh, e = 40, 6
    pol = sp.SeqPolicy(9, 17, e, hh, width, p=p, seed=3)
    _frozen(pol, monkeypatch)
    b = _batch(pol, hh, e, 1)
    adv = torch.randn((hh, e), device="cuda")
    stats = pol.update(b, adv, c_kl=0.1, c_entropy=0.05, clip=0.2).clone()
    w, logits = _network(pol, b, p, 0)
    lp = logits.log_softmax(1)
    a, old, A = b["action"].view(-1).cpu(), b["logp"].view(-1).double().cpu(), adv.view(-1).double().cpu()
    l = lp.gather(1, a[:, None])[:, 0]
    rho, d = (l - old).exp(), old - l
    surr = torch.minimum(rho * A, rho.clamp(0.8, 1.2) * A)
    ent = -(lp.exp() * lp).sum(1)
    loss = (-surr + 0.1 * (d.exp() - d - 1) - 0.05 * ent).mean()
    loss.backward()
    assert abs(stats[0].item() - loss.item()) <= 1e-4 * (1 + abs(loss.item()))
    _compare(pol, w)


def test_preference_update_gradient(sp, monkeypatch):
    hh, e, p = 24, 8, 0.2
    pol = sp.SeqPolicy(5, 7, e, hh, 64, p=p, seed=4)
    _frozen(pol, monkeypatch)
    b = _batch(pol, hh, e, 2)
    stats = pol.preference_update(b, beta=0.3).clone()
    w, logits = _network(pol, b, p, 0)
    l = logits.log_softmax(1).gather(1, b["action"].view(-1, 1).cpu())[:, 0]
    r = (l - b["logp"].view(-1).double().cpu()).view(hh, e).sum(0).view(-1, 2)
    ret = b["reward"].sum(0).cpu().view(-1, 2)
    sign = torch.where(ret[:, 1] > ret[:, 0], -1.0, 1.0).double()
    loss = -torch.nn.functional.logsigmoid(0.3 * sign * (r[:, 0] - r[:, 1])).mean()
    loss.backward()
    assert abs(stats[0].item() - loss.item()) <= 1e-4 * (1 + abs(loss.item()))
    _compare(pol, w)


def test_single_tokens_are_the_sequence(sp):
    hh, e = 30, 5
    pol = sp.SeqPolicy(6, 11, e, hh, 48, p=0.3, seed=5)
    b = _batch(pol, hh, e, 3)
    f = pol.forward(b["obs"], b["done"], b["state"], 0.0, 0)
    state = b["state"].clone()
    for t in range(hh):
        logits = pol.step(b["obs"][t], state)
        state.masked_fill_(b["done"][t, :, None] != 0, 0.0)
        ref = f["logits"].view(hh, e, -1)[t]
        assert (logits - ref).abs().max().item() <= 1e-4 * (1 + ref.abs().max().item())


def test_training_run_learns_and_repeats(sp):
    """Against the same run without updates: the reward per decision of an untrained policy on this
    workload stays near -2.4 from the first iterations on (queues fill whatever is learned)."""
    kw = dict(workload="c3s", envs=512, horizon=128, iters=50, width=64, every=0, seed=7)
    runs = [sp.train(**kw) for _ in range(2)]
    assert runs[0] == runs[1]  # the same bits: no order of atomics anywhere
    assert all(np.isfinite(list(h.values())).all() for h in runs[0])
    frozen = sp.train(lr=0.0, preferences=0, **kw)
    tail = lambda r: np.mean([h["mean_reward"] for h in r[-10:]])  # noqa: E731
    assert tail(runs[0]) > tail(frozen) + 0.5


def test_an_unchanged_policy_is_its_own_reference(sp, monkeypatch):
    """Before any step of the optimiser every ratio is 1 and the KL and all margins are 0, dropout or not, in every
    epoch.  log probabilities of one network and mask, within 1e-6 (1 + |lp|) of each other (|lp| < 10 here): a KL
    of d^2 / 2, margins of 0.1 times 32 such differences."""
    e, hh = 64, 16
    sim = sp.simx.Sim(sp.W.CONFIGS["c3s"](e))
    sim.reset(3)
    dims, has_value = sp.W.mlp_dims("c3s")
    pol = sp.SeqPolicy(sim.D, dims[-1] - int(has_value), e, hh, 64, p=0.3, seed=2)
    _frozen(pol, monkeypatch)
    state = torch.zeros((e, pol.C), device="cuda")
    for _ in range(2):
        b = pol.rollout(sim, state)
        adv = torch.randn((hh, e), device="cuda")
        for _ in range(2):
            s = pol.update(b, adv, c_entropy=0.0).tolist()
            assert abs(s[2]) <= 1e-9 and s[4] == 0.0
            assert abs(s[1] + adv.mean().item()) <= 2e-5 * adv.abs().mean().item()
        q = pol.preference_update(b).tolist()
        assert abs(q[0] - np.log(2)) <= 1e-4 and abs(q[2]) <= 1e-4
    sim.close()


def test_envs_of_equal_return_prefer_neither(sp, monkeypatch):
    """The first pair's returns are equal: loss and gradient are the other pairs' alone, whichever env comes first."""
    hh, e = 12, 6
    pol = sp.SeqPolicy(5, 7, e, hh, 32, p=0.1, seed=6)
    _frozen(pol, monkeypatch)
    b = _batch(pol, hh, e, 4)
    b["reward"][:, 0] = b["reward"][:, 1]
    out = []
    for logp in (-2.0, -1.0):  # of the second env: the pair's margin, not the others'
        b["logp"][:, 1] = logp
        pol.calls = 0
        out.append((pol.preference_update(b, beta=0.3).clone(), pol.grad_flat.clone()))
    assert out[0][1].any() and all(torch.equal(x, y) for x, y in zip(*out))
    b["reward"].zero_()
    stats = pol.preference_update(b, beta=0.3)
    assert not stats.any() and not pol.grad_flat.any()
