"""The operators of sequence policies, as cases that can be timed and compared.

A policy with memory, or one that picks from a large vocabulary, is made of four operators:

* ``token``  the clipped policy loss with its KL and entropy terms, from logits to the
             logits' gradient (``simx.token_loss_grad``);
* ``pref``   the preference loss on pairs of sequences: paired log ratios, from logits to
             the logits' gradient (``simx.preference_loss_grad``);
* ``scan``   the gated linear recurrence h_t = a_t h_{t-1} + (1 - a_t) x_t with
             a_t = sigma(gate_t + bias), forward and backward, and its single-token form
             (``simx.gated_scan``, ``simx.gated_scan_grad``);
* ``norm``   dropout, residual addition and root-mean-square norm in one, forward and
             backward, with a mask that is drawn from counters and never stored
             (``simx.dropout_add_norm``, ``simx.dropout_add_norm_grad``).

With ``own`` false ``run`` computes them from elementary torch operations in 32 bits, rounded
once at the end; with ``own`` true it calls the library.  Sizes of the actions, minibatches and
horizons are the repository's own (48 actions, minibatches of 8192 rows, 512 decisions); the
others are generic.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}

# A drawn case moves no more than the largest listed one of its kind.
MOST_LOGIT_BYTES = 8192 * 131072 * 2
MOST_SCAN = 2 * 65536 * 1024
MOST_NORM = 16384 * 4096


def listed():
    return [
        # One PPO minibatch of the benchmark's 48 actions: the library's own loss shape, but with
        # logits from a network outside it.
        dict(name="token actions 8192x48 f32", kind="token", n=8192, vocab=48, dtype="f32",
             masked=0.0, banned=0, temperature=1.0, kl=0.0, entropy=0.01),
        # A handful of tokens of a large vocabulary: the tail of a batch, latency counts.
        dict(name="token few 8x131072 bf16", kind="token", n=8, vocab=131072, dtype="bf16",
             masked=0.0, banned=0, temperature=1.0, kl=0.05, entropy=0.0),
        # An odd vocabulary in fp32 (rows that start at any alignment), padding and banned tokens.
        dict(name="token ragged 1021x50001 f32", kind="token", n=1021, vocab=50001, dtype="f32",
             masked=0.25, banned=16, temperature=0.7, kl=0.05, entropy=0.01),
        # A training micro-batch of 8192 tokens of a large vocabulary: the largest call.
        dict(name="token large 8192x131072 bf16", kind="token", n=8192, vocab=131072, dtype="bf16",
             masked=0.125, banned=0, temperature=1.0, kl=0.05, entropy=0.0),
        # Four pairs of short answers over a small vocabulary.
        dict(name="pref small 4x64 v4099 f32", kind="pref", pairs=4, longest=64, vocab=4099,
             dtype="f32", smoothing=0.0),
        # A preference-tuning step: 32 pairs of up to 512 tokens.
        dict(name="pref large 32x512 v32768 bf16", kind="pref", pairs=32, longest=512, vocab=32768,
             dtype="bf16", smoothing=0.1),
        # Serving: one token of 256 sequences, the state updated in place.
        dict(name="scan step 256x1x2048 bf16", kind="scan", dir="forward", batch=256, len=1,
             channels=2048, dtype="bf16", layout="batch", done=False),
        # Two long sequences: few rows, a long axis.
        dict(name="scan long 2x65536x1024 bf16", kind="scan", dir="forward", batch=2, len=65536,
             channels=1024, dtype="bf16", layout="packed", done=False),
        # The backward pass over a rollout buffer: time-major, 512 decisions, episodes that end.
        dict(name="scan grad 1024x512x64 f32", kind="scan", dir="grad", batch=1024, len=512,
             channels=64, dtype="f32", layout="time", done=True),
        # The backward pass of a training batch of packed sequences.
        dict(name="scan grad 16x2048x2048 bf16", kind="scan", dir="grad", batch=16, len=2048,
             channels=2048, dtype="bf16", layout="packed", done=True),
        # A training batch: dropout, residual and norm of 16384 tokens.
        dict(name="norm 16384x4096 bf16", kind="norm", dir="forward", n=16384, width=4096,
             dtype="bf16", p=0.1),
        # Its backward pass, at an odd width that leaves rows unaligned.
        dict(name="norm grad 16384x2047 bf16", kind="norm", dir="grad", n=16384, width=2047,
             dtype="bf16", p=0.1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["token", "token", "pref", "scan", "scan", "scan", "norm", "norm"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if kind == "token":
        vocab = _log(rng, 2, 131072)
        n = max(1, min(_log(rng, 1, 65536), MOST_LOGIT_BYTES // (vocab * SIZE[dtype])))
        return dict(kind=kind, n=n, vocab=vocab, dtype=dtype, masked=rng.choice([0.0, 0.25, 0.9]),
                    banned=rng.choice([0, 0, 16]), temperature=rng.choice([1.0, 1.0, 0.7, 1.5]),
                    kl=rng.choice([0.0, 0.05]), entropy=rng.choice([0.0, 0.01]))
    if kind == "pref":
        vocab, longest = _log(rng, 16, 65536), _log(rng, 4, 2048)
        pairs = max(1, min(_log(rng, 1, 64),
                           MOST_LOGIT_BYTES // (2 * longest * vocab * SIZE[dtype])))
        return dict(kind=kind, pairs=pairs, longest=longest, vocab=vocab, dtype=dtype,
                    smoothing=rng.choice([0.0, 0.1]))
    if kind == "scan":
        channels, length = _log(rng, 1, 4096), _log(rng, 1, 65536)
        batch = max(1, min(_log(rng, 1, 1024), MOST_SCAN // (channels * length)))
        return dict(kind=kind, dir=rng.choice(["forward", "grad"]), batch=batch, len=length,
                    channels=channels, dtype=dtype,
                    layout=rng.choice(["batch", "packed", "time"]), done=rng.random() < 0.5)
    width = _log(rng, 16, 8192)
    n = max(1, min(_log(rng, 1, 65536), MOST_NORM // width))
    return dict(kind=kind, dir=rng.choice(["forward", "grad"]), n=n, width=width, dtype=dtype,
                p=rng.choice([0.0, 0.1, 0.5]))


# ---------------------------------------------------------------------------- sizes of a case

def _active(case):
    """Rows of a token case whose weight is not zero."""
    return case["n"] - int(case["n"] * case["masked"])


def _lengths(case):
    """(prompt, whole) lengths of the 2 * pairs sequences of a pref case; the two sequences of a
    pair share their prompt.  Fixed by the case, so that work() knows them."""
    r = random.Random(case["pairs"] * 1000003 + case["longest"])
    out = []
    for _ in range(case["pairs"]):
        prompt = r.randint(0, case["longest"] // 3)
        for _ in range(2):
            out.append((prompt, r.randint(prompt, case["longest"])))
    return out


def work(case):
    es = SIZE[case["dtype"]]
    if case["kind"] == "token":
        read = _active(case) * case["vocab"]
        return {"bytes": (read + case["n"] * case["vocab"]) * es + case["n"] * 32, "flops": 10 * read}
    if case["kind"] == "pref":
        ls = _lengths(case)
        rows, read = sum(l for _, l in ls), sum(l - p for p, l in ls)
        v = case["vocab"]
        return {"bytes": (read + rows) * v * es + rows * 17 + case["pairs"] * 36,
                "flops": 10 * read * v}
    if case["kind"] == "scan":
        bc = case["batch"] * case["channels"]
        m = bc * case["len"]
        done = case["batch"] * case["len"] if case["done"] else 0
        if case["dir"] == "forward":
            return {"bytes": 3 * m * es + 8 * bc + done, "flops": 10 * m}
        return {"bytes": 6 * m * es + 12 * bc + done, "flops": 16 * m}
    m = case["n"] * case["width"]
    if case["dir"] == "forward":
        return {"bytes": 4 * m * es + 4 * case["n"], "flops": 8 * m}
    return {"bytes": 5 * m * es + 4 * case["n"], "flops": 12 * m}


# ---------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _chunks(n, width):
    step = max(1, (1 << 27) // width)
    return [(i, min(n, i + step)) for i in range(0, n, step)]


def _logits(g, n, vocab, dtype, temperature, banned):
    """Logits of a trained-looking policy (standard deviation 2), tokens sampled from them, and
    the tokens' log probabilities.  banned: one token in so many has a logit of -inf."""
    logits = torch.empty((n, vocab), dtype=DT[dtype], device="cuda")
    token = torch.empty(n, dtype=torch.int64, device="cuda")
    logp = torch.empty(n, device="cuda")
    out = None
    if banned and vocab > 1:
        out = torch.rand(vocab, generator=g, device="cuda") < 1.0 / banned
        out[0] = False
    for a, b in _chunks(n, vocab):
        x = (_randn(g, b - a, vocab) * 2.0).to(DT[dtype])
        if out is not None:
            x[:, out] = -math.inf
        logits[a:b] = x
        f = x.float() / temperature
        e = torch.empty_like(f).exponential_(generator=g)
        token[a:b] = (f - e.log()).argmax(1)
        logp[a:b] = f.log_softmax(1).gather(1, token[a:b, None])[:, 0]
    return logits, token, logp


CLIP = (0.2, 0.28)  # below, above


def _prepare_token(case, seed):
    g, n = _gen(seed), case["n"]
    logits, action, lp = _logits(g, n, case["vocab"], case["dtype"], case["temperature"],
                                 case["banned"])
    # log ratios of a few epochs' drift; those on a clip edge (where the loss has a kink and 32
    # bits cannot tell the side) are moved off it
    d = _randn(g, n) * 0.15
    for edge in (math.log1p(-CLIP[0]), math.log1p(CLIP[1])):
        d = torch.where((d - edge).abs() < 1e-3, torch.full_like(d, edge + 1e-3), d)
    weight = torch.full((n,), 1.0 / _active(case), device="cuda")
    weight[torch.randperm(n, generator=g, device="cuda")[_active(case):]] = 0.0
    return dict(logits=logits, action=action, logp_old=lp - d,
                logp_ref=lp + _randn(g, n) * 0.2 if case["kl"] else None,
                adv=_randn(g, n), weight=weight,
                grad=torch.empty_like(logits), stats=torch.empty(5, device="cuda"),
                logp=torch.empty(n, device="cuda"), entropy=torch.empty(n, device="cuda"))


def _prepare_pref(case, seed):
    g, ls = _gen(seed), _lengths(case)
    n = sum(l for _, l in ls)
    start = np.concatenate([[0], np.cumsum([l for _, l in ls])]).astype(np.int64)
    mask = np.zeros(n, np.uint8)
    for (p, l), s in zip(ls, start):
        mask[s + p:s + l] = 1
    logits, token, lp = _logits(g, n, case["vocab"], case["dtype"], 1.0, 0)
    return dict(logits=logits, token=token, seq_start=torch.from_numpy(start).cuda(),
                mask=torch.from_numpy(mask).cuda(), logp_ref=lp + _randn(g, n) * 0.3,
                weight=torch.full((case["pairs"],), 1.0 / case["pairs"], device="cuda"),
                grad=torch.empty_like(logits), stats=torch.empty(3, device="cuda"),
                ratio=torch.empty(2 * case["pairs"], device="cuda"),
                margin=torch.empty(case["pairs"], device="cuda"))


def _sequence(case, parts):
    """`parts` tensors [batch, len, channels] in the case's layout: batch-major, halves of one
    packed projection, or views of time-major buffers."""
    b, t, c, dt = case["batch"], case["len"], case["channels"], DT[case["dtype"]]
    if case["layout"] == "packed":
        return list(torch.empty((b, t, parts * c), dtype=dt, device="cuda").split(c, dim=2))
    if case["layout"] == "time":
        return [torch.empty((t, b, c), dtype=dt, device="cuda").transpose(0, 1) for _ in range(parts)]
    return [torch.empty((b, t, c), dtype=dt, device="cuda") for _ in range(parts)]


def _prepare_scan(case, seed):
    g = _gen(seed)
    b, t, c = case["batch"], case["len"], case["channels"]
    x, gate = _sequence(case, 2)
    x.copy_(_randn(g, b, t, c))
    gate.copy_(_randn(g, b, t, c) * 1.5 + 2.0)  # gates that mostly remember
    s = dict(x=x, gate=gate, bias=_randn(g, c) * 0.5, h0=_randn(g, b, c), done=None)
    if case["done"]:
        done = torch.rand((t, b), generator=g, device="cuda") < 1.0 / 128
        s["done"] = done.to(torch.uint8).t()
    if case["dir"] == "forward":
        s["h"] = _sequence({**case, "layout": "time" if case["layout"] == "time" else "batch"}, 1)[0]
        s["h_last"] = torch.empty((b, c), device="cuda")
        return s
    h = torch.empty_like(x)
    h.copy_(_scan_forward(x, gate, s["bias"], s["h0"], s["done"])[0])  # what the forward pass saved
    s["h"] = h
    s["dh"] = torch.empty_like(h)
    s["dh"].copy_(_randn(g, b, t, c))
    s["dh_last"] = _randn(g, b, c)
    s["dx"], s["dgate"] = _sequence(case, 2)
    s["dbias"] = torch.empty(c, device="cuda")
    s["dh0"] = torch.empty((b, c), device="cuda")
    return s


def _prepare_norm(case, seed):
    g, n, d, dt = _gen(seed), case["n"], case["width"], DT[case["dtype"]]
    s = dict(gain=1.0 + _randn(g, d) * 0.1, seed=int(seed) * 7919 + 12345, step=int(seed) % 1000)
    residual = (_randn(g, n, d) * 1.5).to(dt)
    x = _randn(g, n, d).to(dt)
    if case["dir"] == "forward":
        s.update(x=x, residual=residual, z=torch.empty_like(x), y=torch.empty_like(x),
                 rstd=torch.empty(n, device="cuda"))
        return s
    z = residual.float() + x.float()
    s.update(z=z.to(dt), rstd=(z.square().mean(1) + EPS).rsqrt(), dy=_randn(g, n, d).to(dt),
             dz=_randn(g, n, d).to(dt), dx=torch.empty_like(x), dresidual=torch.empty_like(x),
             dgain=torch.empty(d, device="cuda"))
    return s


EPS = 1e-6


def prepare(case, seed):
    s = {"token": _prepare_token, "pref": _prepare_pref, "scan": _prepare_scan,
         "norm": _prepare_norm}[case["kind"]](case, seed)
    s["case"] = case
    return s


# ---------------------------------------------------------------------------- plain forms

def _rows(logits, token, temperature):
    """(e, s, shifted, log probability of the token) of each row, in 32 bits."""
    x = logits.float()
    x = (x - x.amax(1, keepdim=True)) / temperature
    e = x.exp()
    s = e.sum(1, keepdim=True)
    return e, s, x, x.gather(1, token[:, None])[:, 0] - s[:, 0].log()


def _plain_token(s):
    c = s["case"]
    w, adv = s["weight"], s["adv"]
    on = w != 0
    e, tot, x, lp = _rows(s["logits"], s["action"], c["temperature"])
    p = e / tot
    lps = x - tot.log()
    ent = -torch.where(e > 0, p * lps, 0.0).sum(1)
    rho = (lp - s["logp_old"]).exp()
    a, b = rho * adv, rho.clamp(1 - CLIP[0], 1 + CLIP[1]) * adv
    surr = torch.minimum(a, b)
    clipped = b < a
    if s["logp_ref"] is None:
        kl, dkl = torch.zeros_like(lp), torch.zeros_like(lp)
    else:
        d = s["logp_ref"] - lp
        kl, dkl = d.expm1() - d, -d.expm1()
    off = torch.zeros_like(lp)
    surr, kl, ent, lp = (torch.where(on, v, off) for v in (surr, kl, ent, lp))
    pol, kls, ents = -(w * surr).sum(), (w * kl).sum(), (w * ent).sum()
    stats = torch.stack([pol + c["kl"] * kls - c["entropy"] * ents, pol, kls, ents,
                         (w * clipped).sum()])
    coef = w * (torch.where(clipped, 0.0, -a) + c["kl"] * dkl)
    grad = -coef[:, None] * p
    if c["entropy"]:
        grad += (w * c["entropy"])[:, None] * torch.where(e > 0, p * (lps + ent[:, None]), 0.0)
    grad.scatter_add_(1, s["action"][:, None], coef[:, None])
    grad = torch.where(on[:, None], grad / c["temperature"], 0.0)
    return {"grad": grad.to(s["logits"].dtype), "stats": stats, "logp": lp, "entropy": ent}


BETA = 0.1


def _plain_pref(s):
    c = s["case"]
    eps, w, pairs = c["smoothing"], s["weight"], c["pairs"]
    n = len(s["token"])
    e, tot, _, lp = _rows(s["logits"], s["token"], 1.0)
    at = torch.arange(n, device="cuda")
    seq = (at[:, None] >= s["seq_start"][None, 1:]).sum(1)
    on = s["mask"] != 0
    ratio = torch.zeros(2 * pairs, device="cuda").index_add_(
        0, seq, torch.where(on, lp - s["logp_ref"], 0.0))
    h = BETA * (ratio[0::2] - ratio[1::2])
    soft = lambda v: v.clamp(min=0) + (-v.abs()).exp().log1p()  # noqa: E731
    loss = (1 - eps) * soft(-h) + eps * soft(h)
    dh = w * BETA * (1 / (1 + (-h).exp()) - (1 - eps))
    coef = torch.stack([dh, -dh], 1).reshape(-1)[seq] * on
    grad = -coef[:, None] * (e / tot)
    grad.scatter_add_(1, s["token"][:, None], coef[:, None])
    stats = torch.stack([(w * loss).sum(), (w * (h > 0)).sum(), (w * h).sum()])
    return {"grad": grad.to(s["logits"].dtype), "stats": stats, "ratio": ratio, "margin": h}


def _doubling(a, u):
    """u_t + a_t u_{t-1} + a_t a_{t-1} u_{t-2} + ... along dim 1, in log2(len) sweeps."""
    d = 1
    while d < a.shape[1]:
        u = torch.cat([u[:, :d], u[:, d:] + a[:, d:] * u[:, :-d]], 1)
        a = torch.cat([a[:, :d], a[:, d:] * a[:, :-d]], 1)
        d *= 2
    return u


def _scan_forward(x, gate, bias, h0, done):
    """(h, carried state after the last step) in 32 bits."""
    z = gate.float() + bias
    a, na = torch.sigmoid(z), torch.sigmoid(-z)
    u = na * x.float()
    if done is not None:
        a = a.clone()
        a[:, 1:] = torch.where(done[:, :-1, None] != 0, 0.0, a[:, 1:])
    u[:, 0] += a[:, 0] * h0
    h = _doubling(a, u)
    last = h[:, -1]
    return h, last if done is None else torch.where(done[:, -1:] != 0, 0.0, last)


def _plain_scan(s):
    x, gate, bias, h0, done = s["x"], s["gate"], s["bias"], s["h0"], s["done"]
    if s["case"]["dir"] == "forward":
        h, last = _scan_forward(x, gate, bias, h0, done)
        return {"h": h.to(x.dtype), "h_last": last.contiguous()}
    z = gate.float() + bias
    a, na = torch.sigmoid(z), torch.sigmoid(-z)
    h = s["h"].float()
    carried = torch.cat([h0[:, None], h[:, :-1]], 1)
    keep = torch.ones_like(a[:, :1, :1]) if done is None else (done[:, :, None] == 0).float()
    if done is not None:
        carried[:, 1:] = torch.where(done[:, :-1, None] != 0, 0.0, carried[:, 1:])
    # lambda_t = dh_t + keep_t a_{t+1} lambda_{t+1}, from the last step back
    nxt = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], 1) * keep
    u = s["dh"].float().clone()
    u[:, -1] += nxt[:, -1] * s["dh_last"]
    lam = _doubling(nxt.flip(1), u.flip(1)).flip(1)
    dx = lam * na
    dg = lam * (carried - x.float()) * (a * na)
    return {"dx": dx.to(x.dtype), "dgate": dg.to(x.dtype), "dbias": dg.sum((0, 1)),
            "dh0": a[:, 0] * lam[:, 0]}


_M32 = 0xFFFFFFFF


def _keep(seed, step, n, width, p):
    """(mask [n, width], scale) of the dropout: Philox4x32-10 with the counter
    (column / 8, row, step, 6), eight 16-bit fields a draw, each kept from round(65536 p) on."""
    thr = int(math.floor(p * 65536 + 0.5))
    groups = (width + 7) // 8
    c0 = torch.arange(groups, device="cuda").expand(n, groups)
    c1 = torch.arange(n, device="cuda")[:, None].expand(n, groups)
    c2, c3 = torch.full_like(c0, step), torch.full_like(c0, 6)
    k0, k1 = seed & _M32, (seed >> 32) & _M32
    for _ in range(10):
        m0, m1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((m1 >> 32) & _M32) ^ c1 ^ k0, m1 & _M32, ((m0 >> 32) & _M32) ^ c3 ^ k1, m0 & _M32
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    f = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16,
                     c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], 2)
    return (f >= thr).reshape(n, groups * 8)[:, :width], 65536.0 / (65536 - thr)


def _plain_norm(s):
    c = s["case"]
    n, d, p = c["n"], c["width"], c["p"]
    keep, scale = _keep(s["seed"], s["step"], n, d, p) if p > 0 else (None, 1.0)
    drop = lambda v: v if keep is None else torch.where(keep, v * scale, 0.0)  # noqa: E731
    if c["dir"] == "forward":
        z = s["residual"].float() + drop(s["x"].float())
        r = 1 / (z.square().mean(1) + EPS).sqrt()
        dt = s["x"].dtype
        return {"z": z.to(dt), "y": (z * r[:, None] * s["gain"]).to(dt), "rstd": r}
    zh = s["z"].float() * s["rstd"][:, None]
    dy = s["dy"].float()
    g = dy * s["gain"]
    dz = s["dz"].float() + s["rstd"][:, None] * (g - zh * (g * zh).mean(1, keepdim=True))
    dt = s["z"].dtype
    return {"dx": drop(dz).to(dt), "dresidual": dz.to(dt), "dgain": (dy * zh).sum(0)}


# ---------------------------------------------------------------------------- the library's calls

def _workspace(s, size):
    """The workspace that a program keeps between its calls."""
    if "ws" not in s:
        s["ws"] = torch.empty(max(size(), 16), dtype=torch.uint8, device="cuda")
    return s["ws"]


def _own_token(s):
    from paper_2607_05272_gb300 import simx
    c = s["case"]
    ws = _workspace(s, lambda: simx.token_loss_grad_workspace_size(c["n"]))
    simx.token_loss_grad(s["logits"], s["action"], s["adv"], s["stats"], ws, logp_old=s["logp_old"],
                         logp_ref=s["logp_ref"], weight=s["weight"], clip_low=CLIP[0],
                         clip_high=CLIP[1], c_kl=c["kl"], c_entropy=c["entropy"],
                         temperature=c["temperature"], grad=s["grad"], logp=s["logp"],
                         entropy=s["entropy"])
    return {"grad": s["grad"], "stats": s["stats"], "logp": s["logp"], "entropy": s["entropy"]}


def _own_pref(s):
    from paper_2607_05272_gb300 import simx
    c = s["case"]
    ws = _workspace(s, lambda: simx.preference_loss_grad_workspace_size(len(s["token"]), c["pairs"]))
    simx.preference_loss_grad(s["logits"], s["token"], s["seq_start"], s["stats"], ws,
                              logp_ref=s["logp_ref"], mask=s["mask"], weight=s["weight"], beta=BETA,
                              label_smoothing=c["smoothing"], grad=s["grad"], ratio=s["ratio"],
                              margin=s["margin"])
    return {"grad": s["grad"], "stats": s["stats"], "ratio": s["ratio"], "margin": s["margin"]}


def _own_scan(s):
    from paper_2607_05272_gb300 import simx
    c = s["case"]
    ws = _workspace(s, lambda: simx.gated_scan_workspace_size(c["batch"], c["len"], c["channels"]))
    if c["dir"] == "forward":
        simx.gated_scan(s["x"], s["gate"], s["h"], ws, bias=s["bias"], h0=s["h0"], done=s["done"],
                        h_last=s["h_last"])
        return {"h": s["h"], "h_last": s["h_last"]}
    simx.gated_scan_grad(s["x"], s["gate"], s["h"], s["dh"], s["dx"], s["dgate"], ws,
                         bias=s["bias"], h0=s["h0"], done=s["done"], dh_last=s["dh_last"],
                         dbias=s["dbias"], dh0=s["dh0"])
    return {"dx": s["dx"], "dgate": s["dgate"], "dbias": s["dbias"], "dh0": s["dh0"]}


def _own_norm(s):
    from paper_2607_05272_gb300 import simx
    c = s["case"]
    if c["dir"] == "forward":
        simx.dropout_add_norm(s["x"], s["gain"], s["y"], residual=s["residual"], z=s["z"],
                              rstd=s["rstd"], p=c["p"], eps=EPS, seed=s["seed"], step=s["step"])
        return {"z": s["z"], "y": s["y"], "rstd": s["rstd"]}
    ws = _workspace(s, lambda: simx.dropout_add_norm_grad_workspace_size(c["n"], c["width"]))
    simx.dropout_add_norm_grad(s["z"], s["gain"], s["rstd"], s["dy"], s["dx"], ws, dz=s["dz"],
                               dresidual=s["dresidual"], dgain=s["dgain"], p=c["p"],
                               seed=s["seed"], step=s["step"])
    return {"dx": s["dx"], "dresidual": s["dresidual"], "dgain": s["dgain"]}


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"token": _own_token, "pref": _own_pref, "scan": _own_scan, "norm": _own_norm}[kind](state)
    return {"token": _plain_token, "pref": _plain_pref, "scan": _plain_scan, "norm": _plain_norm}[kind](state)


# ---------------------------------------------------------------------------- 64 bits

def _exact_token(case, s):
    t, n = case["temperature"], case["n"]
    grad = torch.zeros(s["logits"].shape, dtype=torch.float64, device="cuda")
    lp_out = torch.zeros(n, dtype=torch.float64, device="cuda")
    h_out = torch.zeros_like(lp_out)
    sums = torch.zeros(4, dtype=torch.float64, device="cuda")
    for a, b in _chunks(n, case["vocab"] * 2):
        rows = torch.nonzero(s["weight"][a:b])[:, 0] + a
        if not len(rows):
            continue
        w, adv, old = (s[k][rows].double() for k in ("weight", "adv", "logp_old"))
        one = torch.arange(len(rows), device="cuda")
        act = s["action"][rows]
        logp = torch.log_softmax(s["logits"][rows].double() / t, 1)
        p = logp.exp()
        lp = logp[one, act]
        ent = torch.special.entr(p).sum(1)
        ratio = torch.exp(lp - old)
        low, high = 1 - CLIP[0], 1 + CLIP[1]
        over = ((adv > 0) & (ratio > high)) | ((adv < 0) & (ratio < low))
        taken = torch.where(over, torch.where(adv > 0, high, low), ratio)
        co = torch.where(over, 0.0, -ratio * adv)
        k3 = torch.zeros_like(lp)
        if s["logp_ref"] is not None:
            d = s["logp_ref"][rows].double() - lp
            k3 = torch.exp(d) - 1 - d
            co = co + case["kl"] * (1 - torch.exp(d))
        g = -co[:, None] * p
        if case["entropy"]:
            g += case["entropy"] * (p * ent[:, None] - torch.special.entr(p))
        g[one, act] += co
        grad[rows] = g * (w / t)[:, None]
        lp_out[rows], h_out[rows] = lp, ent
        sums += torch.stack([-(w * taken * adv).sum(), (w * k3).sum(), (w * ent).sum(),
                             (w * over).sum()])
    loss = sums[0] + case["kl"] * sums[1] - case["entropy"] * sums[2]
    return {"grad": grad, "stats": torch.cat([loss[None], sums]), "logp": lp_out, "entropy": h_out}


def _exact_pref(case, s):
    start = s["seq_start"].tolist()
    ratios = []
    for a, b in zip(start[:-1], start[1:]):
        r = torch.zeros((), dtype=torch.float64, device="cuda")
        if b > a:
            lp = torch.log_softmax(s["logits"][a:b].double(), 1).gather(1, s["token"][a:b, None])[:, 0]
            r = ((lp - s["logp_ref"][a:b].double()) * s["mask"][a:b].double()).sum()
        ratios.append(r)
    ratio = torch.stack(ratios)
    h = BETA * (ratio[0::2] - ratio[1::2])
    w, eps = s["weight"].double(), case["smoothing"]
    logsig = torch.nn.functional.logsigmoid
    loss = -(1 - eps) * logsig(h) - eps * logsig(-h)
    slope = w * BETA * (eps * torch.sigmoid(h) - (1 - eps) * torch.sigmoid(-h))
    grad = torch.zeros(s["logits"].shape, dtype=torch.float64, device="cuda")
    for q, (a, b) in enumerate(zip(start[:-1], start[1:])):
        if b > a:
            g = -torch.softmax(s["logits"][a:b].double(), 1)
            g[torch.arange(b - a, device="cuda"), s["token"][a:b]] += 1
            sign = 1.0 if q % 2 == 0 else -1.0
            grad[a:b] = g * (sign * slope[q // 2] * s["mask"][a:b].double())[:, None]
    stats = torch.stack([(w * loss).sum(), (w * (h > 0)).sum(), (w * h).sum()])
    return {"grad": grad, "stats": stats, "ratio": ratio, "margin": h}


def _exact_scan(case, s):
    b, t, c = case["batch"], case["len"], case["channels"]
    ends = None if s["done"] is None else s["done"].t() != 0  # [t, b]
    bias, zero = s["bias"].double(), torch.zeros((), dtype=torch.float64, device="cuda")
    if case["dir"] == "forward":
        h = s["h0"].double()
        out = torch.empty((b, t, c), dtype=torch.float64, device="cuda")
        for i in range(t):
            f = torch.sigmoid(s["gate"][:, i].double() + bias)
            h = torch.lerp(s["x"][:, i].double(), h, f)
            out[:, i] = h
            if ends is not None:
                h = torch.where(ends[i][:, None], zero, h)
        return {"h": out, "h_last": h.clone()}
    dx = torch.empty((b, t, c), dtype=torch.float64, device="cuda")
    dg = torch.empty_like(dx)
    back = s["dh_last"].double()  # what reaches the state that step i hands on
    for i in range(t - 1, -1, -1):
        lam = s["dh"][:, i].double()
        lam = lam + (back if ends is None else torch.where(ends[i][:, None], zero, back))
        z = s["gate"][:, i].double() + bias
        f, r = torch.sigmoid(z), torch.sigmoid(-z)
        prev = s["h0"].double() if i == 0 else s["h"][:, i - 1].double()
        if i and ends is not None:
            prev = torch.where(ends[i - 1][:, None], zero, prev)
        dx[:, i] = lam * r
        dg[:, i] = lam * f * r * (prev - s["x"][:, i].double())
        back = lam * f
    return {"dx": dx, "dgate": dg, "dbias": dg.sum((0, 1)), "dh0": back}


def _philox_fields(seed, step, n, width):
    """The 16-bit fields again, in numpy on unsigned 64-bit words."""
    groups = (width + 7) // 8
    u, m, sh = np.uint64, np.uint64(_M32), np.uint64(32)
    x = np.broadcast_to(np.arange(groups, dtype=u), (n, groups))
    y = np.broadcast_to(np.arange(n, dtype=u)[:, None], (n, groups))
    z, v = np.full((n, groups), step, u), np.full((n, groups), 6, u)
    ka, kb = seed & _M32, (seed >> 32) & _M32
    for r in range(10):
        a = u((ka + r * 0x9E3779B9) & _M32)
        b = u((kb + r * 0xBB67AE85) & _M32)
        p, q = x * u(0xD2511F53), z * u(0xCD9E8D57)
        x, y, z, v = (q >> sh) ^ y ^ a, q & m, (p >> sh) ^ v ^ b, p & m
    f = np.stack([x, y, z, v], -1).astype(np.uint32)
    return np.stack([f & 0xFFFF, f >> 16], -1).reshape(n, groups * 8)[:, :width]


def _exact_norm(case, s):
    keep = None
    if case["p"] > 0:
        thr = int(math.floor(case["p"] * 65536 + 0.5))
        f = _philox_fields(s["seed"], s["step"], case["n"], case["width"])
        keep = torch.from_numpy((f >= thr) * (65536.0 / (65536 - thr))).cuda()
    gain = s["gain"].double()
    if case["dir"] == "forward":
        x = s["x"].double()
        z = s["residual"].double() + (x if keep is None else x * keep)
        r = (z.pow(2).sum(1) / case["width"] + EPS).pow(-0.5)
        return {"z": z, "y": z * gain * r[:, None], "rstd": r}
    r = s["rstd"].double()[:, None]
    z, dy = s["z"].double(), s["dy"].double()
    inner = (dy * gain * z).sum(1, keepdim=True) / case["width"]
    dz = s["dz"].double() + r * dy * gain - r.pow(3) * z * inner
    return {"dx": dz if keep is None else dz * keep, "dresidual": dz, "dgain": (dy * z * r).sum(0)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"token": _exact_token, "pref": _exact_pref, "scan": _exact_scan,
            "norm": _exact_norm}[case["kind"]](case, s)
