"""The operators of a training pass over rollouts, as cases that can be timed and compared.

The rollouts that the cache decodes are learnt from by running every token once more, all at the same time: the norms of
queries and keys with the position rotation (`head_norm_rope`), attention over whole packed sequences, each token seeing what the
fixed-size cache let it see (`seq_attn`; without a window, a prompt's attention), and the clipped policy loss with its KL term,
from the logits to their gradient (`policy_loss`, `token_logp`).  `own` selects between the operators in their plain form
(elementary torch operations in 32 bits, 64 for angles and log-probabilities) and the calls a user makes of the library.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"

# Heads, KV heads and head sizes are those of the benchmark's workloads (3B, 7B and 8B shapes, the smallest fp32 one) and generic
# ones.  Queries, keys and values are slices of one projection's output, as a fused projection leaves them.


def listed():
    return [
        # one decode step of a small batch: latency counts; a model with norms of queries and keys
        {"name": "rope one step", "op": "rope", "N": 16, "Hq": 16, "Hkv": 2, "D": 128, "rot": 128, "norm": True, "pairs": "half",
         "far": 60000, "grad": False, "dtype": "bf16"},
        # prompts of a rollout batch, the 7B shape, no norms
        {"name": "rope prompts", "op": "rope", "N": 32768, "Hq": 28, "Hkv": 4, "D": 128, "rot": 128, "norm": False, "pairs": "half",
         "far": 32768, "grad": False, "dtype": "bf16"},
        # a micro-batch of training, the 8B shape with norms: forward and backward
        {"name": "rope training", "op": "rope", "N": 16384, "Hq": 32, "Hkv": 8, "D": 128, "rot": 128, "norm": True, "pairs": "half",
         "far": 8192, "grad": True, "dtype": "bf16"},
        # fp32, neighbouring pairs, a part of the head rotated, an odd number of tokens
        {"name": "rope odd fp32", "op": "rope", "N": 1023, "Hq": 12, "Hkv": 12, "D": 80, "rot": 40, "norm": True, "pairs": "next",
         "far": 100000, "grad": True, "dtype": "fp32"},
        # one short prompt of the 3B shape before its first step: latency
        {"name": "attention one prompt", "op": "attn", "lens": "one", "N": 300, "B": 1, "Hq": 16, "Hkv": 2, "D": 128, "W": 0, "E": 1,
         "prompt": 0, "grad": False, "dtype": "bf16"},
        # one long context, the 7B shape: arithmetic
        {"name": "attention long", "op": "attn", "lens": "one", "N": 16384, "B": 1, "Hq": 28, "Hkv": 4, "D": 128, "W": 0, "E": 1,
         "prompt": 0, "grad": False, "dtype": "bf16"},
        # a packed micro-batch of rollouts under the cache policy of the paper's runs (window, pinned prompts, a quarter leaving at
        # once): forward and backward, odd lengths
        {"name": "attention rollouts", "op": "attn", "lens": "ragged", "N": 24000, "B": 19, "Hq": 28, "Hkv": 4, "D": 128, "W": 1024,
         "E": 256, "prompt": 300, "grad": True, "dtype": "bf16"},
        # long sequences of the 8B shape under full attention: forward and backward
        {"name": "attention training", "op": "attn", "lens": "even", "N": 16384, "B": 2, "Hq": 32, "Hkv": 8, "D": 128, "W": 0, "E": 1,
         "prompt": 0, "grad": True, "dtype": "bf16"},
        # fp32, the smallest configuration's heads, sequences of all lengths
        {"name": "attention fp32", "op": "attn", "lens": "ragged", "N": 3001, "B": 9, "Hq": 4, "Hkv": 1, "D": 64, "W": 0, "E": 1,
         "prompt": 0, "grad": True, "dtype": "fp32"},
        # log-probabilities of one step's tokens: latency
        {"name": "logp one step", "op": "loss", "N": 16, "V": 32000, "grad": False, "kl": False, "masked": 0.0, "dtype": "fp32"},
        # a micro-batch over a large vocabulary, loss and gradient
        {"name": "policy batch", "op": "loss", "N": 4096, "V": 152000, "grad": True, "kl": True, "masked": 0.0, "dtype": "bf16"},
        # fp32 logits of an odd width (no row but the first is aligned), prompt tokens masked
        {"name": "policy odd fp32", "op": "loss", "N": 1001, "V": 65537, "grad": True, "kl": True, "masked": 0.3, "dtype": "fp32"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


HEADS = [(4, 1, 64), (14, 2, 64), (16, 2, 128), (28, 4, 128), (32, 8, 128), (12, 12, 64), (24, 8, 128), (10, 5, 96), (8, 1, 80)]


def draw(rng):
    op = rng.choice(["rope", "attn", "attn", "loss"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    grad = rng.random() < 0.5
    if op == "loss":
        V = _log(rng, 1000, 152000)
        N = max(1, min(_log(rng, 1, 16384), 4096 * 152000 // (V * (1 if dtype == "bf16" else 2))))
        return {"op": op, "N": N, "V": V, "grad": grad, "kl": rng.random() < 0.7, "masked": rng.choice([0.0, 0.2, 0.6]),
                "dtype": dtype}
    Hq, Hkv, D = rng.choice(HEADS)
    if op == "rope":
        N = max(1, min(_log(rng, 1, 32768), 16384 * 40 * 128 // ((Hq + Hkv) * D * (1 if dtype == "bf16" else 2))))
        return {"op": op, "N": N, "Hq": Hq, "Hkv": Hkv, "D": D, "rot": rng.choice([D, D, D // 2]), "norm": rng.random() < 0.6,
                "pairs": rng.choice(["half", "half", "next"]), "far": _log(rng, 100, 1000000), "grad": grad, "dtype": dtype}
    B = _log(rng, 1, 64)
    W = rng.choice([0, 0, _log(rng, 16, 4096)])
    c = {"op": op, "lens": rng.choice(["one", "even", "ragged", "ragged"]) if B > 1 else "one", "N": max(B, _log(rng, 1, 32768)),
         "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "W": W, "E": rng.choice([1, max(1, W // 4)]) if W else 1,
         "prompt": rng.choice([0, W // 4]), "grad": grad, "dtype": dtype}
    if c["lens"] == "one":
        c["B"] = 1
    # no more work than the largest listed case of the type
    most = 4.8e12 if dtype == "bf16" else 6e9
    while c["N"] > c["B"] and work(c)["flops"] > most:
        c["N"] = max(c["B"], c["N"] * 3 // 4)
    return c


# ------------------------------------------------------------------------------------------------------------ inputs
class State:
    pass


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lengths(case):
    """Lengths of the packed sequences: they follow from the case alone.  Ragged ones run from empty to many times the mean."""
    N, B = case["N"], case["B"]
    if case["lens"] == "one":
        return [N]
    if case["lens"] == "even":
        return [N // B + (1 if b < N % B else 0) for b in range(B)]
    rs = np.random.RandomState(N * 131 + B)
    share = rs.exponential(1.0, B)
    share[0] = 0.0                                                   # a sequence of no tokens
    if B > 2:
        share[1] = 1e-9                                              # and one of a token
    if share.sum() == 0:
        share[-1] = 1.0
    lens = np.floor(share / share.sum() * (N - min(B, 2))).astype(int)
    if B > 2:
        lens[1] = 1
    lens[-1] += N - lens.sum()
    return [int(x) for x in lens]


def _pinned(case):
    lens = _lengths(case)
    if not case["prompt"]:
        return [0] * len(lens)
    rs = np.random.RandomState(case["N"] * 7 + 1)
    return [int(x) for x in rs.randint(0, case["prompt"] + 1, len(lens))]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = State()
    s.case = case
    dt = _dtype(case)
    N = case["N"]
    if own:
        import paper_2602_16839_b200 as pt
        s.pt = pt
    if case["op"] == "loss":
        V = case["V"]
        s.logits = torch.empty(N, V, dtype=dt, device=DEV)
        s.tokens = torch.empty(N, dtype=torch.int32, device=DEV)
        lp = torch.empty(N, device=DEV)
        step = max(1, 60_000_000 // V)
        for i in range(0, N, step):                                 # tokens are sampled from the logits, as a rollout's are
            z = (torch.randn(min(step, N - i), V, device=DEV, generator=gen) * 2.5).to(dt)
            s.logits[i:i + step] = z
            z = z.float()
            u = torch.rand(z.shape, device=DEV, generator=gen).clamp_(1e-7, 1 - 1e-7)
            tok = (z - torch.log(-torch.log(u))).argmax(-1)
            s.tokens[i:i + step] = tok.int()
            lp[i:i + step] = z.gather(1, tok[:, None])[:, 0] - torch.logsumexp(z, -1)
        noise = torch.randn(3, N, device=DEV, generator=gen)
        s.old = lp + 0.15 * noise[0]                                # the policy that sampled them, some updates ago
        s.ref = lp + 0.3 * noise[1] if case["kl"] else None
        s.adv = noise[2]                                            # group-normalised rewards
        s.weight = torch.full((N,), 1.0 / N, device=DEV)
        if case["masked"]:
            s.weight[torch.rand(N, device=DEV, generator=gen) < case["masked"]] = 0.0
        if own:
            f = lambda: torch.empty(N, device=DEV)                  # noqa: E731
            s.logp, s.token_loss, s.loss = f(), f(), torch.empty(1, device=DEV)
            s.dlogits = torch.empty_like(s.logits) if case["grad"] else None
        return s
    Hq, Hkv, D = (case[k] for k in ("Hq", "Hkv", "D"))
    H = Hq + 2 * Hkv
    qkv = torch.randn(N, H, D, device=DEV, generator=gen)
    if case["op"] == "attn":
        qkv[:, :Hq] *= 2.0                                          # some tokens matter more than others
    qkv = qkv.to(dt)
    s.q, s.k, s.v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    if case["op"] == "rope":
        s.positions = torch.randint(0, case["far"], (N,), device=DEV, generator=gen, dtype=torch.int32)
        s.inv_freq = (10000.0 ** (-torch.arange(0, case["rot"], 2, device=DEV, dtype=torch.float64) / case["rot"])).float()
        s.wq = s.wk = None
        if case["norm"]:
            s.wq, s.wk = ((1 + 0.2 * torch.randn(D, device=DEV, generator=gen)).to(dt) for _ in range(2))
        if case["grad"]:
            s.gq = torch.randn(N, Hq, D, device=DEV, generator=gen).to(dt)
            s.gk = torch.randn(N, Hkv, D, device=DEV, generator=gen).to(dt)
        if own:
            s.q_out, s.k_out = (torch.empty(N, h, D, dtype=dt, device=DEV) for h in (Hq, Hkv))
            if case["grad"]:
                g = torch.empty(N, Hq + Hkv, D, dtype=dt, device=DEV)
                s.dq, s.dk = g[:, :Hq], g[:, Hq:]
                s.dwq = s.dwk = s.ws = None
                if case["norm"]:
                    s.dwq, s.dwk = torch.empty(D, device=DEV), torch.empty(D, device=DEV)
                    s.ws = torch.empty(s.pt.head_norm_rope_workspace_bytes(D), dtype=torch.uint8, device=DEV)
        return s
    s.cu = torch.tensor(np.concatenate([[0], np.cumsum(_lengths(case))]), dtype=torch.int32, device=DEV)
    s.pinned = torch.tensor(_pinned(case), dtype=torch.int32, device=DEV) if case["W"] else None
    if case["grad"]:
        s.g = torch.randn(N, Hq, D, device=DEV, generator=gen).to(dt)
    if own:
        s.out, s.lse = torch.empty(N, Hq, D, dtype=dt, device=DEV), torch.empty(N, Hq, device=DEV)
        if case["grad"]:
            g = torch.empty(N, H, D, dtype=dt, device=DEV)
            s.dq, s.dk, s.dv = g[:, :Hq], g[:, Hq:Hq + Hkv], g[:, Hq + Hkv:]
            s.ws = torch.empty(s.pt.seq_attn_workspace_bytes(N, Hq), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------------------ plain forms
def _turned(x, cos, sin, case, back=False):
    """Pairs of the first `rot` values of every head turned by their angles (backwards for gradients)."""
    rot = case["rot"]
    if back:
        sin = -sin
    a, rest = x[..., :rot], x[..., rot:]
    if case["pairs"] == "half":
        lo, hi = a[..., :rot // 2], a[..., rot // 2:]
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin, rest], -1)
    lo, hi = a[..., 0::2], a[..., 1::2]
    return torch.cat([torch.stack([lo * cos - hi * sin, hi * cos + lo * sin], -1).flatten(-2), rest], -1)


def _rope_plain(s):
    c = s.case
    angle = s.positions.double()[:, None] * s.inv_freq.double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    out = {}
    for name, x, w in (("q", s.q, s.wq), ("k", s.k, s.wk)):
        x = x.float()
        if c["norm"]:
            inv = (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
            y = x * inv * w.float()
        else:
            y = x
        out[name] = _turned(y, cos, sin, c).to(_dtype(c))
        if not c["grad"]:
            continue
        g = _turned((s.gq if name == "q" else s.gk).float(), cos, sin, c, back=True)
        if c["norm"]:
            n = x * inv
            out["dw" + name] = (g * n).flatten(0, 1).double().sum(0).float()
            g = g * w.float()
            g = inv * (g - n * (g * n).mean(-1, keepdim=True))
        out["d" + name] = g.to(_dtype(c))
    return out


def _seen(case, n, pinned):
    """[n, n] truth values: which tokens of a sequence each of its tokens sees."""
    i = torch.arange(n, device=DEV)
    ok = i[None, :] <= i[:, None]
    if case["W"]:
        cap = case["W"] - pinned
        e = min(case["E"], cap)
        gone = pinned + ((i - pinned + 1 - cap).clamp(min=0) + e - 1) // e * e
        ok = ok & ((i[None, :] < pinned) | (i[None, :] >= gone[:, None]))
    return ok


def _attn_plain(s):
    c = s.case
    Hq, Hkv, D = (c[k] for k in ("Hq", "Hkv", "D"))
    g, scale = Hq // Hkv, c["D"] ** -0.5
    dt = _dtype(c)
    N = c["N"]
    out = {"out": torch.empty(N, Hq, D, dtype=dt, device=DEV), "lse": torch.empty(N, Hq, device=DEV)}
    if c["grad"]:
        out.update(dq=torch.empty(N, Hq, D, dtype=dt, device=DEV), dk=torch.empty(N, Hkv, D, dtype=dt, device=DEV),
                   dv=torch.empty(N, Hkv, D, dtype=dt, device=DEV))
    at = 0
    for n, pinned in zip(_lengths(c), _pinned(c)):
        r = slice(at, at + n)
        at += n
        if n == 0:
            continue
        hide = ~_seen(c, n, pinned)
        for h in range(Hkv):
            hs = slice(h * g, (h + 1) * g)
            q, k, v = s.q[r, hs].float().transpose(0, 1), s.k[r, h].float(), s.v[r, h].float()
            x = (q @ k.T).mul_(scale).masked_fill_(hide, -math.inf)
            m = x.amax(-1, keepdim=True)
            p = x.sub_(m).exp_()
            z = p.sum(-1, keepdim=True)
            out["lse"][r, hs] = (m + torch.log(z))[..., 0].T
            p.div_(z)
            out["out"][r, hs] = (p @ v).transpose(0, 1).to(dt)
            if not c["grad"]:
                continue
            do = s.g[r, hs].float().transpose(0, 1)
            out["dv"][r, h] = (p.flatten(0, 1).T @ do.flatten(0, 1)).to(dt)
            dp = do @ v.T
            dp.sub_((p * dp).sum(-1, keepdim=True)).mul_(p).mul_(scale)
            out["dq"][r, hs] = (dp @ k).transpose(0, 1).to(dt)
            out["dk"][r, h] = (dp.flatten(0, 1).T @ q.flatten(0, 1)).to(dt)
    return out


CLIP_LOW, CLIP_HIGH, KL, TEMPERATURE = 0.2, 0.28, 0.04, 0.9


def _loss_plain(s):
    c = s.case
    N, V = c["N"], c["V"]
    logp, loss = torch.empty(N, device=DEV), torch.empty(N, device=DEV)
    out = {"logp": logp}
    if c["grad"]:
        out["dlogits"] = torch.empty(N, V, dtype=_dtype(c), device=DEV)
    step = max(1, 400_000_000 // V)
    for i in range(0, N, step):
        r = slice(i, i + step)
        z = s.logits[r].float() / TEMPERATURE
        tok = s.tokens[r].long()[:, None]
        m = z.amax(-1, keepdim=True)
        e = torch.exp(z - m)
        total = e.sum(-1, keepdim=True)
        lp = (z.gather(1, tok).double() - m.double() - torch.log(total.double()))[:, 0]
        logp[r] = lp.float()
        if not c["grad"]:
            continue
        w, adv = s.weight[r].double(), s.adv[r].double()
        ratio = torch.exp(lp - s.old[r].double())
        t = -torch.minimum(ratio * adv, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * adv)
        cut = ((adv > 0) & (ratio > 1 + CLIP_HIGH)) | ((adv < 0) & (ratio < 1 - CLIP_LOW))
        d = torch.where(cut, 0.0, -ratio * adv)
        if s.ref is not None:
            over = s.ref[r].double() - lp
            t = t + KL * (torch.exp(over) - over - 1)
            d = d + KL * (1 - torch.exp(over))
        on = w != 0
        logp[r] = torch.where(on, logp[r], 0.0)
        loss[r] = torch.where(on, t, 0.0).float()
        d = torch.where(on, w * d / TEMPERATURE, 0.0).float()[:, None]
        grad = e.div_(total).mul_(-d)
        grad.scatter_add_(1, tok, d)
        out["dlogits"][r] = grad.to(_dtype(c))
    if c["grad"]:
        out["token_loss"] = loss
        out["loss"] = (loss.double() * s.weight.double()).sum().float().reshape(1)
    return out


def run(s):
    c = s.case
    op = c["op"]
    if not own:
        return {"rope": _rope_plain, "attn": _attn_plain, "loss": _loss_plain}[op](s)
    pt = s.pt
    if op == "rope":
        inter = c["pairs"] == "next"
        pt.head_norm_rope(s.q, s.k, s.positions, s.inv_freq, s.q_out, s.k_out, q_weight=s.wq, k_weight=s.wk, interleaved=inter)
        out = {"q": s.q_out, "k": s.k_out}
        if c["grad"]:
            pt.head_norm_rope_backward(s.q, s.k, s.gq, s.gk, s.positions, s.inv_freq, s.dq, s.dk, q_weight=s.wq, k_weight=s.wk,
                                       dq_weight=s.dwq, dk_weight=s.dwk, workspace=s.ws, interleaved=inter)
            out.update(dq=s.dq, dk=s.dk)
            if c["norm"]:
                out.update(dwq=s.dwq, dwk=s.dwk)
        return out
    if op == "attn":
        pt.seq_attn(s.q, s.k, s.v, s.cu, s.out, lse_out=s.lse, n_pinned=s.pinned, window=c["W"], evict_chunk=c["E"])
        out = {"out": s.out, "lse": s.lse}
        if c["grad"]:
            pt.seq_attn_backward(s.q, s.k, s.v, s.out, s.lse, s.g, s.cu, s.dq, s.dk, s.dv, s.ws, n_pinned=s.pinned,
                                 window=c["W"], evict_chunk=c["E"])
            out.update(dq=s.dq, dk=s.dk, dv=s.dv)
        return out
    if not c["grad"]:
        pt.token_logp(s.logits, s.tokens, s.logp, temperature=TEMPERATURE)
        return {"logp": s.logp}
    pt.policy_loss(s.logits, s.tokens, s.adv, s.logp, s.token_loss, s.loss, s.dlogits, old_logp=s.old, ref_logp=s.ref,
                   weight=s.weight, temperature=TEMPERATURE, clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=KL)
    return {"logp": s.logp, "dlogits": s.dlogits, "token_loss": s.token_loss, "loss": s.loss}


# ------------------------------------------------------------------------------------------------------------ work
def _pairs(case):
    """Pairs of tokens that see one another, over all sequences."""
    total = 0
    for n, pinned in zip(_lengths(case), _pinned(case)):
        if not case["W"]:
            total += n * (n + 1) // 2
            continue
        cap = case["W"] - pinned
        e = min(case["E"], cap)
        i = np.arange(n)
        gone = (np.maximum(i - pinned + 1 - cap, 0) + e - 1) // e * e
        total += int((i + 1 - np.where(i >= pinned, gone, 0)).sum())
    return total


def work(case):
    elt = 2 if case["dtype"] == "bf16" else 4
    N = case["N"]
    if case["op"] == "loss":
        row = case["V"] * elt
        if not case["grad"]:
            return {"bytes": float(N) * (row + 8), "flops": float(N) * case["V"] * 4}
        on = 1.0 - case["masked"]                                    # masked rows are not read, their gradient is zero
        return {"bytes": float(N) * (row * (1 + on) + 32), "flops": float(N) * on * case["V"] * 8}
    Hq, Hkv, D = (case[k] for k in ("Hq", "Hkv", "D"))
    if case["op"] == "rope":
        rows = N * (Hq + Hkv) * D
        passes = 2 + (3 if case["grad"] and case["norm"] else 2 if case["grad"] else 0)
        return {"bytes": float(rows * elt * passes + N * 4), "flops": float(rows) * 4 * passes}
    rows = N * D * elt
    fwd = rows * (2 * Hq + 2 * Hkv) + N * Hq * 4
    flops = 4.0 * D * Hq * _pairs(case)
    if case["grad"]:
        return {"bytes": float(fwd + rows * (4 * Hq + 4 * Hkv) + N * Hq * 4), "flops": flops * 3.5}
    return {"bytes": float(fwd), "flops": flops}


# ------------------------------------------------------------------------------------------------------------ in 64 bits
def _exact_rope(s):
    """Each pair as a complex number times e^(i angle); gradients by automatic differentiation."""
    c = s.case
    rot, N = c["rot"], c["N"]
    phase = s.positions.double()[:, None] * s.inv_freq.double()
    turn = torch.polar(torch.ones_like(phase), phase)[:, None]
    out = {}
    for name, x, w in (("q", s.q, s.wq), ("k", s.k, s.wk)):
        x = x.double().detach().requires_grad_(c["grad"])
        leaves = [x]
        y = x
        if c["norm"]:
            w = w.double().detach().requires_grad_(c["grad"])
            leaves.append(w)
            y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["D"] + 1e-6) * w
        part = y[..., :rot].reshape(N, -1, rot // 2, 2) if c["pairs"] == "next" else torch.stack(y[..., :rot].chunk(2, -1), -1)
        z = torch.view_as_real(torch.view_as_complex(part.contiguous()) * turn)
        part = z.flatten(-2) if c["pairs"] == "next" else torch.cat([z[..., 0], z[..., 1]], -1)
        y = torch.cat([part, y[..., rot:]], -1)
        out[name] = y.detach()
        if c["grad"]:
            grads = torch.autograd.grad(y, leaves, (s.gq if name == "q" else s.gk).double())
            out["d" + name] = grads[0]
            if c["norm"]:
                out["dw" + name] = grads[1]
    keys = ["q", "k"] + (["dq", "dk"] if c["grad"] else []) + (["dwq", "dwk"] if c["grad"] and c["norm"] else [])
    return {k: out[k] for k in keys}


def _first_seen(case, n, pinned):
    """The oldest sliding token that each token sees, by running the cache: append, and drop a chunk when it is full."""
    first, held, oldest = [], 0, pinned
    cap = case["W"] - pinned if case["W"] else n + 1
    e = min(case["E"], cap)
    for i in range(n):
        if i < pinned:
            first.append(0)
            continue
        if held == cap:
            oldest, held = oldest + e, held - e
        held += 1
        first.append(oldest)
    return torch.tensor(first, dtype=torch.int64, device=DEV)


def _exact_attn(s):
    c = s.case
    Hq, Hkv, D, N = (c[k] for k in ("Hq", "Hkv", "D", "N"))
    out = {"out": torch.zeros(N, Hq, D, dtype=torch.float64, device=DEV), "lse": torch.zeros(N, Hq, dtype=torch.float64, device=DEV)}
    grads = {"dq": torch.zeros_like(out["out"]), "dk": torch.zeros(N, Hkv, D, dtype=torch.float64, device=DEV)}
    grads["dv"] = torch.zeros_like(grads["dk"])
    at = 0
    for n, pinned in zip(_lengths(c), _pinned(c)):
        r = slice(at, at + n)
        at += n
        if n == 0:
            continue
        col = torch.arange(n, device=DEV)
        first = _first_seen(c, n, pinned)
        step = max(1, 60_000_000 // n)
        for h in range(Hq):                                         # query heads one by one, blocks of rows
            k, v = s.k[r, h * Hkv // Hq].double(), s.v[r, h * Hkv // Hq].double()
            for lo in range(0, n, step):
                rows = torch.arange(lo, min(n, lo + step), device=DEV)
                q = s.q[r, h][rows].double() / math.sqrt(D)
                seen = (col <= rows[:, None]) & ((col >= first[rows][:, None]) | (col < pinned))
                logit = torch.where(seen, q @ k.T, -math.inf)
                lse = torch.logsumexp(logit, -1)
                p = torch.exp(logit - lse[:, None])
                o = p @ v
                out["lse"][at - n + rows, h] = lse
                out["out"][at - n + rows, h] = o
                if c["grad"]:
                    do = s.g[r, h][rows].double()
                    ds = p * (do @ v.T - (do * o).sum(-1, keepdim=True))
                    grads["dq"][at - n + rows, h] = ds @ k / math.sqrt(D)
                    grads["dk"][r, h * Hkv // Hq] += ds.T @ q
                    grads["dv"][r, h * Hkv // Hq] += p.T @ do
    if c["grad"]:
        out.update(grads)
    return out


def _exact_loss(s):
    c = s.case
    N, V = c["N"], c["V"]
    logp, loss = (torch.zeros(N, dtype=torch.float64, device=DEV) for _ in range(2))
    out = {"logp": logp}
    if c["grad"]:
        out["dlogits"] = torch.zeros(N, V, dtype=torch.float64, device=DEV)
    step = max(1, 100_000_000 // V)
    for i in range(0, N, step):
        r = torch.arange(i, min(N, i + step), device=DEV)
        z = s.logits[r].double().requires_grad_(c["grad"])
        lp = torch.log_softmax(z / TEMPERATURE, -1)[torch.arange(len(r), device=DEV), s.tokens[r].long()]
        logp[r] = lp.detach()
        if not c["grad"]:
            continue
        on = (s.weight[r] != 0).double()
        ratio, adv = torch.exp(lp - s.old[r].double()), s.adv[r].double()
        # the pessimistic branch, told apart by the side of the border the ratio is on
        high, low = ratio > 1 + CLIP_HIGH, ratio < 1 - CLIP_LOW
        t = -adv * torch.where((adv > 0) & high, 1 + CLIP_HIGH, torch.where((adv < 0) & low, 1 - CLIP_LOW, ratio))
        if s.ref is not None:
            t = t + KL * (torch.expm1(s.ref[r].double() - lp) - (s.ref[r].double() - lp))
        out["dlogits"][r] = torch.autograd.grad((t * s.weight[r].double()).sum(), z)[0]
        logp[r] *= on
        loss[r] = t.detach() * on
    if c["grad"]:
        out["token_loss"] = loss
        out["loss"] = (loss * s.weight.double()).sum().reshape(1)
    return out


def exact(case, seed):
    global own
    if case["op"] == "loss" and case["N"] * case["V"] > 700_000_000:
        return None
    mine, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = mine
    return {"rope": _exact_rope, "attn": _exact_attn, "loss": _exact_loss}[case["op"]](s)
