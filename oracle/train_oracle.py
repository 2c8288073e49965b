"""Float64 restatement of the training-pass operators: head norms with rotation, attention over packed sequences under the cache
policy, and the clipped policy loss.  Torch tensors in 64 bits on any device; shares no code with the library.

Each function also gives a bound on how far a result computed in fp32 and rounded to the storage type may be, elementwise, from
roundings counted one by one: `half` is the relative half step of the storage type (2^-8 bf16, 2^-24 fp32), U = 2^-24.
"""
import math

import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ------------------------------------------------------------------------------------------------ norms and rotation
def _rotate(y, positions, inv_freq, rot, interleaved, back=False):
    angle = positions.double()[:, None] * inv_freq.double()
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    if back:
        sin = -sin
    out = y.clone()
    idx = torch.arange(rot // 2, device=y.device)
    i, j = (2 * idx, 2 * idx + 1) if interleaved else (idx, idx + rot // 2)
    a, b = y[..., i], y[..., j]
    out[..., i], out[..., j] = a * cos - b * sin, b * cos + a * sin
    return out


def head_norm_rope(x, w, positions, inv_freq, eps, interleaved):
    """x [n, H, D] -> (y, bound).  fp32 work: the mean square ((D / 32 + 6) U relative, halved by the root), root, quotient and two
    products (5 U), a cosine or sine of an angle known to 2 pi U and itself to 2 U, two products and a sum: below
    (D / 64 + 24) U of |a| + |b|."""
    x = x.double()
    rot = 2 * len(inv_freq)
    y = x
    if w is not None:
        y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * w.double()
    out = _rotate(y, positions, inv_freq, rot, interleaved)
    size = y.abs().amax(-1, keepdim=True) * 2
    return out, (x.shape[-1] / 64 + 24) * U * size


def head_norm_rope_backward(x, w, g, positions, inv_freq, eps, interleaved):
    """(dx, bound of dx, dw, bound of dw).  The gradient turned back carries 16 U of |a| + |b|, the norm's factor (D / 64 + 6) U, the
    row's mean of w g n (D / 32 + 8) U of the sum of its magnitudes.  dw adds fewer than 2^13 terms a thread in fp32."""
    x, g = x.double(), g.double()
    rot, D = 2 * len(inv_freq), x.shape[-1]
    t = _rotate(g, positions, inv_freq, rot, interleaved, back=True)
    size = g.abs().amax(-1, keepdim=True) * 2
    if w is None:
        return t, 24 * U * size, None, None
    inv = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    n = x * inv
    wg = t * w.double()
    dx = inv * (wg - n * (wg * n).mean(-1, keepdim=True))
    wmax = w.double().abs().max()
    each = (D / 16 + 48) * U
    bound = each * inv * (size * wmax + n.abs() * (size * wmax * n.abs()).mean(-1, keepdim=True))
    dw = (t * n).sum((0, 1))
    terms = x.shape[0] * x.shape[1]
    return dx, bound, dw, (each + min(terms, 8192) * U) * (size * n.abs()).sum((0, 1))


# ------------------------------------------------------------------------------------------------ attention
def seen(n, window=0, chunk=1, pinned=0, device="cpu"):
    """[n, n] truth values, by running the cache: pinned tokens stay, the others are appended and leave a chunk at a time."""
    mask = torch.zeros(n, n, dtype=torch.bool)
    cap = window - pinned if window else n + 1
    e = min(chunk, cap)
    held = []
    for i in range(n):
        if i < pinned:
            mask[i, :i + 1] = True
            continue
        if len(held) == cap:
            held = held[e:]
        held.append(i)
        mask[i, :pinned] = True
        mask[i, held] = True
    return mask.to(device)


def seq_attn(q, k, v, lens, window=0, chunk=1, pinned=None, scale=None, dout=None, dtype=None, tensor_cores=False):
    """Packed sequences of the given lengths.  Returns a dict: out, lse, their bounds (b_out, b_lse), and with dout the gradients dq,
    dk, dv with theirs; n_dq, n_dk: standard deviations of the error that the rounded output brings into the backward pass.  The bounds: a score is off by E = (D + 4) U scale |q|.|k|, a weight by that, its row's largest E (through the
    maximum and the sum) and 8 U; with tensor cores, weights and score gradients are rounded to bf16 (2^-8)."""
    q, k, v = q.double(), k.double(), v.double()
    N, Hq, D = q.shape
    Hkv = k.shape[1]
    g = Hq // Hkv
    scale = 1 / math.sqrt(D) if scale is None else scale
    h = half_step(dtype) if dtype is not None else 0.0
    pr = 2.0 ** -8 if tensor_cores else 0.0
    r = {x: torch.zeros(N, Hq, D, dtype=torch.float64, device=q.device) for x in ("out", "b_out", "dq", "b_dq")}
    r |= {x: torch.zeros(N, Hkv, D, dtype=torch.float64, device=q.device) for x in ("dk", "b_dk", "dv", "b_dv", "n_dk")}
    r["n_dq"], r["n_out"], r["n_dv"] = torch.zeros_like(r["out"]), torch.zeros_like(r["out"]), torch.zeros_like(r["dv"])
    r |= {x: torch.zeros(N, Hq, dtype=torch.float64, device=q.device) for x in ("lse", "b_lse")}
    at = 0
    for b, n in enumerate(lens):
        rows = slice(at, at + n)
        at += n
        if n == 0:
            continue
        ok = seen(n, window, chunk, int(pinned[b]) if pinned is not None else 0, q.device)
        for hq in range(Hq):
            Q, K, V = q[rows, hq], k[rows, hq // g], v[rows, hq // g]
            s = (Q @ K.T * scale).masked_fill(~ok, -math.inf)
            lse = torch.logsumexp(s, -1, keepdim=True)
            p = torch.exp(s - lse)
            o = p @ V
            E = ((Q.abs() @ K.abs().T) * (scale * (D + 4) * U)).masked_fill(~ok, 0.0)
            top = E.amax(-1, keepdim=True)
            wp = p * (E + top + 8 * U + 2 * U * lse.abs())           # what fp32 makes of a weight
            r["out"][rows, hq], r["lse"][rows, hq] = o, lse[:, 0]
            r["b_out"][rows, hq] = (wp + p * (pr + top + n * U)) @ V.abs() + h * o.abs()
            r["b_lse"][rows, hq] = (top + (n + 8) * U)[:, 0] + 4 * U * (1 + lse.abs())[:, 0]
            if dout is None:
                continue
            do = dout[rows, hq].double()
            dp = do @ V.T
            dot = do.abs() @ V.abs().T
            delta = (do * o).sum(-1, keepdim=True)
            # delta is of the rounded output; it and dp are sums of D terms
            bd = (do.abs() * r["b_out"][rows, hq]).sum(-1, keepdim=True) + (D + 4) * U * (do.abs() * o.abs()).sum(-1, keepdim=True)
            ds = p * (dp - delta)
            bds = (wp + p * r["b_lse"][rows, hq][:, None]) * (dp - delta).abs() + p * (bd + (D + 4) * U * dot) + ds.abs() * (pr + 4 * U)
            dq, dk, dv = ds @ K * scale, ds.T @ Q * scale, p.T @ do
            # what the rounding of the output alone makes of delta, as independent errors: sigma per row, through the products
            sigma = h * (do * o).square().sum(-1, keepdim=True).sqrt()
            r["n_dq"][rows, hq] = scale * sigma * (p @ K).abs()
            r["n_dk"][rows, hq // g] += scale ** 2 * ((p * sigma).square().T @ Q.square())
            r["dq"][rows, hq] = dq
            r["b_dq"][rows, hq] = scale * ((bds + n * U * ds.abs()) @ K.abs()) + h * dq.abs()
            r["dk"][rows, hq // g] += dk
            r["b_dk"][rows, hq // g] += scale * ((bds + g * n * U * ds.abs()).T @ Q.abs())
            r["dv"][rows, hq // g] += dv
            r["b_dv"][rows, hq // g] += (wp + p * (r["b_lse"][rows, hq][:, None] + pr + g * n * U)).T @ do.abs()
    r["n_dk"] = r["n_dk"].sqrt()
    r["b_dk"] += h * r["dk"].abs()
    r["b_dv"] += h * r["dv"].abs()
    return r


# ------------------------------------------------------------------------------------------------ policy loss
def policy_loss(logits, tokens, advantage, old=None, ref=None, weight=None, temperature=1.0, clip_low=0.2, clip_high=0.2, kl_coef=0.0):
    """dict of logp, token_loss, token_kl, loss, dlogits."""
    n, V = logits.shape
    z = logits.double() / temperature
    on = (tokens >= 0) & (tokens < V)
    w = torch.ones(n, dtype=torch.float64, device=z.device) if weight is None else weight.double()
    on = on & (w != 0)
    y = tokens.long().clamp(0, V - 1)
    full = torch.log_softmax(z, -1)
    lp = full.gather(1, y[:, None])[:, 0]
    ratio = torch.ones_like(lp) if old is None else torch.exp(lp - old.double())
    adv = advantage.double()
    surr = torch.minimum(ratio * adv, ratio.clamp(1 - clip_low, 1 + clip_high) * adv)
    inside = ~(((adv > 0) & (ratio > 1 + clip_high)) | ((adv < 0) & (ratio < 1 - clip_low)))
    d = torch.where(inside, -ratio * adv, 0.0)
    kl = torch.zeros_like(lp)
    loss = -surr
    if ref is not None:
        over = ref.double() - lp
        kl = torch.exp(over) - over - 1
        loss = loss + kl_coef * kl
        d = d + kl_coef * (1 - torch.exp(over))
    zero = torch.zeros_like(lp)
    grad = -torch.exp(full)
    grad[torch.arange(n, device=z.device), y] += 1
    grad = grad * (w * d / temperature)[:, None]
    pick = lambda t: torch.where(on, t, zero)                        # noqa: E731
    return {"logp": pick(lp), "token_loss": pick(loss), "token_kl": pick(kl), "loss": (pick(loss) * torch.where(on, w, zero)).sum(),
            "dlogits": torch.where(on[:, None], grad, torch.zeros_like(grad))}
