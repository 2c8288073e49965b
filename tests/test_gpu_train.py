"""The operators of a training pass on the GPU: head norms with rotation, attention over packed sequences, the policy loss."""
import math

import pytest
import torch

import paper_2602_16839_b200 as pt
from oracle import train_oracle as to

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _close(got, ref, bound, what):
    err = (got.double() - ref).abs()
    bad = ~(err <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(err[bad].max()), float((err / bound.clamp(min=1e-300)).nan_to_num(9e9).max()))


def _fused(n, heads, D, dt, gen, pad=0):
    """[n, h, D] slices of one wide row, as a fused projection leaves them."""
    whole = torch.randn(n, (sum(heads) * D) + pad, device=DEV, generator=gen).to(dt)
    out, at = [], 0
    for h in heads:
        out.append(whole[:, at:at + h * D].unflatten(1, (h, D)))
        at += h * D
    return out


# ------------------------------------------------------------------------------------------------------ norms and rotation
ROPE = [  # n, Hq, Hkv, D, rot, norm, interleaved
    (1, 16, 2, 128, 128, True, False), (16, 28, 4, 128, 128, False, False), (37, 14, 2, 64, 64, True, False),
    (5, 3, 1, 8, 8, True, True), (130, 12, 12, 80, 40, True, True), (3, 4, 4, 256, 64, True, False), (67, 4, 1, 96, 96, False, True),
    (9, 2, 1, 72, 36, True, False), (4, 5, 5, 40, 0, True, False), (1000, 32, 8, 128, 64, True, False), (33, 7, 1, 256, 256, True, True),
    (21, 6, 2, 24, 20, False, False),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,Hq,Hkv,D,rot,norm,inter", ROPE)
def test_head_norm_rope_and_its_gradients(n, Hq, Hkv, D, rot, norm, inter, dtype):
    dt, gen = TYPES[dtype], _gen(n + D)
    q, k = _fused(n, (Hq, Hkv), D, dt, gen, pad=16)
    pos = torch.randint(-5, 200000, (n,), device=DEV, generator=gen, dtype=torch.int32)
    freq = (10000.0 ** (-torch.arange(0, rot, 2, device=DEV).double() / max(rot, 1))).float()
    wq, wk = (((1 + 0.3 * torch.randn(D, device=DEV, generator=gen)).to(dt) if norm else None) for _ in range(2))
    if n == 37:
        wk = None                                                    # norms on one side only
    kw = dict(q_weight=wq, k_weight=wk, eps=1e-5, interleaved=inter)
    qo, ko = torch.full((n, Hq, D), 7.0, dtype=dt, device=DEV), torch.full((n, Hkv, D), 7.0, dtype=dt, device=DEV)
    pt.head_norm_rope(q, k, pos, freq, qo, ko, **kw)
    for x, w, y in ((q, wq, qo), (k, wk, ko)):
        ref, b = to.head_norm_rope(x, w, pos, freq, 1e-5, inter)
        _close(y, ref, b + to.half_step(dt) * ref.abs(), "y")
    gq, gk = _fused(n, (Hq, Hkv), D, dt, gen)
    dq, dk = _fused(n, (Hq, Hkv), D, dt, gen, pad=8)
    side = None if dk.shape[0] == 0 else dk[:, :, :].clone()
    dwq, dwk = (torch.full((D,), math.nan, device=DEV) if w is not None else None for w in (wq, wk))
    ws = torch.full((pt.head_norm_rope_workspace_bytes(D) // 4,), math.nan, device=DEV)
    pt.head_norm_rope_backward(q, k, gq, gk, pos, freq, dq, dk, dq_weight=dwq, dk_weight=dwk, workspace=ws, **kw)
    for x, w, g, dx, dw in ((q, wq, gq, dq, dwq), (k, wk, gk, dk, dwk)):
        rx, bx, rw, bw = to.head_norm_rope_backward(x, w, g, pos, freq, 1e-5, inter)
        _close(dx, rx, bx + to.half_step(dt) * rx.abs(), "dx")
        if w is not None:
            _close(dw, rw, bw + to.U * rw.abs(), "dw")
    # in place, and the same bits again
    q2, k2 = q.clone(), k.clone()
    pt.head_norm_rope(q2, k2, pos, freq, q2, k2, **kw)
    assert torch.equal(q2, qo) and torch.equal(k2, ko)
    hq, hk, first = gq.clone(), gk.clone(), [t.clone() for t in (dwq, dwk) if t is not None]
    pt.head_norm_rope_backward(q, k, hq, hk, pos, freq, hq, hk, dq_weight=dwq, dk_weight=dwk, workspace=ws, **kw)
    assert torch.equal(hq, dq) and torch.equal(hk, dk) and all(torch.equal(x, y) for x, y in zip(first, [t for t in (dwq, dwk) if t is not None]))


# ------------------------------------------------------------------------------------------------------ attention
def _attention(lens, Hq, Hkv, D, dt, seed, window=0, chunk=1, pinned=None, scale=None, grad=True, tail=0, size=1.5):
    gen = _gen(seed)
    N = sum(lens) + tail
    q, k, v = _fused(N, (Hq, Hkv, Hkv), D, dt, gen, pad=8)
    q *= size
    dout = torch.randn(N, Hq, D, device=DEV, generator=gen).to(dt)
    cu = torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int32, device=DEV)
    pin = None if pinned is None else torch.tensor(pinned, dtype=torch.int32, device=DEV)
    out, lse = torch.full((N, Hq, D), 3.0, dtype=dt, device=DEV), torch.full((N, Hq), 3.0, device=DEV)
    dq, dk, dv = (torch.full((N, h, D), 3.0, dtype=dt, device=DEV) for h in (Hq, Hkv, Hkv))
    ws = torch.full((pt.seq_attn_workspace_bytes(N, Hq) // 4,), math.nan, device=DEV)
    kw = dict(n_pinned=pin, window=window, evict_chunk=chunk, scale=scale)

    def go():
        pt.seq_attn(q, k, v, cu, out, lse_out=lse, **kw)
        if grad:
            pt.seq_attn_backward(q, k, v, out, lse, dout, cu, dq, dk, dv, ws, **kw)
        return [t.clone() for t in (out, lse, dq, dk, dv)]

    return (q, k, v, dout), go


def _check_attention(lens, Hq, Hkv, D, dtype, window=0, chunk=1, pinned=None, scale=None, grad=True, tail=0, seed=0, size=1.5):
    dt = TYPES[dtype]
    (q, k, v, dout), go = _attention(lens, Hq, Hkv, D, dt, seed, window, chunk, pinned, scale, grad, tail, size)
    got = go()
    assert all(torch.equal(x, y) for x, y in zip(got, go()))
    n = sum(lens)
    ref = to.seq_attn(q[:n], k[:n], v[:n], lens, window, chunk, pinned, scale, dout[:n] if grad else None, dt, dtype == "bf16")
    names = ["out", "lse"] + (["dq", "dk", "dv"] if grad else [])
    for name, t in zip(names, got):
        # half a step is relative only above 2^-126; weights below it may be zero: fewer than 2^10 of them, times less than 2^8
        _close(t[:n], ref[name], ref["b_" + name] + 2.0 ** -108, name)
        assert (t[n:] == 3.0).all(), name                            # rows of no sequence
        # A relative error has a meaning where the result is not itself a difference of roundings (a token that sees itself alone has a
        # weight of exactly one and a score gradient of exactly zero).
        if name != "lse" and n > 200 and ref[name].norm() > ref["b_" + name].norm():
            # roundings of either sign: the 2-norm is far inside the bound.  Two roundings of half a step each, of the weights or
            # score gradients and of the result, have a standard deviation of 2^-8 / sqrt(3) each, 0.82 * 2^-8 together.  The
            # backward pass takes dout . out from the rounded output: where few tokens are seen that sum's error is not small beside
            # the difference it goes into (out has the size of v then), hence the second term.
            off = float((t[:n].double() - ref[name]).norm())
            extra = float(ref["n_" + name].norm()) if grad else 0.0
            # fp32: a weight is off by the roundings of its score, of lse, of lse in base 2 and of their difference, each U of a number
            # of lse's size, and by some U of its own
            rel = 2.0 ** -8 if dtype == "bf16" else 4 * to.U * (16 + float(ref["lse"].abs().max()))
            assert off <= rel * float(ref[name].norm()) + extra, (name, off, float(ref[name].norm()), extra)


SHAPES = [(4, 1, 64), (14, 2, 64), (7, 1, 128), (4, 4, 128), (3, 1, 8), (2, 1, 96), (2, 2, 80), (2, 1, 256), (5, 5, 136)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("Hq,Hkv,D", SHAPES)
def test_attention_of_ragged_sequences(Hq, Hkv, D, dtype):
    _check_attention([0, 1, 65, 0, 127, 128, 129, 300, 2, 64, 0], Hq, Hkv, D, dtype, tail=70)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [1, 2, 31, 63, 64, 65, 127, 128, 129, 255, 256, 257, 383, 385, 640, 1000])
def test_attention_of_one_sequence(n, dtype):
    _check_attention([n], 2, 1, 128 if n % 2 else 64, dtype, seed=n)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("window,chunk,pinned", [
    (1, 1, 0), (2, 1, 1), (17, 1, 0), (64, 16, 0), (64, 64, 0), (100, 25, 37), (128, 1, 127), (200, 50, 128), (129, 129, 1), (300, 75, 130),
    (512, 1, 5), (1 << 30, 1 << 30, 64), (256, 3, 200)])
def test_attention_under_the_cache_policy(window, chunk, pinned, dtype):
    lens = [701, 0, 1, 130, 391]
    pins = [pinned, 0, pinned, min(pinned, 3), max(0, pinned - 1)]
    _check_attention(lens, 4, 2, 128 if window % 2 else 64, dtype, window, chunk, pins, tail=3, seed=window)
    if pinned == 0:
        _check_attention(lens[:3], 2, 1, 64, dtype, window, chunk, None, seed=window)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale,size", [(0.03, 1.0), (1.0, 1.0), (0.125, 30.0)])
def test_attention_of_other_scales_and_large_scores(scale, size, dtype):
    _check_attention([200, 77], 4, 2, 64, dtype, scale=scale, size=size)


# ------------------------------------------------------------------------------------------------------ policy loss
def _loss_case(n, V, dt, seed, mask=True, pad=0):
    gen = _gen(seed)
    z = (torch.randn(n, V + pad, device=DEV, generator=gen) * 3).to(dt)[:, :V]
    tok = torch.randint(0, V, (n,), device=DEV, generator=gen, dtype=torch.int32)
    lp = torch.log_softmax(z.float(), -1).gather(1, tok.long()[:, None])[:, 0]
    r = torch.randn(4, n, device=DEV, generator=gen)
    w = r[3].abs() / n
    if mask and n > 2:
        w[torch.rand(n, device=DEV, generator=gen) < 0.3] = 0
        tok[1] = -1
        tok[2] = V
    return z, tok, dict(advantage=r[0], old_logp=lp + 0.3 * r[1], ref_logp=lp + 0.5 * r[2], weight=w)


def _check_loss(got, ref, dt, V, n, scale, what=""):
    # a sum over V weights, each off by the rounding of its exponent (below 2^5, 2^-20) and its own; 64 bits from there
    rel = (math.sqrt(V) + 40) * to.U + 2.0 ** -20
    _close(got["logp"], ref["logp"], rel * (1 + ref["logp"].abs()), what + "logp")
    rows = {"token_loss": 1.0, "token_kl": 1.0}
    for k in rows:
        if got.get(k) is not None:
            _close(got[k], ref[k], 40 * rel * (1 + ref[k].abs()), what + k)
    if got.get("loss") is not None:
        _close(got["loss"][0], ref["loss"], 40 * rel * (1 + scale), what + "loss")
    if got.get("dlogits") is not None:
        g = ref["dlogits"]
        _close(got["dlogits"], g, (to.half_step(dt) + 40 * rel) * g.abs() + 40 * rel * g.abs().amax(-1, keepdim=True) * 2.0 ** -4 + 1e-37, what + "dlogits")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,V", [(1, 1), (1, 7), (5, 8), (3, 1000), (40, 4099), (7, 32000), (3, 65537), (2, 152000), (600, 130), (2, 300001)])
def test_policy_loss_and_its_gradient(n, V, dtype):
    dt = TYPES[dtype]
    z, tok, kw = _loss_case(n, V, dt, n + V, pad=3 if V % 2 else 0)
    f = lambda: torch.full((n,), math.nan, device=DEV)              # noqa: E731
    got = dict(logp=f(), token_loss=f(), token_kl=f(), loss=torch.full((1,), math.nan, device=DEV), dlogits=torch.full_like(z, math.nan))
    opt = dict(temperature=0.8, clip_low=0.15, clip_high=0.3, kl_coef=0.1)
    pt.policy_loss(z, tok, **kw, **got, **opt)
    ref = to.policy_loss(z, tok, kw["advantage"], kw["old_logp"], kw["ref_logp"], kw["weight"], **opt)
    _check_loss(got, ref, dt, V, n, float((ref["token_loss"].abs() * kw["weight"].double()).sum()))
    # in place: the gradient over the logits; and nothing but some of the outputs
    # (rows that lie alike with respect to 16 bytes are summed in the same order, others need not be)
    z2, z3, g2 = torch.empty_strided(z.shape, z.stride(), dtype=dt, device=DEV).copy_(z), z.clone(), got["dlogits"]
    pt.policy_loss(z2, tok, **kw, logp=f(), dlogits=z2, **opt)
    assert torch.equal(z2, g2) and torch.equal(z, z3)
    lp = f()
    pt.policy_loss(z3, tok, **kw, logp=lp, dlogits=z3, **opt)
    _check_loss(dict(logp=lp, dlogits=z3), ref, dt, V, n, 0)
    lp = f()
    pt.policy_loss(z, tok, **kw, logp=lp, **opt)
    assert torch.equal(lp, got["logp"])
    # no clipping, no reference: one update per rollout
    got = dict(logp=f(), token_loss=f(), dlogits=torch.empty_like(z))
    pt.policy_loss(z, tok, kw["advantage"], **got)
    _check_loss(got, to.policy_loss(z, tok, kw["advantage"]), dt, V, n, 0)
    lp = f()
    pt.token_logp(z, tok, lp, temperature=0.8)
    _check_loss(dict(logp=lp), to.policy_loss(z, tok, kw["advantage"], temperature=0.8), dt, V, n, 0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [37, 5003, 65536])
def test_policy_loss_of_masked_and_extreme_logits(V, dtype):
    """Logits of -inf have no probability, whole stretches of them included; far offsets do not matter; a row that is not a number is
    one, and no other row is."""
    dt, n = TYPES[dtype], 12
    z, tok, kw = _loss_case(n, V, dt, V, mask=False)
    z = z.contiguous()
    z[0, V // 3:] = -math.inf
    z[1, :V - 1] = -math.inf
    z[2] -= 20000
    z[3] += 20000
    z[4] = -3e38
    z[5, V // 2] = math.nan
    z[6] = -math.inf
    z[7, 5] = math.inf
    z[8] = math.nan
    tok[0], tok[1], tok[8] = 1, V - 1, -1
    kw["old_logp"] = torch.log_softmax(z.double(), -1).gather(1, tok.clamp(min=0).long()[:, None])[:, 0].float() + 0.1
    kw["ref_logp"] = kw["old_logp"] - 0.3
    f = lambda: torch.full((n,), 5.0, device=DEV)                   # noqa: E731
    got = dict(logp=f(), token_loss=f(), token_kl=f(), dlogits=torch.full_like(z, 5.0))
    pt.policy_loss(z, tok, **kw, **got, kl_coef=0.1)
    ref = to.policy_loss(z, tok, kw["advantage"], kw["old_logp"], kw["ref_logp"], kw["weight"], kl_coef=0.1)
    bad = torch.tensor([5, 6, 7], device=DEV)
    good = torch.tensor([i for i in range(n) if i not in (5, 6, 7)], device=DEV)
    for k in got:
        assert got[k][bad].isnan().reshape(3, -1).any(1).all(), k
    # offsets of 20000 leave 2^-9 (fp32) or 2^6 (bf16) of a logit: both sides read the same values, the exponents are off by 2^-24 of them
    slack = 20000 * 2.0 ** -22
    for k in ("logp", "token_loss", "token_kl"):
        _close(got[k][good], ref[k][good], slack * (1 + ref[k][good].abs()), k)
    g = ref["dlogits"][good]
    _close(got["dlogits"][good], g, (to.half_step(dt) + 4 * slack) * g.abs() + 4 * slack * g.abs().amax(-1, keepdim=True) + 1e-37, "dlogits")


def test_policy_loss_gradient_against_differences():
    n, V = 6, 1000
    z, tok, kw = _loss_case(n, V, torch.float32, 4, mask=False)
    out = lambda: dict(logp=torch.empty(n, device=DEV), token_loss=torch.empty(n, device=DEV), loss=torch.empty(1, device=DEV))   # noqa: E731
    d, o = torch.empty_like(z), out()
    pt.policy_loss(z, tok, **kw, **o, dlogits=d, kl_coef=0.1)
    for i in range(n):
        for x in (int(tok[i]), 17):
            h = 0.05
            side = []
            for s in (h, -h):
                z2, o2 = z.clone(), out()
                z2[i, x] += s
                pt.policy_loss(z2, tok, **kw, **o2, kl_coef=0.1)
                side.append(float(o2["token_loss"][i].double() * kw["weight"][i].double()))
            slope = (side[0] - side[1]) / (2 * h)
            # a central difference: h^2 / 6 of the third derivative, below 20 of the gradient's size, and the losses' roundings
            assert abs(slope - float(d[i, x])) <= h * h / 6 * 20 * float(d[i].abs().max()) + 2.0 ** -20 / h * float(kw["weight"][i]), (i, x)
