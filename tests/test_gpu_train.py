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


# ------------------------------------------------------------------------------------------------------ what is not seen
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("bf16", 96), ("fp32", 64), ("bf16", 256)])
@pytest.mark.parametrize("which", ["q", "k", "v", "dout"])
@pytest.mark.parametrize("window,chunk,pinned", [(0, 1, 0), (150, 40, 20)])
def test_what_is_not_seen_reaches_no_row(window, chunk, pinned, which, dtype, D):
    """Infinities and NaN in one token, in the packed neighbours and behind the last sequence: rows that do not see them have the bits
    they had without, rows that do are not finite."""
    dt, lens, Hq, Hkv = TYPES[dtype], [330, 200], 4, 2
    pins = [pinned, min(pinned, 3)] if window else None
    (q, k, v, dout), go = _attention(lens, Hq, Hkv, D, dt, 3, window, chunk, pins, tail=60)
    clean = go()
    t = {"q": q, "k": k, "v": v, "dout": dout}[which]
    n = sum(lens)
    t[n:] = math.nan                                                 # nobody's rows
    at = 201                                                         # a token of the first sequence, inside a tile
    t[at, :, 1], t[at, :, 3], t[at, :, 4] = math.nan, math.inf, -math.inf
    got = go()
    seen = to.seen(lens[0], window, chunk, pins[0] if pins else 0, DEV)
    rows = torch.zeros(n + 60, dtype=torch.bool, device=DEV)         # rows whose output or gradient may depend on the token
    if which in ("q", "dout"):
        rows[at] = True
    else:
        rows[:lens[0]] = seen[:, at]
    toks = torch.zeros_like(rows)                                    # tokens that some such row sees
    toks[:lens[0]] = seen[rows[:lens[0]]].any(0)
    if which == "dout":
        out_rows = torch.zeros_like(rows)
    else:
        out_rows = rows
    for name, a, b, hit in (("out", clean[0], got[0], out_rows), ("lse", clean[1], got[1], out_rows if which != "v" else torch.zeros_like(rows)),
                            ("dq", clean[2], got[2], rows), ("dk", clean[3], got[3], toks), ("dv", clean[4], got[4], toks)):
        assert torch.equal(a[~hit], b[~hit]), name
        if name in ("out", "dq", "dk") and hit.any():
            assert (~torch.isfinite(b[hit].float())).flatten(1).any(1).all(), name
    if which == "dout":
        assert (~torch.isfinite(got[4][toks].float())).flatten(1).any(1).all()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp32", 64)])
def test_bad_bounds_are_left_alone(dtype, D):
    """Sequences whose bounds or pinned tokens are out of range are neither read nor written; the others are served."""
    dt = TYPES[dtype]
    (q, k, v, dout), go = _attention([100, 130, 70], 4, 2, D, dt, 5, 64, 8, [3, 5, 0], tail=9)
    ref = go()
    n = q.shape[0]

    def run(cu, pin, window=64):
        o, l = torch.full_like(ref[0], 3.0), torch.full_like(ref[1], 3.0)
        g = [torch.full_like(t, 3.0) for t in ref[2:]]
        ws = torch.empty(pt.seq_attn_workspace_bytes(n, 4), dtype=torch.uint8, device=DEV)
        cu, pin = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (cu, pin))
        pt.seq_attn(q, k, v, cu, o, lse_out=l, n_pinned=pin, window=window, evict_chunk=8)
        pt.seq_attn_backward(q, k, v, o, l, dout, cu, *g, ws, n_pinned=pin, window=window, evict_chunk=8)
        return [o, l, *g]

    for cu, pin, dead in (([0, 100, 230, 300], [3, 64, 0], (100, 230)), ([0, 100, 230, 300], [3, 5, -1], (230, 300)),
                          ([0, 100, 230, n + 5], [3, 5, 0], (230, n)), ([-4, 100, 230, 300], [3, 5, 0], (0, 100)),
                          ([0, 100, 230, 300], [1 << 30, 5, 0], (0, 100))):
        got = run(cu, pin)
        live = torch.ones(n, dtype=torch.bool, device=DEV)
        live[300:] = False
        live[dead[0]:dead[1]] = False
        for a, b in zip(ref, got):
            assert torch.equal(a[live], b[live]) and (b[~live] == 3.0).all()


def test_nothing_to_do():
    e = lambda *s, dt=torch.bfloat16: torch.empty(*s, dtype=dt, device=DEV)      # noqa: E731
    i32, f32 = torch.int32, torch.float32
    q, k = e(0, 4, 64), e(0, 2, 64)
    pt.seq_attn(q, k, k, torch.zeros(3, dtype=i32, device=DEV), q, lse_out=e(0, 4, dt=f32))
    pt.seq_attn_backward(q, k, k, q, e(0, 4, dt=f32), q, torch.zeros(1, dtype=i32, device=DEV), q, k, k, e(0, dt=f32))
    q, k = torch.full((5, 4, 64), 2.0, dtype=torch.bfloat16, device=DEV), torch.ones(5, 2, 64, dtype=torch.bfloat16, device=DEV)
    out = torch.full_like(q, 9.0)
    for cu in ([0], [0, 0, 0], [2, 2]):
        pt.seq_attn(q, k, k, torch.tensor(cu, dtype=i32, device=DEV), out)
    assert (out == 9.0).all()
    freq, w = torch.ones(32, device=DEV), torch.ones(64, dtype=torch.bfloat16, device=DEV)
    q0, k0 = e(0, 4, 64), e(0, 2, 64)
    pt.head_norm_rope(q0, k0, e(0, dt=i32), freq, q0, k0, q_weight=w, k_weight=w)
    dw = [torch.full((64,), 5.0, device=DEV) for _ in range(2)]
    pt.head_norm_rope_backward(q0, k0, q0, k0, e(0, dt=i32), freq, q0, k0, q_weight=w, k_weight=w, dq_weight=dw[0], dk_weight=dw[1],
                               workspace=e(pt.head_norm_rope_workspace_bytes(64), dt=torch.uint8))
    assert (dw[0] == 0).all() and (dw[1] == 0).all()
    loss, z = torch.full((1,), 5.0, device=DEV), e(0, 100)
    pt.policy_loss(z, e(0, dt=i32), e(0, dt=f32), e(0, dt=f32), e(0, dt=f32), loss, z)
    assert float(loss) == 0
    pt.token_logp(z, e(0, dt=i32), e(0, dt=f32))


# ------------------------------------------------------------------------------------------------------ as they are used
@pytest.mark.parametrize("dtype,D,W,E,pins", [("bf16", 128, 40, 10, (0, 13)), ("bf16", 64, 24, 1, (7, 0)), ("fp32", 64, 33, 5, (1, 20))])
def test_attention_of_a_rollout_is_what_its_decode_steps_computed(dtype, D, W, E, pins):
    """Tokens decoded one by one through the cache (prompt pinned, chunks evicted), and the same tokens all at once."""
    dt, Hq, Hkv, T = TYPES[dtype], 4, 2, 150
    gen = _gen(9)
    q, k, v = _fused(2 * T, (Hq, Hkv, Hkv), D, dt, gen)
    cache = pt.Cache(pt.make_config(n_layers=1, batch=2, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, window=W, evict_chunk=E, encode_enabled=0,
                                    dtype=dtype, n_global=8, rank=8))
    pin = torch.tensor(pins, dtype=torch.int32, device=DEV)
    both = lambda t, i: torch.stack([t[i[0]], t[T + i[1]]]).contiguous()       # noqa: E731
    pm = max(pins)
    kp, vp = (torch.stack([t[:pm], t[T:T + pm]]).contiguous() for t in (k, v))
    cache.prefill(0, kp, vp, pin, pm)
    out, lse = torch.empty(2 * T, Hq, D, dtype=dt, device=DEV), torch.empty(2 * T, Hq, device=DEV)
    cu = torch.tensor([0, T, 2 * T], dtype=torch.int32, device=DEV)
    pt.seq_attn(q, k, v, cu, out, lse_out=lse, n_pinned=pin, window=W, evict_chunk=E)
    o, s = torch.empty(2, Hq, D, dtype=dt, device=DEV), torch.empty(2, Hq, device=DEV)
    tol = 2.0 ** -7 * (1 + float(v.abs().max())) if dtype == "bf16" else 1e-5      # each side is off by 2^-8 (|out| + max |v|) at most
    for i in range(T - max(pins)):
        at = (pins[0] + i, pins[1] + i)
        cache.append_evict(0, both(k, at), both(v, at))
        cache.decode_attn(0, both(q, at), o, lse_out=s)
        for b in range(2):
            assert float((out[b * T + at[b]].float() - o[b].float()).abs().max()) <= tol
            assert float((lse[b * T + at[b]] - s[b]).abs().max()) <= 1e-4
    assert cache.status() == 0
    cache.close()


def _pass(P, x, cu, n, opt, own):
    """The update pass of a model of one layer: projections, norms and rotation, attention, logits, loss; gradients of everything."""
    dt = x.dtype
    Hq, Hkv, D = opt["heads"]
    V = P["wo"].shape[0]
    kw = dict(n_pinned=opt["pin"], window=opt["W"], evict_chunk=opt["E"])
    e = lambda *s, d=dt: torch.empty(*s, dtype=d, device=DEV)        # noqa: E731
    H = Hq + 2 * Hkv
    qkv = (x @ P["wqkv"].t()).view(n, H, D)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    qr, kr = e(n, Hq, D), e(n, Hkv, D)
    pt.head_norm_rope(q, k, opt["pos"], opt["freq"], qr, kr, q_weight=P["nq"], k_weight=P["nk"])
    o, lse = e(n, Hq, D), e(n, Hq, d=torch.float32)
    pt.seq_attn(qr, kr, v, cu, o, lse_out=lse, **kw)
    z = o.view(n, Hq * D) @ P["wo"].t()
    f = lambda: e(n, d=torch.float32)                                # noqa: E731
    logp, tl, loss = f(), f(), e(1, d=torch.float32)
    pt.policy_loss(z, opt["tok"], opt["adv"], logp, tl, loss, z, old_logp=opt["old"], ref_logp=opt["ref"], weight=opt["w"], kl_coef=0.05)
    do = (z @ P["wo"]).view(n, Hq, D)
    dqkv = e(n, H, D)
    dqr, dkr = e(n, Hq, D), e(n, Hkv, D)
    ws = e(pt.seq_attn_workspace_bytes(n, Hq), d=torch.uint8)
    pt.seq_attn_backward(qr, kr, v, o, lse, do, cu, dqr, dkr, dqkv[:, Hq + Hkv:], ws, **kw)
    dw = [e(D, d=torch.float32) for _ in range(2)]
    pt.head_norm_rope_backward(q, k, dqr, dkr, opt["pos"], opt["freq"], dqkv[:, :Hq], dqkv[:, Hq:Hq + Hkv], q_weight=P["nq"], k_weight=P["nk"],
                               dq_weight=dw[0], dk_weight=dw[1], workspace=e(pt.head_norm_rope_workspace_bytes(D), d=torch.uint8))
    flat = dqkv.view(n, H * D)
    return {"loss": loss, "logp": logp, "x": flat @ P["wqkv"], "wqkv": flat.t() @ x, "wo": z.t() @ o.view(n, Hq * D), "nq": dw[0], "nk": dw[1]}


def _pass_exact(P, x, lens, opt):
    P = {k: v.double().requires_grad_() for k, v in P.items()}
    x = x.double().requires_grad_()
    Hq, Hkv, D = opt["heads"]
    n = x.shape[0]
    qkv = (x @ P["wqkv"].t()).view(n, -1, D)
    q, _ = to.head_norm_rope(qkv[:, :Hq], P["nq"], opt["pos"], opt["freq"], 1e-6, False)
    k, _ = to.head_norm_rope(qkv[:, Hq:Hq + Hkv], P["nk"], opt["pos"], opt["freq"], 1e-6, False)
    v, outs, at = qkv[:, Hq + Hkv:], [], 0
    for b, m in enumerate(lens):
        r = slice(at, at + m)
        at += m
        s = torch.einsum("ihd,jhd->hij", q[r], k[r].repeat_interleave(Hq // Hkv, 1)) / math.sqrt(D)
        s = s.masked_fill(~to.seen(m, opt["W"], opt["E"], int(opt["pin"][b]), DEV), -math.inf)
        outs.append(torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v[r].repeat_interleave(Hq // Hkv, 1)))
    z = torch.cat(outs).reshape(n, Hq * D) @ P["wo"].t()
    lp = torch.log_softmax(z, -1).gather(1, opt["tok"].long()[:, None])[:, 0]
    ratio = torch.exp(lp - opt["old"].double())
    t = -torch.min(ratio * opt["adv"].double(), ratio.clamp(0.8, 1.2) * opt["adv"].double())
    over = opt["ref"].double() - lp
    t = t + 0.05 * (torch.exp(over) - over - 1)
    loss = (t * opt["w"].double()).sum()
    names = ["x", *P]
    grads = torch.autograd.grad(loss, [x, *P.values()])
    return {"loss": loss.detach().view(1), "logp": (lp * (opt["w"] != 0)).detach(), **dict(zip(names, grads))}


def _pass_case(dtype, D, seed=11):
    dt, gen = TYPES[dtype], _gen(seed)
    lens, Hq, Hkv, dm, V = [150, 1, 77, 260], 4, 2, 64, 500
    n = sum(lens)
    rnd = lambda *s, std=1.0: torch.randn(*s, device=DEV, generator=gen) * std      # noqa: E731
    P = {"wqkv": rnd((Hq + 2 * Hkv) * D, dm, std=dm ** -0.5).to(dt), "wo": rnd(V, Hq * D, std=0.1).to(dt), "nq": (1 + rnd(D, std=0.2)).to(dt),
         "nk": (1 + rnd(D, std=0.2)).to(dt)}
    x = rnd(n, dm).to(dt)
    cu = torch.tensor([0, 150, 151, 228, 488], dtype=torch.int32, device=DEV)
    opt = dict(heads=(Hq, Hkv, D), W=64, E=16, pin=torch.tensor([10, 0, 20, 3], dtype=torch.int32, device=DEV),
               pos=torch.cat([torch.arange(m) for m in lens]).int().to(DEV), freq=(10000.0 ** (-torch.arange(0, D, 2).double() / D)).float().to(DEV),
               tok=torch.randint(0, V, (n,), device=DEV, generator=gen, dtype=torch.int32), adv=rnd(n), w=torch.full((n,), 1.0 / n, device=DEV))
    opt["w"][:10] = 0                                                # prompt tokens
    zero = dict(opt, old=torch.zeros(n, device=DEV), ref=torch.zeros(n, device=DEV))
    lp = _pass_exact(P, x, lens, zero)["logp"].float()
    # ratios away from the border of the clip: what one rounding decides there is a whole row of the gradient
    opt["old"] = lp + torch.where(rnd(n) > 0, 0.05, 0.45) * torch.sign(rnd(n))
    opt["ref"] = lp + 0.3 * rnd(n)
    return P, x, cu, lens, opt


@pytest.mark.parametrize("dtype,D", [("fp32", 64), ("bf16", 128)])
def test_an_update_pass_has_the_gradients_of_the_whole(dtype, D):
    P, x, cu, lens, opt = _pass_case(dtype, D)
    torch.backends.cuda.matmul.allow_tf32 = False
    got = _pass(P, x, cu, x.shape[0], opt, True)
    ref = _pass_exact(P, x, lens, opt)
    # Relative in the 2-norm.  bf16: eleven tensors are rounded on the way (half a step of 2^-8 each, standard deviation 2^-8 / sqrt 3),
    # and the errors of logits of size ~ 2 enter exponentials: 2^-8 * sqrt(11 / 3) * 3 < 2.3e-2.  fp32: sums of up to 500 terms.
    tol = 2.3e-2 if dtype == "bf16" else 2e-5
    for name in ref:
        a, b = got[name].double().flatten(), ref[name].flatten()
        assert float((a - b).norm()) <= tol * float(b.norm()) + (1e-6 if name == "loss" else 0) + (2e-2 if name == "loss" and dtype == "bf16" else 0), (
            name, float((a - b).norm() / b.norm()))


def test_an_update_pass_captured_and_replayed_on_streams():
    """A captured pass replayed with other inputs in place, on a stream of its own, and two passes on two streams at once."""
    P, x, cu, lens, opt = _pass_case("bf16", 128)
    n = x.shape[0]
    x2 = torch.randn(n, 64, device=DEV, generator=_gen(5)).bfloat16()
    ref1, ref2 = _pass(P, x, cu, n, opt, True), _pass(P, x2, cu, n, opt, True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    buf = x.clone()
    with torch.cuda.stream(side):
        _pass(P, buf, cu, n, opt, True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        held = _pass(P, buf, cu, n, opt, True)
    for data, ref in ((x2, ref2), (x, ref1), (x2, ref2)):
        buf.copy_(data)
        graph.replay()
        torch.cuda.synchronize()
        for k in ref:
            assert torch.equal(held[k], ref[k]), k
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for s, data in ((side, x), (other, x2)):
            with torch.cuda.stream(s):
                got.append((_pass(P, data, cu, n, opt, True), ref1 if data is x else ref2))
    torch.cuda.synchronize()
    for g, r in got:
        assert all(torch.equal(g[k], r[k]) for k in r)


# ------------------------------------------------------------------------------------------------------ sizes
def test_packed_rows_past_32_bit_offsets():
    """Tensors of more than 2^31 elements: many short sequences, the last ones checked."""
    N, Hq, Hkv, D = 300_000, 64, 8, 128
    gen = _gen(1)
    q = torch.empty(N, Hq, D, dtype=torch.bfloat16, device=DEV)
    q.view(-1)[:1 << 20] = 1.0
    for i in range(0, N, 50_000):
        q[i:i + 50_000] = torch.randn(50_000, Hq, D, device=DEV, generator=gen, dtype=torch.bfloat16)
    k, v = (torch.randn(N, Hkv, D, device=DEV, generator=gen, dtype=torch.bfloat16) for _ in range(2))
    assert q.numel() > 2 ** 31
    lens = [100] * (N // 100)
    cu = torch.arange(0, N + 1, 100, dtype=torch.int32, device=DEV)
    pos, freq = torch.arange(N, device=DEV, dtype=torch.int32), (10000.0 ** (-torch.arange(0, D, 2).double() / D)).float().to(DEV)
    qr, kr = torch.empty_like(q), torch.empty_like(k)
    pt.head_norm_rope(q, k, pos, freq, qr, kr)
    tail = slice(N - 200, N)
    ref, b = to.head_norm_rope(q[tail], None, pos[tail], freq, 1e-6, False)
    _close(qr[tail], ref, b + to.half_step(torch.bfloat16) * ref.abs(), "rope")
    out, lse = torch.empty_like(q), torch.empty(N, Hq, device=DEV)
    pt.seq_attn(q, k, v, cu, out, lse_out=lse)
    dout = qr
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    ws = torch.empty(pt.seq_attn_workspace_bytes(N, Hq), dtype=torch.uint8, device=DEV)
    pt.seq_attn_backward(q, k, v, out, lse, dout, cu, dq, dk, dv, ws)
    for s in (slice(0, 200), tail):
        r = to.seq_attn(q[s], k[s], v[s], [100, 100], dout=dout[s], dtype=torch.bfloat16, tensor_cores=True)
        for name, t in zip(("out", "lse", "dq", "dk", "dv"), (out, lse, dq, dk, dv)):
            _close(t[s], r[name], r["b_" + name] + 2.0 ** -108, name)


def test_logits_past_32_bit_offsets():
    n, V = 16_500, 131_072 + 8
    z = torch.zeros(n, V, dtype=torch.bfloat16, device=DEV)
    assert z.numel() > 2 ** 31
    z[-3:] = torch.randn(3, V, device=DEV, generator=_gen(2)).bfloat16() * 3
    tok = torch.full((n,), 5, dtype=torch.int32, device=DEV)
    adv, logp = torch.ones(n, device=DEV), torch.empty(n, device=DEV)
    d = torch.empty_like(z)
    pt.policy_loss(z, tok, adv, logp, dlogits=d)
    ref = to.policy_loss(z[-3:], tok[-3:], adv[-3:])
    _check_loss(dict(logp=logp[-3:], dlogits=d[-3:]), ref, torch.bfloat16, V, 3, 0)
    assert float((logp[:-3] + math.log(V)).abs().max()) < 1e-5
