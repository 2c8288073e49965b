"""The operators of a training pass at the edges of what their calls allow."""
import pytest
import torch

import paper_2602_16839_b200 as pt
from oracle import train_oracle as to

import test_gpu_train as whole

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _close(got, ref, bound, what):
    err = (got.double() - ref).abs()
    bad = ~(err <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(err[bad].max()), float((err / bound.clamp(min=1e-300)).nan_to_num(9e9).max()))


# ------------------------------------------------------------------------------------------------------ norms and rotation
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,Hq,Hkv,D,rot,inter", [
    (37, 28, 4, 128, 128, False), (16, 14, 2, 64, 64, False), (5, 16, 2, 128, 64, False), (129, 12, 12, 80, 40, True), (1, 1, 1, 8, 8, True),
    (300, 3, 1, 256, 256, False), (9, 2, 1, 72, 36, False), (2000, 12, 4, 128, 128, False)])
def test_norms_without_eps_whose_heads_do_not_fill_a_step(n, Hq, Hkv, D, rot, inter, dtype):
    """With eps = 0 a group of threads without a head holds zeros, whose norm has no inverse: that reaches no gradient."""
    dt, gen = TYPES[dtype], _gen(n + D)
    rnd = lambda *s: torch.randn(*s, device=DEV, generator=gen)      # noqa: E731
    q, k, gq, gk = (rnd(n, h, D).to(dt) for h in (Hq, Hkv, Hq, Hkv))
    wq, wk = ((1 + 0.3 * rnd(D)).to(dt) for _ in range(2))
    pos = torch.arange(n, device=DEV, dtype=torch.int32) * 7
    freq = (10000.0 ** (-torch.arange(0, rot, 2, device=DEV).double() / rot)).float()
    kw = dict(q_weight=wq, k_weight=wk, eps=0.0, interleaved=inter)
    qo, ko, dq, dk = (torch.empty_like(t) for t in (q, k, q, k))
    dwq, dwk = (torch.empty(D, device=DEV) for _ in range(2))
    ws = torch.empty(pt.head_norm_rope_workspace_bytes(D), dtype=torch.uint8, device=DEV)
    pt.head_norm_rope(q, k, pos, freq, qo, ko, **kw)
    pt.head_norm_rope_backward(q, k, gq, gk, pos, freq, dq, dk, dq_weight=dwq, dk_weight=dwk, workspace=ws, **kw)
    for x, w, y, g, dx, dw in ((q, wq, qo, gq, dq, dwq), (k, wk, ko, gk, dk, dwk)):
        ref, b = to.head_norm_rope(x, w, pos, freq, 0.0, inter)
        _close(y, ref, b + to.half_step(dt) * ref.abs(), "y")
        rx, bx, rw, bw = to.head_norm_rope_backward(x, w, g, pos, freq, 0.0, inter)
        _close(dx, rx, bx + to.half_step(dt) * rx.abs(), "dx")
        # bw allows for 8192 terms added one after another; here a thread adds fewer than 32, its CTA and the other CTAs fewer still
        terms = min(n * x.shape[1], 8192)
        each = (D / 16 + 48) * to.U
        _close(dw, rw, bw * (each + min(terms, 64) * to.U) / (each + terms * to.U) + to.U * rw.abs(), "dw")


# ------------------------------------------------------------------------------------------------------ attention
@pytest.mark.parametrize("D", [128, 64, 8])
@pytest.mark.parametrize("many", [False, True])
def test_non_finite_values_where_a_whole_chunk_leaves_inside_a_tile(many, D):
    """The rows of one tile on both sides of an eviction of 32700 tokens: a value that is no number reaches the rows that see it, in its
    column, and nothing else changes, however long those rows take to find it."""
    lens, Hq, Hkv, W = [33100, 700], 8, 2, 32700
    n, gen = sum(lens), _gen(D)
    q, k, v = (torch.randn(n, h, D, device=DEV, generator=gen).bfloat16() for h in (Hq, Hkv, Hkv))
    cu = torch.tensor([0, lens[0], n], dtype=torch.int32, device=DEV)

    def go():
        out, lse = torch.full((n, Hq, D), 3.0, dtype=torch.bfloat16, device=DEV), torch.full((n, Hq), 3.0, device=DEV)
        pt.seq_attn(q, k, v, cu, out, lse_out=lse, window=W, evict_chunk=W)
        return out, lse

    out, lse = go()
    assert out.isfinite().all() and lse.isfinite().all() and not (lse == 3.0).any()
    first = 100
    v[first:(W if many else first + 1), 0, 5] = float("nan")
    got, lse2 = go()
    assert torch.equal(lse, lse2)
    hit = torch.zeros(n, Hq, D, dtype=torch.bool, device=DEV)
    hit[first:W, :Hq // Hkv, 5] = True                               # rows first .. W - 1 hold what came since the start, the next are empty
    assert got[hit].isnan().all()
    assert torch.equal(got[~hit], out[~hit])


def test_a_chunk_of_two_million_tokens_that_leaves_between_the_halves_of_a_tile():
    """The rows behind the eviction wait while the rows before it go through two million keys."""
    W, Hq, D = 2_000_000, 1, 64                                      # W = 128 modulo 256: the rows of a work item from its second half on
    n, gen = W + 300, _gen(1)
    q, k = (torch.randn(n, Hq, D, device=DEV, generator=gen).bfloat16() for _ in range(2))
    v = torch.ones(n, Hq, D, dtype=torch.bfloat16, device=DEV)
    v[W:] = torch.randn(n - W, Hq, D, device=DEV, generator=gen).bfloat16()
    cu = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    out, lse = torch.full_like(q, 3.0), torch.full((n, Hq), -3.0, device=DEV)
    pt.seq_attn(q, k, v, cu, out, lse_out=lse, window=W, evict_chunk=W)
    # A row's weights add up to one: half a step of bf16 for each weight and for the result, a sum over fewer than 2^14 tiles in fp32.  The
    # other sum is the tensor cores' own, which add the products of 16 tokens at a time and need not round to nearest: each of the n / 16
    # additions is off by less than a whole step, 2^-23 of the sum.
    assert float((out[:W].float() - 1).abs().max()) <= 2 * 2.0 ** -8 + 2.0 ** 14 * to.U + n / 16 * 2.0 ** -23
    assert not (lse[:W] == -3.0).any() and lse.isfinite().all()
    r = to.seq_attn(q[W:], k[W:], v[W:], [n - W], dtype=torch.bfloat16, tensor_cores=True)
    _close(out[W:], r["out"], r["b_out"] + 2.0 ** -108, "out")
    _close(lse[W:], r["lse"], r["b_lse"], "lse")


@pytest.mark.parametrize("D", [128, 64])
def test_gradients_of_rollouts_that_follow_one_another_in_the_same_tensors(D):
    """Other rollouts, bounds and pinned prompts in the same tensors and the same workspace, call after call with nothing in between: the
    launch of the short items, which starts beside that of the long ones, reads this call's numbers."""
    n, Hq, Hkv, W, E, dt = 6000, 8, 2, 256, 64, torch.bfloat16
    kw = dict(window=W, evict_chunk=E)
    sets = []
    for seed, lens, pins in ((1, [2500, 3000, 400, 100], [200, 130, 0, 90]), (2, [300, 5000, 0, 700], [0, 255, 3, 129]),
                             (3, [1500, 1500, 1500, 1500], [128, 1, 250, 64])):
        gen = _gen(seed)
        q, k, v, g = (torch.randn(n, h, D, device=DEV, generator=gen).to(dt) for h in (Hq, Hkv, Hkv, Hq))
        cu = torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int32, device=DEV)
        pin = torch.tensor(pins, dtype=torch.int32, device=DEV)
        sets.append([q, k, v, g, cu, pin])
    bufs = [torch.empty_like(t) for t in sets[0]]
    ws = torch.empty(pt.seq_attn_workspace_bytes(n, Hq), dtype=torch.uint8, device=DEV)
    out, lse = torch.empty(n, Hq, D, dtype=dt, device=DEV), torch.empty(n, Hq, device=DEV)

    def go(q, k, v, g, cu, pin, work):
        grads = [torch.empty_like(t) for t in (q, k, v)]
        pt.seq_attn(q, k, v, cu, out, lse_out=lse, n_pinned=pin, **kw)
        pt.seq_attn_backward(q, k, v, out, lse, g, cu, *grads, work, n_pinned=pin, **kw)
        return grads

    alone = []
    for s in sets:
        alone.append(go(*s, torch.empty_like(ws)))
        torch.cuda.synchronize()
    got = []
    for i in range(30):
        for b, t in zip(bufs, sets[i % 3]):
            b.copy_(t)
        got.append(go(*bufs, ws))
    torch.cuda.synchronize()
    for i, grads in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(alone[i % 3], grads)), i


# ------------------------------------------------------------------------------------------------------ policy loss
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [500_009, 20_000_003, 1 << 28])
def test_rows_of_any_width_add_up(V, dtype):
    """Rows that no cluster holds, of weights that are all alike and of weights that are not: however many there are, their sum is as
    exact as that of a short row."""
    dt, gen = TYPES[dtype], _gen(V)
    z = torch.full((2, V), -0.359375, dtype=dt, device=DEV)          # a weight of 0.698: no sum of them is exact
    z[0, V // 3] = 0.0
    z[1] = torch.randn(V, device=DEV, generator=gen, dtype=dt)
    tok = torch.tensor([5, V - 2], dtype=torch.int32, device=DEV)
    adv, lp = torch.tensor([1.5, -0.7], device=DEV), torch.empty(2, device=DEV)
    only = torch.empty(2, device=DEV)
    pt.token_logp(z, tok, only)
    zd = z.double()
    lse = torch.logsumexp(zd, 1)
    ref = zd[torch.arange(2, device=DEV), tok.long()] - lse
    # Exponents (of the base 2) below 2^4 are off by their own rounding and the factor's, 2^-24 each: weights by 2^-19 log 2, exp2f by 2^-22,
    # a sum of at most 32 of them in fp32 by 2^-19; what the log-probability is rounded to comes beside that.
    rel = 2.0 ** -18
    _close(only, ref, rel + 4 * to.U * ref.abs(), "logp")
    pt.policy_loss(z, tok, adv, lp, dlogits=z)                       # in place
    assert torch.equal(lp, only)
    for i in range(2):
        g = zd[i].sub_(lse[i]).exp_().mul_(adv[i].double())          # -A (onehot - softmax)
        g[int(tok[i])] -= float(adv[i])
        bound = g.abs().mul_(2 * rel + to.half_step(dt)).add_(2.0 ** -126)
        assert (z[i].double().sub_(g).abs_() <= bound).all(), i


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_that_no_cluster_holds_of_masked_and_extreme_logits(dtype):
    whole.test_policy_loss_of_masked_and_extreme_logits(500_009, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("opt", [
    dict(temperature=0.8, clip_low=0.15, clip_high=0.3, kl_coef=0.1), dict(temperature=1.7, kl_coef=2.0), dict(clip_low=0.0, clip_high=0.05)])
@pytest.mark.parametrize("n,V", [(60, 1000), (30, 32000), (20, 152000), (12, 300001), (6, 700003)])
def test_every_entry_of_the_gradient_is_relatively_exact(n, V, opt, dtype):
    """Of the whole loss: old policy, reference, weights, masked tokens.  An entry is compared with its own size, however small a part of
    its row it is."""
    dt = TYPES[dtype]
    z, tok, kw = whole._loss_case(n, V, dt, 3 * n + V)
    lp, dz = torch.empty(n, device=DEV), torch.full_like(z, 5.0)
    pt.policy_loss(z, tok, **kw, logp=lp, dlogits=dz, **opt)
    ref = to.policy_loss(z, tok, kw["advantage"], kw["old_logp"], kw["ref_logp"], kw["weight"], **opt)
    on = (kw["weight"] != 0) & (tok >= 0) & (tok < V)
    assert (dz[~on] == 0).all() and on.sum() >= 2
    T = opt.get("temperature", 1.0)
    p = torch.softmax(z.double() / T, -1)
    rows, own = torch.arange(n, device=DEV)[on], tok[on].long()
    p[rows, own] = 1 - p[rows, own]
    # A weight's exponent (below 2^6 in the base 2) is off by three roundings of 2^-24, its power and the sum by less than 2^-18: 2^-16 with what
    # the entry is multiplied by.  The log-probability is off by less than 2^-17, and with it the ratio and the KL term's factor, each
    # relatively, before one is taken from the other.
    size = (kw["weight"].abs() / T).double() * (torch.exp(ref["logp"] - kw["old_logp"].double()) * kw["advantage"].double().abs()
                                                + opt.get("kl_coef", 0.0) * torch.exp(kw["ref_logp"].double() - ref["logp"]))
    g = ref["dlogits"]
    bound = (to.half_step(dt) + 2.0 ** -16) * g.abs() + 2.0 ** -17 * (size[:, None] * p) + 2.0 ** -126
    _close(dz[on], g[on], bound[on], "dlogits")
    top = g[on].abs().amax(-1, keepdim=True)
    some = top[:, 0] > 0                                             # not cut off by the clip
    few = (g[on][some].abs() < 2.0 ** -6 * top[some]).double().mean()
    assert some.any() and (V < 10000 or few > 0.9)                   # most entries are a small part of their row's largest
