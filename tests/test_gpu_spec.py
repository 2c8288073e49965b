"""GPU parity of the speculative step: tree attention, draft verification and path commit against the float64 oracle.

Tolerances.  Outputs in bf16: the softmax weights and the output are rounded to 8 bits each, half a step at most, so an element
is off by 2^-8 (|o| + sum_j p_j |v_j|) <= 2^-8 (|o| + max|v|), plus what fp32 accumulation and the approximate exp2 add, below
1e-4 for scores of a few units.  fp32 storage, lse and states: the harness's bounds (1e-5; 1e-4 for lse over bf16 inputs, whose
fp32 dot products differ by up to D 2^-24 sum|q||k| from the exact ones; 1e-4 for unit-norm states).  Whole numbers are exact.
"""
import copy

import numpy as np
import pytest
import torch

import paper_2602_16839_b200 as pt
from oracle import spec_oracle as so

from _harness import TOL_LSE, TOL_STATE, Pair, np64

pytestmark = pytest.mark.gpu


def _close(got, want, dtype, vmax):
    tol = 1e-5 if dtype == "fp32" else 2.0 ** -8 * (np.abs(want) + vmax) + 1e-4
    err = np.abs(got - want)
    assert (err <= tol).all(), float((err - tol).max())


def _trees(rng, B, T, kind):
    par = np.full((B, T), -1, np.int32)
    for i in range(1, T):
        par[:, i] = {"chain": i - 1, "star": 0, "forest": -1}.get(kind, 0) if kind != "tree" else rng.integers(-1, i, B)
    return par


def _cuda(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a)).to(dtype).cuda()


def _fill(p, steps, rng=None):
    """Appends `steps` tokens on both sides without attention; with rng, each sequence stops at a length of its own."""
    stop = np.full(p.B, steps) if rng is None else rng.integers(0, steps + 1, p.B)
    for t in range(steps):
        k, v = p.gen.step_kv(t)
        act = (t < stop).astype(np.uint8)
        act_dev = _cuda(act, torch.uint8)
        p.cache.append_evict(-1, k, v, act_dev)
        p.cache.encode(-1)
        for l in range(p.L):
            p.orc.append_evict(l, np64(k[l]), np64(v[l]), act)
            p.orc.encode(l)


def _drafts(p, T, seed=0):
    g = p.gen.generic
    q = g(70 + seed, 0, (p.L, p.B, T, p.Hq, p.D), 1.0)
    k = g(80 + seed, 0, (p.L, p.B, T, p.Hkv, p.D), 1.0)
    v = g(90 + seed, 0, (p.L, p.B, T, p.Hkv, p.D), 1.0)
    return q, k, v


def _check_tree(p, T, parent, n_nodes=None, active=None, per_layer=False, drafts=None):
    q, k, v = _drafts(p, T) if drafts is None else drafts
    out = torch.full((p.L, p.B, T, p.Hq, p.D), 7.5, dtype=p.cache.torch_dtype, device="cuda")
    lse = torch.full((p.L, p.B, T, p.Hq), -3.25, device="cuda")
    before = p.cache.workspace.clone()
    kw = dict(n_nodes=None if n_nodes is None else _cuda(n_nodes), active=None if active is None else _cuda(active, torch.uint8))
    if per_layer:
        for l in range(p.L):
            p.cache.tree_attn(l, q[l], k[l], v[l], _cuda(parent), out[l], lse_out=lse[l], **kw)
    else:
        p.cache.tree_attn(-1, q, k, v, _cuda(parent), out, lse_out=lse, **kw)
    assert p.cache.status() == 0
    for r in (pt.binding.REGION_K, pt.binding.REGION_V, pt.binding.REGION_HEAD, pt.binding.REGION_COUNT,
              pt.binding.REGION_NAPP, pt.binding.REGION_STATE, pt.binding.REGION_TICKETS):
        at, n = p.cache.workspace_region(r)
        at -= p.cache.workspace.data_ptr()
        assert torch.equal(before[at:at + n], p.cache.workspace[at:at + n]), r
    on, ln = np64(out), np64(lse)
    for l in range(p.L):
        o, s, done = so.tree_attn(p.orc, l, np64(q[l]), np64(k[l]), np64(v[l]), parent, n_nodes, active)
        assert (on[l][~done] == 7.5).all() and (ln[l][~done] == -3.25).all()
        _close(on[l][done], o[done], p.dtype, 4.5)
        if done.any():
            assert np.abs(ln[l][done] - s[done]).max() <= TOL_LSE[p.dtype]
    return out, lse


# (storage, H_q, H_kv, D, W, E, T, prompt, tokens appended before, tree)
TREES = [
    ("bf16", 14, 2, 128, 37, 1, 9, 0, 60, "tree"),           # group of 7, ring wrapped, every arrival evicts
    ("bf16", 14, 2, 128, 300, 1, 13, 0, 170, "tree"),        # ring not full: nothing leaves
    ("bf16", 8, 2, 64, 130, 33, 16, 0, 128, "chain"),        # a chunk leaves in the middle of the chain
    ("bf16", 4, 4, 64, 257, 1, 64, 0, 300, "chain"),         # one head per KV head, the longest chain
    ("bf16", 32, 2, 128, 200, 50, 11, 40, 190, "tree"),      # group of 16, pinned prompts
    ("bf16", 16, 2, 128, 260, 1, 33, 0, 270, "tree"),        # several row tiles
    ("bf16", 16, 2, 128, 1, 1, 3, 0, 2, "chain"),            # a window of one token: a node sees itself alone
    ("bf16", 8, 2, 64, 5, 2, 12, 2, 9, "chain"),             # a chain longer than the ring: its own head leaves again
    ("bf16", 8, 1, 128, 64, 64, 7, 0, 64, "star"),           # a full ring that leaves at once for every node
    ("bf16", 7, 1, 128, 129, 1, 1, 0, 0, "chain"),           # an empty cache and one node
    ("bf16", 8, 2, 32, 50, 1, 6, 0, 70, "tree"),             # head size without a tensor-core kernel
    ("fp32", 4, 1, 64, 37, 1, 9, 0, 60, "tree"),
    ("fp32", 12, 3, 128, 200, 50, 20, 40, 190, "tree"),
    ("fp32", 4, 2, 256, 33, 4, 5, 0, 40, "forest"),
    ("fp32", 4, 4, 8, 33, 1, 64, 0, 40, "chain"),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,D,W,E,T,prompt,steps,kind", TREES)
def test_tree_attention_against_the_oracle(dtype, Hq, Hkv, D, W, E, T, prompt, steps, kind):
    rng = np.random.default_rng(W * 100 + T)
    p = Pair(pt, n_layers=2, batch=3, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, window=W, evict_chunk=E, dtype=dtype, seed=4)
    if prompt:
        p.prefill([prompt, 0, max(1, prompt // 3)], prompt)
    _fill(p, steps)
    parent = _trees(rng, 3, T, kind)
    a = _check_tree(p, T, parent)
    b = _check_tree(p, T, parent, per_layer=True)
    for x, y in zip(a, b):                                   # other splits of the work, other summation orders
        assert float((x.float() - y.float()).abs().max()) <= (1e-5 if dtype == "fp32" else 4.5 * 2.0 ** -7)
    p.close()


@pytest.mark.parametrize("dtype,Hq,Hkv,D,W,E,T,prompt,steps,kind", [
    ("bf16", 34, 2, 128, 150, 1, 9, 0, 160, "tree"),         # groups of 17: seven nodes to a row tile, rows left over
    ("bf16", 40, 1, 64, 40, 8, 7, 0, 45, "tree"),            # of 40: three nodes to a row tile
    ("bf16", 96, 2, 64, 130, 1, 6, 0, 140, "chain"),         # of 48: two
    ("bf16", 65, 1, 128, 40, 1, 3, 4, 50, "tree"),           # of 65: one, half the rows of a tile empty
    ("bf16", 100, 1, 128, 33, 1, 5, 0, 40, "star"),
    ("bf16", 128, 1, 128, 20, 1, 64, 0, 25, "tree"),         # of 128, the widest: 32 blocks of rows
    ("bf16", 128, 1, 64, 260, 60, 11, 9, 250, "tree"),
    ("bf16", 129, 1, 64, 20, 1, 3, 0, 25, "tree"),           # wider: the shape-generic kernel
    ("bf16", 8, 2, 96, 130, 1, 9, 0, 140, "tree"),           # head sizes that are no power of two
    ("bf16", 6, 3, 200, 70, 9, 6, 3, 75, "chain"),
    ("bf16", 4, 2, 256, 70, 1, 12, 0, 75, "tree"),
    ("fp32", 8, 2, 96, 130, 1, 9, 0, 140, "tree"),
    ("fp32", 3, 1, 136, 70, 9, 6, 3, 75, "forest"),
    ("fp32", 40, 1, 40, 40, 1, 7, 0, 45, "tree"),
])
def test_tree_attention_of_wide_groups_and_odd_head_sizes(dtype, Hq, Hkv, D, W, E, T, prompt, steps, kind):
    test_tree_attention_against_the_oracle(dtype, Hq, Hkv, D, W, E, T, prompt, steps, kind)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("fp32", 64)])
@pytest.mark.parametrize("E", [1, 24])
def test_tree_attention_ragged(dtype, D, E):
    """Sequences of all lengths, the empty one included, trees of all sizes from no node on, finished sequences."""
    rng = np.random.default_rng(E)
    p = Pair(pt, n_layers=1, batch=9, n_q_heads=14, n_kv_heads=2, head_dim=D, window=96, evict_chunk=E, dtype=dtype, seed=5)
    _fill(p, 130, rng)
    for T in (1, 17):
        n = rng.integers(0, T + 1, 9)
        n[:2] = [0, T]
        active = np.ones(9, np.uint8)
        active[[3, 6]] = 0
        _check_tree(p, T, _trees(rng, 9, T, "tree"), n, active)
    p.close()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp32", 64)])
def test_a_chain_equals_decode_steps(dtype, D):
    """GPU against GPU: node i of a chain is what decode_attn gives after i + 1 real appends."""
    p = Pair(pt, n_layers=2, batch=2, n_q_heads=8, n_kv_heads=2, head_dim=D, window=70, evict_chunk=3, dtype=dtype, seed=6)
    _fill(p, 69)
    T = 12
    q, k, v = _drafts(p, T)
    out = torch.empty(2, 2, T, 8, D, dtype=p.cache.torch_dtype, device="cuda")
    lse = torch.empty(2, 2, T, 8, device="cuda")
    p.cache.tree_attn(-1, q, k, v, _cuda(_trees(None, 2, T, "chain")), out, lse_out=lse)
    o1, l1 = torch.empty_like(out[:, :, 0]), torch.empty(2, 2, 8, device="cuda")
    for i in range(T):
        p.cache.append_evict(-1, k[:, :, i].contiguous(), v[:, :, i].contiguous())
        p.cache.decode_attn(-1, q[:, :, i].contiguous(), o1, None, l1)
        assert float((l1 - lse[:, :, i]).abs().max()) <= 2e-5
        assert float((o1.float() - out[:, :, i].float()).abs().max()) <= (1e-5 if dtype == "fp32" else 2 * 4.5 * 2.0 ** -8 * 2)
    p.close()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("bf16", 32), ("fp32", 64)])
def test_what_a_node_does_not_see_does_not_reach_it(dtype, D):
    """NaN and infinities in nodes off the path, in nodes past n_nodes, in slots that hold nothing, in tokens that have left for
    the deep nodes only, and in other sequences: the rows that do not see them are unchanged bit for bit."""
    W, T = 140, 8
    p = Pair(pt, n_layers=1, batch=3, n_q_heads=14, n_kv_heads=2, head_dim=D, window=W, evict_chunk=1, dtype=dtype, seed=7)
    act = _cuda([1, 1, 0], torch.uint8)
    for t in range(W):
        k, v = p.gen.step_kv(t)
        p.cache.append_evict(-1, k, v, act if t >= 100 else None)         # sequence 2: slots 100.. hold nothing
    q, k, v = _drafts(p, T)
    parent = np.tile(np.array([-1, 0, 1, 0, 3, 2, 5, 6], np.int32), (3, 1))  # 0-1-2-5-6-7 and 0-3-4
    n = np.array([8, 6, 8])

    def run(k, v):
        out = torch.zeros(1, 3, T, 14, D, dtype=p.cache.torch_dtype, device="cuda")
        lse = torch.zeros(1, 3, T, 14, device="cuda")
        p.cache.tree_attn(-1, q, k, v, _cuda(parent), out, n_nodes=_cuda(n), lse_out=lse)
        assert p.cache.status() == 0
        return out, lse

    base = run(k, v)
    assert torch.isfinite(base[0].float()).all() and torch.isfinite(base[1]).all()
    at, size = p.cache.workspace_region(pt.binding.REGION_K)
    base_ptr = p.cache.workspace.data_ptr()
    K = p.cache.workspace[at - base_ptr:at - base_ptr + size].view(p.cache.torch_dtype).view(1, 3, 2, W, D)
    at, size = p.cache.workspace_region(pt.binding.REGION_V)
    V = p.cache.workspace[at - base_ptr:at - base_ptr + size].view(p.cache.torch_dtype).view(1, 3, 2, W, D)

    def same(a, b, rows):
        for x, y in zip(a, b):
            assert torch.equal(x[:, rows[0]][:, rows[1]], y[:, rows[0]][:, rows[1]])

    for bad in (float("nan"), float("inf"), -float("inf")):
        # nodes past n_nodes (sequence 1: nodes 6, 7) and off the path (node 4 for the others)
        k2, v2 = k.clone(), v.clone()
        for t in (k2, v2):
            t[:, 1, 6:] = bad
            t[:, :, 4] = bad
        got = run(k2, v2)
        for b in range(3):
            same(base, got, (b, [i for i in range(n[b]) if i != 4]))
        assert not torch.isfinite(got[0][:, :, 4].float()).any()
        # empty slots of sequence 2
        keep = K.clone(), V.clone()
        K[:, 2, :, 100:], V[:, 2, :, 100:] = bad, bad
        got = run(k, v)
        same(base, got, (slice(None), slice(None)))
        K.copy_(keep[0]), V.copy_(keep[1])
        # the third-oldest token of the full ring of sequence 0 has left for nodes of depth 2 and more; the other sequences
        # never see it
        K[:, 0, :, 2], V[:, 0, :, 2] = bad, bad
        got = run(k, v)
        depth = np.array([0, 1, 2, 1, 2, 3, 4, 5])
        same(base, got, (0, [i for i in range(8) if depth[i] >= 2]))
        for b in (1, 2):
            same(base, got, (b, list(range(n[b]))))
        assert not torch.isfinite(got[0][:, 0, [0, 1, 3]].float()).any()
        K.copy_(keep[0]), V.copy_(keep[1])
    p.close()


@pytest.mark.parametrize("D,Hq,T,E", [(128, 8, 9, 1), (64, 8, 9, 40), (128, 32, 33, 1), (64, 32, 20, 1)])
def test_tree_attention_of_more_blocks_than_the_device_holds(D, Hq, T, E):
    """160 pairs of sequence and KV head: most are worked off whole, one after another, the last ones in parts.  Lengths, trees
    and finished sequences vary, and each call leaves the next one a fresh count of its work."""
    rng = np.random.default_rng(D + T)
    p = Pair(pt, n_layers=1, batch=40, n_q_heads=Hq, n_kv_heads=4, head_dim=D, window=150, evict_chunk=E, seed=14)
    _fill(p, 170, rng)
    parent = _trees(rng, 40, T, "tree")
    _check_tree(p, T, parent)
    n = rng.integers(0, T + 1, 40)
    active = (rng.random(40) < 0.8).astype(np.uint8)
    _check_tree(p, T, parent, n, active)
    _check_tree(p, T, parent, n)
    p.close()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("bf16", 16), ("fp32", 64)])
def test_scores_of_any_size(dtype, D):
    """Scores from -2e5 to 2e5 and more.  Products and sums are whole numbers below 2^24, and 1/sqrt(D) is a power of two for
    D = 16 and 64, so the scores are exact there.  For D = 128 the factor to base 2 is off by 2^-24 relative, which counts for a
    score's distance from the row's largest alone: 24 units at most where the weight is above 2^-24.  The row's reference may be
    off by half a step of 4e5, the same for all its weights."""
    W, T, n = 300, 9, 320
    p = Pair(pt, n_layers=1, batch=2, n_q_heads=8, n_kv_heads=2, head_dim=D, window=W, dtype=dtype, seed=15)
    rng = np.random.default_rng(D)

    def rows(*shape):                                        # large in one place; a last place that tells ties apart by units
        x = np.zeros(shape, np.float32)
        x[..., 0] = rng.integers(-255, 256, shape[:-1])
        x[..., 1] = rng.integers(-3, 4, shape[:-1])
        return x

    for t in range(n):
        k, v = rows(1, 2, 2, D), rng.standard_normal((1, 2, 2, D)).astype(np.float32)
        kt, vt = _cuda(k, p.cache.torch_dtype), _cuda(v, p.cache.torch_dtype)
        p.cache.append_evict(-1, kt, vt)
        p.orc.append_evict(0, np64(kt[0]), np64(vt[0]))
    q = rows(1, 2, T, 8, D)
    q[..., 0] *= 32                                          # 2^13 * 2^8 / sqrt(D): up to 2.6e5 at D = 64
    q = _cuda(q, p.cache.torch_dtype)
    k, v = _cuda(rows(1, 2, T, 2, D), p.cache.torch_dtype), _cuda(rng.standard_normal((1, 2, T, 2, D)), p.cache.torch_dtype)
    out, lse = torch.empty_like(q), torch.empty(1, 2, T, 8, device="cuda")
    parent = _trees(rng, 2, T, "tree")
    p.cache.tree_attn(-1, q, k, v, _cuda(parent), out, lse_out=lse)
    o, s, _ = so.tree_attn(p.orc, 0, np64(q[0]), np64(k[0]), np64(v[0]), parent)
    assert np.abs(s).max() > 5e4
    # the sum's logarithm joins a reference of up to 2.6e5 in natural units, held in fp32 in base 2 and scaled: three roundings
    assert (np.abs(np64(lse)[0] - s) <= 3 * 2.0 ** -23 * np.abs(s) + 1e-4).all()
    # fp32: exponents up to 24 that count, off by 2^-24 relative each for the factor, and exp2 itself
    _close(np64(out)[0], o, "bf16" if dtype == "bf16" else "fp32", 4.5)
    p.close()


@pytest.mark.parametrize("D,B", [(128, 40), (256, 24)])
def test_a_cache_whose_offsets_pass_32_bits(D, B):
    """5 to 6 GB of K and of V: the last sequence of a large batch gives what the same ring gives in a cache of its own, in
    attention and after a commit, and the first sequence's rows stay as they were."""
    Hkv, W, T = 8, 65536, 6
    kw = dict(n_layers=1, n_q_heads=8, n_kv_heads=Hkv, head_dim=D, window=W, n_global=8, rank=8, encode_enabled=0)
    big, small = pt.Cache(pt.make_config(batch=B, **kw)), pt.Cache(pt.make_config(batch=1, **kw))
    gen = torch.Generator(device="cuda").manual_seed(1)

    def word(c, region, dtype):
        at, n = c.workspace_region(region)
        at -= c.workspace.data_ptr()
        return c.workspace[at:at + n].view(dtype)

    for x, y in zip(_rings(big), _rings(small)):
        assert x.numel() > 2 ** 31
        y.normal_(generator=gen)
        x[0, 0].fill_(float("nan"))
        x[0, B - 1].copy_(y[0, 0])
    for c, b in ((big, B - 1), (small, 0)):
        word(c, pt.binding.REGION_COUNT, torch.int32)[b] = W
        word(c, pt.binding.REGION_HEAD, torch.int32)[b] = W - 3
        word(c, pt.binding.REGION_NAPP, torch.int64)[b] = 2 * W - 3
    q, k, v = (torch.randn(1, B, T, h, D, generator=gen, device="cuda").bfloat16() for h in (8, Hkv, Hkv))
    parent = torch.tensor([[-1, 0, 0, 1, 3, 2]] * B, dtype=torch.int32, device="cuda")
    act = torch.zeros(B, dtype=torch.uint8, device="cuda")
    act[B - 1] = 1
    a, b = torch.zeros_like(q), torch.zeros_like(q[:, :1])
    big.tree_attn(-1, q, k, v, parent, a, active=act)
    last = [t[:, B - 1:].contiguous() for t in (q, k, v)]
    small.tree_attn(-1, *last, parent[:1], b)
    assert (a[:, :B - 1] == 0).all()
    # weights of 65536 nearly equal tokens: outputs near 1 / 256, in other orders of summation
    assert float((a[:, B - 1:].float() - b.float()).abs().max()) <= 2.0 ** -8 * float(b.float().abs().max()) + 1e-4
    assert float(b.float().abs().max()) > 2e-3
    path = torch.tensor([[0, 1, 3, 4, -1, -1]] * B, dtype=torch.int32, device="cuda")
    n = torch.full((B,), 4, dtype=torch.int32, device="cuda")
    big.commit_path(-1, k, v, path, n, act)
    small.commit_path(-1, last[1], last[2], path[:1], n[:1])
    for x, y in zip(_rings(big), _rings(small)):
        assert torch.equal(x[0, B - 1], y[0, 0]) and bool(x[0, 0].isnan().all())
    assert big.status() == 0 and small.status() == 0
    big.close(), small.close()


@pytest.mark.parametrize("dtype,D,B", [("bf16", 128, 2), ("bf16", 64, 90), ("fp32", 64, 2)])
def test_tensors_at_the_least_alignment(dtype, D, B):
    """Every tensor 16 bytes (whole numbers 4) behind a 256-byte boundary: the same bits as aligned ones."""
    T = 6
    p = Pair(pt, n_layers=1, batch=B, n_q_heads=8, n_kv_heads=2, head_dim=D, window=70, dtype=dtype, seed=17)
    for t in range(75):
        k, v = p.gen.step_kv(t)
        p.cache.append_evict(-1, k, v)
    q, k, v = _drafts(p, T)
    parent, n = _cuda(_trees(np.random.default_rng(0), B, T, "tree")), torch.full((B,), T, dtype=torch.int32, device="cuda")

    def off(x, nbytes):
        room = torch.zeros(x.numel() * x.element_size() + 256 + nbytes, dtype=torch.uint8, device="cuda")
        start = -room.data_ptr() % 256 + nbytes
        y = room[start:start + x.numel() * x.element_size()].view(x.dtype).view(x.shape)
        y.copy_(x)
        assert y.data_ptr() % 256 == nbytes
        return y

    a, la = torch.zeros_like(q), torch.zeros(1, B, T, 8, device="cuda")
    b, lb = off(a, 16), off(la, 4)
    p.cache.tree_attn(-1, q, k, v, parent, a, n_nodes=n, lse_out=la)
    p.cache.tree_attn(-1, off(q, 16), off(k, 16), off(v, 16), off(parent, 4), b, n_nodes=off(n, 4), lse_out=lb)
    assert torch.equal(a, b) and torch.equal(la, lb) and float(a.abs().max()) > 0
    p.close()


def test_bad_trees_are_left_alone():
    """Parents out of order, counts out of range: that sequence is skipped and the status word says so; the others are served."""
    for D in (128, 32):
        p = Pair(pt, n_layers=1, batch=4, n_q_heads=8, n_kv_heads=2, head_dim=D, window=40, seed=8)
        _fill(p, 50)
        T = 6
        q, k, v = _drafts(p, T)
        parent = _trees(None, 4, T, "chain")
        good = torch.zeros(1, 4, T, 8, D, dtype=torch.bfloat16, device="cuda")
        p.cache.tree_attn(-1, q, k, v, _cuda(parent), good)
        assert p.cache.status() == 0
        parent[0, 3] = 3                                      # itself
        parent[1, 2] = -2
        n = np.array([T, T, T + 1, T])
        out = torch.full_like(good, 2.0)
        p.cache.tree_attn(-1, q, k, v, _cuda(parent), out, n_nodes=_cuda(n))
        assert p.cache.status() == 2
        assert (out[:, :3] == 2.0).all() and torch.equal(out[:, 3], good[:, 3])
        p.cache.reset()
        assert p.cache.status() == 0
        p.close()


def test_calls_that_the_cache_refuses():
    p = Pair(pt, n_layers=1, batch=2, n_q_heads=8, n_kv_heads=2, head_dim=64, window=40, seed=8)
    q, k, v = _drafts(p, 65)
    par = torch.zeros(2, 65, dtype=torch.int32, device="cuda")
    with pytest.raises(pt.PtencError) as e:
        p.cache.tree_attn(-1, q, k, v, par, torch.empty_like(q))
    assert e.value.code == pt.binding.PTENC_ESHAPE
    with pytest.raises(pt.PtencError) as e:
        p.cache.commit_path(-1, k, v, par, par[:, 0].contiguous())
    assert e.value.code == pt.binding.PTENC_ESHAPE
    with pytest.raises(pt.PtencError) as e:
        p.cache.tree_attn(1, q[0], k[0], v[0], par, torch.empty_like(q[0]))
    assert e.value.code == pt.binding.PTENC_EINVAL
    p.close()
    c = pt.Cache(pt.make_config(n_layers=1, batch=2, n_q_heads=8, n_kv_heads=2, head_dim=64, window=40, policy=1))
    q, k, v = q[:, :, :4].contiguous(), k[:, :, :4].contiguous(), v[:, :, :4].contiguous()
    par = par[:, :4].contiguous()
    with pytest.raises(pt.PtencError) as e:
        c.tree_attn(-1, q, k, v, par, torch.empty_like(q))
    assert e.value.code == pt.binding.PTENC_EINVAL
    with pytest.raises(pt.PtencError) as e:
        c.commit_path(-1, k, v, par, par[:, 0].contiguous())
    assert e.value.code == pt.binding.PTENC_EINVAL
    c.close()


# ------------------------------------------------------------------------------------------------------------ commit
COMMITS = [
    # storage, H_kv, D, W, E, T, prompt, steps, normalize, G, r
    ("bf16", 2, 128, 37, 1, 9, 0, 60, 0, 32, 32),
    ("bf16", 4, 64, 37, 1, 9, 12, 30, 0, 32, 32),
    ("bf16", 2, 64, 50, 1, 5, 0, 10, 0, 16, 16),            # not full: nothing leaves
    ("bf16", 2, 128, 64, 16, 12, 0, 70, 0, 32, 32),         # chunks
    ("bf16", 2, 64, 6, 2, 20, 1, 9, 0, 32, 32),             # several chunks per path, a path longer than the ring
    ("bf16", 1, 64, 1, 1, 4, 0, 3, 0, 8, 8),
    ("bf16", 2, 128, 33, 1, 64, 0, 33, 0, 40, 64),          # the longest path, more state rows than a warp
    ("bf16", 2, 64, 20, 1, 7, 0, 25, 1, 32, 32),            # Frobenius
    ("bf16", 2, 64, 20, 1, 7, 0, 25, 2, 32, 32),            # none
    ("bf16", 3, 24, 20, 1, 7, 0, 25, 0, 5, 12),             # odd state and row sizes
    ("bf16", 8, 128, 30, 1, 6, 0, 40, 0, 128, 128),         # the largest state
    ("fp32", 1, 64, 16, 1, 6, 0, 30, 0, 16, 16),
    ("fp32", 2, 32, 24, 7, 10, 3, 30, 1, 9, 5),
]


@pytest.mark.parametrize("dtype,Hkv,D,W,E,T,prompt,steps,norm,G,r", COMMITS)
def test_commit_against_the_oracle(dtype, Hkv, D, W, E, T, prompt, steps, norm, G, r):
    rng = np.random.default_rng(W + T)
    B = 5
    p = Pair(pt, n_layers=2, batch=B, n_q_heads=2 * Hkv, n_kv_heads=Hkv, head_dim=D, window=W, evict_chunk=E, dtype=dtype,
             seed=9, normalize_mode=norm, n_global=G, rank=r, kv_scale=0.5 if norm == 2 else 1.0)
    if prompt:
        p.prefill([prompt, 0, 1, prompt, 0], prompt)
    _fill(p, steps)
    for turn in range(4):
        _, k, v = _drafts(p, T, seed=turn)
        n = rng.integers(0, T + 1, B)
        n[0], n[1] = T, 0
        path = np.full((B, T), -1)
        for b in range(B):
            path[b, :n[b]] = np.sort(rng.choice(T, n[b], replace=False)) if turn != 2 else rng.integers(0, T, n[b])
        active = None
        if turn == 3:
            active = np.array([1, 1, 0, 1, 0], np.uint8)
        ev = torch.full((2, B), -9, dtype=torch.int32, device="cuda")
        if turn % 2:
            for l in range(2):
                p.cache.commit_path(l, k[l], v[l], _cuda(path), _cuda(n), None if active is None else _cuda(active, torch.uint8), ev[l])
        else:
            p.cache.commit_path(-1, k, v, _cuda(path), _cuda(n), None if active is None else _cuda(active, torch.uint8), ev)
        for l in range(2):
            gone = so.commit_path(p.orc, l, np64(k[l]), np64(v[l]), path, n, active)
            assert np.array_equal(ev[l].cpu().numpy(), gone)
        p.check_ring()
        p.check_state(rel=norm == 2)
        _check_rows(p)
    assert p.cache.status() == 0
    p.close()


@pytest.mark.parametrize("W,E,T,prompt,steps,G,r", [
    (20, 16, 20, 12, 40, 32, 32),                            # pinned prompts leave a ring shorter than the chunk: several events
    (64, 64, 64, 0, 70, 32, 32),                             # the whole ring leaves at once
    (300, 129, 40, 0, 290, 16, 64),                          # a chunk that fills no tile evenly
])
def test_commit_of_chunks_against_the_oracle(W, E, T, prompt, steps, G, r):
    test_commit_against_the_oracle("bf16", 2, 64, W, E, T, prompt, steps, 0, G, r)
    test_commit_against_the_oracle("bf16", 8, 128, W, E, T, prompt, steps, 0, G, r)


def _rings(c):
    base = c.workspace.data_ptr()
    f = c.cfg
    for r in (pt.binding.REGION_K, pt.binding.REGION_V):
        at, n = c.workspace_region(r)
        yield c.workspace[at - base:at - base + n].view(c.torch_dtype).view(f.n_layers, f.batch, f.n_kv_heads, f.window, f.head_dim)


def _check_rows(p):
    """Every live token's row, slot by slot."""
    for ring, name in zip(_rings(p.cache), "KV"):
        got = np64(ring)
        for l in range(p.L):
            for b in range(p.B):
                s = p.orc.seqs[l][b]
                sl = list(s.slot_of.values())
                assert np.array_equal(got[l, b][:, sl].transpose(1, 0, 2), getattr(s, name)[sl])


@pytest.mark.parametrize("dtype,E", [("bf16", 1), ("bf16", 9), ("fp32", 1)])
def test_commit_equals_appends_and_encodes(dtype, E):
    """GPU against GPU: the whole decode state after a commit is that after one append and encode per token, the staged rows
    of the last append included (a later ptenc_encode folds the same rows on both sides)."""
    kw = dict(n_layers=2, batch=4, n_q_heads=4, n_kv_heads=2, head_dim=64, window=30, evict_chunk=E, dtype=dtype, seed=10,
              n_global=32, rank=32)
    a, b = Pair(pt, **kw), Pair(pt, **kw)
    for x in (a, b):
        _fill(x, 28)
    rng = np.random.default_rng(1)
    for turn in range(6):
        T = 7
        _, k, v = _drafts(a, T, seed=turn)
        n = rng.integers(1, T + 1, 4)
        path = np.tile(np.arange(T), (4, 1))
        a.cache.commit_path(-1, k, v, _cuda(path), _cuda(n))
        staged = torch.zeros(4, dtype=torch.int64)
        for j in range(T):
            act = _cuda(j < n, torch.uint8)
            b.cache.append_evict(-1, k[:, :, j].contiguous(), v[:, :, j].contiguous(), act)
            b.cache.encode(-1)
        for x, y in zip(_rings(a.cache), _rings(b.cache)):
            assert torch.equal(x, y)
        for l in range(2):
            for x, y in zip(a.cache.get_ring(l), b.cache.get_ring(l)):
                assert torch.equal(x, y)
            assert float((a.cache.get_state(l) - b.cache.get_state(l)).abs().max()) <= 2 * TOL_STATE
    # one more token on every sequence, committed on one side and appended on the other: the staged rows are the same
    _, k, v = _drafts(a, 1, seed=9)
    a.cache.commit_path(-1, k, v, _cuda(np.zeros((4, 1))), _cuda(np.ones(4)))
    b.cache.append_evict(-1, k[:, :, 0].contiguous(), v[:, :, 0].contiguous())
    b.cache.encode(-1)
    for x in (a, b):
        x.cache.encode(-1)
    for l in range(2):
        assert float((a.cache.get_state(l) - b.cache.get_state(l)).abs().max()) <= 2 * TOL_STATE
    for x in (a, b):
        x.close()


def _staging(c):
    """The staging area where the header's workspace layout puts it: evicted K and V rows [L, B, E, H_kv D], their number and the
    first one's token index [L, B]; it ends where the states begin."""
    f, ws = c.cfg, c.workspace
    at, n = c.workspace_region(pt.binding.REGION_NPINNED)
    off, views = at - ws.data_ptr() + n, []
    dims = (f.n_layers, f.batch)
    for shape, dtype in (((*dims, f.evict_chunk, f.n_kv_heads * f.head_dim), c.torch_dtype),) * 2 + ((dims, torch.int32), (dims, torch.int64)):
        off = (off + 1023) // 1024 * 1024
        size = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
        views.append(ws[off:off + size].view(dtype).view(shape))
        off += size
    assert (off + 1023) // 1024 * 1024 == c.workspace_region(pt.binding.REGION_STATE)[0] - ws.data_ptr()
    return views


@pytest.mark.parametrize("dtype,E,B,norm", [("bf16", 1, 5, 0), ("bf16", 5, 5, 0), ("bf16", 16, 5, 0), ("bf16", 16, 4, 2), ("bf16", 29, 5, 0),
                                            ("bf16", 29, 1, 0), ("bf16", 16, 5, 1), ("fp32", 1, 5, 0), ("fp32", 29, 5, 0)])
def test_what_a_commit_leaves_staged(dtype, E, B, norm):
    """Staged rows, their number and their first token after every commit, bit for bit what appending the same tokens one by one
    leaves: the last arrival evicts in some sequences and not in others, and some evict in the middle of their path only."""
    kw = dict(n_layers=2, batch=B, n_q_heads=4, n_kv_heads=2, head_dim=64, window=30, evict_chunk=E, dtype=dtype, seed=20,
              n_global=32, rank=32, normalize_mode=norm)
    a, b = Pair(pt, **kw), Pair(pt, **kw)
    for x in (a, b):
        _fill(x, 34, np.random.default_rng(2))
    rng = np.random.default_rng(E)
    T, seen = 9, set()
    for turn in range(12):
        _, k, v = _drafts(a, T, seed=turn)
        n = rng.integers(0, T + 1, B)
        path = np.tile(np.arange(T), (B, 1))
        a.cache.commit_path(-1, k, v, _cuda(path), _cuda(n))
        want = None
        for j in range(T):
            act = j < n
            b.cache.append_evict(-1, k[:, :, j].contiguous(), v[:, :, j].contiguous(), _cuda(act, torch.uint8))
            b.cache.encode(-1)
            now = [t.clone() for t in _staging(b.cache)]
            if want is None:
                want = now
            else:                                             # a sequence keeps what its own last arrival left
                for w, x in zip(want, now):
                    w[:, torch.as_tensor(act)] = x[:, torch.as_tensor(act)]
        got = _staging(a.cache)
        assert torch.equal(got[2], want[2]) and torch.equal(got[3], want[3])
        for l in range(2):
            for s in range(B):
                m = int(want[2][l, s])
                seen.add((m > 0, int(n[s]) > 0))
                assert torch.equal(got[0][l, s, :m], want[0][l, s, :m]) and torch.equal(got[1][l, s, :m], want[1][l, s, :m])
            for x, y in zip(a.cache.get_ring(l), b.cache.get_ring(l)):
                assert torch.equal(x, y)
            assert float((a.cache.get_state(l) - b.cache.get_state(l)).abs().max()) <= (2 * TOL_STATE if norm != 2 else 2 * TOL_STATE * max(1.0, float(b.cache.get_state(l).abs().max())))
    assert B == 1 or seen >= {(True, True), (False, True), (False, False)}
    assert a.cache.status() == 0 and b.cache.status() == 0
    for x in (a, b):
        x.close()


def _fill_rings(c, gen):
    """Full rings of random rows, the words of which say that the window's tokens came in order."""
    f, ws = c.cfg, c.workspace
    for region in (pt.binding.REGION_K, pt.binding.REGION_V):
        at, n = c.workspace_region(region)
        flat = ws[at - ws.data_ptr():at - ws.data_ptr() + n].view(c.torch_dtype)
        for lo in range(0, flat.numel(), 1 << 30):
            flat[lo:lo + (1 << 30)].normal_(generator=gen)
    for region, dtype in ((pt.binding.REGION_COUNT, torch.int32), (pt.binding.REGION_NAPP, torch.int64)):
        at, n = c.workspace_region(region)
        ws[at - ws.data_ptr():at - ws.data_ptr() + n].view(dtype).fill_(f.window)


def _commit_takes_the_whole_window(c, k, v, append=False):
    """One token more than a full window of evict_chunk == window holds: everything leaves, oldest first, and is staged."""
    f, b1 = c.cfg, dict(dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(5)
    _fill_rings(c, gen)
    rows = torch.cat([torch.arange(0, f.window, max(1, f.window // 97)), torch.arange(f.window - 3, f.window)])
    rings = [r[0, 0][:, rows].clone() for r in _rings(c)]      # [Hkv, rows, D]
    evicted = torch.zeros(1, 1, **b1)
    if append:
        c.append_evict(-1, k[:, :, 0], v[:, :, 0], n_evicted_out=evicted)
    else:
        c.commit_path(-1, k, v, torch.zeros(1, 1, **b1), torch.ones(1, **b1), n_evicted_out=evicted)
    assert evicted.tolist() == [[f.window]] and c.status() == 0
    staged = _staging(c)
    assert int(staged[2]) == f.window and int(staged[3]) == 0
    for ring, stage in zip(rings, staged):
        assert torch.equal(ring.transpose(0, 1).reshape(len(rows), -1), stage[0, 0, rows])
    head, count, n_app = c.get_ring(0)
    assert count.tolist() == [1] and n_app.tolist() == [f.window + 1]
    for r, x in zip(_rings(c), (k, v)):
        assert torch.equal(r[0, 0, :, int(head)], x[0, 0, 0])


def test_commit_of_a_chunk_of_a_million_tokens():
    """evict_chunk 1048577: more groups of sixteen rows than a grid has places in its second direction.  The state after it is
    that of encoding the rows that were staged."""
    W, D, r = (1 << 20) + 1, 64, 16
    gen = torch.Generator(device="cuda").manual_seed(6)
    c = pt.Cache(pt.make_config(n_layers=1, batch=1, n_q_heads=1, n_kv_heads=1, head_dim=D, window=W, evict_chunk=W, n_global=16, rank=r))
    bf = lambda *shape: torch.randn(*shape, generator=gen, device="cuda").to(torch.bfloat16)
    c.set_encoder(0, bf(r, D), bf(r, D), bf(r, D), bf(16, D), bf(16, D), bf(16, D))
    before = c.get_state(0).clone()
    _commit_takes_the_whole_window(c, bf(1, 1, 1, 1, D), bf(1, 1, 1, 1, D))
    after = c.get_state(0).clone()
    at, n = c.workspace_region(pt.binding.REGION_STATE)
    c.workspace[at - c.workspace.data_ptr():at - c.workspace.data_ptr() + n].view(torch.float32).view(before.shape).copy_(before)
    c.encode(-1)                                               # the rows that the commit left staged
    assert float((c.get_state(0) - after).abs().max()) <= 2 * TOL_STATE and not torch.equal(before, after)
    c.close()


@pytest.mark.parametrize("dtype,E,D", [("fp32", 65536, 8), ("fp32", 65537, 8), ("bf16", 131079, 8), ("bf16", 65551, 64)])
def test_chunks_of_more_rows_than_are_counted_together(dtype, E, D):
    """Evicted rows are copied 65536 at a time: chunks of one block, one row more, and three; by an append alike."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    for append in (False, True):
        c = pt.Cache(pt.make_config(n_layers=1, batch=1, n_q_heads=2, n_kv_heads=2, head_dim=D, window=E, evict_chunk=E, dtype=dtype,
                                    encode_enabled=0))
        k, v = (torch.randn(1, 1, 1, 2, D, generator=gen, device="cuda").to(c.torch_dtype) for _ in range(2))
        _commit_takes_the_whole_window(c, k, v, append)
        c.close()


def test_commit_of_a_chunk_of_32_gigabytes():
    """2^31 vectors of 16 bytes in one chunk: rings and staging area fill 137 GB."""
    torch.cuda.empty_cache()
    E = 1 << 20
    cfg = pt.make_config(n_layers=1, batch=1, n_q_heads=32, n_kv_heads=32, head_dim=256, window=E, evict_chunk=E, dtype="fp32",
                         encode_enabled=0)
    if torch.cuda.mem_get_info()[0] < pt.ptenc_workspace_bytes(cfg) + (6 << 30):
        pytest.skip("the device has no room for it")
    gen = torch.Generator(device="cuda").manual_seed(7)
    c = pt.Cache(cfg)
    k, v = (torch.randn(1, 1, 1, 32, 256, generator=gen, device="cuda") for _ in range(2))
    _commit_takes_the_whole_window(c, k, v)
    c.close()
    del c
    torch.cuda.empty_cache()


def test_commit_without_encoder_and_bad_paths():
    p = Pair(pt, n_layers=1, batch=4, n_q_heads=4, n_kv_heads=2, head_dim=64, window=10, seed=11, set_encoder=False)
    _fill(p, 12)
    _, k, v = _drafts(p, 5)
    path = np.tile(np.arange(5), (4, 1))
    n = np.full(4, 5)
    p.cache.commit_path(-1, k, v, _cuda(path), _cuda(n))
    so.commit_path(p.orc, 0, np64(k[0]), np64(v[0]), path, n)
    p.check_ring()
    _check_rows(p)
    assert p.cache.status() == 0
    before = [t.clone() for t in _rings(p.cache)]
    path[0, 3], path[1, 0], n[2] = 5, -1, 6
    ev = torch.full((1, 4), 9, dtype=torch.int32, device="cuda")
    p.cache.commit_path(-1, k, v, _cuda(path), _cuda(n), n_evicted_out=ev)
    assert p.cache.status() == 2 and ev.tolist() == [[0, 0, 0, 5]]
    for x, y in zip(before, _rings(p.cache)):
        assert torch.equal(x[:, :3], y[:, :3]) and not torch.equal(x[:, 3], y[:, 3])
    p.close()
    p = Pair(pt, n_layers=1, batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, window=10, seed=11, encode_enabled=0)
    _fill(p, 12)
    _, k, v = _drafts(p, 5)
    before = p.cache.get_state(0)
    p.cache.commit_path(-1, k, v, _cuda(path[2:, :]), _cuda([5, 5]))
    assert torch.equal(before, p.cache.get_state(0))
    p.close()


# ------------------------------------------------------------------------------------------------------------ verify
def _verify_case(rng, B, T, V, dtype, kind, sharp=2.5, agree=0.9):
    tdt = torch.float32 if dtype == "fp32" else torch.bfloat16
    z = rng.standard_normal((B, T, V)) * sharp
    p = torch.softmax(torch.as_tensor(z), -1).to(tdt)
    q = torch.softmax(torch.as_tensor(agree * z + 0.6 * rng.standard_normal((B, T, V))), -1).to(tdt)
    parent = np.full((B, T), -1, np.int32)
    for i in range(1, T):
        parent[:, i] = {"chain": i - 1, "star": 0}.get(kind, 0) if kind != "tree" else rng.integers(max(0, i - 3), i, B)
    tok = np.full((B, T), V + 5, np.int32)                   # the root's entry is not read
    qn = q.double().numpy()
    for b in range(B):
        for i in range(1, T):
            row = qn[b, parent[b, i]]
            tok[b, i] = rng.choice(V, p=row / row.sum())
    u = rng.random((B, T)).astype(np.float32)
    return p, q, tok, parent, u


def _run_verify(p, q, tok, parent, u, n=None, active=None):
    B, T, V = p.shape
    path = torch.full((B, T), -7, dtype=torch.int32, device="cuda")
    n_path = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    nxt = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    pt.verify_tree(p.cuda(), None if q is None else q.cuda(), _cuda(tok), _cuda(parent), _cuda(u, torch.float32), path, n_path,
                   nxt, None if n is None else _cuda(n), None if active is None else _cuda(active, torch.uint8))
    return path.cpu().numpy(), n_path.cpu().numpy(), nxt.cpu().numpy()


def _check_verify(p, q, tok, parent, u, n=None, active=None):
    path, n_path, nxt = _run_verify(p, q, tok, parent, u, n, active)
    pn, qn = p.double().numpy(), None if q is None else q.double().numpy()
    rejected = 0
    for b in range(p.shape[0]):
        if active is not None and not active[b]:
            assert (path[b] == -7).all() and n_path[b] == -7 and nxt[b] == -7
            continue
        line, x, margin = so.verify_tree(pn[b], None if qn is None else qn[b], tok[b], parent[b], u[b],
                                         None if n is None else n[b])
        assert margin > 1e-13, "a decision on the border: both answers are right, the seed says nothing"
        assert n_path[b] == len(line) and list(path[b, :len(line)]) == line and (path[b, len(line):] == -1).all()
        assert nxt[b] == x, (b, nxt[b], x)
        rejected += len(line) < (p.shape[1] if n is None else n[b])
    return rejected


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,T,V,kind", [(1, 1, 1, "chain"), (3, 4, 2, "tree"), (16, 6, 7, "tree"), (9, 12, 513, "tree"),
                                        (5, 9, 4099, "chain"), (6, 24, 1000, "star"), (4, 64, 129, "tree"),
                                        (3, 5, 50001, "tree"), (2, 3, 131077, "star")])
def test_verify_against_the_oracle(dtype, B, T, V, kind):
    rng = np.random.default_rng(V + T)
    for turn in range(3 if V < 5000 else 1):
        case = _verify_case(rng, B, T, V, dtype, kind, agree=(0.9, 0.3, 1.0)[turn])
        _check_verify(*case)
        p, q, tok, parent, u = case
        _check_verify(p, None, tok, parent, u)
        n = rng.integers(1, T + 1, B)
        active = (rng.random(B) < 0.7).astype(np.uint8)
        _check_verify(p, q, tok, parent, u, n, active)
        _check_verify(p, None, tok, parent, u, n)


def test_verify_where_the_clusters_shrink():
    """Batches around those at which a sequence gets half as many CTAs on a device of 148 SMs: the same answers as sequence by
    sequence, which has the most."""
    rng = np.random.default_rng(6)
    B, T, V = 593, 4, 33001
    gen = torch.Generator(device="cuda").manual_seed(6)
    p, q = (torch.softmax(2.5 * torch.randn(B, T, V, generator=gen, device="cuda"), -1) for _ in range(2))
    parent = np.tile([-1, 0, 0, 1], (B, 1))
    tok, u = rng.integers(0, V, (B, T)), rng.random((B, T)).astype(np.float32)
    tok[:, 1] = p[:, 0].argmax(-1).cpu().numpy()
    for dq in (q, None):
        one = [_run_verify(p[b:b + 1], None if dq is None else dq[b:b + 1], tok[b:b + 1], parent[b:b + 1], u[b:b + 1]) for b in range(B)]
        for n in (74, 75, 148, 149, 296, 297, 592, 593):
            got = _run_verify(p[:n], None if dq is None else dq[:n], tok[:n], parent[:n], u[:n])
            for i, x in enumerate(got):
                assert np.array_equal(x, np.concatenate([o[i] for o in one[:n]]))


def test_verify_flat_rows_draw_the_right_neighbour():
    """Nearly uniform rows of 131071 entries: neighbouring borders lie 7.6e-6 apart and 32-bit sums of them are off by as much."""
    rng = np.random.default_rng(3)
    B, V = 64, 131071
    p = torch.as_tensor(rng.random((B, 1, V)) + 0.5, dtype=torch.float32)
    p /= p.sum(-1, keepdim=True)
    u = rng.random((B, 1)).astype(np.float32)
    u[:4, 0] = [0.0, np.float32(1) - np.float32(2) ** -24, 0.5, 1e-7]
    _check_verify(p, None, np.zeros((B, 1), np.int32), np.full((B, 1), -1, np.int32), u)


def test_verify_rows_that_leave_nothing():
    """Draft and target equal (nothing is left after a rejection), certain targets, rows of zeros, zero draft probability."""
    T, V = 4, 40
    eye = torch.zeros(6, T, V)
    eye[:, :, 5] = 1.0
    parent = np.tile(np.array([-1, 0, 0, 1], np.int32), (6, 1))
    tok = np.tile(np.array([0, 5, 5, 9], np.int32), (6, 1))
    u = np.full((6, T), 0.5, np.float32)
    p, q = eye.clone(), eye.clone()
    q[0] *= 2.5                                               # u q >= p: rejected, and p - q leaves nothing: p again
    q[1, :, 5], q[1, :, 6] = 0.0, 1.0                         # a drafted token the draft gave no probability: taken
    p[2] = 0.0                                                # a row without weight
    p[3, 0] = 0.0
    p[3, 0, 39] = 0.25                                        # rows need not sum to one
    p[4, :, 0] = 1e-30                                        # what a rejection leaves may be tiny: it is all there is
    path, n_path, nxt = _run_verify(p, q, tok, parent, u)
    assert n_path.tolist() == [1, 2, 1, 1, 2, 2] and nxt.tolist() == [5, 5, -1, 39, 0, 5]
    ok = [0, 1, 3, 4, 5]
    for b in ok:
        line, x, _ = so.verify_tree(p[b].double().numpy(), q[b].double().numpy(), tok[b], parent[b], u[b])
        got = _run_verify(p, q, tok, parent, u)
        assert list(got[0][b, :len(line)]) == line and got[2][b] == x


def test_verify_bad_trees_give_no_path():
    rng = np.random.default_rng(5)
    p, q, tok, parent, u = _verify_case(rng, 8, 5, 64, "fp32", "chain")
    n = np.full(8, 5)
    parent[0, 0], parent[1, 2], parent[2, 3], parent[3, 1] = 0, 2, -1, 7
    tok[4, 2], tok[5, 1] = 64, -1
    n[6] = 6
    path, n_path, nxt = _run_verify(p, q, tok, parent, u, n)
    assert (path[:7] == -1).all() and (n_path[:7] == 0).all() and (nxt[:7] == -1).all()
    assert n_path[7] >= 1 and 0 <= nxt[7] < 64


def test_rubbish_in_finished_sequences_is_not_looked_at():
    """What belongs to inactive sequences may hold anything: parents, counts, paths, tokens, probabilities.  Nothing is written
    for them and the status word stays clean; sequences without nodes or path likewise keep what they have."""
    B, T, V = 6, 9, 300
    for dtype, D in (("bf16", 128), ("bf16", 32), ("fp32", 64)):
        p = Pair(pt, n_layers=2, batch=B, n_q_heads=8, n_kv_heads=2, head_dim=D, window=40, dtype=dtype, seed=16)
        _fill(p, 50)
        q, k, v = _drafts(p, T)
        rng = np.random.default_rng(D)
        parent, n = _trees(rng, B, T, "tree"), np.full(B, T)
        active = np.array([1, 0, 1, 0, 1, 1], np.uint8)
        good = torch.full_like(q, 3.0)
        p.cache.tree_attn(-1, q, k, v, _cuda(parent), good, n_nodes=_cuda(n), active=_cuda(active, torch.uint8))
        n[5] = 0
        parent[[1, 3, 5]], n[[1, 3]] = 99, [-5, 1000]
        for x in (q, k, v):
            x[:, [1, 3, 5]] = float("nan")
        out = torch.full_like(q, 3.0)
        p.cache.tree_attn(-1, q, k, v, _cuda(parent), out, n_nodes=_cuda(n), active=_cuda(active, torch.uint8))
        assert p.cache.status() == 0
        assert torch.equal(out[:, [0, 2, 4]], good[:, [0, 2, 4]]) and (out[:, [1, 3, 5]] == 3.0).all()
        before, states = [r.clone() for r in _rings(p.cache)], [p.cache.get_state(l) for l in range(2)]
        path, m = np.tile(np.arange(T), (B, 1)), np.full(B, T)
        path[[1, 3, 5]], m[[1, 3, 5]] = -7, [1000, -3, 0]
        p.cache.commit_path(-1, k, v, _cuda(path), _cuda(m), _cuda(active, torch.uint8))
        assert p.cache.status() == 0
        for x, y in zip(before, _rings(p.cache)):
            assert torch.equal(x[:, [1, 3, 5]], y[:, [1, 3, 5]]) and not torch.equal(x[:, 0], y[:, 0])
        for l in range(2):
            assert torch.equal(states[l][[1, 3, 5]], p.cache.get_state(l)[[1, 3, 5]])
            assert bool(torch.isfinite(p.cache.get_state(l)).all())
        p.close()
    case = _verify_case(np.random.default_rng(1), B, T, V, "fp32", "tree")
    want = _run_verify(*case, active=active)
    p, dq, tok, parent, u = case
    p[[1, 3]], dq[[1, 3]], tok[[1, 3]], parent[[1, 3]] = float("nan"), float("inf"), -9, 77
    for x, y in zip(want, _run_verify(p, dq, tok, parent, u, active=active)):
        assert np.array_equal(x, y)


def test_verify_survives_rows_that_are_no_numbers():
    """The documentation asks for finite rows; others give some answer in range and leave the other sequences alone."""
    rng = np.random.default_rng(2)
    p, q, tok, parent, u = _verify_case(rng, 6, 5, 2051, "fp32", "tree")
    for dq in (q, None):
        want = _run_verify(p, dq, tok, parent, u)
        p2 = p.clone()
        p2[0], p2[1], p2[2, :, ::7] = float("nan"), float("inf"), float("inf")
        p2[3, :, 5] = -1.0
        got = _run_verify(p2, dq, tok, parent, u)
        for x, y in zip(want, got):
            assert np.array_equal(x[4:], y[4:])
        assert ((got[2] >= -1) & (got[2] < 2051)).all() and ((got[1] >= 1) & (got[1] <= 5)).all()


@pytest.mark.parametrize("with_q", [True, False])
def test_verify_rows_past_32_bits(with_q):
    """2.4e9 entries: the last sequence gives what it gives alone, in rows of 1.3e8 entries and of an odd width."""
    B, T, V = 6, 3, 2 ** 27 + 1
    gen = torch.Generator(device="cuda").manual_seed(3)
    p = torch.rand(B, T, V, generator=gen, device="cuda", dtype=torch.bfloat16)
    q = torch.rand(B, T, V, generator=gen, device="cuda", dtype=torch.bfloat16) if with_q else None
    assert p.numel() > 2 ** 31
    tok = torch.randint(0, V, (B, T), generator=gen, device="cuda", dtype=torch.int32)
    parent = torch.tensor([[-1, 0, 0]] * B, dtype=torch.int32, device="cuda")
    u = torch.rand(B, T, generator=gen, device="cuda")
    u[:, 1:] = 1 - 2.0 ** -24                                 # rejected but where the target's entry is the larger one

    def run(lo):
        n, i32 = B - lo, dict(dtype=torch.int32, device="cuda")
        path, n_path, nxt = torch.empty(n, T, **i32), torch.empty(n, **i32), torch.empty(n, **i32)
        pt.verify_tree(p[lo:].clone(), None if q is None else q[lo:].clone(), tok[lo:].clone(), parent[lo:].clone(), u[lo:].clone(),
                       path, n_path, nxt)
        return path, n_path, nxt

    for x, y in zip(run(0), run(B - 1)):
        assert torch.equal(x[-1], y[-1])
    assert int(run(0)[2].min()) >= 0 and int(run(0)[2].max()) > 2 ** 20


def _stretch_rows(dtype):
    """Rows of 50001 entries, of which a cluster's warps sum about 800 each, with two certain drafts at the start of the row that
    are rejected there: (entry 3, entry 7, entry 11); the rest of the row's weight lies from entry 30000 on.  Taking the two
    out of the stretch's sum leaves a residue above zero, one below zero, or hides the third entry altogether."""
    small = dict(fp32=(1e-12, 1e-10, 3e-11), bf16=(1e-16, 1.1e-15, 3e-15))[dtype]
    rows = [(0.3, small[0], 0.0), (0.3, small[1], 0.0), (small[1], 0.3, 0.0), (0.4, small[2], 0.0), (0.3, 0.0, 1e-20),
            (0.3, small[1], 1e-20), (1e-10, 0.3, 1e-25), (0.3, 0.2, 1e-6)]
    p = torch.zeros(len(rows), 50001)
    for x, (a, b, c) in zip(p, rows):
        x[3], x[7], x[11] = a, b, c
        x[30000:30010] = (1 - a - b - c) / 10
    return p.to(torch.float32 if dtype == "fp32" else torch.bfloat16)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_certain_drafts_that_take_nearly_all_of_a_stretch(dtype):
    """u[0] = 0 draws the first token with any weight left, however little it is beside what the rejected drafts held; at a root and
    at a node that was accepted after rejections.  With u[0] = 0 the definition has no rounding: every sum up to the drawn
    token is zero or not."""
    rows = _stretch_rows(dtype)
    B, V = rows.shape
    first = torch.zeros(V)
    first[[3, 40, 49000]] = torch.tensor([0.25, 0.25, 0.5])
    for order in ((3, 7), (7, 3)):
        # at the root: both siblings rejected
        p = rows[:, None].expand(B, 3, V).contiguous()
        tok, par = np.tile([0, *order], (B, 1)), np.tile([-1, 0, 0], (B, 1))
        u = np.tile(np.float32([0.0, 0.99, 0.99]), (B, 1))
        # behind an accepted sibling: entries 3 and 40 of another row come first, the second of them is taken
        deep = torch.stack([first.to(rows.dtype).expand(B, V), rows, rows, rows, rows], 1).contiguous()
        tok2, par2 = np.tile([0, 3, 40, *order], (B, 1)), np.tile([-1, 0, 0, 2, 2], (B, 1))
        u2 = np.tile(np.float32([0.0, 0.9, 0.1, 0.99, 0.99]), (B, 1))
        for q, t, pa, uu, line in ((p, tok, par, u, [0]), (deep, tok2, par2, u2, [0, 2])):
            path, n_path, nxt = _run_verify(q, None, t, pa, uu)
            for b in range(B):
                want = so.verify_tree(q[b].double().numpy(), None, t[b], pa[b], uu[b])
                assert want[0] == line
                assert list(path[b, :n_path[b]]) == line and nxt[b] == want[1], (order, b, nxt[b], want[1])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_certain_drafts_on_peaked_rows(dtype):
    """Rows with a few tokens of weight and zeros elsewhere (what a top-k filter leaves), siblings drawn among those tokens, the same
    token twice included."""
    rng = np.random.default_rng(8)
    B, T, V = 48, 12, 20011
    p = torch.zeros(B, T, V, dtype=torch.float64)
    tok = np.zeros((B, T), np.int32)
    for b in range(B):
        k = int(rng.integers(2, 30))
        where = np.sort(rng.choice(V, k, replace=False)) if b % 2 else int(rng.integers(0, V - 64)) + np.sort(rng.choice(64, k, replace=False))
        for i in range(T):
            w = np.exp(rng.standard_normal(k) * rng.choice([1.0, 8.0, 16.0]))
            p[b, i, where] = torch.as_tensor(w / w.sum())
        tok[b] = where[rng.integers(0, k, T)]
    p = p.to(torch.float32 if dtype == "fp32" else torch.bfloat16)
    parent = np.full((B, T), -1, np.int32)
    for i in range(1, T):
        parent[:, i] = np.where(rng.random(B) < 0.8, 0, rng.integers(0, i, B))
    u = rng.random((B, T)).astype(np.float32)
    for zero in (False, True):
        if zero:
            u[:, 0] = 0.0
        path, n_path, nxt = _run_verify(p, None, tok, parent, u)
        for b in range(B):
            line, x, margin = so.verify_tree(p[b].double().numpy(), None, tok[b], parent[b], u[b])
            if margin <= 1e-12 and not zero:
                continue                                      # on a border up to rounding: both neighbours are right
            assert list(path[b, :n_path[b]]) == line and nxt[b] == x, (zero, b, nxt[b], x)


# ------------------------------------------------------------------------------------------------------------ together
class _Round:
    """One speculative round of a stand-in model: every node's output of the last layer, projected to a vocabulary."""

    def __init__(self, p, T, V, seed=0):
        self.p, self.T, self.V = p, T, V
        rng = np.random.default_rng(seed)
        self.proj = rng.standard_normal((p.Hq * p.D, V)) * 0.7
        self.parent = _trees(rng, p.B, T, "tree")
        self.parent[:, 1:] = np.maximum(self.parent[:, 1:], 0)
        self.n = rng.integers(1, T + 1, p.B)
        self.tok = rng.integers(0, V, (p.B, T))
        self.u = rng.random((p.B, T)).astype(np.float32)


def test_rounds_together_against_the_oracle():
    """Six rounds of attention, verification and commit over all layers, as a rollout runs them; the oracle sees the same
    inputs and, at the one place where a rounding could send the two sides different ways (the probabilities), the GPU's."""
    B, T, V = 4, 10, 50
    p = Pair(pt, n_layers=3, batch=B, n_q_heads=14, n_kv_heads=2, head_dim=128, window=40, evict_chunk=1, seed=12, n_global=32,
             rank=32)
    p.prefill([5, 0, 9, 1], 9)
    _fill(p, 30)
    moved = 0
    for turn in range(6):
        R = _Round(p, T, V, turn)
        drafts = _drafts(p, T, seed=turn)
        out, _ = _check_tree(p, T, R.parent, R.n, drafts=drafts)
        probs = torch.softmax((out[-1].float().reshape(B, T, -1).cpu() @ torch.as_tensor(R.proj, dtype=torch.float32)), -1)
        path, n_path, nxt = _run_verify(probs, None, R.tok, R.parent, R.u, R.n)
        for b in range(B):
            line, x, _ = so.verify_tree(probs[b].double().numpy(), None, R.tok[b], R.parent[b], R.u[b], R.n[b])
            assert list(path[b, :n_path[b]]) == line and nxt[b] == x
        p.cache.commit_path(-1, drafts[1], drafts[2], _cuda(path), _cuda(n_path))
        for l in range(p.L):
            so.commit_path(p.orc, l, np64(drafts[1][l]), np64(drafts[2][l]), path, n_path)
        p.check_ring()
        p.check_state()
        _check_rows(p)
        moved += int(n_path.sum())
    assert moved > 6 * B
    p.step(1000)                                              # and the ordinary step goes on from there
    assert p.cache.status() == 0
    p.close()


def test_a_captured_round_replays_on_another_stream():
    """A round captured into a graph, replayed three times on new inputs in the same buffers, equals eager calls; everything
    runs on a stream other than the default one."""
    B, T, V = 3, 7, 3001
    kw = dict(n_layers=2, batch=B, n_q_heads=8, n_kv_heads=2, head_dim=128, window=33, evict_chunk=1, seed=13, n_global=32, rank=32)
    a, b = Pair(pt, **kw), Pair(pt, **kw)
    for x in (a, b):
        _fill(x, 40)
    rng = np.random.default_rng(0)
    case = [_verify_case(rng, B, T, V, "fp32", "tree") for _ in range(3)]
    parent = _cuda(case[0][3])

    def buffers():
        q, k, v = (t.clone() for t in _drafts(a, T))
        i32 = dict(dtype=torch.int32, device="cuda")
        return dict(q=q, k=k, v=v, out=torch.zeros_like(q), lse=torch.zeros(2, B, T, 8, device="cuda"),
                    p=torch.zeros(B, T, V, device="cuda"), dq=torch.zeros(B, T, V, device="cuda"), tok=torch.zeros(B, T, **i32),
                    u=torch.zeros(B, T, device="cuda"), path=torch.zeros(B, T, **i32), n=torch.zeros(B, **i32),
                    nxt=torch.zeros(B, **i32), par=parent.clone())

    def round_(cache, s):
        cache.tree_attn(-1, s["q"], s["k"], s["v"], s["par"], s["out"], lse_out=s["lse"])
        pt.verify_tree(s["p"], s["dq"], s["tok"], s["par"], s["u"], s["path"], s["n"], s["nxt"])
        cache.commit_path(-1, s["k"], s["v"], s["path"], s["n"])

    def load(s, turn):
        p, q, tok, par, u = case[turn]
        for name, t in (("p", p), ("dq", q), ("tok", _cuda(tok)), ("u", _cuda(u, torch.float32)), ("par", _cuda(par))):
            s[name].copy_(t)
        for name, t in zip("qkv", _drafts(a, T, seed=turn)):
            s[name].copy_(t)

    sa, sb = buffers(), buffers()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        load(sa, 0)
        ws = a.cache.workspace.clone()
        round_(a.cache, sa)                                   # once eagerly: kernels are loaded outside the capture
        a.cache.workspace.copy_(ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            round_(a.cache, sa)
        for turn in range(3):
            load(sa, turn)
            load(sb, turn)
            graph.replay()
            round_(b.cache, sb)
            stream.synchronize()
            for name in ("path", "n", "nxt"):
                assert torch.equal(sa[name], sb[name]), name
            assert torch.equal(sa["out"], sb["out"]) and torch.equal(sa["lse"], sb["lse"])
            for x, y in zip(_rings(a.cache), _rings(b.cache)):
                assert torch.equal(x, y)
            for l in range(2):
                assert torch.equal(a.cache.get_state(l), b.cache.get_state(l))
    torch.cuda.synchronize()
    assert a.cache.status() == 0 and b.cache.status() == 0
    del graph
    for x in (a, b):
        x.close()


def test_two_caches_on_two_streams_at_once():
    """Rounds on two handles, queued on two streams without a wait between them, give the bits of the same rounds one by one."""
    T, turns = 7, 12
    kws = [dict(n_layers=2, batch=24, n_q_heads=8, n_kv_heads=4, head_dim=128, window=300, evict_chunk=1),
           dict(n_layers=2, batch=6, n_q_heads=8, n_kv_heads=2, head_dim=64, window=96, evict_chunk=16)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    pairs = [Pair(pt, seed=18, n_global=32, rank=32, **kw) for kw in kws]
    drafts = [[_drafts(p, T, seed=t) for t in range(turns)] for p in pairs]
    rng = np.random.default_rng(4)
    parents = [_cuda(_trees(rng, kw["batch"], T, "tree")) for kw in kws]
    paths = [[_cuda(np.sort(rng.permuted(np.tile(np.arange(T), (kw["batch"], 1)), axis=1)[:, :4], axis=1)) for _ in range(turns)]
             for kw in kws]
    count = [torch.full((kw["batch"],), 4, dtype=torch.int32, device="cuda") for kw in kws]
    full = [[torch.cat([x, x[:, :3]], 1).contiguous() for x in ps] for ps in paths]

    def turn(i, t, out):
        q, k, v = drafts[i][t]
        pairs[i].cache.tree_attn(-1, q, k, v, parents[i], out)
        pairs[i].cache.commit_path(-1, k, v, full[i][t], count[i])

    for p in pairs:
        for t in range(p.W + 3):
            k, v = p.gen.step_kv(t)
            p.cache.append_evict(-1, k, v)
    start = [p.cache.workspace.clone() for p in pairs]
    results = []
    for together in (False, True):
        for p, ws in zip(pairs, start):
            p.cache.workspace.copy_(ws)
        outs = [[torch.zeros_like(d[0]) for d in ds] for ds in drafts]
        torch.cuda.synchronize()
        for t in range(turns):
            for i in (0, 1):
                with torch.cuda.stream(streams[i]):
                    turn(i, t, outs[i][t])
                if not together:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        assert all(p.cache.status() == 0 for p in pairs)
        results.append((outs, [r.clone() for p in pairs for r in _rings(p.cache)], [p.cache.get_state(l) for p in pairs for l in (0, 1)]))
    for x, y in zip(results[0][0], results[1][0]):
        assert all(torch.equal(a, b) and float(a.float().abs().max()) > 0 for a, b in zip(x, y))
    for part in (1, 2):
        assert all(torch.equal(a, b) for a, b in zip(results[0][part], results[1][part]))
    for p in pairs:
        p.close()
