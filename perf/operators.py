"""The operators of a speculative decode step under the fixed-size cache, as cases that can be timed and compared.

A draft model proposes a tree of tokens per sequence; the target model scores every node against the cache with one pass
over the window (`tree_attn`), the drafted tokens are verified against the target's probabilities from given random
numbers (`verify_tree`), and the accepted path enters the cache, evicting and encoding as token-by-token decoding would
(`commit_path`).  `own` selects between the operators in their plain form (elementary torch operations in 32 bits, 64
where a border or a position decides) and the calls a user makes of the library.
"""
import numpy as np
import torch

own = False

DEV = "cuda"

# Attention shapes: those of the benchmark's workloads (heads, KV heads, head size, window) at one layer per call, which is
# how a model with real weights calls them; the commit also in one call over all layers.  E = 1 evicts one token per
# arriving token, E = W / 4 is the chunk of the paper's runs.  G = r = 32 state rows and rank.


def listed():
    return [
        # one sequence, a short chain: the smallest call, latency counts
        {"name": "tree one chain", "op": "tree", "L": 1, "B": 1, "T": 5, "Hq": 16, "Hkv": 2, "D": 128, "W": 1024, "E": 1,
         "shape": "chain", "fill": "full", "prompt": 0, "mask": False, "dtype": "bf16"},
        # a rollout batch of the 7B shape, trees of 16 nodes, every ring full and evicting
        {"name": "tree batch 16", "op": "tree", "L": 1, "B": 128, "T": 16, "Hq": 28, "Hkv": 4, "D": 128, "W": 2048, "E": 1,
         "shape": "tree", "fill": "full", "prompt": 0, "mask": False, "dtype": "bf16"},
        # large trees over long windows of the 8B shape: as much arithmetic as bandwidth
        {"name": "tree batch 64", "op": "tree", "L": 1, "B": 64, "T": 64, "Hq": 32, "Hkv": 8, "D": 128, "W": 4096, "E": 1,
         "shape": "tree", "fill": "full", "prompt": 0, "mask": False, "dtype": "bf16"},
        # sequences of all lengths and trees of all sizes, a pinned prompt, finished sequences, chunks about to leave
        {"name": "tree ragged", "op": "tree", "L": 2, "B": 23, "T": 13, "Hq": 28, "Hkv": 4, "D": 64, "W": 1000, "E": 250,
         "shape": "tree", "fill": "ragged", "prompt": 100, "mask": True, "dtype": "bf16"},
        # fp32 storage, the smallest configuration's heads
        {"name": "tree fp32", "op": "tree", "L": 1, "B": 16, "T": 8, "Hq": 4, "Hkv": 1, "D": 64, "W": 1024, "E": 1,
         "shape": "tree", "fill": "full", "prompt": 0, "mask": False, "dtype": "fp32"},
        # one sequence, a short chain: the smallest call
        {"name": "verify one chain", "op": "verify", "B": 1, "T": 5, "V": 32000, "shape": "chain", "ragged": False,
         "draft": "sampled", "dtype": "fp32"},
        # a rollout batch with a large vocabulary
        {"name": "verify batch", "op": "verify", "B": 128, "T": 8, "V": 152000, "shape": "tree", "ragged": False,
         "draft": "sampled", "dtype": "fp32"},
        # bf16 rows of an odd width (no row but the first is aligned), trees of different sizes
        {"name": "verify odd bf16", "op": "verify", "B": 61, "T": 16, "V": 65537, "shape": "tree", "ragged": True,
         "draft": "sampled", "dtype": "bf16"},
        # drafts without probabilities (a lookup or a greedy draft): one-hot rows
        {"name": "verify one-hot", "op": "verify", "B": 32, "T": 12, "V": 50001, "shape": "tree", "ragged": True,
         "draft": "onehot", "dtype": "fp32"},
        # one layer of a small batch: latency
        {"name": "commit one layer", "op": "commit", "L": 1, "B": 8, "T": 5, "Hq": 16, "Hkv": 2, "D": 128, "W": 1024, "E": 1,
         "fill": "full", "prompt": 0, "mask": False, "dtype": "bf16"},
        # all layers of a rollout batch in one call, full rings: every accepted token evicts and encodes one
        {"name": "commit all layers", "op": "commit", "L": 28, "B": 32, "T": 8, "Hq": 28, "Hkv": 4, "D": 128, "W": 512, "E": 1,
         "fill": "full", "prompt": 0, "mask": False, "dtype": "bf16"},
        # a quarter of the window leaves at once for the sequences whose rings are about to run over
        {"name": "commit chunks", "op": "commit", "L": 4, "B": 48, "T": 16, "Hq": 28, "Hkv": 4, "D": 128, "W": 516, "E": 129,
         "fill": "ragged", "prompt": 60, "mask": True, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["tree", "tree", "verify", "commit"])
    if op == "verify":
        T = _log(rng, 1, 24)
        V = _log(rng, 1000, 152000)
        B = max(1, min(_log(rng, 1, 160), 128 * 8 * 152000 // (T * V)))
        return {"op": "verify", "B": B, "T": T, "V": V, "shape": rng.choice(["chain", "tree"]),
                "ragged": rng.random() < 0.5, "draft": rng.choice(["sampled", "sampled", "onehot"]),
                "dtype": rng.choice(["fp32", "bf16"])}
    heads = rng.choice([(4, 1, 64), (14, 2, 64), (16, 2, 128), (28, 4, 128), (32, 8, 128), (12, 12, 64), (24, 8, 128)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    W = _log(rng, 33, 4096)
    E = rng.choice([1, 1, max(1, W // 4), max(1, W // 10)])
    c = {"op": op, "L": rng.choice([1, 1, 2, 3]), "B": _log(rng, 1, 128), "T": _log(rng, 1, 64), "Hq": heads[0],
         "Hkv": heads[1], "D": heads[2], "W": W, "E": E, "fill": rng.choice(["full", "ragged"]),
         "prompt": rng.choice([0, 0, W // 5]), "mask": rng.random() < 0.3, "dtype": dtype}
    if op == "tree":
        c["shape"] = rng.choice(["chain", "tree"])
    elif c["T"] > 16:
        c["T"] = 16
    # no more work than the largest listed case of the type
    most = 2.5e11 if dtype == "bf16" else 4e9
    while c["B"] > 1 and (work(c)["flops"] > most or work(c)["bytes"] > 1.0e9):
        c["B"] //= 2
    return c


# ------------------------------------------------------------------------------------------------------------ inputs
class State:
    pass


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _parents(rs, B, T, shape):
    """Parents in topological order: a chain, or a tree that grows from its newest few nodes."""
    par = np.full((B, T), -1, np.int32)
    for i in range(1, T):
        par[:, i] = i - 1 if shape == "chain" else rs.randint(max(0, i - 4), i, B)
    return par


def _dev(a, dtype):
    return torch.as_tensor(np.ascontiguousarray(a)).to(dtype).to(DEV)


def _rings(s, case, rs, gen):
    """The cache of a rollout in progress: rings, ring words, pinned prompts.  The words are the same for every layer, as they
    are when all layers decode the same tokens."""
    L, B, Hkv, W, D, E = (case[k] for k in ("L", "B", "Hkv", "W", "D", "E"))
    ns = rs.randint(0, case["prompt"] + 1, B) if case["prompt"] else np.zeros(B, np.int64)
    C = W - ns
    if case["fill"] == "full":
        count = C.copy()
    else:
        count = rs.randint(0, C + 1)
        near = rs.rand(B) < 0.5                                   # half of them about to run over
        count = np.where(near, np.maximum(0, C - rs.randint(0, 6, B)), count)
    head = np.where(count >= np.maximum(1, C - np.minimum(E, C) + 1), rs.randint(0, C), 0)
    napp = ns + count + head
    words = {"head": head, "count": count, "n_app": napp, "n_sink": ns}
    s.K = torch.randn(L, B, Hkv, W, D, dtype=_dtype(case), device=DEV, generator=gen)
    s.V = torch.randn(L, B, Hkv, W, D, dtype=_dtype(case), device=DEV, generator=gen)
    for k, v in words.items():
        t = _dev(np.broadcast_to(v, (L, B)), torch.int64 if k == "n_app" else torch.int32)
        setattr(s, k, t)


def _cache(s, case):
    """The handle a user's program keeps, holding the same rings: the library's workspace takes their place."""
    import paper_2602_16839_b200 as pt
    s.pt = pt
    s.cache = pt.Cache(pt.make_config(n_layers=case["L"], batch=case["B"], n_q_heads=case["Hq"], n_kv_heads=case["Hkv"],
                                      head_dim=case["D"], window=case["W"], evict_chunk=case["E"], n_global=32, rank=32,
                                      dtype=case["dtype"]))
    base = s.cache.workspace.data_ptr()

    def take(region, t):
        ptr, n = s.cache.workspace_region(region)
        v = s.cache.workspace[ptr - base:ptr - base + n].view(t.dtype).view(t.shape)
        v.copy_(t)
        return v

    s.K, s.V = take(pt.binding.REGION_K, s.K), take(pt.binding.REGION_V, s.V)
    s.head, s.count = take(pt.binding.REGION_HEAD, s.head), take(pt.binding.REGION_COUNT, s.count)
    s.n_app, s.n_sink = take(pt.binding.REGION_NAPP, s.n_app), take(pt.binding.REGION_NPINNED, s.n_sink)
    if case["op"] == "commit":
        for l in range(case["L"]):
            s.cache.set_encoder(l, s.Wq[l], s.Wk[l], s.Wv[l], s.qg[l])
        s.S = take(pt.binding.REGION_STATE, s.S)


def prepare(case, seed):
    rs = np.random.RandomState(seed % (1 << 32))
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = State()
    s.case = case
    B, T = case["B"], case["T"]
    if case["op"] == "verify":
        V = case["V"]
        # target and draft agree mostly, as a draft worth having does; rows of a sampled language model are peaked
        z = torch.randn(B, T, V, device=DEV, generator=gen) * 2.5
        s.p = torch.softmax(z, -1).to(_dtype(case))
        z.mul_(0.9).add_(torch.randn(B, T, V, device=DEV, generator=gen), alpha=0.6)
        q = torch.softmax(z, -1).to(_dtype(case))
        par = _parents(rs, B, T, case["shape"])
        s.parent = _dev(par, torch.int32)
        at = s.parent.clamp(min=0).long()
        s.tokens = torch.zeros(B, T, dtype=torch.int32, device=DEV)
        for i in range(T):                                          # children are drawn from their parent's row
            row = q.gather(1, at[:, i, None, None].expand(B, 1, V))[:, 0].float()
            s.tokens[:, i] = torch.multinomial(row, 1, generator=gen)[:, 0].int()
        s.q = q if case["draft"] == "sampled" else None
        s.n_nodes = _dev(rs.randint(1, T + 1, B) if case["ragged"] else np.full(B, T), torch.int32)
        s.u = torch.rand(B, T, device=DEV, generator=gen)
        if own:
            import paper_2602_16839_b200 as pt
            s.pt = pt
            s.path = torch.empty(B, T, dtype=torch.int32, device=DEV)
            s.n_path = torch.empty(B, dtype=torch.int32, device=DEV)
            s.next = torch.empty(B, dtype=torch.int32, device=DEV)
        return s
    L, Hq, Hkv, D = (case[k] for k in ("L", "Hq", "Hkv", "D"))
    dt = _dtype(case)
    _rings(s, case, rs, gen)
    s.k = torch.randn(L, B, T, Hkv, D, dtype=dt, device=DEV, generator=gen)
    s.v = torch.randn(L, B, T, Hkv, D, dtype=dt, device=DEV, generator=gen)
    s.active = None
    if case["mask"]:
        act = rs.rand(B) < 0.8
        act[0] = True
        s.active = _dev(act, torch.uint8)
    if case["op"] == "tree":
        s.q = torch.randn(L, B, T, Hq, D, dtype=dt, device=DEV, generator=gen)
        s.parent = _dev(_parents(rs, B, T, case["shape"]), torch.int32)
        s.n_nodes = _dev(rs.randint(1, T + 1, B) if case["fill"] == "ragged" else np.full(B, T), torch.int32)
        s.out = torch.zeros(L, B, T, Hq, D, dtype=dt, device=DEV)
        s.lse = torch.zeros(L, B, T, Hq, device=DEV)
    else:
        d_kv, d_q, G, r = Hkv * D, Hq * D, 32, 32
        rnd = lambda *sh, std: (torch.randn(*sh, device=DEV, generator=gen) * std).to(dt)  # noqa: E731
        s.Wq, s.qg = rnd(L, r, d_q, std=d_q ** -0.5), rnd(L, G, d_q, std=r ** -0.5)
        s.Wk, s.Wv = rnd(L, r, d_kv, std=d_kv ** -0.5), rnd(L, r, d_kv, std=(d_kv * r) ** -0.5)
        S = torch.randn(L, B, G, r, device=DEV, generator=gen)
        s.S = S / S.square().sum(-1, keepdim=True).sqrt()
        s.Qa = torch.einsum("lgd,lrd->lgr", s.qg.double(), s.Wq.double()).float()
        n = rs.randint(1, T + 1, B)                                 # accepted: the root and some of the drafted tokens
        path = np.full((B, T), -1)
        for b in range(B):
            path[b, 0] = 0
            path[b, 1:n[b]] = 1 + np.sort(rs.choice(T - 1, n[b] - 1, replace=False)) if n[b] > 1 else []
        s.path, s.n_path = _dev(path, torch.int32), _dev(n, torch.int32)
        s.events = max(1, -(-T // min(case["E"], case["W"] - case["prompt"])))
    if own:
        _cache(s, case)
    return s


# ------------------------------------------------------------------------------------------------------------ plain forms
def _tree_plain(s):
    c = s.case
    L, B, T, Hq, Hkv, D, W, E = (c[k] for k in ("L", "B", "T", "Hq", "Hkv", "D", "W", "E"))
    g = Hq // Hkv
    node = torch.arange(T, device=DEV)
    # which nodes lie on each node's path: the parent relation squared until it is closed
    reach = ((s.parent[:, :, None] == node) | (node[:, None] == node)).float()
    reach = (reach @ reach).clamp(max=1)
    reach = (reach @ reach).clamp(max=1)
    reach = (reach @ reach).clamp(max=1)
    reach = (reach @ reach).clamp(max=1)
    reach = (reach @ reach).clamp(max=1)
    reach = (reach @ reach).clamp(max=1)
    anc = reach > 0
    depth = reach.sum(-1).long() - 1
    ns, head, count = s.n_sink.long()[..., None], s.head.long()[..., None], s.count.long()[..., None]
    cap = W - ns
    e = cap.clamp(max=E)
    over = (count + depth + 1 - cap).clamp(min=0)
    ev = (over + e - 1) // e * e                                    # tokens gone once the path to the node has arrived
    w = torch.arange(W, device=DEV)
    age = torch.where(w >= ns, (w - ns - head) % cap, -1)           # order of arrival of a slot's token
    live = ((age[:, :, None] >= ev[..., None]) & (age < count)[:, :, None]) | (w < ns)[:, :, None]
    kin = anc & (count[..., None] + depth[:, None, :] >= ev[..., None])
    mask = torch.cat([live, kin], -1).repeat_interleave(g, 2)       # rows: node by node, the group's heads inside
    q = s.q.float().view(L, B, T, Hkv, g, D).transpose(2, 3).reshape(L, B, Hkv, T * g, D)
    kt, vt = s.k.float().transpose(2, 3), s.v.float().transpose(2, 3)
    x = torch.cat([q @ s.K.float().transpose(-1, -2), q @ kt.transpose(-1, -2)], -1) * D ** -0.5
    x = x.masked_fill(~mask[:, :, None], float("-inf"))
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - m)
    z = p.sum(-1, keepdim=True)
    o = (p[..., :W] @ s.V.float() + p[..., W:] @ vt) / z
    back = lambda t: t.view(L, B, Hkv, T, g, -1).transpose(2, 3).reshape(L, B, T, Hq, -1)  # noqa: E731
    wanted = node < s.n_nodes[:, None]
    if s.active is not None:
        wanted = wanted & (s.active != 0)[:, None]
    wanted = wanted[None, :, :, None]
    return {"out": torch.where(wanted[..., None], back(o).to(s.out.dtype), s.out),
            "lse": torch.where(wanted, back(m + torch.log(z))[..., 0], s.lse)}


def _verify_plain(s):
    c = s.case
    B, T, V = c["B"], c["T"], c["V"]
    rows = torch.arange(B, device=DEV)
    cur = torch.zeros(B, dtype=torch.int64, device=DEV)
    n = torch.ones(B, dtype=torch.int64, device=DEV)
    path = torch.full((B, T), -1, dtype=torch.int64, device=DEV)
    path[:, 0] = 0
    r = s.p[:, 0].double()
    vocab = torch.arange(V, device=DEV)
    for i in range(1, T):                                           # a child is judged after its elder siblings: a recurrence
        x = s.tokens[:, i].long()
        here = (s.parent[:, i] == cur) & (i < s.n_nodes)
        q = (vocab == x[:, None]).double() if s.q is None else s.q[rows, cur].double()
        ok = here & (s.u[:, i].double() * q[rows, x] < r[rows, x])
        left = (r - q).clamp(min=0)
        total = left.sum(-1, keepdim=True)
        left = torch.where(total > 0, left / total, s.p[rows, cur].double())
        r = torch.where((here & ~ok)[:, None], left, torch.where(ok[:, None], s.p[:, i].double(), r))
        cur = torch.where(ok, i, cur)
        path[rows, torch.where(ok, n, 0)] = torch.where(ok, i, path[:, 0])
        n = n + ok
    cdf = r.cumsum(-1)
    nxt = (cdf <= s.u[:, :1].double() * cdf[:, -1:]).sum(-1)
    return {"path": path.int(), "n_path": n.int(), "next": nxt.int()}


def _commit_plain(s):
    c = s.case
    L, B, T, Hkv, D, W, E = (c[k] for k in ("L", "B", "T", "Hkv", "D", "W", "E"))
    li, bi = torch.arange(L, device=DEV)[:, None, None], torch.arange(B, device=DEV)[None, :, None]
    on = torch.ones(B, dtype=torch.bool, device=DEV) if s.active is None else s.active != 0
    m = torch.where(on, s.n_path, 0).long().expand(L, B)
    ns, head, count = s.n_sink.long(), s.head.long(), s.count.long()
    cap = W - ns
    e = cap.clamp(max=E)
    ev = ((count + m - cap).clamp(min=0) + e - 1) // e * e
    at = s.path.clamp(min=0).long().expand(L, B, T)
    kp, vp = s.k[li, bi, at], s.v[li, bi, at]                       # [L, B, T, Hkv, D], in order of arrival
    slot = lambda o: ns[..., None] + (head[..., None] + o) % cap[..., None]  # noqa: E731
    i = torch.arange(E, device=DEV)
    heads = torch.arange(Hkv, device=DEV)
    for k in range(s.events):                                       # the state is normalised after each eviction: a recurrence
        o = k * e[..., None] + i
        gone = (i < e[..., None]) & (o < ev[..., None])
        old = o < count[..., None]
        at_new = (o - count[..., None]).clamp(0, T - 1)

        def rows(ring, new):
            a = ring[li[..., None], bi[..., None], heads, slot(o)[..., None]]
            return torch.where(old[..., None, None], a, new[li, bi, at_new]).float().reshape(L, B, E, Hkv * D)

        ka = rows(s.K, kp) @ s.Wk.float().transpose(-1, -2)[:, None] * gone[..., None]
        va = rows(s.V, vp) @ s.Wv.float().transpose(-1, -2)[:, None] * gone[..., None]
        t = s.S + s.Qa[:, None] @ (ka.transpose(-1, -2) @ va)
        t = t / t.square().sum(-1, keepdim=True).sqrt().clamp(min=1e-12)
        s.S = torch.where(gone.any(-1)[..., None, None], t, s.S)
    j = torch.arange(T, device=DEV)
    last = (m - 1).clamp(min=0)[..., None]                          # a chain longer than the ring keeps its newest tokens:
    j = torch.where((j <= last) & (count[..., None] + j >= ev[..., None]), j, last)     # the others write the last once more
    to, some = slot(count[..., None] + j)[..., None], (m > 0)[..., None, None, None]
    for ring, new in ((s.K, kp), (s.V, vp)):
        ring[li[..., None], bi[..., None], heads, to] = torch.where(some, new[li, bi, j], ring[li[..., None], bi[..., None], heads, to])
    s.head = ((head + ev) % cap).int()
    s.count = (count + m - ev).int()
    s.n_app = s.n_app + m
    return _ring(s)


def _ring(s):
    return {"K": s.K, "V": s.V, "S": s.S, "head": s.head, "count": s.count, "n_app": s.n_app}


def run(s):
    op = s.case["op"]
    if not own:
        return {"tree": _tree_plain, "verify": _verify_plain, "commit": _commit_plain}[op](s)
    if op == "tree":
        s.cache.tree_attn(-1, s.q, s.k, s.v, s.parent, s.out, n_nodes=s.n_nodes, active=s.active, lse_out=s.lse)
        return {"out": s.out, "lse": s.lse}
    if op == "verify":
        s.pt.verify_tree(s.p, s.q, s.tokens, s.parent, s.u, s.path, s.n_path, s.next, n_nodes=s.n_nodes)
        return {"path": s.path, "n_path": s.n_path, "next": s.next}
    s.cache.commit_path(-1, s.k, s.v, s.path, s.n_path, active=s.active)
    return _ring(s)


# ------------------------------------------------------------------------------------------------------------ work
def work(case):
    """Mean sizes where they depend on the seed: half of the ragged rings run from empty to full, the others are nearly full;
    half of the nodes of ragged trees; half of a path is accepted."""
    elt = 2 if case["dtype"] == "bf16" else 4
    B, T = case["B"], case["T"]
    if case["op"] == "verify":
        rows = 1 if case["draft"] == "onehot" else 2                # the row sampled from, and the draft's beside it
        return {"bytes": float(B) * (case["V"] * elt * rows + T * (16 + 2 * elt)), "flops": float(B) * case["V"] * 4}
    L, Hq, Hkv, D, W = (case[k] for k in ("L", "Hq", "Hkv", "D", "W"))
    act = 0.8 if case["mask"] else 1.0
    d_kv = Hkv * D
    fill = 1.0 if case["fill"] == "full" else 0.75
    if case["op"] == "tree":
        n = fill * W
        t = T if case["fill"] == "full" else (T + 1) / 2
        return {"bytes": act * L * B * ((n + t) * d_kv * 2 * elt + t * Hq * (2 * D * elt + 4)),
                "flops": act * L * B * 4.0 * D * Hq * t * (n + t / 2)}
    m = (T + 1) / 2
    gone = m if case["fill"] == "full" else m / 2                   # evicted rows per sequence
    if case["E"] > 1:
        gone = max(1, case["E"]) * (1.0 if case["fill"] == "full" else 0.4)
    state = 2 * 32 * 32 * 4
    return {"bytes": act * L * B * (2 * d_kv * elt * (2 * m + gone) + state) + L * 2 * 32 * d_kv * elt,
            "flops": act * L * B * gone * (4.0 * d_kv * 32 + 4 * 32 * 32)}


# ------------------------------------------------------------------------------------------------------------ in 64 bits
def _sequential(count, cap, e, arrivals):
    """What a cache of `cap` tokens holds after the arrivals, one by one: (tokens left, tokens gone in order and by event)."""
    held, events = [("old", o) for o in range(count)], []
    for a in arrivals:
        if len(held) == cap:
            events.append(held[:e])
            held = held[e:]
        held.append(("new", a))
    return held, events


def _exact_tree(s):
    c = s.case
    L, B, T, Hq, Hkv, D, W, E = (c[k] for k in ("L", "B", "T", "Hq", "Hkv", "D", "W", "E"))
    g = Hq // Hkv
    out, lse = s.out.double(), s.lse.double()
    par, nn = s.parent.cpu().numpy(), s.n_nodes.cpu().numpy()
    head, count, sink = s.head.cpu().numpy(), s.count.cpu().numpy(), s.n_sink.cpu().numpy()
    act = None if s.active is None else s.active.cpu().numpy()
    for b in range(B):
        if act is not None and not act[b]:
            continue
        h0, n0, ns = int(head[0, b]), int(count[0, b]), int(sink[0, b])
        cap = W - ns
        seen = np.zeros((nn[b], W + T), bool)
        for i in range(nn[b]):
            line, j = [], i
            while j >= 0:
                line.insert(0, j)
                j = int(par[b, j])
            held, _ = _sequential(n0, cap, min(E, cap), line)
            idx = [ns + (h0 + o) % cap if kind == "old" else W + o for kind, o in held]
            seen[i, idx] = True
            seen[i, :ns] = True
        seen = torch.as_tensor(seen).to(DEV)
        for l in range(L):
            K = torch.cat([s.K[l, b], s.k[l, b].transpose(0, 1)], 1).double()
            V = torch.cat([s.V[l, b], s.v[l, b].transpose(0, 1)], 1).double()
            q = s.q[l, b, :nn[b]].double()                           # [n, Hq, D]
            for h in range(Hkv):
                x = torch.einsum("ngd,wd->ngw", q[:, h * g:(h + 1) * g], K[h]) / D ** 0.5
                x = torch.where(seen[:, None], x, -torch.inf)
                y = torch.logsumexp(x, -1)
                lse[l, b, :nn[b], h * g:(h + 1) * g] = y
                out[l, b, :nn[b], h * g:(h + 1) * g] = torch.einsum("ngw,wd->ngd", torch.exp(x - y[..., None]), V[h])
    return {"out": out, "lse": lse}


def _exact_verify(s):
    c = s.case
    B, T = c["B"], c["T"]
    tok, par, nn, u = (t.cpu().numpy() for t in (s.tokens, s.parent, s.n_nodes, s.u))
    path, n_path, nxt = np.full((B, T), -1, np.int32), np.zeros(B, np.int32), np.zeros(B, np.int32)
    get = lambda t, b, i: t[b, i].double().cpu().numpy()             # noqa: E731
    for b in range(B):
        line, searching = [0], True
        while searching:
            searching, at = False, line[-1]
            p = get(s.p, b, at)
            rest = p
            for child in [i for i in range(1, nn[b]) if par[b, i] == at]:
                x = tok[b, child]
                if s.q is None:
                    q = np.zeros_like(p)
                    q[x] = 1
                else:
                    q = get(s.q, b, at)
                if np.float64(u[b, child]) * q[x] < rest[x]:
                    line.append(child)
                    searching = True
                    break
                rest = np.maximum(rest - q, 0)
                rest = rest / rest.sum() if rest.sum() > 0 else p
        acc = np.cumsum(rest)
        path[b, :len(line)], n_path[b] = line, len(line)
        nxt[b] = np.searchsorted(acc, np.float64(u[b, 0]) * acc[-1], side="right")
    return {"path": path, "n_path": n_path, "next": nxt}


def _exact_commit(s):
    c = s.case
    L, B, W, E = (c[k] for k in ("L", "B", "W", "E"))
    K, V, S = s.K.clone(), s.V.clone(), s.S.double()
    head, count, napp, sink = (t.cpu().numpy().copy() for t in (s.head, s.count, s.n_app, s.n_sink))
    path, n = s.path.cpu().numpy(), s.n_path.cpu().numpy()
    act = None if s.active is None else s.active.cpu().numpy()
    Qa = torch.einsum("lgd,lrd->lgr", s.qg.double(), s.Wq.double())
    for b in range(B):
        if act is not None and not act[b]:
            continue
        for l in range(L):
            ns, h0, n0 = int(sink[l, b]), int(head[l, b]), int(count[l, b])
            cap = W - ns
            held, events = _sequential(n0, cap, min(E, cap), [int(i) for i in path[b, :n[b]]])
            for gone in events:
                olds = [ns + (h0 + o) % cap for kind, o in gone if kind == "old"]
                news = [o for kind, o in gone if kind == "new"]
                k = torch.cat([s.K[l, b][:, olds].transpose(0, 1), s.k[l, b, news]]).double().flatten(1)
                v = torch.cat([s.V[l, b][:, olds].transpose(0, 1), s.v[l, b, news]]).double().flatten(1)
                t = S[l, b] + (Qa[l] @ (k @ s.Wk[l].double().T).T) @ (v @ s.Wv[l].double().T)
                S[l, b] = t / t.norm(dim=-1, keepdim=True).clamp(min=1e-12)
            first = n0 + int(n[b]) - len(held)                       # the oldest token still held, by arrival
            for o, (kind, i) in enumerate(held):
                if kind == "new":
                    at = ns + (h0 + first + o) % cap
                    K[l, b, :, at], V[l, b, :, at] = s.k[l, b, i], s.v[l, b, i]
            head[l, b], count[l, b], napp[l, b] = (h0 + first) % cap, len(held), napp[l, b] + n[b]
    return {"K": K, "V": V, "S": S, "head": head, "count": count, "n_app": napp}


def exact(case, seed):
    global own
    if case["op"] == "commit" and case["L"] * case["B"] * case["T"] > 16000:
        return None
    mine, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = mine
    return {"tree": _exact_tree, "verify": _exact_verify, "commit": _exact_commit}[case["op"]](s)
