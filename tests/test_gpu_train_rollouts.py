"""Attention over rollouts: pinned tokens that are seen by far more than others, and calls of very many sequences."""
import math

import pytest
import torch

import paper_2602_16839_b200 as pt

from test_gpu_train import _attention, _check_attention

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("Hq,Hkv,D", [(2, 2, 128), (3, 1, 128), (6, 2, 64), (7, 1, 96), (1, 1, 40)])
@pytest.mark.parametrize("window,chunk,pinned", [(1, 1, 0), (64, 16, 5), (200, 50, 150), (129, 1, 128)])
def test_prompts_that_long_rollouts_keep(window, chunk, pinned, Hq, Hkv, D, dtype):
    lens = [1500, 0, 40, 901, 1]
    _check_attention(lens, Hq, Hkv, D, dtype, window, chunk, [pinned, 0, 0, max(0, pinned - 3), pinned], tail=5, seed=D + window)


@pytest.mark.parametrize("which", ["q", "k", "v", "dout"])
@pytest.mark.parametrize("at", [3, 1100])
def test_a_prompt_that_is_not_a_number(which, at):
    """A token of the prompt, or a late one: what sees it is not finite, the rest keeps its bits."""
    n, window, chunk, pinned = 1300, 64, 16, 20
    (q, k, v, dout), go = _attention([n], 4, 2, 64, torch.bfloat16, 3, window, chunk, [pinned])
    clean = go()
    {"q": q, "k": k, "v": v, "dout": dout}[which][at] = math.nan
    got = go()
    from oracle import train_oracle as to
    seen = to.seen(n, window, chunk, pinned, DEV)
    rows = seen[:, at] if which in ("k", "v") else torch.arange(n, device=DEV) == at
    toks = seen[rows].any(0)
    for name, a, b, hit in (("dq", clean[2], got[2], rows), ("dk", clean[3], got[3], toks), ("dv", clean[4], got[4], toks)):
        assert torch.equal(a[~hit], b[~hit]), name
    assert not torch.isfinite(got[3][toks].float()).flatten(1).all(1).any()
    assert not torch.isfinite(got[2][rows].float()).flatten(1).all(1).any()


@pytest.mark.parametrize("D", [64, 128])
def test_calls_behind_one_another_and_replayed(D):
    """What follows a backward call sees all of its gradients, and every call has the same bits: eager, from a graph, and with the
    gradients consumed at once by the next kernel."""
    lens, Hq, Hkv, window, chunk = [1900, 300, 700], 6, 2, 100, 25
    (q, k, v, dout), go = _attention(lens, Hq, Hkv, D, torch.bfloat16, 8, window, chunk, [90, 40, 99])
    out, lse, dq, dk, dv = go()
    n = sum(lens)
    cu = torch.tensor([0, 1900, 2200, 2900], dtype=torch.int32, device=DEV)
    pin = torch.tensor([90, 40, 99], dtype=torch.int32, device=DEV)
    ws = torch.empty(pt.seq_attn_workspace_bytes(n, Hq), dtype=torch.uint8, device=DEV)
    got = [torch.zeros_like(t) for t in (dq, dk, dv)]
    seen = [torch.zeros_like(t) for t in got]
    pos, freq = torch.zeros(n, dtype=torch.int32, device=DEV), torch.ones(D // 2, device=DEV)

    def call():
        pt.seq_attn_backward(q, k, v, out, lse, dout, cu, *got, ws, n_pinned=pin, window=window, evict_chunk=chunk)
        pt.head_norm_rope(got[0], got[1], pos, freq, seen[0], seen[1])         # turned by nothing: a copy, by one of the library's own
        seen[2].copy_(got[2])
        for t in got:
            t.zero_()

    for _ in range(20):
        call()
        for a, b in zip((dq, dk, dv), seen):
            assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
        call()
    for _ in range(10):
        for t in seen:
            t.zero_()
        graph.replay()
        for a, b in zip((dq, dk, dv), seen):
            assert torch.equal(a, b)


@pytest.mark.parametrize("B", [5000, 1 << 18])
def test_very_many_sequences_most_of_them_empty(B):
    """A few tokens at either end of a long list of empty sequences."""
    lens = [200] + [0] * (B - 3) + [1, 131]
    n, Hq, Hkv, D = sum(lens), 16, 2, 64
    (q, k, v, dout), go = _attention([200, 1, 131], Hq, Hkv, D, torch.bfloat16, 5)
    ref = go()
    cu = torch.full((B + 1,), 200, dtype=torch.int32, device=DEV)
    cu[0], cu[-2], cu[-1] = 0, 201, 332
    out, lse = torch.empty_like(ref[0]), torch.empty_like(ref[1])
    ws = torch.empty(pt.seq_attn_workspace_bytes(n, Hq), dtype=torch.uint8, device=DEV)
    g = [torch.empty_like(t) for t in ref[2:]]
    pt.seq_attn(q, k, v, cu, out, lse_out=lse)
    pt.seq_attn_backward(q, k, v, out, lse, dout, cu, *g, ws)
    for a, b in zip(ref, [out, lse, *g]):
        assert torch.equal(a, b)
