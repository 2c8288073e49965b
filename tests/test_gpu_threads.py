"""Calls from host threads other than the one that made the cache."""
import threading

import pytest
import torch

import paper_2602_16839_b200 as pt

from _harness import Pair

pytestmark = pytest.mark.gpu


def _in_a_new_thread(call):
    """Runs call() as the first thing that a host thread does with CUDA."""
    failure = []

    def run():
        try:
            call()
        except Exception as e:                                # noqa: BLE001
            failure.append(e)

    t = threading.Thread(target=run)
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert not failure, failure[0]


@pytest.mark.parametrize("D", [64, 128])
def test_a_new_thread_gets_the_same_bits(D):
    """Entry points that have the driver describe tensors for the TMA unit, in a thread that no context is bound to yet: the tree's
    attention takes the same kernel as elsewhere, caller rows and caller rings are not refused."""
    B, T, m = 8, 6, 32
    p = Pair(pt, n_layers=1, batch=B, n_q_heads=8, n_kv_heads=2, head_dim=D, window=150, evict_chunk=16, n_global=32, rank=32, seed=3)
    for t in range(160):
        k, v = p.gen.step_kv(t)
        p.cache.append_evict(-1, k, v)
        p.cache.encode(-1)
    g = p.gen.generic
    q, k, v = (g(70 + i, 0, (1, B, T, h, D), 1.0) for i, h in enumerate((8, 2, 2)))
    parent = torch.tensor([[-1, 0, 0, 1, 3, 2]] * B, dtype=torch.int32, device="cuda")
    outs, lses = [torch.zeros_like(q) for _ in range(2)], [torch.zeros(1, B, T, 8, device="cuda") for _ in range(2)]
    tree = [lambda i=i: p.cache.tree_attn(-1, q, k, v, parent, outs[i], lse_out=lses[i]) for i in range(2)]

    Ke, Ve = (g(80 + i, 0, (1, B, m, 2 * D), 1.0) for i in range(2))
    n_ev = torch.full((1, B), m, dtype=torch.int32, device="cuda")
    state0, states = p.cache.get_state(0).clone(), []

    K, V = (g(90 + i, 0, (1, B, 2, 150, D), 1.0) for i in range(2))
    head, count = (torch.full((1, B), x, dtype=torch.int32, device="cuda") for x in (7, 150))
    rings = [torch.zeros(1, B, 8, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    one = q[:, :, 0].contiguous()
    static = [lambda i=i: pt.attn_rings_static(p.cache.cfg, K, V, head, count, one, rings[i]) for i in range(2)]
    encode = lambda: p.cache.encode(-1, Ke, Ve, n_ev, m)
    snapshot = p.cache.workspace.clone()
    torch.cuda.synchronize()
    for call in (tree[0], static[0], encode):
        call()
    torch.cuda.synchronize()
    states.append(p.cache.get_state(0).clone())
    p.cache.workspace.copy_(snapshot)
    torch.cuda.synchronize()
    for call in (tree[1], static[1], encode):
        _in_a_new_thread(call)
    states.append(p.cache.get_state(0).clone())
    assert torch.equal(outs[0], outs[1]) and torch.equal(lses[0], lses[1]) and float(outs[0].float().abs().max()) > 0
    assert torch.equal(rings[0], rings[1]) and float(rings[0].float().abs().max()) > 0
    assert torch.equal(states[0], states[1]) and not torch.equal(states[0], state0)
    assert p.cache.status() == 0
    p.close()
