"""Calls from host threads other than the one that made the cache, and from several at once."""
import os
import subprocess
import sys
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


# First calls, made at the same moment by native threads that start together (Python's own take turns at the interpreter's lock).
NATIVE = r"""
#include <atomic>
#include <cstdint>
#include <thread>
#include <vector>
using Word = uint64_t;
// Calls fn with twelve integer arguments from each of n threads at once.
extern "C" void at_once(int n, void* fn, const Word* args, int* rc) {
  auto f = reinterpret_cast<int (*)(Word, Word, Word, Word, Word, Word, Word, Word, Word, Word, Word, Word)>(fn);
  std::atomic<int> here{0};
  std::vector<std::thread> threads;
  for (int i = 0; i < n; ++i)
    threads.emplace_back([&, i] {
      const Word* a = args + 12 * i;
      here.fetch_add(1);
      while (here.load() < n) {}
      rc[i] = f(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10], a[11]);
    });
  for (auto& t : threads) t.join();
}
"""

SCRIPT = r"""
import ctypes, sys
import torch
import paper_2602_16839_b200 as pt
from paper_2602_16839_b200 import binding as bd

native = ctypes.CDLL(sys.argv[1])
N, T, B = 8, 4, 2
i32 = dict(dtype=torch.int32, device="cuda")


def run(cfg):
    caches = [pt.Cache(pt.make_config(n_layers=1, batch=B, window=6, n_global=32, **cfg)) for _ in range(N + 1)]
    c = caches[0].cfg
    gen = torch.Generator(device="cuda").manual_seed(1)
    rows = lambda h: torch.randn(1, B, T, h, c.head_dim, generator=gen, device="cuda").to(caches[0].torch_dtype)
    q, k, v = rows(c.n_q_heads), rows(c.n_kv_heads), rows(c.n_kv_heads)
    parent, path = torch.tensor([[-1, 0, 1, 2]] * B, **i32), torch.tensor([[0, 1, 2, 3]] * B, **i32)
    n = torch.full((B,), T, **i32)
    outs = [torch.zeros_like(q) for _ in caches]
    streams = [torch.cuda.Stream().cuda_stream for _ in caches]
    torch.cuda.synchronize()

    def together(fn, args):
        words = (ctypes.c_uint64 * (12 * N))(*[x for i in range(N) for x in (list(args(i)) + [0] * 12)[:12]])
        rc = (ctypes.c_int * N)()
        native.at_once(N, ctypes.cast(fn, ctypes.c_void_p), words, rc)
        torch.cuda.synchronize()
        assert list(rc) == [0] * N, (cfg, list(rc))

    handle = lambda i: caches[i]._h.value if hasattr(caches[i]._h, "value") else caches[i]._h
    for _ in range(2):                                        # the second commit evicts
        together(bd.lib.ptenc_tree_attn, lambda i: (handle(i), 0, q.data_ptr(), k.data_ptr(), v.data_ptr(), parent.data_ptr(), 0, T, 0,
                                                    outs[i].data_ptr(), 0, streams[i]))
        together(bd.lib.ptenc_commit_path, lambda i: (handle(i), 0, k.data_ptr(), v.data_ptr(), T, path.data_ptr(), n.data_ptr(), 0,
                                                      0, streams[i]))
        caches[N].tree_attn(0, q[0], k[0], v[0], parent, outs[N][0])
        caches[N].commit_path(0, k[0], v[0], path, n)
        torch.cuda.synchronize()
        for i in range(N):
            assert torch.equal(outs[i], outs[N]) and float(outs[i].float().abs().max()) > 0
            assert all(torch.equal(x, y) for x, y in zip(caches[i].get_ring(0), caches[N].get_ring(0)))
            assert torch.equal(caches[i].get_state(0), caches[N].get_state(0)) and caches[i].status() == 0


for cfg in (dict(dtype="fp32", head_dim=64, n_q_heads=4, n_kv_heads=2, rank=32),
            dict(dtype="fp32", head_dim=128, n_q_heads=32, n_kv_heads=32, rank=128),
            dict(dtype="fp32", head_dim=256, n_q_heads=2, n_kv_heads=2, rank=128),
            dict(dtype="bf16", head_dim=32, n_q_heads=4, n_kv_heads=2, rank=64),
            dict(dtype="bf16", head_dim=128, n_q_heads=4, n_kv_heads=2, rank=32),
            dict(dtype="bf16", head_dim=96, n_q_heads=4, n_kv_heads=2, rank=128),
            dict(dtype="bf16", head_dim=256, n_q_heads=8, n_kv_heads=8, rank=128, normalize_mode=1)):
    run(cfg)
print("fine")
"""


def test_first_calls_from_many_threads(tmp_path):
    """A thread per handle, in a process that has launched none of these kernels before: every call succeeds and gives what the
    same call gives alone."""
    (tmp_path / "at_once.cpp").write_text(NATIVE)
    so = str(tmp_path / "at_once.so")
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-pthread", str(tmp_path / "at_once.cpp"), "-o", so])
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    for _ in range(3):
        r = subprocess.run([sys.executable, "-c", SCRIPT, so], cwd=root, capture_output=True, text=True, timeout=300)
        assert r.returncode == 0 and r.stdout.strip() == "fine", r.stdout + r.stderr
