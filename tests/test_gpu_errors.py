"""A call that fails on the host, and the calls after it."""
import ctypes

import pytest
import torch

import paper_2602_16839_b200 as pt
from paper_2602_16839_b200 import binding as bd

from _harness import Pair

pytestmark = pytest.mark.gpu


class _BrokenCapture:
    """A stream on which launches fail: it is being captured, and the capture has been invalidated by asking the host to wait for
    it.  Nothing of what is called inside runs."""

    def __enter__(self):
        self.rt, self.stream = ctypes.CDLL("libcudart.so.12"), torch.cuda.Stream()
        self.raw = ctypes.c_void_p(self.stream.cuda_stream)
        assert self.rt.cudaStreamBeginCapture(self.raw, 2) == 0
        assert self.rt.cudaStreamSynchronize(self.raw) != 0
        self.on = torch.cuda.stream(self.stream)
        self.on.__enter__()

    def __exit__(self, *what):
        self.on.__exit__(*what)
        graph = ctypes.c_void_p()
        assert self.rt.cudaStreamEndCapture(self.raw, ctypes.byref(graph)) != 0
        self.rt.cudaGetLastError()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp32", 64)])
def test_a_failed_call_is_reported_once(dtype, D):
    """Every entry point that launches: refused with PTENC_ECUDA while launches fail, and fine the next time, with the results of a
    cache on which nothing failed.  A call that reported its predecessor's failure would have run all the same."""
    B, T, V = 3, 4, 50
    kw = dict(n_layers=1, batch=B, n_q_heads=8, n_kv_heads=2, head_dim=D, window=20, evict_chunk=4, dtype=dtype, seed=2, n_global=32, rank=32)
    a, b = Pair(pt, **kw), Pair(pt, **kw)
    for x in (a, b):
        for t in range(22):
            x.cache.append_evict(-1, *x.gen.step_kv(t))
            x.cache.encode(-1)
    g = a.gen.generic
    q, k, v = (g(70 + i, 0, (1, B, T, h, D), 1.0) for i, h in enumerate((8, 2, 2)))
    i32 = dict(dtype=torch.int32, device="cuda")
    parent = torch.tensor([[-1, 0, 0, 1]] * B, **i32)
    probs = torch.softmax(torch.randn(B, T, V, device="cuda"), -1)
    tok, u = torch.zeros(B, T, **i32), torch.full((B, T), 0.5, device="cuda")
    path, n = torch.tensor([[0, 1, 2, 3]] * B, **i32), torch.full((B,), T, **i32)
    outs = {x: dict(tree=torch.zeros_like(q), path=torch.zeros(B, T, **i32), n=torch.zeros(B, **i32), nxt=torch.zeros(B, **i32),
                    one=torch.zeros(1, B, 8, D, dtype=q.dtype, device="cuda")) for x in (a, b)}
    one = [t[:, :, 0].contiguous() for t in (q, k, v)]
    mask = torch.tensor([0, 1, 0], dtype=torch.uint8, device="cuda")
    calls = [
        lambda x: x.cache.tree_attn(-1, q, k, v, parent, outs[x]["tree"]),
        lambda x: pt.verify_tree(probs, None, tok, parent, u, outs[x]["path"], outs[x]["n"], outs[x]["nxt"]),
        lambda x: x.cache.commit_path(-1, k, v, path, n),
        lambda x: x.cache.append_evict(-1, one[1], one[2]),
        lambda x: x.cache.encode(-1),
        lambda x: x.cache.decode_step(-1, *one, outs[x]["one"]),
        lambda x: x.cache.decode_attn(-1, one[0], outs[x]["one"]),
        lambda x: x.cache.reset(mask),
    ]
    torch.cuda.synchronize()
    def fails(call):
        with _BrokenCapture():
            with pytest.raises(pt.PtencError) as e:
                call(a)
        assert e.value.code == bd.PTENC_ECUDA

    for call, other in zip(calls, calls[1:] + calls[:1]):
        for after in (call, other):
            fails(call)
            for x in (a, b):
                after(x)
    torch.cuda.synchronize()
    for l, r in zip(outs[a].values(), outs[b].values()):
        assert torch.equal(l, r)
    assert all(torch.equal(x, y) for x, y in zip(a.cache.get_ring(0), b.cache.get_ring(0)))
    assert torch.equal(a.cache.get_state(0), b.cache.get_state(0))
    assert a.cache.status() == 0 and b.cache.status() == 0
    for x in (a, b):
        x.close()
