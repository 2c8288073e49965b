"""The calls of a training pass: failures of the host, host threads, streams, refusals on the GPU."""
import threading

import pytest
import torch

import paper_2602_16839_b200 as pt
from paper_2602_16839_b200 import binding as bd

from test_gpu_errors import _BrokenCapture

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _calls(dtype, D, seed=0):
    """(call, its outputs) of every entry point, on inputs of their own."""
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    n, Hq, Hkv, V = 300, 4, 2, 777
    rnd = lambda *s: torch.randn(*s, device=DEV, generator=gen).to(dt)         # noqa: E731
    f = lambda *s: torch.zeros(*s, device=DEV)                                 # noqa: E731
    q, k, v, g = rnd(n, Hq, D), rnd(n, Hkv, D), rnd(n, Hkv, D), rnd(n, Hq, D)
    cu = torch.tensor([0, 130, 300], dtype=torch.int32, device=DEV)
    pos, freq, w = torch.arange(n, device=DEV, dtype=torch.int32), torch.rand(D // 2, device=DEV, generator=gen), rnd(D)
    z, tok, adv = rnd(n, V), torch.randint(0, V, (n,), device=DEV, generator=gen, dtype=torch.int32), torch.randn(n, device=DEV, generator=gen)
    out, lse = torch.zeros_like(q), f(n, Hq)
    pt.seq_attn(q, k, v, cu, out, lse_out=lse)
    o2, l2, dq, dk, dv = torch.zeros_like(q), f(n, Hq), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(k)
    qo, ko, gq, gk, wq, wk = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(q), torch.zeros_like(k), f(D), f(D)
    lp, lp2, tl, loss, dz = f(n), f(n), f(n), f(1), torch.zeros_like(z)
    ws = torch.zeros(pt.seq_attn_workspace_bytes(n, Hq), dtype=torch.uint8, device=DEV)
    wr = torch.zeros(pt.head_norm_rope_workspace_bytes(D), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    return [
        (lambda: pt.seq_attn(q, k, v, cu, o2, lse_out=l2), (o2, l2)),
        (lambda: pt.seq_attn_backward(q, k, v, out, lse, g, cu, dq, dk, dv, ws, window=100, evict_chunk=7), (dq, dk, dv)),
        (lambda: pt.head_norm_rope(q, k, pos, freq, qo, ko, q_weight=w, k_weight=w), (qo, ko)),
        (lambda: pt.head_norm_rope_backward(q, k, g, v, pos, freq, gq, gk, q_weight=w, k_weight=w, dq_weight=wq, dk_weight=wk, workspace=wr),
         (gq, gk, wq, wk)),
        (lambda: pt.policy_loss(z, tok, adv, lp, tl, loss, dz), (lp, tl, loss, dz)),
        (lambda: pt.token_logp(z, tok, lp2), (lp2,)),
    ]


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp32", 64), ("bf16", 256)])
def test_a_failed_call_is_reported_once(dtype, D):
    ref, calls = _calls(dtype, D), _calls(dtype, D)
    for call, _ in ref:
        call()
    for i, (call, outs) in enumerate(calls):
        for after in (call, calls[(i + 1) % len(calls)][0]):
            with _BrokenCapture():
                with pytest.raises(pt.PtencError) as e:
                    call()
            assert e.value.code == bd.PTENC_ECUDA
            after()
    torch.cuda.synchronize()
    for (_, a), (_, b) in zip(ref, calls):
        assert all(torch.equal(x, y) for x, y in zip(a, b)) and all(bool(x.abs().max() > 0) for x in a)


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 96), ("fp32", 128)])
def test_new_threads_at_once_get_the_same_bits(dtype, D):
    """Each entry point as the first thing a host thread does with CUDA, eight threads together, a stream each."""
    ref = _calls(dtype, D)
    for call, _ in ref:
        call()
    sets, failures = [_calls(dtype, D) for _ in range(8)], []
    torch.cuda.synchronize()
    start = threading.Barrier(8)

    def run(calls, first):
        try:
            start.wait()
            with torch.cuda.stream(torch.cuda.Stream()):
                for i in range(len(calls)):
                    calls[(first + i) % len(calls)][0]()
        except Exception as e:                                       # noqa: BLE001
            failures.append(e)

    threads = [threading.Thread(target=run, args=(c, i)) for i, c in enumerate(sets)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failures, failures[0]
    for calls in sets:
        for (_, a), (_, b) in zip(ref, calls):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_refusals_on_the_device():
    """What only a GPU tensor can show: overlapping strides, misaligned rows, workspaces that are too small."""
    b16 = dict(dtype=torch.bfloat16, device=DEV)
    base = torch.zeros(64 * 4 * 64 + 64, **b16)
    q, k = base[:64 * 4 * 64].view(64, 4, 64), torch.zeros(64, 2, 64, **b16)
    cu, out = torch.tensor([0, 64], dtype=torch.int32, device=DEV), torch.zeros(64, 4, 64, **b16)

    def refused(code, call, *args, **kw):
        with pytest.raises(pt.PtencError) as e:
            call(*args, **kw)
        assert e.value.code == getattr(bd, "PTENC_" + code)

    refused("EALIGN", pt.seq_attn, base[4:4 + 64 * 4 * 64].view(64, 4, 64), k, k, cu, out)
    refused("EALIGN", pt.seq_attn, torch.zeros(64, 260, **b16)[:, :256].view(64, 4, 64), k, k, cu, out)
    refused("ESHAPE", pt.seq_attn, base.as_strided((64, 4, 64), (128, 64, 1)), k, k, cu, out)         # tokens overlap
    refused("EINVAL", pt.seq_attn, q, k, k, cu, out, window=-1)
    refused("EINVAL", pt.seq_attn, q, k, k, cu, out, window=4, evict_chunk=5)
    refused("EINVAL", pt.seq_attn, q, k, k, cu, out, scale=-1.0)
    refused("EINVAL", pt.seq_attn, q, k, k, cu.cpu(), out)
    refused("ESHAPE", pt.seq_attn, torch.zeros(64, 3, 64, **b16), k, k, cu, torch.zeros(64, 3, 64, **b16))
    lse, ws = torch.zeros(64, 4, device=DEV), torch.zeros(pt.seq_attn_workspace_bytes(64, 4) - 4, dtype=torch.uint8, device=DEV)
    refused("EWORKSPACE", pt.seq_attn_backward, q, k, k, out, lse, out, cu, torch.zeros_like(out), torch.zeros_like(k), torch.zeros_like(k), ws)
    pos, freq, w = torch.zeros(64, dtype=torch.int32, device=DEV), torch.zeros(32, device=DEV), torch.zeros(64, **b16)
    dw = torch.zeros(64, device=DEV)
    refused("EINVAL", pt.head_norm_rope_backward, q, k, out, k, pos, freq, q, k, q_weight=w, k_weight=w, dq_weight=dw, workspace=ws)
    refused("EINVAL", pt.head_norm_rope_backward, q, k, out, k, pos, freq, q, k, q_weight=w, k_weight=w, dq_weight=dw, dk_weight=dw)
    z, n1 = torch.zeros(64, 100, **b16), torch.zeros(64, device=DEV)
    refused("EALIGN", pt.policy_loss, torch.zeros(6404, **b16)[4:].view(64, 100), pos, n1, n1)
    refused("EINVAL", pt.policy_loss, z, pos, n1, n1, loss=torch.zeros(1, device=DEV))
    refused("EINVAL", pt.policy_loss, z, pos, n1, n1, temperature=0.0)
    refused("EINVAL", pt.policy_loss, z, pos, None, n1, old_logp=n1)
    torch.cuda.synchronize()
    assert not base.any()
