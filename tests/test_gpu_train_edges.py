"""The operators of a training pass at the edges of what their calls allow."""
import pytest
import torch

import paper_2602_16839_b200 as pt
from oracle import train_oracle as to

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
