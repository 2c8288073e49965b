"""The policy loss of tokens that the policy is nearly sure of."""
import math

import pytest
import torch

import paper_2602_16839_b200 as pt
from oracle import train_oracle as to

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [2, 9, 1000, 65537, 300001, 500009])
def test_gradient_of_a_token_that_is_nearly_certain(V, dtype):
    """Its logit's gradient is as exact, relatively, as the others': it is the sum of theirs, far below the weights' own rounding."""
    dt, n = TYPES[dtype], 8
    gen = torch.Generator(device=DEV).manual_seed(V)
    z = torch.randn(n, V, device=DEV, generator=gen)
    tok = torch.randint(0, V, (n,), device=DEV, generator=gen, dtype=torch.int32)
    tok[0], tok[1] = 0, V - 1
    z[torch.arange(n, device=DEV), tok.long()] = 3 + torch.tensor([8, 14, 20, 30, 40, 60, 75, 8.0], device=DEV)
    z = z.to(dt)
    adv = torch.randn(n, device=DEV, generator=gen)
    lp, dz = torch.empty(n, device=DEV), torch.empty_like(z)
    pt.policy_loss(z, tok, adv, lp, dlogits=dz)
    ref = to.policy_loss(z, tok, adv)
    # weights are off by the rounding of their exponents, below 2^7 (2^-17 and their own steps), the sum by sqrt(V) U; half a step of the
    # result, which below 2^-126 is absolute
    rel = to.half_step(dt) + 2.0 ** -16 + (math.sqrt(V) + 40) * to.U
    g = ref["dlogits"]
    # 1 - softmax loses what lies below 2^-53 in 64 bits too: the token's own gradient as the sum of the others'
    rows, own = torch.arange(n, device=DEV), tok.long()
    g[rows, own] = 0.0
    g[rows, own] = -g.sum(-1)
    err = (dz.double() - g).abs()
    assert (err <= rel * g.abs() + 2.0 ** -126).all(), float((err / (rel * g.abs() + 2.0 ** -126)).max())
    assert (dz[rows[:4], own[:4]] != 0).all()
    got = dz.clone()
    pt.policy_loss(z, tok, adv, lp, dlogits=z)                      # in place
    assert torch.equal(z, got)
