"""What the training-pass calls hand to the library, without a GPU: the library is a stand-in that keeps the configurations it gets."""
import numpy as np
import pytest
import torch

import paper_2602_16839_b200 as pt
from paper_2602_16839_b200 import binding as bd

from test_train_cpu import _loss, _seq


class _Library:
    def __init__(self):
        self.got = []

    def __getattr__(self, name):
        if name == "ptenc_strerror":
            return pt.lib.ptenc_strerror

        def call(cfg, *args):
            self.got.append({field: getattr(cfg._obj, field) for field, _ in cfg._obj._fields_})
            return bd.PTENC_OK
        return call


@pytest.fixture
def library(monkeypatch):
    fake = _Library()
    monkeypatch.setattr(bd, "lib", fake)
    monkeypatch.setattr(bd, "_device_of", lambda where, t: 0)
    monkeypatch.setattr(bd, "_stream_of", lambda device: 0)
    return fake


def _calls():
    q, k = torch.zeros(6, 4, 64, dtype=torch.bfloat16), torch.zeros(6, 2, 64, dtype=torch.bfloat16)
    cu, pos, freq, w = torch.zeros(3, dtype=torch.int32), torch.zeros(6, dtype=torch.int32), torch.zeros(32), torch.zeros(64, dtype=torch.bfloat16)
    z, f, dw, lse = torch.zeros(6, 9), torch.zeros(6), torch.zeros(64), torch.zeros(6, 4)
    return {
        "rope": lambda **kw: pt.head_norm_rope(q, k, pos, freq, q, k, q_weight=w, k_weight=w, **kw),
        "rope_bwd": lambda **kw: pt.head_norm_rope_backward(q, k, q, k, pos, freq, q, k, q_weight=w, k_weight=w, dq_weight=dw, dk_weight=dw, **kw),
        "attn": lambda **kw: pt.seq_attn(q, k, k, cu, q, **kw),
        "attn_bwd": lambda **kw: pt.seq_attn_backward(q, k, k, q, lse, q, cu, q, k, k, f, **kw),
        "loss": lambda **kw: pt.policy_loss(z, pos, f, f, f, **kw),
        "logp": lambda **kw: pt.token_logp(z, pos, f, **kw),
    }


@pytest.mark.parametrize("call,name", [
    ("rope", "eps"), ("rope_bwd", "eps"), ("attn", "scale"), ("attn_bwd", "scale"), ("loss", "temperature"), ("loss", "clip_low"),
    ("loss", "clip_high"), ("loss", "kl_coef"), ("logp", "temperature")])
@pytest.mark.parametrize("number", [torch.tensor, np.float32, float])
def test_numbers_are_taken_as_they_are_at_the_call(call, name, number, library):
    """A coefficient that is changed in place between two calls, as an annealed one may be."""
    t = number(0.5)
    go = _calls()[call]
    go(**{name: t})
    t *= 0.5
    go(**{name: t})
    assert [c[name] for c in library.got] == [0.5, 0.25]


@pytest.mark.parametrize("call", ["attn", "attn_bwd"])
@pytest.mark.parametrize("name", ["window", "evict_chunk"])
def test_whole_numbers_are_taken_as_they_are_at_the_call(call, name, library):
    go, kw = _calls()[call], dict(window=64, evict_chunk=4)
    t = torch.tensor(8)
    go(**{**kw, name: t})
    t += 3
    go(**{**kw, name: t})
    go(**{**kw, name: np.int64(5)})
    assert [c[name] for c in library.got] == [8, 11, 5]
    with pytest.raises(TypeError):
        go(**{**kw, name: 8.0})


@pytest.mark.parametrize("call", ["attn", "attn_bwd"])
@pytest.mark.parametrize("value", [2 ** 31, 2 ** 32, 2 ** 32 + 5, -2 ** 32 + 5, 2 ** 70])
@pytest.mark.parametrize("name", ["window", "evict_chunk"])
def test_whole_numbers_that_32_bits_do_not_hold_are_refused(call, name, value, library):
    for _ in range(2):
        with pytest.raises(pt.PtencError) as e:
            _calls()[call](**{"window": 64, "evict_chunk": 4, name: value})
        assert e.value.code == bd.PTENC_ESHAPE
    assert library.got == []


def test_vocabularies_and_batches_that_32_bits_do_not_hold_are_refused(library):
    """They would arrive as what 32 bits leave of them.  The tensors have a shape and no memory."""
    meta = dict(device="meta")
    z, n1 = torch.empty(1, 2 ** 32 + 9, dtype=torch.bfloat16, **meta), torch.empty(1, **meta)
    q, k = torch.empty(6, 4, 64, **meta), torch.empty(6, 2, 64, **meta)
    cu, lse, ws = torch.empty(2 ** 32 + 3, dtype=torch.int32, **meta), torch.empty(6, 4, **meta), torch.empty(48, **meta)
    for go in (lambda: pt.token_logp(z, n1.int(), n1), lambda: pt.policy_loss(z, n1.int(), n1, n1, dlogits=torch.empty_like(z)),
               lambda: pt.seq_attn(q, k, k, cu, q), lambda: pt.seq_attn_backward(q, k, k, q, lse, q, cu, q, k, k, ws)):
        with pytest.raises(pt.PtencError) as e:
            go()
        assert e.value.code == bd.PTENC_ESHAPE
    assert library.got == []


@pytest.mark.parametrize("temperature", [1e-45, 1e-39, 1.1e-38])
def test_temperatures_below_the_normal_range_are_refused(temperature):
    """With an inverse that is not finite a row's largest logits would become 0 * inf."""
    assert _loss(T=temperature) == bd.PTENC_EINVAL


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("scale", [2.4e38, 2.9e38])
def test_scales_that_pass_the_range_in_base_2_are_refused(scale, back):
    """A score of zero would become 0 * inf."""
    assert _seq(back, scale=scale) == bd.PTENC_EINVAL
