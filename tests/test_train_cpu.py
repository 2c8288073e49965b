"""The operators of a training pass without a GPU: their oracle against other definitions, and every refusal of the entry points."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2602_16839_b200 as pt
from oracle import train_oracle as to
from oracle.ptenc_oracle import OracleCache
from paper_2602_16839_b200 import binding as bd


# ------------------------------------------------------------------------------------------------------ oracle pins
@pytest.mark.parametrize("inter", [False, True])
def test_rotation_is_a_complex_product_and_its_gradient_the_transpose(inter):
    g = torch.Generator().manual_seed(1)
    x = torch.randn(5, 3, 12, dtype=torch.float64, generator=g, requires_grad=True)
    w = torch.randn(12, dtype=torch.float64, generator=g, requires_grad=True)
    pos, freq = torch.tensor([0, 1, 7, 1000, -3]), torch.tensor([1.0, 0.3, 0.01, 0.002])
    y, _ = to.head_norm_rope(x, w, pos, freq, 1e-3, inter)
    n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-3) * w
    a, b = (n[..., 0:8:2], n[..., 1:8:2]) if inter else (n[..., :4], n[..., 4:8])
    z = torch.complex(a, b) * torch.exp(1j * pos[:, None].double() * freq.double())[:, None]
    c, d = (y[..., 0:8:2], y[..., 1:8:2]) if inter else (y[..., :4], y[..., 4:8])
    assert torch.allclose(z.real, c) and torch.allclose(z.imag, d) and torch.allclose(y[..., 8:], n[..., 8:])
    up = torch.randn(5, 3, 12, dtype=torch.float64, generator=g)
    gx, gw = torch.autograd.grad(y, (x, w), up)
    dx, _, dw, _ = to.head_norm_rope_backward(x.detach(), w.detach(), up, pos, freq, 1e-3, inter)
    assert torch.allclose(gx, dx) and torch.allclose(gw, dw)


@pytest.mark.parametrize("W,E,n0", [(7, 1, 0), (7, 3, 2), (5, 5, 4), (1, 1, 0), (9, 2, 8), (6, 4, 0), (40, 3, 5)])
def test_a_token_sees_what_the_cache_holds(W, E, n0):
    """The mask against the library's closed form, and the attention against decoding token by token."""
    rng, T = np.random.default_rng(0), 23
    q, k, v = (rng.standard_normal((T, h, 8)) for h in (4, 2, 2))
    c = OracleCache(n_layers=1, batch=1, n_q_heads=4, n_kv_heads=2, head_dim=8, window=W, evict_chunk=E, encode_enabled=0)
    if n0:
        c.prefill(0, k[None, :n0], v[None, :n0], [n0])
    r = to.seq_attn(*(torch.from_numpy(x) for x in (q, k, v)), [T], W, E, [n0])
    mask = to.seen(T, W, E, n0)
    cap, e = W - n0, min(E, W - n0)
    for i in range(n0, T):
        c.append_evict(0, k[None, i], v[None, i])
        o, s = c.decode_attn(0, q[None, i])
        assert np.allclose(o[0], r["out"][i].numpy()) and np.allclose(s[0], r["lse"][i].numpy())
        gone = e * max(0, -(-(i - n0 + 1 - cap) // e))
        assert [j for j in range(T) if mask[i, j]] == list(range(n0)) + list(range(n0 + gone, i + 1))
    assert torch.equal(mask[:n0, :n0], torch.ones(n0, n0, dtype=torch.bool).tril()) and not mask[:n0, n0:].any()


def test_attention_gradients_are_those_of_automatic_differentiation():
    g = torch.Generator().manual_seed(2)
    lens = [5, 0, 1, 9]
    q, k, v = (torch.randn(15, h, 8, dtype=torch.float64, generator=g, requires_grad=True) for h in (4, 2, 2))
    up = torch.randn(15, 4, 8, dtype=torch.float64, generator=g)
    r = to.seq_attn(q.detach(), k.detach(), v.detach(), lens, 4, 2, [1, 0, 3, 2], dout=up)
    outs, at = [], 0
    for b, n in enumerate(lens):
        m = to.seen(n, 4, 2, [1, 0, 3, 2][b])
        rows = slice(at, at + n)
        at += n
        if n:
            kk, vv = (t[rows].repeat_interleave(2, 1).transpose(0, 1) for t in (k, v))
            s = (q[rows].transpose(0, 1) @ kk.transpose(1, 2)) / math.sqrt(8)
            outs.append((torch.softmax(s.masked_fill(~m, -math.inf), -1) @ vv).transpose(0, 1))
    o = torch.cat(outs)
    assert torch.allclose(o, r["out"])
    for a, b in zip(torch.autograd.grad(o, (q, k, v), up), (r["dq"], r["dk"], r["dv"])):
        assert torch.allclose(a, b)


def test_policy_loss_gradient_is_that_of_automatic_differentiation_and_of_differences():
    g = torch.Generator().manual_seed(3)
    n, V = 40, 9
    z = torch.randn(n, V, dtype=torch.float64, generator=g, requires_grad=True)
    tok = torch.randint(0, V, (n,), generator=g)
    old, ref, adv, w = (torch.randn(n, dtype=torch.float64, generator=g) for _ in range(4))
    lp0 = torch.log_softmax(z.detach() / 0.7, -1).gather(1, tok[:, None])[:, 0]
    old, ref, w = lp0 + 0.4 * old, lp0 + 0.5 * ref, w.abs()
    w[3] = 0
    opt = dict(old=old, ref=ref, weight=w, temperature=0.7, clip_low=0.2, clip_high=0.3, kl_coef=0.2)
    f = lambda x: to.policy_loss(x, tok, adv, **opt)                 # noqa: E731
    r = f(z.detach())
    lp = torch.log_softmax(z / 0.7, -1).gather(1, tok[:, None])[:, 0]
    ratio = torch.exp(lp - old)
    t = -torch.min(ratio * adv, torch.clamp(ratio, 0.8, 1.3) * adv) + 0.2 * (torch.exp(ref - lp) - (ref - lp) - 1)
    assert torch.allclose(t * (w != 0), r["token_loss"]) and torch.allclose((t * w).sum(), r["loss"])
    assert torch.allclose(torch.autograd.grad((t * w).sum(), z)[0], r["dlogits"])
    for i, x in ((0, 0), (7, 3), (3, 1)):
        d = torch.zeros(n, V, dtype=torch.float64)
        d[i, x] = 1e-5
        slope = (f(z.detach() + d)["loss"] - f(z.detach() - d)["loss"]) / 2e-5
        assert abs(float(slope - r["dlogits"][i, x])) < 1e-8


# ------------------------------------------------------------------------------------------------------ refusals
P = 4096                                                            # an aligned address that is never read


def _rope(**over):
    a = dict(dtype=1, Hq=4, Hkv=2, D=64, rot=64, inter=0, eps=1e-6, q=P, qs=256, k=P, ks=128, wq=P, wk=P, pos=P, f=P, n=5, qo=2 * P, qos=256,
             ko=2 * P, kos=128)
    a.update(over)
    cfg = bd.RopeConfig(a["dtype"], a["Hq"], a["Hkv"], a["D"], a["rot"], a["inter"], a["eps"])
    return pt.lib.ptenc_head_norm_rope(None if a.get("nocfg") else ctypes.byref(cfg), a["q"], a["qs"], a["k"], a["ks"], a["wq"], a["wk"],
                                       a["pos"], a["f"], a["n"], a["qo"], a["qos"], a["ko"], a["kos"], None)


def _rope_bwd(**over):
    a = dict(dtype=1, Hq=4, Hkv=2, D=64, rot=64, inter=0, eps=1e-6, q=P, qs=256, k=P, ks=128, wq=P, wk=P, pos=P, f=P, n=5, gq=P, gqs=256,
             gk=P, gks=128, dq=2 * P, dqs=256, dk=2 * P, dks=128, dwq=P, dwk=P, ws=P, size=1 << 24)
    a.update(over)
    cfg = bd.RopeConfig(a["dtype"], a["Hq"], a["Hkv"], a["D"], a["rot"], a["inter"], a["eps"])
    return pt.lib.ptenc_head_norm_rope_backward(
        None if a.get("nocfg") else ctypes.byref(cfg), a["q"], a["qs"], a["k"], a["ks"], a["wq"], a["wk"], a["pos"], a["f"], a["n"], a["gq"], a["gqs"],
        a["gk"], a["gks"], a["dq"], a["dqs"], a["dk"], a["dks"], a["dwq"], a["dwk"], a["ws"], a["size"], None)


BOTH = [
    (dict(nocfg=True), "EINVAL"), (dict(n=-1), "EINVAL"), (dict(dtype=2), "EINVAL"), (dict(Hq=0), "EINVAL"), (dict(Hkv=0), "EINVAL"),
    (dict(Hq=3), "ESHAPE"), (dict(D=12), "ESHAPE"), (dict(D=264, rot=0), "ESHAPE"), (dict(rot=63), "ESHAPE"), (dict(rot=66), "ESHAPE"),
    (dict(rot=-2), "ESHAPE"), (dict(inter=2), "EINVAL"), (dict(eps=-1.0), "EINVAL"), (dict(eps=math.nan), "EINVAL"), (dict(eps=math.inf), "EINVAL"),
    (dict(n=1 << 31), "ESHAPE"), (dict(q=None), "EINVAL"), (dict(k=None), "EINVAL"), (dict(pos=None), "EINVAL"), (dict(f=None), "EINVAL"),
    (dict(q=P + 8), "EALIGN"), (dict(wk=P + 8), "EALIGN"), (dict(pos=P + 2), "EALIGN"), (dict(f=P + 1), "EALIGN"), (dict(qs=255), "ESHAPE"),
    (dict(qs=260), "EALIGN"), (dict(ks=127), "ESHAPE"), (dict(Hq=32768, Hkv=1), "ESHAPE")]


@pytest.mark.parametrize("over,code", BOTH + [
    (dict(qo=None), "EINVAL"), (dict(ko=None), "EINVAL"), (dict(qo=P + 8), "EALIGN"), (dict(qos=128), "ESHAPE"), (dict(kos=132), "EALIGN"),
    (dict(qo=P, qos=512), "EINVAL"), (dict(ko=P, kos=256), "EINVAL")])
def test_head_norm_rope_refuses(over, code):
    assert _rope(**over) == getattr(bd, "PTENC_" + code)


@pytest.mark.parametrize("over,code", BOTH + [
    (dict(gq=None), "EINVAL"), (dict(gk=None), "EINVAL"), (dict(dq=None), "EINVAL"), (dict(dk=None), "EINVAL"), (dict(dwq=None), "EINVAL"),
    (dict(dwk=None), "EINVAL"), (dict(wq=None), "EINVAL"), (dict(wk=None), "EINVAL"), (dict(ws=None), "EINVAL"), (dict(size=100), "EWORKSPACE"),
    (dict(ws=P + 4), "EALIGN"), (dict(dwq=P + 4), "EALIGN"), (dict(dq=P + 8), "EALIGN"), (dict(dqs=128), "ESHAPE"), (dict(gks=132), "EALIGN"),
    (dict(dq=P, dqs=512), "EINVAL"), (dict(dk=P, dks=256), "EINVAL")])
def test_head_norm_rope_backward_refuses(over, code):
    assert _rope_bwd(**over) == getattr(bd, "PTENC_" + code)


def _seq(back=False, **over):
    a = dict(dtype=1, Hq=4, Hkv=2, D=64, W=0, E=1, scale=0.0, q=P, qs=256, k=P, ks=128, v=P, vs=128, out=P, lse=P, g=P, cu=P, pin=None, B=2, n=10,
             dq=P, dqs=256, dk=P, dks=128, dv=P, dvs=128, ws=P, size=320)
    a.update(over)
    cfg = bd.SeqConfig(a["dtype"], a["Hq"], a["Hkv"], a["D"], a["W"], a["E"], a["scale"])
    cfg = None if a.get("nocfg") else ctypes.byref(cfg)
    if not back:
        return pt.lib.ptenc_seq_attn(cfg, a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["cu"], a["pin"], a["B"], a["n"], a["out"], a["lse"], None)
    return pt.lib.ptenc_seq_attn_backward(cfg, a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["out"], a["lse"], a["g"], a["cu"], a["pin"], a["B"],
                                          a["n"], a["dq"], a["dqs"], a["dk"], a["dks"], a["dv"], a["dvs"], a["ws"], a["size"], None)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("over,code", [
    (dict(nocfg=True), "EINVAL"), (dict(B=-1), "EINVAL"), (dict(n=-1), "EINVAL"), (dict(dtype=9), "EINVAL"), (dict(W=-1), "EINVAL"),
    (dict(W=4, E=0), "EINVAL"), (dict(W=4, E=5), "EINVAL"), (dict(scale=-1.0), "EINVAL"), (dict(scale=math.nan), "EINVAL"),
    (dict(scale=math.inf), "EINVAL"), (dict(Hq=5), "ESHAPE"), (dict(D=20), "ESHAPE"), (dict(D=512), "ESHAPE"), (dict(n=1 << 31), "ESHAPE"),
    (dict(B=1 << 25), "ESHAPE"), (dict(q=None), "EINVAL"), (dict(k=None), "EINVAL"), (dict(v=None), "EINVAL"), (dict(cu=None), "EINVAL"),
    (dict(out=None), "EINVAL"), (dict(q=P + 8), "EALIGN"), (dict(v=P + 2), "EALIGN"), (dict(out=P + 4), "EALIGN"), (dict(cu=P + 2), "EALIGN"),
    (dict(pin=P + 1), "EALIGN"), (dict(lse=P + 2), "EALIGN"), (dict(qs=252), "ESHAPE"), (dict(ks=132), "EALIGN"), (dict(vs=0), "ESHAPE")])
def test_seq_attn_refuses(over, code, back):
    assert _seq(back, **over) == getattr(bd, "PTENC_" + code)


@pytest.mark.parametrize("back", [False, True])
def test_seq_attn_refuses_more_tiles_than_a_launch_has(back):
    many = dict(Hq=128, Hkv=128, qs=8192, ks=8192, vs=8192, dqs=8192, dks=8192, dvs=8192, size=10240)
    assert _seq(back, B=1 << 24, **many) == bd.PTENC_ESHAPE
    assert _seq(back, B=(1 << 24) - 1, n=1 << 30, **many) == bd.PTENC_ESHAPE


@pytest.mark.parametrize("over,code", [
    (dict(lse=None), "EINVAL"), (dict(g=None), "EINVAL"), (dict(dq=None), "EINVAL"), (dict(dk=None), "EINVAL"), (dict(dv=None), "EINVAL"),
    (dict(ws=None), "EINVAL"), (dict(size=319), "EWORKSPACE"), (dict(ws=P + 8), "EALIGN"), (dict(dq=P + 8), "EALIGN"), (dict(g=P + 2), "EALIGN"),
    (dict(dqs=128), "ESHAPE"), (dict(dks=132), "EALIGN"), (dict(dvs=100), "ESHAPE")])
def test_seq_attn_backward_refuses(over, code):
    assert _seq(True, **over) == getattr(bd, "PTENC_" + code)


def _loss(**over):
    a = dict(dtype=1, V=100, T=1.0, lo=0.2, hi=0.2, kl=0.1, z=P, zs=100, tok=P, old=P, ref=P, adv=P, w=P, n=4, lp=P, tl=P, tk=P, loss=P, dz=2 * P, dzs=100)
    a.update(over)
    cfg = bd.PolicyConfig(a["dtype"], a["V"], a["T"], a["lo"], a["hi"], a["kl"])
    return pt.lib.ptenc_policy_loss(None if a.get("nocfg") else ctypes.byref(cfg), a["z"], a["zs"], a["tok"], a["old"], a["ref"], a["adv"], a["w"], a["n"],
                                    a["lp"], a["tl"], a["tk"], a["loss"], a["dz"], a["dzs"], None)


@pytest.mark.parametrize("over,code", [
    (dict(nocfg=True), "EINVAL"), (dict(n=-1), "EINVAL"), (dict(dtype=3), "EINVAL"), (dict(V=0), "EINVAL"), (dict(T=0.0), "EINVAL"),
    (dict(T=-1.0), "EINVAL"), (dict(T=math.nan), "EINVAL"), (dict(T=math.inf), "EINVAL"), (dict(lo=-0.1), "EINVAL"), (dict(hi=math.nan), "EINVAL"),
    (dict(kl=-1.0), "EINVAL"), (dict(V=(1 << 28) + 1, zs=1 << 29), "ESHAPE"), (dict(n=1 << 31), "ESHAPE"), (dict(adv=None), "EINVAL"),
    (dict(tl=None), "EINVAL"), (dict(z=None), "EINVAL"), (dict(tok=None), "EINVAL"), (dict(lp=None), "EINVAL"), (dict(z=P + 2), "EALIGN"),
    (dict(dz=P + 8), "EALIGN"), (dict(w=P + 2), "EALIGN"), (dict(zs=99), "ESHAPE"), (dict(dzs=99), "ESHAPE"), (dict(dz=P, dzs=200), "EINVAL")])
def test_policy_loss_refuses(over, code):
    assert _loss(**over) == getattr(bd, "PTENC_" + code)


def test_nothing_to_do_is_not_an_error():
    assert _seq(n=0) == 0 and _seq(B=0) == 0 and _seq(True, n=0) == 0 and _rope(n=0) == 0
    assert _loss(n=0, loss=None, tl=None) == 0
    assert _rope_bwd(n=0, wq=None, wk=None, dwq=None, dwk=None, ws=None) == 0


def test_workspace_sizes():
    n = ctypes.c_size_t(0)
    assert pt.seq_attn_workspace_bytes(10, 4) == 320 and pt.head_norm_rope_workspace_bytes(128) > 0
    assert pt.lib.ptenc_seq_attn_workspace_bytes(-1, 4, ctypes.byref(n)) == bd.PTENC_EINVAL
    assert pt.lib.ptenc_seq_attn_workspace_bytes(1, 4, None) == bd.PTENC_EINVAL
    assert pt.lib.ptenc_seq_attn_workspace_bytes(1 << 31, 4, ctypes.byref(n)) == bd.PTENC_ESHAPE
    assert pt.lib.ptenc_head_norm_rope_workspace_bytes(12, ctypes.byref(n)) == bd.PTENC_ESHAPE
    assert pt.lib.ptenc_head_norm_rope_workspace_bytes(0, ctypes.byref(n)) == bd.PTENC_EINVAL


def test_the_binding_refuses_what_the_library_cannot_see():
    """Types, shapes and strides, on CPU tensors: the last refusal of a call that is otherwise right is its device."""
    f = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)      # noqa: E731
    q, k, o, p = f(6, 4, 64), f(6, 2, 64), f(6, 4, 64), f(6, 2, 64)
    pos, freq, cu = f(6, dt=torch.int32), f(32, dt=torch.float32), f(3, dt=torch.int32)

    def refused(code, call, *args, **kw):
        with pytest.raises(pt.PtencError) as e:
            call(*args, **kw)
        assert e.value.code == getattr(bd, "PTENC_" + code)

    refused("EINVAL", pt.head_norm_rope, q, k, pos, freq, o, p)                                   # not on a CUDA device
    refused("EINVAL", pt.head_norm_rope, q.half(), k, pos, freq, o, p)
    refused("EINVAL", pt.head_norm_rope, q, k.float(), pos, freq, o, p)
    refused("ESHAPE", pt.head_norm_rope, q, k[:5], pos, freq, o, p)
    refused("ESHAPE", pt.head_norm_rope, q, k, pos, freq, p, p)
    refused("EINVAL", pt.head_norm_rope, q.transpose(1, 2), k, pos, freq, o, p)
    refused("EINVAL", pt.head_norm_rope, q, k, pos.long(), freq, o, p)
    refused("ESHAPE", pt.head_norm_rope, q, k, pos[:3], freq, o, p)
    refused("ESHAPE", pt.head_norm_rope, q, k, pos, freq, o, p, q_weight=f(32))
    refused("EINVAL", pt.head_norm_rope, f(6, 64, 4).transpose(1, 2), k, pos, freq, o, p)
    refused("EINVAL", pt.seq_attn, q, k, k, cu, o)
    refused("EINVAL", pt.seq_attn, q, k, k, cu.long(), o)
    refused("ESHAPE", pt.seq_attn, q, k, k[:, :1], cu, o)
    refused("ESHAPE", pt.seq_attn, q, k, k, cu, o, n_pinned=f(3, dt=torch.int32))
    refused("EINVAL", pt.seq_attn, q, k, k, cu, o, lse_out=f(6, 4))
    refused("EINVAL", pt.seq_attn, q, k, k, cu, f(6, 8, 64)[:, :4])
    refused("ESHAPE", pt.seq_attn_backward, q, k, k, o, f(6, 4, dt=torch.float32), o, cu, q, k, q, f(24, dt=torch.float32))
    z, n1 = f(6, 100, dt=torch.float32), f(6, dt=torch.float32)
    refused("EINVAL", pt.policy_loss, z, pos, n1, n1)
    refused("EINVAL", pt.policy_loss, z.half(), pos, n1, n1)
    refused("EINVAL", pt.policy_loss, z, pos.long(), n1, n1)
    refused("ESHAPE", pt.policy_loss, z, pos, n1[:2], n1)
    refused("EINVAL", pt.policy_loss, z, pos, n1, n1, dlogits=f(100, 6, dt=torch.float32).t())
    refused("EINVAL", pt.policy_loss, z, pos, n1, n1, dlogits=z.bfloat16())
