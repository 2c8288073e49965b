"""Speculative step without a GPU: the oracle against brute force and exact laws, and every refusal of the entry points."""
import ctypes
import itertools

import numpy as np
import pytest
import torch

import paper_2602_16839_b200 as pt
from oracle.ptenc_oracle import OracleCache
from oracle import spec_oracle as so
from paper_2602_16839_b200 import binding as bd


# ------------------------------------------------------------------------------------------------------ oracle pins
@pytest.mark.parametrize("W,E,n0,prompt", [(7, 1, 12, 0), (7, 3, 12, 0), (5, 5, 9, 2), (1, 1, 3, 0), (9, 2, 4, 4), (6, 4, 0, 0)])
def test_what_a_node_sees_follows_the_closed_form(W, E, n0, prompt):
    """Token sets from the counting formula (tokens gone after m appends) against appending for real."""
    c = OracleCache(n_layers=1, batch=1, n_q_heads=1, n_kv_heads=1, head_dim=2, window=W, evict_chunk=E, encode_enabled=0)
    if prompt:
        c.prefill(0, np.zeros((1, prompt, 1, 2)), np.zeros((1, prompt, 1, 2)), [prompt])
    for _ in range(n0):
        c.append_evict(0, np.zeros((1, 1, 2)), np.zeros((1, 1, 2)))
    cap, count = W - prompt, len(c.seqs[0][0].live)
    e = min(E, cap)
    first = c.seqs[0][0].n_appended - count
    for m in range(1, 12):
        c.append_evict(0, np.zeros((1, 1, 2)), np.zeros((1, 1, 2)))
        over = max(0, count + m - cap)
        gone = -(-over // e) * e
        assert list(c.seqs[0][0].live) == list(range(first + gone, first + count + m))


def test_tree_of_one_chain_is_sequential_decoding():
    rng = np.random.default_rng(0)
    c = OracleCache(n_layers=1, batch=2, n_q_heads=4, n_kv_heads=2, head_dim=8, window=6, evict_chunk=2, encode_enabled=0)
    for _ in range(7):
        c.append_evict(0, rng.standard_normal((2, 2, 8)), rng.standard_normal((2, 2, 8)))
    T = 5
    q, k, v = (rng.standard_normal((2, T, h, 8)) for h in (4, 2, 2))
    parent = np.tile(np.arange(-1, T - 1), (2, 1))
    out, lse, done = so.tree_attn(c, 0, q, k, v, parent)
    assert done.all()
    for i in range(T):
        c.append_evict(0, k[:, i], v[:, i])
        o, s = c.decode_attn(0, q[:, i])
        assert np.array_equal(o, out[:, i]) and np.array_equal(s, lse[:, i])


@pytest.mark.parametrize("width", [1, 2, 3])
def test_accepted_and_drawn_token_follows_the_target(width):
    """The first token that leaves the root (accepted child or drawn token) has the target's law, whatever the draft's:
    summed exactly over the draws of `width` siblings and integrated over their random numbers (the acceptance of a child
    is decided at one threshold, so the integral is a weighted sum of two cases)."""
    p = np.array([0.5, 0.2, 0.3, 0.0])
    q = np.array([0.1, 0.6, 0.2, 0.1])
    law = np.zeros(4)
    parent = np.array([-1] + [0] * width)

    def walk(tokens, i, r, weight, law):
        if i == width:
            law += weight * r
            return
        x = tokens[i]
        a = min(1.0, r[x] / q[x])
        law[x] += weight * a
        left = np.maximum(r - q, 0)
        if a < 1.0:
            walk(tokens, i + 1, left / left.sum(), weight * (1 - a), law)

    for tokens in itertools.product(range(4), repeat=width):
        walk(tokens, 0, p, np.prod(q[list(tokens)]), law)
    assert np.allclose(law, p, atol=1e-12)
    # the oracle decides exactly there: just below each threshold it accepts, just above it goes on
    rows = np.tile(p, (width + 1, 1)), np.tile(q, (width + 1, 1))
    for tokens in itertools.product(range(4), repeat=width):
        tok = np.array([0, *tokens])
        r, u = p, np.full(width + 1, 0.5)
        for i in range(1, width + 1):
            a = min(1.0, r[tok[i]] / q[tok[i]])
            if a > 1e-9:
                u[i] = a - 1e-9
                line, _, _ = so.verify_tree(*rows, tok, parent, u)
                assert line == [0, i]
            if a >= 1.0:
                break
            u[i] = a + 1e-9
            line, _, _ = so.verify_tree(*rows, tok, parent, u)
            assert i not in line
            left = np.maximum(r - q, 0)
            r = left / left.sum()


def test_draw_takes_the_first_token_past_the_border():
    p = np.array([[0.0, 0.25, 0.0, 0.5, 0.25, 0.0]])
    for u0, want in ((0.0, 1), (0.2499, 1), (0.25, 3), (0.74, 3), (0.75, 4), (0.9999, 4)):
        assert so.verify_tree(p, p, np.zeros(1, int), np.array([-1]), np.array([u0]))[1] == want
    assert so.verify_tree(np.zeros((1, 6)), None, np.zeros(1, int), np.array([-1]), np.array([0.3]))[1] == -1


def test_certain_drafts_leave_the_rest_of_the_row():
    """A rejected certain draft takes its token out of the row: two rejected siblings leave the other tokens in proportion."""
    p = np.tile(np.array([0.4, 0.3, 0.2, 0.1]), (3, 1))
    tok, parent = np.array([0, 0, 1]), np.array([-1, 0, 0])
    line, nxt, _ = so.verify_tree(p, None, tok, parent, np.array([0.6, 0.9, 0.9]))
    assert line == [0] and nxt == 2                       # rest: 2/3, 1/3 on tokens 2 and 3
    assert so.verify_tree(p, None, tok, parent, np.array([0.7, 0.9, 0.9]))[1] == 3
    # the second sibling is judged by the row without the first: 0.3 / 0.6
    assert so.verify_tree(p, None, tok, parent, np.array([0.7, 0.9, 0.49]))[0] == [0, 2]
    assert so.verify_tree(p, None, tok, parent, np.array([0.7, 0.9, 0.51]))[0] == [0]


# ------------------------------------------------------------------------------------------------------ refusals, C side
GOOD = dict(p=16, q=16, dtype=0, tokens=4, parent=4, n_nodes=None, u=4, active=None, batch=1, max_nodes=4, vocab=10,
            path=4, n_path=4, next_token=4)


def _verify(**patch):
    a = {**GOOD, **patch}
    return bd.lib.ptenc_verify_tree(a["p"], a["q"], a["dtype"], a["tokens"], a["parent"], a["n_nodes"], a["u"], a["active"],
                                    a["batch"], a["max_nodes"], a["vocab"], a["path"], a["n_path"], a["next_token"], None)


@pytest.mark.parametrize("patch,code", [
    (dict(p=None), bd.PTENC_EINVAL), (dict(tokens=None), bd.PTENC_EINVAL), (dict(parent=None), bd.PTENC_EINVAL),
    (dict(u=None), bd.PTENC_EINVAL), (dict(path=None), bd.PTENC_EINVAL), (dict(n_path=None), bd.PTENC_EINVAL),
    (dict(next_token=None), bd.PTENC_EINVAL), (dict(dtype=2), bd.PTENC_EINVAL), (dict(dtype=-1), bd.PTENC_EINVAL),
    (dict(batch=0), bd.PTENC_EINVAL), (dict(max_nodes=0), bd.PTENC_EINVAL), (dict(vocab=0), bd.PTENC_EINVAL),
    (dict(max_nodes=65), bd.PTENC_ESHAPE), (dict(batch=(1 << 24) + 1), bd.PTENC_ESHAPE), (dict(vocab=(1 << 28) + 1), bd.PTENC_ESHAPE),
    (dict(p=24), bd.PTENC_EALIGN), (dict(q=8), bd.PTENC_EALIGN), (dict(u=6), bd.PTENC_EALIGN),
    (dict(path=5), bd.PTENC_EALIGN), (dict(n_nodes=2), bd.PTENC_EALIGN),
])
def test_verify_refuses_on_the_host(patch, code):
    assert _verify(**patch) == code


def test_null_handles_are_errors():
    assert bd.lib.ptenc_tree_attn(None, 0, 16, 16, 16, 16, None, 4, None, 16, None, None) == bd.PTENC_EINVAL
    assert bd.lib.ptenc_commit_path(None, 0, 16, 16, 4, 16, 16, None, None, None) == bd.PTENC_EINVAL


# ------------------------------------------------------------------------------------------------------ refusals, binding
class _NoCall:
    """Stands where the library is: a call that should have been refused before it fails the test."""

    ptenc_strerror = staticmethod(bd.lib.ptenc_strerror)

    def __getattr__(self, name):
        raise AssertionError(f"{name} was reached")


@pytest.fixture
def cache(monkeypatch):
    """A cache object without its device side: the binding's own checks come before any use of it."""
    c = pt.Cache.__new__(pt.Cache)
    c.cfg = pt.make_config(n_layers=2, batch=3, n_q_heads=8, n_kv_heads=2, head_dim=64, window=16)
    c.device, c.torch_dtype, c._h = torch.device("cpu"), torch.bfloat16, None
    monkeypatch.setattr(bd, "lib", _NoCall())
    return c


def _tree_args(T=4, lead=(2, 3)):
    bf = torch.bfloat16
    return dict(q=torch.zeros(*lead, T, 8, 64, dtype=bf), k_tree=torch.zeros(*lead, T, 2, 64, dtype=bf),
                v_tree=torch.zeros(*lead, T, 2, 64, dtype=bf), parent=torch.zeros(3, T, dtype=torch.int32),
                out=torch.zeros(*lead, T, 8, 64, dtype=bf))


@pytest.mark.parametrize("name,bad,code", [
    ("q", lambda t: t.float(), bd.PTENC_EINVAL), ("q", lambda t: t[..., :32].contiguous(), bd.PTENC_ESHAPE),
    ("q", lambda t: t.transpose(-1, -2).contiguous().transpose(-1, -2), bd.PTENC_EINVAL),
    ("k_tree", lambda t: t[:1].contiguous(), bd.PTENC_ESHAPE), ("k_tree", lambda t: t[:, :2].contiguous(), bd.PTENC_ESHAPE),
    ("k_tree", lambda t: t[0], bd.PTENC_ESHAPE), ("v_tree", lambda t: t[:, :, :3].contiguous(), bd.PTENC_ESHAPE),
    ("parent", lambda t: t.long(), bd.PTENC_EINVAL), ("parent", lambda t: t[:, :3].contiguous(), bd.PTENC_ESHAPE),
    ("out", lambda t: t[..., ::2], bd.PTENC_EINVAL),
    ("n_nodes", lambda t: torch.zeros(2, dtype=torch.int32), bd.PTENC_ESHAPE),
    ("active", lambda t: torch.ones(3, dtype=torch.bool), bd.PTENC_EINVAL),
    ("lse_out", lambda t: torch.zeros(2, 3, 4, 8, dtype=torch.bfloat16), bd.PTENC_EINVAL),
])
def test_tree_attn_binding_refuses(cache, name, bad, code):
    a = _tree_args()
    a[name] = bad(a.get(name))
    with pytest.raises(pt.PtencError) as e:
        cache.tree_attn(-1, **a)
    assert e.value.code == code


@pytest.mark.parametrize("name,bad,code", [
    ("k_tree", lambda t: t.half(), bd.PTENC_EINVAL), ("v_tree", lambda t: t[..., :1, :].contiguous(), bd.PTENC_ESHAPE),
    ("path", lambda t: t[:2].contiguous(), bd.PTENC_ESHAPE), ("path", lambda t: t.long(), bd.PTENC_EINVAL),
    ("n_path", lambda t: torch.zeros(4, dtype=torch.int32), bd.PTENC_ESHAPE),
    ("n_evicted_out", lambda t: torch.zeros(3, dtype=torch.int32), bd.PTENC_ESHAPE),
])
def test_commit_path_binding_refuses(cache, name, bad, code):
    a = _tree_args()
    a = dict(k_tree=a["k_tree"], v_tree=a["v_tree"], path=torch.zeros(3, 4, dtype=torch.int32),
             n_path=torch.zeros(3, dtype=torch.int32), n_evicted_out=None)
    a[name] = bad(a[name])
    with pytest.raises(pt.PtencError) as e:
        cache.commit_path(-1, **a)
    assert e.value.code == code


@pytest.mark.parametrize("name,bad,code", [
    ("p", lambda t: t.double(), bd.PTENC_EINVAL), ("p", lambda t: t[0], bd.PTENC_EINVAL),
    ("p", lambda t: t[..., ::2], bd.PTENC_EINVAL), ("q", lambda t: t.bfloat16(), bd.PTENC_EINVAL),
    ("q", lambda t: t[:, :3].contiguous(), bd.PTENC_ESHAPE), ("tokens", lambda t: t.long(), bd.PTENC_EINVAL),
    ("u", lambda t: t.double(), bd.PTENC_EINVAL), ("path", lambda t: t[:1].contiguous(), bd.PTENC_ESHAPE),
    ("u", lambda t: t, bd.PTENC_EINVAL),                     # nothing wrong but the device
])
def test_verify_binding_refuses(monkeypatch, name, bad, code):
    monkeypatch.setattr(bd, "lib", _NoCall())
    a = dict(p=torch.zeros(2, 4, 10), q=torch.zeros(2, 4, 10), tokens=torch.zeros(2, 4, dtype=torch.int32),
             parent=torch.zeros(2, 4, dtype=torch.int32), u=torch.zeros(2, 4), path=torch.zeros(2, 4, dtype=torch.int32),
             n_path=torch.zeros(2, dtype=torch.int32), next_token=torch.zeros(2, dtype=torch.int32))
    a[name] = bad(a[name])
    with pytest.raises(pt.PtencError) as e:
        pt.verify_tree(**a)
    assert e.value.code == code
