"""What the calls between hidden states and token ids refuse, before anything is launched: no GPU is needed."""
import ctypes

import numpy as np
import pytest

import paper_2603_02597_amd as B
from paper_2603_02597_amd import binding

P = 4096            # an address that is not NULL; no refused call reads it


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def _linear(lib, **kw):
    a = dict(x=P, xs=64, w=P, ws=64, dtype=1, m=4, n=8, k=64, bias=None, bt=0, res=None, rs=8, act=0, out=P, os=8, ot=0, work=None, wb=0)
    a.update(kw)
    return lib.bpe_linear(a["x"], a["xs"], a["w"], a["ws"], a["dtype"], a["m"], a["n"], a["k"], a["bias"], a["bt"], a["res"], a["rs"], a["act"], a["out"],
                          a["os"], a["ot"], a["work"], a["wb"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), -1), (dict(w=None), -1), (dict(out=None), -1), (dict(m=-1), -2), (dict(n=1 << 30), -2), (dict(k=-3), -2),
    (dict(xs=63), -2), (dict(ws=63), -2), (dict(os=7), -2), (dict(res=P, rs=7), -2), (dict(dtype=0), -10), (dict(dtype=3), -10),
    (dict(ot=2), -10), (dict(ot=5), -10), (dict(bias=P, bt=9), -10), (dict(act=5), -10), (dict(act=-1), -10), (dict(x=P + 1), -2),
    (dict(w=P + 1), -2), (dict(out=P + 2), -2), (dict(res=P + 2), -2), (dict(bias=P + 2, bt=0), -2)])
def test_linear(lib, kw, code):
    assert _linear(lib, **kw) == code
    assert lib.bpe_last_error()


def test_linear_without_elements_needs_nothing(lib):
    assert _linear(lib, m=0, x=None, out=None) == 0 and _linear(lib, n=0, w=None, out=None) == 0


def test_linear_workspace(lib):
    assert lib.bpe_linear_workspace_bytes(-1, 5, 5) == -2 and lib.bpe_linear_workspace_bytes(5, 1 << 30, 5) == -2
    assert lib.bpe_linear_workspace_bytes(0, 0, 0) == 0
    for m, n, k in ((65, 300, 4096), (100, 256, 65536), (300, 300, 3000)):
        need = lib.bpe_linear_workspace_bytes(m, n, k)
        assert need >= 0
        if need:
            for work, wb in ((None, need), (P, need - 1), (P + 64, need)):
                assert _linear(lib, m=m, n=n, k=k, xs=k, ws=k, os=n, work=work, wb=wb) == -8


def _adjust(lib, rules=None, **kw):
    a = dict(l=P, ls=100, dtype=0, rows=3, vocab=100, out=P, os=100, ot=0)
    a.update(kw)
    r = None
    if rules is not None:
        r = binding._LogitRules(**rules)
        r = ctypes.byref(r)
    return lib.bpe_adjust_logits(a["l"], a["ls"], a["dtype"], a["rows"], a["vocab"], r, a["out"], a["os"], a["ot"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(l=None), -1), (dict(out=None), -1), (dict(rows=-1), -2), (dict(vocab=0), -2), (dict(vocab=1 << 30), -2), (dict(ls=99), -2),
    (dict(os=99), -2), (dict(dtype=4), -10), (dict(ot=1), -10), (dict(dtype=1, ot=2), -10), (dict(l=P + 2), -2), (dict(out=P + 1, dtype=1, ot=1), -2),
    (dict(dtype=1), -10), (dict(ls=200), -10),                     # in place with other types or strides
    (dict(rules=dict(n_history=-1)), -2), (dict(rules=dict(n_history=5)), -1), (dict(rules=dict(n_history=5, history=P)), -1),
    (dict(rules=dict(n_bias=2, bias_ids=P)), -1), (dict(rules=dict(n_bias=1 << 31)), -2), (dict(rules=dict(n_masks=-1)), -2),
    (dict(rules=dict(masks=P, n_masks=3, mask_stride=3)), -2), (dict(rules=dict(masks=P, n_masks=2, mask_stride=4)), -2)])
def test_adjust_logits(lib, kw, code):
    assert _adjust(lib, **kw) == code
    assert lib.bpe_last_error()


def _top(lib, **kw):
    rows, vocab, k = kw.get("rows", 3), kw.get("vocab", 100), kw.get("k", 5)
    need = max(lib.bpe_top_tokens_workspace_bytes(rows, vocab, k), 0)
    a = dict(l=P, ls=100, dtype=0, ids=P, lp=P, ws=P, wb=need)
    a.update(kw)
    return lib.bpe_top_tokens(a["l"], a["ls"], a["dtype"], rows, vocab, k, a["ids"], a["lp"], None, a["ws"], a["wb"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(l=None), -1), (dict(ids=None), -1), (dict(lp=None), -1), (dict(rows=-1), -2), (dict(vocab=0, k=1), -2), (dict(k=0), -2), (dict(k=101), -2),
    (dict(vocab=5000, ls=5000, k=257), -2), (dict(ls=99), -2), (dict(dtype=3), -10), (dict(l=P + 1, dtype=1), -2)])
def test_top_tokens(lib, kw, code):
    assert _top(lib, **kw) == code
    assert lib.bpe_last_error()


def test_top_tokens_workspace(lib):
    for rows, vocab, k in ((1, 50000, 64), (300, 50000, 64)):
        need = lib.bpe_top_tokens_workspace_bytes(rows, vocab, k)
        assert need >= 0
        if need:
            for ws, wb in ((None, need), (P, need - 1), (P + 128, need)):
                assert _top(lib, rows=rows, vocab=vocab, ls=vocab, k=k, ws=ws, wb=wb) == -8


def test_grammar(lib):
    h = ctypes.c_void_p()
    table = np.full((2, 256), -1, dtype=np.int32)
    at = table.ctypes.data_as(ctypes.c_void_p)
    assert lib.bpe_grammar_build(at, None, 2, None) == -1
    assert lib.bpe_grammar_build(None, None, 2, ctypes.byref(h)) == -1
    assert lib.bpe_grammar_build(at, None, 0, ctypes.byref(h)) == -2
    assert lib.bpe_grammar_build(at, None, 65535, ctypes.byref(h)) == -2
    table[1, 7] = 2
    assert lib.bpe_grammar_build(at, None, 2, ctypes.byref(h)) == -3 and b"byte 7 of state 1" in lib.bpe_last_error()
    assert not h.value
    assert lib.bpe_grammar_info(None, None) == -1 and lib.bpe_grammar_free(None) == 0
    assert lib.bpe_grammar_masks(None, None, P, 1, 0, 10, -1, P, 1, None) == -1
    assert lib.bpe_grammar_advance(None, None, P, P, 1, 0, -1, P, None) == -1


def test_the_binding_refuses_what_is_no_matrix_on_the_gpu():
    import torch
    x = torch.zeros(2, 8, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        B.bpe_linear(x, x, torch.zeros(2, 2))
    with pytest.raises(TypeError):
        B.bpe_adjust_logits(torch.zeros(2, 8), torch.zeros(2, 8))
    with pytest.raises(TypeError):
        B.bpe_top_tokens(torch.zeros(2, 8), torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 1), None)
    with pytest.raises(ValueError):
        B.Grammar(np.zeros((2, 256)), accepting=[1])
