"""Refusals of the packed entry points, all before any device work.  Pointers are
never followed."""
import ctypes

import pytest

from paper_2601_21824_amd import binding as b

P = 1 << 20  # stands for an aligned device pointer


def problem(**kw):
    p = b.dash_packed_t(2, 8, 2, 128, 1, 300, 300, 0.0, P, None)
    for t, h in (("q", 8), ("k", 2), ("v", 2), ("o", 8), ("do", 8), ("dq", 8), ("dk", 2), ("dv", 2)):
        setattr(p, t + "_row_stride", h * 128)
        setattr(p, t + "_head_stride", 128)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def fwd(p, ptrs=(P,) * 4, lse=P, ws=None, ws_bytes=0):
    return b.load().dash_attn_packed_fwd(None if p is None else ctypes.byref(p), *ptrs, lse, ws, ws_bytes, None)


def bwd(p, ptrs=(P,) * 9, ws=P, ws_bytes=1 << 40):
    q, k, v, o, do, lse, dq, dk, dv = ptrs
    return b.load().dash_attn_packed_bwd(None if p is None else ctypes.byref(p), q, k, v, o, do, lse, dq, dk, dv, ws, ws_bytes,
                                         None, None)


BOTH = [
    (dict(batch=-1), "batch"), (dict(batch=(1 << 20) + 1), "batch"), (dict(heads_kv=3), "heads_kv"), (dict(heads_q=0), "heads_kv"),
    (dict(d=80), "head dim"), (dict(total_q=-1), "total_q"), (dict(total_k=(1 << 28) + 1), "total_q"),
    (dict(scale=-1.0), "scale"), (dict(scale=float("nan")), "scale"), (dict(cu_q=None), "cu_q"), (dict(total_k=299), "cu_k"),
    (dict(q_row_stride=1028), "q:"), (dict(q_row_stride=64), "q:"), (dict(k_head_stride=-128), "k:"),
    (dict(v_row_stride=1 << 23), "v:"), (dict(o_head_stride=132), "o:"),
]


@pytest.mark.parametrize("change,word", BOTH)
def test_bad_problems(change, word):
    for rc in (fwd(problem(**change)), bwd(problem(**change))):
        assert rc == b.DASH_ERR_INVALID_ARG
        assert word in b.dash_last_error()


@pytest.mark.parametrize("change,word", [
    (dict(dq_head_stride=64), "dq: the strides"), (dict(dk_row_stride=128), "dk: the strides"), (dict(dv_row_stride=100), "dv:"),
    (dict(do_row_stride=8), "dO:")])
def test_bad_gradients(change, word):
    assert bwd(problem(**change)) == b.DASH_ERR_INVALID_ARG
    assert word in b.dash_last_error()


def test_outputs_may_not_overlap_but_inputs_may():
    assert fwd(problem(o_row_stride=128)) == b.DASH_ERR_INVALID_ARG and "o: the strides" in b.dash_last_error()
    # one K/V head read by all through a stride of 0; heads outermost: refused only further on
    assert fwd(problem(k_head_stride=0, v_head_stride=0), lse=None) == b.DASH_ERR_INVALID_ARG and "lse" in b.dash_last_error()
    heads_first = dict(o_row_stride=128, o_head_stride=300 * 128)
    assert fwd(problem(**heads_first), lse=None) == b.DASH_ERR_INVALID_ARG and "lse" in b.dash_last_error()


def test_pointers_and_workspace():
    for i in range(4):
        for bad in (None, P + 8):
            assert fwd(problem(), tuple(bad if j == i else P for j in range(4))) == b.DASH_ERR_INVALID_ARG
    for i in range(9):
        assert bwd(problem(), tuple(None if j == i else P for j in range(9))) == b.DASH_ERR_INVALID_ARG
    assert fwd(None) == b.DASH_ERR_INVALID_ARG and bwd(None) == b.DASH_ERR_INVALID_ARG
    need = b.dash_packed_workspace_size(2, 300, 300, 8, 2, 128)
    assert need >= 300 * 8 * 128 * 4
    for ws, n in ((None, need), (P, need - 1), (P + 16, need)):
        assert bwd(problem(), ws=ws, ws_bytes=n) == b.DASH_ERR_INVALID_ARG and "workspace" in b.dash_last_error()
    for bad in ((2, 300, 300, 8, 3, 128), (2, 300, 300, 8, 2, 100), (-1, 300, 300, 8, 2, 128), (2, -1, 300, 8, 2, 128)):
        assert b.dash_packed_workspace_size(*bad) == 0
    # sizes past 2^31 bytes come through whole
    assert b.dash_packed_workspace_size(64, 1 << 20, 1 << 20, 32, 8, 128) >= (1 << 20) * 32 * 128 * 4


def test_forward_workspace():
    big = dict(total_k=30000, cu_k=P)
    need = b.dash_packed_fwd_workspace_size(2, 300, 30000, 8, 2, 128)
    assert need > 0 and b.dash_packed_fwd_workspace_size(2, 300, 300, 8, 2, 128) == 0
    assert b.dash_packed_fwd_workspace_size(2, 300, 30000, 8, 3, 128) == 0
    for ws, n in ((P, need - 1), (P + 16, need)):
        assert fwd(problem(**big), ws=ws, ws_bytes=n) == b.DASH_ERR_INVALID_ARG and "workspace" in b.dash_last_error()


def test_forward_workspace_of_mostly_empty_sequences():
    """Room for the runs of rows that are there, not of every sequence that could have some."""
    for batch, total_q, total_k, hq, hkv, d in ((1024, 8, 1 << 22, 32, 8, 128), (1 << 15, 1, 1 << 28, 8, 8, 256), (4096, 1, 1 << 24, 1, 1, 64)):
        assert b.dash_packed_fwd_workspace_size(batch, total_q, total_k, hq, hkv, d) <= 8192 * 128 * (d + 2) * 4
    # a token of each of 64 sequences, one of eight, and one alone: split as before
    for batch, total_q, total_k, hq, splits in ((64, 64, 64 * 4096, 4, 2), (8, 1, 8 * 8192, 8, 16), (1, 1, 8192, 32, 16)):
        rows = (total_q // 128 + batch) * hq * splits * 128
        assert b.dash_packed_fwd_workspace_size(batch, total_q, total_k, hq, hq, 128) == rows * 130 * 4


def test_too_many_blocks():
    big = dict(heads_q=4096, heads_kv=4096, total_q=1 << 20, total_k=1 << 20, cu_k=P)
    assert fwd(problem(**big)) == b.DASH_ERR_UNSUPPORTED and "2^24" in b.dash_last_error()
    big = dict(heads_q=4096, heads_kv=4096, total_q=64, total_k=1 << 28, cu_k=P)
    assert bwd(problem(**big)) == b.DASH_ERR_UNSUPPORTED and "2^30" in b.dash_last_error()


def test_empty_calls_are_no_ops():
    none = (None,) * 9
    for p in (problem(batch=0), problem(total_q=0, total_k=0)):
        assert fwd(p, (None,) * 4, None) == b.DASH_OK
        assert bwd(p, none, ws=None, ws_bytes=0) == b.DASH_OK
    assert fwd(problem(total_q=0, cu_k=P), (None, P, P, None), None) == b.DASH_OK  # keys, no queries


def test_binding_checks_tensors():
    import torch
    q, k = torch.zeros(4, 8, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    cu, lse = torch.tensor([0, 4], dtype=torch.int32), torch.zeros(8, 4)
    for call in (lambda: b.dash_attn_packed_fwd(q, k, k, q, lse, cu), lambda: b.dash_attn_packed_fwd(q[0], k, k, q, lse, cu),
                 lambda: b.dash_attn_packed_bwd(q, k, k, q, q, lse, q, k, k, cu)):
        with pytest.raises(b.DashError) as e:
            call()
        assert e.value.code == b.DASH_ERR_INVALID_ARG
