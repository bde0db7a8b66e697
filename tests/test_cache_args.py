"""Refusals of the paged cache's entry points, all before any device work, and
what the library says of them.  Pointers are never followed."""
import ctypes

import pytest

from paper_2601_21824_amd import binding as b

P = 1 << 20  # stands for an aligned device pointer


def cache(**kw):
    c = b.dash_paged_cache_t(2, 8, 2, 128, 10, 16, 4, b.DASH_CACHE_BF16, P, P, 2 * 16 * 128, 16 * 128, 128,
                             2 * 16 * 128, 16 * 128, 128, P, 4, P, None, None)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def append(**kw):
    x = b.dash_append_t(2, None, P, P, P, P, None, 256, 128, 256, 128, 1024, 128, 1024, 128, 0, 0, P, 128, 0)
    for k, v in kw.items():
        setattr(x, k, v)
    return x


def run_append(c, x):
    return b.load().dash_kv_append(None if c is None else ctypes.byref(c), None if x is None else ctypes.byref(x), None, None)


def run_decode(c, q=P, o=P, strides=(1024, 128, 1024, 128), scale=0.0, ws=P, ws_bytes=1 << 30):
    return b.load().dash_attn_decode(None if c is None else ctypes.byref(c), q, strides[0], strides[1], o, strides[2],
                                     strides[3], None, scale, ws, ws_bytes, None, None)


BAD_CACHES = [
    (dict(batch=-1), "batch"), (dict(heads_kv=3), "heads_kv"), (dict(heads_kv=0), "heads_kv"), (dict(d=96), "head dim"),
    (dict(cache_type=2), "cache_type"), (dict(k_scale=P), "E4M3"), (dict(page_size=8), "page_size"),
    (dict(page_size=24), "page_size"), (dict(page_size=1 << 17), "page_size"), (dict(table_width=-1), "table_width"),
    (dict(table_width=1 << 28), "table_width"), (dict(pages=0), "pages"), (dict(lens=None), "lens"),
    (dict(block_table=None), "block_table"), (dict(table_stride=3), "table_stride"), (dict(k_cache=None), "k_cache"),
    (dict(v_cache=P + 8), "v_cache"), (dict(k_row_stride=132), "k_cache"), (dict(v_head_stride=-2048), "v_cache"),
    (dict(k_row_stride=64), "k_cache"), (dict(v_row_stride=1 << 23), "v_cache"), (dict(k_page_stride=-8), "k_cache"),
    (dict(v_page_stride=4), "v_cache"), (dict(cache_type=b.DASH_CACHE_E4M3, k_head_stride=2056), "k_cache"),
]


@pytest.mark.parametrize("change,word", BAD_CACHES)
def test_bad_caches(change, word):
    for rc in (run_append(cache(**change), append()), run_decode(cache(**change))):
        assert rc == b.DASH_ERR_INVALID_ARG
        assert word in b.dash_last_error()


@pytest.mark.parametrize("change,word", [
    (dict(tokens=-1), "tokens"), (dict(tokens=3), "cu"), (dict(rotary_dim=0), "rotary"), (dict(rotary_dim=24), "rotary"),
    (dict(rotary_dim=144), "rotary"), (dict(k=None), "k:"), (dict(v=P + 2), "v:"), (dict(q_out=None), "q_out"),
    (dict(q=None), "q_out"), (dict(q_row_stride=1028), "q:"), (dict(q_out_head_stride=64), "q_out: the strides"),
    (dict(q_out_row_stride=512), "q_out: the strides"), (dict(k_out=P, k_out_row_stride=128, k_out_head_stride=128), "k_out: the strides"),
])
def test_bad_tokens(change, word):
    assert run_append(cache(), append(**change)) == b.DASH_ERR_INVALID_ARG
    assert word in b.dash_last_error()


def test_written_pages_may_not_overlap_but_read_ones_may():
    tight = dict(k_page_stride=16 * 128)
    assert run_append(cache(**tight), append()) == b.DASH_ERR_INVALID_ARG and "pages overlap" in b.dash_last_error()
    # (refused for its workspace, past the checks of the cache)
    assert run_decode(cache(**tight), ws_bytes=0) == b.DASH_ERR_INVALID_ARG and "workspace" in b.dash_last_error()
    # heads outermost: a page's rows of one head, then all other pages of that head
    outer = dict(k_page_stride=16 * 128, k_head_stride=10 * 16 * 128)
    assert run_append(cache(**outer), append(rotary_dim=8)) == b.DASH_ERR_INVALID_ARG and "rotary" in b.dash_last_error()


def test_decode_arguments():
    assert run_decode(None) == b.DASH_ERR_INVALID_ARG
    assert run_append(None, append()) == b.DASH_ERR_INVALID_ARG and run_append(cache(), None) == b.DASH_ERR_INVALID_ARG
    for scale in (-1.0, float("inf"), float("nan")):
        assert run_decode(cache(), scale=scale) == b.DASH_ERR_INVALID_ARG and "scale" in b.dash_last_error()
    assert run_decode(cache(), q=None) == b.DASH_ERR_INVALID_ARG and "q:" in b.dash_last_error()
    assert run_decode(cache(), o=None) == b.DASH_ERR_INVALID_ARG and "o:" in b.dash_last_error()
    assert run_decode(cache(), strides=(1024, 128, 1024, 64)) == b.DASH_ERR_INVALID_ARG and "overlap" in b.dash_last_error()
    need = b.dash_decode_workspace_size(2, 8, 2, 128, 16, 4)
    assert need > 0
    for ws, n in ((None, need), (P, need - 1), (P + 16, need)):
        assert run_decode(cache(), ws=ws, ws_bytes=n) == b.DASH_ERR_INVALID_ARG and "workspace" in b.dash_last_error()
    assert b.dash_decode_workspace_size(1 << 16, 64, 64, 256, 16, 1 << 20) >= (1 << 16) * 64 * 256 * 4  # past 2^31
    assert b.dash_decode_workspace_size(2, 8, 3, 128, 16, 4) == 0
    assert b.dash_decode_workspace_size(2, 8, 2, 96, 16, 4) == 0
    assert b.dash_decode_workspace_size(2, 8, 2, 128, 8, 4) == 0
    assert b.dash_decode_workspace_size(2, 8, 2, 128, 16, 1 << 28) == 0


def test_calls_too_large_for_a_launch():
    """2^32 threads and more: refused by name, before any device work (cases that fit are not run here)."""
    for c in (cache(batch=1 << 20, heads_q=64, heads_kv=64, table_width=1 << 16, table_stride=1 << 16),  # (main kernel and joins)
              cache(batch=1 << 20, heads_q=16, heads_kv=1, table_width=1 << 16, table_stride=1 << 16),  # (joins alone)
              cache(batch=1 << 20, heads_q=16, heads_kv=8)):  # (short tables: eight waves a workgroup)
        assert run_decode(c, strides=(1 << 14, 128, 1 << 14, 128), ws_bytes=1 << 50) == b.DASH_ERR_UNSUPPORTED
        assert "too large" in b.dash_last_error()
    many = dict(tokens=(1 << 26) - 7, cu=P)
    assert run_append(cache(), append(**many)) == b.DASH_ERR_UNSUPPORTED and "tokens" in b.dash_last_error()
    assert run_append(cache(), append(q=None, q_out=None, **dict(many, tokens=(1 << 31) - 1))) == b.DASH_ERR_UNSUPPORTED


def test_empty_calls_are_no_ops():
    assert run_append(cache(batch=0, lens=None, k_cache=None), append(tokens=0)) == b.DASH_OK
    assert run_append(cache(), append(tokens=0, cu=P, k=None)) == b.DASH_OK
    assert run_decode(cache(batch=0, k_cache=None, lens=None), q=None, o=None, ws=None, ws_bytes=0) == b.DASH_OK


def test_binding_checks_tensors():
    import torch
    x = torch.zeros(2, 8, 128, dtype=torch.bfloat16)
    kv = torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16)
    table, lens = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: b.dash_attn_decode(x, kv, kv, table, lens, x),
                 lambda: b.dash_kv_append(x[:, :2], x[:, :2], kv, kv, table, lens),
                 lambda: b.dash_attn_decode(x[0], kv, kv, table, lens, x),
                 lambda: b.dash_kv_append(x[:, :2], x[:, :2], kv, kv, table, lens, q=x)):
        with pytest.raises(b.DashError) as e:
            call()
        assert e.value.code == b.DASH_ERR_INVALID_ARG


def test_binding_checks_shapes():
    """A tensor of as many values in another shape: an L with its dimensions swapped, a matrix of lengths."""
    import torch
    f, i = torch.float32, torch.int32
    at = b._flat  # (device -1: the CPU's)
    for shape in ((3, 5), (1, 5), (3, 1), (0, 4)):
        x = torch.zeros(shape, dtype=f)
        assert at("lse", x, f, -1, *shape) == x.data_ptr()
        for other in (shape[::-1], (shape[0] * shape[1],), (1, *shape)):
            with pytest.raises(b.DashError, match="lse"):
                at("lse", torch.zeros(other, dtype=f), f, -1, *shape)
    for shape in ((6,), (6, 1), (1, 1, 6)):
        assert at("lens", torch.zeros(shape, dtype=i), i, -1, 6) != 0
    for shape in ((2, 3), (5,), (7, 1), (), (6, 0), (1, 2, 3)):
        with pytest.raises(b.DashError, match="lens"):
            at("lens", torch.zeros(shape, dtype=i), i, -1, 6)
    for shape in ((), (1,), (1, 1)):
        assert at("status", torch.zeros(shape, dtype=i), i, -1, 1) != 0
    assert at("status", None, i, -1, 1) == 0
    for bad in (torch.zeros(4, 2, dtype=i)[:, 0], torch.zeros(4, dtype=f)):
        with pytest.raises(b.DashError, match="lens"):
            at("lens", bad, i, -1, 4)
