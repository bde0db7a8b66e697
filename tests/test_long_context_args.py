"""Refusals of the rotary, microscaled cache, read and shared-prefix entry points, all before any device work,
workspace sizes and the frequencies' host computation.  Pointers are never followed."""
import ctypes
import math

import numpy as np
import pytest

from paper_2601_21824_amd import binding as b

P = 1 << 20  # stands for an aligned device pointer


def make(cls, base, kw):
    x = cls(**base)
    for k, v in kw.items():
        setattr(x, k, v)
    return ctypes.byref(x)


ROTARY = dict(rows=4, heads_q=8, heads_k=2, d=128, positions=P, q=P, k=P, q_out=P, k_out=P, q_row_stride=1024, q_head_stride=128,
              k_row_stride=256, k_head_stride=128, q_out_row_stride=1024, q_out_head_stride=128, k_out_row_stride=256,
              k_out_head_stride=128, inv_freq=P, rotary_dim=128, amplitude=1.0)
CACHE = dict(batch=2, heads_q=8, heads_kv=2, d=128, pages=10, page_size=16, table_width=4, cache_type=b.DASH_CACHE_MXFP8, k_cache=P, v_cache=P,
             k_page_stride=2 * 16 * 128, k_head_stride=16 * 128, k_row_stride=128, v_page_stride=2 * 16 * 128, v_head_stride=16 * 128,
             v_row_stride=128, block_table=P, table_stride=4, lens=P, k_mx=P, v_mx=P)
HALF = dict(CACHE, cache_type=b.DASH_CACHE_MXFP4, k_page_stride=2 * 16 * 64, k_head_stride=16 * 64, k_row_stride=64, v_page_stride=2 * 16 * 64,
            v_head_stride=16 * 64, v_row_stride=64)
READ = dict(rows=5, cu=P, k_out=P, v_out=P, k_row_stride=256, k_head_stride=128, v_row_stride=256, v_head_stride=128)


def rotary(**kw):
    return b.load().dash_rotary(make(b.dash_rotary_t, ROTARY, kw), None, None)


def read(cache, **kw):
    return b.load().dash_kv_read(cache, make(b.dash_read_t, READ, kw), None, None)


def append(cache):
    x = b.dash_append_t(2, None, P, P, P, P, None, 256, 128, 256, 128, 1024, 128, 1024, 128, 0, 0, P, 128, 0)
    return b.load().dash_kv_append(cache, ctypes.byref(x), None, None)


def decode(cache, ws_bytes=1 << 30):
    return b.load().dash_attn_decode(cache, P, 1024, 128, P, 1024, 128, None, 0.0, P, ws_bytes, None, None)


def prefix(cache, table=P, width=4, length=P, q=P, o=P, strides=(1024, 128, 1024, 128), scale=0.0, ws=P, ws_bytes=1 << 30):
    return b.load().dash_attn_prefix_decode(cache, table, width, length, q, strides[0], strides[1], o, strides[2], strides[3], None, scale,
                                            ws, ws_bytes, None, None)


def refused(rc, word, code=b.DASH_ERR_INVALID_ARG):
    assert rc == code and word in b.dash_last_error(), (rc, b.dash_last_error())


@pytest.mark.parametrize("kw,word", [
    (dict(rows=-1), "rows"), (dict(rows=1 << 29), "rows"), (dict(d=96), "head dim"), (dict(heads_q=0), "heads"), (dict(heads_k=5000), "heads"),
    (dict(rotary_dim=8), "rotary_dim"), (dict(rotary_dim=136), "rotary_dim"), (dict(rotary_dim=24), "rotary_dim"),
    (dict(amplitude=math.inf), "amplitude"), (dict(amplitude=math.nan), "amplitude"), (dict(q_out=None), "q_out"), (dict(k=None), "k_out"),
    (dict(cu=P), "positions"), (dict(start=P), "positions"), (dict(positions=None), "positions"), (dict(inv_freq=None), "inv_freq"),
    (dict(q=P + 8), "q:"), (dict(k_out=P + 2), "k_out"), (dict(q_row_stride=64), "q:"), (dict(k_head_stride=4), "k:"),
    (dict(q_out=2 * P, q_out_head_stride=0), "overlap"), (dict(q_out_row_stride=2048), "in place"), (dict(positions=None, cu=P, batch=-1), "batch")])
def test_rotary_refuses(kw, word):
    refused(rotary(**kw), word)


def test_rotary_of_nothing():
    assert b.load().dash_rotary(None, None, None) == b.DASH_ERR_INVALID_ARG
    for kw in (dict(rows=0), dict(q=None, q_out=None, k=None, k_out=None), dict(positions=None, cu=P, batch=0)):
        assert rotary(**kw) == b.DASH_OK


@pytest.mark.parametrize("base", [CACHE, HALF])
@pytest.mark.parametrize("kw,word", [
    (dict(k_mx=None), "k_mx"), (dict(v_mx=None), "v_mx"), (dict(k_mx=P + 4), "aligned"), (dict(v_mx=P + 8), "aligned"), (dict(k_scale=P), "E4M3"),
    (dict(v_scale=P), "E4M3"), (dict(cache_type=2), "cache_type"), (dict(cache_type=5), "cache_type"), (dict(k_row_stride=40), "k_cache"),
    (dict(v_row_stride=8), "v_cache"), (dict(k_head_stride=24), "k_cache"), (dict(v_page_stride=8), "v_cache"), (dict(pages=0), "pages"),
    (dict(page_size=24), "page_size"), (dict(batch=-1), "batch"), (dict(heads_q=7), "heads_kv"), (dict(lens=None), "lens")])
def test_microscaled_caches_refused(base, kw, word):
    for call in (append, read, decode, prefix):
        refused(call(make(b.dash_paged_cache_t, base, kw)), word)


def test_rows_of_a_4_bit_cache_are_half_as_long():
    refused(append(make(b.dash_paged_cache_t, HALF, dict(k_row_stride=48))), "k_cache")
    refused(append(make(b.dash_paged_cache_t, HALF, dict(k_head_stride=48))), "overlap")
    refused(append(make(b.dash_paged_cache_t, CACHE, dict(k_row_stride=64))), "k_cache")


@pytest.mark.parametrize("kw,word", [
    (dict(rows=-1), "rows"), (dict(rows=1 << 29), "rows"), (dict(cu=None), "cu"), (dict(k_out=None, v_out=None), "k_out"),
    (dict(k_out=P + 8), "k_out"), (dict(v_row_stride=100), "v_out"), (dict(v_row_stride=64), "v_out"), (dict(k_head_stride=0), "overlap")])
def test_read_refuses(kw, word):
    refused(read(make(b.dash_paged_cache_t, CACHE, {}), **kw), word)


def test_read_of_nothing():
    assert b.load().dash_kv_read(None, make(b.dash_read_t, READ, {}), None, None) == b.DASH_ERR_INVALID_ARG
    assert b.load().dash_kv_read(make(b.dash_paged_cache_t, CACHE, {}), None, None, None) == b.DASH_ERR_INVALID_ARG
    assert read(make(b.dash_paged_cache_t, CACHE, {}), rows=0) == b.DASH_OK
    assert read(make(b.dash_paged_cache_t, CACHE, dict(batch=0))) == b.DASH_OK


@pytest.mark.parametrize("kw,word", [
    (dict(width=-1), "prefix_width"), (dict(width=1 << 28), "prefix_width"), (dict(table=None), "prefix_table"), (dict(length=None), "prefix_len"),
    (dict(q=None), "q:"), (dict(o=P + 4), "o:"), (dict(strides=(1024, 128, 1024, 0)), "overlap"), (dict(scale=-1.0), "scale"),
    (dict(scale=math.inf), "scale"), (dict(ws=None), "workspace"), (dict(ws=P + 128), "workspace"), (dict(ws_bytes=1000), "workspace")])
def test_prefix_refuses(kw, word):
    refused(prefix(make(b.dash_paged_cache_t, CACHE, {}), **kw), word)


def test_prefix_of_nothing_and_its_workspace():
    assert prefix(None) == b.DASH_ERR_INVALID_ARG
    assert prefix(make(b.dash_paged_cache_t, CACHE, dict(batch=0))) == b.DASH_OK
    size = b.dash_prefix_decode_workspace_size
    assert size(64, 32, 8, 128, 16, 3000, 2048) > size(64, 32, 8, 128, 16, 3000, 0) > 0
    for bad in ((-1, 32, 8, 128, 16, 10, 10), (1, 32, 5, 128, 16, 10, 10), (1, 32, 8, 96, 16, 10, 10), (1, 32, 8, 128, 8, 10, 10),
                (1, 32, 8, 128, 16, -1, 10), (1, 32, 8, 128, 16, 10, -1), (1, 32, 8, 128, 16, 10, 1 << 28)):
        assert size(*bad) == 0
    # the prefix's parts stay within what its workgroups leave: (batch G rounded up to 128) rows of 512 at most, or one run
    for batch, hq, hkv, d in ((64, 32, 8, 128), (1, 1, 1, 256), (1000, 8, 1, 64), (1 << 20, 1, 1, 64)):
        rows = (size(batch, hq, hkv, d, 16, 1, 1 << 20) - size(batch, hq, hkv, d, 16, 1, 0)) / (4 * d)
        assert rows <= 512 * 128 * 1.1


def test_frequencies():
    for n in (16, 64, 128, 256):
        i = np.arange(n // 2)
        plain = 10000.0 ** (-2.0 * i / n)
        f, a = b.dash_rotary_frequencies(n)
        assert a == 1.0 and np.allclose(f, plain, rtol=2 ** -23, atol=0)
        f, a = b.dash_rotary_frequencies(n, scaling="linear", factor=4.0)
        assert a == 1.0 and np.allclose(f, plain / 4, rtol=2 ** -23, atol=0)
        f, a = b.dash_rotary_frequencies(n, scaling="base", factor=4.0)
        assert a == 1.0 and f[0] == 1.0 and np.isclose(f[-1], plain[-1] / 4, rtol=2 ** -22)
        f, a = b.dash_rotary_frequencies(n, scaling="parts", factor=8.0, original=4096.0)
        assert np.isclose(a, 0.1 * math.log(8.0) + 1, rtol=2 ** -23)
        turns = 4096 * plain / (2 * math.pi)
        ratio = f / plain
        assert np.all(np.diff(ratio) <= 1e-6) and np.all(ratio >= 0.125 - 1e-6) and np.all(ratio <= 1 + 1e-6)
        step = 10000.0 ** (2.0 / n)  # (the borders are rounded to whole pairs)
        assert np.allclose(ratio[turns > 32 * step], 1, rtol=2 ** -22) and np.allclose(ratio[turns < 1 / step], 0.125, rtol=2 ** -22)
    f, a = b.dash_rotary_frequencies(64, scaling="parts", factor=1.0, original=4096.0)
    assert a == 1.0 and np.allclose(f, 10000.0 ** (-np.arange(0, 64, 2) / 64), rtol=2 ** -23)


@pytest.mark.parametrize("args,kw,word", [
    ((8,), {}, "rotary_dim"), ((24,), {}, "rotary_dim"), ((512,), {}, "rotary_dim"), ((-16,), {}, "rotary_dim"), ((64, 1.0), {}, "base"),
    ((64, math.nan), {}, "base"), ((64,), dict(scaling="other"), "scaling"), ((64,), dict(scaling="linear", factor=0.5), "factor"),
    ((64,), dict(scaling="parts", factor=2.0), "original"), ((64,), dict(scaling="parts", factor=2.0, original=100.0, fast=1.0, slow=2.0), "slow")])
def test_frequencies_refuse(args, kw, word):
    with pytest.raises(b.DashError, match=word):
        b.dash_rotary_frequencies(*args, **kw)


def test_the_package_has_the_calls():
    import paper_2601_21824_amd as dash
    for name in ("dash_rotary", "rotary", "dash_rotary_frequencies", "dash_kv_read", "kv_read", "dash_attn_prefix_decode",
                 "attn_prefix_decode", "dash_prefix_decode_workspace_size"):
        assert getattr(dash, name) is getattr(b, name)


def test_frequencies_by_parts_between_the_borders():
    """dash.h's steps by hand.  n = 128, base 10^4, from 4096 positions: ln(4096 / (64 pi)) = 3.0142 and ln(4096 / (2 pi)) = 6.4799
    over 2 ln 10^4 / 128 = 0.143911 are 20.94 and 45.03, so pairs 20 and 46 are the borders."""
    f, _ = b.dash_rotary_frequencies(128, scaling="parts", factor=8.0, original=4096.0)
    ratio = f / 10000.0 ** (-np.arange(0, 128, 2) / 128)
    for i, want in ((0, 1), (20, 1), (21, 1 - 7 / 8 / 26), (33, 1 - 7 / 16), (40, 1 - 7 / 8 * 20 / 26), (45, 1 - 7 / 8 * 25 / 26), (46, 1 / 8), (63, 1 / 8)):
        assert np.isclose(ratio[i], want, rtol=2 ** -22, atol=0), i
    # n = 16, base 100, from 64 positions, 4 turns and 1: ln(64 / (8 pi)) = 0.9346 and ln(64 / (2 pi)) = 2.3210 over 0.575646
    # are 1.62 and 4.03: pairs 1 and 5
    f, _ = b.dash_rotary_frequencies(16, base=100.0, scaling="parts", factor=2.0, original=64.0, fast=4.0)
    ratio = f / 100.0 ** (-np.arange(0, 16, 2) / 16)
    assert np.allclose(ratio, [1, 1, 0.875, 0.75, 0.625, 0.5, 0.5, 0.5], rtol=2 ** -22, atol=0)
    # one pair where both borders fall together: those before it keep theirs, those behind it take the other
    f, _ = b.dash_rotary_frequencies(16, base=100.0, scaling="parts", factor=2.0, original=2 * math.pi * 100.0 ** (6 / 16), fast=1.0)
    assert set(np.round(f / 100.0 ** (-np.arange(0, 16, 2) / 16), 5)) <= {1.0, 0.75, 0.5}


@pytest.mark.parametrize("n,base,factor,original,fast,slow", [(64, 10000.0, 8.0, 4096.0, 32.0, 1.0), (128, 500000.0, 16.0, 8192.0, 32.0, 1.0),
                                                              (256, 1000.0, 3.0, 100.0, 8.0, 0.5), (96, 10000.0, 2.0, 50.0, 5.0, 1e-4)])
def test_frequencies_by_parts_in_steps(n, base, factor, original, fast, slow):
    """dash.h's steps, one pair at a time."""
    f, a = b.dash_rotary_frequencies(n, base, "parts", factor, original, fast, slow)
    c = [n * math.log(original / (2 * math.pi * t)) / (2 * math.log(base)) for t in (fast, slow)]
    lo, hi = max(math.floor(c[0]), 0), min(math.ceil(c[1]), n - 1)
    for i in range(n // 2):
        x = min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
        g = base ** (-2 * i / n)
        assert abs(f[i] - ((1 - x) * g + x * g / factor)) <= 2.0 ** -23 * g
    assert abs(a - (0.1 * math.log(factor) + 1)) <= 2.0 ** -23 * a
