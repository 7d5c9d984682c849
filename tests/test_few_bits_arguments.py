"""What the calls on few-bit values refuse, as far as it shows without a GPU: the C calls check their arguments before
they launch (no pointer here is ever followed), and the Python calls refuse CPU tensors before the library is entered."""
import ctypes as C
import math

import pytest
import torch

import paper_1610_02132_b200 as Q
from paper_1610_02132_b200.binding import CacheRowsStruct, CacheStruct

NULL, SIZE, ALIGN, LAYOUT, TYPE, SHAPE = -1, -2, -5, -11, -12, -13
BF16, F16, F32 = 2, 1, 0


def cache(data=4096, n_pages=4, page_stride=None, head_stride=None, page_tokens=16, heads=2, head_dim=128, type=BF16):
    one = page_tokens // 16 * 18 * head_dim
    return CacheStruct(data, n_pages, heads * one if page_stride is None else page_stride, one if head_stride is None else head_stride,
                       page_tokens, heads, head_dim, type)


def rows(table=4096, table_stride=4, table_pages=4, sequences=3, lengths=4096, starts=4096, n=5):
    return CacheRowsStruct(table, table_stride, table_pages, sequences, lengths, starts, n)


def store(c=None, r=None, k=4096, ks=(256, 128), v=4096, vs=(256, 128), status=4096, read=False):
    call = Q.binding.lib().qsgd_cache_read if read else Q.binding.lib().qsgd_cache_write
    return call(c or cache(), r or rows(), k, *ks, v, *vs, status, None)


def attend(c=None, r=None, q=4096, qs=(512, 128), heads=4, scale=1.0, out=4096, outs=(512, 128), lse=None, ws=4096, status=4096):
    return Q.binding.lib().qsgd_cache_attend(c or cache(), r or rows(), q, *qs, heads, scale, out, *outs, lse, ws, status, None)


CACHES = [(dict(type=F32), TYPE), (dict(type=7), TYPE), (dict(head_dim=96), LAYOUT), (dict(head_dim=0), LAYOUT), (dict(head_dim=320), LAYOUT),
          (dict(page_tokens=24), LAYOUT), (dict(page_tokens=0, page_stride=4608, head_stride=2304), LAYOUT), (dict(heads=0), LAYOUT),
          (dict(heads=2 ** 17), LAYOUT), (dict(n_pages=0), SHAPE), (dict(n_pages=2 ** 31), SHAPE), (dict(data=None), NULL),
          (dict(data=4104), ALIGN), (dict(page_stride=4616), ALIGN), (dict(head_stride=2312), ALIGN),
          (dict(page_stride=2304), LAYOUT),                 # pages inside one another
          (dict(head_stride=0), LAYOUT), (dict(page_stride=2 ** 41), LAYOUT)]
ROWS = [(dict(table=None), NULL), (dict(lengths=None), NULL), (dict(table=4098), ALIGN), (dict(starts=4097), ALIGN), (dict(table_stride=3), SHAPE),
        (dict(table_pages=0), SHAPE), (dict(n=2 ** 31), SHAPE), (dict(starts=None), SHAPE)]     # (the last: 5 rows of 3 sequences)


@pytest.mark.parametrize("change, code", CACHES)
def test_caches_refused(change, code):
    assert store(cache(**change)) == store(cache(**change), read=True) == attend(cache(**change)) == code


@pytest.mark.parametrize("change, code", ROWS)
def test_rows_refused(change, code):
    assert store(r=rows(**change)) == store(r=rows(**change), read=True) == attend(r=rows(**change)) == code


def test_dense_sides_refused():
    L = Q.binding.lib()
    assert L.qsgd_cache_write(None, rows(), 4096, 256, 128, 4096, 256, 128, 4096, None) == NULL
    assert L.qsgd_cache_write(cache(), None, 4096, 256, 128, 4096, 256, 128, 4096, None) == NULL
    assert store(status=None) == NULL
    for read in (False, True):
        assert store(k=None, read=read) == store(v=None, read=read) == NULL
        assert store(k=4104, read=read) == store(v=4098, read=read) == ALIGN
        assert store(ks=(252, 128), read=read) == store(vs=(256, 132), read=read) == ALIGN
        assert store(ks=(2 ** 41, 128), read=read) == LAYOUT
    assert store(ks=(128, 128), read=True) == LAYOUT          # what is read back would overlap
    assert store(vs=(256, 0), read=True) == LAYOUT
    assert attend(q=None) == attend(out=None) == attend(ws=None) == attend(status=None) == NULL
    assert attend(q=4100) == attend(out=4104) == attend(ws=4100) == attend(lse=4097) == attend(outs=(516, 128)) == ALIGN
    assert attend(heads=0) == attend(heads=3) == attend(scale=math.nan) == attend(scale=math.inf) == LAYOUT
    assert attend(outs=(0, 128)) == attend(outs=(512, 64)) == LAYOUT
    assert attend(r=rows(n=2 ** 30), qs=(16384, 128), outs=(16384, 128), heads=128) == SHAPE


def test_nothing_to_do_launches_nothing():
    assert store(r=rows(n=0)) == store(r=rows(n=0, sequences=0, table=None, lengths=None)) == 0
    assert attend(r=rows(n=0), q=None, out=None, ws=None) == 0
    assert attend(r=rows(sequences=0)) == 0
    L = Q.binding.lib()
    assert L.qsgd_quantize_rows(None, 0, 64, 64, BF16, None, 64, None, None) == 0
    assert L.qsgd_matmul_i8(None, 64, None, None, 64, None, None, 0, 5, 64, None, 5, F32, None, None) == 0
    assert L.qsgd_matmul_i8(None, 64, None, None, 64, None, None, 5, 0, 64, None, 5, F32, None, None) == 0
    assert L.qsgd_linear_i8(None, 64, F32, None, 64, None, None, 0, 5, 64, None, 5, F32, None, None, None) == 0


def test_workspace_sizes():
    for dim in (64, 128, 192, 256):
        small = Q.binding.lib().qsgd_cache_attend_workspace_bytes(cache(head_dim=dim), 2)
        assert 0 < small == Q.binding.lib().qsgd_cache_attend_workspace_bytes(cache(head_dim=dim), 64)
    assert Q.binding.lib().qsgd_cache_attend_workspace_bytes(cache(), 3) == 0
    assert Q.binding.lib().qsgd_cache_attend_workspace_bytes(cache(head_dim=96), 2) == 0
    assert Q.qsgd_linear_i8_workspace_bytes(5, 100) == 5 * 112 + 32
    assert Q.qsgd_linear_i8_workspace_bytes(5, 0) == Q.qsgd_linear_i8_workspace_bytes(5, 131072) == 0


def test_products_refused():
    L = Q.binding.lib()
    rows_ = lambda x=4096, n=3, cols=64, stride=64, type=BF16, codes=4096, cs=64, scale=4096: \
        L.qsgd_quantize_rows(x, n, cols, stride, type, codes, cs, scale, None)
    assert rows_(type=3) == TYPE
    assert rows_(cols=0) == rows_(cols=131072) == rows_(n=2 ** 31) == rows_(cs=63) == rows_(stride=2 ** 41) == SHAPE
    assert rows_(x=None) == rows_(codes=None) == rows_(scale=None) == NULL
    assert rows_(x=4097) == rows_(x=4098, type=F32) == rows_(scale=4098) == ALIGN
    mm = lambda a=4096, sa=4096, b=4096, sb=4096, bias=None, m=3, n=5, cols=64, out=4096, os=5, type=F32, stride=64: \
        L.qsgd_matmul_i8(a, stride, sa, b, 64, sb, bias, m, n, cols, out, os, type, None, None)
    assert mm(type=-1) == TYPE
    assert mm(cols=0) == mm(cols=131072) == mm(m=2 ** 31) == mm(n=2 ** 31) == mm(os=4) == mm(stride=2 ** 40) == SHAPE
    assert mm(a=None) == mm(b=None) == mm(sa=None) == mm(sb=None) == mm(out=None) == NULL
    assert mm(sa=4097) == mm(sb=4098) == mm(bias=4098) == mm(out=4098) == ALIGN
    lin = lambda x=4096, xt=BF16, w=4096, sw=4096, m=3, n=5, cols=64, out=4096, os=5, type=F32, ws=4096: \
        L.qsgd_linear_i8(x, 64, xt, w, 64, sw, None, m, n, cols, out, os, type, ws, None, None)
    assert lin(xt=9) == lin(type=9) == TYPE
    assert lin(cols=0) == lin(m=2 ** 31) == lin(os=4) == SHAPE
    assert lin(x=None) == lin(w=None) == lin(sw=None) == lin(out=None) == lin(ws=None) == NULL
    assert lin(ws=4104) == lin(x=4097) == lin(out=4098) == ALIGN
    for code in (LAYOUT, TYPE, SHAPE):
        assert L.qsgd_status_string(code) != b"unknown status"


def test_cpu_tensors_are_refused():
    with pytest.raises(Q.QsgdError, match="at least one page"):
        Q.Cache(1, 24, 1, 64, device="cpu")
    with pytest.raises(Q.QsgdError, match="at least one page"):
        Q.Cache(1, 16, 1, 64, torch.float32, device="cpu")
    with pytest.raises(Q.QsgdError, match="data must be"):
        Q.Cache(1, 16, 1, 64, device="cpu", data=torch.zeros(1, 1, 1000, dtype=torch.uint8))
    c = Q.Cache(2, 16, 1, 64, device="cpu")
    i32 = torch.zeros(2, 2, dtype=torch.int32)
    x = torch.zeros(2, 1, 64, dtype=torch.bfloat16)
    for call in (Q.qsgd_cache_write, Q.qsgd_cache_read):
        with pytest.raises(Q.QsgdError, match="the cache's data must be a CUDA tensor"):
            call(c, i32, i32[0], x, x, i32[0])
    with pytest.raises(Q.QsgdError, match="the cache's data must be a CUDA tensor"):
        Q.qsgd_cache_attend(c, i32, i32[0], x, x, x, i32[0])
    codes, scale = torch.zeros(2, 64, dtype=torch.int8), torch.zeros(2)
    with pytest.raises(Q.QsgdError, match="x must be a CUDA tensor"):
        Q.qsgd_quantize_rows(x[:, 0], codes, scale)
    with pytest.raises(Q.QsgdError, match="a must be a CUDA tensor"):
        Q.qsgd_matmul_i8(codes, scale, codes, scale, scale)
    with pytest.raises(Q.QsgdError, match="x must be a CUDA tensor"):
        Q.qsgd_linear_i8(None, codes, scale, scale, codes)
