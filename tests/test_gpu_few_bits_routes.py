"""The calls on few-bit values where their kernels divide the work otherwise: many sequences, runs and single tokens in one call, scales of
either sign, very many rows, rows that begin anywhere."""
import math

import pytest
import torch

import few_bits as F
import paper_1610_02132_b200 as Q
from test_gpu_cache import BF16, FP16, Filled, starts_of, values
from test_gpu_cache_ranges import compare, launched
from test_gpu_int8 import check, normal, operands

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sequences, heads, group", [(256, 2, 8), (257, 2, 8), (300, 2, 8), (700, 1, 8), (1300, 1, 12)])
@pytest.mark.parametrize("dim", [64, 128])
def test_tiles_of_many_sequences(sequences, heads, group, dim):
    """Sequences sorted by their lengths and not, counted in one round of a CTA's threads and in several; some without rows, some without tokens."""
    lengths = [(37 * b) % 71 for b in range(sequences)]
    runs = [(5 * b) % 19 for b in range(sequences)]
    f = Filled(lengths, 16, heads, dim, BF16).write_all()
    q, out, lse, launches = launched(f, heads * group, runs, BF16)
    assert launches == 1
    at = 0
    for b, (n, r) in enumerate(zip(lengths, runs)):
        live = min(n, r)
        assert bool((out[at: at + r - live] == 0).all()) and bool((lse[at: at + r - live] == -math.inf).all())
        if live and (b < 5 or b % 23 == 0 or b > sequences - 5):
            one = Filled([0], 16, 1, dim, BF16)
            one.lengths, one.k, one.v = [n], [f.k[b]], [f.v[b]]
            some = slice(at + r - live, at + r)
            compare(one, q[some], out[some], lse[some], 1 / math.sqrt(dim), [live], BF16, tile=True)
        at += r


@pytest.mark.parametrize("scale", [-0.1, 0.0, 0.02, 1.0, -2.0])
@pytest.mark.parametrize("heads", [3, 148])
def test_scales_in_chunks(scale, heads):
    f = Filled([200, 70], 16, heads, 128, BF16).write_all()
    q, out, lse, launches = launched(f, heads, [100, 33], BF16, scale=scale)
    assert (launches == 1) == (heads == 148)
    some = [0, heads - 1]
    f.k, f.v = [x[:, some] for x in f.k], [x[:, some] for x in f.v]
    compare(f, q[:, some], out[:, some], lse[:, some], scale, [100, 33], BF16, tile=launches == 1)


@pytest.mark.parametrize("size", [1e30, 1e-30])
@pytest.mark.parametrize("heads", [3, 148])
def test_keys_outside_fp16(size, heads):
    f = Filled([400], 16, heads, 128, BF16)
    f.k[0] = (f.k[0].float() * size).to(BF16)
    f.k[0][100:200].mul_(2.0 ** -10)
    f.write_all()
    q, out, lse, launches = launched(f, heads, [100], BF16, scale=0.1 / size)
    assert (launches == 1) == (heads == 148)
    some = [0, heads - 1]
    f.k, f.v = [x[:, some] for x in f.k], [x[:, some] for x in f.v]
    compare(f, q[:, some], out[:, some], lse[:, some], 0.1 / size, [100], BF16, tile=launches == 1)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("heads, group, chunk", [(2, 4, 300), (8, 4, 700), (48, 2, 300)])
def test_a_chunk_beside_single_tokens(dtype, heads, group, chunk):
    """A prompt's chunk among other users' single tokens."""
    lengths = [400, 1, 90] + [20 * b + 3 for b in range(12)] + [chunk + 17, 250]
    runs = [1] * 15 + [chunk, 1]
    f = Filled(lengths, 32, heads, 128, dtype).write_all()
    q, out, lse, launches = launched(f, heads * group, runs, dtype)
    some = [0, heads - 1]
    pick = [h * group + i for h in some for i in range(group)]
    at = 0
    for b, (n, r) in enumerate(zip(lengths, runs)):
        one = Filled([0], 16, 1, 128, dtype)
        for i in range(r) if r == 1 else range(0, r, 29):
            m = n - r + i + 1
            one.lengths, one.k, one.v = [m], [f.k[b][:m, some]], [f.v[b][:m, some]]
            compare(one, q[at + i: at + i + 1, pick], out[at + i: at + i + 1, pick], lse[at + i: at + i + 1, pick], 1 / math.sqrt(128), [1], dtype, tile=launches == 1)
        at += r


@pytest.mark.parametrize("m, n, k", [(65535 * 8 + 5, 17, 33), (2 * 65535 * 8 + 300, 3, 19), (1500, 700, 1001), (4000, 333, 515), (700, 4001, 259)])
def test_many_rows_that_begin_anywhere(m, n, k):
    """Several launches above 524280 rows."""
    a, a_scale, b, b_scale = operands(m, n, k, 5, padded=False)
    out = torch.full((m + 1, n + 3), 42.0, device="cuda")
    Q.qsgd_matmul_i8(a, a_scale, b, b_scale, out[:m, :n])
    check(out[:m, :n], a, a_scale, b, b_scale, None, torch.float32)
    assert bool((out[m:] == 42).all()) and bool((out[:, n:] == 42).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m, n, k, padded", [(3000, 700, 1024, True), (1111, 2001, 1000, True), (2000, 300, 777, False)])
def test_linear_of_a_prompt(m, n, k, padded, dtype):
    x, w = normal((m, k), m + k, dtype).cuda(), (normal((n, k), n) * k ** -0.5).cuda()
    codes, w_scale = Q.quantize_rows_alloc(w)
    if not padded:
        codes = codes.contiguous()
    bias, out = normal((n,), 4).cuda(), torch.empty(m, n, dtype=dtype, device="cuda")
    ws = torch.full((Q.qsgd_linear_i8_workspace_bytes(m, k),), 255, dtype=torch.uint8, device="cuda")
    Q.qsgd_linear_i8(x, codes, w_scale, out, ws, bias=bias)
    a, a_scale = F.quantize_rows(x.cpu())
    check(out.cpu(), a, a_scale.float(), codes.cpu(), w_scale.cpu(), bias.cpu(), dtype)
