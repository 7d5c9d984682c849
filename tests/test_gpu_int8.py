"""8-bit rows and their products against their plain statement: codes and sums are exact, the rest within its roundings."""
import math

import pytest
import torch

import few_bits as F
import paper_1610_02132_b200 as Q

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]


def normal(shape, seed, dtype=torch.float32):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, cols, pad", [(1, 1, 0), (3, 7, 0), (5, 64, 0), (2, 4096, 16), (300, 257, 15), (1, 8192, 0), (2, 8200, 0), (2, 20001, 3),
                                             (2000, 40, 8), (1, 131071, 0)])
def test_quantize_rows(dtype, rows, cols, pad):
    x = normal((rows, cols), rows + cols, dtype) * 3
    codes = torch.full((rows, cols + pad), 77, dtype=torch.int8, device="cuda")
    scale = torch.empty(rows, device="cuda")
    Q.qsgd_quantize_rows(x.cuda(), codes[:, :cols], scale)
    want, want_scale = F.quantize_rows(x)
    assert torch.equal(codes[:, :cols].cpu().double(), want)
    assert bool(((scale.cpu().double() - want_scale).abs() <= want_scale * 2.0 ** -24).all())
    assert bool((codes[:, cols:] == 77).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_rows_of_every_sort(dtype):
    x = normal((8, 100), 3, dtype)
    x[0] = 0
    x[1, 50] = math.inf
    x[2, 99] = math.nan
    x[3] = (x[3].float() * 1e-39).to(dtype)                 # below what a scale can stand for (fp16: zeros)
    x[4] = 0
    x[4, 3] = -2
    x[5] = torch.finfo(dtype).max
    x[6] = (torch.arange(100) - 50).to(dtype)
    x[6, 0] = 127                                           # whole numbers are their own codes
    x[7] = (torch.arange(100) - 50).to(dtype) + 0.5         # between two codes: the even one
    x[7, 0] = -127
    codes, scale = torch.empty(8, 100, dtype=torch.int8, device="cuda"), torch.empty(8, device="cuda")
    Q.qsgd_quantize_rows(x.cuda(), codes, scale)
    want, want_scale = F.quantize_rows(x)
    assert torch.equal(codes.cpu().double(), want)
    assert torch.equal(scale.cpu().isnan(), want_scale.isnan()) and bool((scale.cpu()[[0, 3]] == 0).all())
    assert torch.equal(codes[6].cpu()[1:], (torch.arange(100) - 50).to(torch.int8)[1:])


def check(out, a, a_scale, b, b_scale, bias, dtype):
    """Half a step for each of: the sum as fp32, two products, the bias added, the type. From half a step behind the largest number of
    the type on (65520 in fp16) the rounding gives an infinity."""
    total = a.double() @ b.double().T * a_scale.double()[:, None] * b_scale.double()
    ref = total + (0 if bias is None else bias.double())
    tol = 1.01 * (3 * 2.0 ** -24 * total.abs() + (2.0 ** -24 + F.HALF_STEP[dtype]) * ref.abs()) + 1e-30
    over = ref.abs() >= torch.finfo(dtype).max * (1 + F.HALF_STEP[dtype] / 2)
    out, near = out.double(), (ref.abs() - torch.finfo(dtype).max * (1 + F.HALF_STEP[dtype] / 2)).abs() <= 4 * 2.0 ** -24 * ref.abs()
    assert bool((torch.isinf(out) & (out.sign() == ref.sign()))[over & ~near].all())
    off = torch.where(over | near, 0.0, (out - ref).abs())
    assert bool((off <= tol).all()), (off / tol).max()


def operands(m, n, k, seed, padded=True):
    g = torch.Generator().manual_seed(seed)
    row = -(-k // 16) * 16 if padded else k
    out = []
    for rows in (m, n):
        x = torch.full((rows, row), 99, dtype=torch.int8)
        x[:, :k] = torch.randint(-128, 128, (rows, k), generator=g).to(torch.int8)
        out.append(x.cuda()[:, :k])
        out.append((torch.rand(rows, generator=g) + 0.1).cuda())
    return out


SHAPES = [(1, 1, 1), (1, 16, 64), (1, 17, 100), (7, 33, 65), (8, 100, 512), (9, 64, 1000), (16, 40, 31), (17, 300, 130), (33, 129, 2000), (64, 256, 128),
          (65, 257, 129), (100, 96, 4096), (128, 128, 128), (129, 255, 200), (200, 1000, 700), (513, 384, 320), (1, 5000, 16), (9, 8200, 2100), (16, 8192, 2048)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("padded", [True, False])
@pytest.mark.parametrize("m, n, k", SHAPES)
def test_matmul(m, n, k, padded, dtype):
    a, a_scale, b, b_scale = operands(m, n, k, m + n + k, padded)
    bias = None if (m + n) % 2 else torch.randn(n, generator=torch.Generator().manual_seed(1)).cuda()
    out = torch.full((m, n + 3), 42.0, dtype=dtype, device="cuda")
    Q.qsgd_matmul_i8(a, a_scale, b, b_scale, out[:, :n], bias=bias)
    check(out[:, :n], a, a_scale, b, b_scale, bias, dtype)
    assert bool((out[:, n:] == 42).all())


@pytest.mark.parametrize("m", [3, 300])
def test_largest_sums(m):
    """131071 columns of the largest products of one sign: the sum is just inside 32 bits."""
    k = 131071
    a = torch.full((m, k + 1), -128, dtype=torch.int8, device="cuda")[:, :k]
    b = torch.full((130, k + 1), -128, dtype=torch.int8, device="cuda")[:, :k]
    one = torch.ones(300, device="cuda")
    out = torch.empty(m, 130, device="cuda")
    Q.qsgd_matmul_i8(a, one[:m], b, one[:130], out)
    assert bool((out == float(128 * 128 * k)).all())


def test_nothing_to_multiply():
    e = lambda *s: torch.empty(*s, dtype=torch.int8, device="cuda")
    f = lambda *s: torch.empty(*s, device="cuda")
    before = Q.qsgd_launch_count()
    Q.qsgd_matmul_i8(e(0, 64), f(0), e(5, 64), f(5), f(0, 5))
    Q.qsgd_matmul_i8(e(5, 64), f(5), e(0, 64), f(0), f(5, 0))
    Q.qsgd_quantize_rows(f(0, 64), e(0, 64), f(0))
    assert Q.qsgd_launch_count() == before
    with pytest.raises(Q.QsgdError, match="out of|outside"):
        Q.qsgd_matmul_i8(e(5, 0), f(5), e(5, 0), f(5), f(5, 5))


@pytest.mark.parametrize("x_dtype, dtype", [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32), (torch.float32, torch.float16)])
@pytest.mark.parametrize("m, n, k", [(1, 64, 128), (1, 1000, 4096), (5, 33, 77), (40, 512, 1024), (150, 200, 999), (2, 16, 9000), (3, 50, 20000), (11, 8200, 2100), (128, 64, 700),
                                     (129, 64, 700)])
def test_linear(m, n, k, x_dtype, dtype):
    x, w = normal((m, k), m + k, x_dtype).cuda(), normal((n, k), n) * k ** -0.5
    codes, w_scale = Q.quantize_rows_alloc(w.cuda())
    bias = normal((n,), 4).cuda()
    out = torch.empty(m, n, dtype=dtype, device="cuda")
    ws = torch.full((Q.qsgd_linear_i8_workspace_bytes(m, k),), 255, dtype=torch.uint8, device="cuda")
    Q.qsgd_linear_i8(x, codes, w_scale, out, ws, bias=bias)
    a, a_scale = torch.empty(m, k, dtype=torch.int8, device="cuda"), torch.empty(m, device="cuda")
    Q.qsgd_quantize_rows(x, a, a_scale)
    check(out, a, a_scale, codes, w_scale, bias, dtype)


def test_linear_poisoned_row():
    x = normal((4, 256), 1).cuda()
    x[2, 17] = math.inf
    w, w_scale = Q.quantize_rows_alloc(normal((32, 256), 2).cuda())
    out = torch.empty(4, 32, device="cuda")
    ws = torch.empty(Q.qsgd_linear_i8_workspace_bytes(4, 256), dtype=torch.uint8, device="cuda")
    Q.qsgd_linear_i8(x, w, w_scale, out, ws)
    assert bool(out[2].isnan().all()) and not bool(out[[0, 1, 3]].isnan().any())


def test_strided_operands_and_streams():
    a, a_scale, b, b_scale = operands(70, 90, 256, 9)
    out = torch.empty(70, 90, device="cuda")
    Q.qsgd_matmul_i8(a, a_scale, b, b_scale, out)
    wide = torch.zeros(70, 600, dtype=torch.int8, device="cuda")
    for at in (0, 1, 3, 16):                                # rows from any byte on
        view = wide[:, at: at + 256]
        view.copy_(a)
        again = torch.empty(70, 180, device="cuda")[:, ::1][:, 45:135]
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        Q.qsgd_matmul_i8(view, a_scale, b, b_scale, again, stream=s)
        s.synchronize()
        assert torch.equal(again, out)
    every = wide[::2, :256]
    every.copy_(a[:35])
    again = torch.empty(35, 90, device="cuda")
    Q.qsgd_matmul_i8(every, a_scale[:35], b, b_scale, again)
    assert torch.equal(again, out[:35])
    same = a[:1].expand(70, 256)                            # one row for all
    again = torch.empty(70, 90, device="cuda")
    Q.qsgd_matmul_i8(same, a_scale, b, b_scale, again)
    check(again, same, a_scale, b, b_scale, None, torch.float32)


def test_in_a_graph():
    x, (w, w_scale) = normal((6, 512), 1).cuda(), Q.quantize_rows_alloc(normal((300, 512), 2).cuda())
    out, ws = torch.empty(6, 300, device="cuda"), torch.empty(Q.qsgd_linear_i8_workspace_bytes(6, 512), dtype=torch.uint8, device="cuda")
    Q.qsgd_linear_i8(x, w, w_scale, out, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        Q.qsgd_linear_i8(x, w, w_scale, out, ws)
    for seed in (5, 6):
        x.copy_(normal((6, 512), seed))
        g.replay()
        torch.cuda.synchronize()
        again = torch.empty_like(out)
        Q.qsgd_linear_i8(x, w, w_scale, again, torch.empty_like(ws))
        assert torch.equal(out, again)


def test_refusals():
    a, a_scale, b, b_scale = operands(4, 5, 64, 1)
    out = torch.empty(4, 5, device="cuda")
    good = dict(a=a, a_scale=a_scale, b=b, b_scale=b_scale, out=out)
    Q.qsgd_matmul_i8(**good)
    bad = [("a", a.float(), "element type"), ("a", a[0], "2 dimensions"), ("b", b[:, :32], "size 64 in dimension 1"), ("a", a.cpu(), "CUDA tensor"),
           ("a_scale", a_scale[:3], "size 4 in dimension 0"), ("b_scale", b_scale.double(), "element type"), ("out", out.double(), "float32, float16"),
           ("out", out[:3], "size 4 in dimension 0"), ("out", torch.empty(4, 6, device="cuda"), "size 5 in dimension 1"),
           ("out", torch.empty(5, 4, device="cuda").t(), "contiguous along"), ("out", out[:1].expand(4, 5), "outside"),
           ("bias", out[0, :4], "size 5 in dimension 0"), ("bias", b_scale.half(), "element type"), ("b_scale", torch.rand(10, device="cuda")[::2], "contiguous")]
    for name, value, said in bad:
        with pytest.raises(Q.QsgdError, match=said):
            Q.qsgd_matmul_i8(**{**good, name: value})
    x = torch.zeros(4, 64, device="cuda")
    with pytest.raises(Q.QsgdError, match="bytes"):
        Q.qsgd_linear_i8(x, b, b_scale, out, torch.empty(100, dtype=torch.uint8, device="cuda"))
    with pytest.raises(Q.QsgdError, match="float32, float16"):
        Q.qsgd_quantize_rows(x.double(), a, a_scale)
    with pytest.raises(Q.QsgdError, match="outside"):
        Q.qsgd_quantize_rows(x, a[:1].expand(4, 64), a_scale)


def test_a_layer_of_a_generation_step():
    """Projections in 8 bits, the cache in 4: each stage against its plain statement on what the stage before it gave."""
    rows, width, heads, kv_heads, dim, held = 3, 512, 8, 2, 128, [40, 1, 200]
    dtype = torch.bfloat16
    x = normal((rows, width), 1, dtype).cuda()
    w_in, s_in = Q.quantize_rows_alloc((normal(((heads + 2 * kv_heads) * dim, width), 2) * width ** -0.5).cuda())
    w_out, s_out = Q.quantize_rows_alloc((normal((width, heads * dim), 3) * (heads * dim) ** -0.5).cuda())
    n_pages = 20
    cache = Q.Cache(n_pages, 16, kv_heads, dim, dtype)
    table = torch.randperm(n_pages, generator=torch.Generator().manual_seed(1))[:3 * 1 + 13 + 3].to(torch.int32)
    rows_of = torch.zeros(3, 13, dtype=torch.int32)
    rows_of[0, :3], rows_of[1, :1], rows_of[2, :13] = table[:3], table[3:4], table[4:17]
    rows_of = rows_of.cuda()
    status = Q.new_status()
    old_k, old_v = ([normal((n - 1, kv_heads, dim), 10 * i + n, dtype) for n in held] for i in (1, 2))
    before = [n - 1 for n in held]
    starts = torch.tensor([0, before[0], before[0] + before[1], sum(before)], dtype=torch.int32).cuda()
    Q.qsgd_cache_write(cache, rows_of, torch.tensor(before, dtype=torch.int32).cuda(), torch.cat(old_k).cuda(), torch.cat(old_v).cuda(), status,
                       starts=starts)
    lengths = torch.tensor(held, dtype=torch.int32).cuda()
    ws_in, ws_out = (torch.empty(Q.qsgd_linear_i8_workspace_bytes(rows, c), dtype=torch.uint8, device="cuda") for c in (width, heads * dim))
    ws = torch.empty(Q.qsgd_cache_attend_workspace_bytes(cache, heads), dtype=torch.uint8, device="cuda")
    qkv = torch.empty(rows, heads + 2 * kv_heads, dim, dtype=dtype, device="cuda")
    mixed, out = torch.empty(rows, heads, dim, dtype=dtype, device="cuda"), torch.empty(rows, width, dtype=dtype, device="cuda")
    Q.qsgd_linear_i8(x, w_in, s_in, qkv.view(rows, -1), ws_in)
    q, k, v = qkv.split([heads, kv_heads, kv_heads], 1)
    Q.qsgd_cache_write(cache, rows_of, lengths, k, v, status)
    Q.qsgd_cache_attend(cache, rows_of, lengths, q, mixed, ws, status)
    Q.qsgd_linear_i8(mixed.view(rows, -1), w_out, s_out, out, ws_out)
    assert int(status.item()) == 0
    for given, w, s, got in ((x, w_in, s_in, qkv.view(rows, -1)), (mixed.view(rows, -1), w_out, s_out, out)):
        codes, scale = F.quantize_rows(given.cpu())
        check(got.cpu(), codes, scale.float(), w.cpu(), s.cpu(), None, dtype)
    for b in range(rows):
        kk = F.held_value(torch.cat([old_k[b], k[b: b + 1].cpu()]))
        vv = F.held_value(torch.cat([old_v[b], v[b: b + 1].cpu()]))
        ref, _, mean = F.attend(q[b: b + 1].cpu(), kk, vv, 1 / math.sqrt(dim), held[b], 1)
        off = (mixed[b: b + 1].cpu().double() - ref).abs()
        # scores of at most a few units, off by less than 2^-9 (the bound of the cache's own tests); p by twice that
        assert bool((off <= F.HALF_STEP[dtype] * ref.abs() + 2.0 ** -8 * mean + 1e-7).all())
