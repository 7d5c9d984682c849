"""The 4-bit cache against its plain statement: bytes and values are equal, attention within the bounds of its roundings."""
import math
import random

import pytest
import torch

import few_bits as F
import paper_1610_02132_b200 as Q

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16


def values(shape, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    mean = torch.randn(shape[1:], generator=g)
    return (torch.randn(shape, generator=g) * (0.1 + torch.rand(shape[1:], generator=g)) + mean).to(dtype)


class Filled:
    """A cache with random pages behind every sequence and bytes that read as NaN wherever nothing was written."""

    def __init__(self, lengths, page, heads, dim, dtype, seed=0, spare=2, layout="pages"):
        self.lengths, self.page = lengths, page
        pages = [-(-n // page) for n in lengths]
        n = sum(pages) + spare
        one = page // 16 * 18 * dim
        if layout == "pages":
            data = torch.full((n, heads, one), 255, dtype=torch.uint8, device="cuda")
        elif layout == "heads":                             # heads outermost
            data = torch.full((heads, n, one), 255, dtype=torch.uint8, device="cuda").transpose(0, 1)
        else:                                               # room between pages and heads
            data = torch.full((n, heads + 1, one + 48), 255, dtype=torch.uint8, device="cuda")[:, :heads, :one]
        self.cache = Q.Cache(n, page, heads, dim, dtype, data=data)
        order = torch.randperm(n, generator=torch.Generator().manual_seed(seed))
        table = torch.full((len(lengths), max(pages + [1])), -7, dtype=torch.int32)
        at = 0
        for b, m in enumerate(pages):
            table[b, :m] = order[at: at + m].to(torch.int32)
            at += m
        self.table_host, self.table = table, table.cuda()
        self.len = torch.tensor(lengths, dtype=torch.int32).cuda()
        self.status = Q.new_status()
        self.k = [values((m, heads, dim), dtype, 100 + 2 * b + seed) for b, m in enumerate(lengths)]
        self.v = [values((m, heads, dim), dtype, 101 + 2 * b + seed) for b, m in enumerate(lengths)]

    def write_all(self):
        k, v = torch.cat(self.k).cuda(), torch.cat(self.v).cuda()
        Q.qsgd_cache_write(self.cache, self.table, self.len, k, v, self.status, starts=starts_of(self.lengths))
        return self

    def fine(self):
        assert int(self.status.item()) == 0


def starts_of(runs):
    return torch.tensor([sum(runs[:i]) for i in range(len(runs) + 1)], dtype=torch.int32).cuda()


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("dim, heads, page, layout", [(64, 1, 16, "pages"), (128, 3, 32, "heads"), (192, 2, 16, "gaps"), (256, 2, 48, "pages")])
def test_written_bytes(dtype, dim, heads, page, layout):
    """Every byte of whole pages, and not one byte elsewhere."""
    lengths = [page, 2 * page]
    f = Filled(lengths, page, heads, dim, dtype, layout=layout).write_all()
    f.fine()
    before = torch.full_like(f.cache.data, 255)
    for b, n in enumerate(lengths):
        for i in range(n // page):
            for h in range(heads):
                part = slice(i * page, (i + 1) * page)
                want = torch.from_numpy(F.cache_bytes(f.k[b][part, h], f.v[b][part, h]).copy())
                before[int(f.table_host[b, i]), h] = want.cuda()
    assert torch.equal(f.cache.data, before)
    if f.cache.data._base is not None and layout == "gaps":
        base = f.cache.data._base
        assert bool((base[:, heads:] == 255).all()) and bool((base[:, :, -48:] == 255).all())


SPECIAL = ["equal", "zero", "huge", "tiny", "inf", "nan", "one", "ties", "negative zero"]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("kind", SPECIAL)
def test_values_of_every_sort(dtype, kind):
    x = values((16, 1, 128), dtype, 5)
    big, small = (3e38, 1e-40) if dtype == BF16 else (65504.0, 6e-8)
    if kind == "equal": x[:] = 0.3
    if kind == "zero": x[:] = 0
    if kind == "huge": x[:, :, ::2], x[:, :, 1::2], x[3, 0, :64] = big, -big, big
    if kind == "tiny": x = (x.float() * small).to(dtype)
    if kind == "inf": x[2, 0, 70], x[9, 0, 3] = math.inf, -math.inf
    if kind == "nan": x[2, 0, 70] = math.nan
    if kind == "one": x[:] = 0; x[:, :, 5] = 1.0; x[:, :, 100] = -1.0
    if kind == "ties": x[:] = (torch.arange(128) % 31).to(dtype)
    if kind == "negative zero": x[:] = -0.0; x[:, :, 1::2] = 0.0
    f = Filled([16], 16, 1, 128, dtype)
    f.k, f.v = [x], [values((16, 1, 128), dtype, 6)]
    f.write_all()
    want = torch.from_numpy(F.cache_bytes(x[:, 0], f.v[0][:, 0]).copy()).cuda()
    got = f.cache.data[int(f.table_host[0, 0]), 0]
    if kind in ("inf", "nan", "huge"):                      # of a NaN only that it is one is said
        assert torch.equal(got[:1024], want[:1024]) and torch.equal(got[1152:], want[1152:])
    else:
        assert torch.equal(got, want)
    k, v = torch.zeros(2, 16, 1, 128, dtype=dtype, device="cuda")
    Q.qsgd_cache_read(f.cache, f.table, f.len, k, v, f.status, starts=starts_of([16]))
    f.fine()
    held = F.held_value(x)
    assert torch.equal(k.cpu().nan_to_num(7.0, 8.0, 9.0), held.float().to(dtype).nan_to_num(7.0, 8.0, 9.0))


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("dim, heads, page, lengths", [(64, 2, 16, [1, 0, 17, 33]), (128, 8, 64, [5, 200, 64, 1, 0]), (192, 1, 32, [100]),
                                                       (256, 4, 16, [15, 16, 31]), (128, 1, 16, [2500])])
def test_read_back(dtype, dim, heads, page, lengths):
    f = Filled(lengths, page, heads, dim, dtype, layout="gaps").write_all()
    held = torch.cat([F.held_value(x) for x in f.k + f.v])
    total = sum(lengths)
    k = torch.full((total + 3, heads + 1, dim + 8), 42.0, dtype=dtype, device="cuda")     # a view with room on all sides
    v = torch.full((heads, total + 3, dim), 42.0, dtype=dtype, device="cuda").transpose(0, 1)      # heads outermost
    Q.qsgd_cache_read(f.cache, f.table, f.len, k[:, :heads, :dim], v, f.status, starts=starts_of(lengths))
    f.fine()
    want = held.float().to(dtype).cuda()
    assert torch.equal(k[:total, :heads, :dim], want[:total]) and torch.equal(v[:total], want[total:])
    assert bool((k[total:] == 42).all()) and bool((k[:, heads:] == 42).all()) and bool((k[:, :, dim:] == 42).all()) and bool((v[total:] == 42).all())
    # the last token of each, one row a sequence
    if all(lengths):
        k1, v1 = torch.zeros(2, len(lengths), heads, dim, dtype=dtype, device="cuda")
        Q.qsgd_cache_read(f.cache, f.table, f.len, k1, v1, f.status)
        last = torch.tensor(lengths).cumsum(0) - 1
        assert torch.equal(k1, want[:total][last]) and torch.equal(v1, want[total:][last])


def test_more_rows_than_tokens():
    """Rows in front of a sequence's first token are not written, and read back as zero."""
    f = Filled([3, 2], 16, 2, 64, BF16)
    runs, rows = [5, 2], 7
    k, v = values((rows, 2, 64), BF16, 1), values((rows, 2, 64), BF16, 2)
    Q.qsgd_cache_write(f.cache, f.table, f.len, k.cuda(), v.cuda(), f.status, starts=starts_of(runs))
    k2, v2 = torch.full((2, rows, 2, 64), 9.0, dtype=BF16, device="cuda")
    Q.qsgd_cache_read(f.cache, f.table, f.len, k2, v2, f.status, starts=starts_of(runs))
    f.fine()
    for got, x in ((k2, k), (v2, v)):
        want = F.held_value(x).float().to(BF16)
        want[:2] = 0
        assert torch.equal(got.cpu(), want)


def check(out, lse, q, ks, vs, scale, lengths, runs, dtype, wide=False):
    """Bounds. A score: 64 products summed per group in fp32, each at most |q| * (128 + 15) * step (less with centred codes): 68 roundings
    or truncations of 2^-23 of sum |q| * 143 * step, which also covers 2^-17 * 2^-11 of the largest |q| for numbers of q that fp16 does not hold
    exactly, and a few of 2^-22 of the score; p then differs by twice that and by 2^-19 for its exponential and the sums. p * step is rounded to
    fp16, half a step of 2^-11 (for an fp16 output the rest follows: 2^-22), and multiplied by |c - 8| <= 8. The output adds half a step of its type. wide: keys, values and p are rounded to fp16 instead, half a step of 2^-11 of each."""
    at, worst, num, den = 0, 0.0, 0.0, 0.0
    for b, (n, r) in enumerate(zip(lengths, runs)):
        if r == 0:
            continue
        k, v = F.held_value(ks[b]), F.held_value(vs[b])
        qq = q[at: at + r].cpu()
        ref, ref_lse, mean = F.attend(qq, k, v, scale, n, r)
        if n:
            x = ks[b].double().unflatten(-1, (-1, 64))
            step = ((x.amax(-1) - x.amin(-1)) / 15).amax(0) * 1.01                                    # [kv head, group]
            group = qq.shape[1] // step.shape[0]
            asum = qq.double().abs().unflatten(-1, (-1, 64)).sum(-1)                                  # [row, head, group]
            reach = (k.abs().amax(0).repeat_interleave(group, 0)[None] * qq.double().abs()).sum(-1)   # [row, head]: of a score
            err = abs(scale) * ((asum * step.repeat_interleave(group, 0)[None]).sum(-1) * 143 * 68 * 2.0 ** -23 + reach * (2.0 ** -11 if wide else 2.0 ** -20))
        else:
            err = torch.zeros(r, qq.shape[1], dtype=torch.float64)
        y = vs[b].double().unflatten(-1, (-1, 64)) if n else torch.zeros(1, qq.shape[1], qq.shape[2] // 64, 64, dtype=torch.float64)
        width = ((y.amax(-1) - y.amin(-1)) / 15).amax(0) * 1.01                                       # [kv head, group]
        width = width.repeat_interleave(qq.shape[1] // width.shape[0], 0).repeat_interleave(64, 1)[None]
        rounded = (2.0 ** -11 if dtype == BF16 else 2.0 ** -22) * 8 * width
        if wide and n:
            rounded = 2.0 ** -11 * (v.abs().amax(0).repeat_interleave(qq.shape[1] // v.shape[1], 0)[None] + mean)
        tol = F.HALF_STEP[dtype] * ref.abs() + (2 * err[..., None] + 2.0 ** -19) * mean + rounded + 1e-7
        got, got_lse = out[at: at + r].cpu().double(), lse[at: at + r].cpu().double()
        assert bool(((got - ref).abs() <= tol).all()), ((got - ref).abs() / tol).max()
        empty = torch.isinf(ref_lse)
        assert torch.equal(got_lse[empty], ref_lse[empty]) and bool((got[empty] == 0).all())
        assert bool(((got_lse - ref_lse).abs()[~empty] <= (err + 2.0 ** -20 * (2 + ref_lse.abs()))[~empty]).all())
        num, den = num + float((got - ref).square().sum()), den + float(ref.square().sum())
        at += r
    assert math.sqrt(num) <= F.HALF_STEP[dtype] * math.sqrt(den)     # the roundings' mean is smaller than their bound


def run_attend(f, q_heads, runs, dtype, seed=3, scale=None, rows=None, one_each=False):
    total = sum(runs) if rows is None else rows
    dim = f.cache.head_dim
    q = values((total, q_heads, dim), dtype, seed).cuda()
    out = torch.full_like(q, 42.0)
    lse = torch.full((total, q_heads), 42.0, device="cuda")
    ws = torch.full((Q.qsgd_cache_attend_workspace_bytes(f.cache, q_heads),), 255, dtype=torch.uint8, device="cuda")
    Q.qsgd_cache_attend(f.cache, f.table, f.len, q, out, ws, f.status, starts=None if one_each else starts_of(runs), scale=scale, lse=lse)
    f.fine()
    return q, out, lse


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("dim", [64, 128, 192, 256])
@pytest.mark.parametrize("heads, group, page, lengths", [(1, 1, 16, [1]), (2, 4, 16, [16, 17, 0, 5]), (1, 8, 32, [300, 31]), (4, 3, 48, [129, 1, 64]),
                                                         (1, 12, 16, [500]), (1, 64, 16, [700, 90]), (3, 1, 256, [1000] * 3)])
def test_attend_single_tokens(dtype, dim, heads, group, page, lengths):
    f = Filled(lengths, page, heads, dim, dtype).write_all()
    q, out, lse = run_attend(f, heads * group, [1] * len(lengths), dtype, one_each=True)
    check(out, lse, q, f.k, f.v, 1 / math.sqrt(dim), lengths, [1] * len(lengths), dtype)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads, group, lengths, runs", [(2, 1, [20, 40], [20, 3]), (1, 4, [7, 100, 33], [7, 0, 17]), (2, 8, [70], [5]),
                                                         (1, 5, [2, 9], [6, 11])])
def test_attend_runs(dtype, dim, heads, group, lengths, runs):
    """Runs of queries, causal; also more queries than tokens, whose first rows see nothing."""
    f = Filled(lengths, 16, heads, dim, dtype).write_all()
    q, out, lse = run_attend(f, heads * group, runs, dtype, rows=sum(runs) + 2)
    check(out, lse, q, f.k, f.v, 1 / math.sqrt(dim), lengths, runs, dtype)
    assert bool((out[sum(runs):] == 42).all()) and bool((lse[sum(runs):] == 42).all())


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads, group, page, lengths, runs", [(1, 1, 16, [64], [64]), (1, 1, 16, [300], [129]), (2, 4, 64, [200, 65, 130], [70, 65, 33]),
                                                               (1, 8, 16, [5, 700, 0], [40, 33, 7]), (2, 3, 32, [1000, 63], [90, 1]), (1, 2, 48, [64, 128, 192], [32, 64, 96]),
                                                               (1, 12, 16, [17, 16, 2000], [17, 1, 20]), (4, 4, 128, [513], [257])])
def test_attend_chunks(dim, heads, group, page, lengths, runs):
    """Runs that are long enough for tiles of 128 rows; more queries than tokens among them."""
    f = Filled(lengths, page, heads, dim, BF16).write_all()
    assert sum(runs) * group >= 64 * len(runs)
    q, out, lse = run_attend(f, heads * group, runs, BF16, rows=sum(runs) + 2)
    check(out, lse, q, f.k, f.v, 1 / math.sqrt(dim), lengths, runs, BF16, wide=True)
    assert bool((out[sum(runs):] == 42).all()) and bool((lse[sum(runs):] == 42).all())


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads, group, page, lengths, runs", [(28, 4, 16, [300], [129]), (24, 4, 64, [200, 65, 130], [70, 65, 33]), (48, 8, 16, [5, 700, 0], [40, 33, 7]),
                                                               (24, 12, 16, [17, 16, 2000], [17, 9, 30]), (49, 2, 48, [64, 128, 192], [30, 64, 96]),
                                                               (49, 1, 128, [513], [380])])
def test_attend_chunks_that_fill_the_device(dim, heads, group, page, lengths, runs):
    """Rows enough for a tile of 128 to nearly every SM: one kernel, without a second one that joins parts."""
    f = Filled(lengths, page, heads, dim, BF16).write_all()
    torch.cuda.synchronize()
    before = Q.qsgd_launch_count()
    q, out, lse = run_attend(f, heads * group, runs, BF16, rows=sum(runs) + 2)
    assert Q.qsgd_launch_count() - before == 1
    check(out, lse, q, f.k, f.v, 1 / math.sqrt(dim), lengths, runs, BF16, wide=True)
    assert bool((out[sum(runs):] == 42).all()) and bool((lse[sum(runs):] == 42).all())


@pytest.mark.parametrize("heads", [1, 74])
@pytest.mark.parametrize("size_k, size_v", [(1e30, 1e30), (1e-30, 1e-36), (1.0, 3e37), (1e4, 1e-4)])
def test_attend_chunks_of_all_sizes(size_k, size_v, heads):
    """bf16 numbers far outside fp16's range, and tokens of very different sizes side by side."""
    f = Filled([400], 16, heads, 128, BF16)
    sizes = torch.ones(400)
    sizes[100:200] = 1e-4
    f.k[0] = (f.k[0].float() * size_k * sizes[:, None, None]).to(BF16)
    f.v[0] = (f.v[0].float() * size_v * sizes.flip(0)[:, None, None]).to(BF16)
    f.write_all()
    q, out, lse = run_attend(f, 2 * heads, [100], BF16, scale=0.1 / size_k if size_k < 1e20 else 0.0)
    ref, ref_lse, mean = F.attend(q.cpu(), F.held_value(f.k[0]), F.held_value(f.v[0]), 0.1 / size_k if size_k < 1e20 else 0.0, 400, 100)
    err = 0.1 * q.cpu().double().abs().sum(-1, keepdim=True) * 8 * 2.0 ** -11 if size_k < 1e20 else 0.0     # |k| below 8 sizes
    tol = F.HALF_STEP[BF16] * ref.abs() + (2 * err + 2.0 ** -10) * mean + 2.0 ** -11 * f.v[0].double().abs().max()
    assert bool(((out.cpu().double() - ref).abs() <= tol).all())


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("heads, group, dim, lengths", [(2, 4, 128, [20011, 3]), (1, 1, 64, [9000]), (1, 8, 256, [5000, 4999, 1])])
def test_attend_long(dtype, heads, group, dim, lengths):
    """Sequences that many CTAs share."""
    f = Filled(lengths, 64, heads, dim, dtype).write_all()
    q, out, lse = run_attend(f, heads * group, [1] * len(lengths), dtype, one_each=True)
    check(out, lse, q, f.k, f.v, 1 / math.sqrt(dim), lengths, [1] * len(lengths), dtype)


@pytest.mark.parametrize("what", ["huge", "huge and nearly equal", "tiny", "far from zero"])
@pytest.mark.parametrize("lengths, runs", [([9000, 40], [1, 1]), ([600], [1]), ([300, 90], [5, 9])])
def test_attend_values_of_all_sizes(what, lengths, runs):
    """Sums of p v that would not fit 32 bits before they are divided; steps far smaller than the values."""
    f = Filled(lengths, 16, 2, 128, BF16)
    for v in f.v:
        x = v.float()
        v.copy_({"huge": x * 3e37, "huge and nearly equal": 3e38 * (1 - x.abs() * 2.0 ** -8), "tiny": x * 1e-33, "far from zero": 1000 + x}[what])
    f.write_all()
    q, out, lse = run_attend(f, 8, runs, BF16, one_each=max(runs) == 1)
    size = 2.0 ** -100 if "huge" in what else 2.0 ** 100 if what == "tiny" else 1.0
    check(out.double() * size, lse, q, f.k, [(v.double() * size).to(BF16) for v in f.v], 1 / math.sqrt(128), lengths, runs, BF16)     # (exactly)


def test_attend_many_sequences():
    """More sequences than threads of a CTA, some of them empty."""
    lengths = [(7 * i) % 23 for i in range(700)]
    f = Filled(lengths, 16, 1, 64, BF16).write_all()
    q, out, lse = run_attend(f, 2, [1] * 700, BF16, one_each=True)
    check(out, lse, q, f.k, f.v, 0.125, lengths, [1] * 700, BF16)


def test_attend_scales():
    """Large scores (one token takes all), a scale of zero (the mean), a negative one."""
    f = Filled([200], 16, 1, 128, BF16).write_all()
    for scale in (0.0, -0.1, 1.0):
        q, out, lse = run_attend(f, 4, [1], BF16, scale=scale, one_each=True)
        check(out, lse, q, f.k, f.v, scale, [200], [1], BF16)


def test_attend_strided_and_without_lse():
    f = Filled([90, 40], 16, 2, 128, BF16, layout="heads").write_all()
    wide = values((2, 4 + 2 + 2, 128), BF16, 8).cuda()      # queries, keys and values of one projection
    out = torch.full((4, 2, 128 + 8), 42.0, dtype=BF16, device="cuda")
    o = out.transpose(0, 1)[:, :, :128]
    ws = torch.empty(Q.qsgd_cache_attend_workspace_bytes(f.cache, 4), dtype=torch.uint8, device="cuda")
    Q.qsgd_cache_attend(f.cache, f.table, f.len, wide[:, :4], o, ws, f.status)
    whole, lse = torch.empty(2, 4, 128, dtype=BF16, device="cuda"), torch.empty(2, 4, device="cuda")
    Q.qsgd_cache_attend(f.cache, f.table, f.len, wide[:, :4].contiguous(), whole, ws, f.status, lse=lse)
    f.fine()
    assert torch.equal(o, whole) and bool((out[:, :, 128:] == 42).all())
    check(whole, lse, wide[:, :4], f.k, f.v, 1 / math.sqrt(128), [90, 40], [1, 1], BF16)


@pytest.mark.parametrize("n, dim, heads", [(40, 128, 1), (100, 128, 1), (100, 64, 1), (100, 128, 148), (100, 64, 148)])
def test_poisoned_tokens(n, dim, heads):
    """A key that is not finite makes the rows that see it NaN and no others; a value that is not finite, its group of coordinates."""
    f = Filled([n], 16, heads, dim, BF16)
    f.k[0][30, :, 5] = math.inf
    f.v[0][20, :, dim - 58] = math.nan
    f.write_all()
    q, out, lse = run_attend(f, heads, [n], BF16)
    nan = out.isnan()[:, heads // 2]
    assert torch.equal(out.isnan(), nan[:, None].expand(-1, heads, -1))
    assert bool(nan[30:].all()) and not bool(nan[:20].any()) and not bool(nan[20:30, : dim - 64].any()) and bool(nan[20:30, dim - 64:].all())
    assert torch.equal(lse.isnan(), (torch.arange(n).cuda() >= 30)[:, None].expand(-1, heads))
    check(out[:20], lse[:20], q[:20], [f.k[0][:20]], [f.v[0][:20]], 1 / math.sqrt(dim), [20], [20], BF16, wide=n >= 64)


@pytest.mark.parametrize("what", ["page below", "page above", "length", "negative length", "starts"])
def test_places_that_the_cache_has_not(what):
    """They raise the flag, and the other sequences come out as before (but for rows that two sequences claim)."""
    lengths = [50, 40, 30]
    f = Filled(lengths, 16, 1, 64, BF16).write_all()
    starts = starts_of([1, 1, 1])
    q, good, lse = run_attend(f, 2, [1, 1, 1], BF16)
    k, v = torch.zeros(2, 3, 1, 64, dtype=BF16, device="cuda")
    Q.qsgd_cache_read(f.cache, f.table, f.len, k, v, f.status, starts=starts)
    good_k = k.clone()
    f.fine()
    before = f.cache.data.clone()
    if what == "page below": f.table[1, 2] = -1
    if what == "page above": f.table[1, 2] = f.cache.n_pages
    if what == "length": f.len[1] = 16 * f.table.shape[1] + 1
    if what == "negative length": f.len[1] = -3
    if what == "starts": starts[2] = 0
    out, ws = torch.empty_like(q), torch.empty(Q.qsgd_cache_attend_workspace_bytes(f.cache, 2), dtype=torch.uint8, device="cuda")
    for call in ("attend", "read", "write"):
        status = Q.new_status()
        if call == "attend":
            Q.qsgd_cache_attend(f.cache, f.table, f.len, q, out, ws, status, starts=starts)
        elif call == "read":
            Q.qsgd_cache_read(f.cache, f.table, f.len, k, v, status, starts=starts)
        else:
            Q.qsgd_cache_write(f.cache, f.table, f.len, k * 0, v * 0, status, starts=starts)
        assert int(status.item()) == Q.DEV_PAGE, call
    rows = [] if what == "starts" else [0, 2]
    # (where a sequence is split follows from all lengths: two results differ by a rounding each, of the type and of p * step, here below 2^-2)
    assert torch.allclose(out[rows].float(), good[rows].float(), rtol=2 * 2.0 ** -8, atol=2 * 2.0 ** -11 * 8 * 0.25)
    assert torch.equal(k[rows], good_k[rows])
    touched = (f.cache.data != before).flatten(1).any(1).nonzero().flatten().tolist()
    assert set(touched) <= {int(p) for p in f.table_host.flatten() if p >= 0}


@pytest.mark.parametrize("what", ["page below", "page above", "length", "negative length", "starts"])
def test_places_that_the_cache_has_not_in_chunks(what):
    """The same where a tile of 128 rows has all tokens: the other sequences' rows are the same to the bit."""
    f = Filled([50, 40, 35], 16, 48, 128, BF16).write_all()
    starts = starts_of([32, 32, 32])
    q, good, lse = run_attend(f, 192, [32, 32, 32], BF16)
    if what == "page below": f.table[1, 2] = -1
    if what == "page above": f.table[1, 2] = f.cache.n_pages
    if what == "length": f.len[1] = 16 * f.table.shape[1] + 1
    if what == "negative length": f.len[1] = -3
    if what == "starts": starts[2] = 20
    big = torch.full((96 + 8, 192, 128), 42.0, dtype=BF16, device="cuda")
    ws, status = torch.empty(Q.qsgd_cache_attend_workspace_bytes(f.cache, 192), dtype=torch.uint8, device="cuda"), Q.new_status()
    before = Q.qsgd_launch_count()
    Q.qsgd_cache_attend(f.cache, f.table, f.len, q, big[:96], ws, status, starts=starts)
    assert Q.qsgd_launch_count() - before == 1
    assert int(status.item()) == Q.DEV_PAGE
    assert bool((big[96:] == 42).all())
    if what != "starts":
        assert torch.equal(big[:32], good[:32]) and torch.equal(big[64:96], good[64:])


def test_far_pages():
    """Pages whose bytes lie beyond 32 bits of offset."""
    page, heads, dim = 64, 8, 256
    one = Q.qsgd_cache_page_bytes(page, heads, dim)
    n = (5 << 30) // one
    f = Filled([200, 70], page, heads, dim, BF16, spare=n)
    assert f.cache.data.nbytes > 1 << 32
    far = [n - 1, 3, n - 7, n - 20, 1, n - 2]
    f.table_host[0, :4] = torch.tensor(far[:4])
    f.table_host[1, :2] = torch.tensor(far[4:])
    f.table.copy_(f.table_host)
    f.write_all()
    q, out, lse = run_attend(f, 16, [1, 1], BF16, one_each=True)
    check(out, lse, q, f.k, f.v, 1 / 16, [200, 70], [1, 1], BF16)
    k, v = torch.zeros(2, 270, heads, dim, dtype=BF16, device="cuda")
    Q.qsgd_cache_read(f.cache, f.table, f.len, k, v, f.status, starts=starts_of([200, 70]))
    assert torch.equal(k.cpu(), F.held_value(torch.cat(f.k)).float().to(BF16))
    f.fine()


def test_a_generation_in_a_graph():
    """Write and attend captured once, replayed as the sequences grow; beside it another graph with a workspace of its own."""
    f = Filled([64, 64], 16, 2, 128, BF16).write_all()
    new_k, new_v = values((20, 2, 2, 128), BF16, 50), values((20, 2, 2, 128), BF16, 51)
    q = values((2, 4, 128), BF16, 52).cuda()
    k, v, out = torch.zeros(2, 2, 128, dtype=BF16, device="cuda"), torch.zeros(2, 2, 128, dtype=BF16, device="cuda"), torch.zeros_like(q)
    lse = torch.zeros(2, 4, device="cuda")
    out2 = torch.zeros_like(q)
    ws, ws2 = (torch.empty(Q.qsgd_cache_attend_workspace_bytes(f.cache, 4), dtype=torch.uint8, device="cuda") for _ in range(2))
    lengths = [30, 44]
    f.len.copy_(torch.tensor(lengths))
    Q.qsgd_cache_write(f.cache, f.table, f.len, k, v, f.status)          # (the first calls look up launch facts)
    Q.qsgd_cache_attend(f.cache, f.table, f.len, q, out, ws, f.status, lse=lse)
    torch.cuda.synchronize()
    graphs = []
    for o, w in ((out, ws), (out2, ws2)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            if o is out:
                Q.qsgd_cache_write(f.cache, f.table, f.len, k, v, f.status)
            Q.qsgd_cache_attend(f.cache, f.table, f.len, q, o, w, f.status, lse=lse if o is out else None)
        graphs.append(g)
    keys, vals = [x[:n].clone() for x, n in zip(f.k, lengths)], [x[:n].clone() for x, n in zip(f.v, lengths)]
    # (the call above wrote zeros at the last token)
    for b in range(2):
        keys[b][-1] = 0
        vals[b][-1] = 0
    side = torch.cuda.Stream()
    for i in range(4):
        f.len += 1
        lengths = [n + 1 for n in lengths]
        k.copy_(new_k[i])
        v.copy_(new_v[i])
        keys = [torch.cat([x, new_k[i, b: b + 1]]) for b, x in enumerate(keys)]
        vals = [torch.cat([x, new_v[i, b: b + 1]]) for b, x in enumerate(vals)]
        graphs[0].replay()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graphs[1].replay()
        torch.cuda.synchronize()
        f.fine()
        check(out, lse, q, keys, vals, 1 / math.sqrt(128), lengths, [1, 1], BF16)
        assert torch.equal(out, out2)


@pytest.mark.parametrize("lengths, runs, heads", [([900, 300], None, 2), ([9000], None, 2), ([300, 200], [100, 60], 2), ([300, 200], [100, 60], 24)])
def test_every_route_in_a_graph(lengths, runs, heads):
    """Clusters to a segment, the line of units with its second kernel, tiles of 128 rows: replayed with other queries and lengths."""
    f = Filled(lengths, 16, heads, 128, BF16).write_all()
    rows, starts = sum(runs or [1] * len(lengths)), starts_of(runs) if runs else None
    q, out = torch.zeros(rows, 4 * heads, 128, dtype=BF16, device="cuda"), torch.zeros(rows, 4 * heads, 128, dtype=BF16, device="cuda")
    ws = torch.empty(Q.qsgd_cache_attend_workspace_bytes(f.cache, 4 * heads), dtype=torch.uint8, device="cuda")
    Q.qsgd_cache_attend(f.cache, f.table, f.len, q, out, ws, f.status, starts=starts)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        Q.qsgd_cache_attend(f.cache, f.table, f.len, q, out, ws, f.status, starts=starts)
    for seed in (1, 2, 3):
        q.copy_(values((rows, 4 * heads, 128), BF16, seed))
        f.len.copy_(torch.tensor([n - 7 * seed for n in lengths], dtype=torch.int32))
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        again = torch.empty_like(out)
        Q.qsgd_cache_attend(f.cache, f.table, f.len, q, again, torch.empty_like(ws), f.status, starts=starts)
        assert torch.equal(out, again) and bool(out.isfinite().all())
    f.fine()


def test_given_stream_and_repeated_calls():
    f = Filled([3000], 16, 2, 128, FP16).write_all()
    torch.cuda.synchronize()
    q, out, lse = run_attend(f, 8, [1], FP16, one_each=True)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(5):
        again = torch.zeros_like(out)
        ws = torch.empty(Q.qsgd_cache_attend_workspace_bytes(f.cache, 8), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        Q.qsgd_cache_attend(f.cache, f.table, f.len, q, again, ws, f.status, stream=s)
        s.synchronize()
        assert torch.equal(again, out)


def test_both_kernels_and_a_product_on_several_streams():
    """Tiles of 128 rows of both head sizes, the line of units and an 8-bit layer side by side give what they give one after another."""
    cases = [(Filled([900, 500], 16, 24, dim, BF16, seed=dim).write_all(), [100, 64], 96) for dim in (64, 128)]
    cases.append((Filled([3000] * 4, 16, 8, 128, BF16, seed=3).write_all(), None, 32))
    calls = []
    for f, runs, heads in cases:
        q = values((sum(runs) if runs else 4, heads, f.cache.head_dim), BF16, 7).cuda()
        out, ws = torch.empty_like(q), torch.empty(Q.qsgd_cache_attend_workspace_bytes(f.cache, heads), dtype=torch.uint8, device="cuda")
        starts = starts_of(runs) if runs else None
        calls.append((out, lambda s, f=f, q=q, out=out, ws=ws, starts=starts: Q.qsgd_cache_attend(f.cache, f.table, f.len, q, out, ws, f.status,
                                                                                                  starts=starts, stream=s)))
    g = torch.Generator().manual_seed(1)
    x, w = torch.randn(70, 2048, generator=g).to(BF16).cuda(), torch.randint(-127, 128, (3000, 2048), generator=g).to(torch.int8).cuda()
    scale, y = torch.rand(3000, generator=g).cuda(), torch.empty(70, 3000, dtype=BF16, device="cuda")
    space = torch.empty(Q.qsgd_linear_i8_workspace_bytes(70, 2048), dtype=torch.uint8, device="cuda")
    calls.append((y, lambda s: Q.qsgd_linear_i8(x, w, scale, y, space, stream=s)))
    for _, call in calls:
        call(torch.cuda.current_stream())
    torch.cuda.synchronize()
    alone = [out.clone() for out, _ in calls]
    for out, _ in calls:
        out.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(20):
        for s, (_, call) in zip(streams, calls):
            call(s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, out) for a, (out, _) in zip(alone, calls))
    for f, _, _ in cases:
        f.fine()


@pytest.mark.parametrize("seed", range(16))
def test_attend_drawn_shapes(seed):
    r = random.Random(seed)
    dtype, dim, page = r.choice([BF16, BF16, FP16]), r.choice([64, 128, 192, 256]), r.choice([16, 32, 48, 64, 128])
    heads, group, n = r.choice([1, 2, 3, 8, 16, 25, 40]), r.choice([1, 2, 3, 4, 5, 8, 12, 16]), r.choice([1, 2, 3, 5, 9])
    lengths, most = [r.randint(0, r.choice([20, 100, 400, 1200])) for _ in range(n)], max(1, min(200, 40000 // (heads * group * n)))
    runs = [r.randint(0, most) for _ in range(n - 1)] + [r.randint(1, most)]
    f = Filled(lengths + [5], page, heads, dim, dtype, seed=seed).write_all()
    torch.cuda.synchronize()
    before = Q.qsgd_launch_count()
    q, out, lse = run_attend(f, heads * group, runs + [1], dtype, seed=seed, rows=sum(runs) + 1 + r.randint(0, 3))
    check(out, lse, q, f.k, f.v, 1 / math.sqrt(dim), lengths + [5], runs + [1], dtype, wide=Q.qsgd_launch_count() - before == 1)
    assert bool((out[sum(runs) + 1:] == 42).all())


def test_refusals():
    f = Filled([20, 20], 16, 2, 128, BF16).write_all()
    q = torch.zeros(2, 4, 128, dtype=BF16, device="cuda")
    ws = torch.empty(Q.qsgd_cache_attend_workspace_bytes(f.cache, 4), dtype=torch.uint8, device="cuda")
    good = dict(cache=f.cache, table=f.table, lengths=f.len, q=q, out=torch.empty_like(q), workspace=ws, status_dev=f.status)
    Q.qsgd_cache_attend(**good)
    base = torch.zeros(1 + 2 * 4 * 128, dtype=BF16, device="cuda")
    bad = [("q", q.half(), "element type"), ("q", q[:, :3], "multiple of the cache's 2 heads"), ("q", q[:, :, :64], "size 128 in dimension 2"),
           ("q", q[0], "3 dimensions"), ("q", q.cpu(), "CUDA tensor"), ("q", q[:1], "size 1 in dimension 0"),
           ("q", base[1:].view(2, 4, 128), "16-byte"), ("out", q.transpose(1, 2).contiguous().transpose(1, 2), "contiguous along"),
           ("out", q[:, :1].expand(2, 4, 128), "strides"), ("table", f.table.long(), "element type"), ("table", f.table[:1], "size 2 in dimension 0"),
           ("lengths", f.len.float(), "element type"), ("workspace", ws[:-1], "bytes"), ("workspace", ws[1:], "bytes"),
           ("starts", f.len, "size 3 in dimension 0"), ("lse", torch.zeros(2, 3, device="cuda"), "size 4 in dimension 1"),
           ("scale", math.nan, "outside"), ("status_dev", f.len.float(), "element type"), ("q", torch.cat([q, q]), "size 4 in dimension 0")]
    for name, value, said in bad:
        with pytest.raises(Q.QsgdError, match=said):
            Q.qsgd_cache_attend(**{**good, name: value})
    k = torch.zeros(2, 2, 128, dtype=BF16, device="cuda")
    for call in (Q.qsgd_cache_write, Q.qsgd_cache_read):
        with pytest.raises(Q.QsgdError, match="size 2 in dimension 1"):
            call(f.cache, f.table, f.len, k[:, :1], k, f.status)
        with pytest.raises(Q.QsgdError, match="rows or sequences"):
            call(f.cache, f.table, f.len, k[:1], k[:1], f.status)
    with pytest.raises(Q.QsgdError, match="strides"):
        Q.qsgd_cache_read(f.cache, f.table, f.len, k[:, :1].expand(2, 2, 128), k, f.status)
    f.fine()
