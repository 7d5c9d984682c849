"""What the 4-bit cache holds and gives back, against rational numbers: the nearest code and one rounding, where 32 bits do not hold the
differences and sums on the way."""
import math
from fractions import Fraction

import pytest
import torch

import paper_1610_02132_b200 as Q

BF16, FP16 = torch.bfloat16, torch.float16


def next_number(v, dtype, by):
    t = torch.tensor(v, dtype=dtype)
    return float((t.view(torch.int16) + by).view(dtype))


def group_of(x):
    """lo, step and codes of 64 values, in rational numbers: step the smallest number of the type with 15 * step >= span, a code the number
    of borders lo + (i + 1/2) * step below the value."""
    v = [Fraction(float(e)) for e in x]
    lo, span = min(v), max(v) - min(v)
    step = float(torch.tensor(float(span / 15), dtype=torch.float64).to(x.dtype))
    while 15 * Fraction(step) < span:
        step = next_number(step, x.dtype, 1)
    while step > 0 and 15 * Fraction(next_number(step, x.dtype, -1)) >= span:
        step = next_number(step, x.dtype, -1)
    s = Fraction(step)
    return lo, s, [sum(1 for i in range(15) if e - lo > (i + Fraction(1, 2)) * s) for e in v]


def rounded(v, dtype):
    """A rational number as the nearest of the type, the even one of two as near."""
    near = float(torch.tensor(float(v), dtype=torch.float64).to(dtype))
    best = None
    for by in (-1, 0, 1):
        if near == 0 and by:
            continue
        c = next_number(near, dtype, by)
        if not math.isfinite(c):
            continue
        odd = int(torch.tensor(c, dtype=dtype).view(torch.int16)) & 1
        if best is None or (abs(Fraction(c) - v), odd) < best[0]:
            best = (abs(Fraction(c) - v), odd), c
    return best[1]


def groups(dtype):
    """Groups with values beside a border, by less than 32 bits hold beside the difference to the smallest one."""
    tiny = [1e-7, 6e-8, 1e-38, 2.0 ** -24] if dtype == BF16 else [1e-7, 6e-8, 2.0 ** -24, 2.0 ** -23]
    out = []
    g = torch.Generator().manual_seed(7)
    for t in tiny:
        for sign in (1, -1):
            x = torch.zeros(64)
            x[0], x[1], x[2:30], x[30:] = -7.5, 7.5, sign * t, torch.randint(-7, 8, (34,), generator=g).float()
            out.append(x)                                   # step 1, borders at the whole numbers: zero's neighbours
            x = torch.zeros(64)
            # the smallest value next to zero, and values where the borders would be if it were zero (steps 1.96875 and 2.015625)
            x[0], x[1], x[2:20], x[20:] = (sign * t, 29.5, 2.953125, 0.984375) if dtype == BF16 else (sign * t, 30.21875, 5.0390625, 3.0234375)
            out.append(x)
    for k in (3, 5, 11):                                    # symmetric groups of other steps
        x = torch.randn(64, generator=g).to(dtype).float()
        x[0], x[1] = -k * 0.3125, k * 0.3125
        x = x.clamp(-k * 0.3125, k * 0.3125)
        x[2:20] = torch.randn(18, generator=g) * 2.0 ** -torch.randint(10, 40 if dtype == BF16 else 24, (18,), generator=g).float()
        out.append(x)
    return torch.stack(out).to(dtype)


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_groups_are_what_they_are_meant_to_be(dtype):
    """Each of the first ones has a value whose code the difference in 32 bits would not give."""
    differ = 0
    for x in groups(dtype)[:16]:
        lo, s, codes = group_of(x)
        short = (x.float() - x.float().min()).tolist()
        differ += any(sum(1 for i in range(15) if Fraction(d) > (i + Fraction(1, 2)) * s) != c for d, c in zip(short, codes))
    assert differ >= 6


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("dim", [64, 128])
def test_codes_are_the_nearest(dtype, dim):
    x = groups(dtype)
    want = [group_of(g) for g in x]
    tokens = -(-x.shape[0] * 64 // dim // 16) * 16
    k = torch.zeros(tokens * dim, dtype=dtype)
    k[: x.numel()] = x.flatten()
    k = k.view(tokens, 1, dim)
    cache = Q.Cache(1, tokens, 1, dim, dtype)
    table, lengths = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.tensor([tokens], dtype=torch.int32, device="cuda")
    starts, status = torch.tensor([0, tokens], dtype=torch.int32, device="cuda"), Q.new_status()
    Q.qsgd_cache_write(cache, table, lengths, k.cuda(), k.flip(0).cuda(), status, starts=starts)
    k2, v2 = torch.zeros(2, tokens, 1, dim, dtype=dtype, device="cuda")
    Q.qsgd_cache_read(cache, table, lengths, k2, v2, status, starts=starts)
    assert int(status.item()) == 0
    assert torch.equal(k2, v2.flip(0))
    tile = cache.data.cpu().view(tokens // 16, 18 * dim)
    wrong = []
    for i, (lo, step, codes) in enumerate(want):
        token, j = divmod(i, dim // 64)
        held = tile[token // 16, : 8 * dim].view(dim // 64, 16, 32)[j, token % 16]
        got = torch.stack([held & 15, held >> 4], -1).flatten().tolist()
        pair = tile[token // 16, 8 * dim: 9 * dim].view(dtype).view(16, dim // 64, 2)[token % 16, j]
        assert Fraction(float(pair[0])) == lo and Fraction(float(pair[1])) == step
        wrong += [(i, n, a, b) for n, (a, b) in enumerate(zip(got, codes)) if a != b]
    assert not wrong, wrong[:5]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_values_read_back_are_rounded_once(dtype):
    """lo far below step: step * code between two numbers of the type, and lo, beyond 32 bits, says which."""
    pairs = []
    for step in (1.0078125, 1.4921875, 129 / 64, 1.1640625) if dtype == BF16 else (1.0009765625, 1025 / 512, 1.2490234375, 1.0029296875):
        for lo in (2.0 ** -30, -2.0 ** -30, 2.0 ** -40, -2.0 ** -126, 0.0, 2.0 ** -12) if dtype == BF16 else (2.0 ** -24, -2.0 ** -24, 2.0 ** -14, 0.0):
            for size in (1.0, 64.0, -1.0) if dtype == BF16 else (1.0, 512.0, -1.0):
                if size > 0:
                    pairs.append((lo, step * size))
    pairs += [(3.0, 0.0), (-1.0, 2.0), (-0.125, 2.0 ** -9), (1000.0, 0.25)]
    tokens = -(-len(pairs) // 16) * 16
    cache = Q.Cache(1, tokens, 1, 64, dtype)
    data = torch.zeros(tokens // 16, 18 * 64, dtype=torch.uint8)
    for i, (lo, step) in enumerate(pairs):
        tile, slot = divmod(i, 16)
        codes = torch.arange(64) % 16
        for at in (0, 576):
            data[tile, at + slot * 32: at + slot * 32 + 32] = (codes[0::2] | codes[1::2] << 4).to(torch.uint8)
            data[tile, at + 512 + 4 * slot: at + 516 + 4 * slot] = torch.tensor([lo, step], dtype=dtype).view(torch.uint8)
    cache.data.copy_(data.view(1, 1, -1))
    table, lengths = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.tensor([tokens], dtype=torch.int32, device="cuda")
    starts, status = torch.tensor([0, tokens], dtype=torch.int32, device="cuda"), Q.new_status()
    k, v = torch.zeros(2, tokens, 1, 64, dtype=dtype, device="cuda")
    Q.qsgd_cache_read(cache, table, lengths, k, v, status, starts=starts)
    assert int(status.item()) == 0 and torch.equal(k, v)
    wrong = []
    for i, (lo, step) in enumerate(pairs):
        lo, step = (Fraction(float(torch.tensor(e, dtype=dtype))) for e in (lo, step))
        want = [rounded(lo + step * (c % 16), dtype) for c in range(64)]
        wrong += [(float(lo), float(step), c, a, b) for c, (a, b) in enumerate(zip(k[i, 0].tolist(), want)) if a != b]
    assert not wrong, wrong[:5]
