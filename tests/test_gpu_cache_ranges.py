"""Attention over the cache where keys, values and scores are of very different sizes: what a row gives follows from the tokens that it sees, each
with its weight, and from each group of coordinates by itself. Bounds are those of the roundings, of sums over what the row sees."""
import math

import pytest
import torch

import few_bits as F
import paper_1610_02132_b200 as Q
from test_gpu_cache import BF16, FP16, Filled, run_attend, starts_of, values

pytestmark = pytest.mark.gpu

SUBNORMAL = 2.0 ** -25                                      # half the distance of fp16's smallest numbers


def reference(f, b, q, scale, runs):
    """Of sequence b in fp64: out, lse, and sums over what a row sees with its weights p: of |v|, of the steps, and the largest p * size of a
    group. [rows, heads, dim or 1]. `err` bounds a score: see below."""
    k, v = F.held_value(f.k[b]), F.held_value(f.v[b])
    n, group = f.lengths[b], q.shape[1] // k.shape[1]
    g = f.v[b].double().unflatten(-1, (-1, 64))
    step, size = (g.amax(-1) - g.amin(-1)) / 15 * 1.01, torch.maximum((g.amax(-1) - g.amin(-1)) / 15 * 1.01, g.abs().amax(-1) / 1024)
    kg = f.k[b].double().unflatten(-1, (-1, 64))
    kstep = (kg.amax(-1) - kg.amin(-1)) / 15 * 1.01                                                    # [n, kv heads, groups]
    out = dict((name, []) for name in ("out", "lse", "mean", "steps", "most", "err"))
    for i in range(runs):
        m = n - runs + i + 1
        qq = q[i].double().cpu().unflatten(0, (-1, group))                                            # [kv heads, group, dim]
        s = torch.einsum("nkd,kgd->kgn", k[:m], qq) * scale
        p = torch.softmax(s, -1)
        # A score: as in the cache's own tests (rounded sums of |q| * 143 steps, 2^-20 of |q| |k|), but for each token, weighted; where rows of 128 share a
        # tile, keys in fp16: half a step of 2^-11 of |q| |k|, the sums' roundings, and of each group 2^-23 of |q| * the token's largest.
        reach = torch.einsum("nkd,kgd->kgn", k[:m].abs(), qq.abs())
        fine = torch.einsum("nkj,kgj->kgn", kstep[:m], qq.abs().unflatten(-1, (-1, 64)).sum(-1)) * 143 * 68 * 2.0 ** -23 + reach * 2.0 ** -20
        tile = reach * (2.0 ** -12 + 2.0 ** -16) + torch.einsum("nkj,kgj->kgn", k[:m].abs().unflatten(-1, (-1, 64)).amax(-1),
                                                                qq.abs().unflatten(-1, (-1, 64)).sum(-1)) * 2.0 ** -23
        out["err"].append(torch.stack([abs(scale) * (p * e).sum(-1).flatten() + abs(scale) * torch.where(p > 2.0 ** -40, e, 0.0).amax(-1).flatten()
                                       for e in (fine, tile)], -1))
        out["out"].append(torch.einsum("kgn,nkd->kgd", p, v[:m]).flatten(0, 1))
        out["mean"].append(torch.einsum("kgn,nkd->kgd", p, v[:m].abs()).flatten(0, 1))
        out["steps"].append(torch.einsum("kgn,nkj->kgj", p, step[:m]).flatten(0, 1).repeat_interleave(64, -1))
        out["most"].append((p[..., None] * size[:m].permute(1, 0, 2)[:, None]).amax(2).flatten(0, 1).repeat_interleave(64, -1))
        out["lse"].append(torch.logsumexp(s, -1).flatten())
    return {name: torch.stack(x) for name, x in out.items()}


def compare(f, q, out, lse, scale, runs, dtype, tile=False):
    """A coordinate is off by half a step of its type (2^-25, 2^-134 where that is one of the type's smallest numbers, multiples of twice that); by its weights' error, twice a score's and 2^-19, of the sum of p |v|; by the rounding of p * step
    to fp16 (half a step of 2^-11, of 2^-22 for an fp16 output), times |c - 8| <= 8, and where it is one of fp16's smallest numbers by half their distance,
    next to 64 for the largest p * size; in tiles of 128 rows p and v are rounded, 2^-11 together, and v's smallest are 2^-24 of their token's largest."""
    at = 0
    for b, r in enumerate(runs):
        ref = reference(f, b, q[at: at + r], scale, r)
        err = ref["err"][..., 1 if tile else 0, None]
        tol = F.HALF_STEP[dtype] * ref["out"].abs() + (2 * err + 2.0 ** -19) * ref["mean"] + (2.0 ** -25 if dtype == FP16 else 2.0 ** -134)
        small = 8 * f.lengths[b] * SUBNORMAL / 64 * 2 * ref["most"]
        if tile:
            tol += (2.0 ** -11 + 2.0 ** -16) * ref["mean"] + 2.0 ** -13 * 1024 * 16 * ref["most"] * 2.0 ** -10 + small
        else:
            tol += (2.0 ** -12 if dtype == BF16 else 2.0 ** -22) * 8 * ref["steps"] + small
        got = out[at: at + r].double().cpu()
        off = torch.where(ref["out"].isnan() & got.isnan(), 0.0, (got - ref["out"]).abs() / tol)      # (a value that is not finite: its group is not)
        assert bool((off <= 1).all()), (b, float(off.nan_to_num(math.inf).max()), (off.nan_to_num(math.inf) > 1).nonzero()[:3].tolist())
        tol = err[..., 0] + 2.0 ** -19 * (2 + ref["lse"].abs())
        assert bool(((lse[at: at + r].double().cpu() - ref["lse"]).abs() <= tol).all())
        at += r


def launched(f, heads, runs, dtype, scale=None, **more):
    torch.cuda.synchronize()
    before = Q.qsgd_launch_count()
    got = run_attend(f, heads, runs, dtype, scale=scale, **more)
    return (*got, Q.qsgd_launch_count() - before)


# (fp16 caches, sizes within the type)
@pytest.mark.parametrize("dtype, large, small", [(BF16, 1e7, 1.0), (BF16, 1e8, 1.0), (BF16, 1.0, 1e-30), (BF16, 1e30, 1e-30), (FP16, 1.2e4, 1e-3),
                                                 (FP16, 300.0, 3e-6)])
@pytest.mark.parametrize("dim", [128, 256])
@pytest.mark.parametrize("lengths, runs, one", [([2000], [1], True), ([9000, 300], [1, 1], True), ([500], [9], False)])
def test_groups_of_very_different_sizes(dtype, large, small, dim, lengths, runs, one):
    """A group of coordinates has an output of its own: what stands beside it does not blur it."""
    f = Filled(lengths, 16, 2, dim, dtype)
    sizes = torch.ones(dim // 64) * small
    sizes[0] = large
    for v in f.v:
        v.copy_((v.float().clamp(-4, 4) * sizes.repeat_interleave(64)).to(dtype))
    f.write_all()
    q, out, lse = run_attend(f, 8, runs, dtype, one_each=one)
    compare(f, q, out, lse, 1 / math.sqrt(dim), runs, dtype)


@pytest.mark.parametrize("dtype, large", [(BF16, 1e8), (BF16, 1e20), (FP16, 6e7)])
@pytest.mark.parametrize("place", [0, 40, 1990])
@pytest.mark.parametrize("dim", [64, 128])
def test_large_values_of_little_weight(dtype, large, place, dim):
    """A token whose values are large and whose score is low, before or behind the others: its products are small, and theirs are kept."""
    small = 1.0 if dtype == BF16 else 1e-3
    f = Filled([2000], 16, 1, dim, dtype)
    f.k[0].mul_(0.1)
    f.k[0][place] = -80.0 / dim * 4                         # q . k = -320 or so, scale 0.25: weight e^-80
    f.v[0].mul_(small)
    f.v[0][place] = (f.v[0][place].float() * large).to(dtype)
    f.write_all()
    q = values((1, 4, dim), dtype, 3).abs().clamp(0.5, 1.5).cuda()
    out, lse = torch.empty_like(q), torch.empty(1, 4, device="cuda")
    ws = torch.empty(Q.qsgd_cache_attend_workspace_bytes(f.cache, 4), dtype=torch.uint8, device="cuda")
    Q.qsgd_cache_attend(f.cache, f.table, f.len, q, out, ws, f.status, scale=0.25, lse=lse)
    f.fine()
    compare(f, q, out, lse, 0.25, [1], dtype)


@pytest.mark.parametrize("dtype, large", [(BF16, 1e8), (BF16, 1e30), (FP16, 3e7)])
@pytest.mark.parametrize("what", ["keys", "values"])
@pytest.mark.parametrize("dim, heads, group", [(128, 2, 4), (128, 148, 1), (64, 148, 1), (256, 2, 2)])
def test_what_a_row_does_not_see(dtype, large, what, dim, heads, group):
    """Later tokens of any size leave no trace in the rows in front of them (148 heads: tiles of 128 rows in bf16)."""
    small = 1.0 if dtype == BF16 else 1e-3
    f = Filled([150], 16, heads, dim, dtype)
    x = f.k[0] if what == "keys" else f.v[0]
    x.mul_(small)
    x[130:] = (x[130:].float() * large).to(dtype)
    f.write_all()
    scale = (1.0 if what == "values" or dtype == BF16 else 1e3) / math.sqrt(dim)
    q, out, lse, launches = launched(f, heads * group, [100], dtype, scale=scale)
    f.lengths, f.k, f.v = [130], [f.k[0][:130]], [f.v[0][:130]]
    compare(f, q[:80], out[:80], lse[:80], scale, [80], dtype, tile=launches == 1)


@pytest.mark.parametrize("heads", [2, 148])
@pytest.mark.parametrize("large", [2.0 ** 20, 2.0 ** 60])
@pytest.mark.parametrize("what", ["keys", "values", "groups"])
def test_tokens_of_very_different_sizes_in_chunks(what, large, heads):
    """Every other token, or group, much larger; its key points away from the queries, so that the others have the weight."""
    f = Filled([333], 16, heads, 128, BF16)
    if what == "keys":
        f.k[0].mul_(0.1)
        f.k[0][::2] = -(f.k[0][::2].float().abs() * large).to(BF16)
    if what == "values":
        f.k[0].mul_(0.1)
        f.k[0][::2] = (-20.0 * math.log2(large)) / 128
        f.v[0][::2] = (f.v[0][::2].float() * large).to(BF16)
    if what == "groups":
        f.v[0][..., :64] = (f.v[0][..., :64].float() * large).to(BF16)
    f.write_all()
    q = values((100, heads, 128), BF16, 3).abs().clamp(0.5, 1.5).cuda()
    out, lse = torch.empty_like(q), torch.empty(100, heads, device="cuda")
    ws = torch.empty(Q.qsgd_cache_attend_workspace_bytes(f.cache, heads), dtype=torch.uint8, device="cuda")
    before = Q.qsgd_launch_count()
    Q.qsgd_cache_attend(f.cache, f.table, f.len, q, out, ws, f.status, starts=starts_of([100]), scale=0.25, lse=lse)
    assert (Q.qsgd_launch_count() - before == 1) == (heads == 148)
    f.fine()
    compare(f, q, out, lse, 0.25, [100], BF16, tile=heads == 148)


@pytest.mark.parametrize("lengths, runs, heads, one", [([500], [1], 1, True), ([9000], [1], 1, True), ([300], [40], 2, False), ([333], [100], 148, False)])
def test_scores_far_below_zero(lengths, runs, heads, one):
    """All scores lower than any that a fixed number would stand for: the highest one still takes all."""
    f = Filled(lengths, 16, heads, 128, BF16)
    f.k[0][:] = -1e18
    f.k[0][::7] = -0.99e18                                  # (one group's worth of the same number: held as it is)
    f.write_all()
    rows = sum(runs)
    q = torch.full((rows, heads, 128), 1e15, dtype=BF16, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(rows, heads, device="cuda")
    ws = torch.empty(Q.qsgd_cache_attend_workspace_bytes(f.cache, heads), dtype=torch.uint8, device="cuda")
    Q.qsgd_cache_attend(f.cache, f.table, f.len, q, out, ws, f.status, starts=None if one else starts_of(runs), lse=lse)
    f.fine()
    v = F.held_value(f.v[0])
    for i in range(rows):
        n = lengths[0] - rows + i + 1
        want, size = v[0:n:7].mean(0), v[0:n:7].abs().mean(0)
        off = (out[i].double().cpu() - want).abs()
        assert bool((off <= F.HALF_STEP[BF16] * want.abs() + 2.0 ** -10 * size + 2.0 ** -11 * 8 * 0.5).all())
        assert bool(((lse[i].double().cpu() / (-0.9881e18 * 128 * 9.99e14 / math.sqrt(128)) - 1).abs() < 0.01).all())


@pytest.mark.parametrize("n", [1, 40, 64, 65, 128, 150, 192, 200, 256, 300, 330, 400, 449, 520])
@pytest.mark.parametrize("dim", [64, 128])
def test_every_number_of_steps_in_chunks(n, dim):
    """One to nine steps of 64 tokens: the two halves of a tile's softmax have as many, or one has one more. Each ten times, to the bit."""
    f = Filled([n], 16, 296, dim, BF16).write_all()
    runs = [min(n, 128)] if n >= 100 else [128]             # (more rows than tokens: the first see nothing)
    q, out, lse, launches = launched(f, 296, runs, BF16)
    assert launches == 1
    ws = torch.empty(Q.qsgd_cache_attend_workspace_bytes(f.cache, 296), dtype=torch.uint8, device="cuda")
    for _ in range(10):
        again = torch.empty_like(out)
        Q.qsgd_cache_attend(f.cache, f.table, f.len, q, again, ws, f.status, starts=starts_of(runs))
        assert torch.equal(out, again)
    some = [0, 73, 295]                                     # of the heads
    rows = runs[0] - max(0, runs[0] - n)
    f.k, f.v = [x[:, some] for x in f.k], [x[:, some] for x in f.v]
    compare(f, q[-rows:, some], out[-rows:, some], lse[-rows:, some], 1 / math.sqrt(dim), [rows], BF16, tile=True)
    assert bool((out[:-rows] == 0).all()) and bool((lse[:-rows] == -math.inf).all())


@pytest.mark.parametrize("heads", [2, 148])
@pytest.mark.parametrize("large", [2.0 ** 30, 2.0 ** 60, 2.0 ** 100])
@pytest.mark.parametrize("weight", [1, 2])
@pytest.mark.parametrize("place", [0, 128])
def test_large_values_of_little_weight_in_chunks(large, weight, place, heads):
    """64 tokens of large values in one stretch, with weights of about 1 / large, or its square."""
    f = Filled([333], 16, heads, 128, BF16)
    some = slice(place, place + 64)
    f.k[0].mul_(0.1)
    f.k[0][some] = -weight * math.log(large) / 32
    f.v[0][some] = (f.v[0][some].float() * large).to(BF16)
    f.write_all()
    q = values((100, heads, 128), BF16, 3).abs().clamp(0.5, 1.5).cuda()
    out, lse = torch.empty_like(q), torch.empty(100, heads, device="cuda")
    ws = torch.empty(Q.qsgd_cache_attend_workspace_bytes(f.cache, heads), dtype=torch.uint8, device="cuda")
    before = Q.qsgd_launch_count()
    Q.qsgd_cache_attend(f.cache, f.table, f.len, q, out, ws, f.status, starts=starts_of([100]), scale=0.25, lse=lse)
    assert (Q.qsgd_launch_count() - before == 1) == (heads == 148)
    f.fine()
    compare(f, q, out, lse, 0.25, [100], BF16, tile=heads == 148)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page, layout, lengths, runs, group", [(16, "gaps", [150, 0, 40], [100, 3, 60], 2), (48, "heads", [700, 333], [65, 64], 3),
                                                               (128, "pages", [1000], [129], 1)])
def test_tiles_of_wide_ranges_in_every_form(dim, page, layout, lengths, runs, group):
    """Numbers too far apart for a tile's fp16, with pages, rows in front of the first token, heads that share keys, strides, and values that are none."""
    heads = 100
    f = Filled(lengths, page, heads, dim, BF16, layout=layout)
    for k, v in zip(f.k, f.v):
        v[::3] = (v[::3].float() * 1e25).to(BF16)
        k[1::5] = (k[1::5].float() * 1e-20).to(BF16)
    f.k[0][140:], f.v[0][20, :, -1] = math.inf, math.nan
    f.write_all()
    rows = sum(runs)
    wide = values((rows, heads * group + 3, dim + 8), BF16, 8).cuda()
    q, big = wide[:, 1: 1 + heads * group, :dim], torch.full((heads * group, rows + 2, dim + 8), 42.0, dtype=BF16, device="cuda")
    out, lse = big.transpose(0, 1)[:rows, :, :dim], torch.full((rows + 2, heads * group), 42.0, device="cuda")
    ws = torch.empty(Q.qsgd_cache_attend_workspace_bytes(f.cache, heads * group), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    before = Q.qsgd_launch_count()
    Q.qsgd_cache_attend(f.cache, f.table, f.len, q, out, ws, f.status, starts=starts_of(runs), lse=lse[:rows])
    tile = Q.qsgd_launch_count() - before == 1
    assert tile or (dim, runs) == (64, [129])               # (a tile and one row of the next: too few rows for tiles at head size 64)
    f.fine()
    assert bool((big[:, rows:] == 42).all()) and bool((big[:, :, dim:] == 42).all()) and bool((lse[rows:] == 42).all())
    again = torch.empty(rows, heads * group, dim, dtype=BF16, device="cuda")
    Q.qsgd_cache_attend(f.cache, f.table, f.len, q, again, ws, f.status, starts=starts_of(runs))
    assert torch.equal(out.nan_to_num(7.0), again.nan_to_num(7.0))
    at = 0
    for b, (n, r) in enumerate(zip(lengths, runs)):
        seen = torch.arange(n - r + 1, n + 1)               # tokens of each row
        o, s = out[at: at + r], lse[at: at + r]
        assert bool((o[seen <= 0] == 0).all()) and bool((s[seen <= 0] == -math.inf).all())
        if b == 0:
            bad = seen > 140
            assert bool(o[bad].isnan().all()) and bool(s[bad].isnan().all()) and not bool(s[~bad].isnan().any())
            assert bool(o[~bad & (seen > 20)][..., dim - 64:].isnan().all()) and not bool(o[~bad][..., : dim - 64].isnan().any())
        some = [0, heads - 1]
        pick = [h * group + i for h in some for i in range(group)]
        for i in [i for i in range(r) if 0 < seen[i] <= (140 if b == 0 else n)][:: max(1, r // 7)]:
            one = Filled([0], 16, 1, dim, BF16)
            m = int(seen[i])
            one.lengths, one.k, one.v = [m], [f.k[b][:m, some]], [f.v[b][:m, some]]
            compare(one, q[at + i: at + i + 1, pick], o[i: i + 1, pick], s[i: i + 1, pick], 1 / math.sqrt(dim), [1], BF16, tile=tile)
        at += r


@pytest.mark.parametrize("dtype, ratio", [(BF16, 2.0 ** 23), (BF16, 2.0 ** 40), (BF16, 2.0 ** 80), (FP16, 2.0 ** 13)])
@pytest.mark.parametrize("swap", [False, True])
@pytest.mark.parametrize("heads, dim, lengths, runs, one", [(2, 128, [700, 9], [1, 1], True), (2, 256, [5000], [1], True), (2, 128, [150], [40], False), (148, 128, [150], [100], False)])
def test_queries_small_where_keys_are_large(dtype, ratio, swap, heads, dim, lengths, runs, one):
    """A group of coordinates with large keys and small queries counts as much as one with small keys and large queries."""
    f = Filled(lengths, 16, heads, dim, dtype)
    groups = torch.ones(dim // 64)
    groups[1 if swap else 0] = ratio ** 0.5
    for k in f.k:
        k.copy_((k.float() * groups.repeat_interleave(64) / ratio ** 0.25).to(dtype))
    f.write_all()
    q = (values((sum(runs), heads, dim), dtype, 3).float() / groups.repeat_interleave(64) * ratio ** 0.25).to(dtype).cuda()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    ws = torch.empty(Q.qsgd_cache_attend_workspace_bytes(f.cache, heads), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    before = Q.qsgd_launch_count()
    Q.qsgd_cache_attend(f.cache, f.table, f.len, q, out, ws, f.status, starts=None if one else starts_of(runs), lse=lse)
    tile = not one and Q.qsgd_launch_count() - before == 1
    f.fine()
    some = [0, heads - 1]
    f.k, f.v = [x[:, some] for x in f.k], [x[:, some] for x in f.v]
    compare(f, q[:, some], out[:, some], lse[:, some], 1 / math.sqrt(dim), runs, dtype, tile=tile)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("code", [1, 8, 15])
@pytest.mark.parametrize("place", [0, 1, 6])
def test_small_numbers_of_a_query_beside_a_large_one(dtype, code, place):
    """One token, whose score is the log-sum-exp. A product of the query's number and a code is cut off at 2^-18 of the largest |q|, 64 of them (twice, with
    what is added up before), and the rest is fp32."""
    cache, data = Q.Cache(1, 16, 1, 64, dtype), torch.zeros(18 * 64, dtype=torch.uint8)
    codes = torch.full((64,), 15)
    codes[place] = code
    data[:32] = (codes[0::2] | codes[1::2] << 4).to(torch.uint8)
    data[512:516] = torch.tensor([0.0, 1.0], dtype=dtype).view(torch.uint8)
    cache.data.copy_(data.view(1, 1, -1))
    table, lengths, status = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda"), Q.new_status()
    ws = torch.empty(Q.qsgd_cache_attend_workspace_bytes(cache, 1), dtype=torch.uint8, device="cuda")
    for k in range(0, 26, 2):
        q = torch.full((1, 1, 64), 1024.0 * 2.0 ** -k * (1 + 2.0 ** -6), dtype=dtype)
        q[0, 0, place] = 1024.0
        out, lse = torch.empty(1, 1, 64, dtype=dtype, device="cuda"), torch.empty(1, 1, device="cuda")
        Q.qsgd_cache_attend(cache, table, lengths, q.cuda(), out, ws, status, scale=1.0, lse=lse)
        ref = float((q[0, 0].double() * codes).sum())
        assert abs(float(lse) - ref) <= 2 * 64 * 2.0 ** -18 * float(q.max()) * 0.5 + 2.0 ** -21 * abs(ref), k
    assert int(status.item()) == 0


@pytest.mark.parametrize("runs", [[1], [5]])
def test_outputs_that_cancel(runs):
    """One token has nearly all weight and a value of zero made of lo and a code: what is left is the others', of fp16's smallest numbers."""
    f = Filled([25], 16, 1, 128, FP16)
    f.k[0].mul_(0.05)
    f.k[0][10] = 11.0 / 128
    f.v[0].mul_(0.1)
    f.v[0][10] = ((torch.arange(128) % 16) - 7.0) / 16
    f.write_all()
    assert bool((F.held_value(f.v[0])[10, 0, 7::16] == 0).all())
    q = torch.ones(sum(runs), 4, 128, dtype=FP16, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(sum(runs), 4, device="cuda")
    ws = torch.empty(Q.qsgd_cache_attend_workspace_bytes(f.cache, 4), dtype=torch.uint8, device="cuda")
    Q.qsgd_cache_attend(f.cache, f.table, f.len, q, out, ws, f.status, starts=starts_of(runs), scale=1.0, lse=lse)
    f.fine()
    compare(f, q, out, lse, 1.0, runs, FP16)
