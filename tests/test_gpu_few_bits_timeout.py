"""A bounded wait that runs out in the kernels on few-bit values: they raise QSGD_DEV_TIMEOUT, stop, wait for what they have in flight and
return, and the same call is right again with the ordinary bound. The waits are made to run out through the library's test hook (a poll bound
of zero), so nothing here faults, traps or hangs."""
import math

import pytest
import torch

import few_bits as F
import paper_1610_02132_b200 as Q
from test_gpu_cache import BF16, Filled, starts_of, values

pytestmark = pytest.mark.gpu


@pytest.fixture
def zero_polls():
    Q.qsgd_test_set_wait_polls(0)
    try:
        yield
    finally:
        Q.qsgd_test_set_wait_polls(Q.qsgd_test_default_wait_polls())


# clusters to a segment, a CTA to a segment, the line of units with one row a sequence and with several, rows in tiles of 128
@pytest.mark.parametrize("lengths, runs, heads", [([600], None, 2), ([40], None, 1), ([3000] * 9, None, 8), ([700, 300], [100, 64], 1),
                                                  ([700, 300], [100, 64], 24)])
def test_attend_gives_up_and_returns(zero_polls, lengths, runs, heads):
    f = Filled(lengths, 16, heads, 128, BF16).write_all()
    rows = sum(runs or [1] * len(lengths))
    q = values((rows, 4 * heads, 128), BF16, 5).cuda()
    big = torch.full((rows + 8, 4 * heads, 128), 42.0, dtype=BF16, device="cuda")
    ws = torch.empty(Q.qsgd_cache_attend_workspace_bytes(f.cache, 4 * heads), dtype=torch.uint8, device="cuda")
    starts = starts_of(runs) if runs else None
    Q.qsgd_cache_attend(f.cache, f.table, f.len, q, big[:rows], ws, f.status, starts=starts)
    torch.cuda.synchronize()                                  # the kernels came back
    assert int(f.status.item()) & Q.binding.DEV_TIMEOUT
    assert bool((big[rows:] == 42).all())
    Q.qsgd_test_set_wait_polls(Q.qsgd_test_default_wait_polls())
    f.status.zero_()
    out, again = torch.empty_like(q), torch.empty_like(q)
    Q.qsgd_cache_attend(f.cache, f.table, f.len, q, out, ws, f.status, starts=starts)
    Q.qsgd_cache_attend(f.cache, f.table, f.len, q, again, ws, f.status, starts=starts)
    assert int(f.status.item()) == 0 and torch.equal(out, again)
    ref, _, mean = F.attend(q[:runs[0] if runs else 1].cpu(), F.held_value(f.k[0]), F.held_value(f.v[0]), 1 / math.sqrt(128), lengths[0],
                            runs[0] if runs else 1)
    off = (out[: ref.shape[0]].cpu().double() - ref).abs()
    assert bool((off <= 2.0 ** -8 * ref.abs() + 2.0 ** -5 * mean + 0.01).all())      # (the bounds proper are in the tests of the cache)


@pytest.mark.parametrize("m, n, k", [(40, 100, 200), (300, 700, 4096), (2000, 3000, 640)])
def test_product_gives_up_and_returns(zero_polls, m, n, k):
    g = torch.Generator().manual_seed(m)
    a = torch.randint(-128, 128, (m, -(-k // 16) * 16), generator=g).to(torch.int8).cuda()[:, :k]
    b = torch.randint(-128, 128, (n, -(-k // 16) * 16), generator=g).to(torch.int8).cuda()[:, :k]
    one, out, status = torch.ones(max(m, n), device="cuda"), torch.full((m + 3, n), 42.0, device="cuda"), Q.new_status()
    Q.qsgd_matmul_i8(a, one[:m], b, one[:n], out[:m], status_dev=status)
    torch.cuda.synchronize()
    assert int(status.item()) == Q.binding.DEV_TIMEOUT
    assert bool((out[m:] == 42).all())
    Q.qsgd_matmul_i8(a, one[:m], b, one[:n], out[:m])         # without a status word, too, it returns
    torch.cuda.synchronize()
    Q.qsgd_test_set_wait_polls(Q.qsgd_test_default_wait_polls())
    status.zero_()
    Q.qsgd_matmul_i8(a, one[:m], b, one[:n], out[:m], status_dev=status)
    assert int(status.item()) == 0
    assert torch.equal(out[:m], (a.double() @ b.double().T).float())          # the exact sum, rounded to fp32 once
