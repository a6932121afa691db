"""Products on both sides of where the choice of a kernel changes, on the device."""
import pytest
import torch

from paper_2602_23999_amd import rabitq

from product_helpers import assert_scaled, assert_sums, dx64, forward64, i8_64, lists_from, numbers, probes_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("rows,groups,wide", [
    (1024, 1, 1024), (1025, 1, 1024),               # 256 and 272 tiles of 64 columns with 64 rows each
    (512, 1, 1024), (513, 1, 1024),                 # 256 and 272 with 32 rows
    (834, 4, 1024), (900, 4, 1024), (835, 4, 1020), # lists of any lengths
    (20, 40, 1600),                                 # fewer pairs than lists
], ids=str)
def test_shared_tiles_up_to_one_for_each_compute_unit(rows, groups, wide, dtype):
    long = 1048 if dtype == torch.bfloat16 else 264
    off, ids = lists_from(probes_of(rows, rows, 1, groups), groups)
    lists = off.cuda(), ids.cuda(), 1
    x, w = numbers(1, (rows, long), dtype), numbers(2, (groups, wide, long), dtype)
    want, mag, _ = forward64(x, w, off, ids, 1)
    assert_sums(rabitq.grouped_matmul(x.cuda(), w.cuda(), *lists), want, mag, long, dtype)
    w = w.transpose(1, 2).contiguous()
    want, mag, _ = dx64(x, w, off, ids, 1)
    assert_sums(rabitq.grouped_matmul_dx(x.cuda(), w.cuda(), *lists), want, mag, long, dtype)


@pytest.mark.parametrize("m,n,k", [(1024, 1024, 1024), (1408, 768, 1040), (1025, 1000, 2056)])
def test_shared_tiles_of_codes(m, n, k):
    g = torch.Generator().manual_seed(m)
    a, b = (torch.randint(-128, 128, (r, k), generator=g).to(torch.int8) for r in (m, n))
    sa, sb = (torch.exp(torch.randn(r, generator=g)) for r in (m, n))
    assert_scaled(rabitq.matmul_i8(a.cuda(), sa.cuda(), b.cuda(), sb.cuda()), i8_64(a, sa, b, sb), torch.float32)
