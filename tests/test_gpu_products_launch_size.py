"""Products whose launch only the larger tiles hold, on the device."""
import pytest
import torch

from paper_2602_23999_amd import rabitq

from product_helpers import assert_sums, dw64, dx64, forward64, lists_from, numbers

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [1, 16])
def test_one_query_against_more_rows_than_the_smallest_tiles_hold(k):
    n = (1 << 28) + 37
    g = torch.Generator(device="cuda").manual_seed(k)
    b = torch.randint(-128, 128, (n, k), generator=g, device="cuda", dtype=torch.int8)
    a = torch.randint(-128, 128, (1, k), generator=g, device="cuda", dtype=torch.int8)
    sb = torch.exp2(torch.randint(-3, 4, (n,), generator=g, device="cuda").float())
    got = rabitq.matmul_i8(a, torch.full((1,), 0.5, device="cuda"), b, sb)[0]
    for at in range(0, n, 1 << 26):  # sums below 2^19 and scales that are powers of two: everything is exact
        part = slice(at, min(at + (1 << 26), n))
        assert torch.equal(got[part], (b[part].float() * a.float()).sum(1) * 0.5 * sb[part])


def test_more_lists_than_the_smallest_tiles_hold():
    groups, pairs, nprobe = 1 << 20, 100, 1
    gen = torch.Generator().manual_seed(1)
    probes = torch.randint(groups, (pairs, nprobe), generator=gen)
    probes[0], probes[1], probes[2:40] = 0, groups - 1, 77
    off, ids = lists_from(probes, groups)
    lists = off.cuda(), ids.cuda(), nprobe
    small = torch.unique(probes)                 # the lists that have rows, numbered anew
    off_s, ids_s = lists_from(torch.searchsorted(small, probes), small.numel())
    for n, k in ((256, 8), (2, 1024)):           # wide for the forward pass, then for the gradients
        x, dy = numbers(2, (pairs, k), torch.bfloat16), numbers(3, (pairs, n), torch.bfloat16)
        w = torch.full((groups, n, k), float("nan"), dtype=torch.bfloat16, device="cuda")
        w_s = numbers(4, (small.numel(), n, k), torch.bfloat16)
        w[small.cuda()] = w_s.cuda()
        want, mag, _ = forward64(x, w_s, off_s, ids_s, 1)
        assert_sums(rabitq.grouped_matmul(x.cuda(), w, *lists), want, mag, k, torch.bfloat16)
        want, mag, _ = dx64(dy, w_s, off_s, ids_s, 1)
        assert_sums(rabitq.grouped_matmul_dx(dy.cuda(), w, *lists), want, mag, n, torch.bfloat16)
        want, mag = dw64(dy, x, off_s, ids_s, 1)
        got = rabitq.grouped_matmul_dw(dy.cuda(), x.cuda(), *lists, out=w)
        assert_sums(got[small.cuda()], want, mag, 40, torch.bfloat16)
        rest = torch.ones(groups, dtype=torch.bool, device="cuda")
        rest[small.cuda()] = False
        assert not got[rest].any()  # (every element is written: no NaN left)


@pytest.mark.parametrize("rows,k", [((1 << 26) + 73, 8), ((1 << 27) + 1, 5)])
def test_more_rows_to_quantise_than_a_launch_holds(rows, k):
    # whole numbers from -127 to 127, 127 in every row: scale 1, and the codes are the numbers
    g = torch.Generator(device="cuda").manual_seed(k)
    codes = torch.randint(-127, 128, (rows, k), generator=g, device="cuda", dtype=torch.int8)
    codes[:, 3] = 127
    x = torch.empty(rows, k, dtype=torch.bfloat16, device="cuda")
    x.copy_(codes)
    x[-1] *= 2
    got, scale = rabitq.quantize_rows(x)
    assert torch.equal(got, codes)
    assert (scale[:-1] == 1).all() and scale[-1] == 2
