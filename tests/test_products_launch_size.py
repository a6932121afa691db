"""Which launches of the products are refused for their size, on the host.  (Pointers are numbers that nobody follows.)"""
import pytest
import torch

from test_products_refusals import _calls, _ls


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls are not refused, and their pointers lead nowhere")
@pytest.mark.parametrize("name,lists,rest", [
    # around 2^24 workgroups of 16 columns: the kernel for few rows does not hold the launch, larger tiles do
    *[("i8", None, dict(m=m, n=n, k=64, lda=64, ldb=64, ldo=n)) for m in (1, 16, 17) for n in ((1 << 28) - 16, (1 << 28) + 1, 300_000_000)],
    *[("fwd", dict(groups=1 << 20, nprobe=1, pairs=(1 << 23) + d, n=512, k=32), dict(ldx=32, ldw=32, stride=512 * 32, ldo=512)) for d in (0, 1)],
    ("gi8", dict(groups=1 << 20, nprobe=1, pairs=100, n=512, k=32), dict(ldx=32, ldw=32, stride=512 * 32, ldo=512)),
    # around 2^24 workgroups of 64 columns
    *[("i8", None, dict(m=m, n=n, k=64, lda=64, ldb=64, ldo=n)) for m in (1, 17) for n in ((1 << 30) - 1024, (1 << 30) + 64)],
    *[("dx", dict(groups=g, nprobe=1, pairs=100, n=2, k=1024), dict(ldd=2, ldw=1024, stride=2048, ldo=1024)) for g in (1 << 19, 1 << 20, (1 << 21) - 8)],
    *[("dw", dict(groups=g, nprobe=1, pairs=4096 * 100, n=4096, k=4096), dict(ldd=4096, ldx=4096, ldo=4096, stride=1 << 24)) for g in (2048, 4096)],
], ids=str)
def test_launches_that_larger_tiles_hold_are_not_refused(name, lists, rest):
    args = rest if lists is None else dict(rest, ls=_ls(**lists))
    assert _calls()[name](**args) == -3  # (RABITQ_EHIP: it got as far as the launch, and there is no device)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls are not refused, and their pointers lead nowhere")
@pytest.mark.parametrize("rows,k", [((1 << 26) - 4, 64), (1 << 26, 64), ((1 << 31) - 1, 64), (1 << 24, 4096), (1 << 25, 20000)])
def test_rows_of_several_launches_are_not_refused(rows, k):
    assert _calls()["quant"](rows=rows, k=k, ldx=k, ldc=k) == -3
    assert _calls()["quant"](rows=1 << 31, k=k, ldx=k, ldc=k) == -1
