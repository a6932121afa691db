"""The exact comparison of the products sees a lost or doubled part of a long sum, on the host."""
import pytest
import torch

from product_exact import assert_exact, dw_exact, whole
from product_helpers import TYPES


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_a_part_lost_doubled_or_out_of_place_is_seen(dtype):
    rows, n, k, part = 70000, 24, 16, 512
    dy, x = whole(1, (rows, n), dtype), whole(2, (rows, k), dtype)
    off = torch.tensor([0, rows], dtype=torch.int32)
    want = dw_exact(dy, x, off, None, 1)
    assert_exact(want.to(dtype), want, dtype)
    one = lambda at: dy[at:at + part].double().t() @ x[at:at + part].double()
    shifted = dy[part:2 * part].double().t() @ x[:part].double()
    for wrong in (want - one(0), want - one(rows - rows % part - part), want + one(5 * part), want - one(0) + shifted):
        with pytest.raises(AssertionError):
            assert_exact(wrong.to(dtype), want, dtype)
