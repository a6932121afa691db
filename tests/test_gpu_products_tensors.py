"""What the products' binding does with tensors that automatic differentiation watches, on the device."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2602_23999_amd import rabitq

pytestmark = pytest.mark.gpu


def _codes():
    return torch.ones(6, 8, dtype=torch.int8, device="cuda"), torch.ones(6, device="cuda")


def test_tensors_that_carry_a_tangent_are_refused():
    x, w, dy = torch.ones(6, 8, device="cuda"), torch.ones(3, 5, 8, device="cuda"), torch.ones(6, 5, device="cuda")
    off = torch.tensor([0, 2, 2, 6], dtype=torch.int32, device="cuda")
    c, s = _codes()
    with forward_ad.dual_level():
        dual = lambda t: forward_ad.make_dual(t, torch.ones_like(t))
        for call in (lambda: rabitq.grouped_matmul(dual(x), w, off), lambda: rabitq.grouped_matmul(x, dual(w), off),
                     lambda: rabitq.grouped_matmul(x, w, off, out=dual(dy)), lambda: rabitq.grouped_matmul_dx(dual(dy), w, off),
                     lambda: rabitq.grouped_matmul_dw(dy, dual(x), off), lambda: rabitq.quantize_rows(dual(x)),
                     lambda: rabitq.quantize_rows(x, scale=dual(s)), lambda: rabitq.matmul_i8(c, dual(s), c, s),
                     lambda: rabitq.grouped_matmul_i8(c, s, c[:3, None], dual(torch.ones(3, 1, device="cuda")), off)):
            with pytest.raises(rabitq.RabitqError, match="tangent"):
                call()
        assert torch.equal(rabitq.grouped_matmul(x, w, off), torch.full((6, 5), 8.0, device="cuda"))


def test_outputs_of_the_caller_count_as_written():
    x, w, dy = torch.ones(6, 8, device="cuda"), torch.ones(3, 5, 8, device="cuda"), torch.ones(6, 5, device="cuda")
    off = torch.tensor([0, 2, 2, 6], dtype=torch.int32, device="cuda")
    c, s = _codes()
    like = lambda t: torch.zeros_like(t)
    calls = [(like(dy), lambda o: rabitq.grouped_matmul(x, w, off, out=o)), (like(x), lambda o: rabitq.grouped_matmul_dx(dy, w, off, out=o)),
             (like(w), lambda o: rabitq.grouped_matmul_dw(dy, x, off, out=o)), (like(s), lambda o: rabitq.quantize_rows(x, scale=o)),
             (torch.zeros(6, 6, device="cuda"), lambda o: rabitq.matmul_i8(c, s, c, s, out=o)),
             (torch.zeros(6, 1, device="cuda"), lambda o: rabitq.grouped_matmul_i8(c, s, c[:3, None], torch.ones(3, 1, device="cuda"), off, out=o))]
    for buffer, call in calls:
        factor = torch.ones_like(buffer).requires_grad_()
        kept = (buffer * factor).sum()  # saves the buffer for the gradient of the factor
        call(buffer)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            kept.backward()
    codes = like(c)
    before = codes._version
    rabitq.quantize_rows(x, codes=codes)
    assert codes._version > before and x._version == 0 and w._version == 0
    before = codes._version
    with pytest.raises(rabitq.RabitqError):  # (a call that is refused writes nothing)
        rabitq.quantize_rows(x[:, :0], codes=codes[:, :0])
    assert codes._version == before
    with torch.inference_mode():
        assert rabitq.matmul_i8(c, s, c, s, out=torch.zeros(6, 6, device="cuda")).min() == 8
