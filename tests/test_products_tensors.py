"""Tensors that the products' binding refuses whatever their sizes, on the host."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2602_23999_amd import rabitq


class _OnDevice(torch.Tensor):
    """A host tensor that says it lies on device 0, which is all that the checks of an argument ask of it."""

    def get_device(self):
        return 0


def _operand(t):
    return rabitq._operand(t, torch.float32, 2, "x", 0)


def _on_device(*shape):
    return torch.ones(*shape).as_subclass(_OnDevice)


def test_plain_tensors_are_taken():
    ptr, shape, ld, _ = _operand(_on_device(4, 6)[:, :5])
    assert ptr and shape == (4, 5) and ld == 6


def test_tensors_that_require_a_gradient():
    with pytest.raises(rabitq.RabitqError, match="gradient"):
        _operand(_on_device(4, 6).requires_grad_())


def test_tensors_that_carry_a_tangent():
    with forward_ad.dual_level():
        x = _on_device(4, 6)
        assert _operand(x)[1] == (4, 6)  # (a level alone is no tangent)
        dual = forward_ad.make_dual(x, torch.ones(4, 6).as_subclass(_OnDevice))
        for t in (dual, dual[:2], dual[:, :3]):
            assert not t.requires_grad
            with pytest.raises(rabitq.RabitqError, match="tangent"):
                _operand(t)
            with torch.no_grad(), pytest.raises(rabitq.RabitqError, match="tangent"):
                _operand(t)
        assert _operand(forward_ad.unpack_dual(dual).primal)[1] == (4, 6)


def test_views_with_their_sign_turned():
    # the only such views of floats that torch makes have stride 2, which rows of one element pass
    z = torch.complex(torch.zeros(4, 1), torch.ones(4, 1)).conj().imag
    assert z.is_neg() and z.stride() == (2, 2) and (z == -1).all()
    with pytest.raises(rabitq.RabitqError, match="sign"):
        _operand(z.as_subclass(_OnDevice))
    assert _operand(z.resolve_neg().as_subclass(_OnDevice))[1] == (4, 1)
