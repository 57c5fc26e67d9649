"""What the binding refuses before a call reaches the library."""
import pytest
import torch

from paper_1908_04172_amd import he


def test_lazily_conjugated_and_negated_tensors_are_refused():
    """Their memory holds other values than the tensor: contiguous or not, and whatever the device."""
    z = torch.zeros((3, 4), dtype=torch.complex128)
    for t in (z.conj(), z[:1, :1].conj().imag, torch._neg_view(z.real)):
        assert t.is_conj() or t.is_neg()
        with pytest.raises(TypeError, match="conjugated or negated"):
            he._dev_ptr(t, "slots")
    assert z.conj().resolve_conj().is_conj() is False
