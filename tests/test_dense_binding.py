"""What the binding of the dense operators refuses before it asks for a GPU."""

import pytest
import torch
from torch.autograd import forward_ad

from paper_2603_18599_gb300 import dense


def test_tangents_of_forward_mode_are_refused():
    x, cpu = torch.ones(8), torch.device("cpu")
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones(8))
        for tensor in (dual, dual.view(2, 4).view(-1)):
            with pytest.raises(ValueError, match="tangent"):
                dense._vector(tensor, "gain", 8, cpu)
            with torch.no_grad(), pytest.raises(ValueError, match="tangent"):
                dense._vector(tensor, "gain", 8, cpu)
        assert dense._vector(dual.detach(), "gain", 8, cpu) == x.data_ptr()
        assert dense._vector(x, "gain", 8, cpu) == x.data_ptr()
    wants = torch.ones(8, requires_grad=True)
    with pytest.raises(ValueError, match="wants a gradient"):
        dense._vector(wants, "gain", 8, cpu)
    with torch.no_grad():
        assert dense._vector(wants, "gain", 8, cpu) == wants.data_ptr()
