"""What the binding of the Muon step refuses before it looks at a device."""
import pytest
import torch

from paper_2204_01205_amd import binding as B


@pytest.mark.parametrize("coefficients", [(1.5, -0.5), (3.4445,), (), (2.0, -1.5, 0.5, 0.0)])
def test_coefficients_that_are_not_three(coefficients):
    """Two of them would put the number of iterations in the place of the third, and nesterov in the place of that number."""
    tensors = B.MuonTensors((B.FnoMuonTensor * 1)(), 0, None, ())
    with pytest.raises(ValueError, match="three coefficients"):
        B.fno_muon_step(tensors, 0.1, 0.9, torch.empty(256, dtype=torch.uint8), coefficients=coefficients)
