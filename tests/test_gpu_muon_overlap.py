"""Lists of a Muon step whose tensors overlap: two updates of a value, or a gradient in a place that the step writes, have no defined result."""
import pytest
import torch

from paper_2204_01205_amd import binding as B

z = lambda *s: torch.zeros(*s, device="cuda")


@pytest.mark.gpu
def test_tensors_that_overlap_what_the_step_writes_are_refused():
    flat, p, g, m = z(400), z(10, 10), z(10, 10), z(10, 10)
    piece = lambda at: flat[at: at + 100].view(10, 10)
    for params, grads, momentum in (([piece(0), piece(90)], [g, g], [m, z(10, 10)]), ([piece(90), piece(0)], [g, g], [m, z(10, 10)]),
                                    ([piece(0)], [g], [piece(99)]), ([p], [g], [g]), ([p], [p], [m]), ([p], [piece(50)], [piece(149)]),
                                    ([flat[:400].view(20, 20), p], [z(20, 20), g], [z(20, 20), piece(100)]),
                                    ([p, z(5, 4)], [flat[:100].view(10, 10), flat[30:50].view(5, 4)], [piece(100), flat[90:110].view(5, 4)])):
        with pytest.raises(ValueError, match="overlaps"):
            B.make_muon_tensors(params, grads, momentum)


@pytest.mark.gpu
def test_pieces_of_one_tensor_side_by_side_are_a_list():
    flat, g = z(600), z(10, 10)
    piece = lambda at: flat[at: at + 100].view(10, 10)
    B.make_muon_tensors([piece(0), piece(100)], [piece(400), piece(450)], [piece(200), piece(300)])        # gradients may share values
    B.make_muon_tensors([piece(0), piece(100)], [g, g], [piece(200), piece(300)])
    B.make_muon_tensors([flat[:0].view(0, 5), piece(0)], [z(0, 5), g], [flat[:0].view(0, 5), piece(100)])
