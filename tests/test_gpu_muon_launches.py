"""Muon steps of more matrices than one launch takes: those on either side of a cut, the first and the last, against the oracle.  The
tolerances are those of the other tests of the step."""
import numpy as np
import pytest
import torch

from oracle import fno_oracle as O
from paper_2204_01205_amd import binding as B
from test_gpu_muon import bounds, stack

MU = 0.9


def check(params, grads, momentum, places):
    """places: for every tensor of the list the matrices that are looked at."""
    is_complex = params[0].is_complex()
    pick = lambda t, at: stack((t[..., at] if is_complex else t[at]).cpu().numpy())
    places = [torch.tensor(p, device="cuda") for p in places]
    before = [(pick(g, at).astype(np.complex128 if is_complex else np.float64), pick(m, at)) for g, m, at in zip(grads, momentum, places)]
    tensors = B.make_muon_tensors(params, grads, momentum, scale=-1.0)
    B.fno_muon_step(tensors, 1.0, MU, B.alloc_muon_workspace(tensors))
    torch.cuda.synchronize()
    for k, (p, at, (g, m)) in enumerate(zip(params, places, before)):
        u = g + MU * (MU * m + g)
        error = np.sqrt((np.abs(pick(p, at) - O.newton_schulz(u)) ** 2).sum((1, 2)))
        assert np.all(error <= bounds(u, 5)), (k, at[int((error / bounds(u, 5)).argmax())])


def draws(shape, seed, is_complex):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn(shape, dtype=torch.complex64 if is_complex else torch.float32, device="cuda", generator=gen)


@pytest.mark.gpu
@pytest.mark.parametrize("shape,is_complex,cut", [((2 ** 22 + 5, 2, 3), False, 2 ** 22), ((2 ** 22 + 5, 3, 1), False, 2 ** 22),
                                                  ((1, 2, 2 ** 26 + 35), True, 2 ** 26), ((5, 1, 2 ** 26 + 1), True, 2 ** 26)])
def test_a_tensor_that_takes_two_launches(shape, is_complex, cut):
    count = shape[-1] if is_complex else shape[0]
    grads, momentum = draws(shape, 1, is_complex), draws(shape, 2, is_complex)
    check([torch.zeros_like(grads)], [grads], [momentum], [[0, 1, cut // 2, cut - 17, cut - 16, cut - 1, cut, cut + 1 if count > cut + 1 else cut, count - 1]])


@pytest.mark.gpu
def test_tensors_of_17_channels_that_take_two_launches():
    """Thirteen tensors of 81250 blocks of 16 modes: the last one goes on in a second launch.  They share a gradient, which is only read."""
    modes, count = 1300000, 13
    cut = (2 ** 20 - 12 * 81250) * 16
    assert 0 < cut < modes
    grad = draws((17, 17, modes), 3, True)
    momentum = [draws((17, 17, modes), 4 + k, True) for k in range(count)]
    params = [torch.zeros_like(grad) for _ in range(count)]
    ends = [0, 1, modes - 1]
    check(params, [grad] * count, momentum, [ends] * 12 + [ends + [cut - 17, cut - 1, cut, cut + 1, cut + 16]])


@pytest.mark.gpu
def test_more_small_spectral_weights_than_a_launch_takes():
    """Seventy tensors of 5 to 8 channels, 32 a launch, the largest of them among the smallest."""
    shapes = [(5 + k % 4, 8 - k % 3, 65536 if k in (31, 32, 64) else 1 + 7 * k) for k in range(70)]
    params = [torch.zeros(s, dtype=torch.complex64, device="cuda") for s in shapes]
    grads, momentum = ([draws(s, 100 * n + k, True) for k, s in enumerate(shapes)] for n in (1, 2))
    check(params, grads, momentum, [[0, s[2] // 2, s[2] - 1] for s in shapes])
