"""What the operators take as a number (no GPU needed)."""
import fractions

import numpy as np
import pytest
import torch

from paper_2609_39350_amd import operators as ops


@pytest.mark.parametrize("x,want", [(3, 3), (-2**70, -2**70), (True, 1), (np.int64(-5), -5), (np.uint8(7), 7),
                                    (torch.tensor(4), 4), (torch.tensor([4]), 4)])
def test_whole(x, want):
    assert ops._whole("n", x) == want


@pytest.mark.parametrize("x", [None, "3", b"3", 3.0, np.float64(3), 1j, [3], torch.tensor(3.0), torch.zeros(2, dtype=torch.int64)])
def test_not_whole(x):
    with pytest.raises(ValueError, match="n: a whole number"):
        ops._whole("n", x)


@pytest.mark.parametrize("x,want", [(0.1, 0.1), (3, 3.0), (np.float32(0.5), 0.5), (np.int32(2), 2.0), (torch.tensor(0.25), 0.25),
                                    (fractions.Fraction(1, 4), 0.25), (float("inf"), float("inf"))])
def test_real(x, want):
    assert ops._real("x", x) == want


@pytest.mark.parametrize("x", [None, "0.1", b"1", 1j, [0.1], (1.0,), 10**400, torch.zeros(2)])
def test_not_real(x):
    with pytest.raises(ValueError, match="x: a number"):
        ops._real("x", x)


def test_a_routing_of_no_numbers():
    for sizes in (("6", 8, 2), (6, 8.0, 2), (6, 8, None)):
        with pytest.raises(ValueError):
            ops.Routing(*sizes, device="cpu")
