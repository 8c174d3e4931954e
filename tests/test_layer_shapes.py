"""What the modules of a layer refuse by its shape (nothing here needs a GPU)."""
import pytest
import torch

from paper_2104_14129_amd import layers as L


def test_block_norm_takes_inputs_of_one_shape():
    """Rows of another order would be added to each other, rows of another width cut anew."""
    layer = L.QBlockNorm(8)
    x = torch.zeros((2, 3, 8))
    for h, gate in ((torch.zeros((3, 2, 8)), None), (torch.zeros((6, 8)), None), (torch.zeros((2, 3, 4)), None), (x, torch.zeros((3, 2, 8))), (x, torch.zeros(8)), (x, torch.zeros((2, 1, 8)))):
        with pytest.raises(ValueError, match="shape"):
            layer(x, h, gate)
    for x in (torch.zeros((2, 16)), torch.zeros((4, 4)), torch.zeros(16)):
        with pytest.raises(ValueError, match="width"):
            layer(x)
        with pytest.raises(ValueError, match="width"):
            layer(x, x)
