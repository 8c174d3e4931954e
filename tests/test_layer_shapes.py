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


@pytest.mark.parametrize("columns", [193, 199, 201, 256])
def test_linear4_takes_as_many_inputs_as_it_has(columns):
    """Of whole groups a few more or less would meet codes that stand for nothing, or leave weights out."""
    layer = L.Linear4(torch.zeros((5, 32), dtype=torch.int32), torch.zeros((5, 4, 2), dtype=torch.bfloat16), 200)
    for x in (torch.zeros((3, columns)), torch.zeros((2, 3, columns)), torch.zeros(columns), torch.zeros((3, columns), requires_grad=True)):
        with pytest.raises(ValueError, match="200 inputs"):
            layer(x)
    with pytest.raises(ValueError, match="200 inputs"):
        layer(torch.zeros(()))
