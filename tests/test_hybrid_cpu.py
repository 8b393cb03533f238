"""The example model's data and its command's arguments (no GPU)."""
import pytest
import torch

from paper_2507_01652_amd import hybrid


@pytest.mark.parametrize("grid", ((1, 1), (5, 7), (16, 16)))
def test_rows_repeat_turned_by_the_class(grid):
    H, W = grid
    label, tokens = hybrid.images(9, grid, 8, 64, torch.Generator().manual_seed(0))
    assert tokens.shape == (9, H * W) and int(tokens.min()) >= 0 and int(tokens.max()) < 64
    for c, t in zip(label.tolist(), tokens.view(9, H, W)):
        for r in range(1, H):
            assert torch.equal(t[r], t[r - 1].roll(-(1 + c % 3)))
    again = hybrid.images(9, grid, 8, 64, torch.Generator().manual_seed(0))
    assert torch.equal(label, again[0]) and torch.equal(tokens, again[1])


def test_layers_in_turn_and_their_memory():
    model = hybrid.Model(256, 3, (4, 4), 64, 8, window=5)
    assert [type(m) for m in model.layers] == [hybrid.LinearLayer, hybrid.SoftmaxLayer, hybrid.LinearLayer]
    k, v = model.layers[1].begin(2, torch.bfloat16, "cpu")
    assert k.shape == v.shape == (2, 2, 6, 64) and k.dtype == torch.bfloat16
    assert model.layers[0].begin(2, torch.bfloat16, "cpu").shape == (2, 4, 64, 64)
