"""What the Python calls on rows refuse by themselves (no GPU needed)."""
import pytest

from paper_2608_13255_gb300 import build as gbuild


@pytest.fixture(scope="module")
def gc():
    gbuild.build()
    from paper_2608_13255_gb300 import geocache
    geocache.load()
    return geocache


@pytest.mark.parametrize("name", ["relu", "GELU", "", 1, True, ["gelu"], ("silu",)], ids=repr)
def test_an_activation_that_does_not_exist(gc, name):
    import torch
    x, w = torch.zeros((4, 64)).bfloat16(), torch.zeros((32, 64)).bfloat16()
    with pytest.raises(ValueError, match="activation must be"):
        gc.linear(x, w, activation=name)
