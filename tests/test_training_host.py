"""The training modules' checks of what they are built with (no GPU needed)."""
import pytest

from paper_2506_08520_amd import training as T


@pytest.mark.parametrize("make", [
    lambda: T.DifferentialWindowAttention(260, 2, 8, device="cpu"),         # 65 / 130 to a head
    lambda: T.DifferentialTransformerBlock(520, 4, 8, device="cpu"),
    lambda: T.LayerNorm(4097, device="cpu"),
    lambda: T.LayerNorm((8, 32), device="cpu"),
    lambda: T.DifferentialTransformerBlock(8192, 64, 8, device="cpu"),
])
def test_sizes_that_no_kernel_takes_are_refused_at_once(make):
    with pytest.raises(ValueError):
        make()


def test_the_largest_sizes_are_built():
    at = T.DifferentialWindowAttention(256, 2, 8, device="cpu")             # 64 / 128
    assert at.norm.weight.shape == (128,)
    assert T.LayerNorm(4096, device="cpu").weight.shape == (4096,)
    assert T.LayerNorm((64,), device="cpu").weight.shape == (64,)
    assert T.LayerNorm(1, elementwise_affine=False, device="cpu").weight is None
