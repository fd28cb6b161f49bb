"""What ffn's layout of weights refuses, before anything reaches a GPU."""
import pytest
import torch

from paper_2006_11735_amd import ffn


@pytest.mark.parametrize("group", [0, -128, 16, 100, 512, 2 ** 40])
def test_groups_that_the_library_does_not_have(group):
    with pytest.raises(ValueError, match="group"):
        ffn.quantize_weights_s4(torch.zeros((4, 64)), group=group)


@pytest.mark.parametrize("w,kw", [(torch.zeros(64), {}), (torch.zeros((4, 64), dtype=torch.float64), {}), (torch.zeros((2, 4, 64)), {}),
                                  (torch.zeros((4, 64)), dict(scale_dtype=torch.float64)), (torch.zeros((4, 64)), dict(scale_dtype=torch.int8))])
def test_weights_and_scales_of_other_kinds(w, kw):
    with pytest.raises(ValueError, match="weights"):
        ffn.quantize_weights_s4(w, **kw)
