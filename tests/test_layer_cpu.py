"""Arguments of layer.ffn_fwd / ffn_bwd that are refused before anything is computed (CPU only)."""
import pytest
import torch

from paper_2505_18654_amd.layer import ffn_bwd, ffn_fwd


@pytest.mark.parametrize("p", [-0.1, 1.0, float("nan")])
def test_ffn_refuses_what_is_no_probability(p):
    x = torch.zeros(4, 32, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="p_drop"):
        ffn_fwd(x, None, None, None, p)
    with pytest.raises(ValueError, match="p_drop"):
        ffn_bwd(x, {}, None, None, None, p)
