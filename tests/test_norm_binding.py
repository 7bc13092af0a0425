"""What the binding refuses of a norm's results."""
import pytest
import torch

from paper_2408_06995_amd import binding as B


def test_scales_without_codes_are_refused():
    """As the C entry point refuses them: they would stay unwritten."""
    x = torch.zeros(0, 40)
    scales = torch.zeros(0, 2, dtype=torch.uint8)
    with pytest.raises(ValueError, match="code_scales: no codes"):
        B.fpq_rms_norm(x, None, None, 1e-6, x, x, None, None, None, None, None, scales)
