"""GPU: the example's serving from pages, where the chunk at the beginning holds all
tokens or more than there are."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows, prompt", [(4, None), (6, None), (6, 36), (6, 37), (6, 38), (6, 1), (6, 0)])
def test_prompts_as_long_as_the_tokens_and_longer(rows, prompt):
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import token_block
    block = token_block.TokenBlock(rows=rows, cols=rows)
    g = torch.Generator().manual_seed(61)
    how = {} if prompt is None else {"prompt": prompt}
    with torch.no_grad():
        x = block.tokens(torch.rand((3, 3, rows + 2, rows + 2), generator=g).cuda())
        whole = block(x).float()
        served = block.serve_in_pages(x, **how).float()
        assert served.shape == whole.shape
        # bf16 outputs of order 1 to 4: both ways round each of five steps once
        assert (whole - served).abs().max() <= 5 * 4 * 2.0 ** -8
        assert torch.isfinite(block.serve_in_pages(x, kind="e4m3", **how)).all()
