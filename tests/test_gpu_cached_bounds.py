"""Block-wise denoising (cached.py) at the ends of its range."""

import pytest
import torch

from tests.test_gpu_cached import SHAPES, made

pytestmark = pytest.mark.gpu


def test_a_block_that_does_not_fit(abi):
    """A pass or a recording whose positions lie behind the cache's capacity
    is refused, and leaves no status behind."""
    stack, prompt, _ = made(SHAPES[0])                # 96 tokens, blocks of 8
    long = prompt.repeat(1, 3)[:, :90]
    stack.prefill(long)
    with pytest.raises(ValueError):
        stack.capture()
    with pytest.raises(ValueError):
        stack.forward(torch.ones(2, 7, dtype=torch.long, device="cuda"))
    assert torch.isfinite(stack.forward(torch.ones(2, 6, dtype=torch.long, device="cuda"))).all()
    abi.check_status()


def test_no_prompt_and_no_blocks(abi):
    """An answer without a prompt, and none at all."""
    stack, prompt, _ = made(SHAPES[0])
    none = stack.generate(prompt, 0)
    assert none.shape == (2, 0) and none.dtype == torch.long and stack.held == prompt.shape[1]
    alone = stack.generate(prompt[:, :0], 1)
    assert alone.shape == (2, 8) and bool((alone != stack.mask_id).all()) and stack.held == 8
    assert torch.equal(stack.generate(prompt[:, :0], 1), alone)
    abi.check_status()
