"""The example's block on another stream than the one it was made on: its calls go where torch's products go."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import block_step

pytestmark = pytest.mark.gpu


def test_calls_follow_the_current_stream():
    """The stream is compared before anything runs on two."""
    block = block_step.Block(batch=2, length=70, heads=4, kv_heads=2, head_dim=32, hidden=200, dropout=0.2)
    block.x[0].copy_(torch.randn(block.rows, block.width, generator=torch.Generator().manual_seed(3)))
    start, grad = block.x[0].clone(), torch.randn(block.rows, block.width, generator=torch.Generator().manual_seed(4)).cuda()
    want = block.forward().clone()
    grads = {k: t.clone() for k, t in block.backward(grad).items()}
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(other):
        assert block.stream == other
        block.x[0].copy_(start)
        got = block.forward()
        again = block.backward(grad)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and all(torch.equal(again[k], t) for k, t in grads.items())
    assert block.stream != other
