"""The norm, routing, row moves and grouped products together: a training step of the example's
mixture-of-experts block against FP32 PyTorch.

An E4M3 element is off by at most 2^-4 of itself, 0.026 in the mean square; a product of two quantized
operands by 0.026 * sqrt(2) = 0.037 of its norm.  The results depend on one to four such products in a chain:
at most 0.037 * sqrt(4) = 0.074; held to twice that."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,dim,ffn,experts,topk", [(512, 512, 384, 8, 2), (77, 256, 128, 16, 4), (1, 128, 128, 4, 1)])
def test_training_step_against_fp32(tokens, dim, ffn, experts, topk):
    import moe_block
    errors = moe_block.compare(tokens, dim, ffn, experts, topk)
    if topk == 1:
        errors.pop("router")  # a renormalised single choice does not depend on the router
    assert all(e < 0.15 for e in errors.values()), errors


def test_step_does_not_depend_on_what_lies_behind_the_last_group():
    """Rows that no group holds are never read: the same step with poisoned memory."""
    import moe_block
    block = moe_block.MoeBlock(256, 128, 8, 2)
    x, res = (torch.randn(100, 256, device="cuda").bfloat16() for _ in range(2))
    want, saved = block.forward(x, res)
    want_g = block.backward(x, res, saved)
    del saved
    for _ in range(3):
        junk = [torch.full((n,), float("nan"), device="cuda") for n in (1 << 16, 1 << 18, 1 << 20)]
        del junk
        out, saved = block.forward(x, res)
        grads = block.backward(x, res, saved)
        assert torch.equal(out, want) and all(torch.equal(grads[k], want_g[k]) for k in grads)
