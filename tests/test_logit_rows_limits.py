"""Ends of the ranges that the operators on rows of logits allow (no GPU needed)."""
import numpy as np
import pytest

from paper_2605_27081_b200 import binding as rb

B = np.zeros(4096, np.float32)
D = np.zeros(64, np.float32)
CALLS = [
    lambda n, s: rb.remoe_token_logprobs(n, 16, rb.REMOE_F32, B, 16, s, B, 4, B, B, B, B, None),
    lambda n, s: rb.remoe_token_logprobs_backward(n, 16, rb.REMOE_F32, B, 16, s, B, B, B, B, D, 16),
    lambda n, s: rb.remoe_distill_topk(n, 16, rb.REMOE_F32, B, 16, s, 4, B, B, 0, B, B, None, None, 0),
    lambda n, s: rb.remoe_distill_topk_backward(n, 16, rb.REMOE_F32, B, 16, s, 4, B, B, B, B, D, 16),
]


@pytest.mark.parametrize("call", CALLS)
def test_inverse_temperature(call):
    for s in (2.0 ** -100, 1e-30, 1.0, 1e25, 2.0 ** 100):
        assert call(0, s) == rb.REMOE_OK
    for s in (2.0 ** -100 * (1 - 2.0 ** -23), 2.0 ** 100 * (1 + 2.0 ** -23), 1e-45, 2.3e38, 2.4e38, 3.4e38, -2.0 ** -100):
        assert call(0, s) == rb.REMOE_E_ARG and call(2, s) == rb.REMOE_E_ARG
