"""Limits of the experts' products that the header states (no GPU needed)."""
import os
import re

import pytest

from paper_2605_27081_b200 import binding as rb
from test_experts_args import ARG, UNSUPPORTED, _ffn, _ffn_backward


@pytest.mark.parametrize("call", [_ffn, _ffn_backward])
def test_rows_times_channels(call):
    assert call(n_rows=1 << 30, inter=256) == UNSUPPORTED
    assert call(n_rows=1 << 22, inter=65536) == UNSUPPORTED
    assert call(n_rows=(1 << 22) - 1, inter=65536, block_stride=3 * 65536 * 16, **({"d_block_stride": 3 * 65536 * 16} if call is _ffn_backward else {})) \
        in (ARG, rb.REMOE_E_CUDA)                        # (the buffers are the host's)


@pytest.mark.parametrize("call,strides", [(_ffn, ["xs_stride", "ys_stride"]), (_ffn_backward, ["xs_stride", "d_ys_stride", "d_xs_stride"])])
def test_strides_of_rows_and_of_blocks(call, strides):
    for name in strides:
        assert call(**{name: 1 << 38}) == ARG
        assert call(**{name: (1 << 38) - 8}) in (ARG, rb.REMOE_E_CUDA)
    assert call(block_stride=1 << 38) == UNSUPPORTED
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "remoe.h")).read()
    assert re.search(r"below 2\^38 \(from there on ARG for those of rows, UNSUPPORTED for those of blocks\), n_rows \* inter is below 2\^38", text)
