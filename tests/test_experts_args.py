"""Refusals of the operators on tokens sorted by expert: every bad argument is told before anything is launched (no GPU needed)."""
import numpy as np
import pytest

from paper_2605_27081_b200 import binding as rb

N = None
ARG, UNSUPPORTED = rb.REMOE_E_ARG, rb.REMOE_E_UNSUPPORTED
_raw = np.zeros(8192, np.float32)
BUF = (_raw.ctypes.data + 63) // 64 * 64          # 64-byte aligned host memory: refused where a device pointer is asked for


def _sort(**kw):
    a = dict(n_tokens=4, top_k=2, n_experts=8, ids=BUF, rows=BUF, offsets=BUF)
    a.update(kw)
    return rb.remoe_expert_sort(**a)


def _dispatch(**kw):
    a = dict(n_tokens=4, top_k=2, hidden=16, dtype=rb.REMOE_BF16, x=BUF, x_stride=16, rows=BUF, n_rows=8, xs=BUF, xs_stride=16)
    a.update(kw)
    return rb.remoe_expert_dispatch(**a)


def _combine(**kw):
    a = dict(n_tokens=4, top_k=2, hidden=16, dtype=rb.REMOE_BF16, n_rows=8, ys=BUF, ys_stride=16, rows=BUF, gates=BUF, base=BUF + 4096,
             base_stride=16, out=BUF, out_stride=16)
    a.update(kw)
    return rb.remoe_expert_combine(**a)


def _combine_backward(**kw):
    a = dict(n_tokens=4, top_k=2, hidden=16, dtype=rb.REMOE_BF16, d_out=BUF, d_out_stride=16, n_rows=8, ys=BUF, ys_stride=16, rows=BUF,
             gates=BUF, d_ys=BUF + 4096, d_ys_stride=16, d_gates=BUF)
    a.update(kw)
    return rb.remoe_expert_combine_backward(**a)


def _ffn(**kw):
    a = dict(n_rows=8, n_experts=2, hidden=16, inter=8, dtype=rb.REMOE_BF16, xs=BUF, xs_stride=16, offsets=BUF, blocks=BUF, block_stride=384,
             gate_up=BUF, act=BUF, ys=BUF, ys_stride=16)
    a.update(kw)
    return rb.remoe_expert_ffn(**a)


def _ffn_backward(**kw):
    a = dict(n_rows=8, n_experts=2, hidden=16, inter=8, dtype=rb.REMOE_BF16, xs=BUF, xs_stride=16, offsets=BUF, blocks=BUF, block_stride=384,
             gate_up=BUF, d_ys=BUF, d_ys_stride=16, work=BUF, d_xs=BUF + 4096, d_xs_stride=16, d_blocks=BUF, d_block_stride=384)
    a.update(kw)
    return rb.remoe_expert_ffn_backward(**a)


@pytest.mark.parametrize("call", [_sort, _dispatch, _combine, _combine_backward, _ffn, _ffn_backward])
def test_host_memory_is_refused(call):
    assert call() in (ARG, rb.REMOE_E_CUDA)


@pytest.mark.parametrize("kw,code", [
    (dict(n_tokens=-1), ARG), (dict(top_k=0), ARG), (dict(n_experts=0), ARG), (dict(ids=N), ARG), (dict(rows=N), ARG), (dict(offsets=N), ARG),
    (dict(ids=BUF + 2), ARG), (dict(rows=BUF + 1), ARG), (dict(offsets=BUF + 2), ARG), (dict(n_experts=rb.REMOE_SORT_MAX_EXPERTS + 1), UNSUPPORTED),
    (dict(n_tokens=1 << 28, top_k=8), UNSUPPORTED)])
def test_bad_sort(kw, code):
    assert _sort(**kw) == code


@pytest.mark.parametrize("call", [_dispatch, _combine, _combine_backward])
@pytest.mark.parametrize("kw,code", [
    (dict(n_tokens=-1), ARG), (dict(top_k=0), ARG), (dict(hidden=0), ARG), (dict(n_rows=-1), ARG), (dict(rows=N), ARG), (dict(rows=BUF + 2), ARG),
    (dict(dtype=rb.REMOE_FP8_E4M3), UNSUPPORTED), (dict(dtype=rb.REMOE_INT4_G32), UNSUPPORTED), (dict(dtype=5), ARG), (dict(dtype=-1), ARG),
    (dict(n_tokens=1 << 28, top_k=8), UNSUPPORTED), (dict(hidden=rb.REMOE_EXPERT_MAX_HIDDEN + 1), UNSUPPORTED)])
def test_bad_rows(call, kw, code):
    assert call(**kw) == code


@pytest.mark.parametrize("call,names", [(_dispatch, ["x", "xs"]), (_combine, ["ys", "out"]), (_combine_backward, ["d_out", "ys"]),
                                        (_ffn, ["xs", "ys"]), (_ffn_backward, ["xs", "d_ys"])])
def test_bad_matrices(call, names):
    for name in names:
        assert call(**{name: N}) == ARG
        assert call(**{name: BUF + 1}) == ARG
        assert call(**{name + "_stride": 15}) == ARG
        assert call(**{name + "_stride": -16}) == ARG


@pytest.mark.parametrize("call,kw", [
    (_combine, dict(base=BUF + 1)), (_combine, dict(base_stride=15)), (_combine, dict(gates=BUF + 2)), (_combine, dict(base=BUF, base_stride=24)),
    (_combine_backward, dict(d_ys=N, d_gates=N)), (_combine_backward, dict(d_ys=BUF + 1)), (_combine_backward, dict(d_ys_stride=15)),
    (_combine_backward, dict(d_gates=BUF + 2)), (_combine_backward, dict(gates=BUF + 2)), (_combine_backward, dict(d_ys=BUF, d_ys_stride=24))])
def test_bad_combine(call, kw):
    assert call(**kw) == ARG


@pytest.mark.parametrize("call", [_ffn, _ffn_backward])
@pytest.mark.parametrize("kw,code", [
    (dict(n_rows=-1), ARG), (dict(n_experts=0), ARG), (dict(hidden=0), ARG), (dict(inter=0), ARG), (dict(dtype=5), ARG),
    (dict(dtype=rb.REMOE_F32), UNSUPPORTED), (dict(dtype=rb.REMOE_FP8_E4M3), UNSUPPORTED), (dict(dtype=rb.REMOE_INT4_G32), UNSUPPORTED),
    (dict(hidden=20), UNSUPPORTED), (dict(inter=12), UNSUPPORTED), (dict(hidden=rb.REMOE_FFN_MAX_WIDTH + 8), UNSUPPORTED),
    (dict(inter=rb.REMOE_FFN_MAX_WIDTH + 8), UNSUPPORTED), (dict(n_experts=rb.REMOE_SORT_MAX_EXPERTS + 1), UNSUPPORTED),
    (dict(n_rows=(1 << 30) + 1), UNSUPPORTED), (dict(offsets=N), ARG), (dict(offsets=BUF + 2), ARG), (dict(blocks=N), ARG), (dict(blocks=BUF + 8), ARG),
    (dict(block_stride=383), ARG), (dict(block_stride=388), ARG), (dict(xs=BUF + 8), ARG), (dict(xs_stride=20), ARG), (dict(gate_up=BUF + 8), ARG)])
def test_bad_ffn(call, kw, code):
    assert call(**kw) == code


@pytest.mark.parametrize("kw", [dict(act=N), dict(act=BUF + 8), dict(ys=BUF + 8), dict(ys_stride=20)])
def test_bad_ffn_forward(kw):
    assert _ffn(**kw) == ARG


@pytest.mark.parametrize("kw", [dict(gate_up=N), dict(work=N), dict(work=BUF + 8), dict(d_xs=N, d_blocks=N), dict(d_xs=BUF + 8), dict(d_xs_stride=20),
                                dict(d_blocks=BUF + 8), dict(d_block_stride=383), dict(d_block_stride=388), dict(d_xs=BUF),
                                dict(d_xs=BUF, d_blocks=N, d_xs_stride=24)])
def test_bad_ffn_backward(kw):
    assert _ffn_backward(**kw) == ARG


def test_strides_beyond_a_copy():
    far = 1 << 38
    assert _ffn(block_stride=far) == UNSUPPORTED and _ffn_backward(block_stride=far) == UNSUPPORTED
    assert _ffn_backward(d_block_stride=far) == UNSUPPORTED
    assert _ffn(xs_stride=far) == ARG and _ffn_backward(d_ys_stride=far) == ARG


def test_nothing_to_do_is_fine():
    for call in (_dispatch, _combine, _combine_backward):
        assert call(n_tokens=0) == rb.REMOE_OK
        assert call(n_tokens=0, rows=N) == rb.REMOE_OK
    assert _dispatch(n_tokens=0, x=N, rows=N, n_rows=0, xs=N) == rb.REMOE_OK
    assert _dispatch(n_rows=0, xs=N) == rb.REMOE_OK
    assert _ffn(n_rows=0, xs=N, ys=N, act=N, gate_up=N) == rb.REMOE_OK
    assert _ffn_backward(n_rows=0, xs=N, d_ys=N, work=N, gate_up=N, d_xs=N, d_blocks=N) == rb.REMOE_OK


def test_header_and_binding_name_the_same_limits():
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "remoe.h")).read()
    for name in ("REMOE_SORT_MAX_EXPERTS", "REMOE_EXPERT_MAX_HIDDEN", "REMOE_FFN_MAX_WIDTH"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(rb, name)
