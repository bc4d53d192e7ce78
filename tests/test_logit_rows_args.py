"""Refusals of the operators on rows of logits: every bad argument is told before anything is launched (no GPU needed)."""
import numpy as np
import pytest

from paper_2605_27081_b200 import binding as rb

N = None


def _ok_logprobs(**kw):
    buf = np.zeros(4096, np.float32)
    a = dict(n_rows=2, vocab=16, dtype=rb.REMOE_F32, logits=buf, row_stride=16, inv_temperature=1.0, tokens=buf, top_k=4,
             logprob=buf, entropy=buf, top_ids=buf, top_logprob=buf, row_stats=N)
    a.update(kw)
    return rb.remoe_token_logprobs(**a)


def _ok_logprobs_backward(**kw):
    buf = np.zeros(4096, np.float32)
    a = dict(n_rows=2, vocab=16, dtype=rb.REMOE_F32, logits=buf, row_stride=16, inv_temperature=1.0, tokens=buf, row_stats=buf,
             grad_logprob=buf, grad_entropy=buf, d_logits=np.zeros(64, np.float32), d_row_stride=16)
    a.update(kw)
    return rb.remoe_token_logprobs_backward(**a)


def _ok_distill(**kw):
    buf = np.zeros(4096, np.float32)
    a = dict(n_rows=2, vocab=16, dtype=rb.REMOE_F32, logits=buf, row_stride=16, inv_temperature=1.0, n_top=4, teacher_ids=buf,
             teacher_logprobs=buf, tail=0, row_weight=buf, loss=buf, row_stats=N, d_logits=N, d_row_stride=0)
    a.update(kw)
    return rb.remoe_distill_topk(**a)


def _ok_distill_backward(**kw):
    buf = np.zeros(4096, np.float32)
    a = dict(n_rows=2, vocab=16, dtype=rb.REMOE_F32, logits=buf, row_stride=16, inv_temperature=1.0, n_top=4, teacher_ids=buf,
             teacher_logprobs=buf, row_stats=buf, grad_loss=buf, d_logits=np.zeros(64, np.float32), d_row_stride=16)
    a.update(kw)
    return rb.remoe_distill_topk_backward(**a)


ALL = [_ok_logprobs, _ok_logprobs_backward, _ok_distill, _ok_distill_backward]


@pytest.mark.parametrize("call", ALL)
def test_host_memory_is_refused(call):
    # the arguments are in order, but the rows lie in host memory; without a device the runtime call fails instead
    assert call() in (rb.REMOE_E_ARG, rb.REMOE_E_CUDA)


@pytest.mark.parametrize("call", ALL)
@pytest.mark.parametrize("kw,code", [
    (dict(n_rows=-1), rb.REMOE_E_ARG), (dict(vocab=0), rb.REMOE_E_ARG), (dict(logits=N), rb.REMOE_E_ARG),
    (dict(vocab=rb.REMOE_ROWS_MAX_VOCAB + 1, row_stride=1 << 21), rb.REMOE_E_UNSUPPORTED),
    (dict(dtype=rb.REMOE_FP8_E4M3), rb.REMOE_E_UNSUPPORTED), (dict(dtype=rb.REMOE_INT4_G32), rb.REMOE_E_UNSUPPORTED),
    (dict(dtype=5), rb.REMOE_E_ARG), (dict(dtype=-1), rb.REMOE_E_ARG),
    (dict(row_stride=15), rb.REMOE_E_ARG), (dict(row_stride=-16), rb.REMOE_E_ARG),
    (dict(inv_temperature=0.0), rb.REMOE_E_ARG), (dict(inv_temperature=-1.0), rb.REMOE_E_ARG),
    (dict(inv_temperature=float("nan")), rb.REMOE_E_ARG), (dict(inv_temperature=float("inf")), rb.REMOE_E_ARG),
    (dict(logits=4097), rb.REMOE_E_ARG),
])
def test_bad_rows(call, kw, code):
    assert call(**kw) == code


@pytest.mark.parametrize("call", ALL)
def test_no_rows_is_fine(call):
    assert call(n_rows=0) == rb.REMOE_OK


@pytest.mark.parametrize("kw,code", [
    (dict(top_k=-1), rb.REMOE_E_ARG), (dict(top_k=17), rb.REMOE_E_ARG),
    (dict(top_k=257, vocab=512, row_stride=512), rb.REMOE_E_UNSUPPORTED),
    (dict(top_ids=N), rb.REMOE_E_ARG), (dict(top_logprob=N), rb.REMOE_E_ARG), (dict(tokens=N), rb.REMOE_E_ARG),
    (dict(logprob=N, entropy=N, top_k=0), rb.REMOE_E_ARG), (dict(entropy=4098), rb.REMOE_E_ARG), (dict(tokens=4098), rb.REMOE_E_ARG),
])
def test_bad_logprobs(kw, code):
    assert _ok_logprobs(**kw) == code


@pytest.mark.parametrize("kw", [dict(row_stats=N), dict(d_logits=N), dict(d_row_stride=15), dict(tokens=N), dict(d_logits=4098),
                                dict(grad_logprob=N, grad_entropy=N), dict(row_stats=4098)])
def test_bad_logprobs_backward(kw):
    assert _ok_logprobs_backward(**kw) == rb.REMOE_E_ARG


@pytest.mark.parametrize("call", [_ok_distill, _ok_distill_backward])
@pytest.mark.parametrize("kw,code", [
    (dict(n_top=0), rb.REMOE_E_ARG), (dict(n_top=17), rb.REMOE_E_ARG), (dict(n_top=257, vocab=512, row_stride=512, d_row_stride=512), rb.REMOE_E_UNSUPPORTED),
    (dict(teacher_ids=N), rb.REMOE_E_ARG), (dict(teacher_logprobs=N), rb.REMOE_E_ARG), (dict(teacher_ids=4098), rb.REMOE_E_ARG),
    (dict(d_logits=np.zeros(64, np.float32), d_row_stride=15), rb.REMOE_E_ARG),
])
def test_bad_distill(call, kw, code):
    assert call(**kw) == code


@pytest.mark.parametrize("kw", [dict(tail=2), dict(loss=N), dict(row_weight=4098)])
def test_bad_distill_forward(kw):
    assert _ok_distill(**kw) == rb.REMOE_E_ARG


@pytest.mark.parametrize("kw", [dict(row_stats=N), dict(grad_loss=N), dict(d_logits=N)])
def test_bad_distill_backward(kw):
    assert _ok_distill_backward(**kw) == rb.REMOE_E_ARG


def test_in_place_needs_one_stride():
    buf = np.zeros(4096, np.float32)
    assert _ok_logprobs_backward(logits=buf, d_logits=buf, d_row_stride=32) == rb.REMOE_E_ARG
    assert _ok_distill(logits=buf, d_logits=buf, d_row_stride=32) == rb.REMOE_E_ARG
    assert _ok_distill_backward(logits=buf, d_logits=buf, d_row_stride=32) == rb.REMOE_E_ARG


def test_a_stack_takes_no_half_precision_weights():
    shape = dict(n_layers=1, hidden=256, n_routed=8, top_k=2, inter_routed=64, n_shared=0, inter_shared=0, shared_gate=0,
                 renorm_topk=0, weight_dtype=rb.REMOE_F16, batch=1)
    assert rb.remoe_stack_create(shape, 4)[0] == rb.REMOE_E_ARG
