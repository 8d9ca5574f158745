"""Sampling refuses bad arguments on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2607_08642_amd import binding as b
from test_verify_abi import ALIGN, AT, DTYPE, NULL, SHAPE, UNSUPPORTED, WORKSPACE, ref

NAN, INF = float("nan"), float("inf")


def call(logits=AT, stride=1000, rows=4, V=1000, dtype=b.DT_F32, u=AT, tokens=AT, logprobs=AT, ws=AT, size=1 << 30, how=True,
         **kw):
    a = dict(temperature=1.0, top_p=1.0, min_p=0.0, top_k=0, temperatures=None, top_ps=None, min_ps=None, top_ks=None)
    a.update(kw)
    return b.load().dt_sample(logits, stride, rows, V, dtype, u, ref(b.dt_sampling(*a.values())) if how else None, tokens,
                              logprobs, ws, size, None)


@pytest.mark.parametrize("fault,status", [
    (dict(logits=None), NULL), (dict(u=None), NULL), (dict(tokens=None), NULL), (dict(how=False), NULL),
    (dict(dtype=b.DT_F8), DTYPE), (dict(dtype=-1), DTYPE), (dict(rows=0), SHAPE), (dict(V=0), SHAPE), (dict(V=-5), SHAPE),
    (dict(V=(1 << 19) + 1), UNSUPPORTED), (dict(rows=0x7fffffff), UNSUPPORTED), (dict(rows=1 << 23, V=10000), UNSUPPORTED),
    (dict(stride=-1), SHAPE), (dict(temperature=-0.5), SHAPE), (dict(temperature=NAN), SHAPE), (dict(top_k=-1), SHAPE),
    (dict(top_p=-0.1), SHAPE), (dict(top_p=NAN), SHAPE), (dict(min_p=-0.1), SHAPE), (dict(min_p=1.5), SHAPE),
    (dict(min_p=NAN), SHAPE), (dict(logits=AT + 2), ALIGN), (dict(logits=AT + 1, dtype=b.DT_BF16), ALIGN),
    (dict(u=AT + 2), ALIGN), (dict(tokens=AT + 2), ALIGN), (dict(logprobs=AT + 1), ALIGN), (dict(temperatures=AT + 2), ALIGN),
    (dict(top_ks=AT + 2), ALIGN), (dict(top_ps=AT + 2), ALIGN), (dict(min_ps=AT + 2), ALIGN), (dict(ws=None), WORKSPACE),
    (dict(size=8), WORKSPACE), (dict(ws=AT + 64), ALIGN)])
def test_refusals(fault, status):
    assert call(**fault) == status


def test_workspace():
    n = ctypes.c_size_t(7)
    L = b.load()
    assert L.dt_sample_workspace_size(4, 151936, ref(n)) == 0 and n.value > 0
    assert call(V=151936, size=n.value - 1) == WORKSPACE
    m = ctypes.c_size_t(7)
    for rows, V, status in ((0, 10, SHAPE), (4, 0, SHAPE), (4, 1 << 20, UNSUPPORTED), (1 << 30, 100000, UNSUPPORTED)):
        assert L.dt_sample_workspace_size(rows, V, ref(m)) == status and m.value == 7
    assert L.dt_sample_workspace_size(4, 10, None) == NULL


def test_the_binding_refuses_host_tensors():
    with pytest.raises(ValueError):
        b.sample(torch.zeros(2, 8), torch.zeros(2))
