"""What the Python binding does itself, without a GPU: where a call's own workspace comes from."""
import contextlib

import pytest
import torch

from paper_2512_17077_amd import hcsa


class Library:
    """The library's host functions, with every launch left out; says what a call was given."""

    def __init__(self):
        self.real, self.calls = hcsa.lib(), []

    def __getattr__(self, name):
        if name.endswith(("_workspace", "_form_of", "_error", "_slots")):
            return getattr(self.real, name)
        return lambda *args: self.calls.append((name, args)) or hcsa.DLLM_OK


@pytest.fixture
def library(monkeypatch):
    x = Library()
    monkeypatch.setattr(hcsa, "lib", lambda: x)
    return x


def ints(*x):
    return torch.tensor(x, dtype=torch.int32)


def operands(lens, hq=4, hkv=2, d=64):
    """A dense batch, a cache of the same sequences with its batch, and a call's other tensors; one query per sequence."""
    n, total = len(lens), sum(lens)
    cu = ints(*[sum(lens[:b]) for b in range(n + 1)])
    q, cu_q = torch.zeros((n, hq, d), dtype=torch.bfloat16), torch.arange(n + 1, dtype=torch.int32)
    k = torch.zeros((total, hkv, d), dtype=torch.bfloat16)
    codes, scales = torch.zeros((total, hkv, d), dtype=torch.uint8), torch.zeros((hkv, total // 32 + n), dtype=torch.uint8)
    return dict(dense=hcsa.make_batch(q, k, k.clone(), cu_q, cu, 1, max(lens), 0.125),
                cache=hcsa.make_cache(codes, codes.clone(), scales, scales.clone(), 32),
                cached=hcsa.make_cached_batch(q, cu_q, cu, total, hkv, 1, max(lens), 0.125),
                idx=torch.zeros((hq, total), dtype=torch.int32), o=torch.zeros_like(q), cu_k=cu, total=total, most=max(lens))


CALLS = {
    "select": lambda x, **more: hcsa.dllm_hcsa_select(x["dense"], x["cu_k"], x["total"], x["most"], x["idx"], **more),
    "select_ex": lambda x, **more: hcsa.dllm_hcsa_select_ex(x["dense"], x["cu_k"], x["total"], x["most"], x["idx"], **more),
    "attend": lambda x, **more: hcsa.dllm_hcsa_attend(x["dense"], x["idx"], x["cu_k"], x["total"], x["most"], None, x["o"], **more),
    "select_cached": lambda x, **more: hcsa.dllm_hcsa_select_cached(x["cached"], x["cache"], x["cu_k"], x["total"], x["most"], x["idx"], **more),
    "attend_cached": lambda x, **more: hcsa.dllm_hcsa_attend_cached(x["cached"], x["cache"], None, x["cu_k"], x["total"], x["most"], x["o"], **more)}


@pytest.mark.parametrize("call", CALLS)
def test_a_workspace_is_allocated_on_the_stream_that_uses_it(monkeypatch, library, call):
    """Memory of the current stream's pool may still be in use there, and the call's stream would not wait for that."""
    class Side:
        device_index, cuda_stream = None, 77

    now, took = [None], []

    @contextlib.contextmanager
    def on(stream):
        now.append(stream)
        yield
        now.pop()

    def empty(*args, **kind):
        took.append(now[-1])
        return torch.zeros(*args, dtype=kind["dtype"])

    x, side = operands([9000, 4000]), Side()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: None)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 5, raising=False)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda raw, device=None: side)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, stream: None)
    CALLS[call](x, stream=side)
    assert took == [side] and library.calls[-1][1][-1] == 77
    CALLS[call](x)
    assert took == [side, None] and library.calls[-1][1][-1] == 5
    CALLS[call](x, workspace=torch.zeros(64, dtype=torch.uint8), stream=side)
    assert len(took) == 2   # the caller's own
