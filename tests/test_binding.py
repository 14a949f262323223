"""What the Python binding does itself, without a GPU: where a call's own workspace comes from, what it refuses."""
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
    monkeypatch.setattr(hcsa, "_lib", x)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: None)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 5, raising=False)
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
    side.cuda_stream = 0   # no handle of an external stream, but the default one
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: "default")
    CALLS[call](x, stream=side)
    assert took[2:] == ["default"] and library.calls[-1][1][-1] == 0


class Elsewhere(torch.Tensor):
    """A tensor that says it lies on another device."""

    def get_device(self):
        return 1


def elsewhere(t):
    return t.as_subclass(Elsewhere)


def spread(t):
    """t's values, with gaps between them."""
    return torch.stack([t, t], -1)[..., 0]


CU, IDX, O = ints(0, 40, 100), torch.zeros((4, 100), dtype=torch.int32), torch.zeros((2, 4, 64), dtype=torch.bfloat16)


@pytest.mark.parametrize("name,value", [
    ("cu_k", CU.long()), ("cu_k", CU[:2]), ("cu_k", spread(CU)), ("cu_k", elsewhere(CU)), ("cu_k", CU.float()), ("cu_k", torch.cat([CU, CU])),
    ("idx", IDX.long()), ("idx", IDX[:3]), ("idx", IDX[:, :99]), ("idx", IDX.t().contiguous()), ("idx", IDX.t().contiguous().t()),
    ("idx", spread(IDX)), ("idx", elsewhere(IDX)), ("idx", torch.zeros((4, 101), dtype=torch.int32)), ("idx", IDX.reshape(-1)),
    ("idx", torch.zeros((4, 101), dtype=torch.int32)[:, :100]),
    ("o", O.half()), ("o", O.float()), ("o", O[:1]), ("o", O.reshape(2, 256)), ("o", O.transpose(0, 1).contiguous()), ("o", spread(O)),
    ("o", torch.zeros((2, 5, 64), dtype=torch.bfloat16)[:, :4]), ("o", elsewhere(O)),
    ("workspace", elsewhere(torch.zeros(1 << 20, dtype=torch.uint8))), ("workspace", spread(torch.zeros(1 << 20, dtype=torch.uint8)))])
def test_calls_on_the_cache_refuse_tensors_that_their_kernels_would_misread(library, name, value):
    """Types, shapes, gaps and devices: a kernel gets an address only and takes the rest as documented."""
    x = operands([40, 60])

    def calls(x, workspace):
        if name != "o":
            yield lambda: hcsa.dllm_hcsa_select_cached(x["cached"], x["cache"], x["cu_k"], 100, 60, x["idx"], workspace=workspace)
        yield lambda: hcsa.dllm_hcsa_attend_cached(x["cached"], x["cache"], x["idx"], x["cu_k"], 100, 60, x["o"], workspace=workspace)
        if name != "idx":
            yield lambda: hcsa.dllm_hcsa_attend_cached(x["cached"], x["cache"], None, x["cu_k"], 100, 60, x["o"], workspace=workspace)

    good = torch.zeros(1 << 20, dtype=torch.uint8)
    done = 0
    for call in calls(x, good):
        call()
        done += 1
    assert len(library.calls) == done >= 2
    for call in calls(x if name == "workspace" else dict(x, **{name: value}), value if name == "workspace" else good):
        with pytest.raises(AssertionError):
            call()
    assert len(library.calls) == done   # nothing was launched


def test_writes_reads_and_descriptors_refuse_them_too(library):
    x = operands([40, 60])
    rows = torch.zeros((100, 2, 64), dtype=torch.bfloat16)
    cu, at, q = CU.clone(), ints(0, 0), torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    cu_q = ints(0, 1, 2)
    batch = hcsa.make_rows_batch(rows, rows.clone(), cu, 100, 60)
    for bad in (dict(cu_rows=spread(cu)), dict(cu_rows=elsewhere(cu)), dict(cu_rows=cu.long()), dict(cu_rows=cu[:2]), dict(at=spread(at)),
                dict(at=elsewhere(at)), dict(at=at.long()), dict(at=at[:1])):
        args = dict(dict(cu_rows=cu, total_rows=100, max_rows=60, at=at), **bad)
        with pytest.raises(AssertionError):
            hcsa.dllm_hcsa_cache_write(batch, x["cache"], **args)
        with pytest.raises(AssertionError):
            hcsa.dllm_hcsa_cache_read(batch, x["cache"], *batch.tensors[:2], **args)
    for make in (lambda: hcsa.make_rows_batch(rows, elsewhere(rows), cu, 100, 60), lambda: hcsa.make_rows_batch(rows, rows, elsewhere(cu), 100, 60),
                 lambda: hcsa.make_rows_batch(rows, rows, spread(cu), 100, 60), lambda: hcsa.make_rows_batch(rows, rows, cu.long(), 100, 60),
                 lambda: hcsa.make_cached_batch(q, spread(cu_q), cu, 100, 2, 1, 60, 0.1), lambda: hcsa.make_cached_batch(q, cu_q, spread(cu), 100, 2, 1, 60, 0.1),
                 lambda: hcsa.make_cached_batch(q, elsewhere(cu_q), cu, 100, 2, 1, 60, 0.1), lambda: hcsa.make_cached_batch(q, cu_q, elsewhere(cu), 100, 2, 1, 60, 0.1),
                 lambda: hcsa.make_cached_batch(q, cu_q.long(), cu, 100, 2, 1, 60, 0.1), lambda: hcsa.make_cached_batch(q, cu_q, cu[:2], 100, 2, 1, 60, 0.1)):
        with pytest.raises(AssertionError):
            make()
    assert not library.calls
    hcsa.dllm_hcsa_cache_write(batch, x["cache"], cu, 100, 60, at)
    hcsa.dllm_hcsa_cache_read(batch, x["cache"], *batch.tensors[:2], cu, 100, 60)
    assert len(library.calls) == 2


def test_ranges_without_their_sizes_are_refused(library):
    """(Nothing would be moved, and nothing would say so.)"""
    x, rows = operands([40, 60]), torch.zeros((100, 2, 64), dtype=torch.bfloat16)
    batch = hcsa.make_rows_batch(rows, rows.clone(), CU, 100, 60)
    for sizes in ({}, dict(total_rows=100), dict(max_rows=60)):
        with pytest.raises(AssertionError):
            hcsa.dllm_hcsa_cache_write(batch, x["cache"], CU, at=ints(0, 0), **sizes)
        with pytest.raises(AssertionError):
            hcsa.dllm_hcsa_cache_read(batch, x["cache"], *batch.tensors[:2], CU, **sizes)
    assert not library.calls
    hcsa.dllm_hcsa_cache_write(batch, x["cache"], CU, 0, 0)
    hcsa.dllm_hcsa_cache_write(batch, x["cache"])
    assert [call[1][3:5] for call in library.calls] == [(0, 0), (100, 0)]
