"""The calls on the 8-bit cache check their arguments on the host before anything is launched (so these run without a GPU)."""
import ctypes
import random

import pytest
import torch

from paper_2512_17077_amd import hcsa

OK, INVALID, UNSUPPORTED, WORKSPACE = hcsa.DLLM_OK, hcsa.DLLM_ERR_INVALID_ARG, hcsa.DLLM_ERR_UNSUPPORTED, hcsa.DLLM_ERR_WORKSPACE
FAKE = 0x30000   # never dereferenced: every call here fails before a launch, or has nothing to launch


def good_batch():
    b = hcsa.DllmBatch()
    b.dtype = hcsa.DLLM_BF16
    b.batch, b.n_q_heads, b.n_kv_heads, b.head_dim = 2, 8, 2, 128
    b.q = b.k = b.v = 0x10000
    b.q_stride_tok, b.q_stride_head = 8 * 128, 128
    b.kv_stride_tok, b.kv_stride_head = 2 * 128, 128
    b.cu_q = b.cu_kv = 0x20000
    b.total_q, b.total_kv, b.max_q, b.max_kv = 64, 9000, 32, 4000
    b.softmax_scale = 0.088
    return b


def good_cache():
    c = hcsa.DllmCache()
    c.k, c.v, c.k_scale, c.v_scale = 0x40000, 0x50000, 0x60001, 0x60801
    c.stride_tok, c.stride_head = 256, 128
    c.scale_stride_head, c.scale_block = 9000 // 32 + 2, 32
    return c


def write(b, c, cu_rows=FAKE, total=40, most=32, at=FAKE):
    return hcsa.lib().dllm_hcsa_cache_write(b and ctypes.byref(b), c and ctypes.byref(c), cu_rows, total, most, at, None)


def read(b, c, cu_rows=FAKE, total=40, most=32, at=FAKE, k=0x70000, v=0x80000):
    return hcsa.lib().dllm_hcsa_cache_read(b and ctypes.byref(b), c and ctypes.byref(c), cu_rows, total, most, at, k, v, None)


def select(b, c, cu_k=FAKE, total=100, most=50, pool_w=1, forced=0, head_sum=0, idx=FAKE, ws=FAKE, nbytes=1 << 40):
    return hcsa.lib().dllm_hcsa_select_cached(b and ctypes.byref(b), c and ctypes.byref(c), cu_k, total, most, pool_w, forced,
                                              head_sum, idx, ws, nbytes, None)


def attend(b, c, idx=FAKE, cu_k=FAKE, total=100, most=50, o=0x90000, ws=0x30000, nbytes=1 << 40):
    return hcsa.lib().dllm_hcsa_attend_cached(b and ctypes.byref(b), c and ctypes.byref(c), idx, cu_k, total, most, o, ws, nbytes,
                                              None)


EVERY = (write, read, select, attend)


def test_scale_slots_hold_every_sequence_apart():
    slots = hcsa.cache_scale_slots
    assert slots(0, 1, 16) == 1 and slots(500, 2, 32) == 17 and slots(64, 1, 64) == 2
    for bad in ((-1, 1, 32), (10, 0, 32), (10, 1, 8), (10, 1, 0), (10, 1, 33)):
        with pytest.raises(ValueError):
            slots(*bad)
    rng = random.Random(3)
    for _ in range(3000):
        t = rng.choice((16, 32, 64))
        lens = [rng.choice((0, 1, t - 1, t, t + 1, rng.randint(0, 300))) for _ in range(rng.randint(1, 12))]
        end = start = 0
        for b, n in enumerate(lens):
            first = start // t + b
            assert first >= end   # behind the sequence before it
            end, start = first + -(-n // t), start + n
        assert end <= slots(start, len(lens), t)


@pytest.mark.parametrize("call", EVERY)
@pytest.mark.parametrize("field,value,status", [
    ("k", 0, INVALID), ("v", 0, INVALID), ("k_scale", 0, INVALID), ("v_scale", 0, INVALID), ("k", 0x40008, INVALID), ("v", 0x40001, INVALID),
    ("stride_tok", 112, INVALID), ("stride_tok", 264, INVALID), ("stride_head", 64, INVALID), ("stride_head", 136, INVALID),
    ("scale_block", 0, INVALID), ("scale_block", 8, INVALID), ("scale_block", 48, INVALID), ("scale_block", 128, INVALID), ("scale_block", -32, INVALID),
    ("scale_stride_head", 282, INVALID), ("scale_stride_head", 0, INVALID)])
def test_bad_cache_descriptor_is_rejected_everywhere(call, field, value, status):
    c = good_cache()
    setattr(c, field, value)
    assert call(good_batch(), c) == status and hcsa.last_error() != ""
    assert call(good_batch(), None) == INVALID and "cache descriptor" in hcsa.last_error()
    assert call(None, good_cache()) == INVALID


@pytest.mark.parametrize("call,reads_q", [(write, False), (read, False), (select, True), (attend, True)])
def test_a_call_checks_the_part_of_the_batch_that_it_reads(call, reads_q):
    for field, value in (("batch", 0), ("n_kv_heads", 3), ("n_kv_heads", 0), ("head_dim", 96), ("cu_kv", 0), ("max_kv", 9001),
                         ("total_kv", -1), ("dtype", 2)):
        b = good_batch()
        setattr(b, field, value)
        assert call(b, good_cache()) == INVALID, field
    q_fields = (("q", 0), ("cu_q", 0), ("max_q", 65), ("q_stride_head", 64), ("q_stride_tok", 1028), ("q", 0x10002), ("softmax_scale", 0.0),
                ("softmax_scale", float("nan")))
    for field, value in q_fields:
        b = good_batch()
        setattr(b, field, value)
        if reads_q:
            assert call(b, good_cache()) == INVALID, field
        else:   # nothing to move: the call passes its checks and launches nothing
            assert call(b, good_cache(), most=0) == OK, field
    kv_fields = (("kv_stride_tok", 127), ("kv_stride_tok", 260), ("kv_stride_head", 64))
    for field, value in kv_fields:
        b = good_batch()
        setattr(b, field, value)
        if reads_q:   # not read: the next check is the one that fails
            assert call(b, good_cache(), ws=None, nbytes=0, most=4000, total=8000) == WORKSPACE, field
        else:
            assert call(b, good_cache()) == INVALID, field


def test_write_and_read_check_their_ranges_and_tensors():
    for call in (write, read):
        assert call(good_batch(), good_cache(), total=-1) == INVALID
        assert call(good_batch(), good_cache(), total=40, most=41) == INVALID
        assert call(good_batch(), good_cache(), total=5000, most=4001) == INVALID
        assert call(good_batch(), good_cache(), most=-1) == INVALID
        assert call(good_batch(), good_cache(), cu_rows=None, total=8999) == INVALID and "total_kv" in hcsa.last_error()
        empty = good_batch()
        empty.total_kv = empty.max_kv = 0
        assert call(empty, good_cache(), cu_rows=None, total=0) == OK   # nothing to move, nothing launched
        long = good_batch()
        long.n_q_heads = long.n_kv_heads = 1024
        long.total_kv = long.max_kv = 1 << 20
        c = good_cache()
        c.scale_stride_head = 1 << 20
        assert call(long, c, cu_rows=None, total=1 << 20) == UNSUPPORTED and "blocks" in hcsa.last_error()
        huge = good_batch()
        huge.total_kv = 2 ** 31 - 5
        assert call(huge, c) == UNSUPPORTED and "2^31" in hcsa.last_error()
    for k, v in ((0, 0x80000), (0x70000, 0), (0x70008, 0x80000), (0x70000, 0x80002)):
        assert read(good_batch(), good_cache(), k=k, v=v) == INVALID
    b = good_batch()
    b.k = b.v = 0   # what a read does not read
    assert read(b, good_cache(), most=0) == OK and write(b, good_cache()) == INVALID


def test_select_cached_checks():
    b, c = good_batch(), good_cache()
    for what in (dict(cu_k=None), dict(idx=None), dict(total=0), dict(most=0), dict(most=101), dict(most=4001, total=5000), dict(pool_w=2),
                 dict(pool_w=0), dict(pool_w=65), dict(forced=-1), dict(forced=51), dict(head_sum=2)):
        assert select(b, c, **what) == INVALID, what
    need = hcsa.dllm_hcsa_select_cached_workspace(b, c, 50)
    assert need == hcsa.dllm_hcsa_select_workspace(b, 50) > 0
    assert select(b, c, ws=None) == WORKSPACE and select(b, c, ws=FAKE + 16) == WORKSPACE and select(b, c, nbytes=need - 1) == WORKSPACE
    b.dtype = hcsa.DLLM_F32
    assert select(b, c) == UNSUPPORTED and "bf16" in hcsa.last_error() and hcsa.dllm_hcsa_select_cached_workspace(b, c, 50) == 0
    b = good_batch()
    b.total_kv = b.max_kv = 32769
    c.scale_stride_head = 2000
    assert select(b, c) == UNSUPPORTED


def test_attend_cached_checks():
    b, c = good_batch(), good_cache()
    for what in (dict(cu_k=None), dict(o=None), dict(o=0x90008), dict(total=-1, most=-1), dict(most=-1), dict(most=101), dict(most=4001, total=5000)):
        assert attend(b, c, **what) == INVALID, what
    need = hcsa.dllm_hcsa_attend_cached_workspace(b, c, 4000)
    assert need > 0
    assert attend(b, c, ws=None, most=4000, total=8000) == WORKSPACE and attend(b, c, nbytes=need - 1, most=4000, total=8000) == WORKSPACE
    assert hcsa.dllm_hcsa_attend_cached_workspace(b, c, -1) == 0
    b.dtype = hcsa.DLLM_F32
    assert attend(b, c) == UNSUPPORTED and hcsa.dllm_hcsa_attend_cached_workspace(b, c, 50) == 0
    b = good_batch()
    c.stride_tok = 1 << 24   # row offsets inside a sequence are 32 bits wide
    assert attend(b, c) == UNSUPPORTED
    c.stride_tok = (1 << 24) - 16
    b.max_kv = b.total_kv = 4000
    assert attend(b, c) == UNSUPPORTED
    c = good_cache()
    b = good_batch()
    assert attend(b, c, total=(1 << 27) + 1) == UNSUPPORTED and "2^27" in hcsa.last_error()
    b.max_kv = b.total_kv = (1 << 24) + 1
    c.scale_stride_head = 1 << 24
    assert attend(b, c) == UNSUPPORTED


def test_the_largest_lists_that_attention_takes():
    """Pieces of at most 2048 listed rows, at most 65535 of them; without lists the number of rows does not matter."""
    b, c = good_batch(), good_cache()
    most = (1 << 27) - 2048
    assert (most + 2047) // 2048 == 65535
    assert attend(b, c, total=most + 1) == UNSUPPORTED
    assert attend(b, c, total=most, ws=None) == WORKSPACE   # the next check


def test_tensors_of_another_device_are_refused(monkeypatch):
    """The calls launch on the current device."""
    q, cu = torch.zeros((4, 2, 64), dtype=torch.bfloat16), torch.tensor([0, 4], dtype=torch.int32)
    codes, scales = torch.zeros((4, 2, 64), dtype=torch.uint8), torch.zeros((2, 2), dtype=torch.uint8)
    c = hcsa.make_cache(codes, codes.clone(), scales, scales.clone(), 32)
    b, rows = hcsa.make_cached_batch(q, cu, cu, 4, 2, 4, 4, 1.0), hcsa.make_rows_batch(q, q.clone(), cu, 4, 4)
    c.of = b.of = rows.of = c.of[:3] + (1,)   # as if they lay on device 1
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="device 1.*device is 0"):
        hcsa.dllm_hcsa_cache_write(rows, c)
    with pytest.raises(ValueError, match="device 1"):
        hcsa.dllm_hcsa_select_cached(b, c, cu, 4, 4, torch.zeros((2, 4), dtype=torch.int32))
    with pytest.raises(ValueError, match="device 1"):
        hcsa.dllm_hcsa_attend_cached(b, c, None, cu, 4, 4, q)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)

    class OfDevice0:
        device_index, cuda_stream = 0, 0
    with pytest.raises(ValueError, match="stream is on device 0"):
        hcsa.dllm_hcsa_attend_cached(b, c, None, cu, 4, 4, q, stream=OfDevice0())


def shaped(rng):
    b, c = good_batch(), good_cache()
    d, group = rng.choice((64, 128)), rng.choice((1, 2, 4, 5, 8))
    b.batch, b.n_kv_heads, b.head_dim = int(2 ** rng.uniform(0, 8)), rng.choice((1, 2, 4, 8, 16, 32)), d
    b.n_q_heads = b.n_kv_heads * group
    b.q_stride_tok, b.q_stride_head = b.n_q_heads * d, d
    b.max_kv = int(2 ** rng.uniform(0, 14))
    b.total_kv = b.max_kv + int((b.batch - 1) * b.max_kv * rng.random())
    b.max_q = int(2 ** rng.uniform(0, 9))
    b.total_q = b.max_q + int((b.batch - 1) * b.max_q * rng.random())
    c.stride_tok, c.stride_head = b.n_kv_heads * d, d
    c.scale_stride_head = b.total_kv // 32 + b.batch
    return b, c, rng.randint(0, b.max_kv)


def test_an_attend_call_never_takes_more_workspace_than_the_query_asks_for():
    """The query does not know total_k nor whether there are lists: the segments that any call cuts have to fit what it said
    (head_dim + 2 floats per segment, query and head; a head's lists have at most one segment per piece and one per sequence)."""
    rng = random.Random(2)
    whole = cut = 0
    for _ in range(20000):
        b, c, max_k = shaped(rng)
        ws = hcsa.dllm_hcsa_attend_cached_workspace(b, c, max_k)
        for total_k in {max_k, max_k + rng.randint(0, (b.batch - 1) * max_k), b.batch * max_k, b.batch * max_k + 70000}:
            for lists in (False, True):
                piece = hcsa.dllm_hcsa_attend_cached_form_of(b, c, lists, max_k, total_k)
                whole, cut = whole + (piece == 0), cut + (piece > 0)
                assert not (lists and max_k > 2048) or piece > 0   # (what one workgroup can take of a list)
                assert not lists or piece <= 2048
                if piece:
                    pieces = -(-min(total_k, b.batch * max_k) // piece)
                    assert ws >= (pieces + b.batch) * b.max_q * b.n_q_heads * (b.head_dim + 2) * 4, (b.batch, max_k, total_k, lists, piece)
    assert whole > 10000 and cut > 10000


def test_attend_form_of_checks_its_arguments():
    b, c = good_batch(), good_cache()
    for lists, max_k, total_k in ((2, 10, 10), (-1, 10, 10), (0, -1, 10), (0, 11, 10), (1, 4001, 5000), (0, 0, -1)):
        assert hcsa.lib().dllm_hcsa_attend_cached_form_of(ctypes.byref(b), ctypes.byref(c), lists, max_k, total_k) == -1
    b.head_dim = 96
    with pytest.raises(ValueError):
        hcsa.dllm_hcsa_attend_cached_form_of(b, c, True, 10, 10)


def test_the_binding_refuses_tensors_that_do_not_fit():
    k = torch.zeros((40, 2, 64), dtype=torch.uint8)
    scale = torch.zeros((2, 3), dtype=torch.uint8)
    cu = torch.tensor([0, 40], dtype=torch.int32)
    cache = hcsa.make_cache(k, k.clone(), scale, scale.clone(), 32)
    rows = torch.zeros((40, 2, 64), dtype=torch.bfloat16)
    batch = hcsa.make_rows_batch(rows, rows.clone(), cu, 40, 40)
    one = torch.tensor([0, 8], dtype=torch.int32)
    at = torch.zeros(1, dtype=torch.int32)
    for call in (lambda: hcsa.make_cache(k, k.float(), scale, scale, 32), lambda: hcsa.make_cache(k, k, scale, scale, 24),
                 lambda: hcsa.make_cache(k, k, scale[:1], scale[:1], 32), lambda: hcsa.make_cache(k, k, scale.t(), scale.t(), 32),
                 lambda: hcsa.make_cache(k, k, scale.int(), scale.int(), 32), lambda: hcsa.make_cache(k, k[:39], scale, scale, 32),
                 lambda: hcsa.dllm_hcsa_cache_write(hcsa.make_rows_batch(rows[:30], rows[:30], cu, 40, 40), cache),
                 lambda: hcsa.dllm_hcsa_cache_write(batch, hcsa.make_cache(k, k, scale[:, :1], scale[:, :1], 32)),
                 lambda: hcsa.dllm_hcsa_cache_write(batch, cache, one, 41, 8, at), lambda: hcsa.dllm_hcsa_cache_write(batch, cache, one.long(), 8, 8, at),
                 lambda: hcsa.dllm_hcsa_cache_write(batch, cache, one, 8, 8, at.long()), lambda: hcsa.dllm_hcsa_cache_write(batch, cache, at=at),
                 lambda: hcsa.dllm_hcsa_cache_read(batch, cache, rows.clone(), rows.clone()),
                 lambda: hcsa.dllm_hcsa_cache_write(hcsa.make_rows_batch(rows, rows, cu, 39, 39), cache)):
        with pytest.raises(AssertionError):
            call()


def test_python_struct_matches_the_header_layout(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = [f[0] for f in hcsa.DllmCache._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "dllm_hcsa.h"\nint main(void) {\n' +
                   "".join(f'  printf("%zu ", offsetof(dllm_cache, {n}));\n' for n in names) +
                   '  printf("%zu\\n", sizeof(dllm_cache));\n  return 0;\n}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [getattr(hcsa.DllmCache, n).offset for n in names] + [ctypes.sizeof(hcsa.DllmCache)]
