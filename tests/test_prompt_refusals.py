"""What the calls between a prompt and its paged cache refuse, and with which status (host only, nothing is launched), and what
the binding refuses before them."""
import ctypes

import pytest
import torch

import paper_2604_16957_amd as tq
from paper_2604_16957_amd import binding as B

FAKE = 0x10000


def _x(**kw):
    f = dict(q=FAKE, k=FAKE, v=FAKE, q_stride=64 * 128, k_stride=8 * 128, v_stride=8 * 128, n_tokens=100, n_q_heads=64, n_kv_heads=8,
             head_dim=128, dtype=0)
    f.update(kw)
    return B.TqPackedStruct(*[f[n] for n, _ in B.TqPackedStruct._fields_])


def _prefill(x, cu=FAKE, n=1, scale=0.1, window=0, out=FAKE):
    return B.raw().tq_sdpa_prefill(ctypes.byref(x) if x is not None else None, cu, n, scale, window, out, None)


@pytest.mark.parametrize("kw,args,want", [
    (None, {}, B.TQ_ERR_NULL), (dict(q=None), {}, B.TQ_ERR_NULL), (dict(k=None), {}, B.TQ_ERR_NULL), (dict(v=None), {}, B.TQ_ERR_NULL),
    ({}, dict(cu=None), B.TQ_ERR_NULL), ({}, dict(out=None), B.TQ_ERR_NULL),
    (dict(head_dim=64), {}, B.TQ_ERR_SHAPE), (dict(head_dim=192), {}, B.TQ_ERR_SHAPE), (dict(n_kv_heads=0), {}, B.TQ_ERR_SHAPE),
    (dict(n_q_heads=63), {}, B.TQ_ERR_SHAPE), (dict(n_q_heads=0), {}, B.TQ_ERR_SHAPE),
    (dict(k_stride=8 * 128 - 8), {}, B.TQ_ERR_SHAPE), (dict(v_stride=0), {}, B.TQ_ERR_SHAPE), (dict(q_stride=64 * 128 + 4), {}, B.TQ_ERR_SHAPE),
    (dict(k_stride=1 << 24), {}, B.TQ_ERR_SHAPE), (dict(q_stride=-(64 * 128)), {}, B.TQ_ERR_SHAPE),
    (dict(n_tokens=0), {}, B.TQ_ERR_EMPTY), ({}, dict(n=0), B.TQ_ERR_EMPTY), ({}, dict(n=-1), B.TQ_ERR_EMPTY),
    (dict(dtype=2), {}, B.TQ_ERR_UNSUPPORTED), (dict(dtype=-1), {}, B.TQ_ERR_UNSUPPORTED), ({}, dict(window=-1), B.TQ_ERR_UNSUPPORTED),
    ({}, dict(scale=float("nan")), B.TQ_ERR_UNSUPPORTED), ({}, dict(scale=float("inf")), B.TQ_ERR_UNSUPPORTED),
    ({}, dict(n=1 << 30), B.TQ_ERR_UNSUPPORTED), (dict(n_tokens=(1 << 31) - 1), {}, B.TQ_ERR_UNSUPPORTED),
    (dict(q=FAKE + 8), {}, B.TQ_ERR_ALIGN), (dict(k=FAKE + 2), {}, B.TQ_ERR_ALIGN), (dict(v=FAKE + 4), {}, B.TQ_ERR_ALIGN),
    ({}, dict(out=FAKE + 8), B.TQ_ERR_ALIGN), ({}, dict(cu=FAKE + 2), B.TQ_ERR_ALIGN)])
def test_prefill_refuses(kw, args, want):
    assert _prefill(None if kw is None else _x(**kw), **args) == want


def _cache(**kw):
    f = dict(k_codes=FAKE, v_codes=FAKE, k_scale=FAKE, k_zero=FAKE, v_scale=FAKE, v_zero=FAKE,
             batch=16, n_kv_heads=8, head_dim=128, group_size=32, capacity=64, layout=0)
    f.update(kw)
    return B.TqKvCacheStruct(*[f[n] for n, _ in B.TqKvCacheStruct._fields_])


def _store(cache, x, slots=FAKE):
    return B.raw().tq_quantize_kv_slots(ctypes.byref(cache) if cache is not None else None,
                                        ctypes.byref(x) if x is not None else None, slots, None)


@pytest.mark.parametrize("cache,kw,slots,want", [
    (None, {}, FAKE, B.TQ_ERR_NULL), ({}, None, FAKE, B.TQ_ERR_NULL), ({}, {}, None, B.TQ_ERR_NULL), ({}, dict(k=None), FAKE, B.TQ_ERR_NULL),
    (dict(v_zero=None), {}, FAKE, B.TQ_ERR_NULL), (dict(head_dim=64), {}, FAKE, B.TQ_ERR_SHAPE), (dict(group_size=48), {}, FAKE, B.TQ_ERR_SHAPE),
    ({}, dict(head_dim=256, k_stride=2048, v_stride=2048), FAKE, B.TQ_ERR_SHAPE), ({}, dict(n_kv_heads=4), FAKE, B.TQ_ERR_SHAPE),
    ({}, dict(k_stride=0), FAKE, B.TQ_ERR_SHAPE), ({}, dict(n_tokens=0), FAKE, B.TQ_ERR_EMPTY), ({}, dict(dtype=3), FAKE, B.TQ_ERR_UNSUPPORTED),
    (dict(batch=1 << 20, capacity=2048), {}, FAKE, B.TQ_ERR_CAPACITY), (dict(v_codes=FAKE + 4), {}, FAKE, B.TQ_ERR_ALIGN),
    ({}, dict(k=FAKE + 8), FAKE, B.TQ_ERR_ALIGN), ({}, {}, FAKE + 2, B.TQ_ERR_ALIGN)])
def test_store_by_slots_refuses(cache, kw, slots, want):
    assert _store(None if cache is None else _cache(**cache), None if kw is None else _x(**kw), slots) == want


def _state(**kw):
    f = dict(seq_lens=FAKE, block_table=FAKE, free_pages=FAKE, n_free=FAKE, batch=4, max_blocks=8, n_pages=100, page_tokens=64)
    f.update(kw)
    return B.TqPageStateStruct(*[f[n] for n, _ in B.TqPageStateStruct._fields_])


PAGE_STATE = [
    (None, B.TQ_ERR_NULL), (dict(seq_lens=None), B.TQ_ERR_NULL), (dict(block_table=None), B.TQ_ERR_NULL),
    (dict(free_pages=None), B.TQ_ERR_NULL), (dict(n_free=None), B.TQ_ERR_NULL), (dict(batch=0), B.TQ_ERR_SHAPE),
    (dict(max_blocks=0), B.TQ_ERR_SHAPE), (dict(n_pages=0), B.TQ_ERR_SHAPE), (dict(page_tokens=0), B.TQ_ERR_SHAPE),
    (dict(n_pages=1 << 20, page_tokens=2048), B.TQ_ERR_CAPACITY), (dict(n_pages=2147483647, page_tokens=1), B.TQ_ERR_CAPACITY),
    (dict(batch=4097), B.TQ_ERR_UNSUPPORTED), (dict(block_table=FAKE + 2), B.TQ_ERR_ALIGN)]


@pytest.mark.parametrize("kw,want", PAGE_STATE)
def test_page_calls_refuse_a_bad_state(kw, want):
    st = None if kw is None else ctypes.byref(_state(**kw))
    assert B.raw().tq_pages_append(st, FAKE, 16, FAKE, FAKE, FAKE, FAKE, FAKE, None) == want
    assert B.raw().tq_pages_trim(st, FAKE, FAKE, FAKE, None) == want


def test_page_calls_refuse_bad_arguments():
    st = ctypes.byref(_state())
    for i in range(7):
        for bad, want in ((None, B.TQ_ERR_NULL), (FAKE + 2, B.TQ_ERR_ALIGN)):
            if i != 1:
                args = [FAKE, 16, FAKE, FAKE, FAKE, FAKE, FAKE]
                args[i] = bad
                assert B.raw().tq_pages_append(st, *args, None) == want
            if i < 3:
                args = [FAKE, FAKE, FAKE]
                args[i] = bad
                assert B.raw().tq_pages_trim(st, *args, None) == want
    for bound, want in ((0, B.TQ_ERR_EMPTY), (-3, B.TQ_ERR_EMPTY), (2147483647, B.TQ_ERR_CAPACITY)):
        assert B.raw().tq_pages_append(st, FAKE, bound, FAKE, FAKE, FAKE, FAKE, FAKE, None) == want


def test_the_binding_takes_gpu_tensors_only():
    q, k = torch.zeros((4, 8, 128), dtype=torch.float16), torch.zeros((4, 1, 128), dtype=torch.float16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        tq.tq_sdpa_prefill(q, k, k, i, 0.1)
    with pytest.raises(TypeError):
        tq.PageState(i, torch.zeros((2, 3), dtype=torch.int32), i, i[:1], 64)
    with pytest.raises(TypeError):
        tq.KVCache.wrap(*[torch.zeros((1, 1, 32, 64), dtype=torch.uint8)] * 6)
