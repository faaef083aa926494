"""From a prompt to a paged cache on the GPU: attention of packed prompts, their K and V by slots, pages given and taken back,
each against its reference in plain Python or 64 bits, and the four of them together in front of decode steps."""
import ctypes
import math
import random

import numpy as np
import pytest
import torch

import paper_2604_16957_amd as tq
from paper_2604_16957_amd import binding as B
from prompt_common import append, attend, quantize, trim

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _qkv(T, hq, hkv, d, dtype, seed, fused=False, std=1.0):
    gen = torch.Generator().manual_seed(seed)
    row = (torch.randn((T, hq + 2 * hkv, d), generator=gen) * std).to(dtype).cuda()
    q, k, v = row[:, :hq], row[:, hq:hq + hkv], row[:, hq + hkv:]
    return (q, k, v) if fused else (q.contiguous(), k.contiguous(), v.contiguous())


def _cu(lens, first=0):
    return [first + sum(lens[:i]) for i in range(len(lens) + 1)]


def _check_attend(q, k, v, cu, scale, window=0, out=None):
    got = tq.tq_sdpa_prefill(q, k, v, _i32(cu), scale, window=window, out=out)
    want, tol = attend(q, k, v, cu, scale, window)
    err = (got[cu[0]:cu[-1]].double().cpu() - want[cu[0]:cu[-1]]).abs()
    assert torch.isfinite(err).all()
    worst = (err / tol[cu[0]:cu[-1]].clamp(min=1e-30)).max().item() if err.numel() else 0.0
    assert worst <= 1.0, f"error {worst:.2f} of what it may be"
    return got


# ---- attention of prompts ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("hq,hkv,d", [(8, 1, 128), (64, 8, 128), (4, 4, 128), (6, 2, 128), (14, 2, 128), (16, 1, 128), (40, 1, 128), (8, 4, 256),
                                      (8, 1, 256), (3, 3, 256), (32, 1, 512), (4, 2, 512), (3, 1, 512)])
def test_packed_prompts(hq, hkv, d, dtype):
    lens = [1, 0, 33, 130, 2, 0, 0, 64, 31, 200, 0]
    q, k, v = _qkv(sum(lens), hq, hkv, d, dtype, 11 * hq + d, fused=True)
    _check_attend(q, k, v, _cu(lens), 1.0 / math.sqrt(d))


@pytest.mark.parametrize("d,hq,hkv", [(128, 8, 2), (256, 4, 2), (512, 4, 1)])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 515])
def test_every_length_around_a_tile(n, d, hq, hkv):
    q, k, v = _qkv(n, hq, hkv, d, F16, n)
    _check_attend(q, k, v, [0, n], 1.0 / math.sqrt(d))


@pytest.mark.parametrize("window", [1, 2, 31, 64, 65, 100, 128, 1000, 2 ** 31 - 1])
@pytest.mark.parametrize("d,hq,hkv", [(128, 8, 2), (256, 4, 2), (512, 4, 1)])
def test_window(window, d, hq, hkv):
    lens = [300, 1, 70, 129]
    q, k, v = _qkv(sum(lens), hq, hkv, d, F16, window % 1000 + d)
    _check_attend(q, k, v, _cu(lens), 1.0 / math.sqrt(d), window)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("scale", [0.0, -0.09, 1.0, 1e-42, 3.0])
def test_scales_of_any_sign_and_size(scale, dtype):
    q, k, v = _qkv(150, 8, 2, 128, dtype, 5)
    _check_attend(q, k, v, [0, 90, 150], scale)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("d", [128, 256, 512])
def test_sharp_and_growing_scores(d, dtype):
    """Scores that rise with the key (every tile has a new maximum), fall with it, jump, or lie far below zero: weights of very
    different sizes, in heads that see the same keys at different scales and signs side by side."""
    n = 400
    q, k, v = _qkv(n, 4, 1, d, dtype, 21)
    q[:] = 0
    q[:, :, 0] = torch.tensor([1.0, 0.03125, -1.0, 0.5], dtype=dtype).cuda()
    for shape in (torch.arange(n) * 0.75, -torch.arange(n) * 0.75, torch.where(torch.arange(n) % 97 == 50, 60.0, 0.0), torch.full((n,), -300.0)):
        k[:] = 0
        k[:, 0, 0] = shape.to(dtype).cuda()
        _check_attend(q, k, v, [0, n], 1.0)
        _check_attend(q, k, v, [0, 7, n], 1.0, window=150)


@pytest.mark.parametrize("seed", range(12))
def test_drawn_shapes(seed):
    rng = random.Random(100 + seed)
    d = rng.choice([128, 128, 256, 512])
    hkv = rng.choice([1, 2, 3])
    hq = hkv * rng.choice([1, 2, 3, 5, 8, 12])
    lens = [rng.choice([0, 1, rng.randint(2, 40), rng.randint(40, 700)]) for _ in range(rng.randint(1, 9))] + [5]
    window = rng.choice([0, 0, 1, rng.randint(2, 300)])
    dtype = rng.choice([F16, BF16])
    q, k, v = _qkv(sum(lens), hq, hkv, d, dtype, seed, fused=rng.random() < 0.5)
    _check_attend(q, k, v, _cu(lens), rng.choice([1.0, 1.0 / math.sqrt(d), -0.05]), window)


@pytest.mark.parametrize("hq,hkv,d", [(129, 1, 128), (1001, 1, 128), (262, 2, 128), (300, 1, 256), (70, 1, 512)])
def test_more_heads_to_a_group_than_rows_to_a_block(hq, hkv, d):
    lens = [3, 1, 0, 38]
    q, k, v = _qkv(sum(lens), hq, hkv, d, F16, hq, fused=True)
    _check_attend(q, k, v, _cu(lens), 1.0 / math.sqrt(d))


def test_two_calls_at_once():
    """Different prompts on two streams, issued in turn and running side by side: no state is shared."""
    sets = [(_qkv(900, 16, 2, 128, F16, 31), [0, 400, 900]), (_qkv(700, 4, 1, 512, BF16, 32), [0, 1, 700]), (_qkv(800, 8, 4, 256, F16, 33), [0, 800])]
    cus = [_i32(cu) for _, cu in sets]
    want = [tq.tq_sdpa_prefill(*x, cu, 0.1) for (x, _), cu in zip(sets, cus)]
    outs = [[torch.zeros_like(w) for _ in range(4)] for w in want]
    streams = [torch.cuda.Stream() for _ in sets]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for i in range(4):
        for (x, _), cu, s, o in zip(sets, cus, streams, outs):
            tq.tq_sdpa_prefill(*x, cu, 0.1, out=o[i], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for w, several in zip(want, outs) for o in several)


def test_a_longer_prompt():
    q, k, v = _qkv(2311, 16, 2, 128, BF16, 8)
    _check_attend(q, k, v, [0, 2311], 1.0 / math.sqrt(128))


def test_many_short_sequences():
    rng = random.Random(4)
    lens = [rng.choice([0, 1, 1, 2, 3, 5, 8, 40]) for _ in range(700)]
    q, k, v = _qkv(sum(lens), 8, 1, 128, F16, 9)
    _check_attend(q, k, v, _cu(lens), 0.1)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("window", [0, 40])
def test_wide_blocks_at_head_dim_256(window, dtype):
    """Enough rows for blocks of eight waves; and with fewer tokens of the same shape the other instance."""
    rng = random.Random(5)
    lens = [rng.choice([1, 31, 64, 65, 130, 200]) for _ in range(40)]
    lens.append(max(0, 3300 - sum(lens)))
    q, k, v = _qkv(sum(lens), 32, 4, 256, dtype, 17)

    def rows(T):
        x = B.TqPackedStruct(q.data_ptr(), k.data_ptr(), v.data_ptr(), 32 * 256, 4 * 256, 4 * 256, T, 32, 4, 256, 0)
        return B.raw().tq_internal_prefill_rows(ctypes.byref(x))

    assert rows(sum(lens)) == 256 and rows(2000) == 128
    _check_attend(q, k, v, _cu(lens), 1.0 / 16, window)


def test_rows_of_no_sequence_are_left_as_they_were():
    q, k, v = _qkv(400, 8, 2, 128, F16, 3)
    for x in (q, k, v):                                   # what lies outside of the sequences may be anything
        x[:50] = float("nan")
        x[301:] = float("inf")
    out = torch.full_like(q, 7.0)
    _check_attend(q, k, v, [50, 120, 120, 301], 0.1, out=out)
    assert (out[:50] == 7.0).all() and (out[301:] == 7.0).all()


def test_a_neighbours_infinities_stay_with_it():
    q, k, v = _qkv(300, 8, 2, 128, F16, 6)
    want = tq.tq_sdpa_prefill(q, k, v, _i32([0, 77, 200, 300]), 0.1)
    for x in (q, k, v):
        x[77:200] = float("nan")
    got = tq.tq_sdpa_prefill(q, k, v, _i32([0, 77, 200, 300]), 0.1)
    assert torch.equal(got[:77], want[:77]) and torch.equal(got[200:], want[200:])


@pytest.mark.parametrize("cu", [[0, -5, 500, 90], [70, 10, 10, 60], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 100], [5, 5, 5, 5]])
def test_lengths_that_make_no_sense_stay_inside(cu):
    """Not ascending, or outside of the tokens: undefined rows of out, no access outside of the arrays (the guard rows show the writes)."""
    T = 100
    q, k, v = _qkv(T, 8, 2, 128, F16, 2)
    big = torch.full((T + 256, 8, 128), 3.0, dtype=F16, device="cuda")
    tq.tq_sdpa_prefill(q, k, v, _i32(cu), 0.1, out=big[128:128 + T])
    assert (big[:128] == 3.0).all() and (big[128 + T:] == 3.0).all()


def test_same_bits_every_time_and_on_another_stream():
    lens = [500, 3, 260]
    q, k, v = _qkv(sum(lens), 64, 8, 128, F16, 14, fused=True)
    cu = _i32(_cu(lens))
    want = tq.tq_sdpa_prefill(q, k, v, cu, 0.09)
    side = torch.cuda.Stream()
    theirs = [torch.zeros_like(want) for _ in range(3)]
    side.wait_stream(torch.cuda.current_stream())
    outs = [tq.tq_sdpa_prefill(q, k, v, cu, 0.09) for _ in range(3)]
    outs += [tq.tq_sdpa_prefill(q, k, v, cu, 0.09, out=o, stream=side) for o in theirs]
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_a_row_far_into_memory():
    """Rows past 2^31 bytes and elements: a stride near the largest, read at 64-bit offsets."""
    stride, T = (1 << 24) - 8, 200
    flat = torch.zeros(stride * (T - 1) + 2 * 128 * 8, dtype=F16, device="cuda")
    q = flat.as_strided((T, 8, 128), (stride, 128, 1))
    q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(1)).to(F16).cuda())
    k, v = q[:, :2], q[:, 2:4]
    _check_attend(q, k, v, [0, 150, 200], 0.1)


# ---- packed K and V by slots --------------------------------------------------------------------------------------

def _same_cache(cache, slots, k, v, group, before=0xEE):
    """Every stored row holds the reference's bits, every other byte is as it was."""
    page = cache.capacity
    for x, (codes, scale, zero) in ((k, (cache.k_codes, cache.k_scale, cache.k_zero)), (v, (cache.v_codes, cache.v_scale, cache.v_zero))):
        for got, want in zip((codes, scale, zero), quantize(x, group)):
            expected = torch.empty_like(got, device="cpu")
            expected.view(torch.uint8).fill_(before)
            for i, s in enumerate(slots):
                if 0 <= s < cache.batch * page:
                    expected[s // page, :, s % page] = torch.from_numpy(want[i])
            assert torch.equal(got.cpu().view(torch.uint8), expected.view(torch.uint8))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("hkv,d,group,page", [(8, 128, 32, 64), (1, 128, 64, 32), (3, 128, 128, 100), (4, 256, 32, 64), (2, 256, 64, 1), (2, 256, 128, 48),
                                              (1, 512, 32, 32), (2, 512, 128, 64)])
def test_store_by_slots(hkv, d, group, page, dtype):
    T, pages = 133, 300 if page == 1 else 9
    _, k, v = _qkv(T, 1, hkv, d, dtype, d + page, fused=True)
    k[5] = 0.0                                            # a constant group, a tiny one, one with an offset
    k[6] = 2.0 ** -23
    v[7] += 1000.0
    rng = random.Random(page)
    slots = rng.sample(range(pages * page), T)
    for i, s in ((0, -1), (9, -2 ** 31), (10, pages * page), (11, 2 ** 31 - 1)):
        slots[i] = s
    cache = tq.KVCache(pages, hkv, d, page, group_size=group)
    for t in cache.tensors():
        t.view(torch.uint8).fill_(0xEE)
    tq.tq_quantize_kv_slots(cache, k, v, _i32(slots))
    _same_cache(cache, slots, k, v, group)


def test_store_by_slots_of_bf16_outside_of_fp16s_range():
    k = torch.randn((20, 2, 128), generator=torch.Generator().manual_seed(3)).cuda()
    k[0] *= 1e30
    k[1] *= 3e5
    k[2] *= 1e-30
    k[3] = 3e38
    k[4] = k[4].abs() + 1e6
    k[5, :, ::2], k[5, :, 1::2] = 3.3e38, -3.3e38
    k = k.to(BF16)
    v = k.flip(0).contiguous()
    cache = tq.KVCache(1, 2, 128, 20)
    slots = list(range(19, -1, -1))
    tq.tq_quantize_kv_slots(cache, k, v, _i32(slots))
    _same_cache(cache, slots, k, v, 32)


def test_store_by_slots_is_the_append_of_a_contiguous_cache():
    B, hkv, n, d = 3, 4, 57, 128
    k = torch.randn((B, hkv, n, d), generator=torch.Generator().manual_seed(5)).to(F16).cuda()
    v = torch.randn((B, hkv, n, d), generator=torch.Generator().manual_seed(6)).to(F16).cuda()
    a, b = tq.KVCache(B, hkv, d, 80), tq.KVCache(B, hkv, d, 80)
    for c in (a, b):
        for t in c.tensors():
            t.zero_()
    tq.tq_quantize_kv(a, k, v, 11)
    packed = [x.permute(0, 2, 1, 3).reshape(B * n, hkv, d).contiguous() for x in (k, v)]
    tq.tq_quantize_kv_slots(b, *packed, _i32([s * 80 + 11 + i for s in range(B) for i in range(n)]))
    assert all(torch.equal(x, y) for x, y in zip(a.tensors(), b.tensors()))


def test_one_token_and_a_token_per_block_edge():
    for T in (1, 7, 8, 9, 63, 64, 65):
        _, k, v = _qkv(T, 1, 2, 128, F16, T)
        cache = tq.KVCache(2, 2, 128, 64)
        for t in cache.tensors():
            t.view(torch.uint8).fill_(0xEE)
        slots = [127 - i for i in range(T)]
        tq.tq_quantize_kv_slots(cache, k, v, _i32(slots))
        _same_cache(cache, slots, k, v, 32)


# ---- pages ------------------------------------------------------------------------------------------------------

def _random_state(rng, batch, max_blocks, page, spare, longest=None):
    room = max_blocks * page
    lens = [rng.choice([0, 0, page, room, rng.randint(0, min(longest or room, room))]) for _ in range(batch)]
    blocks = [-(-n // page) for n in lens]
    order = list(range(sum(blocks) + spare))
    rng.shuffle(order)
    table, at = [], 0
    for n in blocks:
        table.append(order[at:at + n] + [-7] * (max_blocks - n))
        at += n
    free = order[at:] + [-9] * at
    return lens, table, free, spare


def _state(lens, table, free, n_free, page):
    return tq.PageState(_i32(lens), _i32(table), _i32(free), _i32([n_free]), page)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("batch,max_blocks,page,spare,bound", [(1, 4, 32, 2, 64), (7, 5, 64, 3, 300), (64, 6, 32, 20, 1000), (65, 3, 1, 10, 50),
                                                               (300, 4, 100, 400, 5000), (257, 8, 64, 700, 60000), (1100, 2, 32, 900, 9000),
                                                               (4096, 2, 32, 3000, 4100), (33, 40, 16, 0, 2000)])
def test_pages_append(batch, max_blocks, page, spare, bound, in_place):
    for seed in range(3):
        rng = random.Random(seed * 1000 + batch)
        lens, table, free, n_free = _random_state(rng, batch, max_blocks, page, spare)
        new = [rng.choice([0, 1, 1, -3, page, rng.randint(0, 2 * bound // batch + 2)]) for _ in range(batch)]
        want = append(lens, table, free, n_free, new, page, bound)
        st = _state(lens, table, free, n_free, page)
        after = {} if in_place else dict(seq_lens_after=torch.full_like(st.seq_lens, -5), n_free_after=torch.full_like(st.n_free, -5))
        cu, slots, served = tq.tq_pages_append(st, _i32(new), bound, **after)
        got = dict(cu_seqlens=cu, slots=slots, served=served, block_table=st.block_table,
                   seq_lens=after.get("seq_lens_after", st.seq_lens), n_free=after.get("n_free_after", st.n_free))
        for name, t in got.items():
            assert torch.equal(t.cpu(), torch.tensor(want[name], dtype=torch.int32).reshape(t.shape)), (seed, name)
        assert st.free_pages.tolist() == free
        if not in_place:
            assert st.seq_lens.tolist() == lens and st.n_free.tolist() == [n_free]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("batch,max_blocks,page,spare", [(1, 4, 32, 2), (7, 5, 64, 0), (64, 6, 32, 20), (300, 70, 16, 5), (4096, 5, 32, 1)])
def test_pages_trim(batch, max_blocks, page, spare, in_place):
    for seed in range(3):
        rng = random.Random(seed * 1000 + batch)
        lens, table, free, n_free = _random_state(rng, batch, max_blocks, page, spare)
        keep = [rng.choice([0, -1, n, n + 5, max(0, n - 1), max(0, n - page), rng.randint(0, n)]) for n in lens]
        want = trim(lens, table, free, n_free, keep, page)
        st = _state(lens, table, free, n_free, page)
        after = {} if in_place else dict(seq_lens_after=torch.full_like(st.seq_lens, -5), n_free_after=torch.full_like(st.n_free, -5))
        tq.tq_pages_trim(st, _i32(keep), **after)
        assert after.get("seq_lens_after", st.seq_lens).tolist() == want["seq_lens"]
        assert after.get("n_free_after", st.n_free).tolist() == [want["n_free"]]
        assert st.free_pages.tolist() == want["free_pages"]
        assert st.block_table.tolist() == table


def test_a_state_that_makes_no_sense_stays_inside():
    """Counts and lengths outside of what the arrays hold: clamped, or the sequence is not served; no slot outside of the pool."""
    page, big = 32, 2 ** 31 - 1
    lens, table = [big, -big - 1, 200, 10], [[0, 1], [2, 3], [4, 5], [big, -4]]
    for n_free in (-5, 9, big):
        free = [3, 7, -1, 6, 99]
        new = [big, big, 1, 1]
        st = _state(lens, table, free, n_free, page)
        want = append(lens, table, free, n_free, new, page, 128)
        cu, slots, served = tq.tq_pages_append(st, _i32(new), 128)
        assert (cu.tolist(), slots.tolist(), served.tolist()) == (want["cu_seqlens"], want["slots"], want["served"])
        st = _state(lens, table, free, n_free, page)
        keep = [5, 0, -1, big]
        want = trim(lens, table, free, n_free, keep, page)
        tq.tq_pages_trim(st, _i32(keep))
        assert st.free_pages.tolist() == want["free_pages"] and st.seq_lens.tolist() == want["seq_lens"]
        assert st.n_free.tolist() == [want["n_free"]]


def test_pages_are_never_lost_or_held_twice():
    rng = random.Random(2)
    batch, page, n_pages = 37, 32, 400
    st = tq.PageState.empty(batch, 30, n_pages, page)
    for step in range(40):
        tq.tq_pages_append(st, _i32([rng.choice([0, 1, 1, 1, rng.randint(1, 300)]) for _ in range(batch)]), 20000)
        keep = [rng.choice([n, n, n, max(0, n - rng.randint(0, 7)), 0]) for n in st.seq_lens.tolist()]
        tq.tq_pages_trim(st, _i32(keep))
        lens, table = st.seq_lens.tolist(), st.block_table.tolist()
        pages = [p for b in range(batch) for p in table[b][:-(-lens[b] // page)]] + st.free_pages.tolist()[:st.n_free.item()]
        assert sorted(pages) == list(range(n_pages)), f"step {step}"


# ---- together ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("hq,hkv,d", [(16, 2, 128), (8, 4, 256)])
def test_prompts_then_decode_steps(hq, hkv, d):
    """A server's life in small: prompts come in (attended, stored), every sequence decodes, one ends, another takes its row; each decode
    step against softmax over the tokens that the sequence has seen, dequantised."""
    page, batch, n_pages = 32, 4, 40
    scale = 1.0 / math.sqrt(d)
    st = tq.PageState.empty(batch, 12, n_pages, page)
    pool = tq.KVCache(n_pages, hkv, d, page)
    for t in pool.tensors():
        t.zero_()
    seen = [([], []) for _ in range(batch)]               # dequantised K and V of every sequence, token by token
    gen = torch.Generator().manual_seed(d)

    def remember(b, k, v):
        for kept, x in zip(seen[b], (k, v)):
            codes, s, z = quantize(x, 32)
            c = np.stack([codes & 15, codes >> 4], -1).reshape(x.shape).astype(np.float64)
            kept.append((c - np.repeat(z.astype(np.float64), 32, -1)) * np.repeat(s.astype(np.float64), 32, -1))

    def prompts(new):
        cu, slots, served = tq.tq_pages_append(st, _i32(new), 512)
        assert served.tolist() == [1] * batch
        qkv = torch.randn((512, hq + 2 * hkv, d), generator=gen).to(F16).cuda()
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        out = tq.tq_sdpa_prefill(q, k, v, cu, scale)
        tq.tq_quantize_kv_slots(pool, k, v, slots)
        ends = cu.tolist()
        want, tol = attend(q, k, v, ends, scale)
        assert ((out[:ends[-1]].double().cpu() - want[:ends[-1]]).abs() <= tol[:ends[-1]]).all()
        for b in range(batch):
            if ends[b + 1] > ends[b]:
                remember(b, k[ends[b]:ends[b + 1]], v[ends[b]:ends[b + 1]])

    def decode():
        tq.tq_pages_append(st, _i32([1] * batch), 128)
        qkv = torch.randn((batch, hq + 2 * hkv, d), generator=gen).to(F16).cuda()
        q, k, v = (x.contiguous() for x in (qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]))
        out = tq.tq_sdpa_int4_append_decode_paged(pool, st.block_table, k.unsqueeze(2), v.unsqueeze(2), q, st.seq_lens, 12 * page, scale)
        for b in range(batch):
            remember(b, k[b:b + 1], v[b:b + 1])
            kd, vd = (torch.from_numpy(np.concatenate(x)) for x in seen[b])
            assert st.seq_lens[b].item() == kd.shape[0]
            g = hq // hkv
            for h in range(hq):
                w = torch.softmax(kd[:, h // g] @ q[b, h].double().cpu() * scale, 0)
                assert (out[b, h].double().cpu() - w @ vd[:, h // g]).abs().max() <= 2e-3

    prompts([70, 1, 129, 33])
    for _ in range(3):
        decode()
    lens = st.seq_lens.tolist()
    tq.tq_pages_trim(st, _i32([lens[0], lens[1], 0, lens[3] - 2]))
    seen[2] = ([], [])
    for x in seen[3]:
        x[:] = [np.concatenate(x)[:-2]]
    prompts([0, 0, 45, 0])
    for _ in range(2):
        decode()


def test_captured_step_with_pages_in_place():
    """A graph of page bookkeeping, prompt attention and store, replayed with new lengths in its buffers between eager work."""
    batch, page, bound, hq, hkv, d = 5, 32, 640, 8, 2, 128
    q, k, v = _qkv(bound, hq, hkv, d, F16, 77, fused=True)
    new = torch.zeros(batch, dtype=torch.int32, device="cuda")
    bufs = dict(cu_seqlens=torch.zeros(batch + 1, dtype=torch.int32, device="cuda"), slots=torch.zeros(bound, dtype=torch.int32, device="cuda"),
                served=torch.zeros(batch, dtype=torch.int32, device="cuda"))
    states = [tq.PageState.empty(batch, 40, 120, page) for _ in range(2)]
    pools = [tq.KVCache(120, hkv, d, page) for _ in range(2)]
    for pool in pools:
        for t in pool.tensors():
            t.zero_()
    outs = [torch.zeros((bound, hq, d), dtype=F16, device="cuda") for _ in range(2)]

    def step(i):
        tq.tq_pages_append(states[i], new, bound, **bufs)
        tq.tq_sdpa_prefill(q, k, v, bufs["cu_seqlens"], 0.1, out=outs[i])
        tq.tq_quantize_kv_slots(pools[i], k, v, bufs["slots"])

    step(0)                                               # (nothing asked for: the state stays as it is)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    for lens in ([3, 0, 100, 1, 40], [1, 1, 1, 1, 1], [200, 33, 0, 1, 128], [0, 0, 0, 0, 0], [1, 500, 2, 64, 7]):
        new.copy_(_i32(lens))
        graph.replay()
        torch.cuda.synchronize()
        step(1)
        torch.cuda.synchronize()
        for a, b in ((states[0].seq_lens, states[1].seq_lens), (states[0].block_table, states[1].block_table), (states[0].n_free, states[1].n_free),
                     (outs[0], outs[1]), *zip(pools[0].tensors(), pools[1].tensors())):
            assert torch.equal(a, b)


# ---- what the binding refuses -------------------------------------------------------------------------------------

def test_the_binding_refuses_what_the_kernels_would_misread():
    q, k, v = _qkv(10, 8, 2, 128, F16, 1)
    cu = _i32([0, 10])
    for bad in (q.float(), q.to(BF16)):
        with pytest.raises(TypeError):
            tq.tq_sdpa_prefill(bad, k, v, cu, 0.1)
    for args in ((q, k, v[:9], cu), (q, k[:9], v[:9], cu), (q, k.transpose(0, 1), v, cu), (q[..., ::2], k, v, cu), (q, k, v, cu.long())):
        with pytest.raises((ValueError, TypeError)):
            tq.tq_sdpa_prefill(*args, 0.1)
    with pytest.raises(ValueError):
        tq.tq_sdpa_prefill(q, k, v, cu, 0.1, out=torch.empty_like(k))
    with pytest.raises(tq.TqError):
        tq.tq_sdpa_prefill(q, k, v, cu, 0.1, window=-1)
    with pytest.raises(tq.TqError):                        # a broadcast row has no stride
        tq.tq_sdpa_prefill(q, k[:1].expand(10, 2, 128), v, cu, 0.1)
    cache = tq.KVCache(2, 2, 128, 32)
    with pytest.raises(ValueError):
        tq.tq_quantize_kv_slots(cache, k, v, _i32([0] * 9))
    with pytest.raises(tq.TqError):
        tq.tq_quantize_kv_slots(cache, q, q, _i32(list(range(10))))
    st = tq.PageState.empty(3, 4, 10, 32)
    with pytest.raises(ValueError):
        tq.tq_pages_append(st, _i32([1, 1]), 10)
    with pytest.raises(tq.TqError):
        tq.tq_pages_append(st, _i32([1, 1, 1]), 0)
    with pytest.raises(ValueError):
        tq.tq_pages_trim(st, _i32([1, 1, 1]), seq_lens_after=_i32([0, 0]))
