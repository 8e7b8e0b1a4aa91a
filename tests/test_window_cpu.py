"""Windows with sinks, shared prefixes and slot maps, without a GPU: the test statement of what is seen against brute force,
and the refusals that come before any device call."""
import ctypes

import numpy as np
import pytest

import window_util as W
from paper_2602_02599_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding._lib()


@pytest.mark.parametrize("n_sink,window", [(0, 1), (0, 7), (1, 1), (4, 3), (4, 100), (9, 2)])
def test_what_a_query_sees(n_sink, window):
    for i in range(40):
        assert W.seen(i, n_sink, window) == [j for j in range(i + 1) if j < n_sink or j > i - window]


@pytest.mark.parametrize("n_sink,s_cap", [(0, 8), (1, 8), (4, 16), (7, 8), (4, 64)])
def test_rolling_rows_hold_the_newest_positions(n_sink, s_cap):
    rows = {}
    for p in range(60):
        rows[W.slot(p, n_sink, s_cap)] = p
        held = set(rows.values())
        assert held == set(range(min(n_sink, p + 1))) | set(range(max(n_sink, p + 1 - (s_cap - n_sink)), p + 1))
        if p < s_cap:
            assert W.slot(p, n_sink, s_cap) == p
    assert all(0 <= r < s_cap for r in rows)


def test_slot_maps_by_hand():
    start, seq, pos, at, after = W.slots([0, 5, 30], [2, 0, 3], [0, 0, 100], 2, 8)
    assert start.tolist() == [0, 2, 2, 5] and seq.tolist() == [0, 0, 2, 2, 2] and pos.tolist() == [0, 1, 130, 131, 132]
    assert at.tolist() == [0, 1, 2 + 28 % 6, 2 + 29 % 6, 2 + 30 % 6] and after.tolist() == [2, 5, 33]
    # nine tokens on six rolling rows: the first three are overwritten by later ones of the same call
    assert W.slots([2], [9], None, 2, 8)[3].tolist() == [-1, -1, -1, 5, 6, 7, 2, 3, 4]


def test_refusals_before_any_device_call(lib):
    E, A, H, C, S = binding.RAP_EINVAL, binding.RAP_EALIGN, binding.RAP_ESHAPE, binding.RAP_ECAPACITY, binding.RAP_ESTATE
    desc = binding.rap_model_desc(1, 64, 4, 2, 64, 10000.0, 0, 1, 3, 4)
    a = [1 << 20 | i << 12 for i in range(9)]          # addresses that no device ever sees
    import torch
    if torch.cuda.is_available():
        pytest.skip("with a device the checks behind these are tested on it")
    ctx = ctypes.c_void_p()
    assert lib.rap_create(ctypes.byref(desc), ctypes.byref(ctx)) == binding.RAP_ECUDA
    try:
        def build_slots(**kw):
            d = dict(B=3, past=a[0], new=a[1], base=None, T=5, n_sink=2, S_cap=16, start=a[2], seq=a[3], pos=a[4], slot=a[5], after=a[6])
            d.update(kw)
            return lib.rap_build_slots(ctx, d["B"], d["past"], d["new"], d["base"], d["T"], d["n_sink"], d["S_cap"], d["start"], d["seq"],
                                       d["pos"], d["slot"], d["after"], None)

        for name in ("past", "new", "start", "seq", "pos", "slot"):
            assert build_slots(**{name: None}) == E
            assert build_slots(**{name: a[8] + 4}) == A
        assert build_slots(base=a[8] + 8) == A and build_slots(after=a[8] + 4) == A
        assert build_slots(B=-1) == E and build_slots(T=-1) == E and build_slots(n_sink=-1) == E and build_slots(n_sink=16) == E
        assert build_slots(S_cap=0) == E and build_slots(S_cap=12) == A and build_slots(B=4) == H
        assert build_slots(seq=a[4]) == E and build_slots(start=a[0]) == E and build_slots(slot=a[3] + 16) == E
        assert build_slots(after=a[1]) == E and build_slots(after=a[2]) == E and build_slots(base=a[6]) == E
        # nothing to refuse but the missing device
        assert build_slots() not in (E, A, H, C) and build_slots(after=a[0]) not in (E, A, H, C) and build_slots(after=None) not in (E, A, H, C)
        # the attention calls want tables first, and pointers before that
        assert lib.rap_decode_attn_window(ctx, 0, 1, a[0], a[1], a[2], 16, a[3], 8, 2, 4, a[4], None) == S
        assert lib.rap_decode_attn_window(ctx, 0, 1, None, a[1], a[2], 16, a[3], 8, 2, 4, a[4], None) == E
        assert lib.rap_prefill_attn_window(ctx, 0, 1, 4, a[0], a[1], a[2], 16, a[3], a[4], 4, 8, 2, 4, a[5], None) == S
        assert lib.rap_prefill_attn_window(ctx, 0, 1, 4, a[0], a[1], a[2], 16, None, a[4], 4, 8, 2, 4, a[5], None) == E
        assert lib.rap_decode_attn_shared(ctx, 0, 1, a[0], 1, a[1], a[2], 16, a[3], a[4], 8, a[5], a[6], 16, a[7], 8, a[8], None) == S
        assert lib.rap_decode_attn_shared(ctx, 0, 1, a[0], 1, a[1], a[2], 16, a[3], None, 8, a[5], a[6], 16, a[7], 8, a[8], None) == E
    finally:
        lib.rap_destroy(ctx)


def blocks(rows):
    return [max(1, (n + 31) // 32) for n in rows]


# (KV heads, visible rows, partials of a prefix, rows of K and V both of a multiple of 16 bytes)
LONG_UNITS = [(2, [16384, 4096], 0, False), (2, [16384, 4096], 0, True), (4, [16860, 999, 364], 0, False), (4, [3230, 14656], 0, False),
              (2, [8224], 0, True), (4, [8224], 0, True), (2, [8704], 0, True), (4, [9120], 0, True), (4, [248, 5744], 20, False),
              (2, [128, 6976, 96, 448, 3264, 9152], 0, False), (2, [96, 160, 7328, 3904, 96, 7360], 10, False), (4, [1696, 9504], 0, False)]


@pytest.mark.parametrize("kv,rows,n_pre,padded", LONG_UNITS)
def test_every_partial_has_a_place(lib, kv, rows, n_pre, padded):
    most, places = binding.rap_debug_window_plan(148, kv, blocks(rows), n_pre, padded)
    assert 1 <= most <= places == 64 - n_pre


def test_every_partial_has_a_place_in_random_batches(lib):
    """Batches of every kind: alike, spread over the logarithm, a long sequence among short ones at either end."""
    r = np.random.RandomState(11)
    for i in range(30000):
        kv, B = r.randint(1, 17), int(np.exp(r.uniform(0, np.log(60))))
        most_rows = np.exp(r.uniform(0, np.log(65536)))
        rows = np.exp(r.uniform(0, np.log(most_rows + 1), B)).astype(int) if i % 3 else np.full(B, int(most_rows)) - r.randint(0, 40, B)
        if i % 3 == 2:
            rows[r.choice([0, B - 1])] = int(np.exp(r.uniform(np.log(2000), np.log(65536))))
        n_pre = r.choice([0, 0, r.randint(1, 41)])
        most, places = binding.rap_debug_window_plan(r.choice([148, 148, 132, 7]), kv, blocks(np.maximum(rows, 0)), n_pre, i % 2)
        assert 1 <= most <= places, (kv, rows.tolist(), n_pre, i % 2)
    for bad in ([], [0], [2 ** 27]):
        with pytest.raises(binding.RapError):
            binding.rap_debug_window_plan(148, 8, bad)
    with pytest.raises(binding.RapError):
        binding.rap_debug_window_plan(148, 8, [4], n_pre=41)
