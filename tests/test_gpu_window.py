"""Attention with a window and sinks (one token, ragged blocks), over shared prefixes, and slot maps, on the GPU against plain
64-bit statements of them (window_util).  Caches hold NaN wherever nothing is seen."""
import math

import numpy as np
import pytest
import torch

import window_util as W
from paper_2602_02599_b200 import binding

pytestmark = pytest.mark.gpu

SHAPES = [(45, 90, 4), (58, 115, 3), (51, 102, 1), (32, 64, 8), (64, 128, 4), (64, 128, 5), (45, 90, 5), (1, 1, 2), (3, 5, 7), (8, 16, 4), (9, 17, 6),
          (16, 33, 2), (20, 128, 4), (64, 16, 3), (22, 45, 8), (37, 73, 1), (48, 96, 2), (63, 127, 6)]


def decode(H, lens, n_sink, window, s_cap, stream=None):
    """Random caches of the lengths, the call, and the reference."""
    B = len(lens)
    K, V = H.caches(B, s_cap)
    rows = [[W.slot(p, n_sink, s_cap) for p in W.seen(n - 1, n_sink, window)] if n else [] for n in lens]
    for b, r in enumerate(rows):
        H.fill(K, b, r)
        H.fill(V, b, r)
    q, out = H.query(B), H.out(B)
    H.ctx.rap_decode_attn_window(0, B, q, K, V, s_cap, H.ints(lens), max(lens), n_sink, window, out)
    want = [H.reference(q[b], [(K, V, b, rows[b])]) for b in range(B)]
    return out, torch.stack([w[0] for w in want]), torch.stack([w[1] for w in want])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_sink,window,s_cap", [(4, 100, 128), (0, 64, 64), (4, 60, 64), (17, 300, 512), (1, 1, 8), (130, 33, 200), (0, 1000, 1000), (3, 2 ** 31 - 1, 1504)])
def test_decode_lengths_at_every_border(n_sink, window, s_cap, dtype):
    H = W.Heads(2, 4, 45, 90, dtype, 24)
    rolling = window <= s_cap - n_sink
    near = {0, 1, 2, 7, 8, 9, 31, 32, 33, n_sink, n_sink + 1, s_cap - 1, s_cap}
    if window < 10 ** 6:
        near |= {window - 1, window, window + 1, n_sink + window, n_sink + window + 1, n_sink + window + 9}
    if rolling:
        near |= {s_cap + 1, s_cap + 5, 2 * s_cap + 3, 2 * s_cap - n_sink, 7 * s_cap + 11, 2 ** 31 - 1}
    lens = sorted(n for n in near if 0 <= n and (rolling or n <= s_cap))
    lens = lens[::2] + lens[1::2]
    if window < 10 ** 6:
        got, want, bound = decode(H, lens[:24], n_sink, window, s_cap)
    else:                                             # a window beyond every length is plain attention
        got, want, bound = decode(H, lens[:24], n_sink, s_cap, s_cap)
        again = H.out(len(lens))
        H.g.manual_seed(5)
        K, V, q = H.randn(len(lens), 2, s_cap, 90), H.randn(len(lens), 2, s_cap, 90), H.query(len(lens))
        H.ctx.rap_decode_attn_window(0, len(lens), q, K, V, s_cap, H.ints(lens), max(lens), n_sink, window, again)
        ref = [H.reference(q[b], [(K, V, b, range(n))]) for b, n in enumerate(lens)]
        W.check(again, torch.stack([r[0] for r in ref]), torch.stack([r[1] for r in ref]))
    W.check(got, want, bound)
    if 0 in lens:
        assert (got[lens.index(0)] == 0).all()
    H.clean()
    H.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs,vch,group", SHAPES)
def test_decode_head_shapes(pairs, vch, group, dtype):
    H = W.Heads(3, group, pairs, vch, dtype, 5)
    W.check(*decode(H, [333, 1, 0, 130, 2000], 5, 200, 400))
    W.check(*decode(H, [333, 1, 0, 130, 399], 0, 333, 400))
    H.clean()
    H.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_wide_heads(dtype):
    H = W.Heads(1, 3, 128, 256, dtype, 3, head_dim=256)
    W.check(*decode(H, [70, 0, 555], 2, 65, 72))
    H.close()


@pytest.mark.parametrize("B,kv,lens", [(1, 1, 5000), (1, 8, 4500), (200, 1, 300), (70, 8, 260), (3, 2, 9000)])
def test_decode_batches(B, kv, lens):
    """From one unit that all SMs share to hundreds of short ones."""
    H = W.Heads(kv, 4, 45, 90, "bf16", B)
    lens = [max(0, lens - 37 * b) for b in range(B)]
    W.check(*decode(H, lens, 4, 4096, 4112))
    W.check(*decode(H, lens[::-1], 0, 100, 9000 // 8 * 8 + 8))
    H.clean()
    H.close()


def prefill(H, past, new, n_sink, window, s_cap, pad=0):
    B, T = len(new), sum(new) + pad
    K, V = H.caches(B, s_cap)
    lens = [p + n for p, n in zip(past, new)]
    rows = [[[W.slot(p, n_sink, s_cap) for p in W.seen(i, n_sink, window)] for i in range(past[b], lens[b])] for b in range(B)]
    for b in range(B):
        every = {r for i in rows[b] for r in i}
        H.fill(K, b, every)
        H.fill(V, b, every)
    start = [0] + list(np.cumsum(new))
    q, out = H.query(T), H.out(T, fill=7.25)
    H.ctx.rap_prefill_attn_window(0, B, T, q, K, V, s_cap, H.ints(start), H.ints(lens), max(new), max(lens), n_sink, window, out)
    assert (out[start[-1]:] == 7.25).all()             # rows behind the last sequence
    want, bound = [], []
    for b in range(B):
        # queries that see the same number of rows at a time
        some = range(new[b]) if new[b] <= 80 else sorted(set(list(range(0, 40)) + list(range(new[b] // 2 - 20, new[b] // 2 + 20)) + list(range(new[b] - 40, new[b]))))
        for i in some:
            o, e = H.reference(q[start[b] + i], [(K, V, b, rows[b][i])])
            want.append((start[b] + i, o, e))
    if want:
        at = torch.tensor([w[0] for w in want], device=H.device)
        W.check(out[at], torch.stack([w[1] for w in want]), torch.stack([w[2] for w in want]))
    assert torch.isfinite(out).all()
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_sink,window", [(4, 100), (0, 64), (17, 30), (1, 1), (0, 1), (130, 65), (64, 1000)])
@pytest.mark.parametrize("rolling", [False, True])
def test_prefill_ragged(n_sink, window, rolling, dtype):
    new = [1, 0, 63, 130, 64, 0, 7, 1, 65]
    past = [0, 5, 200, 333, 0, 0, 1000, 129, 61]
    s_cap = (n_sink + window + max(new) + 7) // 8 * 8 if rolling else 1136
    H = W.Heads(2, 4, 45, 90, dtype, len(new))
    prefill(H, past, new, n_sink, window, s_cap, pad=5)
    H.clean()
    H.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs,vch,group", SHAPES)
def test_prefill_head_shapes(pairs, vch, group, dtype):
    H = W.Heads(2, group, pairs, vch, dtype, 3)
    prefill(H, [0, 300, 77], [150, 1, 70], 3, 90, 248, pad=1)
    H.clean()
    H.close()


def test_prefill_wide_heads():
    for dtype in ("bf16", "f32"):
        H = W.Heads(1, 2, 100, 200, dtype, 2, head_dim=256)
        prefill(H, [10, 0], [20, 30], 2, 25, 56)
        H.close()


def test_prefill_long_blocks():
    H = W.Heads(2, 4, 45, 90, "bf16", 2)
    prefill(H, [0, 3000], [2500, 700], 4, 1024, 3704)
    prefill(H, [900, 0], [1, 2000], 0, 5000, 2000)
    H.clean()
    H.close()


def shared(H, prefix, groups, lens, p_cap, s_cap):
    B, N = len(lens), len(prefix)
    KP, VP = H.caches(N, p_cap)
    K, V = H.caches(B, s_cap)
    start = [0] + list(np.cumsum(groups))
    for n in range(N):
        H.fill(KP, n, range(prefix[n]))
        H.fill(VP, n, range(prefix[n]))
    for b in range(B):
        H.fill(K, b, range(lens[b]))
        H.fill(V, b, range(lens[b]))
    q, out = H.query(B), H.out(B)
    H.ctx.rap_decode_attn_shared(0, B, q, N, KP, VP, p_cap, H.ints(start), H.ints(prefix), max(prefix), K, V, s_cap, H.ints(lens), max(lens), out)
    want = []
    for n in range(N):
        for b in range(start[n], start[n + 1]):
            want.append(H.reference(q[b], [(KP, VP, n, range(prefix[n])), (K, V, b, range(lens[b]))]))
    W.check(out, torch.stack([w[0] for w in want]), torch.stack([w[1] for w in want]))
    for b, n in enumerate(np.repeat(np.arange(N), groups)):
        if prefix[n] + lens[b] == 0:
            assert (out[b] == 0).all()
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefix,groups,lens", [
    ([1000], [5], [0, 1, 31, 32, 100]), ([1], [3], [0, 0, 5]), ([0], [3], [0, 4, 70]), ([63, 64, 65, 0, 128], [2, 0, 1, 2, 3], [0, 9, 64, 0, 33, 1, 2, 3]),
    ([5000, 3], [1, 1], [1, 1]), ([2049], [40], [7 * (b % 5) for b in range(40)]), ([700, 900], [70, 33], [b % 3 for b in range(103)])])
def test_shared_prefixes(prefix, groups, lens, dtype):
    H = W.Heads(2, 4, 45, 90, dtype, len(lens))
    shared(H, prefix, groups, lens, (max(prefix) + 8) // 8 * 8, (max(lens) + 8) // 8 * 8)
    H.clean()
    H.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs,vch,group", SHAPES)
def test_shared_head_shapes(pairs, vch, group, dtype):
    H = W.Heads(3, group, pairs, vch, dtype, 6)
    shared(H, [130, 77], [4, 2], [0, 40, 3, 1, 65, 12], 136, 72)
    H.clean()
    H.close()


def test_shared_wide_heads():
    H = W.Heads(2, 2, 120, 250, "bf16", 3, head_dim=256)
    shared(H, [130], [3], [0, 40, 3], 136, 48)
    H.close()


def test_shared_without_a_group():
    """Sequences behind the last group have no prefix."""
    H = W.Heads(2, 4, 45, 90, "bf16", 4)
    KP, VP = H.randn(1, 2, 64, 90), H.randn(1, 2, 64, 90)
    K, V, q, out = H.randn(4, 2, 16, 90), H.randn(4, 2, 16, 90), H.query(4), H.out(4)
    H.ctx.rap_decode_attn_shared(0, 4, q, 1, KP, VP, 64, H.ints([0, 2]), H.ints([64]), 64, K, V, 16, H.ints([3, 0, 16, 5]), 16, out)
    for b, n in enumerate([3, 0, 16, 5]):
        W.check(out[b], *H.reference(q[b], ([(KP, VP, 0, range(64))] if b < 2 else []) + [(K, V, b, range(n))]))
    H.clean()
    H.close()


def slot_call(H, past, new, base, T, n_sink, s_cap, in_place=False):
    B = len(past)
    p, n, a = H.ints(past), H.ints(new), None if base is None else H.ints(base)
    start = H.ints([-7] * (B + 1))
    seq, pos, at = [H.ints([-7] * T) for _ in range(3)]
    after = p if in_place else H.ints([-7] * B)
    H.ctx.rap_build_slots(B, p, n, a, T, n_sink, s_cap, start, seq, pos, at, after)
    return [x.cpu().numpy() for x in (start, seq, pos, at, after)]


@pytest.mark.parametrize("past,new,base", [
    ([0], [1], None), ([5, 0, 9], [0, 0, 0], None), ([7], [0], None), ([3, 30, 300, 1000], [1, 1, 1, 1], None), ([0, 17, 100], [40, 0, 13], [0, 5, 100000]),
    (list(range(0, 700 * 3, 3)), [i % 7 for i in range(700)], None), ([11] * 1500, [1] * 1500, [4] * 1500), ([0, 2 ** 31 - 60], [3000, 50], None),
    ([100000, 5, 0], [9000, 1, 20000], None)])
@pytest.mark.parametrize("in_place", [False, True])
def test_slot_maps(past, new, base, in_place):
    H = W.Heads(2, 4, 45, 90, "bf16", len(past))
    for n_sink, s_cap in [(0, 24000), (4, 24000), (19, 20024)]:
        want = W.slots(past, new, base, n_sink, s_cap)
        T = sum(new)
        got = slot_call(H, past, new, base, T + 9, n_sink, s_cap, in_place)
        for g, w, name in zip(got, want, ("row_start", "seq_id", "pos", "slot", "len_out")):
            assert np.array_equal(g[: len(w)], w), name
            assert (g[len(w):] == -7).all(), name
        H.clean()
    H.close()


def test_slot_maps_report_what_cannot_be():
    H = W.Heads(2, 4, 45, 90, "bf16", 3)
    # more new tokens than a rolling cache has rows: the earlier ones of a row lose it
    got = slot_call(H, [2, 50, 0], [9, 2, 3], None, 14, 2, 8)
    assert np.array_equal(got[3], W.slots([2, 50, 0], [9, 2, 3], None, 2, 8)[3]) and (got[3] == -1).sum() == 3
    assert H.ctx.rap_get_last_device_status() == (binding.RAP_ECAPACITY, 0)
    # fewer rows than tokens
    got = slot_call(H, [2, 50, 0], [4, 2, 3], None, 5, 2, 64)
    assert got[0].tolist() == [0, 4, 5, 5] and got[1].tolist() == [0, 0, 0, 0, 1]
    assert H.ctx.rap_get_last_device_status()[0] == binding.RAP_ECAPACITY
    # negative lengths count as none
    got = slot_call(H, [2, -50, 0], [4, 2, -3], None, 6, 2, 64)
    assert got[0].tolist() == [0, 4, 6, 6] and got[2].tolist() == [2, 3, 4, 5, 0, 1] and got[4].tolist() == [6, 2, 0]
    assert H.ctx.rap_get_last_device_status()[0] == binding.RAP_EINVAL
    # positions beyond 31 bits
    got = slot_call(H, [2 ** 31 - 2, 3, 0], [1, 1, 0], [1, 2 ** 31 - 3, 0], 2, 2, 64)
    assert got[2].tolist() == [2 ** 31 - 1, -7]
    assert H.ctx.rap_get_last_device_status() == (binding.RAP_EINVAL, 1)
    H.clean()
    H.close()


def test_no_rows_no_sequences():
    H = W.Heads(2, 4, 45, 90, "bf16", 3)
    got = slot_call(H, [1, 2, 3], [0, 0, 0], None, 0, 0, 8)
    assert got[0].tolist() == [0, 0, 0, 0] and got[4].tolist() == [1, 2, 3]
    start = H.ints([-7])
    H.ctx.rap_build_slots(0, start, start, None, 0, 0, 8, H.ints([0]), *[H.ints([0]) for _ in range(3)], None)
    K, V = H.caches(1, 8)
    q, out = H.query(1), H.out(1, fill=3.0)
    H.ctx.rap_decode_attn_window(0, 0, q, K, V, 8, start, 0, 0, 1, out)
    H.ctx.rap_prefill_attn_window(0, 0, 1, q, K, V, 8, start, start, 0, 0, 0, 1, out)
    H.ctx.rap_prefill_attn_window(0, 1, 0, q, K, V, 8, H.ints([0, 0]), H.ints([4]), 0, 4, 0, 1, out)
    H.ctx.rap_prefill_attn_window(0, 1, 1, q, K, V, 8, H.ints([0, 0]), H.ints([4]), 0, 4, 0, 1, out)
    H.ctx.rap_decode_attn_shared(0, 0, q, 1, K, V, 8, start, start, 0, K, V, 8, start, 0, out)
    assert (out == 3.0).all()
    H.clean()
    H.close()


def test_special_values_stay_where_they_are_seen():
    """A NaN or an infinity in a row that is seen reaches its KV head's outputs and no others; 0 times infinity in rows that
    are not seen reaches nothing."""
    H = W.Heads(2, 4, 45, 90, "bf16", 3)
    K, V, q = H.randn(3, 2, 64, 90), H.randn(3, 2, 64, 90), H.query(3)
    K[0, 1, 40, 3] = math.nan
    V[1, 0, 41, 5] = math.inf
    K[2, :, 20] = math.inf                             # position 20 is neither a sink nor in the window
    V[2, :, 20] = -math.inf
    out = H.out(3)
    H.ctx.rap_decode_attn_window(0, 3, q, K, V, 64, H.ints([50, 50, 50]), 50, 4, 16, out)
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[0, 4:] = True
    bad[1, :4, 5] = True
    assert torch.equal(~torch.isfinite(out), bad)
    assert torch.isnan(out[0, 4:]).all() and (out[1, :4, 5] == math.inf).all()
    H.clean()
    H.close()


def test_large_logits():
    """Weights of one row of many, and logits far beyond fp32's exponents of 2."""
    H = W.Heads(1, 4, 45, 90, "bf16", 2)
    K, V = H.randn(2, 1, 512, 90, scale=30.0), H.randn(2, 1, 512, 90)
    q, out = H.randn(2, 4, 90, scale=40.0), H.out(2)
    lens = [512, 400]
    H.ctx.rap_decode_attn_window(0, 2, q, K, V, 512, H.ints(lens), 512, 4, 300, out)
    for b, n in enumerate(lens):
        want, bound = H.reference(q[b], [(K, V, b, W.seen(n - 1, 4, 300))])
        assert ((out[b] - want).abs() <= bound).all()
    H.close()


@pytest.mark.parametrize("pairs,vch", [(45, 90), (64, 128)])
def test_a_wait_that_runs_out_is_reported(pairs, vch):
    """One stage is armed and nothing copied into it: the launch ends, says so, and the next ones are right again."""
    H = W.Heads(2, 4, pairs, vch, "bf16", 3)
    K, V, q = H.randn(3, 2, 512, 2 * pairs), H.randn(3, 2, 512, vch), H.query(3)
    lens, want = [500, 30, 400], []
    for b, n in enumerate(lens):
        want.append(H.reference(q[b], [(K, V, b, W.seen(n - 1, 4, 300))]))

    def call():
        out = H.out(3)
        H.ctx.rap_decode_attn_window(0, 3, q, K, V, 512, H.ints(lens), 500, 4, 300, out)
        return out

    H.ctx.rap_debug_arm_wait_timeout()
    call()
    assert H.ctx.rap_get_last_device_status()[0] == binding.RAP_ETIMEOUT
    H.ctx.rap_debug_arm_wait_timeout()
    call()                                              # counters left behind, and not asked for
    for _ in range(3):
        out = call()
        W.check(out, torch.stack([w[0] for w in want]), torch.stack([w[1] for w in want]))
    assert H.ctx.rap_get_last_device_status()[0] == binding.RAP_ETIMEOUT
    out = H.out(3)
    H.ctx.rap_decode_attn_shared(0, 3, q, 1, K, V, 512, H.ints([0, 3]), H.ints([512]), 512, K, V, 512, H.ints(lens), 500, out)
    for b, n in enumerate(lens):
        W.check(out[b], *H.reference(q[b], [(K, V, 0, range(512)), (K, V, b, range(n))]))
    H.clean()
    H.close()


def refused(status, f, *a):
    with pytest.raises(binding.RapError) as e:
        f(*a)
    assert e.value.status == status


def test_refusals():
    H = W.Heads(2, 4, 45, 90, "bf16", 2)
    K, V = H.caches(2, 64)
    q, out, n, s = H.query(2), H.out(2, fill=1.0), H.ints([3, 4]), H.ints([0, 1, 2])
    E, A, S, C = binding.RAP_EINVAL, binding.RAP_EALIGN, binding.RAP_ESHAPE, binding.RAP_ECAPACITY
    D = H.ctx.rap_decode_attn_window
    refused(E, D, 1, 2, q, K, V, 64, n, 4, 0, 8, out)
    refused(E, D, 0, -1, q, K, V, 64, n, 4, 0, 8, out)
    refused(E, D, 0, 2, q, K, V, 64, n, -1, 0, 8, out)
    refused(E, D, 0, 2, q, K, V, 64, n, 4, -1, 8, out)
    refused(E, D, 0, 2, q, K, V, 64, n, 4, 64, 8, out)
    refused(E, D, 0, 2, q, K, V, 64, n, 4, 0, 0, out)
    refused(S, D, 0, 3, q, K, V, 64, n, 4, 0, 8, out)
    refused(A, D, 0, 2, q, K, V, 60, n, 4, 0, 8, out)
    refused(A, D, 0, 2, q, K.data_ptr() + 4, V, 64, n, 4, 0, 8, out)
    refused(C, D, 0, 2, q, K, V, 64, n, 65, 4, 61, out)
    D(0, 2, q, K, V, 64, H.ints([0, 0]), 65, 4, 60, H.out(2))
    P = H.ctx.rap_prefill_attn_window
    refused(E, P, 0, 2, 2, q, K, V, 64, None, n, 1, 4, 0, 8, out)
    refused(E, P, 0, 2, -1, q, K, V, 64, s, n, 1, 4, 0, 8, out)
    refused(E, P, 0, 2, 2, q, K, V, 64, s, n, 5, 4, 0, 8, out)
    refused(E, P, 0, 2, 2, q, K, V, 64, s, n, 1, 4, 0, 0, out)
    refused(S, P, 0, 3, 2, q, K, V, 64, s, n, 1, 4, 0, 8, out)
    refused(A, P, 0, 2, 2, q, K, V, 64, s.data_ptr() + 4, n, 1, 4, 0, 8, out)
    refused(C, P, 0, 2, 2, q, K, V, 64, s, n, 10, 65, 4, 52, out)
    F = H.ctx.rap_decode_attn_shared
    refused(E, F, 0, 2, q, 0, K, V, 64, s, n, 4, K, V, 64, n, 4, out)
    refused(E, F, 0, 2, q, 1, K, V, 64, s, n, -1, K, V, 64, n, 4, out)
    refused(E, F, 0, 2, q, 1, K, V, 64, s, n, 4, None, V, 64, n, 4, out)
    refused(S, F, 0, 3, q, 1, K, V, 64, s, n, 4, K, V, 64, n, 4, out)
    refused(A, F, 0, 2, q, 1, K, V, 60, s, n, 4, K, V, 64, n, 4, out)
    refused(A, F, 0, 2, q, 1, K, V, 64, s, n, 4, K, V, 64, n, 4, out.data_ptr() + 4)
    refused(C, F, 0, 2, q, 1, K, V, 64, s, n, 65, K, V, 64, n, 4, out)
    refused(C, F, 0, 2, q, 1, K, V, 64, s, n, 4, K, V, 64, n, 65, out)
    R = H.ctx.rap_build_slots
    t = [H.ints([0] * 8) for _ in range(4)]
    refused(E, R, 2, n, n, None, 4, 64, 64, *t, None)
    refused(E, R, 2, n, s, None, 4, 0, 64, t[0], t[1], t[1], t[2], None)
    refused(E, R, 2, n, s, None, 4, 0, 64, *t, s)
    refused(S, R, 3, n, s, None, 4, 0, 64, *t, None)
    refused(A, R, 2, n, s, None, 4, 0, 60, *t, None)
    assert (out == 1.0).all()
    H.clean()
    H.close()


def test_calls_back_to_back_and_replayed():
    """Calls of unlike batches one behind the other without a wait, then the same captured and replayed with lengths that the
    graph itself advances: the results are those of calls waited for one by one, to the bit."""
    H = W.Heads(2, 4, 45, 90, "bf16", 40, max_rows=64)
    n_sink, window, s_cap = 4, 200, 264
    K, V = H.randn(40, 2, s_cap, 90), H.randn(40, 2, s_cap, 90)
    KP, VP = H.randn(1, 2, 504, 90), H.randn(1, 2, 504, 90)
    q = H.query(40)
    sizes = [40, 3, 17, 1, 40]

    def decode_once(B, lens, out):
        H.ctx.rap_decode_attn_window(0, B, q, K, V, s_cap, lens, 5000, n_sink, window, out)

    def shared_once(B, lens, out):
        H.ctx.rap_decode_attn_shared(0, B, q, 1, KP, VP, 504, H_group[B], H_pre, 500, K, V, s_cap, lens, s_cap, out)

    H_group, H_pre = {B: H.ints([0, B]) for B in sizes}, H.ints([500])
    lens = H.ints([(31 * b) % 260 for b in range(40)])
    alone, packed = [], []
    for B in sizes:
        for f in (decode_once, shared_once):
            o = H.out(40)
            f(B, lens, o)
            torch.cuda.synchronize()
            alone.append(o[:B].clone())
    for B in sizes:
        for f in (decode_once, shared_once):
            o = H.out(40)
            f(B, lens, o)
            packed.append(o[:B])
    torch.cuda.synchronize()
    assert all(torch.equal(a, p) for a, p in zip(alone, packed))
    # a step that advances its own lengths, captured
    steps, B = 6, 17
    one = H.ints([1] * B)
    maps = [H.ints([0] * 24) for _ in range(4)]

    def step(lens, outs):
        H.ctx.rap_build_slots(B, lens, one, None, B, n_sink, s_cap, *maps, lens)
        decode_once(B, lens, outs[0])
        shared_once(B, lens, outs[1])
        H.ctx.rap_prefill_attn_window(0, B, B, q, K, V, s_cap, maps[0], lens, 1, 5000, n_sink, window, outs[2])

    want, start = [], H.ints([10 * b for b in range(B)])
    lens = start.clone()
    outs = [H.out(40, fill=0.5) for _ in range(3)]
    for _ in range(steps):
        step(lens, outs)
        torch.cuda.synchronize()
        want.append([o.clone() for o in outs])
    lens.copy_(start)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(lens, outs)
    torch.cuda.synchronize()
    lens.copy_(start)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(lens, outs)
    for i in range(steps):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want[i])), i
    lens.copy_(start)
    for i in range(steps):                              # no wait in between
        graph.replay()
    decode_once(40, lens, H.out(40))                     # and an eager call of another size behind it
    graph.replay()
    torch.cuda.synchronize()
    assert lens.tolist() == [n + steps + 1 for n in start.tolist()]
    H.clean()
    H.close()


def test_two_contexts_on_two_streams():
    streams = [torch.cuda.Stream() for _ in range(2)]
    sides = []
    for s in streams:
        with torch.cuda.stream(s):
            H = W.Heads(8, 4, 45, 90, "bf16", 8)
            K, V, q = H.randn(8, 8, 2048, 90), H.randn(8, 8, 2048, 90), H.query(8)
            sides.append((s, H, K, V, q, H.ints([2000 - 100 * b for b in range(8)]), [H.out(8) for _ in range(6)]))
    torch.cuda.synchronize()
    for i in range(6):
        for s, H, K, V, q, n, outs in sides:
            with torch.cuda.stream(s):
                if i % 2:
                    H.ctx.rap_decode_attn_window(0, 8, q, K, V, 2048, n, 2000, 4, 1000, outs[i])
                else:
                    H.ctx.rap_decode_attn_shared(0, 8, q, 1, K, V, 2048, H.ints([0, 8]), H.ints([2048]), 2048, K, V, 2048, n, 2000, outs[i])
    torch.cuda.synchronize()
    for s, H, K, V, q, n, outs in sides:
        for i in (2, 3, 4, 5):
            assert torch.equal(outs[i], outs[i % 2])
        W.check(outs[1][3], *H.reference(q[3], [(K, V, 3, W.seen(1699, 4, 1000))]))
        W.check(outs[0][3], *H.reference(q[3], [(K, V, 0, range(2048)), (K, V, 3, range(1700))]))
        H.clean()
        H.close()


def test_against_the_calls_beside_them():
    """A window beyond every length gives rap_decode_attn's and rap_prefill_attn's results."""
    H = W.Heads(4, 4, 45, 90, "bf16", 3)
    K, V, q = H.randn(3, 4, 1024, 90), H.randn(3, 4, 1024, 90), H.query(3)
    n = H.ints([1000, 17, 512])
    a, b = H.out(3), H.out(3)
    H.ctx.rap_decode_attn(0, 3, q, K, V, 1024, n, 1000, 0, a)
    H.ctx.rap_decode_attn_window(0, 3, q, K, V, 1024, n, 1000, 4, 1024, b)
    # 1e-5: the older call's weights carry 17 bits too
    assert float((a - b).norm() / a.norm()) <= 1e-5
    T = 100
    q = H.query(3 * T)
    a, b = H.out(3 * T), H.out(3 * T)
    H.ctx.rap_prefill_attn(0, 3, T, q, K, V, 1024, H.ints([900, 0, 412]), 900, a)
    H.ctx.rap_prefill_attn_window(0, 3, 3 * T, q, K, V, 1024, H.ints([0, T, 2 * T, 3 * T]), H.ints([1000, T, 512]), T, 1000, 0, 1024, b)
    # the older call rounds a weight to one bf16 number: 2^-8 of itself at most
    assert float((a - b).norm() / a.norm()) <= 2.0 ** -8
    H.close()


def test_far_rows():
    """Rows behind 2^31 numbers and 2^32 bytes of a cache."""
    H = W.Heads(2, 2, 64, 128, "bf16", 2)
    s_cap = 9 * 2 ** 20                                  # 2 x 2 x 9M x 128 numbers: 9.7 GB a cache
    K, V = [torch.empty((2, 2, s_cap, 128), dtype=torch.bfloat16, device=H.device) for _ in range(2)]
    n_sink, window, lens = 3, 700, [s_cap + 300, s_cap]
    rows = [[W.slot(p, n_sink, s_cap) for p in W.seen(n - 1, n_sink, window)] for n in lens]
    for b in range(2):
        H.fill(K, b, rows[b])
        H.fill(V, b, rows[b])
    q, out = H.query(2), H.out(2)
    H.ctx.rap_decode_attn_window(0, 2, q, K, V, s_cap, H.ints(lens), max(lens), n_sink, window, out)
    for b in range(2):
        W.check(out[b], *H.reference(q[b], [(K, V, b, rows[b])]))
    out = H.out(2)
    H.ctx.rap_prefill_attn_window(0, 2, 2, q, K, V, s_cap, H.ints([0, 1, 2]), H.ints(lens), 1, max(lens), n_sink, window, out)
    for b in range(2):
        W.check(out[b], *H.reference(q[b], [(K, V, b, rows[b])]))
    H.ctx.rap_decode_attn_shared(0, 1, q, 1, K[1:], V[1:], s_cap, H.ints([0, 1]), H.ints([3]), 3, K, V, 8, H.ints([3]), 8, out)
    H.clean()
    H.close()


@pytest.mark.parametrize("rolling", [False, True])
def test_a_conversation_on_a_cache(rolling):
    """Prompt and answer as a server runs them: slot maps from the lengths, projection with append, block attention over the
    prompt's chunks of unlike sizes, then one token at a time -- all from one device-side length array; the attention is
    compared with the definition on the positions' own K and V rows, kept apart from the cache."""
    B, hidden, n_sink, window = 3, 256, 2, 40
    H = W.Heads(2, 4, 45, 90, "bf16", B, hidden=hidden, max_rows=64)
    heads, n_out = 8, (8 + 2) * 90 + 2 * 90
    wq = H.randn(n_out, hidden, scale=0.1)
    s_cap = 88 if rolling else 256
    K, V = H.caches(B, s_cap)
    lens = H.ints([0] * B)
    held = [[] for _ in range(B)]                        # every position's K and V rows as they were appended
    chunks = [[30, 0, 1], [5, 33, 20], [0, 17, 40], [31, 1, 2]] + [[1, 1, 1]] * 60
    past = [0] * B
    for new in chunks:
        T = sum(new)
        maps = [H.ints([-1] * (n + 8)) for n in (B + 1, T, T, T)]
        start, seq, pos, at = maps
        H.ctx.rap_build_slots(B, lens, H.ints(new), None, T, n_sink, s_cap, start, seq, pos, at, lens)
        x, q = H.randn(T, hidden), torch.empty((T, heads, 90), dtype=H.dt, device=H.device)
        H.ctx.rap_qkv_rope_append(0, T, x, wq, None, seq, pos, at, s_cap - 1, H.tables[3], q, K, V, B, s_cap)
        longest = max(p + n for p, n in zip(past, new))
        out = H.out(T)
        if max(new) == 1 and min(new) == 1:
            H.ctx.rap_decode_attn_window(0, B, q, K, V, s_cap, lens, longest, n_sink, window, out)
        else:
            H.ctx.rap_prefill_attn_window(0, B, T, q, K, V, s_cap, start, lens, max(new), longest, n_sink, window, out)
        r = 0
        for b in range(B):
            for p in range(past[b], past[b] + new[b]):
                s = W.slot(p, n_sink, s_cap)
                held[b].append((K[b, :, s].clone(), V[b, :, s].clone()))
        for b in range(B):
            for p in range(past[b], past[b] + new[b]):
                if new[b] == 1 or p % 7 == 0:
                    rows = W.seen(p, n_sink, window)
                    kk, vv = [torch.stack([held[b][j][i] for j in rows], 1)[None] for i in range(2)]
                    W.check(out[r], *H.reference(q[r], [(kk, vv, 0, range(len(rows)))]))
                r += 1
        past = [p + n for p, n in zip(past, new)]
    assert lens.tolist() == past
    H.clean()
    H.close()


def test_a_batch_behind_one_prompt():
    """A prompt prefilled once, then several answers that share it: positions run on from the prompt's, each sequence appends to
    its own cache, and every step equals attention over the whole conversation."""
    B, hidden, prompt = 5, 256, 70
    H = W.Heads(2, 4, 45, 90, "bf16", B, hidden=hidden, max_rows=128)
    wq = H.randn((8 + 2) * 90 + 2 * 90, hidden, scale=0.1)
    KP, VP = H.caches(1, 72)
    K, V = H.caches(B, 16)

    def append(T, seq, pos, at, k, v, n, cap):
        q = torch.empty((T, 8, 90), dtype=H.dt, device=H.device)
        H.ctx.rap_qkv_rope_append(0, T, H.randn(T, hidden), wq, None, seq, pos, at, cap - 1, H.tables[3], q, k, v, n, cap)
        return q

    plen = H.ints([0])
    m = [H.ints([0] * 128) for _ in range(4)]
    H.ctx.rap_build_slots(1, plen, H.ints([prompt]), None, prompt, 0, 72, *m, plen)
    append(prompt, *m[1:], KP, VP, 1, 72)
    lens, base, group = H.ints([0] * B), H.ints([prompt] * B), H.ints([0, B])
    for step in range(12):
        H.ctx.rap_build_slots(B, lens, H.ints([1] * B), base, B, 0, 16, *m, lens)
        assert m[2][:B].tolist() == [prompt + step] * B and m[3][:B].tolist() == [step] * B
        q = append(B, *m[1:], K, V, B, 16)
        out = H.out(B)
        H.ctx.rap_decode_attn_shared(0, B, q, 1, KP, VP, 72, group, plen, 72, K, V, 16, lens, 16, out)
        for b in range(B):
            W.check(out[b], *H.reference(q[b], [(KP, VP, 0, range(prompt)), (K, V, b, range(step + 1))]))
    H.clean()
    H.close()


@pytest.mark.parametrize("pairs,vch,group", [(45, 90, 4), (58, 115, 3), (64, 128, 4), (64, 127, 5), (22, 45, 8)])
def test_prefill_over_many_rows(pairs, vch, group):
    """Sums that leave tensor memory on the way: every 2560 rows, here none to five times, and right at the border."""
    H = W.Heads(1, group, pairs, vch, "bf16", 4)
    prefill(H, [12000, 4088, 8190, 4096], [5, 8, 70, 0], 4, 10 ** 6, 12008, pad=1)
    prefill(H, [30000, 4088, 8190, 16000], [5, 9, 70, 1], 130, 9000, 9200)
    prefill(H, [2552, 2552, 5110, 2550], [8, 9, 12, 70], 0, 10 ** 6, 5128)
    H.clean()
    H.close()


@pytest.mark.parametrize("rising", [False, True])
def test_prefill_maxima_that_move_over_many_rows(rising):
    """The largest logits in the last rows, or in the first."""
    for pairs, vch in ((45, 90), (64, 128)):
        H = W.Heads(1, 4, pairs, vch, "bf16", 1)
        n, m = 13000, 300
        K, V = H.caches(1, n)
        slope = torch.linspace(0.2, 8.0, n, device=H.device)[:, None]
        K[0, 0] = (H.randn(n, 2 * pairs).float() * (slope if rising else slope.flip(0))).to(H.dt)
        V[0, 0] = H.randn(n, vch)
        q, out = H.query(m), H.out(m)
        H.ctx.rap_prefill_attn_window(0, 1, m, q, K, V, n, H.ints([0, m]), H.ints([n]), m, n, 0, 2 ** 31 - 1, out)
        for i in (0, 1, 63, 64, 130, m - 1):
            want, bound = H.reference(q[i], [(K, V, 0, range(n - m + i + 1))])
            assert ((out[i] - want).abs() <= bound).all()
        H.clean()
        H.close()


@pytest.mark.parametrize("pairs,vch,group", [(45, 90, 4), (58, 115, 3), (64, 128, 4)])
def test_shared_prefixes_of_many_rows_a_split(pairs, vch, group):
    H = W.Heads(8, group, pairs, vch, "bf16", 8)       # 64 pieces: splits of 77 tiles of 64 rows on 148 SMs
    shared(H, [6400, 6399, 6337, 6400, 4097, 4096, 6400, 6400], [1] * 8, [0, 3, 1, 40, 7, 0, 64, 9], 6400, 64)
    H.clean()
    H.close()


@pytest.mark.parametrize("kv,lens,shape", [
    (2, [16384, 4096], (45, 90, 4)), (2, [16384, 4096], (48, 96, 4)), (4, [16860, 999, 364], (45, 90, 4)), (4, [3230, 14656], (58, 115, 3)),
    (2, [8224], (48, 96, 4)), (4, [8224], (48, 96, 4)), (2, [8704], (48, 96, 5)), (4, [9120], (48, 96, 2)),
    (2, [128, 6976, 96, 448, 3264, 9152], (64, 128, 4)), (4, [1696, 9504], (32, 64, 8))])
def test_decode_long_units(kv, lens, shape):
    """Few units, one far longer than the others: as many CTAs share it as there are places for partials."""
    pairs, vch, group = shape
    H = W.Heads(kv, group, pairs, vch, "bf16", len(lens))
    s_cap = (max(lens) + 7) // 8 * 8
    for order in (lens, lens[::-1]):
        W.check(*decode(H, order, 0, s_cap, s_cap))
    H.clean()
    H.close()


@pytest.mark.parametrize("kv,prefix,lens,shape", [(4, 1280, [248, 5744], (45, 90, 4)), (2, 640, [96, 160, 7328, 3904, 96, 7360], (45, 90, 4)),
                                                  (4, 1280, [248, 5744], (48, 96, 4)), (2, 4000, [9000], (48, 96, 3))])
def test_shared_long_units(kv, prefix, lens, shape):
    pairs, vch, group = shape
    H = W.Heads(kv, group, pairs, vch, "bf16", len(lens))
    shared(H, [prefix], [len(lens)], lens, prefix, (max(lens) + 7) // 8 * 8)
    H.clean()
    H.close()


@pytest.mark.parametrize("pairs,vch,group,dtype", [(45, 90, 4, "bf16"), (58, 115, 3, "bf16"), (64, 128, 5, "bf16"), (45, 90, 4, "f32")])
@pytest.mark.parametrize("end", [2 ** 31 - 1, 2 ** 31 - 40, 2 ** 31 - 64])
def test_prefill_at_the_last_positions(end, pairs, vch, group, dtype):
    """Rolling caches bound no length: blocks that end right below 2^31."""
    H = W.Heads(2, group, pairs, vch, dtype, 4)
    new = [130, 1, 0, 70]
    prefill(H, [end - n for n in new], new, 4, 100, 240, pad=2)
    prefill(H, [end - n for n in new], new, 0, 33, 168)
    H.clean()
    H.close()


def test_caches_of_too_many_rows_are_refused():
    """Rows and the blocks that reach beyond the last one are counted in 32 bits."""
    H = W.Heads(2, 4, 45, 90, "bf16", 2)
    K, V = H.caches(2, 64)
    q, out, n, s = H.query(2), H.out(2, fill=1.0), H.ints([0, 0]), H.ints([0, 1, 2])
    most, S = 2 ** 31 - 72, binding.RAP_ESHAPE
    for rows in (most + 8, 2 ** 31 - 8):
        refused(S, H.ctx.rap_decode_attn_window, 0, 2, q, K, V, rows, n, 0, 0, 8, out)
        refused(S, H.ctx.rap_prefill_attn_window, 0, 2, 2, q, K, V, rows, s, n, 1, 1, 0, 8, out)
        refused(S, H.ctx.rap_decode_attn_shared, 0, 2, q, 1, K, V, rows, s, n, 0, K, V, 64, n, 0, out)
        refused(S, H.ctx.rap_decode_attn_shared, 0, 2, q, 1, K, V, 64, s, n, 0, K, V, rows, n, 0, out)
    assert (out == 1.0).all()
    H.ctx.rap_decode_attn_window(0, 2, q, K, V, most, n, 0, 0, 8, out)      # nothing is seen, nothing is read
    assert (out == 0.0).all()
    H.clean()
    H.close()


@pytest.mark.parametrize("offset", [0.0, 1.0])
@pytest.mark.parametrize("pairs,vch,group,n", [(45, 90, 4, 65536), (64, 128, 5, 40000), (58, 115, 3, 40000), (48, 96, 8, 50000)])
def test_decode_many_rows_a_warp(pairs, vch, group, n, offset):
    """More units than there are CTAs, so that a warp sums a quarter of a unit's rows (of 40,000 to 65,536) alone; V of zero mean
    and around one."""
    B = 40
    H = W.Heads(8, group, pairs, vch, "bf16", B)
    K, V = H.randn(B, 8, n, 2 * pairs), H.randn(B, 8, n, vch)
    V += offset
    q, out = H.query(B), H.out(B)
    lens = [n - 37 * b for b in range(B)]
    H.ctx.rap_decode_attn_window(0, B, q, K, V, n, H.ints(lens), n, 0, 2 ** 31 - 1, out)
    for b in (0, 1, B // 2, B - 1):
        W.check(out[b], *H.reference(q[b], [(K, V, b, range(lens[b]))]))
    H.clean()
    H.close()


@pytest.mark.parametrize("pairs,vch,group", [(45, 90, 4), (58, 115, 3), (64, 128, 4), (32, 64, 8), (48, 96, 5), (9, 17, 6), (16, 33, 2), (64, 127, 6), (64, 128, 7), (8, 128, 1)])
def test_decode_long_sums_at_every_border(pairs, vch, group):
    """A launch whose bounds allow many rows a warp, with units of every length: none, one row, and around the blocks after which
    sums leave the accumulators."""
    lens = [9000, 0, 1, 31, 33, 100, 3073, 4063, 4064, 4065, 4095, 4096, 4097, 4127, 4129, 4191, 4193, 4223, 4225, 6144, 6145, 8190, 8192, 8193,
            8225, 8256, 8257, 8289, 8321, 8449, 8999, 700, 2048, 5000, 0, 12, 7777, 128, 129, 64]
    H = W.Heads(8, group, pairs, vch, "bf16", len(lens))
    W.check(*decode(H, lens, 3, 10 ** 6, 9000))
    H.clean()
    H.close()


def test_decode_long_sums_of_special_values():
    B, n = 40, 9000
    H = W.Heads(8, 4, 45, 90, "bf16", B)
    K, V, q = H.randn(B, 8, n, 90), H.randn(B, 8, n, 90), H.query(B)
    K[0, 1, 5000, 3] = math.nan
    V[1, 0, 41, 5] = math.inf                          # before sums have left the accumulators, and behind
    V[2, 0, 8900, 76] = -math.inf
    V[3, 7, 8950, 89] = math.inf
    K[4, :, n - 40:] = math.inf                        # not seen
    V[4, :, n - 40:] = math.nan
    out, lens = H.out(B), [n] * 4 + [n - 40] * 36
    H.ctx.rap_decode_attn_window(0, B, q, K, V, n, H.ints(lens), n, 0, n, out)
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[0, 4:8] = True
    bad[1, :4, 5] = bad[2, :4, 76] = bad[3, 28:, 89] = True
    assert torch.equal(~torch.isfinite(out), bad)
    assert torch.isnan(out[0, 4:8]).all() and (out[1, :4, 5] == math.inf).all() and (out[2, :4, 76] == -math.inf).all() and (out[3, 28:, 89] == math.inf).all()
    W.check(out[4], *H.reference(q[4], [(K, V, 4, range(n - 40))]))
    H.clean()
    H.close()


@pytest.mark.parametrize("rising", [False, True])
def test_decode_maxima_that_move_over_many_rows(rising):
    """The largest logits in the last rows, or in the first."""
    B, n = 40, 20000
    for pairs, vch, group in ((45, 90, 4), (64, 128, 8)):
        H = W.Heads(8, group, pairs, vch, "bf16", B)
        slope = torch.linspace(0.2, 8.0, n, device=H.device)[:, None]
        K = torch.empty((B, 8, n, 2 * pairs), dtype=H.dt, device=H.device)
        for b in range(B):
            K[b] = (H.randn(8, n, 2 * pairs).float() * (slope if rising else slope.flip(0))).to(H.dt)
        V, q, out = H.randn(B, 8, n, vch), H.query(B), H.out(B)
        H.ctx.rap_decode_attn_window(0, B, q, K, V, n, H.ints([n] * B), n, 0, n, out)
        for b in (0, 17, B - 1):
            want, bound = H.reference(q[b], [(K, V, b, range(n))])
            assert ((out[b] - want).abs() <= bound).all()
        H.clean()
        H.close()


def test_shared_long_sums():
    """Many own rows behind a prefix."""
    for pairs, vch, group in ((45, 90, 4), (48, 96, 3)):
        H = W.Heads(8, group, pairs, vch, "bf16", 40)
        shared(H, [500, 0, 1300], [20, 1, 19], [9000 - 300 * (b % 30) for b in range(40)], 1304, 9000)
        H.clean()
        H.close()


@pytest.mark.parametrize("pairs,vch", [(45, 90), (64, 128), (48, 96)])
def test_a_join_that_runs_out_is_reported(pairs, vch):
    """Joins that wait for more than is copied: the launch ends, says so, and the next ones are right again."""
    H = W.Heads(2, 4, pairs, vch, "bf16", 3)
    K, V, q = H.randn(3, 2, 2048, 2 * pairs), H.randn(3, 2, 2048, vch), H.query(3)
    lens, start, plen = H.ints([2000, 30, 1900]), H.ints([0, 3]), H.ints([700])
    window = [H.reference(q[b], [(K, V, b, W.seen(n - 1, 4, 1500))]) for b, n in enumerate(lens.tolist())]
    behind = [H.reference(q[b], [(K, V, 0, range(700)), (K, V, b, range(n))]) for b, n in enumerate(lens.tolist())]

    def call(prefix):
        out = H.out(3)
        if prefix:
            H.ctx.rap_decode_attn_shared(0, 3, q, 1, K, V, 2048, start, plen, 700, K, V, 2048, lens, 2000, out)
        else:
            H.ctx.rap_decode_attn_window(0, 3, q, K, V, 2048, lens, 2000, 4, 1500, out)
        return out

    for prefix in (False, True):
        H.ctx.rap_debug_arm_join_timeout()
        call(prefix)
        assert H.ctx.rap_get_last_device_status()[0] == binding.RAP_ETIMEOUT
        H.ctx.rap_debug_arm_join_timeout()
        call(prefix)                                     # counters left behind, and not asked for
        for again in (True, False, True):
            want = behind if again else window
            W.check(call(again), torch.stack([w[0] for w in want]), torch.stack([w[1] for w in want]))
        assert H.ctx.rap_get_last_device_status()[0] == binding.RAP_ETIMEOUT
    H.clean()
    H.close()


@pytest.mark.parametrize("pairs,vch,group,dtype", [(45, 90, 4, "bf16"), (58, 115, 3, "bf16"), (64, 128, 4, "bf16"), (45, 90, 4, "f32")])
def test_special_values_in_blocks(pairs, vch, group, dtype):
    """A NaN in a K row reaches the queries that see it, an infinity in a V row its channel: as an infinity in fp32; in bf16, where
    a weight is a rounding and a remainder, as an infinity if the remainder is positive and as NaN (inf - inf, or 0 inf) if not, and
    for queries of the block that do not see the row too.  What no query sees may hold anything."""
    H = W.Heads(2, group, pairs, vch, dtype, 3)
    n_sink, window, s_cap = 4, 60, 400
    new, past = [70, 40, 5], [100, 60, 300]
    K, V = H.randn(3, 2, s_cap, 2 * pairs), H.randn(3, 2, s_cap, vch)
    K[0, 1, 120, 3] = math.nan
    V[1, 0, 80, 5] = math.inf
    K[2, :, 5:240], V[2, :, 5:240] = math.nan, -math.inf
    K[:, :, 305:], V[:, :, 305:] = math.inf, math.nan
    T, start, lens = sum(new), [0, 70, 110, 115], [p + n for p, n in zip(past, new)]
    q, out = H.query(T), H.out(T)
    H.ctx.rap_prefill_attn_window(0, 3, T, q, K, V, s_cap, H.ints(start), H.ints(lens), max(new), max(lens), n_sink, window, out)
    for b in range(3):
        for i in range(new[b]):
            pos, o = past[b] + i, out[start[b] + i]
            rows = W.seen(pos, n_sink, window)
            want, bound = H.reference(q[start[b] + i], [(K, V, b, rows)])
            good = torch.ones_like(o, dtype=torch.bool)
            if b == 0 and 120 in rows:
                assert torch.isnan(o[group:]).all()
                good[group:] = False
            if b == 1 and (80 in rows or dtype == "bf16"):
                assert 80 not in rows or ((o[:group, 5] == math.inf) if dtype == "f32" else ~torch.isfinite(o[:group, 5])).all()
                good[:group, 5] = False
            assert torch.isfinite(o[good]).all() and ((o - want).abs() <= bound + 1e-30)[good].all()
    H.clean()
    H.close()


@pytest.mark.parametrize("pairs,vch,group,dtype", [(45, 90, 4, "bf16"), (58, 115, 3, "bf16"), (64, 128, 4, "bf16"), (45, 90, 4, "f32")])
def test_special_values_behind_prefixes(pairs, vch, group, dtype):
    """The same of a prefix: a NaN in K reaches its group's outputs of that KV head, an infinity in V its channel, as an infinity
    (fp32) or that or NaN (bf16); in a sequence's own rows it gives an infinity, in rows that are not seen nothing."""
    H = W.Heads(2, group, pairs, vch, dtype, 5)
    prefix, groups, lens = [200, 333], [3, 2], [9, 0, 40, 33, 5]
    KP, VP = H.randn(2, 2, 400, 2 * pairs), H.randn(2, 2, 400, vch)
    K, V, q, out = H.randn(5, 2, 64, 2 * pairs), H.randn(5, 2, 64, vch), H.query(5), H.out(5)
    VP[0, 1, 70, 7] = math.inf
    KP[1, 0, 332, 1] = math.nan
    V[2, 0, 39, 9] = -math.inf
    for n, p in enumerate(prefix):
        KP[n, :, p:], VP[n, :, p:] = math.nan, math.inf
    for b, n in enumerate(lens):
        K[b, :, n:], V[b, :, n:] = math.inf, math.nan
    H.ctx.rap_decode_attn_shared(0, 5, q, 2, KP, VP, 400, H.ints([0, 3, 5]), H.ints(prefix), 333, K, V, 64, H.ints(lens), 40, out)
    for b in range(5):
        n = 0 if b < 3 else 1
        want, bound = H.reference(q[b], [(KP, VP, n, range(prefix[n])), (K, V, b, range(lens[b]))])
        good = torch.ones_like(out[b], dtype=torch.bool)
        if n == 0:
            hit = out[b][group:, 7]
            assert ((hit == math.inf) if dtype == "f32" else ~torch.isfinite(hit)).all()
            good[group:, 7] = False
        else:
            assert torch.isnan(out[b][:group]).all()
            good[:group] = False
        if b == 2:
            assert (out[b][:group, 9] == -math.inf).all()
            good[:group, 9] = False
        assert torch.isfinite(out[b][good]).all() and ((out[b] - want).abs() <= bound + 1e-30)[good].all()
    H.clean()
    H.close()


def test_far_rows_behind_a_prefix():
    """A prefix whose group lies behind 2^31 numbers and 2^32 bytes of its cache, and own rows as far."""
    H = W.Heads(2, 2, 64, 128, "bf16", 2)
    cap = 9 * 2 ** 20
    K, V = [torch.empty((2, 2, cap, 128), dtype=torch.bfloat16, device=H.device) for _ in range(2)]
    for c in (K, V):
        H.fill(c, 1, range(700))
        H.fill(c, 0, range(40))
    q, out = H.query(2), H.out(2)
    H.ctx.rap_decode_attn_shared(0, 2, q, 2, K, V, cap, H.ints([0, 1, 2]), H.ints([3, 700]), 700, K, V, cap, H.ints([40, 500]), 500, out)
    for b, p in enumerate((3, 700)):
        W.check(out[b], *H.reference(q[b], [(K, V, b, range(p)), (K, V, b, range((40, 500)[b]))]))
    H.clean()
    H.close()
