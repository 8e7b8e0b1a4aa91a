"""The cache held in 4 bits on the GPU: conversion both ways, the quantising append, the attention and whole decode steps,
against the fp64 oracle through the C ABI."""
from dataclasses import replace

import numpy as np
import pytest
import torch

from oracle import rap_oracle as O
from paper_2602_02599_b200 import binding, synth
from paper_2602_02599_b200.stack import DecodeStack

import q4_util
import util

pytestmark = pytest.mark.gpu


def _bare_stack(w=None, **kw):
    w = w or synth.scaled_down(synth.LLAMA_8B, n_layers=1, batch=1, seq=8, hidden=256)
    return DecodeStack(w, s_cap=kw.pop("s_cap", 8), alloc_cache=False, **kw)


def _ok(st):
    torch.cuda.synchronize()
    assert st.ctx.rap_get_last_device_status() == (0, 0)


def _kind(dtype):
    return binding.RAP_F32 if dtype == "f32" else binding.RAP_BF16


# ---- rows ----------------------------------------------------------------------------------------------------------------


def _rows(n, W, dtype, seed):
    rng = np.random.default_rng(seed)
    x = (rng.normal(0, 1, (n, W)) * rng.lognormal(0, 3, (n, 1)) + rng.normal(0, 2, (n, 1))).astype(np.float32)
    x[0] = 0.0
    if n > 8:
        x[1] = -0.3                                       # one value (not a bf16 number when fp32)
        x[2, : min(W, 4)] = np.array([7.5, -7.5, 1.0, -2.0], dtype=np.float32)[: min(W, 4)]     # s = 1, z = 0: ties to even
        x[2, 4:] = 0.0
        x[3, W // 2] = np.nan
        x[4, 0] = np.inf
        x[5, W - 1] = -np.inf
        x[6] = 1e-40
        x[7] = np.where(np.arange(W) % 2, 3e38, -3e38)
        x[8] = 3.4e38
    return O.round_bf16(x).astype(np.float32) if dtype == "bf16" else x


@pytest.mark.parametrize("W", [1, 2, 3, 7, 8, 9, 31, 32, 33, 48, 64, 90, 115, 116, 128, 129, 255, 256])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 9, 1003])
def test_rows_both_ways_bit_exact(W, dtype, n):
    """Bytes of rap_quantize_rows_q4 and values of rap_dequantize_rows_q4 equal the oracle's: rows of very different
    magnitudes, special rows, ties; what lies behind the last row stays as it was."""
    st = _bare_stack()
    x = _rows(n, W, dtype, W + n)
    tdt = torch.float32 if dtype == "f32" else torch.bfloat16
    dx = torch.from_numpy(x).to(st.device).to(tdt)
    rb = binding.rap_q4_row_bytes(W)
    packed = torch.full((n + 3, rb), 0xAB, dtype=torch.uint8, device=st.device)
    st.ctx.rap_quantize_rows_q4(_kind(dtype), n, W, dx, packed)
    back = torch.full((n + 3, W), 77.0, dtype=tdt, device=st.device)
    st.ctx.rap_dequantize_rows_q4(_kind(dtype), n, W, packed, back)
    wide = torch.full((n + 3, W), 77.0, dtype=torch.float32, device=st.device)
    st.ctx.rap_dequantize_rows_q4(binding.RAP_F32, n, W, packed, wide)
    _ok(st)
    held = O.quantize_rows_q4(x)
    got = packed.cpu().numpy()
    assert np.array_equal(got[:n], q4_util.pack(*held))
    assert np.all(got[n:] == 0xAB) and torch.all(back[n:] == 77.0) and torch.all(wide[n:] == 77.0)
    with np.errstate(over="ignore"):
        want = O.dequantize_rows_q4(*held).astype(np.float32)          # exact in 64 bits, one rounding
    assert np.array_equal(wide[:n].cpu().numpy(), want, equal_nan=True)
    if dtype == "bf16":
        assert np.array_equal(util.to_np64(back[:n]), O.round_bf16(want), equal_nan=True)
    st.close()


def test_rows_on_another_stream_and_an_empty_call():
    st = _bare_stack()
    x = torch.randn((4096, 90), device=st.device)
    packed = torch.zeros((4096, 52), dtype=torch.uint8, device=st.device)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        st.ctx.rap_quantize_rows_q4(binding.RAP_F32, 4096, 90, x, packed)
        st.ctx.rap_quantize_rows_q4(binding.RAP_F32, 0, 90, x, packed)
        st.ctx.rap_dequantize_rows_q4(binding.RAP_F32, 0, 90, packed, x)
    side.synchronize()
    assert np.array_equal(packed.cpu().numpy(), q4_util.pack(*O.quantize_rows_q4(x.cpu().numpy())))
    st.close()


@pytest.mark.parametrize("name", ["8b", "3b", "sweep0.5", "tiny"])
@pytest.mark.parametrize("lens", [[40], [0, 1, 7, 39, 40, 17, 0, 8]])
def test_read_cache_up_to_every_length(name, lens):
    base = synth.CONFIGS[name]
    w = replace(base, batch=len(lens), seq=40, n_layers=1)
    st = DecodeStack(w, s_cap=48)
    st.build_tables(*synth.draw_scores(w))
    k4, v4 = q4_util.caches(st, 0)
    g = torch.Generator(device=st.device).manual_seed(1)
    want = []
    for packed, W in ((k4, 2 * w.n_pairs), (v4, w.n_vch)):
        x = torch.empty(packed.shape[:3] + (W,), device=st.device).normal_(0.2, 1, generator=g)
        st.ctx.rap_quantize_rows_q4(binding.RAP_F32, x.shape[0] * x.shape[1] * x.shape[2], W, x, packed)
        back = torch.empty(x.shape, dtype=st.dt, device=st.device)
        st.ctx.rap_dequantize_rows_q4(_kind(w.dtype), x.shape[0] * x.shape[1] * x.shape[2], W, packed, back)
        for b, n in enumerate(lens):
            back[b, :, n:] = 5.0
            packed[b, :, n:] = 0xFF                  # not to be read as numbers
        want.append(back)
    st.k_cache[0].fill_(5.0)
    st.v_cache[0].fill_(5.0)
    dl = torch.tensor(lens, dtype=torch.int32, device=st.device)
    st.ctx.rap_read_cache_q4(0, len(lens), k4, v4, 48, dl, max(lens), st.k_cache[0], st.v_cache[0])
    _ok(st)
    assert torch.equal(st.k_cache[0], want[0]) and torch.equal(st.v_cache[0], want[1])
    st.ctx.rap_read_cache_q4(0, len(lens), k4, v4, 48, torch.zeros_like(dl), 0, st.k_cache[0], st.v_cache[0])
    _ok(st)
    assert torch.equal(st.k_cache[0], want[0])
    st.close()


# ---- append ----------------------------------------------------------------------------------------------------------------


def _append_case(st, w, T, seed, with_bias=False):
    rng = np.random.default_rng(seed)
    seq_id = rng.integers(0, st.B, size=T).astype(np.int32)
    slot = np.zeros(T, np.int32)
    for b in range(st.B):                                # distinct slots per sequence
        m = seq_id == b
        slot[m] = rng.permutation(st.s_cap)[: m.sum()]
    pos = rng.integers(0, 100000, size=T).astype(np.int32)
    up = lambda a: torch.from_numpy(a).to(st.device)
    bias = None
    if with_bias:
        bias = rng.normal(0, 2, st.n_out(0)).astype(np.float32)
    return seq_id, slot, pos, up(seq_id), up(slot), up(pos), bias


@pytest.mark.parametrize("T", [1, 5, 70])
@pytest.mark.parametrize("with_bias", [False, True])
def test_append_fp32_equals_the_plain_append_then_the_row_quantiser(T, with_bias):
    """An fp32 stack's plain append writes the unrounded K and V rows, so the quantising append has to write exactly what
    rap_quantize_rows_q4 makes of them, and nothing else; q~ is the same bit for bit."""
    w = replace(synth.TINY, batch=3, seq=96)
    ks, vs = synth.draw_scores(w)
    st, tabs, w_host = util.build_small_stack(w, ks, vs, s_cap=96, max_rows=128)
    seq_id, slot, pos, dsid, dslot, dpos, bias = _append_case(st, w, T, T, with_bias)
    dbias = None if bias is None else torch.from_numpy(bias).to(st.device)
    dx = torch.from_numpy(synth.draw_hidden(w, 0, 1, T)).to(st.device)
    st.k_cache[0].zero_()
    st.v_cache[0].zero_()
    q1, q2 = (torch.full((T, w.n_q_heads, 2 * w.n_pairs), float("nan"), device=st.device) for _ in range(2))
    st.ctx.rap_qkv_rope_append(0, T, dx, st.w_qkv[0], dbias, dsid, dpos, dslot, int(slot.max()), st.inv_freq, q1, st.k_cache[0],
                               st.v_cache[0], st.B, st.s_cap)
    k4, v4 = q4_util.caches(st, 0)
    st.ctx.rap_qkv_rope_append_q4(0, T, dx, st.w_qkv[0], dbias, dsid, dpos, dslot, int(slot.max()), st.inv_freq, q2, k4, v4, st.B,
                                  st.s_cap)
    _ok(st)
    assert torch.equal(q1, q2)
    written = np.zeros((st.B, w.n_kv_heads, st.s_cap), bool)
    written[seq_id, :, slot] = True
    for packed, plain in ((k4, st.k_cache[0]), (v4, st.v_cache[0])):
        got = packed.cpu().numpy()
        assert not got[~written].any()
        want = q4_util.pack(*O.quantize_rows_q4(plain.cpu().numpy()))
        assert np.array_equal(got[written], want[written])
    st.close()


@pytest.mark.parametrize("name,T", [("8b", 1), ("8b", 32), ("3b", 17), ("sweep1.0", 5), ("8b", 100), ("sweep0.5", 300)])
def test_append_bf16_holds_the_oracle_rows(name, T):
    """Decode-sized and prompt-sized calls: q~ as the plain append writes it, and every appended row within half a step of
    the oracle's own fp64 projection and rotation (plus the fp32 sum's error, 1e-3 of the row's largest entry), its step
    within a bf16 step and a bit of the oracle's."""
    w = synth.scaled_down(synth.CONFIGS[name], n_layers=1, batch=4, seq=64, hidden=512)
    ks, vs = synth.draw_scores(w)
    st, tabs, w_host = util.build_small_stack(w, ks, vs, s_cap=160, max_rows=512)
    seq_id, slot, pos, dsid, dslot, dpos, _ = _append_case(st, w, T, T)
    P, dv = w.n_pairs, w.n_vch
    X = synth.draw_hidden(w, 0, 2, T)
    dx = torch.from_numpy(X).to(st.device).to(st.dt)
    q1, q2 = (torch.full((T, w.n_q_heads, 2 * P), float("nan"), dtype=st.dt, device=st.device) for _ in range(2))
    k4, v4 = q4_util.caches(st, 0)
    st.ctx.rap_qkv_rope_append_q4(0, T, dx, st.w_qkv[0], None, dsid, dpos, dslot, int(slot.max()), st.inv_freq, q1, k4, v4, st.B,
                                  st.s_cap)
    st.qkv_rope_append(0, dx, dsid, dpos, dslot, int(slot.max()), q_out=q2)
    _ok(st)
    assert torch.equal(q1, q2)
    _, k, v = O.qkv_rope(O.round_storage(X, w.dtype), w_host[0], None, pos, tabs["inv_freq"][0], w.n_q_heads, w.n_kv_heads, P, dv)
    written = np.zeros((st.B, w.n_kv_heads, st.s_cap), bool)
    written[seq_id, :, slot] = True
    for packed, rows, W in ((k4, k, 2 * P), (v4, v, dv)):
        got = packed.cpu().numpy()
        assert not got[~written].any()
        c, s, z = (a[seq_id, :, slot] for a in q4_util.unpack(got, W))
        off = 1e-3 * np.abs(rows).max(-1)
        assert np.all(np.abs(O.dequantize_rows_q4(c, s, z) - rows) <= (0.5 * s * (1 + 2.0 ** -16) + off)[..., None])
        want_s = O.quantize_rows_q4(rows)[1]
        assert np.all(np.abs(s - want_s) <= want_s * 2.0 ** -7 + off / 3)      # z may sit a bf16 step apart: /7.5 of it
    st.close()


@pytest.mark.parametrize("name,T,seed", [("8b", 4000, 1), ("8b", 4000, 2), ("sweep1.0", 2500, 3), ("8b", 30, 4), ("tiny", 600, 5)])
def test_append_writes_the_codes_of_the_rotation_as_it_is_defined(name, T, seed):
    """Every byte of the appended rows is the row quantiser's on O.rotate_k_q4 of the projection (V: on the projection).
    Activations and weights lie on a coarse grid, so that the projection's sums -- multiples of 2^-12 below 2^8 -- are exact in
    fp32 in any order, and far positions.  (The two sides' fp64 sines differ by an ulp or two, which moves an fp32 rounding
    once in 2^26 numbers, and then a code once in a million: nothing in 6 million numbers.)"""
    w = replace(synth.scaled_down(synth.CONFIGS[name], n_layers=1, batch=2, seq=16, hidden=256), seq=16)
    S = (T // 2 + 24) // 8 * 8
    st, tabs, _ = util.build_small_stack(w, *synth.draw_scores(w), s_cap=S, max_rows=T)
    rng = np.random.default_rng(seed)
    X = (np.round(rng.normal(0, 8, (T, w.hidden))) / 8).astype(np.float32)
    Wq = (np.round(rng.normal(0, 0.02 * 512, (st.n_out(0), w.hidden))) / 512).astype(np.float32)
    up = lambda a: torch.from_numpy(a).to(st.device)
    seq_id = np.repeat(np.arange(2), (T + 1) // 2)[:T].astype(np.int32)
    slot = (np.arange(T) - np.where(seq_id, (T + 1) // 2, 0)).astype(np.int32)
    pos = (slot + np.where(seq_id, 91234, 3)).astype(np.int32)
    k4, v4 = q4_util.caches(st, 0)
    q = torch.empty((T, w.n_q_heads, 2 * w.n_pairs), dtype=st.dt, device=st.device)
    st.ctx.rap_qkv_rope_append_q4(0, T, up(X).to(st.dt), up(Wq).to(st.dt), None, up(seq_id), up(pos), up(slot), int(slot.max()), st.inv_freq, q,
                                  k4, v4, 2, S)
    _ok(st)
    H, P2, dv = w.n_kv_heads, 2 * w.n_pairs, w.n_vch
    Y = X.astype(np.float64) @ Wq[w.n_q_heads * P2:].astype(np.float64).T
    assert np.array_equal(Y, Y.astype(np.float32))
    freq = st.inv_freq[0, :, : w.n_pairs].cpu().numpy()
    K = O.rotate_k_q4(Y[:, : H * P2].reshape(T, H, P2), pos, freq)
    V = Y[:, H * P2:].reshape(T, H, dv).astype(np.float32)
    for packed, rows in ((k4, K), (v4, V)):
        got = packed.cpu().numpy()[seq_id, :, slot]
        assert np.array_equal(got, q4_util.pack(*O.quantize_rows_q4(rows)))
    st.close()


def test_append_skips_rows_out_of_range_and_reports_them():
    w = synth.scaled_down(synth.LLAMA_8B, n_layers=1, batch=2, seq=16, hidden=256)
    ks, vs = synth.draw_scores(w)
    st, _, _ = util.build_small_stack(w, ks, vs, s_cap=16, max_rows=8)
    k4, v4 = q4_util.caches(st, 0)
    dx = torch.from_numpy(synth.draw_hidden(w, 0, 1, 4)).to(st.device).to(st.dt)
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device=st.device)
    q = torch.empty((4, w.n_q_heads, 2 * w.n_pairs), dtype=st.dt, device=st.device)
    st.ctx.rap_qkv_rope_append_q4(0, 4, dx, st.w_qkv[0], None, i32(0, 2, -1, 1), i32(1, 2, 3, 4), i32(3, 3, 3, 16), 15, st.inv_freq, q,
                                  k4, v4, 2, 16)
    torch.cuda.synchronize()
    code, detail = st.ctx.rap_get_last_device_status()
    assert code == binding.RAP_ECAPACITY and detail in (1, 2, 3)
    touched = k4.cpu().numpy().any(axis=(-1)) | v4.cpu().numpy().any(axis=-1)
    want = np.zeros_like(touched)
    want[0, :, 3] = True
    assert np.array_equal(touched, want)
    st.close()


# ---- attention ---------------------------------------------------------------------------------------------------------------


def _attn_stack(w, lens, seed=0, gain=1.0, s_cap=None, shift=0.0):
    """(stack, q, k4, v4, lengths): caches quantised from random rows of unlike magnitudes; rows past the end are 0xFF."""
    st = DecodeStack(w, s_cap=s_cap or ((max(lens) + 8 + 7) // 8) * 8, alloc_cache=False)
    st.build_tables(*synth.draw_scores(w))
    g = torch.Generator(device=st.device).manual_seed(seed)
    packed = []
    for cache, W in zip(q4_util.caches(st, 0), (2 * w.n_pairs, w.n_vch)):
        ramp = (1.0 + 0.02 * torch.arange(st.s_cap, device=st.device) % 3.0).view(1, 1, -1, 1)
        x = torch.empty(cache.shape[:3] + (W,), device=st.device).normal_(shift, 1.28, generator=g) * ramp
        st.ctx.rap_quantize_rows_q4(binding.RAP_F32, x.numel() // W, W, x, cache)
        for b, n in enumerate(lens):
            cache[b, :, n:] = 0xFF
        packed.append(cache)
    q = torch.empty((len(lens), w.n_q_heads, 2 * w.n_pairs), dtype=st.dt, device=st.device).normal_(0, 1.28 * gain, generator=g)
    return st, q, packed[0], packed[1], torch.tensor(lens, dtype=torch.int32, device=st.device)


def _run_attn(st, w, q, k4, v4, dl, n_split=0, bound=None):
    out = torch.full((q.shape[0], w.n_q_heads, w.n_vch), float("nan"), dtype=torch.float32, device=st.device)
    st.ctx.rap_decode_attn_q4(0, q.shape[0], q, k4, v4, st.s_cap, dl, int(dl.max()) if bound is None else bound, n_split, out)
    return out


def _attn_case(w, lens, n_split=0, variant=0, **kw):
    st, q, k4, v4, dl = _attn_stack(w, lens, **kw)
    st.ctx.rap_set_attn_variant(variant)
    out = _run_attn(st, w, q, k4, v4, dl, n_split)
    _ok(st)
    held = [q4_util.unpack(c, W) for c, W in ((k4, 2 * w.n_pairs), (v4, w.n_vch))]
    generic = variant == 1 or w.dtype == "f32" or max(2 * w.n_pairs, w.n_vch) > 128
    q4_util.check_attn(util.to_np64(out), util.to_np64(q), held[0], held[1], lens, w.head_dim, 1 if generic else 16)
    st.close()


def _small(name="8b", **kw):
    return replace(synth.scaled_down(synth.CONFIGS[name], n_layers=1, batch=1, seq=64), **kw)


EDGES = [[1], [2, 31, 32, 33, 63], [0, 300, 0, 1, 129, 0], [0, 0], [255, 256, 257, 511, 512, 513], [1] * 9]


@pytest.mark.parametrize("lens", EDGES)
@pytest.mark.parametrize("n_split", [0, 1, 4])
@pytest.mark.parametrize("variant", [0, 1])
def test_attention_lengths_at_every_border(lens, n_split, variant):
    _attn_case(_small(batch=len(lens)), lens, n_split, variant, seed=len(lens))


@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("P,dv", [(45, 90), (58, 115), (32, 64), (64, 128), (51, 102)])
def test_attention_head_shapes(G, P, dv):
    w = _small(batch=2, n_pairs=P, n_vch=dv, n_q_heads=2 * G, n_kv_heads=2)
    _attn_case(w, [777, 130], seed=G)


@pytest.mark.parametrize("P", [1, 2, 4, 5, 11, 16, 17, 23, 31, 33, 48, 49, 63])
def test_attention_odd_widths(P):
    """Any retained counts, K and V apart: fewer numbers than a word of codes, one more than a group of 32."""
    for dv in (1, 2 * P, 129 - 2 * P, 33, 97):
        _attn_case(_small(batch=2, n_pairs=P, n_vch=dv, n_q_heads=6, n_kv_heads=2), [300, 45], seed=P + dv)


@pytest.mark.parametrize("n_split", [0, 7])
@pytest.mark.parametrize("name", ["3b", "8b", "14b"])
def test_attention_longer_sequences(name, n_split):
    _attn_case(replace(_small(name), batch=3), [6000, 2500, 33], n_split, seed=5)


@pytest.mark.parametrize("gain", [0.0, 1e-30, 0.05, 12.0, 1e6])
def test_attention_flat_and_peaked(gain):
    """q of any size: all weights equal, one weight left, a q far outside fp16's range."""
    _attn_case(_small(batch=2), [1500, 40], seed=7, gain=gain)


@pytest.mark.parametrize("G", [1, 4, 5, 8])
@pytest.mark.parametrize("size", [1.0, 2.0 ** 20, 2.0 ** 100])
def test_attention_one_row_left_of_many(G, size):
    """A q far out of fp16's range (the K steps make up for it), and one row 40 binary places above the rest, another one for every
    query head: the outputs are that row's V numbers, which a tolerance made of sum |q| could not tell.  The rest, 2000 rows of
    2^-40, counts 2^-29; the row's own weight 2^-19 of its size for five heads and more (two fp16 numbers of it, the second rounded),
    2^-27 for up to four; V numbers are off by that and three fp32 roundings."""
    n, P = 2000, 16
    w = _small(n_pairs=P, n_vch=90, n_q_heads=G, n_kv_heads=1)
    st = DecodeStack(w, s_cap=n, alloc_cache=False)
    st.build_tables(*synth.draw_scores(w))
    rng = np.random.default_rng(G)
    one = np.ones((1, 1, n))
    rows = rng.permutation(n)[:G]
    k_codes, v_codes = np.zeros((1, 1, n, 2 * P), dtype=np.uint8), rng.integers(0, 16, (1, 1, n, 90)).astype(np.uint8)
    k_codes[0, 0, rows, np.arange(G)] = 15          # head g asks dimension g
    held = [(k_codes, one / size, 0 * one), (v_codes, one, 0 * one)]
    k4, v4 = (torch.from_numpy(q4_util.pack(*h)).to(st.device) for h in held)
    q = torch.zeros((1, G, 2 * P), dtype=st.dt, device=st.device)
    for g in range(G):
        q[0, g, g] = 41 * float(np.sqrt(w.head_dim) * np.log(2)) / 15 * size
    want = v_codes[0, 0, rows] - 7.5
    for n_split in (0, 1, 5):
        out = util.to_np64(_run_attn(st, w, q, k4, v4, torch.tensor([n], dtype=torch.int32, device=st.device), n_split))[0]
        _ok(st)
        assert np.all(np.abs(out - want) <= 7.5 * (2 * 2.0 ** -29 + (2.0 ** -19 if G > 4 else 2.0 ** -26) + 4 * 2.0 ** -24)), np.abs(out - want).max()
    st.close()


@pytest.mark.parametrize("shift", [50.0, -3.0])
def test_attention_rows_off_centre(shift):
    _attn_case(_small(batch=2), [1100, 200], seed=8, shift=shift)


@pytest.mark.parametrize("scale", [1e-20, 1e-6, 3e4, 1e20])
def test_attention_v_of_any_magnitude(scale):
    """Steps of V far outside fp16's range, and unlike ones side by side: the weights carry them."""
    lens = [700, 350]
    w = _small(batch=2)
    st, q, k4, v4, dl = _attn_stack(w, lens, seed=9)
    g = torch.Generator(device=st.device).manual_seed(3)
    spread = torch.exp(3 * torch.randn((2, w.n_kv_heads, st.s_cap, 1), generator=g, device=st.device))
    x = torch.randn((2, w.n_kv_heads, st.s_cap, w.n_vch), generator=g, device=st.device) * spread * scale
    st.ctx.rap_quantize_rows_q4(binding.RAP_F32, x.numel() // w.n_vch, w.n_vch, x, v4)
    out = _run_attn(st, w, q, k4, v4, dl)
    _ok(st)
    q4_util.check_attn(util.to_np64(out), util.to_np64(q), q4_util.unpack(k4, 2 * w.n_pairs), q4_util.unpack(v4, w.n_vch), lens, w.head_dim)
    st.close()


@pytest.mark.parametrize("G", [1, 4, 5, 8])
@pytest.mark.parametrize("middle", [0.0, 0.75, -3e30])
def test_attention_logits_that_rise_over_v_rows_without_a_step(G, middle):
    """Constant V rows have no step, so their weights never come near a limit of weight times step: a logit far above those of the
    blocks before must still raise the reference, or the row sums leave fp32.  40 of 1000 rows lie `bits` binary places above the
    others; with d_v' = 1 all rows are constant.  (Where the 40 are zero rows the others, 2^-60 of them and less, make the output:
    a weight is right to 2^-27 of the largest.)"""
    n = 1000
    for dv, bits in ((48, 60), (48, 100), (48, 124), (48, 127.9), (48, 300), (1, 60), (1, 124), (1, 400)):
        w = _small(n_pairs=16, n_vch=dv, n_q_heads=G, n_kv_heads=1)
        st = DecodeStack(w, s_cap=n, alloc_cache=False)
        st.build_tables(*synth.draw_scores(w))
        rng = np.random.default_rng(dv)
        k_codes, v_codes = np.zeros((1, 1, n, 32), dtype=np.uint8), rng.integers(0, 16, (1, 1, n, dv)).astype(np.uint8)
        k_codes[:, :, 600:640, 0] = 15
        one = np.ones((1, 1, n))
        v_step, v_mid = 0.25 * one, O.round_bf16(rng.normal(0, 1, (1, 1, n)))
        if dv == 1:
            v_step[:] = 0.0
        v_step[:, :, 600:640], v_mid[:, :, 600:640] = 0.0, O.round_bf16(middle * (1 + 0.5 * rng.random(40)))
        held = [(k_codes, one, 0 * one), (v_codes, v_step, v_mid)]
        k4, v4 = (torch.from_numpy(q4_util.pack(*h)).to(st.device) for h in held)
        q = torch.zeros((1, G, 32), dtype=st.dt, device=st.device)
        q[:, :, 0] = bits * float(np.sqrt(w.head_dim) * np.log(2)) / 15
        for n_split in (0, 1, 3):
            out = _run_attn(st, w, q, k4, v4, torch.tensor([n], dtype=torch.int32, device=st.device), n_split)
            _ok(st)
            assert torch.isfinite(out).all(), (dv, bits, n_split)
            want = O.decode_attn_q4(util.to_np64(q), held[0], held[1], [n], w.head_dim)
            tol = q4_util.attn_bound(util.to_np64(q), held[0], held[1], [n], w.head_dim) + n * 2.0 ** -27 * 7.5 * 0.25
            assert np.all(np.abs(util.to_np64(out) - want) <= tol), (dv, bits, n_split)
        st.close()


@pytest.mark.parametrize("G", [1, 4, 5, 8])
@pytest.mark.parametrize("scale", [1.0, 1e-6, 1e20, 1e30])
@pytest.mark.parametrize("gain", [0.0, 1.0])
def test_attention_over_blocks_of_constant_v_rows(G, scale, gain):
    """Rows without a V step, or with next to none, at the front or in the middle -- zeroed slots, zero rows, constant rows, noise --
    say nothing about the weights that the rows behind them need; and they count in the row sums however far apart the steps lie."""
    lens = [2000, 700]
    w = _small(batch=2, n_q_heads=2 * G, n_kv_heads=2)
    st, q, k4, v4, dl = _attn_stack(w, lens, seed=14, gain=gain)
    g = torch.Generator(device=st.device).manual_seed(G)
    x = torch.randn((2, 2, st.s_cap, w.n_vch), generator=g, device=st.device) * scale
    st.ctx.rap_quantize_rows_q4(binding.RAP_F32, x.numel() // w.n_vch, w.n_vch, x, v4)
    kept = v4.clone()
    one = lambda step, middle: torch.from_numpy(q4_util.pack(np.arange(w.n_vch, dtype=np.uint8)[None] % 16, np.array([step]), O.round_bf16(np.array([middle])))).to(st.device)
    constant, noise = one(0.0, 0.75 * scale), one(2.0 ** -90, 0.0)
    for first, last in ((0, 32), (0, 256), (0, 512), (32, 64), (512, 768), (64, 1900), (0, 1999), (0, 2000)):
        for row in (torch.zeros_like(constant), constant, noise):
            v4.copy_(kept)
            v4[:, :, first:last] = row
            held = [q4_util.unpack(c, W) for c, W in ((k4, 2 * w.n_pairs), (v4, w.n_vch))]
            for n_split in (0, 1):
                out = _run_attn(st, w, q, k4, v4, dl, n_split)
                _ok(st)
                want = np.concatenate([O.decode_attn_q4(util.to_np64(q)[b:b + 1], *(tuple(a[b:b + 1] for a in h) for h in held), [n], w.head_dim)
                                       for b, n in enumerate(lens)])
                # (steps as small as the noise's: a row's weight is cut at 2^-97 of the largest exponential)
                tol = q4_util.attn_bound(util.to_np64(q), held[0], held[1], lens, w.head_dim) + max(lens) * 7.5 * 2.0 ** -97
                assert np.all(np.abs(util.to_np64(out) - want) <= tol), (first, last, n_split)
    st.close()


@pytest.mark.parametrize("G", [1, 4, 5, 8])
@pytest.mark.parametrize("bits,step", [(130, 2.0 ** 66), (130, 2.0 ** 120), (40, 2.0 ** 66), (180, 2.0 ** 100)])
def test_attention_steps_that_count_far_below_the_largest_logit(G, bits, step):
    """Zero rows with the largest logits and, in their block, rows `bits` binary places below with steps so large that their weight
    times step counts (2^-130 relative to the largest is no fp32 number): they make the output, or nearly nothing of it."""
    n = 96
    w = _small(n_pairs=16, n_vch=48, n_q_heads=G, n_kv_heads=1)
    st = DecodeStack(w, s_cap=n, alloc_cache=False)
    st.build_tables(*synth.draw_scores(w))
    rng = np.random.default_rng(7)
    k_codes, v_codes = np.zeros((1, 1, n, 32), dtype=np.uint8), rng.integers(0, 16, (1, 1, n, 48)).astype(np.uint8)
    k_codes[..., 0] = 15
    low = np.arange(n) % 7 == 3
    k_codes[:, :, low, 0] = 0
    one = np.ones((1, 1, n))
    held = [(k_codes, one, 0 * one), (v_codes, np.where(low, step, 0.0) * one, 0 * one)]
    k4, v4 = (torch.from_numpy(q4_util.pack(*h)).to(st.device) for h in held)
    q = torch.zeros((1, G, 32), dtype=st.dt, device=st.device)
    q[:, :, 0] = bits * float(np.sqrt(w.head_dim) * np.log(2)) / 15
    want = O.decode_attn_q4(util.to_np64(q), held[0], held[1], [n], w.head_dim)
    # (a product of weight and step is cut at 2^-97 of the largest weight, a sum of weights at 2^-149)
    tol = q4_util.attn_bound(util.to_np64(q), held[0], held[1], [n], w.head_dim) + n * 7.5 * 2.0 ** -97
    for n_split in (0, 1):
        out = util.to_np64(_run_attn(st, w, q, k4, v4, torch.tensor([n], dtype=torch.int32, device=st.device), n_split))
        _ok(st)
        assert np.all(np.abs(out - want) <= tol), (np.abs(out - want).max(), np.abs(want).max())
    st.close()


def test_attention_fp32_and_wide_heads():
    _attn_case(replace(synth.TINY, batch=2, seq=200), [200, 77], seed=2)
    _attn_case(replace(synth.TINY, batch=2, seq=200), [200, 77], 3, seed=3)
    w = _small(batch=2, head_dim=256, n_pairs=90, n_vch=179, n_q_heads=4, n_kv_heads=2)
    _attn_case(w, [500, 65], seed=4)


@pytest.mark.parametrize("variant", [0, 1])
@pytest.mark.parametrize("where", ["k", "v"])
def test_a_nan_row_reaches_its_own_heads_only(variant, where):
    lens = [900, 400]
    w = _small(batch=2)
    st, q, k4, v4, dl = _attn_stack(w, lens, seed=6)
    st.ctx.rap_set_attn_variant(variant)
    clean = _run_attn(st, w, q, k4, v4, dl)
    (k4 if where == "k" else v4)[1, 3, 222] = 0xFF
    out = _run_attn(st, w, q, k4, v4, dl)
    _ok(st)
    hit = torch.zeros((2, w.n_q_heads), dtype=torch.bool, device=st.device)
    hit[1, 3 * w.group: 4 * w.group] = True
    assert torch.isnan(out[hit]).all()
    assert torch.equal(out[~hit], clean[~hit])
    st.close()


def test_attention_offsets_past_32_bits():
    """A cache of more than 2^32 bytes whose last sequence alone is in use."""
    w = _small(batch=32)
    st = DecodeStack(w, s_cap=330000, alloc_cache=False)
    st.build_tables(*synth.draw_scores(w))
    k4, v4 = q4_util.caches(st, 0)
    assert k4.numel() > 2 ** 32
    n = 1500
    g = torch.Generator(device=st.device).manual_seed(2)
    for cache, W in ((k4, 2 * w.n_pairs), (v4, w.n_vch)):
        x = torch.randn((w.n_kv_heads, n, W), generator=g, device=st.device)
        packed = torch.empty((w.n_kv_heads, n, cache.shape[-1]), dtype=torch.uint8, device=st.device)
        st.ctx.rap_quantize_rows_q4(binding.RAP_F32, w.n_kv_heads * n, W, x, packed)
        cache[31, :, :n] = packed
    q = torch.randn((32, w.n_q_heads, 2 * w.n_pairs), generator=g, device=st.device).to(st.dt)
    lens = [0] * 31 + [n]
    dl = torch.tensor(lens, dtype=torch.int32, device=st.device)
    out = _run_attn(st, w, q, k4, v4, dl)
    _ok(st)
    assert not out[:31].any()
    one = lambda c, W: q4_util.unpack(c[31:, :, :n].contiguous(), W)
    q4_util.check_attn(util.to_np64(out[31:]), util.to_np64(q[31:]), one(k4, 2 * w.n_pairs), one(v4, w.n_vch), [n], w.head_dim)
    st.close()


def test_attention_repeats_bit_for_bit_on_one_split_and_on_a_side_stream():
    w = _small(batch=5)
    st, q, k4, v4, dl = _attn_stack(w, [3000, 5, 0, 911, 64], seed=3)
    first = _run_attn(st, w, q, k4, v4, dl)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = [_run_attn(st, w, q, k4, v4, dl) for _ in range(5)]
    torch.cuda.current_stream().wait_stream(side)
    _ok(st)
    assert all(torch.equal(first, a) for a in again)
    st.close()


def test_attention_captured_and_replayed():
    """Two graphs on one context, replayed in turns, with lengths that change between replays (within the bound)."""
    w = _small(batch=3)
    lens = [2000, 700, 0]
    st, q, k4, v4, dl = _attn_stack(w, [2000, 2000, 2000], seed=4)
    dl.copy_(torch.tensor(lens, dtype=torch.int32))
    outs = [torch.zeros((3, w.n_q_heads, w.n_vch), dtype=torch.float32, device=st.device) for _ in range(2)]
    _run_attn(st, w, q, k4, v4, dl, bound=2000)
    torch.cuda.synchronize()
    graphs = []
    for o in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            st.ctx.rap_decode_attn_q4(0, 3, q, k4, v4, st.s_cap, dl, 2000, 0, o)
        graphs.append(g)
    held = [q4_util.unpack(c, W) for c, W in ((k4, 2 * w.n_pairs), (v4, w.n_vch))]
    for lens in ([2000, 700, 0], [1, 0, 1999], [64, 64, 64]):
        dl.copy_(torch.tensor(lens, dtype=torch.int32))
        for i in (0, 1, 0, 0):
            outs[i].fill_(float("nan"))
            graphs[i].replay()
            torch.cuda.synchronize()
            q4_util.check_attn(util.to_np64(outs[i]), util.to_np64(q), held[0], held[1], lens, w.head_dim)
    assert st.ctx.rap_get_last_device_status() == (0, 0)
    del graphs
    st.close()


@pytest.mark.parametrize("G", [3, 8])
def test_attention_large_q_on_small_rows_and_an_infinity_in_q(G):
    w = _small(batch=2, n_q_heads=2 * G, n_kv_heads=2)
    lens = [400, 35]
    st, q, k4, v4, dl = _attn_stack(w, lens, seed=10, gain=1e33)
    g = torch.Generator(device=st.device).manual_seed(3)
    x = torch.randn((2, w.n_kv_heads, st.s_cap, 2 * w.n_pairs), generator=g, device=st.device) * 1e-33
    st.ctx.rap_quantize_rows_q4(binding.RAP_F32, x.numel() // x.shape[-1], x.shape[-1], x, k4)
    held = [q4_util.unpack(c, W) for c, W in ((k4, 2 * w.n_pairs), (v4, w.n_vch))]
    out = _run_attn(st, w, q, k4, v4, dl)
    _ok(st)
    q4_util.check_attn(util.to_np64(out), util.to_np64(q), held[0], held[1], lens, w.head_dim)
    for value in (float("inf"), float("-inf"), float("nan")):
        q2 = q.clone()
        q2[0, G + 1, 5] = value
        got = _run_attn(st, w, q2, k4, v4, dl)
        _ok(st)
        assert torch.isnan(got[0, G + 1]).all()
        got[0, G + 1] = out[0, G + 1]
        q4_util.check_attn(util.to_np64(got), util.to_np64(q), held[0], held[1], lens, w.head_dim)
    st.close()


@pytest.mark.parametrize("G", [1, 4, 5])
def test_attention_one_cta_over_a_long_sequence_of_the_largest_codes(G):
    """140,000 rows on one CTA: 547 blocks a warp, past what one filling of the accumulators may hold.  The first tiles' rows weigh
    2^-3.9 of the others, so that the weights stay just below the size at which the reference is raised.  All rows have the same V, so
    the outputs are its numbers."""
    n, dv = 140000, 64
    w = _small(n_pairs=16, n_vch=dv, n_q_heads=G, n_kv_heads=1)
    st = DecodeStack(w, s_cap=n, alloc_cache=False)
    st.build_tables(*synth.draw_scores(w))
    codes = np.zeros((1, 1, n, 32), dtype=np.uint8)
    codes[:, :, 2048:, 0] = 15
    one = np.ones((1, 1, n))
    v_codes = np.where(np.arange(dv) < 40, 15, np.arange(dv) % 16).astype(np.uint8) * np.ones((1, 1, n, 1), dtype=np.uint8)
    k4, v4 = (torch.from_numpy(q4_util.pack(c, one, 0 * one)).to(st.device) for c in (codes, v_codes))
    q = torch.zeros((1, G, 32), dtype=st.dt, device=st.device)
    q[:, :, 0] = 3.9 * float(np.sqrt(w.head_dim) * np.log(2)) / 15
    out = util.to_np64(_run_attn(st, w, q, k4, v4, torch.tensor([n], dtype=torch.int32, device=st.device), 1))
    _ok(st)
    # the codes' sums are exact (G <= 4) or rounded once per 16 blocks; the row sums, fp32, take 4 * 547 additions a lane
    want = v_codes[0, 0, 0] - 7.5
    assert np.all(np.abs(out[0] - want) <= 2.0 ** -24 * (4 * 547 + 600) * np.abs(want).max())
    st.close()


@pytest.mark.parametrize("G", [1, 4, 5])
def test_attention_one_large_weight_over_a_long_flat_tail(G):
    """One row outweighs each of 60,000 equal ones by 2^25.5 or so: what a narrow weight loses of each must not add up."""
    n = 60000
    w = _small(n_pairs=16, n_vch=48, n_q_heads=G, n_kv_heads=1)
    st = DecodeStack(w, s_cap=n, alloc_cache=False)
    st.build_tables(*synth.draw_scores(w))
    k_codes, v_codes = np.zeros((1, 1, n, 32), dtype=np.uint8), np.full((1, 1, n, 48), 15, dtype=np.uint8)
    k_codes[:, :, 5] = 15
    v_codes[:, :, 5] = 0
    one = np.ones((1, 1, n))
    held = [(c, one, 0 * one) for c in (k_codes, v_codes)]
    k4, v4 = (torch.from_numpy(q4_util.pack(*h)).to(st.device) for h in held)
    q = torch.zeros((1, G, 32), dtype=st.dt, device=st.device)
    q[:, :, 0] = torch.tensor([25.3 + 0.1 * g for g in range(G)]) * float(np.sqrt(w.head_dim) * np.log(2)) / 15
    want = O.decode_attn_q4(util.to_np64(q), held[0], held[1], [n], w.head_dim)
    for n_split in (0, 1):
        out = util.to_np64(_run_attn(st, w, q, k4, v4, torch.tensor([n], dtype=torch.int32, device=st.device), n_split))
        _ok(st)
        # The logits, up to 26 / log2(e), may be off by 2^-22 of that.  The row sums, fp32, take 30 or so additions of eight blocks each
        # and one per row among eight blocks: 40 times 2^-24.
        # G <= 4: a weight's fraction counts up to 2^-27 of the largest weight and is cut at points that follow the golden section: of a
        # lane's N equal weights per row of a block at most 2 + log2 N too many or too few are cut up; 8 lanes x 4 rows x 8 warps hold
        # N <= 235 each.  (Cut alike, the tail would be off by up to 60000 2^-28 = 2.2e-4.)
        # G > 4: fp16 ends 2^-33 below the largest weight, 60000 times half of that; the splitting's 2^-19 of the tail; and the MMAs
        # cut their running sums off: those of 16 blocks, 64 MMAs, by 2^-23 of at most 15 (the large row, complemented), and 7.5 times
        # the sum of the weights by as much of 7.5.  (Later ones start from nothing.)
        tail = (n - 1) * 2.0 ** -25.2
        tol = 7.5 * (2 * tail * (26 * 2.0 ** -22 + 2.0 ** -19) + 40 * 2.0 ** -24 + 2.0 ** -20)
        tol += 7.5 * 256 * 10 * 2.0 ** -27 if G <= 4 else 7.5 * n * 2.0 ** -34 + 64 * 2.0 ** -23 * (15 + 7.5)
        assert np.all(np.abs(out - want) <= tol), (np.abs(out - want).max(), tol)
    st.close()


def test_attention_of_twenty_thousand_sequences():
    """More than the plan in shared memory holds: sequences of every length 0 .. 49, the same fifty again and again."""
    B, w = 20000, _small(n_q_heads=8, n_kv_heads=2)
    lens = list(range(50))
    st, q, k4, v4, dl = _attn_stack(replace(w, batch=50), lens, seed=12, s_cap=56)
    small = _run_attn(st, w, q, k4, v4, dl)
    _ok(st)
    held = [q4_util.unpack(c, W) for c, W in ((k4, 2 * w.n_pairs), (v4, w.n_vch))]
    q4_util.check_attn(util.to_np64(small), util.to_np64(q), held[0], held[1], lens, w.head_dim)
    st.close()
    big = DecodeStack(replace(w, batch=B), s_cap=56, alloc_cache=False)
    big.build_tables(*synth.draw_scores(w))
    out = _run_attn(big, w, q.repeat(B // 50, 1, 1), k4.repeat(B // 50, 1, 1, 1), v4.repeat(B // 50, 1, 1, 1), dl.repeat(B // 50), bound=49)
    _ok(big)
    assert torch.equal(out, small.repeat(B // 50, 1, 1))
    big.close()


def test_read_cache_of_many_sequences():
    """More sequences than one plan of the read-back covers."""
    B, S = 2500, 24
    w = _small(batch=B, n_q_heads=2, n_kv_heads=1, n_pairs=3, n_vch=5)
    st = DecodeStack(w, s_cap=S)
    st.build_tables(*synth.draw_scores(w))
    k4, v4 = q4_util.caches(st, 0)
    g = torch.Generator(device=st.device).manual_seed(2)
    dl = torch.randint(0, S + 1, (B,), generator=g, device=st.device, dtype=torch.int32)
    dl[100:1400] = 0
    used = (torch.arange(S, device=st.device)[None, :] < dl[:, None])[:, None, :, None]
    want = []
    for packed, W, cache in ((k4, 6, st.k_cache[0]), (v4, 5, st.v_cache[0])):
        x = torch.randn(packed.shape[:3] + (W,), generator=g, device=st.device)
        st.ctx.rap_quantize_rows_q4(binding.RAP_F32, B * S, W, x, packed)
        back = torch.empty(x.shape, dtype=st.dt, device=st.device)
        st.ctx.rap_dequantize_rows_q4(_kind(w.dtype), B * S, W, packed, back)
        cache.fill_(7.0)
        want.append(torch.where(used, back, torch.full_like(back, 7.0)))
    st.ctx.rap_read_cache_q4(0, B, k4, v4, S, dl, S, st.k_cache[0], st.v_cache[0])
    _ok(st)
    assert torch.equal(st.k_cache[0], want[0]) and torch.equal(st.v_cache[0], want[1])
    st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_read_cache_at_every_width_of_long_calls(dtype):
    """Rows of every width up to 256, K as wide as V or narrower, with enough rows for the longest chunks: whatever the width,
    what a chunk takes of shared memory has to fit beside the plan."""
    lens, S = [640, 639, 0, 300], 640
    for W in list(range(57, 81)) + list(range(113, 257)) if dtype == "bf16" else list(range(33, 90)) + list(range(90, 257, 9)):
        w = replace(_small(batch=4), head_dim=256, dtype=dtype, n_q_heads=8, n_kv_heads=8, n_pairs=W // 2 if W % 3 else 5, n_vch=W)
        st = DecodeStack(w, s_cap=S)
        st.build_tables(*synth.draw_scores(w))
        g = torch.Generator(device=st.device).manual_seed(W)
        used = (torch.arange(S, device=st.device)[None, :] < torch.tensor(lens, device=st.device)[:, None])[:, None, :, None]
        held, want = q4_util.caches(st, 0), []
        for packed, width, cache in zip(held, (2 * w.n_pairs, W), (st.k_cache[0], st.v_cache[0])):
            x = torch.randn(packed.shape[:3] + (width,), generator=g, device=st.device)
            st.ctx.rap_quantize_rows_q4(binding.RAP_F32, 4 * 8 * S, width, x, packed)
            back = torch.empty(x.shape, dtype=st.dt, device=st.device)
            st.ctx.rap_dequantize_rows_q4(_kind(dtype), 4 * 8 * S, width, packed, back)
            cache.fill_(7.0)
            want.append(torch.where(used, back, torch.full_like(back, 7.0)))
        dl = torch.tensor(lens, dtype=torch.int32, device=st.device)
        st.ctx.rap_read_cache_q4(0, 4, held[0], held[1], S, dl, S, st.k_cache[0], st.v_cache[0])
        _ok(st)
        assert torch.equal(st.k_cache[0], want[0]) and torch.equal(st.v_cache[0], want[1]), W
        st.close()


def test_two_contexts_on_two_streams():
    cases = [_attn_stack(_small(batch=3), [3000, 911, 64], seed=s) for s in (20, 21)]
    w = _small(batch=3)
    alone = [_run_attn(st, w, q, k4, v4, dl) for st, q, k4, v4, dl in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [[], []]
    for _ in range(6):
        for i, (st, q, k4, v4, dl) in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                outs[i].append(_run_attn(st, w, q, k4, v4, dl, bound=3000))
    torch.cuda.synchronize()
    for i, (st, *_rest) in enumerate(cases):
        assert all(torch.equal(alone[i], o) for o in outs[i])
        assert st.ctx.rap_get_last_device_status() == (0, 0)
        st.close()


def test_a_wait_that_runs_out_is_reported_and_the_next_launch_is_right():
    w = _small(batch=5)
    lens = [900, 5, 0, 411, 64]
    st, q, k4, v4, dl = _attn_stack(w, lens, seed=13)
    want = _run_attn(st, w, q, k4, v4, dl)
    _ok(st)
    st.ctx.rap_debug_arm_wait_timeout()
    got = _run_attn(st, w, q, k4, v4, dl)                  # returns: the wait is bounded
    torch.cuda.synchronize()
    assert torch.isnan(got[0, : w.group]).all()            # the first unit was never finished
    done = ~torch.isnan(got).any(-1)
    assert int((~done).sum()) <= 2 * w.group and torch.equal(got[done], want[done])
    for _ in range(2):
        assert torch.equal(_run_attn(st, w, q, k4, v4, dl), want)
    torch.cuda.synchronize()
    code, _detail = st.ctx.rap_get_last_device_status()
    assert code == binding.RAP_ETIMEOUT and st.ctx.rap_get_last_device_status() == (0, 0)
    st.close()


@pytest.mark.parametrize("scan", ["q4", "bf16"])
def test_a_wait_that_runs_out_at_a_large_batch_then_a_small_one_then_the_large_one(scan):
    """What a launch that gave up leaves in the arrival counters of units beyond a following smaller batch must not reach the next
    large one.  CTA 0, which gives up, has a part of the second sequence (the first is empty); others finish theirs.  The calls' q
    differ, so that a unit merged from an older call's partials shows.  The status is read at the end (that clears the counters)."""
    w = _small(batch=40, n_kv_heads=1, n_q_heads=4)
    lens = [0] + [9000] * 39
    if scan == "q4":
        st, q, k, v, dl = _attn_stack(w, lens, seed=15)
        call = st.ctx.rap_decode_attn_q4
    else:
        st, q, _k4, _v4, dl = _attn_stack(w, lens, seed=15)
        g = torch.Generator(device=st.device).manual_seed(15)
        k, v = (torch.randn((40, 1, st.s_cap, W), generator=g, device=st.device).to(st.dt) for W in (2 * w.n_pairs, w.n_vch))
        call = st.ctx.rap_decode_attn

    def run(x, B=40):
        out = torch.full((B, w.n_q_heads, w.n_vch), float("nan"), dtype=torch.float32, device=st.device)
        call(0, B, x, k, v, st.s_cap, dl, 9000, 0, out)
        return out

    qs = [q, q.flip(0).contiguous(), (q * 0.5).contiguous()]
    want = [run(x) for x in qs]
    _ok(st)
    for first in (0, 1):                         # from either of the two sets of counters
        if first:
            run(q)
        st.ctx.rap_debug_arm_wait_timeout()
        gave_up = run(qs[0])
        assert not run(q, 1).any()
        for i in (1, 2, 0, 1, 2):
            got = run(qs[i])
            assert torch.equal(got, want[i]), i
        assert torch.isnan(gave_up[1]).all() and torch.equal(gave_up[0], want[0][0])
        assert st.ctx.rap_get_last_device_status()[0] == binding.RAP_ETIMEOUT
    st.close()


# ---- together ------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("name", ["8b", "3b", "tiny"])
def test_decode_step_equals_the_separate_calls(name):
    """rap_decode_step_q4 against rap_qkv_rope_append_q4 + rap_decode_attn_q4 per layer, bit for bit, caches and outputs;
    the lengths advance; the attention against the oracle on the device's own rows."""
    base = synth.CONFIGS[name]
    w = replace(base, batch=2, seq=300) if name == "tiny" else synth.scaled_down(base, n_layers=3, batch=2, seq=300, hidden=512)
    lens = np.array([300, 211], dtype=np.int32)
    ks, vs = synth.draw_scores(w)
    st, _, _ = util.build_small_stack(w, ks, vs, full_weights=False, max_rows=256)
    B, L = w.batch, w.n_layers
    g = torch.Generator(device=st.device).manual_seed(11)
    k4, v4 = [], []
    for l in range(L):
        pair = q4_util.caches(st, l)
        for packed, W in zip(pair, (2 * st.n_pairs[l], st.n_vch[l])):
            x = torch.empty(packed.shape[:3] + (W,), device=st.device).normal_(0, 1, generator=g)
            st.ctx.rap_quantize_rows_q4(binding.RAP_F32, x.numel() // W, W, x, packed)
        k4.append(pair[0])
        v4.append(pair[1])
    k4_ref, v4_ref = [t.clone() for t in k4], [t.clone() for t in v4]
    x = torch.empty((L, B, w.hidden), device=st.device).normal_(0, 1, generator=g).to(st.dt)
    st.seq_len.copy_(torch.from_numpy(lens))
    for step in range(2):
        dl = torch.from_numpy(lens + step).to(st.device)
        sid = torch.arange(B, dtype=torch.int32, device=st.device)
        want = []
        for l in range(L):
            q = torch.empty((B, w.n_q_heads, 2 * st.n_pairs[l]), dtype=st.dt, device=st.device)
            st.ctx.rap_qkv_rope_append_q4(l, B, x[l], st.w_qkv[l], None, sid, dl, dl, int(lens.max()) + step, st.inv_freq, q, k4_ref[l],
                                          v4_ref[l], B, st.s_cap)
            o = torch.empty((B, w.n_q_heads, st.n_vch[l]), dtype=torch.float32, device=st.device)
            st.ctx.rap_decode_attn_q4(l, B, q, k4_ref[l], v4_ref[l], st.s_cap, dl + 1, int(lens.max()) + step + 1, 0, o)
            want.append((q, o))
        st.out.fill_(float("nan"))
        st.ctx.rap_decode_step_q4(B, x, st.w_qkv, None, st.inv_freq, k4, v4, st.s_cap, st.seq_len, int(lens.max()) + step, 0,
                                  st.q_scratch, st.out, st.out_stride, 1)
        _ok(st)
        assert np.array_equal(st.seq_len.cpu().numpy(), lens + step + 1)
        for l in range(L):
            assert torch.equal(k4[l], k4_ref[l]) and torch.equal(v4[l], v4_ref[l])
            assert torch.equal(st.out[l][: want[l][1].numel()].view_as(want[l][1]), want[l][1])
    l = L - 1
    held = [q4_util.unpack(c, W) for c, W in ((k4[l], 2 * st.n_pairs[l]), (v4[l], st.n_vch[l]))]
    q4_util.check_attn(util.to_np64(want[l][1]), util.to_np64(want[l][0]), held[0], held[1], lens + 2, w.head_dim,
                       1 if w.dtype == "f32" else 16)
    st.close()


@pytest.mark.parametrize("name", ["8b", "tiny"])
def test_decode_steps_back_to_back_and_replayed(name):
    """Six steps that advance the lengths, each waited for; the same six enqueued back to back; and one captured step replayed six
    times: caches, lengths and the last outputs are equal bit for bit (a position read too early would be the step before's)."""
    base = synth.CONFIGS[name]
    w = replace(base, batch=3, seq=120) if name == "tiny" else synth.scaled_down(base, n_layers=3, batch=3, seq=120, hidden=512)
    st, _, _ = util.build_small_stack(w, *synth.draw_scores(w), full_weights=False, max_rows=64)
    L = w.n_layers
    g = torch.Generator(device=st.device).manual_seed(5)
    start = []
    for l in range(L):
        pair = q4_util.caches(st, l)
        for packed, W in zip(pair, (2 * st.n_pairs[l], st.n_vch[l])):
            x = torch.empty(packed.shape[:3] + (W,), device=st.device).normal_(0, 1, generator=g)
            st.ctx.rap_quantize_rows_q4(binding.RAP_F32, x.numel() // W, W, x, packed)
        start.append(pair)
    lens = torch.tensor([120, 0, 57], dtype=torch.int32, device=st.device)
    x = torch.empty((L, w.batch, w.hidden), device=st.device).normal_(0, 1, generator=g).to(st.dt)

    def case():
        return [p[0].clone() for p in start], [p[1].clone() for p in start], lens.clone(), torch.zeros_like(st.out)

    def step(k4, v4, dl, out):
        st.ctx.rap_decode_step_q4(w.batch, x, st.w_qkv, None, st.inv_freq, k4, v4, st.s_cap, dl, 126, 0, st.q_scratch, out, st.out_stride, 1)

    ran = []
    for wait in (True, False):
        c = case()
        torch.cuda.synchronize()
        for _ in range(6):
            step(*c)
            if wait:
                torch.cuda.synchronize()
        _ok(st)
        ran.append(c)
    c = case()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*c)
    for _ in range(6):
        graph.replay()
    _ok(st)
    ran.append(c)
    assert torch.equal(ran[0][2], lens + 6)
    for other in ran[1:]:
        assert torch.equal(other[2], ran[0][2]) and torch.equal(other[3], ran[0][3])
        assert all(torch.equal(a, b) for i in (0, 1) for a, b in zip(other[i], ran[0][i]))
    del graph
    st.close()


def test_prompt_chunk_behind_a_quantised_prefix_then_decode():
    """As a server uses them: a prompt's first part appended in 4 bits, the rows read back, the second part attended over
    them by rap_prefill_attn, appended in 4 bits too, then a decode step of the attention over everything."""
    w = synth.scaled_down(synth.LLAMA_8B, n_layers=1, batch=2, seq=400, hidden=512)
    ks, vs = synth.draw_scores(w)
    st, tabs, w_host = util.build_small_stack(w, ks, vs, s_cap=448, max_rows=512)
    B, T1, T2, P, dv = 2, 250, 128, w.n_pairs, w.n_vch
    k4, v4 = q4_util.caches(st, 0)

    def append(first, count, seed):
        sid = torch.arange(B, dtype=torch.int32, device=st.device).repeat_interleave(count)
        pos = torch.arange(first, first + count, dtype=torch.int32, device=st.device).repeat(B)
        x = torch.from_numpy(synth.draw_hidden(w, 0, seed, B * count)).to(st.device).to(st.dt)
        q = torch.empty((B * count, w.n_q_heads, 2 * P), dtype=st.dt, device=st.device)
        st.ctx.rap_qkv_rope_append_q4(0, B * count, x, st.w_qkv[0], None, sid, pos, pos, first + count - 1, st.inv_freq, q, k4, v4, B,
                                      st.s_cap)
        return q

    append(0, T1, 1)
    q = append(T1, T2, 2)
    dl = torch.full((B,), T1 + T2, dtype=torch.int32, device=st.device)
    start = torch.full((B,), T1, dtype=torch.int32, device=st.device)
    st.ctx.rap_read_cache_q4(0, B, k4, v4, st.s_cap, dl, T1 + T2, st.k_cache[0], st.v_cache[0])
    out = torch.empty((B, T2, w.n_q_heads, dv), dtype=torch.float32, device=st.device)
    st.ctx.rap_prefill_attn(0, B, T2, q, st.k_cache[0], st.v_cache[0], st.s_cap, start, T1, out)
    _ok(st)
    held = [q4_util.unpack(c, W) for c, W in ((k4, 2 * P), (v4, dv))]
    K, V = (O.round_bf16(O.dequantize_rows_q4(*h)) for h in held)
    want = O.prefill_attn(util.to_np64(q).reshape(B, T2, w.n_q_heads, 2 * P), K, V, np.full(B, T1), w.head_dim)
    util.check_attn(util.to_np64(out), want, "bf16")
    q1 = append(T1 + T2, 1, 3)
    o1 = _run_attn(st, w, q1, k4, v4, dl + 1)
    _ok(st)
    held = [q4_util.unpack(c, W) for c, W in ((k4, 2 * P), (v4, dv))]
    q4_util.check_attn(util.to_np64(o1), util.to_np64(q1), held[0], held[1], [T1 + T2 + 1] * B, w.head_dim)
    st.close()


def test_refusals():
    w = synth.scaled_down(synth.LLAMA_8B, n_layers=1, batch=2, seq=16, hidden=256)
    ks, vs = synth.draw_scores(w)
    st, _, _ = util.build_small_stack(w, ks, vs, s_cap=16, max_rows=8)
    k4, v4 = q4_util.caches(st, 0)
    dl = torch.tensor([3, 4], dtype=torch.int32, device=st.device)
    q = torch.zeros((2, w.n_q_heads, 2 * w.n_pairs), dtype=st.dt, device=st.device)
    out = torch.zeros((2, w.n_q_heads, w.n_vch), dtype=torch.float32, device=st.device)
    x = torch.zeros((2, w.hidden), dtype=st.dt, device=st.device)

    def refused(status, f, *a):
        with pytest.raises(binding.RapError) as e:
            f(*a)
        assert e.value.status == status

    A = st.ctx.rap_decode_attn_q4
    refused(binding.RAP_EINVAL, A, 1, 2, q, k4, v4, 16, dl, 4, 0, out)
    refused(binding.RAP_EINVAL, A, 0, 2, None, k4, v4, 16, dl, 4, 0, out)
    refused(binding.RAP_EINVAL, A, 0, 2, q, k4, v4, 16, dl, 4, -1, out)
    refused(binding.RAP_ESHAPE, A, 0, 3, q, k4, v4, 16, dl, 4, 0, out)
    refused(binding.RAP_ESHAPE, A, 0, 2, q, k4, v4, 16, dl, 4, 65, out)
    refused(binding.RAP_EALIGN, A, 0, 2, q, k4, v4, 12, dl, 4, 0, out)
    refused(binding.RAP_EALIGN, A, 0, 2, q, k4.data_ptr() + 4, v4, 16, dl, 4, 0, out)
    refused(binding.RAP_ECAPACITY, A, 0, 2, q, k4, v4, 16, dl, 17, 0, out)
    A(0, 0, q, k4, v4, 16, dl, 4, 0, out)
    R = st.ctx.rap_read_cache_q4
    refused(binding.RAP_EINVAL, R, 0, 2, k4, v4, 16, None, 4, st.k_cache[0], st.v_cache[0])
    refused(binding.RAP_EINVAL, R, -1, 2, k4, v4, 16, dl, 4, st.k_cache[0], st.v_cache[0])
    refused(binding.RAP_ESHAPE, R, 0, 3, k4, v4, 16, dl, 4, st.k_cache[0], st.v_cache[0])
    refused(binding.RAP_EALIGN, R, 0, 2, k4, v4, 12, dl, 4, st.k_cache[0], st.v_cache[0])
    refused(binding.RAP_ECAPACITY, R, 0, 2, k4, v4, 16, dl, 17, st.k_cache[0], st.v_cache[0])
    P = st.ctx.rap_qkv_rope_append_q4
    refused(binding.RAP_ESHAPE, P, 0, 9, x, st.w_qkv[0], None, dl, dl, dl, 4, st.inv_freq, q, k4, v4, 2, 16)
    refused(binding.RAP_ECAPACITY, P, 0, 2, x, st.w_qkv[0], None, dl, dl, dl, 16, st.inv_freq, q, k4, v4, 2, 16)
    refused(binding.RAP_EINVAL, P, 0, 2, x, st.w_qkv[0], None, None, dl, dl, 4, st.inv_freq, q, k4, v4, 2, 16)
    refused(binding.RAP_EALIGN, P, 0, 2, x, st.w_qkv[0], None, dl, dl, dl, 4, st.inv_freq, q, k4.data_ptr() + 8, v4, 2, 16)
    S = st.ctx.rap_decode_step_q4
    refused(binding.RAP_ECAPACITY, S, 2, x, st.w_qkv, None, st.inv_freq, [k4], [v4], 16, dl, 16, 0, st.q_scratch, st.out, st.out_stride, 0)
    refused(binding.RAP_EINVAL, S, 2, x, st.w_qkv, None, st.inv_freq, [None], [v4], 16, dl, 4, 0, st.q_scratch, st.out, st.out_stride, 0)
    refused(binding.RAP_ESHAPE, S, 2, x, st.w_qkv, None, st.inv_freq, [k4], [v4], 16, dl, 4, 0, st.q_scratch, st.out, 4, 0)
    refused(binding.RAP_ESHAPE, st.ctx.rap_quantize_rows_q4, binding.RAP_F32, 1, 257, x, k4)
    _ok(st)
    assert not k4.any() and not v4.any()
    st.close()


def test_conversions_refuse_buffers_that_overlap():
    w = synth.scaled_down(synth.LLAMA_8B, n_layers=1, batch=2, seq=16, hidden=256)
    st = DecodeStack(w, s_cap=16)
    st.build_tables(*synth.draw_scores(w))
    k4, v4 = q4_util.caches(st, 0)
    dl = torch.tensor([3, 4], dtype=torch.int32, device=st.device)
    K, V = st.k_cache[0], st.v_cache[0]
    rows = torch.randn((64, 90), device=st.device)
    for call in (lambda: st.ctx.rap_quantize_rows_q4(binding.RAP_F32, 64, 90, rows, rows),
                 lambda: st.ctx.rap_dequantize_rows_q4(binding.RAP_F32, 8, 90, rows.data_ptr() + 64, rows),
                 lambda: st.ctx.rap_read_cache_q4(0, 2, K, v4, 16, dl, 4, K, V),
                 lambda: st.ctx.rap_read_cache_q4(0, 2, k4, V, 16, dl, 4, K, V),
                 lambda: st.ctx.rap_read_cache_q4(0, 2, k4, v4, 16, dl, 4, K, K.data_ptr() + 16)):
        with pytest.raises(binding.RapError) as e:
            call()
        assert e.value.status == binding.RAP_EINVAL
    before = rows.clone()
    st.ctx.rap_read_cache_q4(0, 2, k4, k4, 16, dl, 4, K, V)          # the same source twice is no overlap
    _ok(st)
    assert torch.equal(rows, before)
    st.close()
