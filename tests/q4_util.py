"""Helpers of the 4-bit cache tests: the byte layout written down apart from the library, random caches, and the error
bound of the attention."""
import numpy as np
import torch

from oracle import rap_oracle as O
from paper_2602_02599_b200 import binding


def row_words(W):
    n = -(-(-(-W // 2) + 4) // 4)
    return n if n % 2 else n + 1


def pack(codes, steps, middles):
    """(codes [..., W], steps, middles) -> uint8 [..., row bytes]."""
    codes = np.asarray(codes, dtype=np.uint8)
    W = codes.shape[-1]
    out = np.zeros(codes.shape[:-1] + (4 * row_words(W),), dtype=np.uint8)
    for i in range(W):
        out[..., i // 2] |= codes[..., i] << (4 * (i % 2))
    for at, v in ((-4, steps), (-2, middles)):
        v = np.asarray(v)
        bits = (v.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
        bits = np.where(np.isnan(v), 0x7FFF, bits)
        out[..., at], out[..., at + 1] = bits & 0xFF, bits >> 8
    return out


def unpack(t, W):
    """uint8 [..., row bytes] (tensor or array) -> (codes, steps, middles)."""
    a = t.detach().cpu().numpy() if isinstance(t, torch.Tensor) else t
    codes = np.stack([a[..., : (W + 1) // 2] & 15, a[..., : (W + 1) // 2] >> 4], -1).reshape(a.shape[:-1] + (-1,))[..., :W]

    def number(at):
        return ((a[..., at].astype(np.uint32) | (a[..., at + 1].astype(np.uint32) << 8)) << 16).astype(np.uint32).view(np.float32).astype(np.float64)

    return codes, number(-4), number(-2)


def attn_bound(q, k_held, v_held, lens, head_dim, rows_per_add=16):
    """Elementwise bound on |kernel - fp64| of decode_attn_q4, [B][H_q][1].

    The logits are fp32 sums of at most 33 partial products groups (one per step of 16 dims, plus the split into step and
    middle), each off by at most 2^-23 of the largest intermediate sum, and an MMA may lose one more place to alignment:
    d = 2^-17 (sum |q|) max_j(|z_j| + 15 s_j) / sqrt(D) covers them (the codes run to 15, their offset of 7.5 comes off
    later).  A logit off by d moves every weight by at most e^(2 d) - 1; a weight itself is off by 2^-22 (split into two
    16-bit numbers) plus 2^-21 (the exponential and the row sum).  Adding n rows in fp32 loses at most 2^-23 of the
    running sum per addition (16 rows at a time on the tensor cores, 1 in the shape-generic kernel), and the running sum
    is at most A = sum p (|zV| + 15 sV)."""
    q = np.asarray(q, dtype=np.float64)
    B, Hq, _ = q.shape
    Hkv = k_held[0].shape[1]
    G = Hq // Hkv
    out = np.zeros((B, Hq, 1))
    for b in range(B):
        n = int(lens[b])
        for g in range(Hq if n else 0):
            h = g // G
            K = O.dequantize_rows_q4(*(a[b, h, :n] for a in k_held))
            s = K @ q[b, g] / np.sqrt(head_dim)
            p = np.exp(s - s.max())
            p /= p.sum()
            A = (p * (np.abs(v_held[2][b, h, :n]) + 15 * v_held[1][b, h, :n])).sum()
            reach = (np.abs(k_held[2][b, h, :n]) + 15 * k_held[1][b, h, :n]).max()
            d = 2.0 ** -17 * np.abs(q[b, g]).sum() * reach / np.sqrt(head_dim)
            out[b, g] = A * (np.expm1(min(2 * d, 50.0)) + 2.0 ** -20 + 2.0 ** -23 * (8 + n / rows_per_add))
    return out


def check_attn(got, q, k_held, v_held, lens, head_dim, rows_per_add=16):
    """got [B][H_q][d_v'] against the oracle on the values that the device's own rows stand for."""
    lens = [int(n) for n in lens]
    want = np.zeros(got.shape)
    for b, n in enumerate(lens):
        if n:
            one = lambda held: tuple(a[b:b + 1] for a in held)
            want[b] = O.decode_attn_q4(np.asarray(q)[b:b + 1], one(k_held), one(v_held), [n], head_dim)[0]
    tol = attn_bound(q, k_held, v_held, lens, head_dim, rows_per_add)
    err = np.abs(got - want)
    assert np.all(err <= tol), (float(err.max()), float((err / np.maximum(tol, 1e-300)).max()))
    return float(err.max())


def caches(st, l):
    """Zeroed packed caches of layer l of a stack."""
    kb, vb = binding.rap_q4_row_bytes(2 * st.n_pairs[l]), binding.rap_q4_row_bytes(st.n_vch[l])
    shape = (st.B, st.w.n_kv_heads, st.s_cap)
    return (torch.zeros(shape + (kb,), dtype=torch.uint8, device=st.device), torch.zeros(shape + (vb,), dtype=torch.uint8, device=st.device))
