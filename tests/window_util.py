"""Attention with a window and sinks, over shared prefixes, and slot maps, stated plainly in 64 bits for the tests."""
import math

import numpy as np
import torch

from paper_2602_02599_b200 import binding


def slot(p, n_sink, s_cap):
    """The cache row of position p."""
    return p if p < n_sink else n_sink + (p - n_sink) % (s_cap - n_sink)


def seen(i, n_sink, window):
    """The positions that a query at position i sees, in order."""
    return [j for j in range(min(n_sink, i + 1))] + list(range(max(n_sink, i - window + 1), i + 1))


def slots(past, new, base, n_sink, s_cap):
    """(row_start, seq_id, pos, slot, len_out) of a ragged batch."""
    start, seq, pos, at = [0], [], [], []
    for b, (n, m) in enumerate(zip(past, new)):
        for p in range(n, n + m):
            later = p >= n_sink and p + s_cap - n_sink < n + m       # a later token of the call takes the row
            seq.append(b)
            pos.append(p + (base[b] if base else 0))
            at.append(-1 if later else slot(p, n_sink, s_cap))
        start.append(len(seq))
    return [np.array(x, dtype=np.int32) for x in (start, seq, pos, at, [n + m for n, m in zip(past, new)])]


def attend(q, k, v, head_dim):
    """fp64 q [G][W], k [n][W], v [n][dv] -> (output, bound): softmax(q k / sqrt(D)) v and how far an fp32 evaluation may be
    off, by its roundings.  A logit (base 2) sums W exact products of bf16 numbers, or rounded ones of fp32, with an error
    of at most W 2^-23 times the sum of their magnitudes (2^-24 a step, twice that where the adder truncates); taking off the
    maximum and the exponential add 2^-22 and 2^-24 of the largest exponent; a weight is rounded to two bf16 numbers, 2^-17
    of itself; each of the two sums over n rows adds n 2^-24 of its terms' magnitudes; merging and dividing 2^-21."""
    n, w = k.shape
    if n == 0:
        z = torch.zeros((q.shape[0], v.shape[1]), dtype=torch.float64, device=q.device)
        return z, z
    s = q @ k.T / math.sqrt(head_dim)
    p = torch.softmax(s, -1)
    size = (q.abs() @ k.abs().T).amax(-1, keepdim=True) / math.sqrt(head_dim) * math.log2(math.e)
    spread = (s.amax(-1, keepdim=True) - s.amin(-1, keepdim=True)) * math.log2(math.e)
    off = 2 * (math.log(2) * (w * size * 2.0 ** -23 + spread * 2.0 ** -24) + 2.0 ** -22) + 2.0 ** -17 + 2 * n * 2.0 ** -24 + 2.0 ** -21
    return p @ v, off * (p @ v.abs())


REL_L2 = 1e-5      # of a whole output: the roundings above are independent, rms 2.4e-6 (weights) and below (the rest), so a quarter of this


def check(got, want, bound):
    got = got.double()
    assert torch.isfinite(got).all()
    off = (got - want).abs()
    assert (off <= bound + 1e-30).all(), f"{int((off > bound + 1e-30).sum())} entries off, worst {float((off / (bound + 1e-30)).max()):.3g} of the bound"
    norm = float(want.norm())
    rel = float((got - want).norm()) / norm if norm else float((got - want).norm())
    assert rel <= REL_L2, f"rel-L2 {rel:.3e}"
    return rel


class Heads:
    """A context for one head shape, and caches of random rows."""

    def __init__(self, kv_heads, group, pairs, vch, dtype, batch, head_dim=128, device="cuda:0", hidden=64, max_rows=1):
        self.kv, self.group, self.w, self.dv, self.head_dim = kv_heads, group, 2 * pairs, vch, head_dim
        self.device, self.batch = torch.device(device), batch
        self.dt = torch.float32 if dtype == "f32" else torch.bfloat16
        torch.cuda.set_device(self.device)
        self.ctx = binding.RapContext(1, hidden, kv_heads * group, kv_heads, head_dim, 10000.0, binding.RAP_PAIR_HALF,
                                      binding.RAP_F32 if dtype == "f32" else binding.RAP_BF16, batch, max_rows)
        r = np.random.RandomState(0)
        self.tables = [torch.empty((1, kv_heads, n), dtype=t, device=self.device) for n, t in
                       ((head_dim // 2, torch.int32), (head_dim, torch.int32), (head_dim, torch.int32), (head_dim // 2, torch.float64))]
        self.ctx.rap_build_tables(r.rand(1, kv_heads, head_dim // 2), r.rand(1, kv_heads, head_dim), [pairs], [vch], *self.tables)
        self.g = torch.Generator(device=self.device).manual_seed(pairs * 1000 + vch * 10 + group)

    def randn(self, *shape, scale=1.0):
        return (torch.randn(shape, generator=self.g, device=self.device) * scale).to(self.dt)

    def ints(self, values):
        return torch.tensor(list(values), dtype=torch.int32, device=self.device)

    def out(self, rows, fill=math.nan):
        return torch.full((rows, self.kv * self.group, self.dv), fill, dtype=torch.float32, device=self.device)

    def caches(self, rows, s_cap):
        """K and V of NaN, to be written where something is seen: [rows][H_kv][s_cap][..]."""
        return [torch.full((rows, self.kv, s_cap, n), math.nan, dtype=self.dt, device=self.device) for n in (self.w, self.dv)]

    def fill(self, cache, b, rows):
        rows = torch.as_tensor(sorted(set(rows)), device=self.device, dtype=torch.long)
        if len(rows):
            cache[b, :, rows] = self.randn(self.kv, len(rows), cache.shape[-1])

    def query(self, rows):
        return self.randn(rows, self.kv * self.group, self.w, scale=1.5)

    def reference(self, q, parts):
        """One token: q [H_q][W]; parts: (cache K, cache V, b, rows) one behind the other."""
        outs, bounds = [], []
        for h in range(self.kv):
            at = [torch.as_tensor(rows, device=self.device, dtype=torch.long) for _, _, _, rows in parts]
            k = torch.cat([K[b, h][r].double() for (K, _, b, _), r in zip(parts, at)])
            v = torch.cat([V[b, h][r].double() for (_, V, b, _), r in zip(parts, at)])
            o, e = attend(q[h * self.group: (h + 1) * self.group].double(), k, v, self.head_dim)
            outs.append(o)
            bounds.append(e)
        return torch.cat(outs), torch.cat(bounds)

    def clean(self):
        assert self.ctx.rap_get_last_device_status() == (binding.RAP_OK, 0)

    def close(self):
        self.ctx.close()
