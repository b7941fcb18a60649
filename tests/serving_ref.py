"""Plain references of the serving operators, in 64 bits and by their definitions, for the tests (CPU torch and numpy;
none of the library's code)."""
import math

import numpy as np
import torch


def code_offsets(d):
    """Byte of the K code of (token, channel) and of the V code in an 8-bit block: numpy [16][d] each."""
    t, c = np.arange(16)[:, None], np.arange(d)[None, :]
    k = 512 * (c // 32) + 64 * (t % 8) + 16 * (c % 32 // 8) + 8 * (t // 8) + c % 8
    v = 16 * d + 512 * (c // 32) + 64 * (c % 8) + 16 * (t % 8 // 2) + 4 * (c % 32 // 8) + 2 * (t // 8) + t % 2
    return k, v


class Cache8:
    """Host model of the 8-bit cache: codes (int) and ranges per (slot block, KV head), by the definition."""

    def __init__(self, n_blocks, H_kv, d):
        self.codes = [np.zeros((n_blocks, H_kv, 16, d), np.int64) for _ in range(2)]
        self.range = [np.zeros((n_blocks, H_kv)) for _ in range(2)]
        self.d = d

    def append(self, k, v, slots):
        """k, v: float64 [n][H][d] holding values of a 16-bit type."""
        i, n = 0, len(slots)
        while i < n:
            if slots[i] < 0:
                i += 1
                continue
            j = i + 1
            while j < n and slots[j] == slots[j - 1] + 1 and slots[j] % 16:
                j += 1
            blk, off = int(slots[i]) // 16, int(slots[i]) % 16
            for part, x in ((0, k), (1, v)):
                x = x[i:j]
                old = self.range[part][blk] if off else np.zeros_like(self.range[part][blk])
                new = np.maximum(old, np.abs(x).max((0, 2)))
                safe = np.where(new > 0, new, 1.0)
                codes = self.codes[part][blk]
                # numpy rounds halves to even; the quotients of exact products are themselves exact at a half
                codes[:, :off] = np.rint(codes[:, :off] * old[:, None, None] / safe[:, None, None]).astype(np.int64)
                codes[:, off:off + j - i] = np.rint(127.0 * x.transpose(1, 0, 2) / safe[:, None, None]).astype(np.int64)
                self.range[part][blk] = new
            i = j

    def values(self, slots):
        """K and V of the slots, float64 [n][H][d]."""
        s = np.asarray(slots)
        return [c[s // 16, :, s % 16] * (r[s // 16] / 127.0)[..., None] for c, r in zip(self.codes, self.range)]


def read_device_cache(blocks, d):
    """Codes and ranges of a device cache's blocks (uint8 [...][H][blocks][bytes] -> Cache8 numbered like slots / 16)."""
    x = blocks.cpu().numpy()
    P, H, n, _ = x.shape
    x = x.transpose(0, 2, 1, 3).reshape(P * n, H, -1)
    out = Cache8(P * n, H, d)
    for part, at in enumerate(code_offsets(d)):
        out.codes[part] = x[:, :, at].astype(np.int64) - 128
        out.range[part] = np.ascontiguousarray(x[:, :, 32 * d + 4 * part:32 * d + 4 * part + 4]).view(np.float32)[..., 0].astype(np.float64)
    return out


def slots_of(lens, new, table, page_tokens, S_cap=0):
    """Slots of the tokens lens[b] .. lens[b] + new[b] - 1 of every sequence, packed (table None: contiguous)."""
    out = []
    for b, (a, n) in enumerate(zip(lens, new)):
        for p in range(a, a + n):
            out.append(b * S_cap + p if table is None else int(table[b][p // page_tokens]) * page_tokens + p % page_tokens)
    return np.array(out, np.int64)


def attention(q, k, v, alpha, seen=None):
    """softmax(alpha q k^T) v in float64 with what the error bounds need: (out, sum p |v|, largest p, largest |alpha| sum
    |q||k|).  q [n][d], k, v [m][d]; seen [n][m] bool or None.  Rows that see nothing are zero."""
    q, k, v = (torch.as_tensor(x, dtype=torch.float64) for x in (q, k, v))
    z = alpha * (q @ k.T)
    mag = abs(alpha) * (q.abs() @ k.abs().T)
    if seen is None:
        seen = torch.ones_like(z, dtype=torch.bool)
    z = z.masked_fill(~seen, -math.inf)
    some = seen.any(1, keepdim=True)
    p = torch.where(some, torch.softmax(torch.where(some, z, 0.0), -1), 0.0).masked_fill(~seen, 0.0)
    # what a query does not see takes no part, whatever it is (0 * inf is not 0)
    vv = torch.where(torch.isfinite(v), v, 0.0)
    out = p @ vv
    bad = ~torch.isfinite(v)
    if bad.any():
        for j in torch.nonzero(bad.any(1)).flatten().tolist():
            rows = seen[:, j]
            out[rows] = out[rows] + torch.where(bad[j], v[j], 0.0)
    return out, p @ vv.abs(), p.amax(1, keepdim=True), mag.masked_fill(~seen, 0.0).amax(1, keepdim=True)


def bound(ref, weighed, p_max, mag, n, d, weight_eps, v_max, out_eps, subnormal=2.0 ** -25):
    """How far an attention output may be from the definition: weights rounded to 16 bits (relative weight_eps, or an absolute step of
    `subnormal` of the largest weight where they are subnormal), scores accumulated in fp32 over d products (relative 2^-24
    per addition; d / 16 + 8 additions deep, times 2: numerator and denominator), the fast exponential and logarithm
    (2^-21), sums over n weights in fp32 (2^-24 times their depth, n / 16 + 64 at most), then the output's own rounding."""
    rel = weight_eps + 2 * mag * (d / 16 + 8) * 2.0 ** -24 + mag * 2.0 ** -22 + 2.0 ** -20 + (n / 16 + 64) * 2.0 ** -24
    return weighed * rel + n * subnormal * p_max * v_max + ref.abs() * out_eps + 1e-37
