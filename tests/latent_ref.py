"""Plain references of the latent-attention operators, in 64 bits and by their definitions, for the tests (CPU torch and
numpy; none of the library's code)."""
import numpy as np
import torch

import serving_ref as R

ROPE = 64
LARGEST = {torch.float16: 65504.0, torch.bfloat16: float(torch.finfo(torch.bfloat16).max)}


def code_offsets(d_c):
    """Byte of the code of (token, channel) in a block: numpy [16][d_c]."""
    t, c = np.arange(16)[:, None], np.arange(d_c)[None, :]
    return d_c * t + 128 * (c // 128) + 16 * (c % 64 // 8) + 8 * (c % 128 // 64) + c % 8


def held(x):
    """What the cache takes a 16-bit tensor's values for, float64: NaN 0, an infinity the type's largest number, magnitudes
    up to 2^64."""
    y = torch.nan_to_num(x.double(), nan=0.0, posinf=LARGEST[x.dtype], neginf=-LARGEST[x.dtype])
    return y.clamp(-2.0 ** 64, 2.0 ** 64).cpu().numpy()


class Cache:
    """Host model: codes, ranges, positional keys (their fp16 numbers) and powers of two by slot."""

    def __init__(self, n_slots, d_c):
        self.codes, self.a = np.zeros((n_slots, d_c), np.int64), np.zeros(n_slots)
        self.r, self.s = np.zeros((n_slots, ROPE), np.float16), np.ones(n_slots)
        self.d_c = d_c

    def append(self, c, r, slots):
        """c [n][d_c], r [n][64]: 16-bit tensors; slots: numpy [n], negative ones are skipped."""
        c, r = held(c), held(r)
        a = np.abs(c).max(1)
        a[a < 2.0 ** -64] = 0.0
        # numpy rounds halves to even; the quotients of exact products are themselves exact at a half
        codes = np.where(a[:, None] > 0, np.rint(127.0 * c / np.where(a > 0, a, 1.0)[:, None]), 0.0).astype(np.int64)
        top = np.abs(r).max(1)
        s = np.exp2(np.maximum(np.floor(np.log2(np.where(top > 0, top, 2.0 ** 15))) - 15, -126))
        on = slots >= 0
        at = slots[on]
        self.codes[at], self.a[at], self.r[at], self.s[at] = codes[on], a[on], (r / s[:, None]).astype(np.float16)[on], s[on]

    def values(self, slots):
        """Latents and positional keys, float64."""
        return self.codes[slots] * (self.a[slots] / 127.0)[:, None], self.r[slots].astype(np.float64) * self.s[slots][:, None]


def read_device_cache(blocks, d_c):
    """The model of a device cache's blocks (uint8 [...][blocks][bytes]), numbered like slots."""
    x = np.ascontiguousarray(blocks.cpu().numpy().reshape(-1, 16 * (d_c + 136)))
    n = len(x)
    out = Cache(16 * n, d_c)
    out.codes = x[:, code_offsets(d_c)].reshape(16 * n, d_c).astype(np.int64) - 128
    out.r = np.ascontiguousarray(x[:, 16 * d_c:16 * d_c + 2048]).view(np.float16).reshape(16 * n, ROPE)
    scales = np.ascontiguousarray(x[:, 16 * d_c + 2048:]).view(np.float32).reshape(16 * n, 2).astype(np.float64)
    out.a, out.s = scales[:, 0], scales[:, 1]
    return out


def attention(q_c, q_r, c, r, alpha):
    """The absorbed form: R.attention over keys [c | r] and values c, with its bounds' terms."""
    q = torch.cat([torch.as_tensor(q_c).double(), torch.as_tensor(q_r).double()], -1)
    return R.attention(q, np.concatenate([c, r], 1), c, alpha)


def bound(ref, weighed, p, mag, n, d_c, c, out_eps):
    """How far the absorbed form may be from its definition.  R.bound's terms hold with d_c + 64 products in a score: the
    weights are rounded to fp16 (2^-11), the scores' four further roundings (by the token's range and power of two, the
    scale, the sum of both parts) are 4 x 2^-24 of mag within its 8 spare additions; log2 of the range is off by 2^-22 at
    most and its sum with the score (|log2 a / 127| <= 71) by 71 x 2^-24, both once for the numerator and once for the
    denominator, where they nearly cancel: 2 x (2^-22 + 71 x 2^-24) x ln 2 = 2^-17.3 at the very most.  Weights times
    ranges of less than 2^-14 are rounded by 2^-25, where the largest is at least 2^8: 2^-33 of the largest p_t a_t."""
    top = np.abs(c).max() if len(c) else 0.0
    return R.bound(ref, weighed, p, mag, n, d_c + ROPE, 2.0 ** -11, top, out_eps, 2.0 ** -33) + weighed * 2.0 ** -17


def prompt_keys(k_n, k_r):
    """[n][H][d + 64] keys of the expanded form."""
    return torch.cat([k_n, k_r[:, None].expand(-1, k_n.shape[1], -1)], -1)
