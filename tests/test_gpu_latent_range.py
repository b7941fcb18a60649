"""Latent decode of tokens whose ranges lie as far apart as the cache holds them, from 2^-64 to 2^64: a token of small range takes no
part in the output, but its weight is in the sum that the output is divided by."""
import numpy as np
import pytest

import latent_ref as L
import serving_ref as R
from test_gpu_latent import _cache, _dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2604_16957_b200 import tq
    assert torch.cuda.is_available()
    return tq, torch


def _check_wide(torch, out, q_c, q_r, model, slots, alpha):
    """As _check_decode, with 2^-33 of the largest contribution p_t a_t instead of the largest weight by the largest value."""
    c, r = model.values(slots)
    ref, weighed, p, mag = L.attention(q_c.double().cpu(), q_r.double().cpu(), c, r, alpha)
    z = alpha * torch.cat([q_c, q_r], -1).double().cpu() @ torch.as_tensor(np.concatenate([c, r], 1)).T
    most = (torch.softmax(z, -1) * torch.as_tensor(model.a[slots])).amax(1, keepdim=True)
    tol = L.bound(ref, weighed, 0 * p, mag, len(slots), c.shape[1], c[:0], 0.0) + len(slots) * 2.0 ** -33 * most
    err = (out.double().cpu() - ref).abs()
    assert torch.all(err <= tol), float((err / tol).max())


def _filled(tq, torch, x, lens, d_c):
    """A contiguous cache of the rows x [sum of lens][d_c + 64] (float64), appended as bf16, with its model and slots by sequence."""
    x = torch.from_numpy(x).bfloat16().cuda()
    cap = -(-max(lens) // 16) * 16
    cache, _ = _cache(tq, torch, len(lens), d_c, 0, cap, 0)
    slots = R.slots_of([0] * len(lens), lens, None, 0, cap)
    tq.tq_latent_append(cache, x[:, :d_c], x[:, d_c:], torch.from_numpy(slots).cuda())
    cache.seq_lens.copy_(_dev(torch, lens))
    model = L.Cache(len(lens) * cap, d_c)
    model.append(x[:, :d_c], x[:, d_c:], slots)
    return cache, model, np.split(slots, np.cumsum(lens)[:-1])


# n tokens of size `small` (0: zeros) around one of size `big`, each of which has 2^weight times the big one's weight
FAR = [(128, 0.0, 2.0 ** 62, 0), (2, 0.0, 2.0 ** 64, 0), (3000, 2.0 ** -64, 2.0 ** 64, 0), (1000, 0.0, 2.0 ** 63, 30), (131072, 0.0, 2.0 ** 50, -13),
       (131072, 0.0, 2.0 ** 50, -18), (131072, 2.0 ** -60, 2.0 ** 64, -17), (131072, 0.0, 2.0 ** 40, -24), (70000, 2.0 ** -63, 2.0 ** 64, -30)]


@pytest.mark.parametrize("n,small,big,weight", FAR)
@pytest.mark.parametrize("H", [4, 20, 40])
def test_a_large_token_among_small_ones(gpu, n, small, big, weight, H):
    """In the first tile, in the middle and at the end: alone in its part of the sequence, or met after the small ones."""
    tq, torch = gpu
    d_c = 128
    rng = np.random.default_rng(n)
    q_c, q_r = torch.zeros((1, H, d_c), device="cuda").bfloat16(), torch.zeros((1, H, 64), device="cuda").bfloat16()
    q_r[0, :, 0] = -float(weight)
    q_r[0, 0, 0] = 0.0                                             # and a head of equal weights
    work, out = tq.alloc_latent_workspace(1, H, d_c), torch.empty((1, H, d_c), device="cuda")
    x = np.zeros((n, d_c + 64))
    x[:, :d_c] = rng.uniform(-small, small, (n, d_c))
    for where in sorted({0, n // 2 + 7 if n > 2 else 0, n - 1}):
        y = x.copy()
        y[where, :d_c], y[where, d_c] = rng.uniform(-big, big, d_c), 1.0
        cache, model, slots = _filled(tq, torch, y, [n], d_c)
        tq.tq_sdpa_latent_decode(cache, q_c, q_r, float(np.log(2.0)), 0, 0, work, out)
        _check_wide(torch, out[0], q_c[0], q_r[0], model, slots[0], float(np.float32(np.log(2.0))))


@pytest.mark.parametrize("H", [3, 16, 30, 64, 128])
@pytest.mark.parametrize("lens", [[6000], [500, 90, 1, 1400] * 20, [30000, 64]])
def test_ranges_of_any_size(gpu, lens, H):
    """Ranges spread evenly over the powers of two from 2^-64 to 2^64 and zero, weights over 2^80."""
    tq, torch = gpu
    d_c, n = 128, sum(lens)
    rng = np.random.default_rng(H + n)
    x = np.concatenate([rng.uniform(-1, 1, (n, d_c)) * 2.0 ** rng.integers(-64, 65, (n, 1)).astype(np.float64), rng.uniform(-1, 1, (n, 64))], 1)
    x[rng.random(n) < 0.05, :d_c] = 0.0
    cache, model, slots = _filled(tq, torch, x, lens, d_c)
    B = len(lens)
    q_c, q_r = torch.zeros((B, H, d_c), device="cuda").bfloat16(), torch.zeros((B, H, 64), device="cuda").bfloat16()
    q_r[:, :, :2] = torch.randn((B, H, 2), device="cuda").bfloat16() * 30.0
    out = torch.empty((B, H, d_c), device="cuda")
    tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.7, 0, 0, tq.alloc_latent_workspace(B, H, d_c), out)
    for b in range(min(B, 8)):
        _check_wide(torch, out[b], q_c[b], q_r[b], model, slots[b], float(np.float32(0.7)))
