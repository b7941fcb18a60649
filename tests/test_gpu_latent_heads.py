"""Latent decode: no head's result depends on what the other heads attend."""
import numpy as np
import pytest

import latent_ref as L
import serving_ref as R
from test_gpu_latent import _cache, _check_decode, _dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2604_16957_b200 import tq
    assert torch.cuda.is_available()
    return tq, torch


@pytest.mark.parametrize("H", [2, 17, 33])
def test_a_head_beside_one_whose_weights_grow(gpu, H):
    """1200 sequences of two tiles: tokens of score 0 and range 127, then tokens of a range between 508 and 2032, one of whose
    scores brings the exponent of head 0 to within a rounding of where weights are rescaled (2^15.5 times that range,
    when the first tile's are 2^8).  Head 1 has a score there that needs rescaling, or none: head 0 gives the same bits."""
    tq, torch = gpu
    B, d_c = 1200, 128
    rng = np.random.default_rng(H)
    a = np.floor(rng.uniform(508.0, 2032.0, B))                   # exact in fp16
    lg = np.log2(a / 127.0)
    # the smallest score, a multiple of `grid`, with (score + 8) + log2(range / 127) above 15.5
    grid = np.where(np.arange(B) % 2, 2.0 ** -18, 2.0 ** -20)
    steps = np.rint(np.ceil((7.5 - lg) / grid) * grid * 2.0 ** 20).astype(np.int64)
    x = np.zeros((B, 128, d_c + 64))
    x[:, :, :d_c] = rng.integers(-127, 128, (1, 128, d_c))
    x[:, :, 0] = 127.0
    x[:, 64:, :d_c] = np.floor(x[:, 64:, :d_c] * (a / 127.0)[:, None, None])
    x[:, 64:, 0] = a[:, None]
    x[:, 100, d_c:d_c + 3] = 4096.0, 64.0, 1.0                     # score of digits to the base 64, times 2^-20
    x = torch.from_numpy(x.reshape(-1, d_c + 64)).half().cuda()
    cache, _ = _cache(tq, torch, B, d_c, 0, 128, 0)
    slots = np.arange(B * 128)
    tq.tq_latent_append(cache, x[:, :d_c], x[:, d_c:], torch.from_numpy(slots).cuda())
    cache.seq_lens.fill_(128)
    alpha = float(np.float32(np.log(2.0)) * np.float32(2.0 ** -20))
    q_c, q_r = torch.zeros((B, H, d_c), device="cuda").half(), torch.zeros((B, H, 64), device="cuda").half()
    digits = np.stack([steps >> 12, steps >> 6 & 63, steps & 63], 1)
    assert digits.max() < 2048
    q_r[:, 0, :3] = torch.from_numpy(digits).half().cuda()
    work = tq.alloc_latent_workspace(B, H, d_c)
    outs = []
    for far in (0.0, 16384.0):                                     # 64 log2 units
        q_r[:, 1, 0] = far
        out = torch.empty((B, H, d_c), device="cuda")
        tq.tq_sdpa_latent_decode(cache, q_c, q_r, alpha, 0, 0, work, out)
        outs.append(out)
    model = L.Cache(B * 128, d_c)
    model.append(x[:, :d_c], x[:, d_c:], slots)
    for b in (0, 1, 611, B - 1):
        for out, far in zip(outs, (0.0, 16384.0)):
            q_r[:, 1, 0] = far
            _check_decode(torch, out[b:b + 1], q_c[b:b + 1], q_r[b:b + 1], [model.values(slots[128 * b:128 * b + 128])], alpha, 0)
    assert torch.equal(outs[0][:, 0], outs[1][:, 0]), int((outs[0][:, 0] != outs[1][:, 0]).any(1).sum())
    assert not torch.equal(outs[0][:, 1], outs[1][:, 1])
