"""Latent decode of batches whose sequences are cut into very different numbers of parts: long ones among many that are short or empty."""
import numpy as np
import pytest

from test_gpu_latent import _check_decode, _dev, _filled, _queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2604_16957_b200 import tq
    assert torch.cuda.is_available()
    return tq, torch


BATCHES = [[40000] + [1] * 63, [0] * 200 + [30000], [3, 0, 9000] * 20, [20000, 20000] + [64, 65, 0] * 100, [1200] * 60, [700] * 17 + [16000] + [50] * 400,
           [14000] * 9 + [7], [33000, 31000, 2, 35000, 34000]]


@pytest.mark.parametrize("lens", BATCHES)
@pytest.mark.parametrize("H,d_c,kind", [(5, 128, "fp16"), (16, 512, "bf16"), (24, 256, "fp16"), (100, 128, "bf16")])
def test_long_sequences_among_short_ones(gpu, lens, H, d_c, kind):
    tq, torch = gpu
    B = len(lens)
    cache, values = _filled(tq, torch, lens, d_c, 16, kind, B + H)
    q_c, q_r = _queries(torch, B, H, d_c, kind)
    alpha, status = (d_c + 64) ** -0.5, _dev(torch, [0])
    work = tq.alloc_latent_workspace(B, H, d_c)
    work.fill_(0x11)
    guard = torch.full(((B + 2) * H * d_c,), float("nan"), device="cuda").view(-1, H, d_c)
    out = guard[1:-1]
    tq.tq_sdpa_latent_decode(cache, q_c, q_r, alpha, 0, 0, work, out, status)
    assert int(status.item()) == (tq.TQ_STATUS_EMPTY_SEQ if 0 in lens else 0)
    longest = np.argsort(lens)[-4:].tolist()
    _check_decode(torch, out, q_c, q_r, values, alpha, 0, rows=sorted({0, 1, B // 2, B - 1, *longest}))
    assert torch.all(torch.isnan(guard[0])) and torch.all(torch.isnan(guard[-1])) and torch.all(torch.isfinite(out))
    # with a bound on the lengths, into other junk
    work.fill_(0x22)
    again = torch.full_like(out, float("nan"))
    tq.tq_sdpa_latent_decode(cache, q_c, q_r, alpha, 0, max(lens), work, again)
    _check_decode(torch, again, q_c, q_r, values, alpha, 0, rows=longest)
    assert torch.all(torch.isfinite(again))
