"""Attention of the serving operators where its numbers are hard: many tokens of a tiny weight each beside a dominant one,
and scores far from zero."""
import numpy as np
import pytest

import serving_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2604_16957_b200 import tq
    assert torch.cuda.is_available()
    return tq, torch


def _dominant_and_tail(n, H, d, offset):
    """K and V of n tokens (float64 [n][H][d]): the first of every 16 scores 0 with q = e_0 and has the value e_0; the others
    score `offset` (in units of log 2 / alpha) and have the value 1 in every other channel."""
    k, v = np.zeros((n, H, d)), np.zeros((n, H, d))
    tail = np.arange(n) % 16 != 0
    k[tail, :, 0] = offset
    v[tail, :, 1:] = 1.0
    v[~tail, :, 0] = 1.0
    return k, v


# one unit in a thread block; cut units; several whole units per warp; many units on one line; wide heads
@pytest.mark.parametrize("lens,H_q,H_kv,d,kind", [
    ([500], 8, 2, 64, "fp16"), ([20000], 8, 1, 128, "fp16"), ([400] * 40, 16, 8, 64, "bf16"), ([2500] * 40, 8, 8, 64, "fp16"),
    ([3000], 4, 2, 256, "bf16"), ([300], 4, 1, 512, "fp16")])
@pytest.mark.parametrize("offset", [-22.5, -18.25])
def test_decode_keeps_a_tail_of_small_weights(gpu, lens, H_q, H_kv, d, kind, offset):
    """The tail's weights are 2^-22.5 of the largest contribution each.  They enter the matrix product in 16 bits: a weight may be
    off by 2^-11 of itself, or by half a step of the subnormals, which lie 2^7 below the place that the largest contribution has:
    2^-25 / 2^7 = 2^-32 of it."""
    tq, torch = gpu
    t = {"fp16": torch.float16, "bf16": torch.bfloat16}[kind]
    B, n = len(lens), max(lens)
    cap = -(-n // 16) * 16
    k, v = _dominant_and_tail(n, H_kv, d, offset)
    cache = tq.KV8Cache(B, H_kv, cap, d)
    rows = torch.cat([torch.arange(x) + b * cap for b, x in enumerate(lens)]).cuda()
    kk, vv = (torch.cat([torch.from_numpy(y[:x]) for x in lens]).to(t).cuda() for y in (k, v))
    tq.tq_kv8_append(cache, kk, vv, rows)
    cache.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    model = R.Cache8(cap // 16, H_kv, d)
    model.append(k, v, np.arange(n))
    km, vm = model.values(np.arange(n))
    q = torch.zeros((B, H_q, d), dtype=t, device="cuda")
    q[..., 0] = 1.0
    out = torch.empty((B, H_q, d), device="cuda")
    alpha = float(np.log(2.0))
    tq.tq_sdpa_int8_decode(cache, q, alpha, 0, 0, tq.alloc_int8_workspace(B, H_kv, H_q, d), out)
    ref, weighed, p, mag = R.attention(q[0, :1].double().cpu(), km[:, 0], vm[:, 0], alpha)
    tol = R.bound(ref, weighed, p, mag, n, d, 2.0 ** -11, 1.0, 0.0, subnormal=2.0 ** -32)
    got = out.double().cpu()
    assert torch.all((got - ref).abs() <= tol), float(((got - ref).abs() / tol).max())
    assert float((tol / ref)[0, 1]) < 0.003     # (the bound says something)


@pytest.mark.parametrize("B,n", [(1, 3000), (160, 50)])   # a cut unit; whole units by warp
@pytest.mark.parametrize("size", [2.0 ** -120])
def test_decode_of_tiny_values(gpu, B, n, size):
    """bf16 values near the smallest normal numbers: what undoes the scaling of the weights does not make zeros of them."""
    tq, torch = gpu
    d, H = 64, 4
    rng = np.random.default_rng(4)
    cap = -(-n // 16) * 16
    cache = tq.KV8Cache(B, H, cap, d)
    k = torch.from_numpy(rng.standard_normal((n, H, d))).bfloat16()
    v = (torch.from_numpy(rng.uniform(0.25, 1.0, (n, H, d))) * size).bfloat16()
    tq.tq_kv8_append(cache, k.repeat(B, 1, 1).cuda(), v.repeat(B, 1, 1).cuda(),
                     torch.cat([torch.arange(n) + b * cap for b in range(B)]).cuda())
    cache.seq_lens.fill_(n)
    model = R.Cache8(cap // 16, H, d)
    model.append(k.double().numpy(), v.double().numpy(), np.arange(n))
    km, vm = model.values(np.arange(n))
    q = torch.from_numpy(rng.standard_normal((1, H, d))).bfloat16()
    out = torch.empty((B, H, d), device="cuda")
    tq.tq_sdpa_int8_decode(cache, q.repeat(B, 1, 1).cuda(), 0.125, 0, 0, tq.alloc_int8_workspace(B, H, H, d), out)
    for h in range(H):
        ref, weighed, p, mag = R.attention(q[0, h:h + 1].double(), km[:, h], vm[:, h], 0.125)
        # 127 l products of 2^-120 / 127 / l: the last factor may be subnormal, 2^-120 / 127 / 3000 = 2^-139 in steps of 2^-149
        tol = R.bound(ref, weighed, p, mag, n, d, 2.0 ** -11, size, 0.0, subnormal=2.0 ** -32) + ref.abs() * 2.0 ** -10
        assert torch.all((out[:, h].double().cpu() - ref).abs() <= tol)


def test_decode_joins_huge_values(gpu):
    """Parts of a cut unit whose values are near the largest number: their weighted sum does not overflow on its way."""
    tq, torch = gpu
    d, n = 64, 6000
    cache = tq.KV8Cache(1, 1, n, d)
    k = torch.randn((n, 1, d)).bfloat16()
    v = torch.full((n, 1, d), 2.0 ** 127, dtype=torch.bfloat16)
    v[:, :, 1::2] *= -1
    tq.tq_kv8_append(cache, k.cuda(), v.cuda(), torch.arange(n, device="cuda"))
    cache.seq_lens.fill_(n)
    out = torch.empty((1, 3, d), device="cuda")
    tq.tq_sdpa_int8_decode(cache, torch.randn((1, 3, d), device="cuda").bfloat16(), 0.125, 0, 0, tq.alloc_int8_workspace(1, 1, 3, d), out)
    # weights of equal values: their rounding in 16 bits is all that is left of the error, 2^-11 of the value
    assert torch.all((out.double().cpu() / v[:1].double() - 1).abs() <= 2.0 ** -11 + 2.0 ** -16)


@pytest.mark.parametrize("B,n", [(1, 1), (1, 40), (1, 5000), (160, 50)])
@pytest.mark.parametrize("size", [-1.3671875 * 2.0 ** 52, -1.3671875 * 2.0 ** -46, 1.3671875 * 2.0 ** -46, 1.3671875 * 2.0 ** 52])
def test_decode_of_scores_far_from_zero(gpu, B, n, size):
    """Every score near 2^18 or 2^118, of either sign: equal keys weigh their values equally, whatever the score is."""
    tq, torch = gpu
    d, H = 64, 4
    cap = -(-n // 16) * 16
    cache = tq.KV8Cache(B, H, cap, d)
    k = torch.full((B * n, H, d), 2.0 ** 60, dtype=torch.bfloat16, device="cuda")
    v = (torch.rand((n, H, d)) + 0.5).bfloat16()
    tq.tq_kv8_append(cache, k, v.repeat(B, 1, 1).cuda(), torch.cat([torch.arange(n) + b * cap for b in range(B)]).cuda())
    cache.seq_lens.fill_(n)
    model = R.Cache8(cap // 16, H, d)
    model.append(np.zeros((n, H, d)), v.double().numpy(), np.arange(n))
    q = torch.full((B, H, d), size, dtype=torch.bfloat16, device="cuda")
    out = torch.empty((B, H, d), device="cuda")
    tq.tq_sdpa_int8_decode(cache, q, 1.0, 0, 0, tq.alloc_int8_workspace(B, H, H, d), out)
    ref = torch.as_tensor(model.values(np.arange(n))[1].mean(0))
    assert torch.all((out.double().cpu() - ref).abs() <= 2.0 ** -11 * 1.5 + 2.0 ** -15)   # weights in 16 bits, values up to 1.5


@pytest.mark.parametrize("padded", [0, 200])   # one tile per thread block, and two
@pytest.mark.parametrize("d", [64, 128, 256, 512])
@pytest.mark.parametrize("offset", [-22.5, -18.25])
def test_prompt_keeps_a_tail_of_small_weights(gpu, padded, d, offset):
    """As for decode: fp16 weights are off by 2^-11 of themselves or by 2^-32 of the largest one."""
    tq, torch = gpu
    n, H_q, H = 300, 4, 2
    k, v = _dominant_and_tail(n, H, d, offset)
    k, v = (torch.from_numpy(x).half().cuda() for x in (k, v))
    q = torch.zeros((n, H_q, d), dtype=torch.float16, device="cuda")
    q[..., 0] = 1.0
    at = torch.tensor([0, n] + [n] * padded, dtype=torch.int32, device="cuda")
    out = torch.empty((n, H_q, d), device="cuda")
    alpha = float(np.log(2.0))
    tq.tq_sdpa_prompt(q, k, v, at, at, alpha, out)
    seen = torch.arange(n)[None, :] <= torch.arange(n)[:, None]
    ref, weighed, p, mag = R.attention(q[:, 0].double().cpu(), k[:, 0].double().cpu(), v[:, 0].double().cpu(), alpha, seen)
    tol = R.bound(ref, weighed, p, mag, n, d, 2.0 ** -11, 1.0, 0.0, subnormal=2.0 ** -32)
    got = out.double().cpu()
    for h in range(H_q):
        assert torch.all((got[:, h] - ref).abs() <= tol), float(((got[:, h] - ref).abs() / tol).max())
    # the bound says something (in the last row: it counts all n tokens as seen, row i sees i + 1)
    assert float((tol / ref)[-1, 1]) < 0.003


@pytest.mark.parametrize("padded", [0, 200])
@pytest.mark.parametrize("d", [64, 128, 256, 512])
@pytest.mark.parametrize("size", [-1.3671875 * 2.0 ** 52, -1.3671875 * 2.0 ** -46, 1.3671875 * 2.0 ** -46, 1.3671875 * 2.0 ** 52])
def test_prompt_of_scores_far_from_zero(gpu, padded, d, size):
    """Every score near 2^18 or 2^118 or beyond, of either sign: equal keys weigh their values equally, whatever the score is.  A query
    of zeros among the others (weights of 1) is not disturbed."""
    tq, torch = gpu
    n, H = 300, 2
    k = torch.full((n, H, d), 2.0 ** 60, dtype=torch.bfloat16, device="cuda")
    v = (torch.rand((n, H, d)) + 0.5).bfloat16().cuda()
    q = torch.full((n, 4, d), size, dtype=torch.bfloat16, device="cuda")
    q[100:110] = 0
    at = torch.tensor([0, n] + [n] * padded, dtype=torch.int32, device="cuda")
    out = torch.empty((n, 4, d), device="cuda")
    tq.tq_sdpa_prompt(q, k, v, at, at, 1.0, out)
    ref = (v.double().cumsum(0) / torch.arange(1, n + 1, device="cuda")[:, None, None]).repeat_interleave(2, 1)
    assert torch.all((out.double() - ref).abs() <= 1.5 * 2.0 ** -8)   # weights in bf16, values up to 1.5


@pytest.mark.parametrize("padded", [0, 200])
@pytest.mark.parametrize("d", [64, 256])
@pytest.mark.parametrize("size", [-44800.0, -11.0, 1.37, 3.3, 11.0, 44800.0])
def test_prompt_of_fp16_scores_far_from_zero(gpu, padded, d, size):
    """The same in fp16, whose weights have less room: scores of 2^22 to 2^38."""
    tq, torch = gpu
    n, H = 300, 2
    k = torch.full((n, H, d), 42112.0, dtype=torch.float16, device="cuda")
    v = (torch.rand((n, H, d)) + 0.5).half().cuda()
    q = torch.full((n, 4, d), size, dtype=torch.float16, device="cuda")
    at = torch.tensor([0, n] + [n] * padded, dtype=torch.int32, device="cuda")
    out = torch.empty((n, 4, d), device="cuda")
    tq.tq_sdpa_prompt(q, k, v, at, at, 1.0, out)
    ref = (v.double().cumsum(0) / torch.arange(1, n + 1, device="cuda")[:, None, None]).repeat_interleave(2, 1)
    assert torch.all((out.double() - ref).abs() <= 1.5 * (2.0 ** -11 + 2.0 ** -15))


@pytest.mark.parametrize("padded", [0, 200])
@pytest.mark.parametrize("d", [64, 128, 256, 512])
@pytest.mark.parametrize("size", [2.0 ** 127, 2.0 ** -100])
def test_prompt_of_huge_and_tiny_values(gpu, padded, d, size):
    """bf16 values near the largest number: the sum of a row's weighted values does not overflow before it is divided.  And small
    ones, of which nothing is lost for that."""
    tq, torch = gpu
    n, H = 1500, 1
    v = torch.full((n, H, d), size, dtype=torch.bfloat16, device="cuda")
    v[..., 1::2] *= -1
    q, k = torch.randn((n, 2, d), device="cuda").bfloat16(), torch.randn((n, H, d), device="cuda").bfloat16()
    at = torch.tensor([0, n] + [n] * padded, dtype=torch.int32, device="cuda")
    out = torch.empty((n, 2, d), device="cuda")
    tq.tq_sdpa_prompt(q, k, v, at, at, d ** -0.5, out)
    # equal values: what is left of the error is the rounding of the weights, 2^-8
    assert torch.all((out.double() / v.double() - 1).abs() <= 2.0 ** -8 + 2.0 ** -15)


@pytest.mark.parametrize("B,n,H_q,H,d,kind", [(1, 300, 16, 2, 128, "fp16"), (200, 60, 12, 4, 64, "bf16"), (3, 9000, 16, 2, 128, "bf16"),
                                              (1, 5000, 8, 1, 256, "fp16")])
def test_a_query_of_infinities_or_nans_stays_in_its_row(gpu, B, n, H_q, H, d, kind):
    """Decode and prompt attention: the other heads and tokens give the same bits as without it."""
    tq, torch = gpu
    t = {"fp16": torch.float16, "bf16": torch.bfloat16}[kind]
    cap = -(-n // 16) * 16
    cache = tq.KV8Cache(B, H, cap, d)
    k, v = (torch.randn((B * n, H, d), device="cuda").to(t) for _ in range(2))
    tq.tq_kv8_append(cache, k, v, torch.cat([torch.arange(n, device="cuda") + b * cap for b in range(B)]))
    cache.seq_lens.fill_(n)
    work = tq.alloc_int8_workspace(B, H, H_q, d)
    at = torch.tensor([0, 200, 300], dtype=torch.int32, device="cuda")
    for rows, call in ((B, lambda q, o: tq.tq_sdpa_int8_decode(cache, q, 0.1, 0, 0, work, o)),
                       (300, lambda q, o: tq.tq_sdpa_prompt(q, k[:300], v[:300], at, at, 0.1, o))):
        q = torch.randn((rows, H_q, d), device="cuda").to(t)
        bad = torch.zeros((rows, H_q), dtype=torch.bool, device="cuda")
        outs = []
        for _ in range(2):
            outs.append(torch.empty((rows, H_q, d), device="cuda"))
            call(q, outs[-1])
            for b, h, c, x in ((0, 1, 3, "nan"), (-1, -1, 0, "inf"), (rows // 2, 4, 5, "-inf")):
                q[b, h, c] = float(x)
                bad[b, h] = True
        assert torch.equal(outs[0][~bad], outs[1][~bad]) and torch.isnan(outs[1][bad]).any(-1).all()
