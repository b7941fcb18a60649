"""Prompt attention in forms that the other tests pass by: wide heads (d = 512) with windows, without the causal mask, with
NaN and infinities and over many key tiles, and chunks whose past comes back from the 8-bit cache."""
import numpy as np
import pytest

import serving_ref as R
from test_gpu_serving import _check_prompt, _packed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2604_16957_b200 import tq
    assert torch.cuda.is_available()
    return tq, torch


def _dev(torch, x, t=None):
    return torch.tensor(x, dtype=t or torch.int32, device="cuda")


@pytest.mark.parametrize("lq,past,H_q,H_kv,kind,causal,window", [
    ([1], 0, 2, 1, "fp16", True, 0), ([700, 33], 0, 4, 2, "bf16", True, 0), ([300, 1, 0, 65], 0, 8, 2, "fp16", True, 100),
    ([130], 0, 6, 2, "bf16", True, 1), ([200, 31], 45, 4, 1, "fp16", False, 0), ([64, 5], 700, 8, 8, "bf16", True, 0),
    ([100], 333, 3, 1, "fp16", True, 50), ([40], -12, 2, 2, "bf16", True, 0), ([90] * 30, 0, 8, 4, "fp16", True, 0)])
def test_prompt_with_wide_heads(gpu, lq, past, H_q, H_kv, kind, causal, window):
    tq, torch = gpu
    d = 512
    rng = np.random.default_rng(sum(lq) + 1)
    lk = [max(0, n + past) if n else 0 for n in lq]
    fused = past == 0
    q, k, v = _packed(torch, rng, lq, lk, H_q, H_kv, d, kind, fused, 3)
    q_at, k_at = np.concatenate([[0], np.cumsum(lq)]).tolist(), np.concatenate([[0], np.cumsum(lk)]).tolist()
    dq, dk = _dev(torch, q_at), _dev(torch, k_at)
    status = _dev(torch, [0])
    for out_t in (torch.float32, q.dtype):
        guard = torch.full(((len(q) + 2) * H_q * d,), 5.0, dtype=out_t, device="cuda")
        out = guard.view(-1, H_q, d)[1:-1]
        tq.tq_sdpa_prompt(q, k, v, dq, dq if fused else dk, d ** -0.5, out, causal=causal, window=window, status=status)
        assert int(status.item()) == 0
        assert torch.all(guard.view(-1, H_q, d)[0] == 5.0) and torch.all(guard.view(-1, H_q, d)[1 + sum(lq):] == 5.0)
        _check_prompt(torch, out, q, k, v, q_at, k_at, d ** -0.5, causal, window)


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("window", [0, 20])
def test_infinities_and_nans_with_wide_heads(gpu, kind, window):
    """In both halves of the channels, which different thread blocks compute: of another sequence, of later tokens, outside the window, and
    seen."""
    tq, torch = gpu
    d, H_q, H = 512, 4, 2
    q, k, v = (x.contiguous() for x in _packed(torch, np.random.default_rng(5), [150, 90, 60], [150, 90, 60], H_q, H, d, kind, True, 2))
    at = [0, 150, 240, 300]
    v[150:240], k[150:240] = float("nan"), float("inf")
    v[100, 0, 3], v[101, 1, 300], v[240, 0, 511], v[77, 1, 256] = float("inf"), float("nan"), -float("inf"), float("inf")
    v[300:], k[300:] = float("nan"), float("nan")
    out = torch.empty(q.shape, device="cuda")
    tq.tq_sdpa_prompt(q, k, v, _dev(torch, at), _dev(torch, at), d ** -0.5, out, window=window)
    assert torch.isnan(out[150:240]).all()
    _check_prompt(torch, out[:150], q[:150], k[:150], v[:150], [0, 150], [0, 150], d ** -0.5, True, window)
    _check_prompt(torch, out[240:], q[240:300], k[240:300], v[240:300], [0, 60], [0, 60], d ** -0.5, True, window)


@pytest.mark.parametrize("d,kind,window", [(64, "fp16", 0), (128, "bf16", 0), (128, "fp16", 100), (256, "bf16", 300), (512, "fp16", 0)])
def test_chunked_prompts_over_the_cache(gpu, d, kind, window):
    """Prompts admitted in chunks: the pages and slots of a chunk, its attention over the past that the cache gives back and its own
    tokens, and the append.  A token's slot is page_table[b][p / page_tokens] * page_tokens + p % page_tokens."""
    tq, torch = gpu
    t = {"fp16": torch.float16, "bf16": torch.bfloat16}[kind]
    rng = np.random.default_rng(d + window)
    B, H_q, H, P, pages = 3, 4, 2, 16, 60
    table, lens = torch.zeros((B, 20), dtype=torch.int32, device="cuda"), _dev(torch, [0] * B)
    free, count, offsets, status = torch.randperm(pages).int().cuda(), _dev(torch, [pages]), _dev(torch, [0] * (B + 1)), _dev(torch, [0])
    cache = tq.PagedKV8Cache.over(torch.full((pages, H, 1, tq.TQ_BLOCK8_BYTES(d)), 0xA5, dtype=torch.uint8, device="cuda"), lens, table)
    work, model = tq.alloc_pages_workspace(B), R.Cache8(pages, H, d)
    for new in ([37, 100, 1], [64, 0, 150], [1, 90, 33], [120, 1, 0]):
        cached = lens.tolist()
        n = sum(new)
        slots = torch.empty(n, dtype=torch.int64, device="cuda")
        tq.tq_pages_assign(table, lens, _dev(torch, new), P, pages, free, count, lens, count, offsets, slots, work, status)
        x = torch.from_numpy(rng.standard_normal((n, H_q + 2 * H, d))).to(t).cuda()
        q, k, v = x[:, :H_q], x[:, H_q:H_q + H], x[:, H_q + H:]
        # the past of every sequence, then its chunk
        old = [torch.arange(c, device="cuda") for c in cached]
        past = torch.cat([table[b, p // P].long() * P + p % P for b, p in enumerate(old)])
        pk, pv = (torch.empty((len(past), H, d), dtype=t, device="cuda") for _ in range(2))
        tq.tq_kv8_gather(cache, past, pk, pv, status)
        assert all(np.array_equal(got.double().cpu().numpy(), torch.from_numpy(want).float().to(t).double().numpy())
                   for got, want in zip((pk, pv), model.values(past.cpu().numpy())))
        at, p0 = offsets.tolist(), np.concatenate([[0], np.cumsum(cached)]).tolist()
        ks, vs = (torch.cat([torch.cat([old_[p0[b]:p0[b + 1]], new_[at[b]:at[b + 1]]]) for b in range(B)]) for old_, new_ in ((pk, k), (pv, v)))
        k_at = np.concatenate([[0], np.cumsum([c + m for c, m in zip(cached, new)])]).tolist()
        out = torch.empty((n, H_q, d), device="cuda")
        tq.tq_sdpa_prompt(q, ks, vs, offsets, _dev(torch, k_at), d ** -0.5, out, window=window, status=status)
        _check_prompt(torch, out, q, ks, vs, at, k_at, d ** -0.5, True, window)
        tq.tq_kv8_append(cache, k, v, slots, status)
        model.append(k.double().cpu().numpy(), v.double().cpu().numpy(), slots.cpu().numpy())
    assert int(status.item()) == 0 and lens.tolist() == [222, 191, 184]


@pytest.mark.parametrize("padded", [0, 200])
def test_a_scale_that_is_no_number(gpu, padded):
    """It gives NaN, as it does in decode, and no average of the values; queries that see nothing stay zero."""
    tq, torch = gpu
    q, k, v = _packed(torch, np.random.default_rng(7), [70], [70], 4, 2, 64, "fp16", True)
    out = torch.empty(q.shape, device="cuda")
    tq.tq_sdpa_prompt(q, k[:40], v[:40], _dev(torch, [0, 70] + [70] * padded), _dev(torch, [0, 40] + [40] * padded), float("nan"), out)
    assert torch.isnan(out[30:]).all() and torch.all(out[:30] == 0)
    cache = tq.KV8Cache(1, 2, 64, 64)
    tq.tq_kv8_append(cache, k[:40], v[:40], torch.arange(40, device="cuda"))
    cache.seq_lens.fill_(40)
    out = torch.empty((1, 4, 64), device="cuda")
    tq.tq_sdpa_int8_decode(cache, q[:1], float("nan"), 0, 0, tq.alloc_int8_workspace(1, 2, 4, 64), out)
    assert torch.isnan(out).all()
