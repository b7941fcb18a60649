"""The serving operators as a server uses them: other streams, captured graphs, side by side, many sequences, caches and
tensors beyond 4 GB, calls that the binding refuses."""
import numpy as np
import pytest

import serving_ref as R
from test_gpu_serving import _cache, _check_cache, _check_decode, _check_prompt, _filled, _packed, _rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2604_16957_b200 import tq
    assert torch.cuda.is_available()
    return tq, torch


def _dev(torch, x, t=None):
    return torch.tensor(x, dtype=t or torch.int32, device="cuda")


def test_streams_side_by_side(gpu):
    """Prompt attention, append and decode on two streams at a time, each with a workspace of its own, against the same calls
    one after the other on the default stream: bit for bit."""
    tq, torch = gpu
    rng = np.random.default_rng(1)
    jobs = []
    for seed in (3, 4):
        cache, _ = _filled(tq, torch, [3000, 70, 900], 2, 128, 16, "fp16", seed, cap=3200)
        q, k, v = _packed(torch, rng, [300, 40], [300, 40], 8, 2, 128, "bf16", True)
        jobs.append(dict(cache=cache, dq=torch.randn((3, 16, 128), device="cuda").half(), q=q, k=k, v=v, at=_dev(torch, [0, 300, 340])))

    def run(j, stream=None):
        work = tq.alloc_int8_workspace(3, 2, 16, 128)
        torch.cuda.synchronize()
        outs = [torch.zeros((3, 16, 128), device="cuda") for _ in range(20)] + [torch.zeros(j["q"].shape, device="cuda") for _ in range(5)]
        torch.cuda.synchronize()
        for o in outs[:20]:
            tq.tq_sdpa_int8_decode(j["cache"], j["dq"], 0.09, 0, 0, work, o, stream=stream)
        for o in outs[20:]:
            tq.tq_sdpa_prompt(j["q"], j["k"], j["v"], j["at"], j["at"], 0.09, o, stream=stream)
        return outs

    want = [run(j) for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for j, s in zip(jobs, streams):
        got.append(run(j, s))
    for s in streams:
        s.synchronize()
    for a, b in zip(want, got):
        for x, y in zip(a, b):
            assert torch.equal(x, y) and x.abs().sum() > 0


def test_captured_prompt_follows_the_offsets(gpu):
    """One captured launch of prompt attention, replayed with other lengths and other data in the same tensors."""
    tq, torch = gpu
    rng = np.random.default_rng(2)
    n, H_q, H, d = 400, 8, 2, 128
    x = torch.zeros((n, H_q + 2 * H, d), dtype=torch.float16, device="cuda")
    q, k, v = x[:, :H_q], x[:, H_q:H_q + H], x[:, H_q + H:]
    at = _dev(torch, [0, 0, 0, 0])
    out = torch.zeros((n, H_q, d), device="cuda")
    tq.tq_sdpa_prompt(q, k, v, at, at, d ** -0.5, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tq.tq_sdpa_prompt(q, k, v, at, at, d ** -0.5, out)
    for lens in ([400, 0, 0], [1, 2, 3], [0, 129, 200], [100, 100, 200]):
        x.copy_(torch.from_numpy(rng.standard_normal(x.shape)).half())
        cum = np.concatenate([[0], np.cumsum(lens)]).tolist()
        at.copy_(torch.tensor(cum, dtype=torch.int32))
        out.fill_(5.0)
        g.replay()
        _check_prompt(torch, out, q, k, v, cum, cum, d ** -0.5, True, 0)
        assert torch.all(out[cum[-1]:] == 5.0)


def test_two_captured_decode_graphs(gpu):
    """Two graphs over one cache, each with a workspace of its own, replayed on two streams at once; then both on one stream
    with the workspaces that they share with eager calls."""
    tq, torch = gpu
    cache, values = _filled(tq, torch, [5000, 1, 2500], 2, 64, 0, "fp16", 9)
    qs = [torch.randn((3, 8, 64), device="cuda").half() for _ in range(2)]
    outs = [torch.zeros((3, 8, 64), device="cuda") for _ in range(2)]
    works = [tq.alloc_int8_workspace(3, 2, 8, 64) for _ in range(2)]
    graphs = []
    for q, o, w in zip(qs, outs, works):
        tq.tq_sdpa_int8_decode(cache, q, 0.125, 0, 0, w, o)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(10):
                tq.tq_sdpa_int8_decode(cache, q, 0.125, 0, 0, w, o)
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for q, o in zip(qs, outs):
        _check_decode(torch, o, q, values, 0.125, 0, 64)
    for g, q, o, w in zip(graphs, qs, outs, works):
        o.zero_()
        g.replay()
        tq.tq_sdpa_int8_decode(cache, q, 0.125, 0, 0, w, o)
        _check_decode(torch, o, q, values, 0.125, 0, 64)


def test_many_sequences(gpu):
    """More sequences than a round of the decode kernel's scan, most of them short or empty; hundreds of tiny prompts."""
    tq, torch = gpu
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 40, 1300).tolist()
    lens[7], lens[1299] = 700, 33
    cache, values = _filled(tq, torch, lens, 2, 64, 16, "bf16", 6)
    q = torch.randn((1300, 4, 64), device="cuda").bfloat16()
    out = torch.full((1300, 4, 64), 9.0, device="cuda")
    status = _dev(torch, [0])
    tq.tq_sdpa_int8_decode(cache, q, 0.125, 0, 0, tq.alloc_int8_workspace(1300, 2, 4, 64), out, status)
    assert int(status.item()) == tq.TQ_STATUS_EMPTY_SEQ
    _check_decode(torch, out, q, values, 0.125, 0, 64)
    lq = rng.integers(0, 4, 700).tolist()
    q, k, v = _packed(torch, rng, lq, lq, 4, 4, 64, "fp16", True)
    cum = np.concatenate([[0], np.cumsum(lq)]).tolist()
    at = _dev(torch, cum)
    out = torch.empty(q.shape, device="cuda")
    tq.tq_sdpa_prompt(q, k, v, at, at, 0.125, out)
    _check_prompt(torch, out, q, k, v, cum, cum, 0.125, True, 0)


def test_a_workspace_serves_another_shape_once_zeroed(gpu):
    tq, torch = gpu
    work = torch.zeros(8 << 20, dtype=torch.uint8, device="cuda")
    for seed, (lens, H_q, H, d) in enumerate([([4000], 8, 1, 64), ([3000, 2000, 1000], 64, 8, 128), ([2500], 2, 2, 256)]):
        cache, values = _filled(tq, torch, lens, H, d, 0, "fp16", 20 + seed)
        q = torch.randn((len(lens), H_q, d), device="cuda").half()
        out = torch.empty((len(lens), H_q, d), device="cuda")
        work.zero_()
        for _ in range(3):
            out.fill_(3.0)
            tq.tq_sdpa_int8_decode(cache, q, d ** -0.5, 0, 0, work, out)
            _check_decode(torch, out, q, values, d ** -0.5, 0, d)


def test_cache_beyond_4_gb(gpu):
    """The last sequence of a contiguous cache of 4.6 GB, and the last page of a pool of that size: append, gather, decode."""
    tq, torch = gpu
    rng = np.random.default_rng(8)
    H, d, n = 8, 128, 300
    for paged in (False, True):
        if paged:
            pages = 17 * 1024
            cache = tq.PagedKV8Cache.over(torch.empty((pages, H, 8, tq.TQ_BLOCK8_BYTES(d)), dtype=torch.uint8, device="cuda"),
                                          _dev(torch, [n]), _dev(torch, [[pages - 1, pages - 3, pages - 2]]))
            table = [[pages - 1, pages - 3, pages - 2]]
            slots = R.slots_of([0], [n], table, 128)
        else:
            cache = tq.KV8Cache.over(torch.empty((17, H, 8192, tq.TQ_BLOCK8_BYTES(d)), dtype=torch.uint8, device="cuda"),
                                     _dev(torch, [0] * 16 + [n]))
            slots = np.arange(n) + 16 * 131072
        assert cache.blocks.numel() > 1 << 32
        k, v = _rows(torch, rng, n, H, d, "fp16")
        s = torch.from_numpy(slots).cuda()
        tq.tq_kv8_append(cache, k, v, s)
        ko, vo = (torch.empty((n, H, d), device="cuda") for _ in range(2))
        tq.tq_kv8_gather(cache, s, ko, vo)
        model = R.Cache8(20, H, d)
        model.append(k.double().cpu().numpy(), v.double().cpu().numpy(), np.arange(n))
        values = model.values(np.arange(n))
        assert np.allclose(ko.cpu().numpy(), values[0], rtol=2.0 ** -22) and np.allclose(vo.cpu().numpy(), values[1], rtol=2.0 ** -22)
        B = 1 if paged else 17
        q = torch.randn((B, 16, d), device="cuda").half()
        out = torch.full((B, 16, d), 3.0, device="cuda")
        tq.tq_sdpa_int8_decode(cache, q, d ** -0.5, 0, 0, tq.alloc_int8_workspace(B, H, 16, d), out)
        _check_decode(torch, out[-1:], q[-1:], [values], d ** -0.5, 0, d)
        assert torch.all(out[:-1] == 0)
        del cache
        torch.cuda.empty_cache()


def test_prompt_rows_beyond_4_gb(gpu):
    """Sequences at the far end of packed tensors of more than 2^31 elements."""
    tq, torch = gpu
    n, H_q, H, d = 225000, 64, 8, 128
    x = torch.empty((n, H_q + 2 * H, d), dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 1 << 31
    x[-300:] = torch.randn((300, H_q + 2 * H, d), device="cuda").bfloat16()
    out = torch.empty((n, H_q, d), dtype=torch.bfloat16, device="cuda")
    out[-320:] = 5.0
    q, k, v = x[:, :H_q], x[:, H_q:H_q + H], x[:, H_q + H:]
    at = _dev(torch, [n - 300, n - 100, n - 4])
    tq.tq_sdpa_prompt(q, k, v, at, at, d ** -0.5, out)
    assert torch.all(out[-320:-300] == 5.0) and torch.all(out[-4:] == 5.0)
    tail = slice(n - 300, n)
    _check_prompt(torch, out[tail], q[tail], k[tail], v[tail], [0, 200, 296], [0, 200, 296], d ** -0.5, True, 0)


def test_results_do_not_depend_on_the_run(gpu):
    """The same call twice gives the same bits: no atomics on results, a fixed split."""
    tq, torch = gpu
    cache, _ = _filled(tq, torch, [20000, 300], 4, 128, 64, "bf16", 30)
    q = torch.randn((2, 32, 128), device="cuda").bfloat16()
    work = tq.alloc_int8_workspace(2, 4, 32, 128)
    a, b = (torch.empty((2, 32, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for _ in range(10):
        tq.tq_sdpa_int8_decode(cache, q, 0.09, 0, 0, work, a)
        tq.tq_sdpa_int8_decode(cache, q, 0.09, 0, 0, work, b)
        assert torch.equal(a, b)


def test_the_binding_refuses(gpu):
    """Shapes, types and strides that the library could not use raise before anything is launched."""
    tq, torch = gpu
    cache = tq.KV8Cache(2, 2, 64, 128)
    work = tq.alloc_int8_workspace(2, 2, 8, 128)
    z = lambda *s, t=torch.float16: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    slots = z(3, t=torch.int64)
    at = _dev(torch, [0, 3])
    kv4 = tq.KVCache(2, 2, 64, 128)
    bad = [
        lambda: tq.tq_kv8_append(kv4, z(3, 2, 128), z(3, 2, 128), slots),
        lambda: tq.tq_kv8_append(cache, z(3, 2, 64), z(3, 2, 64), slots),
        lambda: tq.tq_kv8_append(cache, z(2, 2, 128), z(2, 2, 128), slots),
        lambda: tq.tq_kv8_append(cache, z(3, 2, 128, t=torch.float32), z(3, 2, 128, t=torch.float32), slots),
        lambda: tq.tq_kv8_append(cache, z(3, 2, 128), z(3, 2, 128, t=torch.bfloat16), slots),
        lambda: tq.tq_kv8_append(cache, z(3, 4, 128)[:, ::2], z(3, 2, 128), slots),
        lambda: tq.tq_kv8_append(cache, z(1, 2, 128).expand(3, 2, 128), z(3, 2, 128), slots),
        lambda: tq.tq_kv8_append(cache, z(3, 2, 128), z(3, 2, 128), slots.int()),
        lambda: tq.tq_kv8_append(cache, z(3, 2, 128).cpu(), z(3, 2, 128), slots),
        lambda: tq.tq_kv8_gather(cache, slots, z(3, 2, 128), z(3, 2, 128, t=torch.float32)),
        lambda: tq.tq_kv8_gather(cache, slots, z(3, 3, 128)[:, :2], z(3, 2, 128)),
        lambda: tq.tq_sdpa_int8_decode(kv4, z(2, 8, 128), 1.0, 0, 0, work, z(2, 8, 128)),
        lambda: tq.tq_sdpa_int8_decode(cache, z(3, 8, 128), 1.0, 0, 0, work, z(3, 8, 128)),
        lambda: tq.tq_sdpa_int8_decode(cache, z(2, 7, 128), 1.0, 0, 0, work, z(2, 7, 128)),
        lambda: tq.tq_sdpa_int8_decode(cache, z(2, 8, 128), 1.0, 0, 0, work[:100], z(2, 8, 128)),
        lambda: tq.tq_sdpa_int8_decode(cache, z(2, 8, 128), 1.0, 0, 0, work, z(2, 8, 128, t=torch.bfloat16)),
        lambda: tq.tq_sdpa_int8_decode(cache, z(2, 8, 128), 1.0, -1, 0, work, z(2, 8, 128)),
        lambda: tq.tq_sdpa_prompt(z(3, 4, 96), z(3, 2, 96), z(3, 2, 96), at, at, 1.0, z(3, 4, 96)),
        lambda: tq.tq_sdpa_prompt(z(3, 4, 64), z(3, 2, 64), z(4, 2, 64), at, at, 1.0, z(3, 4, 64)),
        lambda: tq.tq_sdpa_prompt(z(3, 4, 64), z(3, 2, 64), z(3, 2, 64), at, _dev(torch, [0, 1, 3]), 1.0, z(3, 4, 64)),
        lambda: tq.tq_sdpa_prompt(z(3, 4, 64), z(3, 2, 64), z(3, 2, 64), at, at, 1.0, z(3, 4, 64), causal=False, window=4),
        lambda: tq.tq_sdpa_prompt(z(3, 4, 65)[..., :64], z(3, 2, 64), z(3, 2, 64), at, at, 1.0, z(3, 4, 64)),
        lambda: tq.tq_sdpa_prompt(z(3, 4, 64), z(3, 3, 64), z(3, 3, 64), at, at, 1.0, z(3, 4, 64)),
        lambda: tq.tq_pages_assign(z(2, 4, t=torch.int32), _dev(torch, [1, 2, 3]), _dev(torch, [1, 2, 3]), 16, 9, z(9, t=torch.int32), _dev(torch, [9]),
                                   z(3, t=torch.int32), z(1, t=torch.int32), z(4, t=torch.int32), slots, tq.alloc_pages_workspace(3)),
        lambda: tq.tq_pages_assign(z(3, 4, t=torch.int32), _dev(torch, [1, 2, 3]), _dev(torch, [1, 2, 3]), 16, 9, z(8, t=torch.int32), _dev(torch, [8]),
                                   z(3, t=torch.int32), z(1, t=torch.int32), z(4, t=torch.int32), slots, tq.alloc_pages_workspace(3)),
        lambda: tq.tq_pages_release(z(3, 4, t=torch.int32), _dev(torch, [1, 2, 3]), z(3, t=torch.int32), 16, 9, z(9, t=torch.int32), _dev(torch, [0]),
                                    z(3, t=torch.int32), z(1, t=torch.int32)),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(tq.TqError):
            call()
            raise AssertionError(i)
    # nothing to do is no error
    tq.tq_kv8_append(cache, z(0, 2, 128), z(0, 2, 128), slots[:0])
    tq.tq_kv8_gather(cache, slots[:0], z(0, 2, 128), z(0, 2, 128))
    tq.tq_sdpa_prompt(z(0, 4, 64), z(0, 2, 64), z(0, 2, 64), _dev(torch, [0, 0]), _dev(torch, [0, 0]), 1.0, z(0, 4, 64))
    # a single row of any stride
    x = z(1, 6, 128)
    tq.tq_kv8_append(cache, x.as_strided((1, 2, 128), (3, 128, 1)), x[:, 2:4], _dev(torch, [0], torch.int64))
    torch.cuda.synchronize()


def test_one_workspace_for_batches_of_any_shape(gpu):
    """Zeroed once, it goes from call to call whatever their batch, heads and head dimension: a server's batch changes from step to
    step."""
    tq, torch = gpu
    shapes = [([9000, 50], 16, 2, 128), ([2500, 700] * 32, 8, 8, 64), ([3000], 4, 2, 256), ([1500] * 40, 32, 8, 128), ([30000], 8, 1, 128),
              ([20, 2500, 300] * 15, 16, 8, 64), ([600, 900], 8, 2, 512)]
    work = torch.zeros(max(int(tq._lib.tq_int8_workspace_bytes(len(l), H, H_q, d)) for l, H_q, H, d in shapes), dtype=torch.uint8, device="cuda")
    filled = [_filled(tq, torch, l, H, d, 0, "fp16", 40 + i) for i, (l, H_q, H, d) in enumerate(shapes)]
    for turn in range(2):
        for (lens, H_q, H, d), (cache, values) in zip(shapes, filled):
            q = torch.randn((len(lens), H_q, d), device="cuda").half()
            out = torch.full((len(lens), H_q, d), 3.0, device="cuda")
            tq.tq_sdpa_int8_decode(cache, q, d ** -0.5, 0, 0, work, out)
            _check_decode(torch, out, q, values, d ** -0.5, 0, d)


def test_pages_for_the_4_bit_cache(gpu):
    """Pages from tq_pages_assign serve a paged 4-bit cache whose lengths the append advances: bit for bit the contiguous
    cache's contents and attention."""
    tq, torch = gpu
    B, H, d, P, pages = 3, 2, 128, 16, 30
    paged, plain = tq.PagedKVCache(B, H, P, 8, pages, d), tq.KVCache(B, H, 128, d)
    free, count = torch.randperm(pages).int().cuda(), _dev(torch, [pages])
    after, offsets, status = _dev(torch, [0] * B), _dev(torch, [0] * (B + 1)), _dev(torch, [0])
    work = tq.alloc_pages_workspace(B)
    for T in (37, 1, 1, 16, 9, 1):
        slots = torch.empty(B * T, dtype=torch.int64, device="cuda")
        tq.tq_pages_assign(paged.page_table, paged.seq_lens, _dev(torch, [T] * B), P, pages, free, count, after, count, offsets, slots, work,
                           status)
        k, v = (torch.randn((B, H, T, d), device="cuda").half() for _ in range(2))
        for cache in (paged, plain):
            tq.tq_kv_quantize_append(cache, k, v, status)
        assert paged.seq_lens.tolist() == after.tolist() == plain.seq_lens.tolist()
    n = plain.seq_lens.tolist()[0]
    assert n == 65 and count.tolist() == [pages - 3 * 5] and int(status.item()) == 0
    for a, b in zip(paged.arrays_token_major(), plain.arrays_token_major()):
        assert torch.equal(a[:, :, :n], b[:, :, :n])
    q = torch.randn((B, 8, d), device="cuda").half()
    outs = []
    for cache in (paged, plain):
        o, m, l = tq.alloc_partials(B, 8, d, 2)
        out = torch.empty((B, 8, d), device="cuda")
        tq.tq_sdpa_int4_decode(cache, q, 0.09, 2, o, m, l, status)
        tq.tq_sdpa_int4_combine(o, m, l, out)
        outs.append(out)
    assert torch.equal(*outs) and outs[0].abs().sum() > 0
