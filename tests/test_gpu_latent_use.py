"""Latent attention as a server uses it: other streams, captured graphs, side by side, many sequences, caches and tensors beyond
4 GB, one workspace for every shape, calls that the binding refuses, waits that run out."""
import numpy as np
import pytest

import latent_ref as L
import serving_ref as R
from test_gpu_latent import _check, _check_decode, _dev, _filled, _operands, _queries, _rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2604_16957_b200 import tq
    assert torch.cuda.is_available()
    return tq, torch


def test_streams_side_by_side(gpu):
    """Decode and prompt attention on two streams at a time, each with a workspace of its own, against the same calls one after the
    other on the default stream: bit for bit."""
    tq, torch = gpu
    rng = np.random.default_rng(1)
    jobs = []
    for seed, H in ((3, 40), (4, 16)):
        cache, _ = _filled(tq, torch, [3000, 70, 900], 512, 16, "fp16", seed, cap=3200)
        jobs.append(dict(cache=cache, q=_queries(torch, 3, H, 512, "bf16"), H=H, ops=_operands(torch, rng, [300, 40], [300, 40], 3, 128, "bf16", "fused"),
                         at=_dev(torch, [0, 300, 340])))

    def run(j, stream=None):
        work = tq.alloc_latent_workspace(3, j["H"], 512)
        outs = [torch.zeros((3, j["H"], 512), device="cuda") for _ in range(20)] + [torch.zeros((340, 3, 128), device="cuda") for _ in range(5)]
        torch.cuda.synchronize()
        for o in outs[:20]:
            tq.tq_sdpa_latent_decode(j["cache"], *j["q"], 0.05, 0, 0, work, o, stream=stream)
        for o in outs[20:]:
            tq.tq_sdpa_latent_prompt(*j["ops"], j["at"], j["at"], 0.07, o, stream=stream)
        return outs

    want = [run(j) for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [run(j, s) for j, s in zip(jobs, streams)]
    for s in streams:
        s.synchronize()
    for a, b in zip(want, got):
        for x, y in zip(a, b):
            assert torch.equal(x, y) and x.abs().sum() > 0


def test_captured_decode_follows_the_lengths(gpu):
    """One captured launch, replayed with other lengths, pages and queries in the same tensors; two graphs on two streams."""
    tq, torch = gpu
    cache, values = _filled(tq, torch, [5000, 300, 2500], 256, 16, "fp16", 9)
    jobs = []
    for H in (8, 70):
        q_c, q_r = _queries(torch, 3, H, 256, "fp16")
        out, work = torch.zeros((3, H, 256), device="cuda"), tq.alloc_latent_workspace(3, H, 256)
        call = lambda q_c=q_c, q_r=q_r, out=out, work=work: tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.06, 0, 0, work, out)  # noqa: E731
        call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(5):
                call()
        jobs.append((g, q_c, q_r, out, call))
    for lens in ([5000, 300, 2500], [0, 1, 64], [4999, 0, 0], [17, 300, 2049]):
        cache.seq_lens.copy_(_dev(torch, lens))
        for g, q_c, q_r, out, _ in jobs:
            q_c.copy_(torch.randn_like(q_c.float()).half())
            out.fill_(7.0)
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        for (g, *_), s in zip(jobs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for g, q_c, q_r, out, call in jobs:
            cut = [tuple(x[:n] for x in v) for v, n in zip(values, lens)]
            _check_decode(torch, out, q_c, q_r, cut, 0.06, 0)
            g.replay()
            call()                                                 # the same workspace, eagerly behind the graph
            _check_decode(torch, out, q_c, q_r, cut, 0.06, 0)


def test_captured_prompt_follows_the_offsets(gpu):
    tq, torch = gpu
    rng = np.random.default_rng(2)
    n, H, d = 400, 3, 128
    ops = _operands(torch, rng, [n], [n], H, d, "fp16", "fused")
    at, out = _dev(torch, [0, 0, 0, 0]), torch.zeros((n, H, d), device="cuda")
    tq.tq_sdpa_latent_prompt(*ops, at, at, 0.07, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tq.tq_sdpa_latent_prompt(*ops, at, at, 0.07, out)
    for lens in ([400, 0, 0], [1, 2, 3], [0, 129, 200], [100, 100, 200]):
        cum = np.concatenate([[0], np.cumsum(lens)]).tolist()
        at.copy_(torch.tensor(cum, dtype=torch.int32))
        out.fill_(5.0)
        g.replay()
        _check(torch, out, ops, cum, cum, 0.07, True, 0)
        assert torch.all(out[cum[-1]:] == 5.0)


@pytest.mark.parametrize("H", [4, 100])
def test_many_sequences(gpu, H):
    """More sequences than a round of the kernel's scan, most of them short or empty."""
    tq, torch = gpu
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 40, 1300).tolist()
    lens[7], lens[700], lens[1299] = 700, 3000, 33
    cache, values = _filled(tq, torch, lens, 128, 16, "bf16", 6)
    q_c, q_r = _queries(torch, 1300, H, 128, "bf16")
    out, status = torch.full((1300, H, 128), 9.0, device="cuda"), _dev(torch, [0])
    tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.07, 0, 0, tq.alloc_latent_workspace(1300, H, 128), out, status)
    assert int(status.item()) == tq.TQ_STATUS_EMPTY_SEQ
    _check_decode(torch, out, q_c, q_r, values, 0.07, 0)


def test_one_workspace_for_batches_of_any_shape(gpu):
    tq, torch = gpu
    shapes = [([9000, 50], 16, 512), ([2500, 700] * 16, 8, 128), ([3000], 100, 256), ([1500] * 20, 32, 512), ([30000], 1, 128), ([20, 2500, 300] * 5, 64, 256)]
    work = torch.randint(0, 256, (max(int(tq._lib.tq_latent_workspace_bytes(len(l), H, d)) for l, H, d in shapes),), dtype=torch.uint8, device="cuda")
    filled = [_filled(tq, torch, l, d, 0, "fp16", 40 + i) for i, (l, H, d) in enumerate(shapes)]
    for turn in range(2):
        for (lens, H, d), (cache, values) in zip(shapes, filled):
            q_c, q_r = _queries(torch, len(lens), H, d, "fp16")
            out = torch.full((len(lens), H, d), 3.0, device="cuda")
            tq.tq_sdpa_latent_decode(cache, q_c, q_r, (d + 64) ** -0.5, 0, 0, work, out)
            _check_decode(torch, out, q_c, q_r, values, (d + 64) ** -0.5, 0)


def test_results_do_not_depend_on_the_run(gpu):
    """The same call twice gives the same bits: no atomics on results, a fixed split."""
    tq, torch = gpu
    for H in (16, 32, 128):
        cache, _ = _filled(tq, torch, [20000, 300], 512, 64, "bf16", 30)
        q_c, q_r = _queries(torch, 2, H, 512, "bf16")
        work = tq.alloc_latent_workspace(2, H, 512)
        a, b = (torch.empty((2, H, 512), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.05, 0, 0, work, a)
        for _ in range(10):
            work.fill_(0xFF)
            tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.05, 0, 0, work, b)
            assert torch.equal(a, b)


def test_cache_beyond_4_gb(gpu):
    """The last sequence of a contiguous cache of 5.4 GB, and the last pages of a pool of that size: append, gather, decode."""
    tq, torch = gpu
    rng = np.random.default_rng(8)
    d_c, n = 512, 300
    for paged in (False, True):
        if paged:
            pages = 65 * 1024
            cache = tq.PagedLatentCache.over(torch.empty((pages, 8, tq.TQ_BLOCK_LATENT_BYTES(d_c)), dtype=torch.uint8, device="cuda"),
                                             _dev(torch, [n]), _dev(torch, [[pages - 1, pages - 3, pages - 2]]))
            slots = R.slots_of([0], [n], [[pages - 1, pages - 3, pages - 2]], 128)
        else:
            cache = tq.LatentCache.over(torch.empty((65, 8192, tq.TQ_BLOCK_LATENT_BYTES(d_c)), dtype=torch.uint8, device="cuda"),
                                        _dev(torch, [0] * 64 + [n]))
            slots = np.arange(n) + 64 * 131072
        assert cache.blocks.numel() > 1 << 32
        c, r = _rows(torch, rng, n, d_c, "fp16")
        s = torch.from_numpy(slots).cuda()
        tq.tq_latent_append(cache, c, r, s)
        co, ro = torch.empty((n, d_c), device="cuda"), torch.empty((n, 64), device="cuda")
        tq.tq_latent_gather(cache, s, co, ro)
        model = L.Cache(304, d_c)
        model.append(c, r, np.arange(n))
        values = model.values(np.arange(n))
        assert np.allclose(co.cpu().numpy(), values[0], rtol=2.0 ** -22) and np.allclose(ro.cpu().numpy(), values[1], rtol=2.0 ** -22)
        B = 1 if paged else 65
        q_c, q_r = _queries(torch, B, 16, d_c, "fp16")
        out = torch.full((B, 16, d_c), 3.0, device="cuda")
        tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.005, 0, 0, tq.alloc_latent_workspace(B, 16, d_c), out)
        _check_decode(torch, out[-1:], q_c[-1:], q_r[-1:], [values], 0.005, 0)
        assert torch.all(out[:-1] == 0)
        del cache
        torch.cuda.empty_cache()


def test_prompt_rows_beyond_4_gb(gpu):
    """Sequences at the far end of packed tensors of more than 2^31 elements."""
    tq, torch = gpu
    n, H, d = 70000, 128, 128
    kv = torch.empty((n, H, 2 * d), dtype=torch.bfloat16, device="cuda")
    q = torch.empty((n, H, d + 64), dtype=torch.bfloat16, device="cuda")
    k_r = torch.randn((n, 64), device="cuda").bfloat16()
    assert kv.numel() > 1 << 31
    kv[-300:], q[-300:] = torch.randn((300, H, 2 * d), device="cuda").bfloat16(), torch.randn((300, H, d + 64), device="cuda").bfloat16()
    out = torch.empty((n, H, d), dtype=torch.bfloat16, device="cuda")
    out[-320:] = 5.0
    at = _dev(torch, [n - 300, n - 100, n - 4])
    ops = (q[..., :d], q[..., d:], kv[..., :d], k_r, kv[..., d:])
    tq.tq_sdpa_latent_prompt(*ops, at, at, 0.07, out)
    assert torch.all(out[-320:-300] == 5.0) and torch.all(out[-4:] == 5.0)
    tail = slice(n - 300, n)
    few = tuple((x[tail, :3] if x.dim() == 3 else x[tail]) for x in ops)
    _check(torch, out[tail, :3], few, [0, 200, 296], [0, 200, 296], 0.07, True, 0)
    few = tuple((x[tail, -2:] if x.dim() == 3 else x[tail]) for x in ops)
    _check(torch, out[tail, -2:], few, [0, 200, 296], [0, 200, 296], 0.07, True, 0)


def test_the_binding_refuses(gpu):
    """Shapes, types and strides that the library could not use raise before anything is launched."""
    tq, torch = gpu
    cache = tq.LatentCache(2, 64, 256)
    kv8 = tq.KV8Cache(2, 2, 64, 128)
    work = tq.alloc_latent_workspace(2, 8, 256)
    z = lambda *s, t=torch.float16: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    slots, at = z(3, t=torch.int64), _dev(torch, [0, 3])
    f32, bf = torch.float32, torch.bfloat16
    app, gat, dec, pro = tq.tq_latent_append, tq.tq_latent_gather, tq.tq_sdpa_latent_decode, tq.tq_sdpa_latent_prompt
    qc, qr, o = z(2, 8, 256), z(2, 8, 64), z(2, 8, 256)
    p = dict(q_n=z(3, 4, 128), q_r=z(3, 4, 64), k_n=z(3, 4, 128), k_r=z(3, 64), v=z(3, 4, 128), q_offsets=at, kv_offsets=at, attn_scale=1.0, out=z(3, 4, 128))
    bad = [
        lambda: app(kv8, z(3, 256), z(3, 64), slots),
        lambda: app(cache, z(3, 128), z(3, 64), slots),
        lambda: app(cache, z(3, 256), z(3, 32), slots),
        lambda: app(cache, z(2, 256), z(2, 64), slots),
        lambda: app(cache, z(3, 256, t=f32), z(3, 64, t=f32), slots),
        lambda: app(cache, z(3, 256), z(3, 64, t=bf), slots),
        lambda: app(cache, z(256, 3).T, z(3, 64), slots),
        lambda: app(cache, z(1, 256).expand(3, 256), z(3, 64), slots),
        lambda: app(cache, z(3, 260)[:, 4:], z(3, 64), slots),
        lambda: app(cache, z(3, 256), z(3, 64), slots.int()),
        lambda: app(cache, z(3, 256).cpu(), z(3, 64), slots),
        lambda: gat(cache, slots, z(3, 256), z(3, 64, t=f32)),
        lambda: gat(cache, slots, z(3, 257)[:, :256], z(3, 64)),
        lambda: gat(cache, slots, z(2, 256), z(2, 64)),
        lambda: dec(kv8, qc, qr, 1.0, 0, 0, work, o),
        lambda: dec(cache, z(3, 8, 256), z(3, 8, 64), 1.0, 0, 0, work, z(3, 8, 256)),
        lambda: dec(cache, qc, z(2, 7, 64), 1.0, 0, 0, work, o),
        lambda: dec(cache, qc, z(2, 8, 128)[..., ::2], 1.0, 0, 0, work, o),
        lambda: dec(cache, z(2, 8, 260)[..., :256].transpose(0, 1).contiguous().transpose(0, 1)[..., :255], qr, 1.0, 0, 0, work, z(2, 8, 255)),
        lambda: dec(cache, qc, qr.bfloat16(), 1.0, 0, 0, work, o),
        lambda: dec(cache, qc.float(), qr.float(), 1.0, 0, 0, work, o.float()),
        lambda: dec(cache, qc, qr, 1.0, 0, 0, work, o.bfloat16()),
        lambda: dec(cache, qc, qr, 1.0, 0, 0, work[:1000], o),
        lambda: dec(cache, qc, qr, 1.0, -1, 0, work, o),
        lambda: dec(cache, qc, qr, 1.0, 0, 0, work, z(2, 256, 8).transpose(1, 2)),
        lambda: dec(cache, z(1, 8, 256).expand(2, 8, 256), qr, 1.0, 0, 0, work, o),
        lambda: pro(**{**p, "q_n": z(3, 4, 96), "out": z(3, 4, 96)}),
        lambda: pro(**{**p, "k_n": z(3, 2, 128)}),
        lambda: pro(**{**p, "k_r": z(2, 64)}),
        lambda: pro(**{**p, "k_r": z(3, 64, t=bf)}),
        lambda: pro(**{**p, "v": z(4, 4, 128)}),
        lambda: pro(**{**p, "kv_offsets": _dev(torch, [0, 1, 3])}),
        lambda: pro(**{**p, "causal": False, "window": 4}),
        lambda: pro(**{**p, "k_n": z(3, 1, 128).expand(3, 4, 128)}),
        lambda: pro(**{**p, "out": z(3, 4, 64)}),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(tq.TqError):
            call()
            raise AssertionError(i)
    # nothing to do is no error
    app(cache, z(0, 256), z(0, 64), slots[:0])
    gat(cache, slots[:0], z(0, 256), z(0, 64))
    pro(z(0, 4, 64), z(0, 4, 64), z(0, 4, 64), z(0, 64), z(0, 4, 64), _dev(torch, [0, 0]), _dev(torch, [0, 0]), 1.0, z(0, 4, 64))
    # queries without a single key give zeros
    out = torch.full((3, 4, 128), 7.0, dtype=torch.float16, device="cuda")
    pro(**{**p, "k_n": z(0, 4, 128), "k_r": z(0, 64), "v": z(0, 4, 128), "kv_offsets": _dev(torch, [0, 0]), "out": out})
    assert torch.all(out == 0)
    # a single row or head of any stride
    app(cache, z(1, 300).as_strided((1, 256), (3, 1)), z(1, 64), slots[:1])
    dec(tq.LatentCache(1, 64, 256), z(1, 8, 256).as_strided((1, 8, 256), (5, 256, 1)), z(1, 8, 64), 1.0, 0, 0, work, z(1, 8, 256))
    torch.cuda.synchronize()


def test_tensors_under_a_cache(gpu):
    """A cache follows its tensors' storage; one of another shape is refused."""
    tq, torch = gpu
    cache, values = _filled(tq, torch, [100], 128, 0, "fp16", 3, cap=160)
    q_c, q_r = _queries(torch, 1, 4, 128, "fp16")
    out, work = torch.empty((1, 4, 128), device="cuda"), tq.alloc_latent_workspace(1, 4, 128)
    other = cache.blocks.clone()
    cache.blocks.zero_()
    cache.blocks.set_(other.untyped_storage(), 0, other.shape)
    tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.07, 0, 0, work, out)
    _check_decode(torch, out, q_c, q_r, values, 0.07, 0)
    cache.blocks.resize_(1, 5, other.shape[2])
    with pytest.raises(tq.TqError):
        tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.07, 0, 0, work, out)


# ------------------------------------------------------------------------------------------------------------ waits

def _hooked(tq, torch, call, limit, fault):
    tq._test_hook(tq.HOOK_SPIN_LIMIT, limit)
    tq._test_hook(tq.HOOK_FAULT_BLOCK, fault)
    try:
        call()
        torch.cuda.synchronize()   # returns
    finally:
        tq._test_hook(tq.HOOK_SPIN_LIMIT, 0)
        tq._test_hook(tq.HOOK_FAULT_BLOCK, -1)


# one thread block's worth and cut sequences, with every number of columns; many pieces of work in a thread block
WAITS = [([1000], 16), ([20000, 700], 20), ([9000, 3000, 50], 64), ([100, 30] * 200, 16), ([20, 2500, 300] * 15, 128)]


@pytest.mark.parametrize("lens,H", WAITS)
@pytest.mark.parametrize("fault", [0, 2])
def test_decode_gives_up_on_a_tile(gpu, lens, H, fault):
    """The operands of one tile of every thread block are never announced: status, no write elsewhere, and the next call is
    right."""
    tq, torch = gpu
    B, d_c = len(lens), 512
    cache, values = _filled(tq, torch, lens, d_c, 16, "fp16", 3)
    q_c, q_r = _queries(torch, B, H, d_c, "bf16")
    work, status = tq.alloc_latent_workspace(B, H, d_c), _dev(torch, [0])
    work.fill_(0x7F)
    guard = torch.full((B * H * d_c + 128,), 5.0, device="cuda")
    out = guard[64:-64].view(B, H, d_c)
    _hooked(tq, torch, lambda: tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.05, 0, 0, work, out, status), 100000, fault)
    # (a third tile is something that not every batch has in one thread block)
    assert int(status.item()) in ((tq.TQ_STATUS_TIMEOUT,) if fault == 0 else (0, tq.TQ_STATUS_TIMEOUT))
    assert torch.all(guard[:64] == 5.0) and torch.all(guard[-64:] == 5.0)
    status.zero_()
    tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.05, 0, 0, work, out, status)
    assert int(status.item()) == 0
    _check_decode(torch, out, q_c, q_r, values, 0.05, 0)


@pytest.mark.parametrize("lens,H", WAITS)
@pytest.mark.parametrize("limit", [1, 3000])
def test_decode_with_short_waits(gpu, lens, H, limit):
    """Whether a wait is caught depends on timing: the call returns either way, and a clean status means a right result."""
    tq, torch = gpu
    B, d_c = len(lens), 512
    cache, values = _filled(tq, torch, lens, d_c, 16, "fp16", 4)
    q_c, q_r = _queries(torch, B, H, d_c, "fp16")
    work, status = tq.alloc_latent_workspace(B, H, d_c), _dev(torch, [0])
    out = torch.empty((B, H, d_c), device="cuda")
    _hooked(tq, torch, lambda: tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.05, 0, 0, work, out, status), limit, -1)
    assert int(status.item()) in (0, tq.TQ_STATUS_TIMEOUT)
    if int(status.item()):
        tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.05, 0, 0, work, out)
    _check_decode(torch, out, q_c, q_r, values, 0.05, 0)


@pytest.mark.parametrize("lq,H,window", [([300], 3, 0), ([700, 40], 64, 0), ([130] * 30, 8, 100)])
@pytest.mark.parametrize("limit,fault", [(100000, 0), (100000, 1), (2000, -1)])
def test_prompt_gives_up_on_a_tile(gpu, lq, H, window, limit, fault):
    tq, torch = gpu
    ops = _operands(torch, np.random.default_rng(len(lq)), lq, lq, H, 128, "fp16", "fused")
    cum = np.concatenate([[0], np.cumsum(lq)]).tolist()
    at, status = _dev(torch, cum), _dev(torch, [0])
    guard = torch.full(((cum[-1] + 2) * H * 128,), 5.0, device="cuda").view(-1, H, 128)
    out = guard[1:-1]
    call = lambda: tq.tq_sdpa_latent_prompt(*ops, at, at, 0.07, out, window=window, status=status)  # noqa: E731
    _hooked(tq, torch, call, limit, fault)
    assert int(status.item()) == tq.TQ_STATUS_TIMEOUT if fault >= 0 else int(status.item()) in (0, tq.TQ_STATUS_TIMEOUT)
    assert torch.all(guard[0] == 5.0) and torch.all(guard[-1] == 5.0)
    status.zero_()
    call()
    assert int(status.item()) == 0
    few = [h for h in (0, H // 2, H - 1)]
    _check(torch, out[:, few], tuple(x[:, few] if x.dim() == 3 else x for x in ops), cum, cum, 0.07, True, window)
