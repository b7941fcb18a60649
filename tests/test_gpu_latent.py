"""Latent attention against its definitions in 64 bits (tests/latent_ref.py): the 8-bit cache, the absorbed form over it, the
expanded form over packed prompts, and a run of them together."""
import numpy as np
import pytest

import latent_ref as L
import serving_ref as R
from test_gpu_serving import _check_prompt, _types

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2604_16957_b200 import tq
    assert torch.cuda.is_available()
    return tq, torch


def _dev(torch, x, t=None):
    return torch.tensor(x, dtype=t or torch.int32, device="cuda")


# ----------------------------------------------------------------------------------------------------------- cache

def _cache(tq, torch, B, d_c, page, cap, seed):
    """A cache with junk in it (every byte 0xFF: codes 127, scales and positional keys NaN) and its page table."""
    if page == 0:
        c = tq.LatentCache(B, cap, d_c)
        c.blocks.fill_(0xFF)
        return c, None
    cols = -(-cap // page)
    c = tq.PagedLatentCache(B, page, cols, B * cols + 3, d_c)
    c.blocks.fill_(0xFF)
    table = np.random.default_rng(seed).permutation(B * cols + 3)[:B * cols].reshape(B, cols).astype(np.int32)
    c.page_table.copy_(torch.from_numpy(table))
    return c, table


def _rows(torch, rng, n, d_c, kind, fused=True):
    """Latents and positional keys whose sizes vary from token to token: slices of one tensor, or apart."""
    x = rng.standard_normal((n, d_c + 72)) * 10.0 ** rng.uniform(-2, 2, (n, 1))
    x[:, d_c + 8:] *= 10.0 ** rng.uniform(-2, 2, (n, 1))
    x = torch.from_numpy(x).to(_types(torch)[kind]).cuda()
    c, r = x[:, :d_c], x[:, d_c + 8:]
    return (c, r) if fused else (c.contiguous(), r.contiguous())


def _check_cache(cache, model, slots):
    got = L.read_device_cache(cache.blocks, model.d_c)
    s = np.unique(slots[slots >= 0])
    assert np.array_equal(got.a[s], model.a[s]) and np.array_equal(got.s[s], model.s[s])
    assert np.array_equal(got.codes[s], model.codes[s])
    assert np.array_equal(got.r[s].view(np.uint16) & 0x7fff, model.r[s].view(np.uint16) & 0x7fff)
    assert np.array_equal(got.r[s], model.r[s])


@pytest.mark.parametrize("B,d_c,page,kind,fused", [(1, 512, 0, "fp16", True), (3, 512, 16, "bf16", True), (2, 256, 64, "fp16", False),
                                                   (4, 128, 32, "bf16", True), (2, 128, 0, "fp16", False), (5, 256, 128, "bf16", True)])
def test_append_and_gather(gpu, B, d_c, page, kind, fused):
    """Prompts of odd lengths, then tokens one by one, rows of padding among them; bit for bit.  Nothing else changes."""
    tq, torch = gpu
    rng = np.random.default_rng(B + d_c)
    cap = 160
    cache, table = _cache(tq, torch, B, d_c, page, cap, 3)
    model = L.Cache(cache.blocks.numel() // (d_c + 136), d_c)
    lens, used, status = [0] * B, [], _dev(torch, [0])
    for new in ([37 + 11 * b for b in range(B)], [1] * B, [0, 5, 1, 2, 16][:B], [1] * B):
        slots = R.slots_of(lens, new, table, page, cap)
        slots = np.concatenate([slots, [-1, -7]])
        if new[0] == 1:
            slots = slots[rng.permutation(len(slots))]           # any order
        c, r = _rows(torch, rng, len(slots), d_c, kind, fused)
        tq.tq_latent_append(cache, c, r, torch.from_numpy(slots).cuda(), status)
        model.append(c, r, slots)
        lens = [a + b for a, b in zip(lens, new)]
        used.append(slots)
    used = np.concatenate(used)
    used = used[used >= 0]
    _check_cache(cache, model, used)
    got = L.read_device_cache(cache.blocks, d_c)
    rest = np.setdiff1d(np.arange(len(got.a)), used)
    assert np.all(got.codes[rest] == 127) and np.all(np.isnan(got.a[rest])) and np.all(np.isnan(got.r[rest])) and np.all(np.isnan(got.s[rest]))
    # read back, in any order, twice, with rows of zeros
    ask = np.concatenate([used[rng.permutation(len(used))], used[:3], [-1]])
    want = model.values(np.where(ask < 0, 0, ask))
    for t in (torch.float32, torch.float16, torch.bfloat16):
        co, ro = torch.full((len(ask), d_c), 7.0, dtype=t, device="cuda"), torch.full((len(ask), 64), 7.0, dtype=t, device="cuda")
        tq.tq_latent_gather(cache, torch.from_numpy(ask).cuda(), co, ro, status)
        # two roundings in binary32 (of a / 127 and of the product), then the type's own, with half a step of fp16's subnormals
        eps = 2.0 ** -23 + (0.0 if t == torch.float32 else torch.finfo(t).eps / 2)
        for out, ref in ((co, want[0]), (ro, want[1])):
            ref = np.where(ask[:, None] < 0, 0.0, ref)
            out = out.double().cpu().numpy()
            small = np.abs(ref) < 65504 if t == torch.float16 else np.ones_like(ref, bool)
            assert np.all(np.abs(out - ref)[small] <= (np.abs(ref) * eps + (2.0 ** -25 if t == torch.float16 else 0.0))[small])
    assert int(status.item()) == 0


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("d_c", [128, 512])
def test_append_edge_values(gpu, d_c, kind):
    """Zeros, single values, subnormals, halves between codes, NaN, infinities, values beyond 2^64 and below 2^-64."""
    tq, torch = gpu
    t = _types(torch)[kind]
    rows, n = [], d_c
    def row(c, r=0.0):  # noqa: E306
        x = torch.zeros(d_c + 64, dtype=torch.float64)
        x[:d_c], x[d_c:] = c, r
        rows.append(x)
        return x
    row(0.0)
    row(0.0)[5] = 1.0
    row(1.0)[d_c + 63] = -3.0
    row(torch.arange(n) - 63.5)[7] = 127.0                         # 127 x / a = x: halves, to even
    row(torch.finfo(t).smallest_normal / 8)[d_c] = torch.finfo(t).smallest_normal / 8
    row(float("nan"), float("nan"))
    row(0.5, 0.25)[3] = float("nan")
    row(0.5, 0.25)[[3, d_c + 1]] = float("inf")
    row(0.5, 0.25)[[4, d_c + 2]] = -float("inf")
    row(1.0, 1e-3)[d_c] = 60000.0
    row(1e-7, 6e-8)
    if kind == "bf16":
        row(2.0 ** 70, -2.0 ** 64)[1] = 2.0 ** 63
        row(2.0 ** -65, 2.0 ** -120)
        row(2.0 ** -64, 2.0 ** -130)[0] = -2.0 ** -70
        row(2.0 ** 64, 1.0)[d_c + 5] = 2.0 ** -31                  # kept, and 2^-36 of the largest: a step of 2^-39
        row(1.0, 1.0)[d_c + 5] = 1.171875 * 2.0 ** -36
    x = torch.stack(rows).to(t).cuda()
    cache, _ = _cache(tq, torch, 1, d_c, 0, 32, 0)
    slots = np.arange(len(rows))[::-1].copy()
    tq.tq_latent_append(cache, x[:, :d_c], x[:, d_c:], torch.from_numpy(slots).cuda())
    model = L.Cache(32, d_c)
    model.append(x[:, :d_c], x[:, d_c:], slots)
    _check_cache(cache, model, slots)


@pytest.mark.parametrize("d_c,n", [(512, 20001), (128, 90007)])
def test_append_and_gather_many(gpu, d_c, n):
    """So many rows that a warp has two on their way; an odd number of them, scattered over the cache."""
    tq, torch = gpu
    rng = np.random.default_rng(n)
    cache, _ = _cache(tq, torch, 1, d_c, 0, -(-n // 16) * 16, 0)
    slots = rng.permutation(cache.S_cap)[:n]
    slots[::97] = -1
    c, r = _rows(torch, rng, n, d_c, "bf16")
    s = torch.from_numpy(slots).cuda()
    tq.tq_latent_append(cache, c, r, s)
    model = L.Cache(cache.S_cap, d_c)
    model.append(c, r, slots)
    _check_cache(cache, model, slots)
    co, ro = torch.empty((n, d_c), device="cuda"), torch.empty((n, 64), device="cuda")
    tq.tq_latent_gather(cache, s, co, ro)
    on = slots >= 0
    want = model.values(np.where(on, slots, 0))
    for out, ref in ((co, want[0]), (ro, want[1])):
        ref = np.where(on[:, None], ref, 0.0)
        assert np.all(np.abs(out.double().cpu().numpy() - ref) <= 2.0 ** -23 * np.abs(ref))


def test_append_and_gather_refuse_bad_slots(gpu):
    tq, torch = gpu
    cache, _ = _cache(tq, torch, 2, 256, 0, 32, 0)
    status = _dev(torch, [0])
    c, r = _rows(torch, np.random.default_rng(1), 4, 256, "fp16", False)
    before = cache.blocks.clone()
    tq.tq_latent_append(cache, c, r, _dev(torch, [64, 1 << 40, -1, (1 << 62)], torch.int64), status)
    assert int(status.item()) == tq.TQ_STATUS_BAD_SLOT and torch.equal(before, cache.blocks)
    status.zero_()
    tq.tq_latent_append(cache, c, r, _dev(torch, [63, 64, 0, -1], torch.int64), status)
    model = L.Cache(64, 256)
    model.append(c, r, np.array([63, -1, 0, -1]))
    _check_cache(cache, model, np.array([63, 0]))
    assert int(status.item()) == tq.TQ_STATUS_BAD_SLOT
    status.zero_()
    co, ro = torch.full((4, 256), 7.0, device="cuda"), torch.full((4, 64), 7.0, device="cuda")
    tq.tq_latent_gather(cache, _dev(torch, [0, 64, 1 << 40, -5], torch.int64), co, ro, status)
    assert int(status.item()) == tq.TQ_STATUS_BAD_SLOT and torch.all(co[1:] == 0) and torch.all(ro[1:] == 0) and torch.all(co[0] != 7.0)


# ---------------------------------------------------------------------------------------------------------- decode

def _filled(tq, torch, lens, d_c, page, kind, seed, cap=None):
    """A cache filled through append (one call), with the values it holds."""
    rng = np.random.default_rng(seed)
    B = len(lens)
    cap = cap or -(-max(max(lens), 1) // 16) * 16
    cache, table = _cache(tq, torch, B, d_c, page, cap, seed)
    slots = R.slots_of([0] * B, lens, table, page, cap)
    model = L.Cache(cache.blocks.numel() // (d_c + 136), d_c)
    if len(slots):
        x = rng.standard_normal((len(slots), d_c + 64)) * 10.0 ** rng.uniform(-0.5, 0.5, (len(slots), 1))
        x[:, d_c:d_c + 2] *= 5.0
        x = torch.from_numpy(x).to(_types(torch)[kind]).cuda()
        tq.tq_latent_append(cache, x[:, :d_c], x[:, d_c:], torch.from_numpy(slots).cuda())
        model.append(x[:, :d_c], x[:, d_c:], slots)
    cache.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    starts = np.concatenate([[0], np.cumsum(lens)])
    return cache, [model.values(slots[starts[b]:starts[b + 1]]) for b in range(B)]


def _queries(torch, B, H, d_c, kind, layout="split"):
    """q_c, q_r of N(0, 1): slices of one tensor, heads before rows, or apart."""
    t = _types(torch)[kind]
    if layout == "fused":
        x = torch.randn((B, H, d_c + 64), device="cuda").to(t)
        return x[..., :d_c], x[..., d_c:]
    if layout == "heads":
        return torch.randn((H, B, d_c), device="cuda").to(t).transpose(0, 1), torch.randn((B, H, 192), device="cuda").to(t)[..., 128:]
    return torch.randn((B, H, d_c), device="cuda").to(t), torch.randn((B, H, 64), device="cuda").to(t)


def _check_decode(torch, out, q_c, q_r, values, alpha, window, rows=None):
    d_c = q_c.shape[-1]
    qc, qr, od = q_c.double().cpu(), q_r.double().cpu(), out.double().cpu()
    out_eps = 0.0 if out.dtype == torch.float32 else torch.finfo(out.dtype).eps / 2
    worst = 0.0
    for b in range(len(values)) if rows is None else rows:
        c, r = values[b]
        n = len(c)
        lo = max(0, n - window) if window else 0
        if n == 0:
            assert torch.all(od[b] == 0)
            continue
        ref, weighed, p, mag = L.attention(qc[b], qr[b], c[lo:], r[lo:], alpha)
        tol = L.bound(ref, weighed, p, mag, n - lo, d_c, c[lo:], out_eps)
        if out.dtype == torch.float16:
            tol = tol + 2.0 ** -25  # half a step of the subnormals
        err = (od[b] - ref).abs()
        assert torch.all(err <= tol), (b, float((err / tol).max()))
        worst = max(worst, float((err / tol).max()))
    return worst


DECODES = [
    # lens, H, d_c, page, kind, window, layout
    ([1], 1, 512, 0, "fp16", 0, "split"), ([17], 16, 512, 0, "fp16", 0, "fused"), ([64], 5, 128, 0, "bf16", 0, "heads"),
    ([65, 63, 0, 128, 1], 16, 512, 16, "bf16", 0, "fused"), ([1000], 128, 512, 0, "bf16", 0, "split"),
    ([5000, 0, 33, 16, 2047], 64, 512, 64, "bf16", 0, "heads"), ([700, 1300], 20, 256, 16, "fp16", 0, "split"),
    ([3001], 32, 256, 0, "fp16", 0, "fused"), ([100, 1, 900], 33, 128, 32, "bf16", 0, "split"), ([500, 77], 100, 512, 16, "fp16", 0, "heads"),
    ([2500], 17, 512, 128, "bf16", 0, "split"), ([1500, 100, 64, 63], 12, 512, 16, "fp16", 64, "fused"), ([4000], 64, 256, 0, "fp16", 1000, "split"),
    ([2000, 5], 40, 512, 64, "bf16", 1, "split"), ([20] * 300, 8, 128, 16, "fp16", 0, "fused"), ([20000], 16, 512, 0, "fp16", 0, "split"),
    ([333] * 40, 130, 256, 16, "bf16", 0, "split"), ([70, 3], 300, 128, 0, "fp16", 50, "heads"), ([6000, 4000, 9000], 128, 512, 64, "fp16", 0, "split")]


@pytest.mark.parametrize("lens,H,d_c,page,kind,window,layout", DECODES)
def test_latent_decode(gpu, lens, H, d_c, page, kind, window, layout):
    tq, torch = gpu
    B = len(lens)
    cache, values = _filled(tq, torch, lens, d_c, page, kind, len(lens) + H)
    q_c, q_r = _queries(torch, B, H, d_c, kind, layout)
    alpha, status = (d_c + 64) ** -0.5, _dev(torch, [0])
    work = tq.alloc_latent_workspace(B, H, d_c)
    work.fill_(0xFF)                                               # its contents mean nothing
    for out_t in (torch.float32, _types(torch)[kind]):
        guard = torch.full(((B + 2) * H * d_c,), 5.0, dtype=out_t, device="cuda")
        out = guard.view(-1, H, d_c)[1:-1]
        for bound in (0, max(lens) + 3):
            status.zero_()
            tq.tq_sdpa_latent_decode(cache, q_c, q_r, alpha, window, bound, work, out, status)
            assert int(status.item()) == (tq.TQ_STATUS_EMPTY_SEQ if 0 in lens else 0)
            _check_decode(torch, out, q_c, q_r, values, alpha, window)
        assert torch.all(guard.view(-1, H, d_c)[0] == 5.0) and torch.all(guard.view(-1, H, d_c)[-1] == 5.0)


def test_latent_decode_of_a_cache_of_the_other_type(gpu):
    """fp16 queries over latents that were bf16, and the other way round: the cache has no type."""
    tq, torch = gpu
    for kind, other in (("fp16", "bf16"), ("bf16", "fp16")):
        cache, values = _filled(tq, torch, [300, 20], 512, 16, other, 5)
        q_c, q_r = _queries(torch, 2, 16, 512, kind)
        out = torch.empty((2, 16, 512), device="cuda")
        tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.05, 0, 0, tq.alloc_latent_workspace(2, 16, 512), out)
        _check_decode(torch, out, q_c, q_r, values, 0.05, 0)


@pytest.mark.parametrize("n,H", [(1, 3), (50, 16), (3000, 20), (3000, 64)])
@pytest.mark.parametrize("alpha", [-0.05, 0.0, 1.0, 30.0])
def test_latent_decode_of_odd_scales(gpu, n, H, alpha):
    """A negative scale, none, and scores in the thousands, whose largest takes everything."""
    tq, torch = gpu
    cache, values = _filled(tq, torch, [n], 512, 0, "fp16", 6)
    q_c, q_r = _queries(torch, 1, H, 512, "fp16")
    out = torch.empty((1, H, 512), device="cuda")
    tq.tq_sdpa_latent_decode(cache, q_c, q_r, alpha, 0, 0, tq.alloc_latent_workspace(1, H, 512), out)
    _check_decode(torch, out, q_c, q_r, values, alpha, 0)
    tq.tq_sdpa_latent_decode(cache, q_c, q_r, float("nan"), 0, 0, tq.alloc_latent_workspace(1, H, 512), out)
    assert torch.all(torch.isnan(out))


@pytest.mark.parametrize("n,H", [(40, 16), (5000, 16), (700, 70)])
def test_a_query_of_infinities_or_nans_stays_in_its_head(gpu, n, H):
    tq, torch = gpu
    for kind in ("fp16", "bf16"):
        cache, values = _filled(tq, torch, [n, n], 256, 16, kind, 7)
        q_c, q_r = _queries(torch, 2, H, 256, kind)
        want = torch.empty((2, H, 256), device="cuda")
        work = tq.alloc_latent_workspace(2, H, 256)
        tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.06, 0, 0, work, want)
        q_c[0, 3, 17], q_c[1, H - 1, 255], q_r[0, 0, 63] = float("nan"), float("inf"), -float("inf")
        q_r[1, 2] = float("nan")
        got = torch.empty((2, H, 256), device="cuda")
        tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.06, 0, 0, work, got)
        bad = torch.zeros((2, H), dtype=torch.bool)
        bad[0, 3] = bad[1, H - 1] = bad[0, 0] = bad[1, 2] = True
        assert torch.all(torch.isnan(got[bad])) and torch.equal(got[~bad], want[~bad])


@pytest.mark.parametrize("H", [4, 64])
@pytest.mark.parametrize("n", [300, 6000])
def test_latent_decode_of_values_of_very_different_size(gpu, n, H):
    """Ranges from 2^-40 to 2^40 side by side (positional keys decide the scores): the largest token with next to no
    weight, and with all of it."""
    tq, torch = gpu
    d_c = 128
    rng = np.random.default_rng(9)
    cache, _ = _cache(tq, torch, 1, d_c, 0, -(-n // 16) * 16, 0)
    size = 2.0 ** rng.integers(-40, 20, (n, 1)).astype(np.float64)
    size[n // 3] = 2.0 ** 40
    x = torch.from_numpy(np.concatenate([rng.standard_normal((n, d_c)) * size, rng.standard_normal((n, 64))], 1)).bfloat16().cuda()
    x[n // 3, d_c:] = 0.0
    x[n // 3, d_c] = 4.0
    slots = np.arange(n)
    tq.tq_latent_append(cache, x[:, :d_c], x[:, d_c:], torch.from_numpy(slots).cuda())
    cache.seq_lens.fill_(n)
    model = L.Cache(cache.S_cap, d_c)
    model.append(x[:, :d_c], x[:, d_c:], slots)
    c, r = model.values(slots)
    q_c, q_r = torch.zeros((1, H, d_c), device="cuda").bfloat16(), torch.randn((1, H, 64), device="cuda").bfloat16()
    q_r[0, 0], q_r[0, 1], q_r[0, 2] = 0.0, 0.0, 0.0
    q_r[0, 1, 0], q_r[0, 2, 0] = -40.0, 40.0
    out = torch.empty((1, H, d_c), device="cuda")
    tq.tq_sdpa_latent_decode(cache, q_c, q_r, 1.0, 0, 0, tq.alloc_latent_workspace(1, H, d_c), out)
    ref, weighed, p, mag = L.attention(q_c[0].double().cpu(), q_r[0].double().cpu(), c, r, 1.0)
    z = torch.softmax(torch.cat([q_c[0], q_r[0]], -1).double().cpu() @ torch.as_tensor(np.concatenate([c, r], 1)).T, -1)
    # 2^-33 of the largest contribution p_t a_t instead of the largest weight by the largest value
    tol = L.bound(ref, weighed, 0 * p, mag, n, d_c, c[:0], 0.0) + n * 2.0 ** -33 * (z * torch.as_tensor(model.a[:n])).amax(1, keepdim=True)
    err = (out[0].double().cpu() - ref).abs()
    assert torch.all(err <= tol), float((err / tol).max())


@pytest.mark.parametrize("n", [200, 4000, 20000])
@pytest.mark.parametrize("H", [2, 64])
def test_latent_decode_keeps_a_tail_of_small_weights(gpu, n, H):
    """One token far above the others, whose own weights of 2^-20 add up: the tail keeps its digits, wherever the large one
    stands."""
    tq, torch = gpu
    d_c = 128
    for where in (0, n // 2, n - 1):
        x = torch.zeros((n, d_c + 64), device="cuda")
        x[:, :d_c] = torch.from_numpy(np.random.default_rng(3).uniform(0.5, 1.0, (n, d_c))).cuda()
        x[where, :d_c] *= -1.0
        x[where, d_c] = 1.0
        x = x.half()
        cache, _ = _cache(tq, torch, 1, d_c, 0, -(-n // 16) * 16, 0)
        slots = np.arange(n)
        tq.tq_latent_append(cache, x[:, :d_c], x[:, d_c:], torch.from_numpy(slots).cuda())
        cache.seq_lens.fill_(n)
        model = L.Cache(cache.S_cap, d_c)
        model.append(x[:, :d_c], x[:, d_c:], slots)
        q_c, q_r = torch.zeros((1, H, d_c), device="cuda").half(), torch.zeros((1, H, 64), device="cuda").half()
        q_r[0, :, 0] = torch.linspace(10.0, 18.0, H)               # e^-10 .. e^-18 of the large one
        out = torch.empty((1, H, d_c), device="cuda")
        tq.tq_sdpa_latent_decode(cache, q_c, q_r, 1.0, 0, 0, tq.alloc_latent_workspace(1, H, d_c), out)
        c, r = model.values(slots)
        _check_decode(torch, out, q_c, q_r, [(c, r)], 1.0, 0)
        # the tail itself: what is left when the large token's share is taken away, by 2^-11 of each of its weights
        z = torch.softmax(torch.cat([q_c[0], q_r[0]], -1).double().cpu() @ torch.as_tensor(np.concatenate([c, r], 1)).T, -1)
        big = z[:, where:where + 1] * torch.as_tensor(c[where])[None, :]
        tail = z @ torch.as_tensor(c) - big
        err = (out[0].double().cpu() - big - tail).abs()
        assert torch.all(err <= 2.0 ** -10 * (big.abs() + tail.abs()) + n * 2.0 ** -33)


@pytest.mark.parametrize("size", [-1.3671875 * 2.0 ** 52, 1.3671875 * 2.0 ** -46, 1.3671875 * 2.0 ** 12, 1.3671875 * 2.0 ** 30])
@pytest.mark.parametrize("n,H", [(1, 1), (200, 16), (5000, 40)])
def test_latent_decode_of_scores_far_from_zero(gpu, n, H, size):
    """Equal scores of any size give the mean of the latents, whose ranges differ."""
    tq, torch = gpu
    d_c = 128
    rng = np.random.default_rng(4)
    x = torch.from_numpy(rng.standard_normal((n, d_c + 64))).bfloat16().cuda()
    x[:, d_c:] = 0.0
    x[:, d_c] = 1.0
    cache, _ = _cache(tq, torch, 1, d_c, 0, -(-n // 16) * 16, 0)
    slots = np.arange(n)
    tq.tq_latent_append(cache, x[:, :d_c], x[:, d_c:], torch.from_numpy(slots).cuda())
    cache.seq_lens.fill_(n)
    model = L.Cache(cache.S_cap, d_c)
    model.append(x[:, :d_c], x[:, d_c:], slots)
    q_c, q_r = torch.zeros((1, H, d_c), device="cuda").bfloat16(), torch.zeros((1, H, 64), device="cuda").bfloat16()
    q_r[..., 0] = size
    out = torch.empty((1, H, d_c), device="cuda")
    tq.tq_sdpa_latent_decode(cache, q_c, q_r, 1.0, 0, 0, tq.alloc_latent_workspace(1, H, d_c), out)
    c = torch.as_tensor(model.values(slots)[0])
    # each weight is rounded to fp16, and log2 of its token's range is off by 2^-22 (see latent_ref.bound)
    tol = c.abs().mean(0) * (2.0 ** -11 + 2.0 ** -17 + (n / 16 + 64) * 2.0 ** -24)
    assert torch.all((out[0].double().cpu() - c.mean(0)).abs() <= tol)


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("n,H,d_c", [(70, 16, 512), (3000, 16, 256), (500, 9, 128), (3000, 20, 512)])
def test_latent_decode_of_queries_at_the_limits(gpu, n, H, d_c, kind):
    """Heads whose channels are all as large as the largest, of either sign; whose two parts, or whose channels, differ by
    2^10; with one channel, or none; over rows of which all channels are as large.  Queries times 2^8 with a scale times
    2^-8 give the same bits."""
    tq, torch = gpu
    top = 2.0 - 2 * torch.finfo(_types(torch)[kind]).eps
    rng = np.random.default_rng(n + H)
    x = rng.standard_normal((n, d_c + 64))
    x[0, :d_c], x[1, :d_c], x[2, :d_c] = 1.0, -1.0, np.where(np.arange(d_c) % 2, 1.0, -1.0)
    x[:, 0] = 0.0
    x = torch.from_numpy(x).to(_types(torch)[kind]).cuda()
    cache, table = _cache(tq, torch, 1, d_c, 16, -(-n // 16) * 16, 3)
    slots = R.slots_of([0], [n], table, 16, cache.S_cap)
    tq.tq_latent_append(cache, x[:, :d_c], x[:, d_c:], torch.from_numpy(slots).cuda())
    cache.seq_lens.fill_(n)
    model = L.Cache(cache.blocks.numel() // (d_c + 136), d_c)
    model.append(x[:, :d_c], x[:, d_c:], slots)
    c, r = model.values(slots)
    q_c, q_r = torch.from_numpy(rng.standard_normal((1, H, d_c))), torch.from_numpy(rng.standard_normal((1, H, 64)))
    q_c[0, 0], q_c[0, 1] = top, -top
    q_c[0, 2] = torch.tensor([top, -top]).repeat(d_c // 2)
    q_r[0, 0], q_r[0, 1] = top, -top
    q_r[0, 3] *= 2.0 ** -10
    q_c[0, 4] *= 2.0 ** -10
    q_c[0, 5] = 0.0
    q_c[0, 5, 7] = top
    q_c[0, 6] *= 2.0 ** -10                                        # (the largest channel meets zeros)
    q_c[0, 6, 0] = top
    q_r[0, 6] *= 2.0 ** -10
    q_c[0, 7], q_c[0, 8], q_r[0, 8] = 0.0, 0.0, 0.0
    q_c, q_r = q_c.to(_types(torch)[kind]).cuda(), q_r.to(_types(torch)[kind]).cuda()
    work = tq.alloc_latent_workspace(1, H, d_c)
    out, same = torch.empty((1, H, d_c), device="cuda"), torch.empty((1, H, d_c), device="cuda")
    for alpha, rows in (((d_c + 64) ** -0.5, range(H)), (64.0, [6])):
        tq.tq_sdpa_latent_decode(cache, q_c, q_r, alpha, 0, 0, work, out)
        tq.tq_sdpa_latent_decode(cache, q_c * 256, q_r * 256, alpha / 256, 0, 0, work, same)
        assert torch.equal(out, same)
        for h in rows:
            ref, weighed, p, mag = L.attention(q_c[0, h:h + 1].double().cpu(), q_r[0, h:h + 1].double().cpu(), c, r, alpha)
            # a score is off by the query's rounding, 2^-26 of its largest channel; twice that, numerator and denominator
            delta = alpha * 2.0 ** -26 * float(q_c[0, h].abs().max()) * float(np.abs(c).sum(1).max())
            tol = L.bound(ref, weighed, p, mag, n, d_c, c, 0.0) + weighed * 2.0 * np.expm1(delta)
            err = (out[0, h:h + 1].double().cpu() - ref).abs()
            assert torch.all(err <= tol), (h, alpha, float((err / tol).max()))


def test_latent_decode_status_bits(gpu):
    tq, torch = gpu
    cache, values = _filled(tq, torch, [64, 64], 256, 16, "fp16", 8)
    q_c, q_r = _queries(torch, 2, 4, 256, "fp16")
    work, status = tq.alloc_latent_workspace(2, 4, 256), _dev(torch, [0])
    out = torch.empty((2, 4, 256), device="cuda")
    run = lambda: tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.06, 0, 0, work, out, status)  # noqa: E731
    cache.seq_lens.copy_(_dev(torch, [65, -1]))                    # S_cap is 64
    run()
    assert int(status.item()) == tq.TQ_STATUS_BAD_LEN | tq.TQ_STATUS_EMPTY_SEQ and torch.all(out[1] == 0)
    _check_decode(torch, out, q_c, q_r, values, 0.06, 0, rows=[0])
    cache.seq_lens.copy_(_dev(torch, [64, 64]))
    for bad in (-1, cache.num_pages, 1 << 30):
        status.zero_()
        held = cache.page_table[1, 2].clone()
        cache.page_table[1, 2] = bad
        run()
        assert int(status.item()) == tq.TQ_STATUS_BAD_PAGE
        _check_decode(torch, out, q_c, q_r, values, 0.06, 0, rows=[0])
        # entries behind the last token's page are not looked at
        cache.seq_lens[1] = 32
        status.zero_()
        run()
        assert int(status.item()) == 0
        _check_decode(torch, out, q_c, q_r, [values[0], tuple(x[:32] for x in values[1])], 0.06, 0)
        cache.seq_lens[1] = 64
        cache.page_table[1, 2] = held


# ---------------------------------------------------------------------------------------------------------- prompt

def _operands(torch, rng, lq, lk, H, d, kind, layout, extra=0):
    t = _types(torch)[kind]
    make = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(t).cuda()  # noqa: E731
    n_q, n_kv = sum(lq) + extra, sum(lk) + extra
    if layout == "fused":                                          # slices of the projections' outputs
        q, kv, x = make(n_q, H, d + 64), make(n_kv, H, 2 * d), make(n_kv, 512 + 64)
        return q[..., :d], q[..., d:], kv[..., :d], x[:, 512:], kv[..., d:]
    if layout == "heads":                                          # heads before rows
        return (make(H, n_q, d).transpose(0, 1), make(H, n_q, 64).transpose(0, 1), make(H, n_kv, d).transpose(0, 1), make(n_kv, 64),
                make(H, n_kv, d).transpose(0, 1))
    return make(n_q, H, d), make(n_q, H, 64), make(n_kv, H, d), make(n_kv, 64), make(n_kv, H, d)


def _check(torch, out, ops, q_at, k_at, alpha, causal, window):
    q_n, q_r, k_n, k_r, v = (x.cpu() for x in ops)
    q, k, v = torch.cat([q_n, q_r], -1), L.prompt_keys(k_n, k_r), v
    # (the check cuts its head dimension from q: 64 channels more than the output has)
    _check_prompt(torch, out, q, k, v, q_at, k_at, alpha, causal, window)


PROMPTS = [
    # lq, past, H, d, kind, causal, window, layout
    ([1], 0, 1, 64, "fp16", True, 0, "split"), ([5], 0, 3, 128, "bf16", True, 0, "fused"), ([129], 0, 4, 64, "fp16", True, 0, "fused"),
    ([300], 0, 2, 128, "fp16", True, 0, "heads"), ([64, 1, 0, 77, 256, 3], 0, 5, 128, "bf16", True, 0, "fused"),
    ([200, 31], 0, 6, 64, "bf16", True, 0, "heads"), ([33, 128, 1], 200, 4, 128, "fp16", True, 0, "fused"),
    ([100], 517, 7, 64, "bf16", True, 128, "split"), ([513], 0, 2, 128, "fp16", True, 100, "fused"),
    ([70, 130], 45, 2, 128, "bf16", False, 0, "fused"), ([20], -12, 4, 128, "fp16", True, 0, "fused"), ([30], 0, 9, 64, "fp16", False, 0, "split"),
    ([1, 1, 1], 1000, 4, 128, "fp16", True, 1, "heads"), ([1100], 0, 3, 128, "fp16", True, 0, "fused"), ([700], 0, 2, 64, "bf16", True, 0, "fused")]
# Empty sequences behind the others: a padded batch.  They also count towards the tiles by which the kernel's form is
# chosen (two tiles per thread block where there are more tiles than SMs).
PADDED = pytest.mark.parametrize("padded", [0, 200])


@PADDED
@pytest.mark.parametrize("lq,past,H,d,kind,causal,window,layout", PROMPTS)
def test_latent_prompt(gpu, lq, past, H, d, kind, causal, window, layout, padded):
    """past < 0: fewer keys than queries, so the first queries see nothing.  Rows behind the last sequence stay."""
    tq, torch = gpu
    rng = np.random.default_rng(sum(lq) + d)
    lq = lq + [0] * padded
    lk = [max(0, n + past) if n else 0 for n in lq]
    ops = _operands(torch, rng, lq, lk, H, d, kind, layout, 3)
    q_at, k_at = np.concatenate([[0], np.cumsum(lq)]).tolist(), np.concatenate([[0], np.cumsum(lk)]).tolist()
    dq, dk = _dev(torch, q_at), _dev(torch, k_at)
    status, alpha = _dev(torch, [0]), (d + 64) ** -0.5
    for out_t in (torch.float32, _types(torch)[kind]):
        guard = torch.full(((len(ops[0]) + 2) * H * d,), 5.0, dtype=out_t, device="cuda")
        out = guard.view(-1, H, d)[1:-1]
        tq.tq_sdpa_latent_prompt(*ops, dq, dk, alpha, out, causal=causal, window=window, status=status)
        assert int(status.item()) == 0
        assert torch.all(guard.view(-1, H, d)[0] == 5.0) and torch.all(guard.view(-1, H, d)[1 + sum(lq):] == 5.0)
        _check(torch, out, ops, q_at, k_at, alpha, causal, window)


@PADDED
@pytest.mark.parametrize("d,kind", [(64, "bf16"), (128, "fp16")])
@pytest.mark.parametrize("layout", ["fused", "heads"])
def test_latent_prompt_infinities_and_nans_stay_with_their_readers(gpu, d, kind, layout, padded):
    """NaN and infinities in keys and values: of a neighbouring sequence, of later tokens, of tokens outside the window, and of
    tokens that are seen."""
    tq, torch = gpu
    rng = np.random.default_rng(5)
    lq = [150, 90] + [0] * padded
    for window in (0, 40):
        q_n, q_r, k_n, k_r, v = _operands(torch, rng, lq, lq, 3, d, kind, layout)
        for i, x in ((0, float("inf")), (70, -float("inf")), (100, float("nan")), (149, float("inf")), (200, float("nan"))):
            v[i, 1, i % d] = x
        k_r[120, 3], k_n[130, 2, 5], k_r[239, 63] = float("nan"), float("nan"), float("nan")
        at = np.concatenate([[0], np.cumsum(lq)]).tolist()
        out = torch.empty((240, 3, d), device="cuda")
        tq.tq_sdpa_latent_prompt(q_n, q_r, k_n, k_r, v, _dev(torch, at), _dev(torch, at), 0.07, out, window=window)
        _check(torch, out, (q_n, q_r, k_n, k_r, v), at, at, 0.07, True, window)


@PADDED
def test_latent_prompt_offsets_outside_the_buffers(gpu, padded):
    tq, torch = gpu
    rng = np.random.default_rng(6)
    ops = _operands(torch, rng, [100], [100], 2, 128, "fp16", "fused")
    out, status = torch.full((100, 2, 128), 9.0, device="cuda"), _dev(torch, [0])
    q_at, k_at = [0, 60, 140] + [140] * padded, [0, 60, 1000] + [1000] * padded
    tq.tq_sdpa_latent_prompt(*ops, _dev(torch, q_at), _dev(torch, k_at), 0.07, out, status=status)
    assert int(status.item()) == tq.TQ_STATUS_BAD_LEN
    _check(torch, out, ops, [0, 60, 100], [0, 60, 100], 0.07, True, 0)
    status.zero_()
    tq.tq_sdpa_latent_prompt(*ops, _dev(torch, [0, 50, 100]), _dev(torch, [0, 100, 100]), 0.07, out, status=status)
    assert int(status.item()) == tq.TQ_STATUS_EMPTY_SEQ and torch.all(out[50:] == 0)


# ------------------------------------------------------------------------------------------------------- together

@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("d_c", [512, 256])
def test_a_serving_loop(gpu, d_c, captured):
    """One layer of a model with latent attention, three slots: prompts go through the expanded form (in two chunks, the first
    of which is read back from the cache) and into the cache, steps through the absorbed form with the same expansions;
    both forms, up to the cache's rounding, are one attention.  The decode steps run eagerly or from one captured graph."""
    tq, torch = gpu
    torch.manual_seed(3)
    B, H, d, P, num_pages = 3, 6, 128, 32, 30
    t, alpha = torch.float16, (d + 64) ** -0.5
    w_k, w_v = ((torch.randn((H, d, d_c), device="cuda") * d_c ** -0.5).to(t) for _ in range(2))
    table, lens = torch.zeros((B, 8), dtype=torch.int32, device="cuda"), _dev(torch, [0] * B)
    free, count = torch.randperm(num_pages).int().cuda(), _dev(torch, [num_pages])
    cache = tq.PagedLatentCache.over(torch.full((num_pages, P // 16, tq.TQ_BLOCK_LATENT_BYTES(d_c)), 0xFF, dtype=torch.uint8, device="cuda"), lens, table)
    pwork, work = tq.alloc_pages_workspace(B), tq.alloc_latent_workspace(B, H, d_c)
    status, offsets = _dev(torch, [0]), _dev(torch, [0] * (B + 1))
    model = L.Cache(num_pages * P, d_c)
    place = [[] for _ in range(B)]

    def tokens(n):
        return torch.randn((n, d_c + 64), device="cuda").to(t), torch.randn((n, H, d + 64), device="cuda").to(t)

    def expand(c):
        return torch.einsum("nc,hdc->nhd", c.float(), w_k.float()).to(t), torch.einsum("nc,hdc->nhd", c.float(), w_v.float()).to(t)

    def note(new, slots):
        at = 0
        for b, n in enumerate(new):
            place[b] += slots[at:at + n]
            at += n

    def admit(new, done):
        """A chunk of every sequence with new tokens, behind what is cached of it."""
        tq.tq_pages_release(table, lens, _dev(torch, done, torch.uint8), P, num_pages, free, count, lens, count, status)
        for b in range(B):
            if done[b]:
                place[b] = []
        past = [len(p) for p in place]
        n = sum(new)
        slots = torch.empty(n, dtype=torch.int64, device="cuda")
        tq.tq_pages_assign(table, lens, _dev(torch, new), P, num_pages, free, count, lens, count, offsets, slots, pwork, status)
        x, q = tokens(n)
        tq.tq_latent_append(cache, x[:, :d_c], x[:, d_c:], slots, status)
        model.append(x[:, :d_c], x[:, d_c:], np.array(slots.tolist()))
        note(new, slots.tolist())
        # keys of the chunk's sequences: everything that is cached, read back and expanded
        keys = [place[b] if new[b] else [] for b in range(B)]
        k_at = np.concatenate([[0], np.cumsum([len(k) for k in keys])]).tolist()
        ask = torch.tensor(sum(keys, []), dtype=torch.int64, device="cuda")
        c, r = torch.empty((len(ask), d_c), dtype=t, device="cuda"), torch.empty((len(ask), 64), dtype=t, device="cuda")
        tq.tq_latent_gather(cache, ask, c, r, status)
        k_n, v = expand(c)
        out = torch.full((n, H, d), 9.0, device="cuda")
        ops = (q[..., :d], q[..., d:], k_n, r, v)
        tq.tq_sdpa_latent_prompt(*ops, offsets, _dev(torch, k_at), alpha, out, status=status)
        _check(torch, out, ops, offsets.tolist(), k_at, alpha, True, 0)
        return past

    ones, none = _dev(torch, [1] * B), _dev(torch, [0] * B, torch.uint8)
    s_slots = torch.zeros(B, dtype=torch.int64, device="cuda")
    s_x, s_q = tokens(B)
    s_qc, s_out = torch.empty((H, B, d_c), dtype=t, device="cuda"), torch.zeros((B, H, d_c), device="cuda")

    def step():
        tq.tq_pages_release(table, lens, none, P, num_pages, free, count, lens, count, status)
        tq.tq_pages_assign(table, lens, ones, P, num_pages, free, count, lens, count, offsets, s_slots, pwork, status)
        tq.tq_latent_append(cache, s_x[:, :d_c], s_x[:, d_c:], s_slots, status)
        torch.bmm(s_q[..., :d].transpose(0, 1), w_k, out=s_qc)     # the query times the key's expansion, heads first
        tq.tq_sdpa_latent_decode(cache, s_qc.transpose(0, 1), s_q[..., d:], alpha, 0, 0, work, s_out, status)

    assert admit([37, 16, 50], [0, 0, 0]) == [0, 0, 0]
    assert admit([20, 0, 64], [0, 0, 0]) == [37, 16, 50]
    graph = None
    if captured:
        step_lens, step_table, step_free, step_count = lens.clone(), table.clone(), free.clone(), count.clone()
        step()                                                     # (the library product's set-up is not for a capture)
        for x, y in ((lens, step_lens), (table, step_table), (free, step_free), (count, step_count)):
            x.copy_(y)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    for turn in range(14):
        if turn == 9:
            assert admit([0, 30, 0], [0, 1, 0]) == [57 + 9, 0, 114 + 9]
        for x, y in zip((s_x, s_q), tokens(B)):
            x.copy_(y)
        graph.replay() if graph else step()
        slots = s_slots.tolist()
        note([1] * B, slots)
        model.append(s_x[:, :d_c], s_x[:, d_c:], np.array(slots))
        values = [model.values(np.array(place[b])) for b in range(B)]
        _check_decode(torch, s_out, s_qc.transpose(0, 1), s_q[..., d:], values, alpha, 0)
        if turn in (0, 13):
            # the absorbed form's result, expanded, against the expanded form of the same token
            ask = torch.tensor(sum(place, []), dtype=torch.int64, device="cuda")
            k_at = np.concatenate([[0], np.cumsum([len(p) for p in place])]).tolist()
            c, r = torch.empty((len(ask), d_c), dtype=t, device="cuda"), torch.empty((len(ask), 64), dtype=t, device="cuda")
            tq.tq_latent_gather(cache, ask, c, r, status)
            k_n, v = expand(c)
            out = torch.empty((B, H, d), device="cuda")
            tq.tq_sdpa_latent_prompt(s_q[..., :d], s_q[..., d:], k_n, r, v, _dev(torch, list(range(B + 1))), _dev(torch, k_at), alpha, out, status=status)
            absorbed = torch.einsum("bhc,hdc->bhd", s_out, w_v.float())
            # keys, values and queries were rounded to fp16 on the way (2^-11 each, scores of up to a few units)
            assert (absorbed - out).abs().max() <= 0.02 * v.float().abs().max()
    assert int(status.item()) == 0
    assert lens.tolist() == [len(p) for p in place]
    assert count.tolist() == [num_pages - sum(-(-len(p) // P) for p in place)]
