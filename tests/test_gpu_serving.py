"""The serving operators against their definitions in 64 bits (tests/serving_ref.py): page bookkeeping, the 8-bit cache,
decode attention over it, attention of packed prompts, and a run of them together."""
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


def _types(torch):
    return {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


# ---------------------------------------------------------------------------------------------------------- pages

def ref_release(table, lens, done, P, num_pages, free, count):
    free, lens = list(free), list(lens)
    pages = [int(table[b][i]) for b in range(len(lens)) if done[b] for i in range(-(-lens[b] // P))]
    if count + len(pages) > num_pages:
        return lens, free, count, True
    free[count:count + len(pages)] = pages
    return [0 if done[b] else lens[b] for b in range(len(lens))], free, count + len(pages), False


def ref_assign(table, lens, new, P, free, count, n_slots):
    table = [list(r) for r in table]
    cap = P * len(table[0])
    status, wanted, offsets, slots, out, granted, ends = 0, 0, [0], [], [], 0, 0
    for b, (a, n) in enumerate(zip(lens, new)):
        bad = 4 if n < 0 or not 0 <= a <= cap else 0
        n = max(n, 0)
        ends += n
        fits = not bad and a + n <= cap
        if not bad and not fits:
            bad |= 1
        need = -(-(a + n) // P) - -(-a // P) if fits else 0
        wanted += need
        ok = fits
        if ends > n_slots:
            if n > 0:
                bad |= 4
                ok = False
        if ok and need and wanted > count:
            bad |= 32
            ok = False
        status |= bad
        offsets.append(min(ends, n_slots))
        if ok:
            for i in range(need):
                table[b][-(-a // P) + i] = free[count - 1 - (wanted - need) - i]
            granted = max(granted, wanted) if need else granted
        out.append(a + n if ok else a)
        slots += [table[b][p // P] * P + p % P if ok else -1 for p in range(a, a + n)]
    slots = slots[:n_slots] + [-1] * (n_slots - len(slots))
    return table, out, count - granted, offsets, slots, status


def _pool(rng, lens, P, spare, extra_cols=2):
    pages = [-(-n // P) for n in lens]
    total = sum(pages) + spare
    perm = rng.permutation(total)
    cols = max(pages + [1]) + extra_cols
    table = np.full((len(lens), cols), -1, np.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = perm[at:at + n]
        at += n
    free = np.full(total, -1, np.int32)
    free[:spare] = perm[at:]
    return table, free, spare, total


@pytest.mark.parametrize("B,P,hi,new_hi,spare,pad,seed", [
    (1, 16, 0, 1, 1, 0, 1), (1, 64, 100, 1, 4, 3, 2), (16, 64, 3000, 1, 16, 0, 3), (7, 16, 300, 200, 100, 5, 4),
    (64, 16, 500, 400, 60, 0, 5),        # the pool runs out half way
    (300, 32, 200, 90, 1000, 17, 6),     # more slots than the one-launch form writes (and a second warp row of sequences)
    (2500, 16, 60, 20, 3500, 1, 7),      # several rounds of the scan
])
def test_release_and_assign(gpu, B, P, hi, new_hi, spare, pad, seed):
    tq, torch = gpu
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, hi + 1, B)
    lens[rng.integers(0, B)] = 0
    new = rng.integers(0, new_hi + 1, B)
    new[-1] = new_hi
    done = rng.random(B) < 0.2
    table, free, count, total = _pool(rng, lens, P, spare)
    dev = lambda x, t=torch.int32: torch.tensor(np.asarray(x), dtype=t, device="cuda")  # noqa: E731
    d_table, d_free, d_count, d_lens = dev(table), dev(free), dev([count]), dev(lens)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    l1, c1 = torch.empty_like(d_lens), torch.empty_like(d_count)
    tq.tq_pages_release(d_table, d_lens, dev(done, torch.bool), P, total, d_free, d_count, l1, c1, status)
    want_l, want_free, want_c, refused = ref_release(table, lens, done, P, total, free, count)
    assert not refused and int(status.item()) == 0
    assert l1.tolist() == [int(x) for x in want_l] and c1.tolist() == [want_c] and d_free.tolist() == [int(x) for x in want_free]
    n = int(new.sum()) + pad
    if n == 0:
        n = 1
    offsets = torch.full((B + 1,), 77, dtype=torch.int32, device="cuda")
    slots = torch.full((n + 8,), 99, dtype=torch.int64, device="cuda")
    work = tq.alloc_pages_workspace(B)
    # the lengths and the count in place, as a serving loop keeps them
    tq.tq_pages_assign(d_table, l1, dev(new), P, total, d_free, c1, l1, c1, offsets, slots[:n], work, status)
    table2, lens2, count2, offsets2, slots2, status2 = ref_assign(table, want_l, new, P, want_free, want_c, n)
    assert int(status.item()) == status2
    assert l1.tolist() == [int(x) for x in lens2] and c1.tolist() == [count2] and offsets.tolist() == [int(x) for x in offsets2]
    assert slots[:n].tolist() == [int(x) for x in slots2] and slots[n:].tolist() == [99] * 8
    assert np.array_equal(d_table.cpu().numpy(), np.array(table2, np.int32))


def test_assign_refusals_on_the_device(gpu):
    """Sequences that do not fit their table, the slots or the range of lengths are refused one by one; the others go on."""
    tq, torch = gpu
    P = 16
    dev = lambda x, t=torch.int32: torch.tensor(x, dtype=t, device="cuda")  # noqa: E731
    lens, new = [30, -3, 5, 1000, 0, 40], [3, 4, -2, 1, 16, 20]     # rows of 3 pages: 48 tokens
    table = np.arange(18, dtype=np.int32).reshape(6, 3)
    free = list(range(18, 30))
    for n_slots in (44, 30, 4):
        want = ref_assign(table, lens, new, P, free, 12, n_slots)
        d_table, out, cnt = dev(table), torch.empty(6, dtype=torch.int32, device="cuda"), dev([12])
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        offsets, slots = torch.empty(7, dtype=torch.int32, device="cuda"), torch.empty(n_slots, dtype=torch.int64, device="cuda")
        tq.tq_pages_assign(d_table, dev(lens), dev(new), P, 30, dev(free + [0] * 18), cnt, out, cnt, offsets, slots,
                           tq.alloc_pages_workspace(6), status)
        assert out.tolist() == want[1] and cnt.tolist() == [want[2]] and offsets.tolist() == want[3]
        assert slots.tolist() == want[4] and int(status.item()) == want[5] and d_table.tolist() == [list(map(int, r)) for r in want[0]]
    # pages outside the pool: flagged, their tokens skipped
    status.zero_()
    slots = torch.empty(20, dtype=torch.int64, device="cuda")
    tq.tq_pages_assign(dev(table), dev([0] * 6), dev([20, 0, 0, 0, 0, 0]), P, 30, dev([50, 7] + [0] * 28), dev([2]), out, cnt, offsets, slots,
                       tq.alloc_pages_workspace(6), status)
    assert int(status.item()) == tq.TQ_STATUS_BAD_PAGE and slots.tolist() == [7 * 16 + i for i in range(16)] + [-1] * 4


def test_release_refuses_more_pages_than_the_pool_has(gpu):
    tq, torch = gpu
    dev = lambda x, t=torch.int32: torch.tensor(x, dtype=t, device="cuda")  # noqa: E731
    lens, free, count = dev([40, 16]), dev([5, 4, 3, -1]), dev([3])
    out, cnt, status = torch.empty_like(lens), torch.empty_like(count), dev([0])
    tq.tq_pages_release(dev([[0, 1, 2], [3, 0, 0]]), lens, dev([1, 0], torch.uint8), 16, 4, free, count, out, cnt, status)
    assert int(status.item()) == tq.TQ_STATUS_BAD_PAGE and out.tolist() == [40, 16] and cnt.tolist() == [3]
    assert free.tolist() == [5, 4, 3, -1]


def test_pages_of_contiguous_caches(gpu):
    tq, torch = gpu
    dev = lambda x, t=torch.int32: torch.tensor(x, dtype=t, device="cuda")  # noqa: E731
    lens, status = dev([5, 90, 0]), dev([0])
    tq.tq_pages_release(None, lens, dev([0, 1, 0], torch.uint8), 96, 0, None, None, lens, None, status)
    assert lens.tolist() == [5, 0, 0]
    offsets, slots = dev([0] * 4), torch.empty(12, dtype=torch.int64, device="cuda")
    tq.tq_pages_assign(None, lens, dev([2, 3, 4]), 96, 0, None, None, lens, None, offsets, slots, tq.alloc_pages_workspace(3), status)
    assert lens.tolist() == [7, 3, 4] and offsets.tolist() == [0, 2, 5, 9] and int(status.item()) == 0
    assert slots.tolist() == [5, 6, 96, 97, 98, 192, 193, 194, 195, -1, -1, -1]


# ------------------------------------------------------------------------------------------------------ 8-bit cache

def _cache(tq, torch, B, H, d, page, cap, seed):
    """A cache with junk in it (every byte 0xA5) and its page table (None: contiguous)."""
    if page == 0:
        c = tq.KV8Cache(B, H, cap, d)
        c.blocks.fill_(0xA5)
        return c, None
    cols = -(-cap // page)
    c = tq.PagedKV8Cache(B, H, page, cols, B * cols + 3, d)
    c.blocks.fill_(0xA5)
    table = np.random.default_rng(seed).permutation(B * cols + 3)[:B * cols].reshape(B, cols).astype(np.int32)
    c.page_table.copy_(torch.from_numpy(table))
    return c, table


def _rows(torch, rng, n, H, d, kind, fused=True):
    """Packed 16-bit K and V rows with magnitudes that vary from token to token: slices of a fused tensor, or apart."""
    t = _types(torch)[kind]
    x = torch.from_numpy(rng.standard_normal((n, 3 + 2 * H, d)) * 10.0 ** rng.uniform(-2, 2, (n, 1, 1))).to(t).cuda()
    k, v = x[:, 3:3 + H], x[:, 3 + H:]
    return (k, v) if fused else (k.contiguous(), v.contiguous())


def _check_cache(cache, model, slots, d):
    got = R.read_device_cache(cache.blocks, d)
    s = np.unique(slots[slots >= 0])
    for part in (0, 1):
        assert np.array_equal(got.range[part][s // 16], model.range[part][s // 16])
        assert np.array_equal(got.codes[part][s // 16, :, s % 16], model.codes[part][s // 16, :, s % 16])


@pytest.mark.parametrize("B,H,d,page,kind,seed", [
    (1, 1, 64, 0, "fp16", 1), (3, 2, 128, 16, "fp16", 2), (2, 3, 128, 64, "bf16", 3), (4, 1, 256, 32, "bf16", 4),
    (2, 2, 512, 16, "fp16", 5), (2, 5, 64, 128, "bf16", 6)])
def test_append_and_gather(gpu, B, H, d, page, kind, seed):
    """Appends of one token, of odd chunks and of a long prompt in turn: every code and range is the definition's, and
    gather gives the values back in any order."""
    tq, torch = gpu
    rng = np.random.default_rng(seed)
    cap = 256
    cache, table = _cache(tq, torch, B, H, d, page, cap, seed)
    total = cache.blocks.shape[0] * cache.blocks.shape[2]
    model = R.Cache8(total, H, d)
    lens, seen = [0] * B, np.zeros(0, np.int64)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for step, most in enumerate([1, 1, 1, 7, 1, 40, 1, 1, 100, 2, 1]):
        new = [int(rng.integers(0, most + 1)) for _ in range(B)]
        new[step % B] = most
        slots = R.slots_of(lens, new, table, page, cap)
        padded = np.concatenate([slots, [-1] * (step % 3)]).astype(np.int64)
        k, v = _rows(torch, rng, len(padded), H, d, kind, fused=step % 2 == 0)
        tq.tq_kv8_append(cache, k, v, torch.from_numpy(padded).cuda(), status)
        model.append(k.double().cpu().numpy(), v.double().cpu().numpy(), padded)
        lens = [a + n for a, n in zip(lens, new)]
        seen = np.concatenate([seen, slots])
        _check_cache(cache, model, seen, d)
    assert int(status.item()) == 0
    order = rng.permutation(np.concatenate([seen, seen[:5], [-1, -1]]))
    for out, eps in ((torch.float32, 2.0 ** -23), (_types(torch)[kind], torch.finfo(_types(torch)[kind]).eps / 2 + 2.0 ** -23)):
        k, v = (torch.full((len(order), H, d), 7.0, dtype=out, device="cuda") for _ in range(2))
        tq.tq_kv8_gather(cache, torch.from_numpy(order).cuda(), k, v, status)
        for got, want in zip((k, v), model.values(np.maximum(order, 0))):
            want[order < 0] = 0.0
            got = got.double().cpu().numpy()
            assert np.all(np.abs(got - want) <= np.abs(want) * eps + 1e-7 * (out == torch.float16))
    assert int(status.item()) == 0


def test_append_edge_values(gpu):
    """Exact halves, zeros, subnormals, the types' largest values, NaN and infinities."""
    tq, torch = gpu
    H, d = 1, 64
    for kind, top, tiny in (("fp16", 65504.0, 2.0 ** -24), ("bf16", float(torch.finfo(torch.bfloat16).max), 2.0 ** -133)):
        rows = []
        a = np.zeros((3, d))
        a[0, 0] = 254.0                       # range 254: 127 x / 254 = x / 2, halves for every odd x
        a[0, 1:] = np.arange(1, d) * 1.0
        a[1] = -a[0] + 1
        rows += [a, np.zeros((2, d)), np.full((1, d), tiny), np.linspace(-1, 1, d)[None] * 127 * tiny, np.full((2, d), top) * np.linspace(-1, 1, d)]
        x = np.concatenate(rows)
        t = torch.from_numpy(x).to(_types(torch)[kind])
        t[-1, 3], t[-1, 4], t[-1, 5] = float("nan"), float("inf"), -float("inf")
        clean = t.double().numpy().copy()
        clean[-1, 3], clean[-1, 4], clean[-1, 5] = 0.0, top, -top
        t, clean = t[:, None, :], clean[:, None, :]
        cache, _ = _cache(tq, torch, 1, H, d, 0, 256, 0)
        model = R.Cache8(16, H, d)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        slots = np.arange(len(x)) * 16        # a block each, then all of them into one block, one by one
        for s in [slots] + [np.array([240 + i]) for i in range(len(x))]:
            i0 = 0 if len(s) > 1 else int(s[0]) - 240
            rows_t = t[i0:i0 + len(s)].cuda().contiguous()
            tq.tq_kv8_append(cache, rows_t, rows_t, torch.from_numpy(s).cuda(), status)
            model.append(clean[i0:i0 + len(s)], clean[i0:i0 + len(s)], s)
            _check_cache(cache, model, s, d)
        _check_cache(cache, model, np.arange(240, 240 + len(x)), d)
        assert int(status.item()) == 0


def test_append_and_gather_refuse_bad_slots(gpu):
    """Slots outside the cache and rows out of order are flagged and skipped; nothing else is touched."""
    tq, torch = gpu
    cache, _ = _cache(tq, torch, 1, 2, 128, 0, 64, 0)
    rng = np.random.default_rng(0)
    k, v = _rows(torch, rng, 6, 2, 128, "fp16")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for bad in ([0, 1, 64, 1 << 40, 16, 17], [0, 1, 3, 4, 16, 17], [0, 1, 1, 1, 16, 17], [0, 1, 0, 1, 16, 17]):
        cache.blocks.fill_(0xA5)
        status.zero_()
        s = np.array(bad, np.int64)
        tq.tq_kv8_append(cache, k, v, torch.from_numpy(s).cuda(), status)
        assert int(status.item()) == tq.TQ_STATUS_BAD_SLOT
        model = R.Cache8(4, 2, 128)
        good = np.array([0, 1, -1, -1, 16, 17], np.int64)
        model.append(k.double().cpu().numpy(), v.double().cpu().numpy(), good)
        _check_cache(cache, model, good, 128)
        assert torch.all(cache.blocks[:, :, 2:] == 0xA5)
    status.zero_()
    ko, vo = (torch.full((4, 2, 128), 7.0, device="cuda") for _ in range(2))
    tq.tq_kv8_gather(cache, torch.tensor([0, 64, 1 << 40, -5], device="cuda"), ko, vo, status)
    assert int(status.item()) == tq.TQ_STATUS_BAD_SLOT and torch.all(ko[1:] == 0) and torch.all(vo[1:] == 0)


# ---------------------------------------------------------------------------------------------------------- decode

def _filled(tq, torch, lens, H, d, page, kind, seed, cap=None):
    """A cache filled through append (one call), with its host model."""
    rng = np.random.default_rng(seed)
    B = len(lens)
    cap = cap or -(-max(max(lens), 1) // 16) * 16
    cache, table = _cache(tq, torch, B, H, d, page, cap, seed)
    slots = R.slots_of([0] * B, lens, table, page, cap)
    model = R.Cache8(cache.blocks.shape[0] * cache.blocks.shape[2], H, d)
    if len(slots):
        t = _types(torch)[kind]
        k = torch.from_numpy(rng.standard_normal((len(slots), H, d))).cuda()
        k[..., :2] *= 10.0
        v = torch.from_numpy(rng.standard_normal((len(slots), H, d)) * 10.0 ** rng.uniform(-1, 1, (len(slots), 1, 1))).cuda()
        k, v = k.to(t), v.to(t)
        tq.tq_kv8_append(cache, k, v, torch.from_numpy(slots).cuda())
        model.append(k.double().cpu().numpy(), v.double().cpu().numpy(), slots)
    cache.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    starts = np.concatenate([[0], np.cumsum(lens)])
    return cache, [model.values(slots[starts[b]:starts[b + 1]]) for b in range(B)]


def _check_decode(torch, out, q, values, alpha, window, d):
    B, H_q, _ = q.shape
    qd, od = q.double().cpu(), out.double().cpu()
    out_eps = 0.0 if out.dtype == torch.float32 else torch.finfo(out.dtype).eps / 2
    worst = 0.0
    for b in range(B):
        k, v = values[b]
        n = len(k)
        lo = max(0, n - window) if window else 0
        if n == 0:
            assert torch.all(od[b] == 0)
            continue
        H = k.shape[1]
        G = H_q // H
        for h in range(H):
            ref, weighed, p, mag = R.attention(qd[b, h * G:(h + 1) * G], k[lo:, h], v[lo:, h], alpha)
            tol = R.bound(ref, weighed, p, mag, n - lo, d, 2.0 ** -11, np.abs(v[lo:, h]).max(), out_eps)
            if out.dtype == torch.float16:
                tol = tol + 2.0 ** -25  # half a step of the subnormals
            err = (od[b, h * G:(h + 1) * G] - ref).abs()
            assert torch.all(err <= tol), (b, h, float((err / tol).max()))
            worst = max(worst, float((err / tol).max()))
    return worst


@pytest.mark.parametrize("lens,H_q,H_kv,d,page,kind,window,seed", [
    ([1], 1, 1, 64, 0, "fp16", 0, 1), ([17], 8, 1, 128, 0, "fp16", 0, 2), ([1000], 64, 8, 128, 0, "bf16", 0, 3),
    ([5000, 0, 33, 16, 2047], 16, 2, 128, 64, "bf16", 0, 4), ([700, 1300], 24, 8, 128, 16, "fp16", 0, 5),
    ([3001], 32, 16, 256, 0, "fp16", 0, 6), ([100, 1, 900], 6, 2, 256, 32, "bf16", 0, 7),
    ([500, 77], 8, 2, 512, 16, "fp16", 0, 8), ([2500], 40, 2, 64, 128, "bf16", 0, 9),       # 20 heads: three tiles
    ([1500, 100, 64, 63], 8, 2, 128, 16, "fp16", 64, 10), ([4000], 64, 8, 128, 0, "fp16", 1000, 11),
    ([2000, 5], 12, 4, 256, 64, "bf16", 1, 12), ([20] * 300, 4, 4, 64, 16, "fp16", 0, 13), ([20000], 8, 1, 128, 0, "fp16", 0, 14),
    # units of a few blocks each: one per thread block, several per warp; wide heads, where a warp never takes a unit
    ([5, 118, 0, 33] * 4, 64, 8, 128, 0, "fp16", 0, 15), ([3, 0, 70, 200] * 20, 24, 8, 128, 16, "bf16", 0, 16),
    ([40, 1] * 60, 8, 4, 256, 16, "fp16", 20, 17), ([9, 300] * 30, 20, 4, 512, 32, "bf16", 0, 18), ([16] * 700, 3, 1, 64, 0, "bf16", 0, 19),
    ([400, 0, 390] * 60, 2, 2, 128, 64, "fp16", 0, 20),
    # more units than thread blocks, long and short ones on one line; a padded batch with one long sequence; equal shares
    ([20, 2500, 300] * 15, 8, 8, 64, 0, "bf16", 0, 21), ([2500] * 6 + [17] * 40, 16, 4, 128, 64, "fp16", 0, 22),
    ([0] * 30 + [9000] + [0] * 25, 24, 4, 128, 16, "bf16", 0, 23), ([1900, 40] * 20, 8, 4, 256, 32, "bf16", 1500, 24),
    ([1500, 10, 0] * 13, 32, 8, 512, 16, "fp16", 0, 25), ([700, 3, 1], 8, 4, 64, 0, "fp16", 0, 26), ([6000, 5900, 1], 16, 2, 128, 16, "fp16", 0, 27)])
def test_int8_decode(gpu, lens, H_q, H_kv, d, page, kind, window, seed):
    tq, torch = gpu
    rng = np.random.default_rng(100 + seed)
    cache, values = _filled(tq, torch, lens, H_kv, d, page, kind, seed)
    B = len(lens)
    wide = torch.from_numpy(rng.standard_normal((B, H_q + 3, d))).to(_types(torch)[kind]).cuda()
    work = tq.alloc_int8_workspace(B, H_kv, H_q, d)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    alpha = d ** -0.5
    for q, out_t in ((wide[:, :H_q], torch.float32), (wide[:, 3:].contiguous(), _types(torch)[kind])):
        guard = torch.full((B * H_q * d + 128,), 5.0, dtype=out_t, device="cuda")
        out = guard[64:-64].view(B, H_q, d)
        status.zero_()
        tq.tq_sdpa_int8_decode(cache, q, alpha, window, 0, work, out, status)
        assert int(status.item()) == (tq.TQ_STATUS_EMPTY_SEQ if 0 in lens else 0)
        assert torch.all(guard[:64] == 5.0) and torch.all(guard[-64:] == 5.0)
        _check_decode(torch, out, q, values, alpha, window, d)
        assert torch.all(work[:int(tq._lib.tq_int8_counter_bytes(B, H_kv, H_q))] == 0)  # left as it was found
        again = torch.empty_like(out)
        tq.tq_sdpa_int8_decode(cache, q, alpha, window, max(max(lens), 1), work, again, status)
        _check_decode(torch, again, q, values, alpha, window, d)


def test_int8_decode_values_of_very_different_size(gpu):
    """Blocks of V whose ranges span the whole of fp16, against scores that favour the small ones: the weights are
    referred to the largest contribution, so the small blocks' values keep their precision where they dominate."""
    tq, torch = gpu
    d, n = 64, 512
    rng = np.random.default_rng(5)
    cache, _ = _cache(tq, torch, 1, 1, d, 0, n, 0)
    k = torch.zeros((n, 1, d), dtype=torch.float16)
    k[:, 0, 0] = torch.linspace(0, 12, n)                 # later tokens score higher ...
    v = torch.from_numpy(rng.standard_normal((n, 1, d)) * np.exp2(np.linspace(14, -12, n))[:, None, None]).half()  # ... and are smaller
    slots = np.arange(n)
    tq.tq_kv8_append(cache, k.cuda(), v.cuda(), torch.from_numpy(slots).cuda())
    cache.seq_lens.fill_(n)
    model = R.Cache8(n // 16, 1, d)
    model.append(k.double().numpy(), v.double().numpy(), slots)
    q = torch.zeros((1, 3, d), dtype=torch.float16, device="cuda")
    q[0, 1, 0], q[0, 2, 0] = 4.0, 60.0
    out = torch.empty((1, 3, d), device="cuda")
    tq.tq_sdpa_int8_decode(cache, q, 1.0, 0, 0, tq.alloc_int8_workspace(1, 1, 3, d), out)
    kk, vv = model.values(slots)
    ref, weighed, p, mag = R.attention(q[0].double().cpu(), kk[:, 0], vv[:, 0], 1.0)
    # per token the error is 2^-11 of its own contribution, or 2^-25 of the largest contribution p_j a_j
    z = torch.softmax(q[0].double().cpu() @ torch.as_tensor(kk[:, 0]).T, -1)
    a = torch.as_tensor(np.repeat(model.range[1][:, 0], 16))
    tol = R.bound(ref, weighed, 0 * p, mag, n, d, 2.0 ** -11, 0.0, 0.0) + n * 2.0 ** -25 * (z * a).amax(1, keepdim=True)
    assert torch.all((out[0].double().cpu() - ref).abs() <= tol)


def test_int8_decode_extreme_queries(gpu):
    """bf16 queries far outside the range of fp16, zero queries, a negative and a zero scale."""
    tq, torch = gpu
    lens, H, d = [100], 2, 128
    cache, values = _filled(tq, torch, lens, H, d, 0, "bf16", 21)
    q = torch.randn((1, 16, d), device="cuda").to(torch.bfloat16)
    q[0, :8] *= 2.0 ** 60
    q[0, 8:12] *= 2.0 ** -60
    q[0, 12:] = 0
    work = tq.alloc_int8_workspace(1, H, 16, d)
    for alpha in (2.0 ** -62, -(2.0 ** -60), 0.0):
        out = torch.empty((1, 16, d), device="cuda")
        tq.tq_sdpa_int8_decode(cache, q, alpha, 0, 0, work, out)
        _check_decode(torch, out, q, values, alpha, 0, d)


def test_int8_decode_status_bits(gpu):
    tq, torch = gpu
    cache, values = _filled(tq, torch, [40, 60], 2, 64, 16, "fp16", 31)
    work, status = tq.alloc_int8_workspace(2, 2, 4, 64), torch.zeros(1, dtype=torch.int32, device="cuda")
    q, out = torch.randn((2, 4, 64), device="cuda").half(), torch.empty((2, 4, 64), device="cuda")
    cache.page_table[1, 3] = 10000                      # behind no token of sequence 0, the last page of sequence 1
    tq.tq_sdpa_int8_decode(cache, q, 0.125, 0, 0, work, out, status)
    assert int(status.item()) == tq.TQ_STATUS_BAD_PAGE
    _check_decode(torch, out[:1], q[:1], values[:1], 0.125, 0, 64)
    status.zero_()
    cache.seq_lens[0] = 65                              # S_cap is 64
    cache.seq_lens[1] = -1
    tq.tq_sdpa_int8_decode(cache, q, 0.125, 0, 0, work, out, status)
    assert int(status.item()) == tq.TQ_STATUS_BAD_LEN | tq.TQ_STATUS_EMPTY_SEQ and torch.all(out[1] == 0)


# ---------------------------------------------------------------------------------------------------------- prompt

def _check_prompt(torch, out, q, k, v, q_at, k_at, alpha, causal, window):
    H_q, H, d = q.shape[1], k.shape[1], q.shape[2]
    G = H_q // H
    qd, kd, vd, od = (x.double().cpu() for x in (q, k, v, out))
    out_eps = 0.0 if out.dtype == torch.float32 else torch.finfo(out.dtype).eps / 2
    w_eps = torch.finfo(q.dtype).eps / 2
    for b in range(len(q_at) - 1):
        lq, lk = q_at[b + 1] - q_at[b], k_at[b + 1] - k_at[b]
        if lq <= 0:
            continue
        i, j = torch.arange(lq)[:, None] + lk - lq, torch.arange(lk)[None, :]
        seen = (j <= i) if causal else torch.ones((lq, lk), dtype=torch.bool)
        if window:
            seen = seen & (j > i - window)
        for h in range(H_q):
            qq, kk, vv = qd[q_at[b]:q_at[b + 1], h], kd[k_at[b]:k_at[b + 1], h // G], vd[k_at[b]:k_at[b + 1], h // G]
            ref, weighed, p, mag = R.attention(qq, kk, vv, alpha, seen)
            finite = torch.where(torch.isfinite(vv), vv, 0.0)
            tol = R.bound(ref, weighed, p, mag, lk, d, w_eps, float(finite.abs().max()) if lk else 0.0, out_eps,
                          2.0 ** -25 if q.dtype == torch.float16 else 0.0)
            got = od[q_at[b]:q_at[b + 1], h]
            assert torch.equal(torch.isnan(got), torch.isnan(ref)), (b, h)
            fine = torch.isfinite(ref)
            assert torch.equal(got[~fine & ~torch.isnan(ref)], ref[~fine & ~torch.isnan(ref)]), (b, h)
            err = torch.where(fine, (got - ref).abs(), 0.0)
            assert torch.all(err <= torch.where(fine, tol, 1.0)), (b, h, float((err / tol)[fine].max()))


def _packed(torch, rng, lq, lk, H_q, H_kv, d, kind, fused, extra=0):
    t = _types(torch)[kind]
    make = lambda n, h: torch.from_numpy(rng.standard_normal((n, h, d)).astype(np.float32)).to(t).cuda()  # noqa: E731
    n_q, n_kv = sum(lq) + extra, sum(lk) + extra
    if fused:
        x = make(n_q, H_q + 2 * H_kv)
        return x[:, :H_q], x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:]
    return make(n_q, H_q), make(n_kv, H_kv), make(n_kv, H_kv)


PROMPTS = [
    # lq, past, H_q, H_kv, d, kind, causal, window
    ([1], 0, 1, 1, 64, "fp16", True, 0), ([5], 0, 8, 1, 128, "bf16", True, 0), ([129], 0, 4, 4, 64, "fp16", True, 0),
    ([300], 0, 8, 1, 128, "fp16", True, 0), ([64, 1, 0, 77, 256, 3], 0, 4, 2, 128, "bf16", True, 0),
    ([200, 31], 0, 6, 2, 64, "bf16", True, 0), ([150], 0, 5, 1, 256, "fp16", True, 0), ([90, 20], 0, 4, 2, 256, "bf16", True, 50),
    ([40, 7], 0, 3, 3, 512, "fp16", True, 0), ([33, 128, 1], 200, 8, 2, 128, "fp16", True, 0), ([100], 517, 16, 2, 64, "bf16", True, 128),
    ([513], 0, 8, 8, 128, "fp16", True, 100), ([70, 130], 45, 4, 1, 128, "bf16", False, 0), ([20], -12, 4, 2, 128, "fp16", True, 0),
    ([260], 0, 64, 1, 128, "bf16", True, 0), ([30], 0, 20, 1, 64, "fp16", False, 0), ([1, 1, 1], 1000, 8, 1, 128, "fp16", True, 1),
    ([1100], 0, 8, 2, 128, "fp16", True, 0), ([700], 0, 2, 1, 256, "bf16", True, 0)]


# Empty sequences behind the others: a padded batch.  They also count towards the tiles by which the kernel's form is
# chosen (d <= 128: two tiles per thread block where there are more tiles than SMs).
PADDED = pytest.mark.parametrize("padded", [0, 200])


@PADDED
@pytest.mark.parametrize("lq,past,H_q,H_kv,d,kind,causal,window", PROMPTS)
def test_prompt(gpu, lq, past, H_q, H_kv, d, kind, causal, window, padded):
    """past < 0: fewer keys than queries, so the first queries see nothing.  Rows behind the last sequence stay."""
    tq, torch = gpu
    rng = np.random.default_rng(sum(lq) + d)
    lq = lq + [0] * padded
    lk = [max(0, n + past) if n else 0 for n in lq]
    fused = past == 0
    extra = 3
    q, k, v = _packed(torch, rng, lq, lk, H_q, H_kv, d, kind, fused, extra)
    q_at, k_at = np.concatenate([[0], np.cumsum(lq)]).tolist(), np.concatenate([[0], np.cumsum(lk)]).tolist()
    dq, dk = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (q_at, k_at))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for out_t in (torch.float32, _types(torch)[kind]):
        guard = torch.full(((len(q) + 2) * H_q * d,), 5.0, dtype=out_t, device="cuda")
        out = guard.view(-1, H_q, d)[1:-1]
        tq.tq_sdpa_prompt(q, k, v, dq, dq if fused else dk, d ** -0.5, out, causal=causal, window=window, status=status)
        assert int(status.item()) == 0
        assert torch.all(guard.view(-1, H_q, d)[0] == 5.0) and torch.all(guard.view(-1, H_q, d)[1 + sum(lq):] == 5.0)
        _check_prompt(torch, out, q, k, v, q_at, k_at, d ** -0.5, causal, window)


@PADDED
@pytest.mark.parametrize("d,kind", [(64, "bf16"), (128, "fp16"), (256, "bf16")])
def test_prompt_infinities_and_nans_stay_with_their_readers(gpu, d, kind, padded):
    """NaN and infinities in K and V: of a neighbouring sequence, of later tokens of the same sequence, of tokens outside
    the window, and of tokens that are seen."""
    tq, torch = gpu
    rng = np.random.default_rng(d)
    lq, H_q, H_kv = [150, 90, 60], 4, 2
    q, k, v = (x.contiguous() for x in _packed(torch, rng, lq, lq, H_q, H_kv, d, kind, True, 2))
    at = [0, 150, 240, 300]
    v[150:240] = float("nan")              # the whole second sequence
    k[150:240] = float("inf")
    v[100, 0, 3], v[101, 1, 5], v[240, 0, 7] = float("inf"), float("nan"), -float("inf")
    k[120, 1, 2] = float("nan")
    v[300:], k[300:] = float("nan"), float("nan")
    dq = torch.tensor(at + [300] * padded, dtype=torch.int32, device="cuda")
    for window in (0, 20):
        out = torch.empty(q.shape, dtype=torch.float32, device="cuda")
        tq.tq_sdpa_prompt(q, k, v, dq, dq, d ** -0.5, out, window=window)
        o = out[:300]
        assert torch.isnan(o[150:240]).all()
        kk = k.clone()
        kk[120, 1, 2] = 0                   # queries that see it give NaN throughout; the others as if it were not there
        readers = range(120, min(150, 120 + window) if window else 150)
        G = H_q // H_kv
        assert torch.isnan(o[list(readers), G:]).all()
        keep = [i for i in range(150) if i not in readers]
        ref = torch.empty_like(out)
        tq.tq_sdpa_prompt(q, kk, v, dq, dq, d ** -0.5, ref, window=window)
        assert torch.equal(torch.nan_to_num(o[keep]), torch.nan_to_num(ref[keep]))
        assert torch.equal(torch.isnan(o[keep]), torch.isnan(ref[keep]))
        first = [0, 150]
        _check_prompt(torch, ref[:150], q[:150], kk[:150], v[:150], first, first, d ** -0.5, True, window)
        _check_prompt(torch, o[240:], q[240:300], k[240:300], v[240:300], [0, 60], [0, 60], d ** -0.5, True, window)


@PADDED
def test_prompt_large_scores_and_odd_scales(gpu, padded):
    """Scores far beyond the range of exp, a negative and a zero scale."""
    tq, torch = gpu
    rng = np.random.default_rng(9)
    q, k, v = _packed(torch, rng, [200], [200], 4, 2, 128, "fp16", True)
    q = q * 30
    at = torch.tensor([0, 200] + [200] * padded, dtype=torch.int32, device="cuda")
    for alpha in (1.0, -0.3, 0.0):
        out = torch.empty(q.shape, dtype=torch.float32, device="cuda")
        tq.tq_sdpa_prompt(q, k, v, at, at, alpha, out)
        _check_prompt(torch, out, q, k, v, [0, 200], [0, 200], alpha, True, 0)


@PADDED
def test_prompt_offsets_outside_the_buffers(gpu, padded):
    tq, torch = gpu
    q, k, v = _packed(torch, np.random.default_rng(3), [64], [64], 2, 1, 64, "fp16", False)
    dev = lambda x: torch.tensor(x + x[-1:] * (padded if len(x) > 1 else 0), dtype=torch.int32, device="cuda")  # noqa: E731
    status = dev([0])
    out = torch.full(q.shape, 5.0, device="cuda")
    tq.tq_sdpa_prompt(q, k, v, dev([0, 20, 90]), dev([0, 20, 90]), 0.125, out, status=status)   # the second one ends at row 64
    assert int(status.item()) == tq.TQ_STATUS_BAD_LEN
    _check_prompt(torch, out, q, k, v, [0, 20, 64], [0, 20, 64], 0.125, True, 0)
    status.zero_()
    out.fill_(5.0)
    tq.tq_sdpa_prompt(q, k, v, dev([0, 20, 40]), dev([0, 0, 20]), 0.125, out, status=status)    # no keys for the first
    assert int(status.item()) == tq.TQ_STATUS_EMPTY_SEQ and torch.all(out[:20] == 0) and torch.all(out[40:] == 5.0)


# ------------------------------------------------------------------------------------------------------- together

@pytest.mark.parametrize("captured", [False, True])
def test_a_serving_loop(gpu, captured):
    """Two layers, three slots: prompts are admitted, attended and cached, steps are decoded, a sequence leaves and another
    takes its slot; every layer uses the same lengths, page table, offsets and slots.  The decode steps run eagerly or
    from one captured graph."""
    tq, torch = gpu
    rng = np.random.default_rng(77)
    B, H_q, H, d, P, layers, num_pages = 3, 8, 2, 128, 16, 2, 40
    t, alpha = torch.float16, 128 ** -0.5
    dev = lambda x, ty=torch.int32: torch.tensor(x, dtype=ty, device="cuda")  # noqa: E731
    table, lens = torch.zeros((B, 12), dtype=torch.int32, device="cuda"), dev([0] * B)
    free, count = torch.randperm(num_pages).int().cuda(), dev([num_pages])
    caches = [tq.PagedKV8Cache.over(torch.full((num_pages, H, 1, tq.TQ_BLOCK8_BYTES(d)), 0xA5, dtype=torch.uint8, device="cuda"), lens, table)
              for _ in range(layers)]
    pwork, work = tq.alloc_pages_workspace(B), tq.alloc_int8_workspace(B, H, H_q, d)
    status, offsets = dev([0]), dev([0] * (B + 1))
    history = [[[] for _ in range(B)] for _ in range(layers)]   # (k, v) rows by layer and sequence
    models = [R.Cache8(num_pages, H, d) for _ in range(layers)]
    place = [[] for _ in range(B)]                              # slots of every sequence, in order

    def qkv(n):
        return torch.from_numpy(rng.standard_normal((n, H_q + 2 * H, d))).to(t).cuda()

    def note(new, slots):
        at = 0
        for b, n in enumerate(new):
            place[b] += slots[at:at + n]
            at += n

    def admit(new, done):
        tq.tq_pages_release(table, lens, dev(done, torch.uint8), P, num_pages, free, count, lens, count, status)
        for b in range(B):
            if done[b]:
                place[b] = []
        n = sum(new)
        slots = torch.empty(n + 2, dtype=torch.int64, device="cuda")
        tq.tq_pages_assign(table, lens, dev(new), P, num_pages, free, count, lens, count, offsets, slots, pwork, status)
        note(new, slots.tolist())
        at = offsets.tolist()
        for i, cache in enumerate(caches):
            x = qkv(n + 2)
            q, k, v = x[:, :H_q], x[:, H_q:H_q + H], x[:, H_q + H:]
            out = torch.full((n + 2, H_q, d), 9.0, dtype=torch.float32, device="cuda")
            tq.tq_sdpa_prompt(q, k, v, offsets, offsets, alpha, out, status=status)
            tq.tq_kv8_append(cache, k, v, slots, status)
            _check_prompt(torch, out, q, k, v, at, at, alpha, True, 0)
            assert torch.all(out[n:] == 9.0)
            models[i].append(k.double().cpu().numpy(), v.double().cpu().numpy(), np.array(slots.tolist()))

    ones, none = dev([1] * B), dev([0] * B, torch.uint8)
    s_slots, s_x = torch.zeros(B, dtype=torch.int64, device="cuda"), [qkv(B) for _ in range(layers)]
    s_out = [torch.zeros((B, H_q, d), dtype=torch.float32, device="cuda") for _ in range(layers)]

    def step():
        tq.tq_pages_release(table, lens, none, P, num_pages, free, count, lens, count, status)
        tq.tq_pages_assign(table, lens, ones, P, num_pages, free, count, lens, count, offsets, s_slots, pwork, status)
        for cache, x, out in zip(caches, s_x, s_out):
            tq.tq_kv8_append(cache, x[:, H_q:H_q + H], x[:, H_q + H:], s_slots, status)
            tq.tq_sdpa_int8_decode(cache, x[:, :H_q], alpha, 0, 0, work, out, status)

    admit([37, 16, 50], [0, 0, 0])
    graph = None
    if captured:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    for turn in range(20):
        if turn == 9:
            admit([0, 30, 0], [0, 1, 0])
        for x in s_x:
            x.copy_(qkv(B))
        graph.replay() if graph else step()
        slots = s_slots.tolist()
        note([1] * B, slots)
        for i, (x, out) in enumerate(zip(s_x, s_out)):
            models[i].append(x[:, H_q:H_q + H].double().cpu().numpy(), x[:, H_q + H:].double().cpu().numpy(), np.array(slots))
            _check_decode(torch, out, x[:, :H_q], [models[i].values(np.array(place[b])) for b in range(B)], alpha, 0, d)
    assert int(status.item()) == 0
    assert lens.tolist() == [len(p) for p in place]
    used = sum(-(-len(p) // P) for p in place)
    assert count.tolist() == [num_pages - used]
    live = set(free.tolist()[:num_pages - used]) | {s // P for p in place for s in p}
    assert live == set(range(num_pages))                        # no page lost, none twice


def test_a_step_that_only_ends_sequences(gpu):
    """Every sequence leaves and none comes: no rows, no slots; the pages are back.  Queries without a single key give zeros."""
    tq, torch = gpu
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    lens, table = ints([20, 16]), ints([[3, 1], [2, 0]])
    free, count = ints([0, 4, 0, 0, 0]), ints([2])
    offsets, slots = ints([9, 9, 9]), torch.empty(0, dtype=torch.int64, device="cuda")
    status = ints([0])
    tq.tq_pages_release(table, lens, torch.ones(2, dtype=torch.bool, device="cuda"), 16, 5, free, count, lens, count, status)
    tq.tq_pages_assign(table, lens, ints([0, 0]), 16, 5, free, count, lens, count, offsets, slots, tq.alloc_pages_workspace(2), status)
    assert lens.tolist() == [0, 0] and count.tolist() == [5] and free.tolist() == [0, 4, 3, 1, 2]
    assert offsets.tolist() == [0, 0, 0] and status.tolist() == [0]
    tq.tq_pages_assign(table, lens, ints([1, 0]), 16, 5, free, count, lens, count, offsets, slots, tq.alloc_pages_workspace(2), status)
    assert lens.tolist() == [0, 0] and count.tolist() == [5] and offsets.tolist() == [0, 0, 0] and status.tolist() == [tq.TQ_STATUS_BAD_LEN]
    cache = tq.PagedKV8Cache(2, 2, 16, 2, 5, 64)
    none = torch.empty((0, 2, 64), dtype=torch.float16, device="cuda")
    tq.tq_kv8_append(cache, none, none, slots)
    tq.tq_kv8_gather(cache, slots, none, none)
    q = torch.ones((3, 4, 64), dtype=torch.float16, device="cuda")
    out = torch.full_like(q, 7.0)
    status.zero_()
    tq.tq_sdpa_prompt(q, none, none, ints([0, 2, 2]), ints([0, 0, 0]), 1.0, out, status=status)
    assert (out[:2] == 0).all() and (out[2] == 7).all() and status.tolist() == [tq.TQ_STATUS_EMPTY_SEQ]
    tq.tq_sdpa_prompt(q[:0], none, none, ints([0, 0]), ints([0, 0]), 1.0, out[:0])
