"""Measured cases of the serving operators: page bookkeeping (tq_pages_release, tq_pages_assign), the 8-bit KV cache
(tq_kv8_append, tq_kv8_gather), decode attention over it (tq_sdpa_int8_decode) and attention of whole prompts
(tq_sdpa_prompt).

A pass runs either the framework's kernels (`own` true) or the same operators written with elementary torch
operations.  The formulas:

pages     A pool of pages of `page` tokens; free_pages[0 .. free_count) is a stack.  Release pushes the pages of every
          finished sequence, sequences and pages in ascending order.  Assign appends new_lens[b] tokens to sequence b:
          need_b = ceil((len + new) / page) - ceil(len / page) pages come off the stack in sequence order; token n of
          the packed new tokens gets the slot table[b][pos / page] * page + pos % page, and -1 behind the last token.
append    Tokens are kept in blocks of 16.  A block of one KV head has one range a = max |x| for K and one for V over
          its tokens so far; the code of x is round_half_even(127 x / a), its value code * a / 127.  When a token
          raises the range, the older codes c of the block become round_half_even(c a_old / a_new).
gather    The values of given slots.
decode    softmax(alpha q . K^T) V of one query token per sequence over its cached tokens (the last `window` of them).
prompt    The same for every token of packed sequences, causal: query i of a sequence with lq queries and lk keys sees
          the keys j with i + lk - lq - window < j <= i + lk - lq.

Layout of a block of one KV head (32 d + 16 bytes): K codes, V codes (code + 128 in a byte each), range of K, range of
V (fp32), 8 bytes unused.  Byte of the K code of (token, channel c): 512 (c / 32) + 64 (token % 8) + 16 (c % 32 / 8)
+ 8 (token / 8) + c % 8.  Byte of the V code: 512 (c / 32) + 64 (c % 8) + 16 (token % 8 / 2) + 4 (c % 32 / 8) +
2 (token / 8) + token % 2.
"""
import math

import torch

own = False

_TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # bookkeeping of one decode step of 16 running sequences, one of them finished: pure latency
        dict(name="pages step 16", op="pages", B=16, page=64, len_lo=4096, len_hi=65536, fresh=0, new_hi=1, finished=1),
        # admission of 60 new prompts of up to 8K tokens among 64 slots, small pages
        dict(name="pages prompts 64", op="pages", B=64, page=16, len_lo=100, len_hi=8000, fresh=60, new_hi=8192, finished=2),
        # the decode step's append: one token of each of 16 sequences, into partly filled blocks
        dict(name="append step 16", op="append", B=16, H_q=64, H_kv=8, d=128, page=64, len_lo=4096, len_hi=65536, new_lo=1, new_hi=1, type="bf16"),
        # packed prompts into the cache: 16 ragged prompts, K and V as slices of the fused projection's output
        dict(name="append prompts 16", op="append", B=16, H_q=64, H_kv=8, d=128, page=64, len_lo=0, len_hi=40, new_lo=1024, new_hi=8192, type="fp16"),
        # decode of one short and one long conversation, Llama-shaped heads
        dict(name="decode 1K", op="decode", B=1, H_q=64, H_kv=8, d=128, page=0, len_lo=1024, len_hi=1024, window=0, type="fp16"),
        dict(name="decode 128K", op="decode", B=1, H_q=64, H_kv=8, d=128, page=0, len_lo=131072, len_hi=131072, window=0, type="fp16"),
        # a ragged batch served from a page pool
        dict(name="decode ragged 16", op="decode", B=16, H_q=64, H_kv=8, d=128, page=64, len_lo=4096, len_hi=65536, window=0, type="bf16"),
        # wide heads, few queries per KV head, odd length
        dict(name="decode d256 32K", op="decode", B=1, H_q=32, H_kv=16, d=256, page=0, len_lo=32749, len_hi=32749, window=0, type="bf16"),
        # a burst of short prompts through a small model: latency
        dict(name="prompt short", op="prompt", B=16, H_q=4, H_kv=1, d=64, q_lo=1, q_hi=300, past=0, window=0, type="fp16"),
        # one 8K prompt, Llama-shaped heads: arithmetic
        dict(name="prompt 8K", op="prompt", B=1, H_q=64, H_kv=8, d=128, q_lo=8192, q_hi=8192, past=0, window=0, type="fp16"),
        # packed prompts of different lengths
        dict(name="prompt ragged 8", op="prompt", B=8, H_q=64, H_kv=8, d=128, q_lo=256, q_hi=2048, past=0, window=0, type="bf16"),
        # a chunk of a longer prompt (its first tokens are cached) in a sliding-window layer with wide heads
        dict(name="prompt chunk d256", op="prompt", B=2, H_q=32, H_kv=16, d=256, q_lo=1000, q_hi=1024, past=3000, window=1024, type="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    d = rng.choice([64, 128, 128, 128, 256])
    H_kv = rng.choice([1, 2, 4, 8, 8] + ([16] if d > 64 else []))
    G = rng.choice([1, 2, 3, 4, 8, 8])
    return d, H_kv, H_kv * G


def draw(rng):
    op = rng.choice(["pages", "append", "decode", "decode", "prompt", "prompt"])
    kind = rng.choice(["fp16", "bf16"])
    if op == "pages":
        B = _log_int(rng, 1, 256)
        fresh = rng.randint(0, B)
        return dict(op=op, B=B, page=rng.choice([16, 32, 64, 128]), len_lo=1, len_hi=_log_int(rng, 64, 16384), fresh=fresh,
                    new_hi=_log_int(rng, 1, max(1, min(8192, 500000 // B))), finished=rng.randint(0, B - fresh))
    d, H_kv, H_q = _heads(rng)
    page = rng.choice([0, 16, 64, 128])
    if op == "append":
        B = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, max(1, (16 * 4096 * 1024) // (B * H_kv * d)))
        return dict(op=op, B=B, H_q=H_q, H_kv=H_kv, d=d, page=page, len_lo=0, len_hi=_log_int(rng, 16, 4096), new_lo=max(1, hi // 8), new_hi=hi, type=kind)
    if op == "decode":
        B = _log_int(rng, 1, 64)
        hi = _log_int(rng, 16, min(131072, (16 * 32768 * 1024) // (B * H_kv * d)))
        return dict(op=op, B=B, H_q=H_q, H_kv=H_kv, d=d, page=page, len_lo=max(1, hi // 16), len_hi=hi, window=rng.choice([0, 0, 0, 1024, 1000]), type=kind)
    B = _log_int(rng, 1, 16)
    hi = _log_int(rng, 2, min(4096, int(math.sqrt(64 * 2048 * 2048 * 8 / (B * H_q)))))
    past = rng.choice([0, 0, 0, rng.randint(1, 1000)])
    if B * H_q * hi * (hi + past) * d > 64 * 2048 * 2048 * 8 * 128:
        past = 0
    return dict(op=op, B=B, H_q=H_q, H_kv=H_kv, d=d, q_lo=max(1, hi // 8), q_hi=hi, past=past, window=rng.choice([0, 0, 0, 1024, 100]), type=kind)


# ----------------------------------------------------------------------------------------------------------- inputs

def _lengths(case, lo, hi):
    """Lengths of the case's sequences: spread evenly over [lo, hi] by a fixed stride, so that they (and with them
    every size of the case) do not depend on the seed."""
    B = case["B"]
    return [lo + ((2 * i + 1) * 7919 * (hi - lo + 1) // (2 * B)) % (hi - lo + 1) if hi > lo else lo for i in range(B)]


def _pages_lengths(case):
    """(cached, new, finished) of every sequence: `fresh` empty ones that take a prompt, `finished` ones that leave,
    the others take one token."""
    B, fresh = case["B"], case["fresh"]
    lens = _lengths(case, case["len_lo"], case["len_hi"])
    new = _lengths(case, 1, case["new_hi"])
    done = [fresh <= i < fresh + case["finished"] for i in range(B)]
    cached = [0 if i < fresh else lens[i] for i in range(B)]
    return cached, [new[i] if i < fresh else 0 if done[i] else 1 for i in range(B)], done


def _ceil(a, b):
    return -(-a // b)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def _pool(lens, page, B, g):
    """A page table whose rows name random pages of a pool, and the stack of the pages that are left."""
    pages = [_ceil(n, page) for n in lens]
    max_pages = max(1, max(pages))
    num_pages = sum(pages) + 5
    perm = torch.randperm(num_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros((B, max_pages), dtype=torch.int32, device="cuda")
    at = torch.arange(max_pages, device="cuda")[None, :] < _ints(pages)[:, None]
    table[at] = perm[:sum(pages)]
    return table, perm[sum(pages):], num_pages


def _normal(shape, g, kind, outliers=None):
    x = torch.randn(shape, generator=g, device="cuda")
    if outliers is not None:
        x[..., outliers] *= 10.0
    return x.to(_TYPES[kind])


def _fill_cache(pages, H_kv, blocks, d, g):
    """A cache of random contents: pages * H_kv * blocks blocks with codes of normally distributed values (K with
    four channels ten times the others, as outlier channels of trained models are) and their ranges."""
    n = pages * H_kv * blocks
    out = torch.zeros((n, 32 * d + 16), dtype=torch.uint8, device="cuda")
    channels = torch.randperm(d, generator=g, device="cuda")[:4]
    step = max(1, (1 << 28) // (16 * d))
    for s in range(0, n, step):
        m = min(step, n - s)
        for part in (0, 1):
            x = torch.randn((m, 16, d), generator=g, device="cuda")
            if part == 0:
                x[..., channels] *= 10.0
            a = x.half().float().abs().amax((1, 2))
            c = torch.round(x.half().float() * 127.0 / a[:, None, None]) + 128.0
            out[s:s + m, part * 16 * d:(part + 1) * 16 * d] = _put[part](c.to(torch.uint8))
            out[s:s + m, 32 * d + 4 * part:32 * d + 4 * part + 4] = a[:, None].contiguous().view(torch.uint8)
    return out.view(pages, H_kv, blocks, 32 * d + 16)


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    if case["op"] == "pages":
        cached, new, done = _pages_lengths(case)
        page, B = case["page"], case["B"]
        max_pages = max(_ceil(c + n, page) for c, n in zip(cached, new)) + 1
        table, left, _ = _pool(cached, page, B, g)
        wanted = sum(_ceil(c + n, page) - _ceil(c, page) for c, n in zip(cached, new))
        used = sum(_ceil(c, page) for c in cached)
        num_pages = used + wanted + 5
        perm = torch.randperm(num_pages, generator=g, device="cuda").to(torch.int32)
        full = torch.full((B, max_pages), -1, dtype=torch.int32, device="cuda")
        at = torch.arange(max_pages, device="cuda")[None, :] < _ints([_ceil(c, page) for c in cached])[:, None]
        full[at] = perm[:used]
        free = torch.full((num_pages,), -1, dtype=torch.int32, device="cuda")
        free[:num_pages - used] = perm[used:]
        s.update(table=full, free=free, count=_ints([num_pages - used]), lens=_ints(cached), new=_ints(new),
                 done=_ints([int(x) for x in done], torch.uint8), n=sum(new), num_pages=num_pages, work=_workspace(16 * B + 256))
        return s
    H_q, H_kv, d, B, kind = case["H_q"], case["H_kv"], case["d"], case["B"], case["type"]
    if case["op"] == "prompt":
        lq = _lengths(case, case["q_lo"], case["q_hi"])
        lk = [n + case["past"] for n in lq]
        outliers = torch.randperm(d, generator=g, device="cuda")[:4]
        # q, k, v as a model has them: slices of one projection's output where the prompt has no past
        if case["past"]:
            q, k, v = (_normal((sum(n), h, d), g, kind, o) for n, h, o in ((lq, H_q, None), (lk, H_kv, outliers), (lk, H_kv, None)))
        else:
            x = _normal((sum(lq), H_q + 2 * H_kv, d), g, kind)
            x[:, H_q:H_q + H_kv, outliers] *= 10.0
            q, k, v = x[:, :H_q], x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:]
        cum = lambda ns: _ints([sum(ns[:i]) for i in range(len(ns) + 1)])  # noqa: E731
        s.update(q=q, k=k, v=v, q_at=cum(lq), k_at=cum(lk), alpha=d ** -0.5, most_q=max(lq), most_k=max(lk))
        return s
    page = case["page"]
    lens = _lengths(case, case["len_lo"], case["len_hi"])
    new = _lengths(case, case["new_lo"], case["new_hi"]) if case["op"] == "append" else [0] * B
    most = _ceil(max(a + b for a, b in zip(lens, new)), 16) * 16
    if page:
        table, _, pages = _pool([a + b for a, b in zip(lens, new)], page, B, g)
    else:
        table, pages, page = None, B, most
    blocks = _fill_cache(pages, H_kv, page // 16, d, g)
    s.update(blocks=blocks, lens=_ints(lens), table=table, page_tokens=page, paged=table is not None)
    if case["op"] == "append":
        n = sum(new)
        x = _normal((n, H_q + 2 * H_kv, d), g, kind)
        x[:, H_q:H_q + H_kv, torch.randperm(d, generator=g, device="cuda")[:4]] *= 10.0
        at = _slots_of(lens, new, table, page)
        # what is read back: every token of the blocks that the new tokens fall into
        whole = _slots_of([a // 16 * 16 for a in lens], [a % 16 + b for a, b in zip(lens, new)], table, page)
        s.update(k=x[:, H_q:H_q + H_kv], v=x[:, H_q + H_kv:], slots=at, read=whole)
        return s
    # room for more splits of a sequence than fill the GPU several times
    splits = min(256, 1 + 4096 // (B * H_kv))
    s.update(q=_normal((B, H_q, d), g, kind), alpha=d ** -0.5, work=_workspace(8 * B * H_kv + 4 * B * H_q * splits * (d + 2) + 4096))
    return s


def _workspace(n):
    return torch.zeros(n, dtype=torch.uint8, device="cuda")


def _slots_of(lens, new, table, page):
    rows, at = [], []
    for b, (a, n) in enumerate(zip(lens, new)):
        pos = torch.arange(a, a + n, device="cuda")
        rows.append(torch.full_like(pos, b))
        at.append(pos)
    rows, at = torch.cat(rows), torch.cat(at)
    pages = rows if table is None else table[rows, at // page].long()
    return pages * page + at % page


# ------------------------------------------------------------------------------------- the operators in plain torch

def _k_put(c):
    m, _, d = c.shape  # [m][16][d] -> [m][16 d] in the order of the layout
    return c.view(m, 2, 8, d // 32, 4, 8).permute(0, 3, 2, 4, 1, 5).reshape(m, 16 * d)


def _v_put(c):
    m, _, d = c.shape
    return c.view(m, 2, 4, 2, d // 32, 4, 8).permute(0, 4, 6, 2, 5, 1, 3).reshape(m, 16 * d)


def _k_get(x):
    m, d = x.shape[0], x.shape[1] // 16
    return x.view(m, d // 32, 8, 4, 2, 8).permute(0, 4, 2, 1, 3, 5).reshape(m, 16, d)


def _v_get(x):
    m, d = x.shape[0], x.shape[1] // 16
    return x.view(m, d // 32, 8, 4, 4, 2, 2).permute(0, 5, 3, 6, 1, 4, 2).reshape(m, 16, d)


_put, _get = (_k_put, _v_put), (_k_get, _v_get)


def _plain_release(s):
    page, B, wide = s["page"], s["B"], s["table"].shape[1]
    pages = torch.where(s["done"].bool(), (s["lens"] + page - 1) // page, 0)
    mine = torch.arange(wide, device="cuda")[None, :] < pages[:, None]
    at = s["count"] + (torch.cumsum(mine.flatten(), 0) - 1).view(B, wide)
    s["free"][at[mine]] = s["table"][mine]
    return torch.where(s["done"].bool(), 0, s["lens"]), s["count"] + pages.sum().to(torch.int32)


def _plain_assign(s, lens, count):
    page, table, free, n = s["page"], s["table"], s["free"], s["n"]
    wide = table.shape[1]
    old, new = lens.long(), s["new"].long()
    ends = torch.cumsum(new, 0)
    starts = ends - new
    fits = (old + new <= wide * page) & (ends <= n)
    first, last = (old + page - 1) // page, (old + new + page - 1) // page
    need = torch.where(fits, last - first, 0)
    upto = torch.cumsum(need, 0)
    ok = fits & ((need == 0) | (upto <= count))
    i = torch.arange(wide, device="cuda")[None, :]
    fresh = ok[:, None] & (i >= first[:, None]) & (i < last[:, None])
    at = count - 1 - ((upto - need)[:, None] + i - first[:, None])
    table[fresh] = free[at[fresh]]
    taken = torch.where(ok, upto, 0).amax()
    token = torch.arange(n, device="cuda")
    row = torch.searchsorted(ends, token, right=True).clamp(max=len(old) - 1)
    pos = old[row] + token - starts[row]
    slots = table[row, (pos // page).clamp(max=wide - 1)].long() * page + pos % page
    slots = torch.where(ok[row] & (token < ends[-1]), slots, -1)
    offsets = torch.cat([torch.zeros_like(ends[:1]), ends]).to(torch.int32)
    return dict(lens=torch.where(ok, old + new, old).to(torch.int32), count=(count - taken).to(torch.int32), offsets=offsets,
                slots=slots, table=table, free=free)


def _block_rows(s, ids):
    """(page, block) of the blocks whose number in slots / 16 is ids."""
    per = s["page_tokens"] // 16
    return ids // per, ids % per


def _plain_append(s):
    blocks, slots, d = s["blocks"], s["slots"], s["d"]
    ids, off = slots // 16, slots % 16
    leader = torch.ones_like(ids, dtype=torch.bool)
    leader[1:] = ids[1:] != ids[:-1]
    run = torch.cumsum(leader, 0) - 1
    page, block = _block_rows(s, ids[leader])
    before = off[leader]
    R, H = len(before), s["H_kv"]
    older = (torch.arange(16, device="cuda")[None, :] < before[:, None])[:, None, :, None]
    bytes_ = blocks[page, :, block]
    out = torch.empty_like(bytes_)
    ranges = bytes_[..., 32 * d:32 * d + 8].contiguous().view(torch.float32)
    made = torch.zeros_like(ranges)
    for part, x in ((0, s["k"].float()), (1, s["v"].float())):
        a_old = torch.where(before[:, None] > 0, ranges[..., part], 0.0)
        a_new = a_old.clone().scatter_reduce_(0, run[:, None].expand(-1, H), x.abs().amax(-1), "amax")
        div = torch.where(a_new > 0, a_new, 1.0)
        codes = _get[part](bytes_[..., 16 * d * part:16 * d * (part + 1)].reshape(R * H, 16 * d)).view(R, H, 16, d).float() - 128.0
        codes = torch.where(older, torch.round(codes * a_old[..., None, None] / div[..., None, None]), 0.0)
        codes[run, :, off] = torch.round(x * 127.0 / div[run][..., None])
        out[..., 16 * d * part:16 * d * (part + 1)] = _put[part]((codes + 128.0).to(torch.uint8).view(R * H, 16, d)).view(R, H, 16 * d)
        made[..., part] = a_new
    out[..., 32 * d:32 * d + 8] = made.view(torch.uint8)
    out[..., 32 * d + 8:] = 0
    blocks[page, :, block] = out


def _plain_gather(s):
    blocks, slots, d, H = s["blocks"], s["read"], s["d"], s["H_kv"]
    ids, inverse = torch.unique_consecutive(slots // 16, return_inverse=True)
    page, block = _block_rows(s, ids)
    bytes_ = blocks[page, :, block]
    ranges = bytes_[..., 32 * d:32 * d + 8].contiguous().view(torch.float32)
    back = []
    for part in (0, 1):
        codes = _get[part](bytes_[..., 16 * d * part:16 * d * (part + 1)].reshape(-1, 16 * d)).view(-1, H, 16, d)
        x = (codes[inverse, :, slots % 16].float() - 128.0) * (ranges[..., part] / 127.0)[inverse][..., None]
        back.append(x.to(_TYPES[s["type"]]))
    return back


def _plain_decode(s):
    blocks, d, B, H = s["blocks"], s["d"], s["B"], s["H_kv"]
    page, G = s["page_tokens"], s["H_q"] // s["H_kv"]
    bytes_ = blocks[s["table"].long()] if s["paged"] else blocks[:, None]  # [B][pages][H][blocks][bytes]
    S = bytes_.shape[1] * page
    bytes_ = bytes_.permute(0, 2, 1, 3, 4).reshape(B, H, S // 16, 32 * d + 16)
    ranges = bytes_[..., 32 * d:32 * d + 8].contiguous().view(torch.float32) / 127.0
    values = [_get[p](bytes_[..., 16 * d * p:16 * d * (p + 1)].reshape(-1, 16 * d)).view(B, H, S // 16, 16, d).float().sub_(128.0)
              .mul_(ranges[..., p, None, None]).view(B, H, S, d) for p in (0, 1)]
    q = s["q"].float().view(B, H, G, d)
    scores = torch.matmul(q, values[0].transpose(-1, -2)) * s["alpha"]
    at = torch.arange(S, device="cuda")[None, :]
    lens = s["lens"][:, None]
    seen = at < lens
    if s["window"]:
        seen = seen & (at >= lens - s["window"])
    scores = scores.masked_fill(~seen[:, None, None, :], -math.inf)
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    out = torch.matmul(p, values[1].masked_fill(~seen[:, None, :, None], 0.0)) / p.sum(-1, keepdim=True)
    return out.view(B, H * G, d).to(_TYPES[s["type"]])


def _plain_prompt(s):
    B, H, d, G = s["B"], s["H_kv"], s["d"], s["H_q"] // s["H_kv"]
    q_at, k_at = s["q_at"].long(), s["k_at"].long()
    lq, lk = q_at[1:] - q_at[:-1], k_at[1:] - k_at[:-1]
    i, j = torch.arange(s["most_q"], device="cuda"), torch.arange(s["most_k"], device="cuda")
    has_q, has_k = i[None, :] < lq[:, None], j[None, :] < lk[:, None]
    q = s["q"][(q_at[:-1, None] + i).clamp(max=len(s["q"]) - 1)].float()  # [B][Lq][H_q][d]
    k, v = (x[(k_at[:-1, None] + j).clamp(max=len(x) - 1)].float().masked_fill(~has_k[..., None, None], 0.0).permute(0, 2, 1, 3)
            for x in (s["k"], s["v"]))
    q = q.view(B, -1, H, G, d).permute(0, 2, 3, 1, 4).reshape(B, H, G * len(i), d)
    scores = torch.matmul(q, k.transpose(-1, -2)).mul_(s["alpha"]).view(B, H, G, len(i), len(j))
    reach = i[None, :, None] + (lk - lq)[:, None, None]
    hidden = (j > reach) | ~has_k[:, None, :]
    if s["window"]:
        hidden = hidden | (j <= reach - s["window"])
    scores.masked_fill_(hidden[:, None, None], -math.inf)
    most = scores.amax(-1, keepdim=True)
    scores.sub_(torch.where(most == -math.inf, 0.0, most)).exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.matmul(scores.view(B, H, -1, len(j)), v).view(B, H, G, len(i), d) / torch.where(total == 0, 1.0, total)
    out = out.permute(0, 3, 1, 2, 4).reshape(B, len(i), H * G, d)
    return out[has_q].to(_TYPES[s["type"]])


# -------------------------------------------------------------------------------------------------------------- run

def _cache(s):
    from paper_2604_16957_b200 import tq
    if s["paged"]:
        return tq.PagedKV8Cache.over(s["blocks"], s["lens"], s["table"])
    return tq.KV8Cache.over(s["blocks"], s["lens"])


def run(s):
    op = s["op"]
    if not own:
        if op == "pages":
            return _plain_assign(s, *_plain_release(s))
        if op == "append":
            _plain_append(s)
            return _plain_gather(s)
        return _plain_decode(s) if op == "decode" else _plain_prompt(s)
    from paper_2604_16957_b200 import tq
    if op == "pages":
        lens, count = torch.empty_like(s["lens"]), torch.empty_like(s["count"])
        offsets = torch.empty(s["B"] + 1, dtype=torch.int32, device="cuda")
        slots = torch.empty(s["n"], dtype=torch.int64, device="cuda")
        tq.tq_pages_release(s["table"], s["lens"], s["done"], s["page"], s["num_pages"], s["free"], s["count"], lens, count)
        tq.tq_pages_assign(s["table"], lens, s["new"], s["page"], s["num_pages"], s["free"], count, lens, count, offsets, slots, s["work"])
        return dict(lens=lens, count=count, offsets=offsets, slots=slots, table=s["table"], free=s["free"])
    if op == "append":
        cache = _cache(s)
        tq.tq_kv8_append(cache, s["k"], s["v"], s["slots"])
        shape = (len(s["read"]), s["H_kv"], s["d"])
        k, v = (torch.empty(shape, dtype=_TYPES[s["type"]], device="cuda") for _ in range(2))
        tq.tq_kv8_gather(cache, s["read"], k, v)
        return [k, v]
    if op == "decode":
        out = torch.empty_like(s["q"])
        tq.tq_sdpa_int8_decode(_cache(s), s["q"], s["alpha"], s["window"], 0, s["work"], out)
        return out
    out = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
    tq.tq_sdpa_prompt(s["q"], s["k"], s["v"], s["q_at"], s["k_at"], s["alpha"], out, causal=True, window=s["window"])
    return out


# ------------------------------------------------------------------------------------------------------------- work

def work(case):
    if case["op"] == "pages":
        cached, new, done = _pages_lengths(case)
        page = case["page"]
        moved = sum(_ceil(c, page) for c, x in zip(cached, done) if x)
        taken = sum(_ceil(c + n, page) - _ceil(c, page) for c, n in zip(cached, new))
        # lengths in and out, offsets; a released or a taken page is read once and written once; 8 bytes a slot
        return dict(bytes=17 * case["B"] + 8 * (moved + taken) + 8 * sum(new), flops=0)
    H_q, H_kv, d, B = case["H_q"], case["H_kv"], case["d"], case["B"]
    if case["op"] == "append":
        lens, new = _lengths(case, case["len_lo"], case["len_hi"]), _lengths(case, case["new_lo"], case["new_hi"])
        older, n = sum(a % 16 for a in lens), sum(new)
        row = 2 * H_kv * d  # values of a token
        # new tokens read (16 bits) and their codes written, older codes of their blocks read and written again; then
        # the blocks' codes read and their values written (16 bits)
        return dict(bytes=row * (2 * n + n + 2 * older) + row * 3 * (n + older), flops=4 * row * (n + older))
    if case["op"] == "decode":
        lens = _lengths(case, case["len_lo"], case["len_hi"])
        tokens = sum(min(n, case["window"]) if case["window"] else n for n in lens)
        return dict(bytes=tokens * H_kv * (2 * d + 0.5) + 4 * B * H_q * d, flops=4 * tokens * H_q * d)
    lq = _lengths(case, case["q_lo"], case["q_hi"])
    past, w = case["past"], case["window"]
    pairs = sum(_pairs(n, past, w) for n in lq)
    return dict(bytes=4 * sum(lq) * H_q * d + 4 * sum(n + past for n in lq) * H_kv * d, flops=4 * pairs * H_q * d)


def _pairs(n, past, w):
    """Pairs (query, key) that n queries behind `past` keys see through a window w (0: none)."""
    if not w or past + n <= w:
        return n * past + n * (n + 1) // 2
    full = min(n, max(0, past + n - w + 1))  # queries that see w keys
    return full * w + sum(range(past + 1, past + n - full + 1))


# ------------------------------------------------------------------------------------------- the definition, 64 bits

def _bytes_of(d):
    """Byte of the K and of the V code of (token, channel) in a block: int64 [16][d] each, from the formulas above."""
    t = torch.arange(16, device="cuda")[:, None]
    c = torch.arange(d, device="cuda")[None, :]
    k = 512 * (c // 32) + 64 * (t % 8) + 16 * (c % 32 // 8) + 8 * (t // 8) + c % 8
    v = 16 * d + 512 * (c // 32) + 64 * (c % 8) + 16 * (t % 8 // 2) + 4 * (c % 32 // 8) + 2 * (t // 8) + t % 2
    return k, v


def _read64(blocks, page, h, block, d):
    """K and V codes (fp64, [m][16][d]) and ranges ([m][2]) of the blocks (page, h, block)."""
    x = blocks[page, h, block]
    k, v = (x[:, b.flatten()].view(-1, 16, d).double() - 128.0 for b in _bytes_of(d))
    return k, v, x[:, 32 * d:32 * d + 8].contiguous().view(torch.float32).double()


def exact(case, seed):
    if case["op"] == "pages":
        return None  # whole numbers
    s = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(s)
    return _exact_decode(s) if case["op"] == "decode" else _exact_prompt(s)


def _exact_append(s):
    d, H, slots = s["d"], s["H_kv"], s["slots"]
    total = s["blocks"].shape[0] * s["blocks"].shape[2]  # blocks of the cache, numbered as slots / 16
    per = s["blocks"].shape[2]
    first = torch.full((total,), 16, device="cuda", dtype=torch.int64)
    first.scatter_reduce_(0, slots // 16, slots % 16, "amin")  # first new token of each block
    touched = torch.unique(slots // 16)
    back = [torch.empty((len(s["read"]), H, d), dtype=torch.float64, device="cuda") for _ in range(2)]
    where = torch.full((total,), -1, device="cuda", dtype=torch.int64)
    where[touched] = torch.arange(len(touched), device="cuda")
    for h in range(H):
        k, v, a = _read64(s["blocks"], touched // per, h, touched % per, d)
        for part, codes, x in ((0, k, s["k"]), (1, v, s["v"])):
            x = x[:, h].double()
            start = first[touched]
            old = torch.where(start > 0, a[:, part], 0.0)
            top = torch.zeros((total,), dtype=torch.float64, device="cuda").scatter_reduce_(0, slots // 16, x.abs().amax(1), "amax")[touched]
            new = torch.maximum(old, top)
            safe = torch.where(new > 0, new, 1.0)[:, None, None]
            codes = torch.round(codes * old[:, None, None] / safe)
            mine = where[slots // 16]
            codes[mine, slots % 16] = torch.round(127.0 * x / safe[mine, 0])
            values = codes * (new / 127.0)[:, None, None]
            back[part][:, h] = values[where[s["read"] // 16], s["read"] % 16]
    return back


def _exact_decode(s):
    d, H, G = s["d"], s["H_kv"], s["H_q"] // s["H_kv"]
    per = s["blocks"].shape[2]
    out = torch.zeros((s["B"], s["H_q"], d), dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["lens"].tolist()):
        low = max(0, n - s["window"]) if s["window"] else 0
        j = torch.arange(low // 16, _ceil(n, 16), device="cuda")
        page = torch.full_like(j, b) if not s["paged"] else s["table"][b, j // per].long()
        for h in range(H):
            k, v, a = _read64(s["blocks"], page, h, j % per, d)
            k = (k * (a[:, 0] / 127.0)[:, None, None]).view(-1, d)[low % 16:low % 16 + n - low]
            v = (v * (a[:, 1] / 127.0)[:, None, None]).view(-1, d)[low % 16:low % 16 + n - low]
            z = s["q"][b, h * G:(h + 1) * G].double() @ k.T * s["alpha"]
            out[b, h * G:(h + 1) * G] = torch.softmax(z, -1) @ v
    return out


def _exact_prompt(s):
    G, H = s["H_q"] // s["H_kv"], s["H_kv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    q_at, k_at = s["q_at"].tolist(), s["k_at"].tolist()
    for b in range(s["B"]):
        lq, lk = q_at[b + 1] - q_at[b], k_at[b + 1] - k_at[b]
        i = torch.arange(lq, device="cuda")[:, None] + lk - lq
        j = torch.arange(lk, device="cuda")[None, :]
        seen = (j <= i) & ((j > i - s["window"]) if s["window"] else (j >= 0))
        for h in range(H):
            k, v = (x[k_at[b]:k_at[b + 1], h].double() for x in (s["k"], s["v"]))
            for g in range(G):
                z = s["q"][q_at[b]:q_at[b + 1], h * G + g].double() @ k.T * s["alpha"]
                out[q_at[b]:q_at[b + 1], h * G + g] = torch.softmax(z.masked_fill(~seen, -math.inf), -1) @ v
    return out
