"""Measured cases of the latent-attention operators: the cache of latent vectors in 8 bits (tq_latent_append,
tq_latent_gather), attention of single tokens over it in the absorbed form (tq_sdpa_latent_decode) and attention of whole
prompts in the expanded form (tq_sdpa_latent_prompt).

A token has one latent vector c (d_c channels) and one positional key r (64 channels), shared by all heads.  Head h of a
model expands c into a key and a value; the absorbed form multiplies the query by the key's expansion instead, so that
all heads attend the latents themselves.  A pass runs either the framework's kernels (`own` true) or the same operators
written with elementary torch operations.  The formulas:

append    Per token a = max |c|, codes round_half_even(127 c / a) with the value code * a / 127; r as fp16(r / s) with the
          value s * that, s the power of two that brings max |r| into [2^15, 2^16).  Magnitudes above 2^64 count as 2^64, a
          latent without any magnitude of 2^-64 as zero; s is at least 2^-126.
gather    The values of given slots.
decode    o_h = sum_t p_ht c_t,  p_h = softmax_t(alpha (qc_h . c_t + qr_h . r_t)),  over the cached tokens of the sequence
          (the last `window` of them).
prompt    o_ih = sum_j p_ihj v_jh,  p_ih = softmax_j(alpha (qn_ih . kn_jh + qr_ih . kr_j)), causal: query i of a sequence
          with lq queries and lk keys sees the keys j with i + lk - lq - window < j <= i + lk - lq.

Layout of a block of 16 tokens, 16 (d_c + 136) bytes: codes (two's complement + 128, one byte each), the positional keys
(fp16 [16][64]), and {a, s} (fp32) of each token.  Byte of the code of (token t, channel c): d_c t + 128 (c / 128) +
16 (c % 64 / 8) + 8 (c % 128 / 64) + c % 8.
"""
import math

import torch

own = False

_TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
_DR = 64  # channels of the positional key


# ------------------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # one decode step's append: a token of each of 32 sequences, into pages: pure latency
        dict(name="append step 32", op="append", B=32, d_c=512, page=64, len_lo=2048, len_hi=16384, new_lo=1, new_hi=1, type="bf16"),
        # packed prompts into the cache, latents and positional keys as slices of the down projection's output
        dict(name="append prompts 16", op="append", B=16, d_c=512, page=64, len_lo=0, len_hi=40, new_lo=1024, new_hi=8192, type="fp16"),
        # decode of one short conversation, 16 heads
        dict(name="decode 1K 16 heads", op="decode", B=1, H=16, d_c=512, page=0, len_lo=1024, len_hi=1024, window=0, type="fp16"),
        # one long conversation, 16 heads: bytes
        dict(name="decode 128K 16 heads", op="decode", B=1, H=16, d_c=512, page=0, len_lo=131072, len_hi=131072, window=0, type="fp16"),
        # one long conversation, all of 128 heads on one GPU
        dict(name="decode 32K 128 heads", op="decode", B=1, H=128, d_c=512, page=64, len_lo=32749, len_hi=32749, window=0, type="bf16"),
        # a ragged batch served from a page pool, 128 heads: arithmetic
        dict(name="decode ragged 32", op="decode", B=32, H=128, d_c=512, page=64, len_lo=2000, len_hi=16384, window=0, type="bf16"),
        # many short conversations with a smaller model's latents, an odd number of heads
        dict(name="decode short 60", op="decode", B=60, H=20, d_c=256, page=16, len_lo=100, len_hi=1500, window=0, type="fp16"),
        # a burst of short prompts through a small model: latency
        dict(name="prompt short", op="prompt", B=16, H=4, d=64, q_lo=1, q_hi=300, past=0, window=0, type="fp16"),
        # one 4K prompt, 64 heads: arithmetic
        dict(name="prompt 4K", op="prompt", B=1, H=64, d=128, q_lo=4096, q_hi=4096, past=0, window=0, type="bf16"),
        # packed prompts of different lengths
        dict(name="prompt ragged 8", op="prompt", B=8, H=32, d=128, q_lo=256, q_hi=2048, past=0, window=0, type="bf16"),
        # chunks of longer prompts, whose first tokens were read back from the cache and expanded
        dict(name="prompt chunk", op="prompt", B=2, H=16, d=128, q_lo=500, q_hi=512, past=3500, window=0, type="fp16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "decode", "decode", "decode", "prompt", "prompt"])
    kind = rng.choice(["fp16", "bf16"])
    if op == "prompt":
        d = rng.choice([64, 128, 128])
        H = _log_int(rng, 1, 64)
        B = _log_int(rng, 1, 16)
        most = 64 * 4096 * 4096 // 2
        hi = _log_int(rng, 2, min(4096, int(math.sqrt(most / (B * H)))))
        past = rng.choice([0, 0, 0, rng.randint(1, 3000)])
        if B * H * hi * (hi + past) > most:
            past = 0
        return dict(op=op, B=B, H=H, d=d, q_lo=max(1, hi // 8), q_hi=hi, past=past, window=rng.choice([0, 0, 0, 1024, 100]), type=kind)
    d_c = rng.choice([512, 512, 512, 256, 128])
    page = rng.choice([0, 16, 64, 128])
    if op == "append":
        B = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, min(32768, 16 * 4096 // B))
        return dict(op=op, B=B, d_c=d_c, page=page, len_lo=0, len_hi=_log_int(rng, 16, 4096), new_lo=max(1, hi // 8), new_hi=hi, type=kind)
    B = _log_int(rng, 1, 64)
    H = _log_int(rng, 1, 128)
    hi = _log_int(rng, 16, min(131072, 32 * 8192 // B))
    return dict(op=op, B=B, H=H, d_c=d_c, page=page, len_lo=max(1, hi // 16), len_hi=hi, window=rng.choice([0, 0, 0, 1024, 1000]), type=kind)


# ----------------------------------------------------------------------------------------------------------- inputs

def _lengths(case, lo, hi):
    """Lengths of the case's sequences: spread evenly over [lo, hi] by a fixed stride, so that they (and with them
    every size of the case) do not depend on the seed."""
    B = case["B"]
    return [lo + ((2 * i + 1) * 7919 * (hi - lo + 1) // (2 * B)) % (hi - lo + 1) if hi > lo else lo for i in range(B)]


def _ceil(a, b):
    return -(-a // b)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def _pool(lens, page, B, g):
    """A page table whose rows name random pages of a pool."""
    pages = [_ceil(n, page) for n in lens]
    num_pages = sum(pages) + 5
    perm = torch.randperm(num_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros((B, max(1, max(pages))), dtype=torch.int32, device="cuda")
    at = torch.arange(table.shape[1], device="cuda")[None, :] < _ints(pages)[:, None]
    table[at] = perm[:sum(pages)]
    return table, num_pages


def _latents(n, d_c, g):
    """Normalised latents as a model has them: channels of different gain, tokens of different size; positional keys with
    a few strong channels (fp32 [n][d_c + 64])."""
    x = torch.randn((n, d_c + _DR), generator=g, device="cuda")
    gain = torch.exp(0.3 * torch.randn((d_c + _DR,), generator=g, device="cuda"))
    gain[d_c + torch.randperm(_DR, generator=g, device="cuda")[:4]] *= 4.0
    return x.mul_(gain).mul_(torch.exp(0.1 * torch.randn((n, 1), generator=g, device="cuda")))


def _fill_cache(pages, blocks, d_c, g):
    """A cache of random contents: pages * blocks blocks that hold quantised latents."""
    n = pages * blocks
    out = torch.empty((n, 16 * (d_c + 136)), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // (16 * d_c))
    for s in range(0, n, step):
        m = min(step, n - s)
        x = _latents(16 * m, d_c, g).half().float()
        out[s:s + m] = _encode(x[:, :d_c], x[:, d_c:]).view(m, -1)
    return out.view(pages, blocks, -1)


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    B, kind = case["B"], _TYPES[case["type"]]
    if case["op"] == "prompt":
        H, d = case["H"], case["d"]
        lq = _lengths(case, case["q_lo"], case["q_hi"])
        lk = [n + case["past"] for n in lq]
        # the projections' outputs, of which the operands are slices: queries per head [d | 64], keys and values [d | d]
        q = torch.randn((sum(lq), H, d + _DR), generator=g, device="cuda").to(kind)
        kv = torch.randn((sum(lk), H, 2 * d), generator=g, device="cuda").to(kind)
        r = _latents(sum(lk), d, g)[:, d:].to(kind)
        cum = lambda ns: _ints([sum(ns[:i]) for i in range(len(ns) + 1)])  # noqa: E731
        s.update(q_n=q[..., :d], q_r=q[..., d:], k_n=kv[..., :d], v=kv[..., d:], k_r=r, q_at=cum(lq), k_at=cum(lk),
                 alpha=(d + _DR) ** -0.5, most_q=max(lq), most_k=max(lk))
        return s
    d_c, page = case["d_c"], case["page"]
    lens = _lengths(case, case["len_lo"], case["len_hi"])
    new = _lengths(case, case["new_lo"], case["new_hi"]) if case["op"] == "append" else [0] * B
    most = _ceil(max(a + b for a, b in zip(lens, new)), 16) * 16
    if page:
        table, pages = _pool([a + b for a, b in zip(lens, new)], page, B, g)
    else:
        table, pages, page = None, B, most
    s.update(blocks=_fill_cache(pages, page // 16, d_c, g), lens=_ints(lens), table=table, page_tokens=page, paged=table is not None)
    if case["op"] == "append":
        x = _latents(sum(new), d_c, g).to(kind)
        rows = torch.repeat_interleave(torch.arange(B, device="cuda"), _ints(new, torch.int64))
        first = _ints([sum(new[:b]) - lens[b] for b in range(B)], torch.int64)
        pos = torch.arange(sum(new), device="cuda") - first[rows]
        held = rows if table is None else table[rows, pos // page].long()
        s.update(c=x[:, :d_c], r=x[:, d_c:], slots=held * page + pos % page)
        return s
    H = case["H"]
    # absorbed queries: per head the latent part and the positional part, scaled so that scores are a few units apart
    q = torch.randn((B, H, d_c + _DR), generator=g, device="cuda").to(kind)
    s.update(q_c=q[..., :d_c], q_r=q[..., d_c:], alpha=1.5 * (d_c + _DR) ** -0.5,
             work=torch.zeros(4096 + 64 * B + 2 * 160 * 64 * (d_c + 8) * 4, dtype=torch.uint8, device="cuda"))
    return s


# ------------------------------------------------------------------------------------- the operators in plain torch

def _order(x):
    """[n][d_c] from channel order into the order of a block's bytes (and _channels back)."""
    n, d_c = x.shape
    return x.reshape(n, d_c // 128, 2, 8, 8).transpose(2, 3).reshape(n, d_c)


def _channels(x):
    n, d_c = x.shape
    return x.reshape(n, d_c // 128, 8, 2, 8).transpose(2, 3).reshape(n, d_c)


def _quantise(c, r):
    """Codes, positional keys (fp16) and {a, s} of fp32 rows."""
    c = c.clamp(-2.0 ** 64, 2.0 ** 64)
    a = c.abs().amax(1)
    a = torch.where(a < 2.0 ** -64, 0.0, a)
    codes = torch.where(a[:, None] > 0, torch.round(c * 127.0 / torch.where(a > 0, a, 1.0)[:, None]), 0.0)
    r = r.clamp(-2.0 ** 64, 2.0 ** 64)
    top = r.abs().amax(1)
    e = torch.where(top > 0, torch.frexp(top).exponent - 16, 0).clamp(min=-126)
    s = torch.ldexp(torch.ones_like(top), e)
    return codes, torch.ldexp(r, -e[:, None]).half(), a, s


def _encode(c, r):
    """Bytes of whole blocks from fp32 rows [16 m][...]."""
    m, d_c = c.shape[0] // 16, c.shape[1]
    codes, r, a, s = _quantise(c, r)
    out = torch.empty((m, 16 * (d_c + 136)), dtype=torch.uint8, device=c.device)
    out[:, :16 * d_c] = _order(codes + 128.0).to(torch.uint8).view(m, 16 * d_c)
    out[:, 16 * d_c:16 * d_c + 2048] = r.contiguous().view(torch.uint8).view(m, 2048)
    out[:, 16 * d_c + 2048:] = torch.stack([a, s], 1).contiguous().view(torch.uint8).view(m, 128)
    return out


def _decode(blocks, d_c):
    """fp32 latents [n][16][d_c] and positional keys [n][16][64] of blocks [n][bytes]."""
    n = blocks.shape[0]
    codes = _channels(blocks[:, :16 * d_c].reshape(16 * n, d_c)).float() - 128.0
    r = blocks[:, 16 * d_c:16 * d_c + 2048].contiguous().view(torch.float16).view(16 * n, _DR).float()
    a, s = blocks[:, 16 * d_c + 2048:].contiguous().view(torch.float32).view(16 * n, 2).unbind(1)
    return (codes * (a / 127.0)[:, None]).view(n, 16, d_c), (r * s[:, None]).view(n, 16, _DR)


def _plain_append(s):
    flat, slots, d_c = s["blocks"].view(-1, s["blocks"].shape[-1]), s["slots"], s["d_c"]
    codes, r, a, scale = _quantise(s["c"].float(), s["r"].float())
    at, t = slots // 16, slots % 16
    flat[:, :16 * d_c].view(-1, 16, d_c)[at, t] = _order(codes + 128.0).to(torch.uint8)
    flat[:, 16 * d_c:16 * d_c + 2048].view(-1, 16, 2 * _DR)[at, t] = r.contiguous().view(torch.uint8)
    flat[:, 16 * d_c + 2048:].view(-1, 16, 8)[at, t] = torch.stack([a, scale], 1).contiguous().view(torch.uint8)


def _plain_gather(s):
    flat, slots = s["blocks"].view(-1, s["blocks"].shape[-1]), s["slots"]
    ids, where = torch.unique_consecutive(slots // 16, return_inverse=True)
    c, r = _decode(flat[ids], s["d_c"])
    return [c[where, slots % 16].to(_TYPES[s["type"]]), r[where, slots % 16].to(_TYPES[s["type"]])]


def _plain_decode(s):
    blocks, d_c, B = s["blocks"], s["d_c"], s["B"]
    blocks = blocks[s["table"].long()] if s["paged"] else blocks[:, None]  # [B][pages][blocks][bytes]
    c, r = (x.view(B, -1, x.shape[-1]) for x in _decode(blocks.reshape(-1, blocks.shape[-1]), d_c))
    scores = torch.matmul(s["q_c"].float(), c.transpose(1, 2))
    scores = (scores + torch.matmul(s["q_r"].float(), r.transpose(1, 2))) * s["alpha"]
    at, lens = torch.arange(c.shape[1], device="cuda")[None, :], s["lens"][:, None]
    seen = at < lens
    if s["window"]:
        seen = seen & (at >= lens - s["window"])
    scores = scores.masked_fill(~seen[:, None], -math.inf)
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    out = torch.matmul(p, c.masked_fill(~seen[..., None], 0.0)) / p.sum(-1, keepdim=True)
    return out.to(_TYPES[s["type"]])


def _plain_prompt(s):
    q_at, k_at = s["q_at"].long(), s["k_at"].long()
    lq, lk = q_at[1:] - q_at[:-1], k_at[1:] - k_at[:-1]
    i, j = torch.arange(s["most_q"], device="cuda"), torch.arange(s["most_k"], device="cuda")
    has_q, has_k = i[None, :] < lq[:, None], j[None, :] < lk[:, None]
    rows_q = (q_at[:-1, None] + i).clamp(max=len(s["q_n"]) - 1)
    rows_k = (k_at[:-1, None] + j).clamp(max=len(s["k_n"]) - 1)
    q_n, q_r = (s[x][rows_q].float().transpose(1, 2) for x in ("q_n", "q_r"))  # [B][H][Lq][d]
    k_n, v = (s[x][rows_k].float().masked_fill(~has_k[..., None, None], 0.0).transpose(1, 2) for x in ("k_n", "v"))
    k_r = s["k_r"][rows_k].float().masked_fill(~has_k[..., None], 0.0)[:, None]
    scores = torch.matmul(q_n, k_n.transpose(-1, -2))
    scores.add_(torch.matmul(q_r, k_r.transpose(-1, -2))).mul_(s["alpha"])
    reach = i[None, :, None] + (lk - lq)[:, None, None]
    hidden = (j > reach) | ~has_k[:, None, :]
    if s["window"]:
        hidden = hidden | (j <= reach - s["window"])
    scores.masked_fill_(hidden[:, None], -math.inf)
    most = scores.amax(-1, keepdim=True)
    scores.sub_(torch.where(most == -math.inf, 0.0, most)).exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.matmul(scores, v) / torch.where(total == 0, 1.0, total)
    return out.transpose(1, 2)[has_q].to(_TYPES[s["type"]])


# -------------------------------------------------------------------------------------------------------------- run

def _cache(s):
    from paper_2604_16957_b200 import tq
    if s["paged"]:
        return tq.PagedLatentCache.over(s["blocks"], s["lens"], s["table"])
    return tq.LatentCache.over(s["blocks"], s["lens"])


def run(s):
    op = s["op"]
    if not own:
        if op == "append":
            _plain_append(s)
            return _plain_gather(s)
        return _plain_decode(s) if op == "decode" else _plain_prompt(s)
    from paper_2604_16957_b200 import tq
    if op == "append":
        cache = _cache(s)
        tq.tq_latent_append(cache, s["c"], s["r"], s["slots"])
        c, r = (torch.empty((len(s["slots"]), d), dtype=_TYPES[s["type"]], device="cuda") for d in (s["d_c"], _DR))
        tq.tq_latent_gather(cache, s["slots"], c, r)
        return [c, r]
    if op == "decode":
        out = torch.empty(s["q_c"].shape, dtype=s["q_c"].dtype, device="cuda")
        tq.tq_sdpa_latent_decode(_cache(s), s["q_c"], s["q_r"], s["alpha"], s["window"], 0, s["work"], out)
        return out
    out = torch.empty(s["q_n"].shape, dtype=s["q_n"].dtype, device="cuda")
    tq.tq_sdpa_latent_prompt(s["q_n"], s["q_r"], s["k_n"], s["k_r"], s["v"], s["q_at"], s["k_at"], s["alpha"], out, causal=True,
                             window=s["window"])
    return out


# ------------------------------------------------------------------------------------------------------------- work

def work(case):
    B = case["B"]
    if case["op"] == "append":
        n, d_c = sum(_lengths(case, case["new_lo"], case["new_hi"])), case["d_c"]
        # 16-bit rows read and their blocks' bytes written; then the other way round; slots twice
        return dict(bytes=n * (2 * (2 * (d_c + _DR) + d_c + 136) + 16), flops=6 * n * d_c)
    if case["op"] == "decode":
        lens, H, d_c = _lengths(case, case["len_lo"], case["len_hi"]), case["H"], case["d_c"]
        tokens = sum(min(n, case["window"]) if case["window"] else n for n in lens)
        return dict(bytes=tokens * (d_c + 136) + 2 * B * H * (2 * d_c + _DR), flops=2 * tokens * H * (2 * d_c + _DR))
    H, d, past, w = case["H"], case["d"], case["past"], case["window"]
    lq = _lengths(case, case["q_lo"], case["q_hi"])
    pairs = sum(_pairs(n, past, w) for n in lq)
    keys = sum(n + past for n in lq)
    return dict(bytes=2 * sum(lq) * H * (2 * d + _DR) + 2 * keys * (2 * H * d + _DR), flops=2 * pairs * H * (2 * d + _DR))


def _pairs(n, past, w):
    """Pairs (query, key) that n queries behind `past` keys see through a window w (0: none)."""
    if not w or past + n <= w:
        return n * past + n * (n + 1) // 2
    full = min(n, max(0, past + n - w + 1))  # queries that see w keys
    return full * w + sum(range(past + 1, past + n - full + 1))


# ------------------------------------------------------------------------------------------- the definition, 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "decode": _exact_decode, "prompt": _exact_prompt}[case["op"]](s)


def _exact_append(s):
    c, r = s["c"].double(), s["r"].double()
    a = c.abs().amax(1, keepdim=True)
    c = torch.round(127.0 * c / a) * a / 127.0
    # fp16 with the largest magnitude in [2^15, 2^16): a step of 2^-10 relative, or of 2^-24 below 2^-14
    scale = torch.exp2(torch.floor(torch.log2(r.abs().amax(1, keepdim=True))) - 15.0)
    x = r / scale
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -14))) - 10.0)
    return [c, torch.round(x / step) * step * scale]


def _exact_tokens(s, b, positions):
    """Latents and positional keys of sequence b at the positions, in 64 bits, byte by byte of the layout."""
    d_c, page = s["d_c"], s["page_tokens"]
    held = s["table"][b, positions // page].long() if s["paged"] else torch.full_like(positions, b)
    blocks = s["blocks"][held, positions % page // 16]
    t = (positions % 16)[:, None]
    ch = torch.arange(d_c, device="cuda")[None, :]
    codes = torch.gather(blocks, 1, d_c * t + 128 * (ch // 128) + 16 * (ch % 64 // 8) + 8 * (ch % 128 // 64) + ch % 8).double() - 128.0
    pick = lambda at, n: torch.gather(blocks, 1, at + torch.arange(n, device="cuda")[None, :]).contiguous()  # noqa: E731
    r = pick(16 * d_c + 128 * t, 128).view(torch.float16).double()
    scales = pick(16 * d_c + 2048 + 8 * t, 8).view(torch.float32).double()
    return codes * scales[:, :1] / 127.0, r * scales[:, 1:]


def _exact_decode(s):
    out = torch.zeros(s["q_c"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["lens"].tolist()):
        low = max(0, n - s["window"]) if s["window"] else 0
        c, r = _exact_tokens(s, b, torch.arange(low, n, device="cuda"))
        z = s["alpha"] * (s["q_c"][b].double() @ c.T + s["q_r"][b].double() @ r.T)
        out[b] = torch.softmax(z, -1) @ c
    return out


def _exact_prompt(s):
    out = torch.zeros(s["q_n"].shape, dtype=torch.float64, device="cuda")
    q_at, k_at = s["q_at"].tolist(), s["k_at"].tolist()
    for b in range(s["B"]):
        lq, lk = q_at[b + 1] - q_at[b], k_at[b + 1] - k_at[b]
        rows, keys = slice(q_at[b], q_at[b + 1]), slice(k_at[b], k_at[b + 1])
        i = torch.arange(lq, device="cuda")[:, None] + lk - lq
        j = torch.arange(lk, device="cuda")[None, :]
        hidden = (j > i) | ((j <= i - s["window"]) if s["window"] else (j < 0))
        for h in range(s["H"]):
            z = torch.cat([s["q_n"][rows, h], s["q_r"][rows, h]], 1).double() @ torch.cat([s["k_n"][keys, h], s["k_r"][keys]], 1).double().T
            out[rows, h] = torch.softmax((s["alpha"] * z).masked_fill(hidden, -math.inf), -1) @ s["v"][keys, h].double()
    return out
