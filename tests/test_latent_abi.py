"""The latent-attention operators' layout helpers, sizes and refusals, without a GPU: every bad argument is answered before
anything is launched."""
import ctypes as C

import pytest

import latent_ref as L


@pytest.fixture(scope="module")
def tq():
    from paper_2604_16957_b200 import build
    build.build()
    from paper_2604_16957_b200 import tq
    return tq


def test_block_layout(tq):
    for d_c in (128, 256, 512):
        at = L.code_offsets(d_c)
        assert sorted(at.flatten().tolist()) == list(range(16 * d_c))
        for t in range(16):
            for c in range(d_c):
                assert tq._lib.tq_cache_latent_code_offset(d_c, t, c) == at[t, c]
        assert tq.TQ_BLOCK_LATENT_BYTES(d_c) == 16 * (d_c + 2 * 64 + 8) == tq._lib.tq_cache_latent_bytes(1, 16, d_c)
    assert tq._lib.tq_cache_latent_bytes(3, 33, 512) == 3 * 3 * 10368 and tq._lib.tq_cache_latent_bytes(0, 33, 512) == 0


def test_workspace_sizes(tq):
    size = tq._lib.tq_latent_workspace_bytes
    assert size(0, 16, 512) == size(1, 0, 512) == size(1, 1025, 512) == 0
    for B, H, d_c in ((1, 1, 128), (1, 128, 512), (64, 20, 256), (65535, 1024, 512)):
        # at least the partial results of a thread block per SM: rows, maxima and sums
        assert size(B, H, d_c) >= 148 * min(H, 16) * (d_c + 2) * 4 and size(B, H, d_c) % 4 == 0
        assert size(B + 1, H, d_c) >= size(B, H, d_c)


F = 0x1000  # never dereferenced: validation fails first


def _cache(tq, **kw):
    return tq.tq_latent_cache(**{**dict(blocks=F, seq_lens=F, B=1, S_cap=64, d_c=512), **kw})


def _paged(tq, **kw):
    return _cache(tq, **{**dict(S_cap=128, page_table=F, page_tokens=32, max_pages=4, num_pages=9), **kw})


def _caches(tq):
    for bad in [dict(d_c=64), dict(d_c=1024), dict(d_c=0), dict(S_cap=60), dict(S_cap=0), dict(B=70000), dict(B=0)]:
        yield _cache(tq, **bad), tq.TQ_ERR_SHAPE
    for bad in [dict(page_tokens=48), dict(page_tokens=8), dict(max_pages=3), dict(num_pages=0)]:
        yield _paged(tq, **bad), tq.TQ_ERR_SHAPE
    yield _cache(tq, blocks=F + 8), tq.TQ_ERR_ALIGN
    yield _cache(tq, seq_lens=F + 2), tq.TQ_ERR_ALIGN
    yield _paged(tq, page_table=F + 2), tq.TQ_ERR_ALIGN
    yield _cache(tq, blocks=None), tq.TQ_ERR_NULL
    yield _cache(tq, seq_lens=None), tq.TQ_ERR_NULL


def _vary(good, changes):
    for at, value, code in changes:
        args = list(good)
        args[at] = value
        yield args, code


def _check_all(call, good, changes, tq):
    for args, code in _vary(good, changes):
        assert call(*args) == code, args
    for bad, code in _caches(tq):
        assert call(C.byref(bad), *good[1:]) == code


def test_append_and_gather_refuse(tq):
    N, S, A = tq.TQ_ERR_NULL, tq.TQ_ERR_SHAPE, tq.TQ_ERR_ALIGN
    ok = _cache(tq)
    good = [C.byref(ok), F, F, tq.TQ_FP16, 576, 576, F, 5, None, None]
    _check_all(tq._lib.tq_latent_append, good, [
        (0, None, N), (1, None, N), (2, None, N), (6, None, N), (3, tq.TQ_FP32, S), (3, 7, S), (4, 504, S), (4, 516, S), (5, 56, S),
        (5, 68, S), (7, -1, S), (7, 1 << 31, S), (1, F + 8, A), (2, F + 2, A), (6, F + 4, A), (8, F + 2, A)], tq)
    good = [C.byref(ok), F, 5, F, F, tq.TQ_BF16, None, None]
    _check_all(tq._lib.tq_latent_gather, good, [
        (0, None, N), (1, None, N), (3, None, N), (4, None, N), (2, -1, S), (2, 1 << 31, S), (5, 9, S), (1, F + 4, A), (3, F + 8, A),
        (4, F + 8, A), (6, F + 2, A)], tq)
    # nothing to do is no error, and no address is looked at
    assert tq._lib.tq_latent_append(C.byref(ok), None, None, 0, 0, 0, None, 0, None, None) == tq.TQ_OK
    assert tq._lib.tq_latent_gather(C.byref(ok), None, 0, None, None, 0, None, None) == tq.TQ_OK


def _heads(tq, data=F, row=8192, head=512):
    return C.byref(tq.tq_heads(data, row, head))


def test_decode_refuses(tq):
    N, S, A, W = tq.TQ_ERR_NULL, tq.TQ_ERR_SHAPE, tq.TQ_ERR_ALIGN, tq.TQ_ERR_WORKSPACE
    ok = _cache(tq)
    need = tq._lib.tq_latent_workspace_bytes(1, 16, 512)
    good = [C.byref(ok), _heads(tq), _heads(tq, head=64), tq.TQ_BF16, 16, 0.1, 0, 0, F, need, F, tq.TQ_BF16, None, None]
    _check_all(tq._lib.tq_sdpa_latent_decode, good, [
        (0, None, N), (1, None, N), (2, None, N), (1, _heads(tq, data=None), N), (2, _heads(tq, data=None), N), (8, None, N), (10, None, N),
        (4, 0, S), (4, 1025, S), (3, tq.TQ_FP32, S), (11, tq.TQ_FP16, S), (6, -1, S), (7, -1, S), (1, _heads(tq, head=504), S),
        (1, _heads(tq, row=504), S), (1, _heads(tq, row=8196), S), (2, _heads(tq, head=68), S), (2, _heads(tq, head=56), S),
        (1, _heads(tq, data=F + 8), A), (2, _heads(tq, data=F + 2), A), (8, F + 8, A), (10, F + 4, A), (12, F + 2, A), (9, need - 1, W)], tq)
    # line positions are 30 bits
    big = _cache(tq, B=60000, S_cap=1 << 21)
    assert tq._lib.tq_sdpa_latent_decode(C.byref(big), *good[1:]) == S


def test_prompt_refuses(tq):
    N, S, A = tq.TQ_ERR_NULL, tq.TQ_ERR_SHAPE, tq.TQ_ERR_ALIGN
    h = lambda **kw: _heads(tq, **{**dict(row=1024, head=256), **kw})  # noqa: E731
    good = [h(), h(), h(), F, 64, h(), tq.TQ_BF16, 9, 9, F, F, 1, 4, 128, 0.1, 1, 0, F, tq.TQ_BF16, None, None]
    for args, code in _vary(good, [
            (0, None, N), (1, None, N), (2, None, N), (5, None, N), (0, h(data=None), N), (1, h(data=None), N), (2, h(data=None), N),
            (3, None, N), (5, h(data=None), N), (9, None, N), (10, None, N), (17, None, N), (11, 0, S), (11, 65536, S), (12, 0, S),
            (12, 4097, S), (13, 96, S), (13, 256, S), (7, -1, S), (8, -1, S), (6, tq.TQ_FP32, S), (18, tq.TQ_FP16, S), (16, -1, S),
            (0, h(head=120), S), (0, h(row=132), S), (1, h(head=56), S), (2, h(row=64), S), (5, h(head=252), S), (4, 56, S), (4, 68, S),
            (0, h(row=1 << 40), S), (0, h(data=F + 8), A), (1, h(data=F + 8), A), (2, h(data=F + 8), A), (5, h(data=F + 8), A),
            (3, F + 8, A), (9, F + 2, A), (10, F + 2, A), (17, F + 8, A), (19, F + 2, A)]):
        assert tq._lib.tq_sdpa_latent_prompt(*args) == code, args
    args = list(good)
    args[15], args[16] = 0, 5   # a window without a causal mask
    assert tq._lib.tq_sdpa_latent_prompt(*args) == S
    args = list(good)
    args[7] = 0                 # no queries
    assert tq._lib.tq_sdpa_latent_prompt(*args) == tq.TQ_OK


def test_cache_objects_refuse(tq):
    import torch
    z = lambda *s, t=torch.uint8: torch.zeros(s, dtype=t)  # noqa: E731
    lens = z(2, t=torch.int32)
    c = tq.LatentCache.over(z(2, 4, 10368), lens)
    assert (c.B, c.S_cap, c.d_c) == (2, 64, 512)
    p = tq.PagedLatentCache.over(z(5, 2, 6272), lens, z(2, 3, t=torch.int32))
    assert (p.B, p.S_cap, p.d_c, p.page_tokens, p.max_pages, p.num_pages) == (2, 96, 256, 32, 3, 5)
    s = p.struct()
    assert (s.B, s.S_cap, s.d_c, s.num_pages) == (2, 96, 256, 5) and s.blocks == p.blocks.data_ptr()
    for bad in (lambda: tq.LatentCache.over(z(2, 4, 10369), lens), lambda: tq.LatentCache.over(z(3, 4, 10368), lens),
                lambda: tq.LatentCache.over(z(2, 4, 10368, t=torch.int8), lens), lambda: tq.LatentCache.over(z(2, 10368), lens),
                lambda: tq.LatentCache.over(z(2, 4, 2176), lens), lambda: tq.LatentCache.over(z(2, 4, 16), lens),
                lambda: tq.LatentCache.over(z(2, 4, 10368), lens.long()), lambda: tq.LatentCache.over(z(2, 8, 10368)[:, ::2], lens),
                lambda: tq.PagedLatentCache.over(z(5, 2, 6272), lens, z(3, 3, t=torch.int32)),
                lambda: tq.PagedLatentCache.over(z(5, 2, 6272), lens, z(2, 3, t=torch.int64)),
                lambda: tq.LatentCache(1, 60, 512, device="cpu"), lambda: tq.LatentCache(1, 64, 100, device="cpu"),
                lambda: tq.PagedLatentCache(1, 48, 2, 3, 512, device="cpu"), lambda: tq.LatentCache.over(3, lens)):
        with pytest.raises(tq.TqError):
            bad()
    # a call with another kind of cache, or on the host
    kv8 = tq.KV8Cache(1, 2, 64, 128, device="cpu")
    for cache in (kv8, c, None):
        with pytest.raises(tq.TqError):
            tq.tq_latent_gather(cache, z(1, t=torch.int64), z(1, 512, t=torch.float32), z(1, 64, t=torch.float32))
    c.blocks.resize_(2, 3, 10368)
    with pytest.raises(tq.TqError):
        c.struct()
