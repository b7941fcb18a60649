"""The serving operators' layout helpers and refusals, without a GPU: every bad argument is answered before anything is
launched."""
import ctypes as C

import pytest

import serving_ref as R


@pytest.fixture(scope="module")
def tq():
    from paper_2604_16957_b200 import build
    build.build()
    from paper_2604_16957_b200 import tq
    return tq


def test_block_layout(tq):
    for d in (64, 128, 256, 512):
        k, v = R.code_offsets(d)
        seen = set()
        for t in range(16):
            for c in range(d):
                assert tq._lib.tq_cache8_code_offset(d, 0, t, c) == k[t, c]
                assert tq._lib.tq_cache8_code_offset(d, 1, t, c) == v[t, c]
                seen.update((int(k[t, c]), int(v[t, c])))
        assert seen == set(range(32 * d))
        assert tq.TQ_BLOCK8_BYTES(d) == 32 * d + 16 == tq._lib.tq_cache8_bytes(1, 1, 16, d)
    assert tq._lib.tq_cache8_bytes(2, 8, 33, 128) == 2 * 8 * 3 * 4112 and tq._lib.tq_cache8_bytes(0, 8, 33, 128) == 0


def test_workspace_sizes(tq):
    assert tq._lib.tq_pages_workspace_bytes(0) == 0 and tq._lib.tq_pages_workspace_bytes(7) >= 64
    assert tq._lib.tq_int8_counter_bytes(3, 2, 34) >= 4 * 3 * 2 * 3 and tq._lib.tq_int8_counter_bytes(1, 4, 2) == 0
    # 148 thread blocks, 8 units: 156 parts of 8 rows, 8 maxima and 8 sums; many units: two parts per thread block
    assert tq._lib.tq_int8_workspace_bytes(1, 8, 64, 128) == tq._lib.tq_int8_counter_bytes(1, 8, 64) + 156 * 8 * 130 * 4
    assert tq._lib.tq_int8_workspace_bytes(64, 8, 24, 64) == tq._lib.tq_int8_counter_bytes(64, 8, 24) + 296 * (3 * 64 + 8) * 4
    assert tq._lib.tq_int8_workspace_bytes(1, 1, 1, 64) == 256 + 149 * 68 * 4


F = 0x1000  # never dereferenced: validation fails first


def _cache(tq, **kw):
    return tq.tq_kv8_cache(**{**dict(blocks=F, seq_lens=F, B=1, H_kv=2, S_cap=64, d=128), **kw})


def _paged(tq, **kw):
    return _cache(tq, **{**dict(S_cap=128, page_table=F, page_tokens=32, max_pages=4, num_pages=9), **kw})


BAD_CACHES = [dict(d=100), dict(S_cap=60), dict(H_kv=0), dict(B=70000), dict(B=0)]
BAD_PAGED = [dict(page_tokens=48), dict(page_tokens=8), dict(max_pages=3), dict(num_pages=0)]


def _caches(tq):
    for bad in BAD_CACHES:
        yield _cache(tq, **bad), tq.TQ_ERR_SHAPE
    for bad in BAD_PAGED:
        yield _paged(tq, **bad), tq.TQ_ERR_SHAPE
    yield _cache(tq, blocks=F + 8), tq.TQ_ERR_ALIGN
    yield _paged(tq, page_table=F + 2), tq.TQ_ERR_ALIGN
    yield _cache(tq, blocks=None), tq.TQ_ERR_NULL


def _vary(good, changes):
    for at, value, code in changes:
        args = list(good)
        args[at] = value
        yield args, code


def test_append_and_gather_refuse(tq):
    N, S, A = tq.TQ_ERR_NULL, tq.TQ_ERR_SHAPE, tq.TQ_ERR_ALIGN
    ok = _cache(tq)
    good = [C.byref(ok), F, F, tq.TQ_FP16, 256, 256, F, 5, None, None]
    for args, code in _vary(good, [(0, None, N), (1, None, N), (2, None, N), (6, None, N), (3, tq.TQ_FP32, S), (3, 7, S), (4, 255, S),
                                   (4, 248, S), (5, 260, S), (7, -1, S), (7, 1 << 31, S), (1, F + 8, A), (2, F + 2, A),
                                   (6, F + 4, A), (8, F + 2, A)]):
        assert tq._lib.tq_kv8_append(*args) == code, args
    for c, code in _caches(tq):
        assert tq._lib.tq_kv8_append(C.byref(c), *good[1:]) == code
    good = [C.byref(ok), F, 5, F, F, tq.TQ_FP32, None, None]
    for args, code in _vary(good, [(0, None, N), (1, None, N), (3, None, N), (4, None, N), (5, 3, S), (2, -1, S), (1, F + 4, A), (3, F + 8, A),
                                   (6, F + 1, A)]):
        assert tq._lib.tq_kv8_gather(*args) == code, args
    for c, code in _caches(tq):
        assert tq._lib.tq_kv8_gather(C.byref(c), *good[1:]) == code


def test_decode_refuses(tq):
    N, S, A = tq.TQ_ERR_NULL, tq.TQ_ERR_SHAPE, tq.TQ_ERR_ALIGN
    ok = _cache(tq)
    room = tq._lib.tq_int8_workspace_bytes(1, 2, 8, 128)
    good = [C.byref(ok), F, tq.TQ_FP16, 1024, 8, 1.0, 0, 0, F, room, F, tq.TQ_FP16, None, None]
    for args, code in _vary(good, [(0, None, N), (1, None, N), (8, None, N), (10, None, N), (2, tq.TQ_FP32, S), (11, tq.TQ_BF16, S),
                                   (11, 9, S), (3, 1016, S), (3, 1028, S), (4, 7, S), (4, 0, S), (4, 2 * 65, S), (6, -1, S), (7, -1, S),
                                   (9, room - 1, tq.TQ_ERR_WORKSPACE), (1, F + 8, A), (8, F + 8, A), (10, F + 4, A), (12, F + 2, A)]):
        assert tq._lib.tq_sdpa_int8_decode(*args) == code, args
    for c, code in _caches(tq):
        assert tq._lib.tq_sdpa_int8_decode(C.byref(c), *good[1:]) == code
    huge = _paged(tq, B=65535, H_kv=8, S_cap=1 << 20, page_tokens=1 << 16, max_pages=16, num_pages=9)
    assert tq._lib.tq_sdpa_int8_decode(C.byref(huge), *good[1:]) == S


def test_prompt_refuses(tq):
    N, S, A = tq.TQ_ERR_NULL, tq.TQ_ERR_SHAPE, tq.TQ_ERR_ALIGN
    #       q  k  v  dtype       strides          n_q n_kv offsets B  Hq Hk d    scale c  w  out dtype status stream
    good = [F, F, F, tq.TQ_BF16, 1024, 256, 256, 10, 10, F, F, 2, 8, 2, 128, 1.0, 1, 0, F, tq.TQ_FP32, None, None]
    for args, code in _vary(good, [(0, None, N), (1, None, N), (2, None, N), (9, None, N), (10, None, N), (18, None, N), (3, tq.TQ_FP32, S),
                                   (3, 5, S), (4, 1016, S), (4, 1025, S), (5, 250, S), (6, 128, S), (7, -1, S), (8, -1, S), (11, 0, S),
                                   (11, 65536, S), (12, 7, S), (12, 0, S), (13, 0, S), (14, 96, S), (17, -1, S), (19, tq.TQ_FP16, S),
                                   (0, F + 8, A), (1, F + 2, A), (2, F + 8, A), (9, F + 2, A), (18, F + 8, A), (20, F + 1, A)]):
        assert tq._lib.tq_sdpa_prompt(*args) == code, args
    windowed = list(good)
    windowed[16], windowed[17] = 0, 5                  # a window without the causal mask
    assert tq._lib.tq_sdpa_prompt(*windowed) == S
    many = list(good)
    many[4], many[12] = 2 * 65 * 128, 2 * 65           # 65 query heads on a KV head
    assert tq._lib.tq_sdpa_prompt(*many) == S


def test_pages_refuse(tq):
    N, S, A = tq.TQ_ERR_NULL, tq.TQ_ERR_SHAPE, tq.TQ_ERR_ALIGN
    #       table lens done B page cols pool free count lens_out count_out status stream
    good = [F, F, F, 4, 16, 8, 30, F, F, F, F, None, None]
    for args, code in _vary(good, [(1, None, N), (2, None, N), (7, None, N), (8, None, N), (9, None, N), (10, None, N), (3, 0, S), (3, 65536, S),
                                   (4, 24, S), (4, 8, S), (5, 0, S), (5, 1 << 28, S), (6, 0, S), (0, F + 2, A), (1, F + 1, A), (7, F + 2, A),
                                   (8, F + 2, A), (9, F + 2, A), (10, F + 2, A), (11, F + 2, A)]):
        assert tq._lib.tq_pages_release(*args) == code, args
    #       table lens new B page cols pool free count lens_out count_out offsets slots n ws bytes status stream
    room = tq._lib.tq_pages_workspace_bytes(4)
    good = [F, F, F, 4, 16, 8, 30, F, F, F, F, F, F, 9, F, room, None, None]
    for args, code in _vary(good, [(1, None, N), (2, None, N), (7, None, N), (8, None, N), (9, None, N), (10, None, N), (11, None, N), (12, None, N),
                                   (14, None, N), (13, -1, S), (13, 1 << 31, S), (4, 17, S), (15, room - 1, tq.TQ_ERR_WORKSPACE), (12, F + 4, A),
                                   (14, F + 8, A), (11, F + 2, A)]):
        assert tq._lib.tq_pages_assign(*args) == code, args
    contiguous = list(good)
    contiguous[0], contiguous[4] = None, 24            # a capacity that is no multiple of 16
    assert tq._lib.tq_pages_assign(*contiguous) == S


def test_a_step_without_tokens_is_no_error(tq):
    """A batch of which every sequence has just ended: no rows, so no addresses either."""
    c, bad = _cache(tq), _cache(tq, d=100)
    assert tq._lib.tq_kv8_append(C.byref(c), None, None, tq.TQ_FP16, 256, 256, None, 0, None, None) == tq.TQ_OK
    assert tq._lib.tq_kv8_gather(C.byref(c), None, 0, None, None, tq.TQ_FP32, None, None) == tq.TQ_OK
    assert tq._lib.tq_kv8_append(C.byref(bad), None, None, tq.TQ_FP16, 256, 256, None, 0, None, None) == tq.TQ_ERR_SHAPE
    prompt = [None, None, None, tq.TQ_BF16, 1024, 256, 256, 0, 0, F, F, 2, 8, 2, 128, 1.0, 1, 0, None, tq.TQ_FP32, None, None]
    assert tq._lib.tq_sdpa_prompt(*prompt) == tq.TQ_OK
    prompt[7] = 3                                      # queries, but no address of theirs
    assert tq._lib.tq_sdpa_prompt(*prompt) == tq.TQ_ERR_NULL


def test_a_cache_follows_its_tensors(tq):
    """Storage that was swapped under a tensor is found again; a tensor of another size is refused; the attributes cannot
    be set past the cache."""
    import torch
    cache = tq.KV8Cache(2, 2, 32, 64, device="cpu")
    cache.blocks.data = cache.blocks.clone()
    assert cache.struct().blocks == cache.blocks.data_ptr()
    with pytest.raises(AttributeError):
        cache.seq_lens = torch.zeros(2, dtype=torch.int32)
    cache.blocks.data = cache.blocks[:1].clone()
    with pytest.raises(tq.TqError) as e:
        cache.struct()
    assert e.value.code == tq.TQ_ERR_SHAPE and "resized" in str(e.value)


def test_the_binding_refuses_tensors_it_cannot_use(tq):
    """CPU tensors, wrong types and shapes raise before the library is called; an int8 cache is no int4 cache."""
    import torch
    z = lambda *s, t=torch.float16: torch.zeros(s, dtype=t)  # noqa: E731
    cache = tq.KV8Cache(1, 2, 32, 64, device="cpu")
    if not torch.cuda.is_available():
        calls = (lambda: tq.tq_kv8_append(cache, z(3, 2, 64), z(3, 2, 64), z(3, t=torch.int64)),
                 lambda: tq.tq_sdpa_prompt(z(3, 2, 64), z(3, 2, 64), z(3, 2, 64), z(2, t=torch.int32), z(2, t=torch.int32), 1.0, z(3, 2, 64)),
                 lambda: tq.tq_pages_release(None, z(3, t=torch.int32), z(3, t=torch.uint8), 16, 0, None, None, z(3, t=torch.int32), None))
        for call in calls:
            with pytest.raises(tq.TqError) as e:
                call()
            assert e.value.code == tq.TQ_ERR_SHAPE and "CUDA" in str(e.value)
    for bad in (lambda: tq.KV8Cache.over(z(1, 2, 2, 100, t=torch.uint8), z(1, t=torch.int32)),
                lambda: tq.KV8Cache.over(cache.blocks, z(2, t=torch.int32)),
                lambda: tq.KV8Cache.over(cache.blocks, z(1, t=torch.int64)),
                lambda: tq.KV8Cache(1, 1, 30, 64, device="cpu"),
                lambda: tq.PagedKV8Cache(1, 1, 24, 2, 2, 64, device="cpu"),
                lambda: tq.tq_kv8_gather(tq.KVCache(1, 2, 32, 64, device="cpu"), z(1, t=torch.int64), z(1, 2, 64), z(1, 2, 64))):
        with pytest.raises(tq.TqError):
            bad()
    with pytest.raises((C.ArgumentError, TypeError)):
        tq._lib.tq_sdpa_int4_decode(C.byref(cache.struct()), F, 8, 1.0, 1, F, F, F, None, None)
    paged = tq.PagedKV8Cache(3, 2, 32, 4, 9, 128, device="cpu")
    assert (paged.B, paged.H_kv, paged.S_cap, paged.d, paged.page_tokens, paged.max_pages, paged.num_pages) == (3, 2, 128, 128, 32, 4, 9)
    c = paged.struct()
    assert (c.blocks, c.seq_lens, c.page_table) == (paged.blocks.data_ptr(), paged.seq_lens.data_ptr(), paged.page_table.data_ptr())


def test_a_cache_refuses_tensors_of_another_type_or_shape(tq):
    """What stands in a tensor's place has to be of its type and shape, not of as many elements alone: an int64 or int16 table
    would be read as int32."""
    import torch
    for name, swap in (("seq_lens", lambda t: t.long()), ("seq_lens", lambda t: t.to(torch.int16)), ("page_table", lambda t: t.to(torch.uint8)),
                       ("page_table", lambda t: t.t().contiguous()), ("blocks", lambda t: t.to(torch.float32)),
                       ("blocks", lambda t: t.reshape(t.shape[1], t.shape[0], *t.shape[2:]))):
        cache = tq.PagedKV8Cache(3, 2, 32, 4, 9, 128, device="cpu")
        assert cache.struct().B == 3
        tensor = getattr(cache, name)
        tensor.data = swap(tensor)
        with pytest.raises(tq.TqError) as e:
            cache.struct()
        assert e.value.code == tq.TQ_ERR_SHAPE, name


def test_a_cache_struct_outlives_its_cache(tq):
    """The C struct is the caller's own: it stays as it is when the cache object is gone, and when it is used again."""
    import gc
    import torch
    blocks, lens = torch.zeros((3, 2, 2, tq.TQ_BLOCK8_BYTES(64)), dtype=torch.uint8), torch.zeros(3, dtype=torch.int32)
    c = tq.KV8Cache.over(blocks, lens).struct()
    gc.collect()
    others = [tq.KV8Cache.over(torch.zeros((1, 1, 1, tq.TQ_BLOCK8_BYTES(128)), dtype=torch.uint8), torch.zeros(1, dtype=torch.int32))
              for _ in range(50)]
    assert (c.blocks, c.seq_lens, c.B, c.H_kv, c.S_cap, c.d) == (blocks.data_ptr(), lens.data_ptr(), 3, 2, 32, 64)
    cache = tq.KV8Cache.over(blocks, lens)
    first = cache.struct()
    blocks.data = blocks.clone()
    assert cache.struct().blocks == blocks.data_ptr() != first.blocks
    del others


def _python(code):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    return subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)


@pytest.mark.parametrize("there", [False, True])
def test_without_its_binding_only_the_serving_operators_are_missing(tq, tmp_path, there):
    """The extension module is missing, or is none: the rest of tq imports and works, and the serving operators say why not."""
    path = tmp_path / "_tq_bind.other.so"
    if there:
        path.write_bytes(b"made for something else")
    p = _python(f"""
from paper_2604_16957_b200 import build
build.binding_path = lambda: {str(path)!r}
from paper_2604_16957_b200 import tq
assert "sm_100a" in tq.tq_version() and tq.KVCache(1, 2, 32, 64, device="cpu").struct().H_kv == 2
assert tq.tq_auto_splits(1, 8, 64, 128, 1000) > 0
import torch
z = torch.zeros(1, dtype=torch.int32)
for call in (lambda: tq.KV8Cache(1, 2, 32, 64, device="cpu"), lambda: tq.PagedKV8Cache(1, 2, 32, 2, 2, 64, device="cpu"),
             lambda: tq.tq_pages_release(None, z, z, 16, 0, None, None, z, None),
             lambda: tq.tq_sdpa_prompt(z, z, z, z, z, 1.0, z)):
    try:
        call()
    except ImportError as e:
        assert "_tq_bind.other.so" in str(e) and "build" in str(e), e
    else:
        raise AssertionError("no error")
print("fine")
""")
    assert p.returncode == 0 and p.stdout.strip() == "fine", p.stderr


def test_the_binding_is_named_after_what_it_was_built_for(monkeypatch):
    """Another torch, another Python: another file, which is then built and not taken over."""
    import sysconfig

    import torch
    from paper_2604_16957_b200 import build
    here = build.binding_path()
    assert here.endswith(sysconfig.get_config_var("EXT_SUFFIX"))
    monkeypatch.setattr(torch, "__version__", "9.9.0+other")
    assert build.binding_path() != here
    monkeypatch.undo()
    real = sysconfig.get_config_var
    monkeypatch.setattr(sysconfig, "get_config_var", lambda k: ".cpython-399.so" if k == "EXT_SUFFIX" else real(k))
    assert build.binding_path() != here
    monkeypatch.undo()
    commands = []
    monkeypatch.setattr(torch, "__version__", "9.9.0+other")
    monkeypatch.setattr(build.subprocess, "run", lambda cmd, **kw: (commands.append(cmd), open(cmd[cmd.index("-o") + 1], "w").close()))
    out = build.build_binding()
    try:
        assert len(commands) == 1 and out == build.binding_path() and out != here
    finally:
        build.os.remove(out)
