"""Latent attention where few calls go: caches of the other type with many heads, a first call that is captured, operands that are missing
for one particular tile."""
import subprocess
import sys

import pytest

from test_gpu_latent import _check_decode, _dev, _filled, _queries
from test_gpu_latent_use import _hooked

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2604_16957_b200 import tq
    assert torch.cuda.is_available()
    return tq, torch


@pytest.mark.parametrize("H", [20, 64, 90])
@pytest.mark.parametrize("kind,other", [("fp16", "bf16"), ("bf16", "fp16")])
def test_a_cache_of_the_other_type_with_many_heads(gpu, H, kind, other):
    tq, torch = gpu
    cache, values = _filled(tq, torch, [700, 20, 0, 65], 256, 16, other, 5)
    q_c, q_r = _queries(torch, 4, H, 256, kind, "heads")
    out = torch.empty((4, H, 256), device="cuda")
    tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.05, 0, 0, tq.alloc_latent_workspace(4, H, 256), out)
    _check_decode(torch, out, q_c, q_r, values, 0.05, 0)


FIRST = """
import torch
from paper_2604_16957_b200 import tq
B, H, d_c, n = 2, {H}, 512, 700
x = torch.randn((B * n, d_c + 64), device="cuda").half()
cache = tq.LatentCache(B, 704, d_c)
slots = (torch.arange(B * n, device="cuda") // n * 704 + torch.arange(B * n, device="cuda") % n)
cache.seq_lens.fill_(n)
q = torch.randn((B, H, d_c + 64), device="cuda").half()
work, out = tq.alloc_latent_workspace(B, H, d_c), [torch.zeros((B, H, d_c), device="cuda") for _ in range(2)]
back = [torch.zeros((B * n, d), device="cuda") for d in (d_c, 64)]
k = torch.randn((50, 4, 128), device="cuda").half()
at, prompt = torch.tensor([0, 50], dtype=torch.int32, device="cuda"), [torch.zeros((50, 4, 128), device="cuda") for _ in range(2)]
def step(i):
    tq.tq_latent_append(cache, x[:, :d_c], x[:, d_c:], slots)
    tq.tq_sdpa_latent_decode(cache, q[..., :d_c], q[..., d_c:], 0.05, 0, 0, work, out[i])
    tq.tq_latent_gather(cache, slots, *back)
    tq.tq_sdpa_latent_prompt(k, k[..., :64], k, k[:, 0, :64], k, at, at, 0.07, prompt[i])
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    step(0)
g.replay()
step(1)
torch.cuda.synchronize()
assert torch.equal(*out) and torch.equal(*prompt) and all(t.abs().sum() > 0 for t in (*out, *prompt, *back))
print("same")
"""


@pytest.mark.parametrize("H", [16, 128])
def test_the_first_call_of_a_process_is_captured(gpu, H):
    r = subprocess.run([sys.executable, "-c", FIRST.format(H=H)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stderr[-2000:]


# lengths, heads; whether some thread block has a third tile, by the shares of the line
THIRD = [([1000], 16, False), ([9000, 3000, 50], 64, False), ([20000, 700], 20, True), ([100, 30] * 200, 16, True), ([20, 2500, 300] * 15, 128, True)]


@pytest.mark.parametrize("lens,H,reached", THIRD)
def test_a_third_tile_without_operands(gpu, lens, H, reached):
    """A call that reaches such a tile says so; one that does not is right."""
    tq, torch = gpu
    B, d_c = len(lens), 512
    # (a thread block's share of the tiles and the 3 places in front of each sequence, over 148 of them for each 64 heads)
    lines = torch.cuda.get_device_properties(0).multi_processor_count // -(-H // 64)
    assert (-(-sum(-(-n // 64) + 3 for n in lens) // lines) > 2) == reached
    cache, values = _filled(tq, torch, lens, d_c, 16, "fp16", 3)
    q_c, q_r = _queries(torch, B, H, d_c, "bf16")
    work, status, out = tq.alloc_latent_workspace(B, H, d_c), _dev(torch, [0]), torch.empty((B, H, d_c), device="cuda")
    _hooked(tq, torch, lambda: tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.05, 0, 0, work, out, status), 1000000, 2)
    assert int(status.item()) == (tq.TQ_STATUS_TIMEOUT if reached else 0)
    if reached:
        tq.tq_sdpa_latent_decode(cache, q_c, q_r, 0.05, 0, 0, work, out)
    _check_decode(torch, out, q_c, q_r, values, 0.05, 0, rows=range(min(B, 6)))


def test_tensors_without_rows_have_no_strides(gpu):
    """What has no elements may come with any strides (those of an empty numpy array are all zero)."""
    tq, torch = gpu
    none = lambda *s: torch.zeros((0, *s), dtype=torch.float16, device="cuda").as_strided((0, *s), (0,) * (1 + len(s)))  # noqa: E731
    out, at = torch.full((5, 3, 128), 7.0, dtype=torch.float16, device="cuda"), [_dev(torch, [0, n]) for n in (0, 5)]
    q = torch.randn((5, 3, 192), device="cuda").half()
    tq.tq_sdpa_latent_prompt(q[..., :128], q[..., 128:], none(3, 128), none(64), none(3, 128), at[1], at[0], 0.1, out)
    assert torch.all(out == 0)
    tq.tq_sdpa_latent_prompt(none(3, 128), none(3, 64), q[..., :128], q[:, 0, :64], q[..., :128], at[0], at[1], 0.1, out[:0])
    out.fill_(7.0)
    tq.tq_sdpa_prompt(q[..., :128].contiguous(), none(3, 128), none(3, 128), at[1], at[0], 0.1, out)
    assert torch.all(out == 0)
    slots = torch.zeros((0,), dtype=torch.int64, device="cuda")
    tq.tq_latent_append(tq.LatentCache(1, 16, 128), none(128), none(64), slots)
    tq.tq_kv8_append(tq.KV8Cache(1, 2, 16, 64), none(2, 64), none(2, 64), slots)
    torch.cuda.synchronize()
