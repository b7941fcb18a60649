"""The bounded waits of the serving operators' kernels: when a copy does not arrive in time, the call sets
TQ_STATUS_TIMEOUT and returns, and the next one is right.  As in test_gpu_timeout.py the instrumented instantiations make one
chosen copy's barrier expect 16 bytes that never arrive (the data itself lands), or shorten the limit.  Nothing here faults,
traps or waits without a bound."""
import numpy as np
import pytest

from test_gpu_serving import _check_decode, _check_prompt, _filled, _packed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2604_16957_b200 import tq
    assert torch.cuda.is_available()
    return tq, torch


def _hooked(tq, torch, call, limit, fault):
    tq._test_hook(tq.HOOK_SPIN_LIMIT, limit)
    tq._test_hook(tq.HOOK_FAULT_BLOCK, fault)
    try:
        call()
        torch.cuda.synchronize()   # returns
    finally:
        tq._test_hook(tq.HOOK_SPIN_LIMIT, 0)
        tq._test_hook(tq.HOOK_FAULT_BLOCK, -1)


# one unit in a thread block; cut units; whole units by warp; more units than thread blocks on one line
DECODES = [([1000], 16, 2), ([20000, 700], 16, 2), ([100, 30] * 20, 64, 8), ([20, 2500, 300] * 15, 8, 8)]


@pytest.mark.parametrize("lens,H_q,H_kv", DECODES)
@pytest.mark.parametrize("fault", [0, 5])
def test_decode_gives_up_on_a_copy(gpu, lens, H_q, H_kv, fault):
    tq, torch = gpu
    B, d = len(lens), 128
    cache, values = _filled(tq, torch, lens, H_kv, d, 16, "fp16", 3)
    q = torch.randn((B, H_q, d), device="cuda").half()
    work, status = tq.alloc_int8_workspace(B, H_kv, H_q, d), torch.zeros(1, dtype=torch.int32, device="cuda")
    guard = torch.full((B * H_q * d + 128,), 5.0, device="cuda")
    out = guard[64:-64].view(B, H_q, d)
    _hooked(tq, torch, lambda: tq.tq_sdpa_int8_decode(cache, q, 0.09, 0, 0, work, out, status), 100000, fault)
    assert int(status.item()) == tq.TQ_STATUS_TIMEOUT
    assert torch.all(guard[:64] == 5.0) and torch.all(guard[-64:] == 5.0)
    work[:int(tq._lib.tq_int8_counter_bytes(B, H_kv, H_q))].zero_()   # as tq.h asks after a timeout
    status.zero_()
    tq.tq_sdpa_int8_decode(cache, q, 0.09, 0, 0, work, out, status)
    assert int(status.item()) == 0
    _check_decode(torch, out, q, values, 0.09, 0, d)


@pytest.mark.parametrize("lens,H_q,H_kv", DECODES)
@pytest.mark.parametrize("limit", [1, 2000])
def test_decode_with_short_waits(gpu, lens, H_q, H_kv, limit):
    """Whether a wait is caught depends on timing: the call returns either way, and a clean status means a right result."""
    tq, torch = gpu
    B, d = len(lens), 128
    cache, values = _filled(tq, torch, lens, H_kv, d, 16, "fp16", 4)
    q = torch.randn((B, H_q, d), device="cuda").half()
    work, status = tq.alloc_int8_workspace(B, H_kv, H_q, d), torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.empty((B, H_q, d), device="cuda")
    _hooked(tq, torch, lambda: tq.tq_sdpa_int8_decode(cache, q, 0.09, 0, 0, work, out, status), limit, -1)
    assert int(status.item()) in (0, tq.TQ_STATUS_TIMEOUT)
    if int(status.item()):
        work.zero_()
        tq.tq_sdpa_int8_decode(cache, q, 0.09, 0, 0, work, out)
    _check_decode(torch, out, q, values, 0.09, 0, d)


# one tile per thread block, and two; thread blocks that take over several pieces of work; a window
PROMPTS = [([300], 8, 1, 0), ([700, 40], 64, 8, 0), ([400, 1, 900, 33], 32, 8, 100), ([130] * 30, 16, 8, 0)]


def _prompt(tq, torch, lq, H_q, H):
    d = 128
    q, k, v = _packed(torch, np.random.default_rng(len(lq)), lq, lq, H_q, H, d, "fp16", True)
    cum = np.concatenate([[0], np.cumsum(lq)]).tolist()
    guard = torch.full(((len(q) + 2) * H_q * d,), 5.0, device="cuda")
    return q, k, v, cum, torch.tensor(cum, dtype=torch.int32, device="cuda"), guard, guard.view(-1, H_q, d)[1:-1]


@pytest.mark.parametrize("lq,H_q,H,window", PROMPTS)
@pytest.mark.parametrize("fault", [0, 1, 2])
def test_prompt_gives_up_on_a_tile(gpu, lq, H_q, H, window, fault):
    tq, torch = gpu
    q, k, v, cum, at, guard, out = _prompt(tq, torch, lq, H_q, H)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    _hooked(tq, torch, lambda: tq.tq_sdpa_prompt(q, k, v, at, at, 0.09, out, window=window, status=status), 100000, fault)
    assert int(status.item()) == tq.TQ_STATUS_TIMEOUT
    assert torch.all(guard.view(-1, H_q, 128)[0] == 5.0) and torch.all(guard.view(-1, H_q, 128)[-1] == 5.0)
    status.zero_()
    tq.tq_sdpa_prompt(q, k, v, at, at, 0.09, out, window=window, status=status)
    assert int(status.item()) == 0
    _check_prompt(torch, out, q, k, v, cum, cum, 0.09, True, window)


@pytest.mark.parametrize("lq,H_q,H,window", PROMPTS)
@pytest.mark.parametrize("limit", [1, 2000])
def test_prompt_with_short_waits(gpu, lq, H_q, H, window, limit):
    tq, torch = gpu
    q, k, v, cum, at, guard, out = _prompt(tq, torch, lq, H_q, H)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    _hooked(tq, torch, lambda: tq.tq_sdpa_prompt(q, k, v, at, at, 0.09, out, window=window, status=status), limit, -1)
    assert int(status.item()) in (0, tq.TQ_STATUS_TIMEOUT)
    if int(status.item()):
        tq.tq_sdpa_prompt(q, k, v, at, at, 0.09, out, window=window)
    _check_prompt(torch, out, q, k, v, cum, cum, 0.09, True, window)
