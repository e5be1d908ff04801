"""Bounded waits of the packed attention that run out: the status a caller sees, and the calls after it.

A barrier is set up for an arrival that never comes, so that a wait for it ends by its own limit: nothing hangs.
"""
import time

import pytest
import torch

pytestmark = pytest.mark.gpu

LIMIT = 20_000_000


@pytest.fixture(scope="module")
def M():
    from paper_2606_15615_gb300 import moeca
    return moeca


@pytest.fixture
def stall(M):
    yield lambda barrier: M.moeca_probe_attention_stall(barrier, LIMIT)
    M.moeca_probe_attention_stall(M.MOECA_ATTENTION_NONE)


@pytest.mark.parametrize("barrier", ["COPIES", "SCORES", "WEIGHTS", "SLOTS"])
@pytest.mark.parametrize("q_n,H,n", [(300, 2, 2000), (40, 2, 700), (600, 1, 600)])
def test_a_wait_that_runs_out_is_reported(M, stall, barrier, q_n, H, n):
    g = torch.Generator().manual_seed(q_n)
    q = torch.randn(q_n, H, 128, generator=g).bfloat16().cuda()
    k, v = (torch.randn(n, H, 128, generator=g).bfloat16().cuda() for _ in range(2))
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    want = M.attention(q, k, v, causal=True, status=status)
    torch.cuda.synchronize()
    assert status.tolist() == [0, 0]
    stall(getattr(M, "MOECA_ATTENTION_" + barrier))
    t0 = time.monotonic()
    M.attention(q, k, v, causal=True, status=status)
    torch.cuda.synchronize()
    # A wait, a drain of one second for each of the copies that never report, and what launches take.
    assert 1e-9 * LIMIT <= time.monotonic() - t0 < 10
    assert status[0].item() == M.MOECA_ERR_TIMEOUT and 710 <= status[1].item() <= 713
    M.attention(q, k, v, causal=True)  # without a status word
    torch.cuda.synchronize()
    stall(M.MOECA_ATTENTION_NONE)
    status.zero_()
    assert torch.equal(M.attention(q, k, v, causal=True, status=status), want) and status.tolist() == [0, 0]


@pytest.mark.parametrize("bad", [(-1, LIMIT), (5, LIMIT), (1, 999_999), (1, 1_000_000_001)])
def test_stall_refusals(M, bad):
    with pytest.raises(M.MoecaError):
        M.moeca_probe_attention_stall(*bad)
