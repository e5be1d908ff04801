"""Bounded waits that run out in both forms of the packed attention's tile kernel, at keys that end inside a fragment
(whose foreign values a warp clears while others may give up), and the calls after them.

A barrier is set up for an arrival that never comes, so that a wait for it ends by its own limit: nothing hangs.
"""
import time

import pytest
import torch

from test_gpu_packed_attention_forms import form, offsets, qkv

pytestmark = pytest.mark.gpu

LIMIT = 5_000_000


@pytest.fixture(scope="module")
def M():
    from paper_2606_15615_gb300 import moeca
    return moeca


@pytest.fixture
def stall(M):
    yield lambda barrier: M.moeca_probe_attention_stall(barrier, LIMIT)
    M.moeca_probe_attention_stall(M.MOECA_ATTENTION_NONE)


@pytest.mark.parametrize("barrier", ["COPIES", "SCORES", "WEIGHTS", "SLOTS"])
@pytest.mark.parametrize("q_len,k_len,H,d,name,cut", [
    ([40, 100], [137, 900], 2, 64, "TILE", False), ([64], [9001], 2, 72, "TILE", True), ([150, 129], [4103, 4999], 77, 64, "TILES", False),
    ([200, 131] * 9, [197, 1003] * 9, 9, 128, "TILES", False), ([300], [9001], 2, 96, "TILES", True)], ids=range(5))
def test_a_wait_that_runs_out_is_reported(M, stall, barrier, q_len, k_len, H, d, name, cut):
    q, k, v = qkv(d, sum(q_len), sum(k_len), H, H, d)
    got, chunk = form(M, q, k, v, q_len, k_len, max(q_len))
    assert got == getattr(M, "MOECA_ATTENTION_FORM_" + name) and (chunk > 0) == cut
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    args = dict(q_offsets=offsets(q_len), k_offsets=offsets(k_len), max_q=max(q_len), status=status)
    want = M.attention(q, k, v, **args)
    torch.cuda.synchronize()
    assert status.tolist() == [0, 0]
    stall(getattr(M, "MOECA_ATTENTION_" + barrier))
    t0 = time.monotonic()
    M.attention(q, k, v, **args)
    torch.cuda.synchronize()
    # A wait, and a drain of one second for each of the copies that never report, in each round of blocks.
    assert 1e-9 * LIMIT <= time.monotonic() - t0 < 20
    assert status[0].item() == M.MOECA_ERR_TIMEOUT and 710 <= status[1].item() <= 713
    stall(M.MOECA_ATTENTION_NONE)
    status.zero_()
    assert torch.equal(M.attention(q, k, v, **args), want) and status.tolist() == [0, 0]
