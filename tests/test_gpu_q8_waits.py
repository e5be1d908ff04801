"""Bounded waits of the 8-bit calls that run out: a barrier waits for an arrival that nothing makes, the kernel gives
up after the set limit, says so in the status word and leaves the GPU in order.  No GPU fault is made."""
import time

import pytest
import torch

from test_gpu_q8 import M, filled, ints  # noqa: F401  (M: a fixture)

pytestmark = pytest.mark.gpu

LIMIT = 20_000_000  # ns


@pytest.fixture
def stall(M):
    yield lambda barrier: M.moeca_probe_q8_stall(barrier, LIMIT)
    M.moeca_probe_q8_stall(M.MOECA_Q8_NONE, LIMIT)


def status_words():
    return torch.zeros(2, dtype=torch.int32, device="cuda")


def test_stall_arguments(M):
    for barrier, ns in ((-1, LIMIT), (5, LIMIT), (1, 0), (1, 1_000_000_001)):
        with pytest.raises(M.MoecaError):
            M.moeca_probe_q8_stall(barrier, ns)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float8_e4m3fn])
@pytest.mark.parametrize("rows", [3, 9000])  # one tile, several a pair: the pair's MMAs run when the wait begins
@pytest.mark.parametrize("barrier", ["MOECA_Q8_OPERANDS", "MOECA_Q8_SCALES", "MOECA_Q8_ACCUMULATORS"])
def test_matmul_wait_runs_out(M, stall, barrier, rows, dtype):
    a, _ = filled(M, 1, rows, 1500, "e4m3")
    b, _ = filled(M, 2, 2 * 700, 1500, "e4m3")
    off = ints([0, rows // 3, rows])
    call = lambda status: M.q8_matmul(a, b, off, dtype=dtype, status=status)  # noqa: E731
    bits = lambda r: r.q.view(torch.uint8) if isinstance(r, M.Q8) else r  # noqa: E731
    status = status_words()
    want = bits(call(status)).clone()
    assert status.tolist() == [0, 0]
    stall(getattr(M, barrier))
    t0 = time.monotonic()
    call(status)
    torch.cuda.synchronize()
    assert time.monotonic() - t0 < 20
    assert status[0].item() == M.MOECA_ERR_TIMEOUT and 700 <= status[1].item() < 710
    call(None)  # nobody asked: the call still ends
    torch.cuda.synchronize()
    stall(M.MOECA_Q8_NONE)
    status.zero_()
    for _ in range(3):  # all SMs' TMEM and barriers are in order again
        assert torch.equal(bits(call(status)), want)
    assert status.tolist() == [0, 0]


@pytest.mark.parametrize("call", ["read", "combine", "combine unaligned"])
def test_staged_copies_run_out(M, stall, call):
    """Every warp gives up on its first token, and waits as long again for the copies that are under way."""
    width = 1001 if "unaligned" in call else 1152
    c, _ = filled(M, 3, 3000, width, "e4m3")
    rows = torch.arange(3000, dtype=torch.int32, device="cuda")[:, None].repeat(1, 4)
    x = torch.randn(3000, width, device="cuda")
    if call == "read":
        run = lambda status: M.q8_read(c, dtype=torch.float32, status=status)  # noqa: E731
    else:
        run = lambda status: M.q8_combine(c, rows, x=x, status=status)  # noqa: E731
    status = status_words()
    want = run(status).clone()
    assert status.tolist() == [0, 0]
    stall(M.MOECA_Q8_COPIES)
    torch.cuda.synchronize()
    t0 = time.monotonic()
    run(status)
    torch.cuda.synchronize()
    assert 2e-9 * LIMIT <= time.monotonic() - t0 < 10
    assert status.tolist() == [M.MOECA_ERR_TIMEOUT, 710]
    run(None)
    torch.cuda.synchronize()
    stall(M.MOECA_Q8_NONE)
    status.zero_()
    assert torch.equal(run(status), want) and status.tolist() == [0, 0]


def test_a_snapshot_that_was_not_read_back_is_not_loaded(M, stall):
    """Stack.set_state from 8-bit rows raises when their copies do not arrive, and leaves the stack as it was."""
    from paper_2606_15615_gb300 import workloads as W
    T, D, E, k, F = 512, 128, 8, 2, 256
    w = W.tiny_layer(43, T, D, E, k, F, dtype="bf16", wscale=0.05)[0]
    cfg = M.moeca_config_default(n_layers=1, hidden=D, ffn=F, n_experts=E, top_k=k, max_tokens=T, tau0=0.75)
    s = M.Stack(cfg, [w])
    x = torch.randn(T, D, device="cuda").bfloat16()
    s.step(x, 1)
    small = s.get_state(0, q8=torch.float8_e4m3fn)
    s.step(2 * x, 1)
    before = s.get_state(0)
    stall(M.MOECA_Q8_COPIES)
    with pytest.raises(M.MoecaError) as e:
        s.set_state(0, small)
    assert e.value.status == M.MOECA_ERR_TIMEOUT
    stall(M.MOECA_Q8_NONE)
    after = s.get_state(0)
    assert all(torch.equal(before[n], after[n]) for n in ("cache_h", "cache_e", "cache_w", "cache_norm", "ema"))
    s.set_state(0, small)
    assert torch.equal(s.get_state(0)["cache_h"].view(T * k, D), M.q8_read(small["cache_h"]))
    s.close()
