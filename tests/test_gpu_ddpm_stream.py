"""Eq. 1 on a stream that is not the current one."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_a_new_x_prev_has_memory_of_its_own():
    """Memory that the current stream has freed but may still write is not given to a result of another stream."""
    from paper_2606_15615_gb300 import moeca as M
    x, eps = torch.randn(4096, 64, device="cuda"), torch.randn(4096, 64, device="cuda")
    want = M.ddpm_step(x, eps, 0.99, 0.5, 0.0).clone()
    side = torch.cuda.Stream()
    torch.empty_like(want).fill_(5.0)  # loads the fill's kernel, which would wait for the stream
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    stale = torch.empty_like(want)
    stale.fill_(5.0)  # runs once the current stream is free again
    del stale
    got = M.ddpm_step(x, eps, 0.99, 0.5, 0.0, stream=side.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
