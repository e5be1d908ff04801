"""The forms of the packed attention's kernels: what a row's result may depend on, and which form takes which sizes."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    from paper_2606_15615_gb300 import moeca
    return moeca


def offsets(lengths):
    return torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device="cuda")


def qkv(seed, Tq, Tk, H, Hk, d, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(n, h, d, generator=g).to(dtype).cuda() for n, h in ((Tq, H), (Tk, Hk), (Tk, Hk))]


# The last rows of a sequence share their warps with rows of the next one's queries.
@pytest.mark.parametrize("q_len,k_len,H,Hk", [([120, 40], [1000, 300], 2, 2), ([38, 30], [1500, 300], 3, 1),
                                              ([250, 100] * 12, [900, 300] * 12, 8, 8)], ids=["tile", "group", "pairs"])
@pytest.mark.parametrize("d", [64, 72, 128])
def test_rows_do_not_depend_on_other_sequences(M, q_len, k_len, H, Hk, d):
    q, k, v = qkv(d, sum(q_len), sum(k_len), H, Hk, d)
    first = torch.cat([torch.full((n,), i % 2 == 0) for i, n in enumerate(q_len)]).cuda()
    args = dict(q_offsets=offsets(q_len), k_offsets=offsets(k_len), causal=False)
    want = M.attention(q, k, v, **args)[first]
    for factor in (0.0, 30.0, 1e6, float("inf"), float("nan")):
        other = torch.where(first[:, None, None], q, q * factor)
        assert torch.equal(M.attention(other, k, v, **args)[first], want)


@pytest.mark.parametrize("H", [3, 5, 48])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_do_not_depend_on_what_shared_memory_held(M, H, d):
    """128 is no multiple of the group: a tile's last rows are of no query."""
    q, k, v = qkv(H, 400, 1300, H, 1, d)
    fill = qkv(1, 128 * 320, 128 * 320, 1, 1, d)
    res = []
    for value in (0.0, 1e30, -3e3, float("nan")):
        M.attention(fill[0], fill[1], torch.full_like(fill[2], value), n_seqs=320)  # results leave through shared memory
        res.append(M.attention(q, k, v))
    assert all(torch.equal(r, res[0]) for r in res) and bool(res[0].isfinite().all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("most", [3, 40, 300])
def test_offsets_written_right_before_the_call(M, dtype, most):
    """Offsets that a kernel of the same graph writes before the call, others in every replay; the key axis is cut."""
    n, keys, B = 3 * most, 20_000, 3
    q, k, v = qkv(most, n, keys, 4, 2, 64, dtype)
    rng = np.random.default_rng(most)

    def cuts(total, longest):
        while True:
            c = np.concatenate([[0], np.sort(rng.integers(0, total + 1, B - 1)), [total]])
            if np.diff(c).max() <= longest:
                return torch.tensor(c, dtype=torch.int32, device="cuda")

    source = [torch.zeros(B + 1, dtype=torch.int32, device="cuda") for _ in range(2)]
    off = [torch.zeros_like(s) for s in source]

    def step():
        for a, b in zip(off, source):
            torch.add(b, 0, out=a)
        return M.attention(q, k, v, q_offsets=off[0], k_offsets=off[1], causal=True, max_q=most, lse=True)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = step()
    for _ in range(6):
        new = [cuts(n, most), cuts(keys, keys)]
        for s, c in zip(source, new):
            s.copy_(c)
        graph.replay()
        want = M.attention(q, k, v, q_offsets=new[0], k_offsets=new[1], causal=True, max_q=most, lse=True)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
