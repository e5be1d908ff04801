"""The forms of the packed attention's kernels: what a row's result may depend on, and which form takes which sizes."""
import numpy as np
import pytest
import torch

from test_gpu_packed_attention import check as against_64_bits

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
    n, keys, B = 2 * most, 20_000, 3
    q, k, v = qkv(most, n, keys, 4, 2, 64, dtype)
    rng = np.random.default_rng(most)

    def cuts(total, longest):  # lengths of at most `longest` each
        a = int(rng.integers(max(total - 2 * longest, 0), min(total, longest) + 1))
        b = int(rng.integers(max(total - longest, a), min(total, a + longest) + 1))
        return torch.tensor([0, a, b, total], dtype=torch.int32, device="cuda")

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


def form(M, q, k, v, q_len, k_len, max_q=0):
    """The form of a call with offsets."""
    def heads(t):
        return M.moeca_heads(t.data_ptr(), t.stride(0), t.stride(1), t.shape[1])
    out = torch.empty_like(q)
    off = offsets(q_len)
    return M.moeca_probe_attention_form(M.moeca_attention_args(
        heads(q), heads(k), heads(v), heads(out), off.data_ptr(), off.data_ptr(), None, None, None, q.shape[0], k.shape[0], len(q_len),
        max_q, M.MOECA_BF16, q.shape[2], 1, 0, 0.1))


# Shapes of two tiles a block: whole and cut keys, one and more sequences, tails of every kind, blocks whose second
# tile has no queries or fewer keys.
PAIRS = [
    ([129 + 11 * i % 72 for i in range(20)], [129 + 11 * i % 72 for i in range(20)], 8, 8, False),
    ([200 - 3 * i for i in range(20)], [150 + 17 * i for i in range(20)], 16, 8, False),
    ([385, 130, 0, 260] * 3, [385, 130, 9, 260] * 3, 11, 11, False),
    ([300, 17, 260, 1], [4100, 4500, 4097, 5003], 2, 2, True),
    ([300], [9001], 2, 2, True),
    ([150, 290], [9000, 5007], 4, 2, True),
]


@pytest.mark.parametrize("q_len,k_len,H,Hk,cut", PAIRS, ids=range(len(PAIRS)))
@pytest.mark.parametrize("causal,d", [(False, 40), (False, 72), (False, 128), (True, 64), (True, 96), (True, 128)])
def test_two_tiles_a_block(M, q_len, k_len, H, Hk, cut, causal, d):
    q, k, v = qkv(d, sum(q_len), sum(k_len), H, Hk, d)
    got, chunk = form(M, q, k, v, q_len, k_len, max(q_len))
    assert got == M.MOECA_ATTENTION_FORM_TILES and (chunk > 0) == cut
    against_64_bits(M, q, k, v, q_len, k_len, causal, max_q=max(q_len))


@pytest.mark.parametrize("causal,d", [(False, 72), (True, 64)])
def test_two_tiles_a_block_over_long_keys(M, causal, d):
    """Whole key axes above 4096 keys, tiles of 1 to 256 queries."""
    q_len, k_len = [150, 17, 260, 1], [4100, 4500, 4097, 5003]
    q, k, v = qkv(d, sum(q_len), sum(k_len), 16, 16, d)
    assert form(M, q, k, v, q_len, k_len, max(q_len)) == (M.MOECA_ATTENTION_FORM_TILES, 0)
    against_64_bits(M, q, k, v, q_len, k_len, causal, max_q=max(q_len))


@pytest.mark.parametrize("causal,d", [(False, 64), (False, 96), (True, 72), (True, 128)])
def test_two_tiles_a_block_of_equal_lengths(M, causal, d):
    q, k, v = qkv(d, 21 * 150, 21 * 170, 8, 8, d)
    assert form(M, q, k, v, [150] * 21, [170] * 21, 150) == (M.MOECA_ATTENTION_FORM_TILES, 0)
    against_64_bits(M, q, k, v, [150] * 21, [170] * 21, causal, given=False, n_seqs=21)
    own = q.clone()
    want = M.attention(q, k, v, n_seqs=21, causal=causal)
    assert M.attention(own, k, v, n_seqs=21, causal=causal, out=own) is own and torch.equal(own, want)


@pytest.mark.parametrize("d", [64, 72, 128])
def test_two_tiles_a_block_with_foreign_values(M, d):
    """Rising maxima, and NaN and infinities in every other sequence."""
    n = 20
    q_len, k_len = [140 + i for i in range(n)], [200 + 7 * i for i in range(n)]
    q, k, v = qkv(d, sum(q_len), sum(k_len), 8, 8, d)
    assert form(M, q, k, v, q_len, k_len, max(q_len))[0] == M.MOECA_ATTENTION_FORM_TILES
    at = torch.cat([torch.linspace(0.1, 20, m) for m in k_len]).cuda()
    k *= at[:, None, None].to(k.dtype)
    against_64_bits(M, q, k, v, q_len, k_len, True, max_q=max(q_len))
    args = dict(q_offsets=offsets(q_len), k_offsets=offsets(k_len), max_q=max(q_len))
    want = M.attention(q, k, v, **args)
    bad_q, bad_k = (torch.cat([torch.full((m,), i % 2 == 1) for i, m in enumerate(x)]).cuda() for x in (q_len, k_len))
    k[bad_k], v[bad_k] = float("inf"), float("nan")
    out = M.attention(q, k, v, **args)
    assert torch.equal(out[~bad_q], want[~bad_q]) and bool(out[bad_q].isnan().all())


# Sequences of very different lengths, of which only those far above the mean are cut: the long ones first, last, among
# others, two of them; sequences without keys or queries.
UNEVEN = [[12000] + [100] * 38 + [4200], [9, 0] * 15 + [18000] + [150, 40, 0] * 3, [0] * 39 + [20000], [2100, 0, 4100, 6200, 1] * 2 + [13] * 30]


@pytest.mark.parametrize("k_len", UNEVEN, ids=range(len(UNEVEN)))
@pytest.mark.parametrize("first", [(0, 0), (3, 2500)])
@pytest.mark.parametrize("d,H,Hk,causal", [(64, 2, 2, True), (72, 6, 2, False), (128, 2, 1, True)])
def test_uneven_lengths(M, k_len, first, d, H, Hk, causal):
    q_len = [20, 0, 7, 33] * 10
    q, k, v = qkv(d, sum(q_len) + first[0] + 5, sum(k_len) + first[1] + 40, H, Hk, d)
    got, chunk = form(M, q, k, v, q_len, k_len, max(q_len))
    assert got == M.MOECA_ATTENTION_FORM_TILE and max(k_len) > chunk > 1536
    q[:first[0]], k[:first[1]], v[:first[1]] = float("nan"), float("inf"), float("nan")
    against_64_bits(M, q, k, v, q_len, k_len, causal, first=first, max_q=max(q_len))
    args = dict(q_offsets=offsets(q_len) + first[0], k_offsets=offsets(k_len) + first[1], causal=causal, max_q=max(q_len))
    again = M.attention(q, k, v, **args, lse=True)
    assert all(torch.equal(x, y) for x, y in zip(again, M.attention(q, k, v, **args, lse=True)))


@pytest.mark.parametrize("bad", [[-5, 12000, 100, 20000], [0, 25000, 3, 9000], [15000, 0, 0, 15000], [-2 ** 31, 2 ** 31 - 1, 0, 5],
                                 [19999, 20000, 19000, 20001]])
def test_wrong_offsets_of_uneven_lengths_stay_inside(M, bad):
    """Offsets out of range or order: clamped, and nothing outside the tensors is touched."""
    n = 40
    q, k, v = qkv(3, 20 * n, 20_000, 2, 2, 64)
    rng = np.random.default_rng(1)
    off = torch.tensor(np.concatenate([bad, rng.integers(-100, 20_100, n + 1 - len(bad))]), dtype=torch.int32, device="cuda")
    buf = torch.full((20 * n + 20, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(20 * n, 2, device="cuda")
    for q_off in (offsets([20] * n), off):
        M.attention(q, k, v, q_offsets=q_off, k_offsets=off, max_q=20, out=buf[10:-10], lse=lse)
        M.attention(q, k, v, q_offsets=q_off, k_offsets=off, max_q=20, lse=True)
    torch.cuda.synchronize()
    assert bool((buf[:10] == 5).all()) and bool((buf[-10:] == 5).all()) and not bool(buf.isnan().any())


@pytest.mark.parametrize("d", [64, 72, 33])
def test_parts_of_a_buffer_with_heads_first(M, d):
    """[heads, tokens, 3, d]: the norm in place of queries and keys, attention in place of the queries."""
    H, T = 3, 150
    g = torch.Generator().manual_seed(d)
    buf = torch.randn(H, T, 3, d, generator=g).bfloat16().cuda()
    q, k, v = (buf[:, :, i].permute(1, 0, 2) for i in range(3))
    nq, nk = M.qk_norm_rope(q.contiguous(), k.contiguous())
    want, values = M.attention(nq, nk, v.contiguous()), v.clone()
    M.qk_norm_rope(q, k, q_out=q, k_out=k)
    assert torch.equal(q, nq) and torch.equal(k, nk)
    M.attention(q, k, v, out=q)
    assert torch.equal(q, want) and torch.equal(k, nk) and torch.equal(v, values)


@pytest.mark.parametrize("d", [8, 16, 24, 48, 56, 88, 104, 112, 120])
@pytest.mark.parametrize("causal", [False, True])
def test_head_sizes_between_the_kernels_steps(M, d, causal):
    for q_len, k_len, H, Hk, name in (([1, 3], [300, 77], 4, 2, "ROWS"), ([40, 90], [133, 500], 2, 2, "TILE"),
                                      ([129 + i for i in range(20)], [129 + 9 * i for i in range(20)], 8, 8, "TILES")):
        q, k, v = qkv(d, sum(q_len), sum(k_len), H, Hk, d)
        assert form(M, q, k, v, q_len, k_len, max(q_len))[0] == getattr(M, "MOECA_ATTENTION_FORM_" + name)
        against_64_bits(M, q, k, v, q_len, k_len, causal, max_q=max(q_len))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_as_many_sequences_as_there_may_be(M, dtype):
    """A million sequences of one token and one key: the result is the value."""
    n = 1 << 20
    q, k, v = qkv(1, n, n, 1, 1, 8, dtype)
    off = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    for args in (dict(n_seqs=n), dict(q_offsets=off, k_offsets=off), dict(q_offsets=off, k_offsets=off, max_q=1)):
        assert torch.equal(M.attention(q, k, v, causal=True, **args), v)
    two = torch.arange(0, n + 1, 2, dtype=torch.int32, device="cuda")  # two queries and keys each: the first sees one key
    assert torch.equal(M.attention(q, k, v, q_offsets=two, k_offsets=two, causal=True)[::2], v[::2])
    with pytest.raises(M.MoecaError):
        M.attention(q, k, v, n_seqs=n + 1)
