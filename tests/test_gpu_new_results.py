"""Results that a call allocates are whole: what it does not compute is 0 (or -inf), whatever the memory held; given
tensors keep it.  The allocator hands out memory that held NaN before."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def M():
    from paper_2606_15615_gb300 import moeca
    return moeca


def offsets(lengths, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(lengths)]), dtype=torch.int32, device="cuda")


def poison(*tensors):
    """The next tensors of these sizes lie where NaN was."""
    for t in tensors:
        keep = [torch.full_like(t, float("nan"), memory_format=torch.contiguous_format) for _ in range(4)]
        del keep


# query lengths, key lengths, max_q, first query token: single tokens, one tile, many blocks, few blocks for long tails, cut keys.
CASES = [([30, 1, 20], [100, 5, 300], 1, 0), ([30, 20], [100, 300], 12, 3), ([300, 40, 0, 7] * 9, [300, 40, 0, 7] * 9, 130, 5),
         ([5000], [10], 1, 0), ([3000, 2], [5000, 6000], 2, 1), ([2] * 700, [3] * 700, 1, 0), ([400, 500], [9000, 30], 64, 2)]


@pytest.mark.parametrize("q_len,k_len,max_q,first", CASES, ids=range(len(CASES)))
@pytest.mark.parametrize("H,Hk", [(2, 1), (8, 8)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new_out,new_lse", [(True, True), (False, True), (True, False), (False, False)])
def test_attention(M, q_len, k_len, max_q, first, H, Hk, dtype, new_out, new_lse):
    g = torch.Generator().manual_seed(first)
    T = sum(q_len) + first + 4
    q, k, v = (torch.randn(n, h, 64, generator=g).to(TYPES[dtype]).cuda() for n, h in ((T, H), (sum(k_len), Hk), (sum(k_len), Hk)))
    done = torch.zeros(T, dtype=torch.bool)
    for n, at in zip(q_len, first + np.cumsum([0] + q_len)):
        done[at:at + min(n, max_q)] = True
    rest = (~done).cuda()
    args = dict(q_offsets=offsets(q_len, first), k_offsets=offsets(k_len), max_q=max_q)
    lse = torch.full((T, H), 7.0, device="cuda")
    out = torch.full_like(q, 5.0)
    poison(q, lse)
    got = M.attention(q, k, v, out=None if new_out else out, lse=True if new_lse else lse, **args)
    assert (got[0] is out) != new_out and (got[1] is lse) != new_lse
    assert bool((got[0][rest] == (0.0 if new_out else 5.0)).all())
    assert bool((got[1][rest] == (-float("inf") if new_out or new_lse else 7.0)).all())
    assert bool(got[0][~rest].isfinite().all()) and not bool((got[0][~rest] == 5.0).all(-1).any())
    seen = torch.cat([torch.full((n,), m > 0) for n, m in zip(q_len, k_len)])
    live = (~rest)[first:T - 4] & seen.cuda()
    assert bool(got[1][first:T - 4][live].isfinite().all())
    if new_out and new_lse:  # neither result alone nor the memory changes the other
        poison(q)
        assert torch.equal(M.attention(q, k, v, **args), got[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("max_q", [1, 20])
def test_attention_of_equal_lengths(M, dtype, max_q):
    q, k, v = (torch.randn(4 * 50, 2, 64, device="cuda").to(TYPES[dtype]) for _ in range(3))
    poison(q)
    out, lse = M.attention(q, k, v, n_seqs=4, max_q=max_q, lse=True)
    rest = torch.arange(200, device="cuda") % 50 >= max_q
    assert bool((out[rest] == 0).all()) and bool((lse[rest] == -float("inf")).all())
    assert bool(lse[~rest].isfinite().all()) and bool(out[~rest].isfinite().all()) and not bool((out[~rest] == 0).all(-1).any())


@pytest.mark.parametrize("max_q", [1, 16])
def test_attention_in_place_keeps_its_queries(M, max_q):
    q, k, v = (torch.randn(100, 2, 64, device="cuda").bfloat16() for _ in range(3))
    own = q.clone()
    M.attention(own, k, v, q_offsets=offsets([60, 30], 5), k_offsets=offsets([60, 40]), max_q=max_q, out=own)
    done = torch.zeros(100, dtype=torch.bool)
    done[5:5 + max_q] = done[65:65 + max_q] = True
    assert torch.equal(own[~done], q[~done]) and not bool((own[done.cuda()] == q[done.cuda()]).all(-1).any())


@pytest.mark.parametrize("T,H,Hk,d,rot", [(40, 3, 2, 64, 64), (40, 3, 2, 72, 36), (9, 1, 1, 5, 2), (33, 2, 2, 512, 512), (2000, 16, 8, 128, 96),
                                          (3, 2, 1, 511, 254)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("new_q,new_k", [(True, True), (True, False), (False, True), (False, False)])
def test_norm_of_tokens_without_a_position(M, T, H, Hk, d, rot, dtype, pairs, new_q, new_k):
    g = torch.Generator().manual_seed(T)
    q, k = (torch.randn(T, h, d, generator=g).to(TYPES[dtype]).cuda() for h in (H, Hk))
    table = M.rope_table(torch.arange(20), rot).cuda()
    pos = torch.randint(-15, 35, (T,), generator=g).to(torch.int32)
    out = ((pos < 0) | (pos >= 20)).cuda()
    pos = pos.cuda()
    given_q, given_k = torch.full_like(q, 5.0), torch.full_like(k, 5.0)
    poison(q, k)
    got = M.qk_norm_rope(q, k, table, pos=pos, pairs=pairs, eps=0.0, q_out=None if new_q else given_q, k_out=None if new_k else given_k)
    want = M.qk_norm_rope(q, k, table, pos=pos.clamp(0, 19), pairs=pairs, eps=0.0)
    for x, w, new in zip(got, want, (new_q, new_k)):
        assert torch.equal(x[~out], w[~out]) and bool((x[out] == (0.0 if new else 5.0)).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_behind_a_short_table(M, dtype):
    q = torch.randn(30, 2, 48, device="cuda").to(TYPES[dtype])
    poison(q)
    y, _ = M.qk_norm_rope(q, None, M.rope_table(torch.arange(11), 48).cuda())  # the tokens' numbers are the positions
    assert bool((y[11:] == 0).all()) and bool(y[:11].isfinite().all()) and not bool((y[:11] == 0).all(-1).any())
    poison(q)
    z, _ = M.qk_norm_rope(q, q.clone(), torch.empty(0, 24, 2, device="cuda"))
    assert bool((z == 0).all())
