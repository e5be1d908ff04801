"""Scores far beyond the exponential's range: every kernel of the packed attention gives the mean of the values whose
keys score highest, whatever the scores' size.

Keys come in groups; all keys of a group are the same, and a group's score is a whole multiple of another's, so that in
exact arithmetic p is 1 for the keys of the highest group that a row sees and 0 (below 2^-500) for the others.  A
score is d equal products of two numbers of 8 bits: 16 + 7 bits, exact in fp32 in any order.  So p is exactly 1 or 0,
the sum of n values is off by n 2^-22 of the sum of magnitudes, normalising and joining by 16 roundings of 2^-24, and
the result is rounded by 2^-8 (bf16) or 2^-24.  The log of the sum is the score times scale, eight
roundings of 2^-24 at most (scale and its base-2 form, two constants, two products, a sum), and log(n), off by 2^-21.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def M():
    from paper_2606_15615_gb300 import moeca
    return moeca


def offsets(lengths):
    return torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device="cuda")


def check(M, q_len, k_len, H, Hk, d, dtype, power, sign, order, by, causal, drift=0.0):
    """Scores of sign 2^power in base 2 (times 1, 2 and 3 along the keys, in the given order); values that drift along the keys."""
    g = torch.Generator().manual_seed(d + power)
    product = 2.0 ** power / np.log2(np.e) / d ** 0.5  # |q k| of a channel, with scale d^-0.5
    scale = d ** -0.5
    if by == "scale":
        product, scale = 1.0, scale * product
    a, b = torch.tensor([product ** 0.5 / 1.5, product ** 0.5 * 1.5]).to(torch.bfloat16).tolist()
    factor = torch.cat([torch.tensor(order, dtype=torch.float32).repeat_interleave(-(-n // len(order)))[:n] for n in k_len])
    q = torch.full((sum(q_len), H, d), a).to(TYPES[dtype]).cuda()
    k = (factor[:, None, None] * (sign * b)).to(torch.bfloat16).expand(-1, Hk, d).contiguous().to(TYPES[dtype]).cuda()
    v = torch.randn(sum(k_len), Hk, d, generator=g) + drift * torch.linspace(-1, 1, sum(k_len))[:, None, None]
    v = v.to(TYPES[dtype]).cuda()
    out, lse = M.attention(q, k, v, q_offsets=offsets(q_len), k_offsets=offsets(k_len), causal=causal, scale=scale, lse=True)
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    key = k[:, 0, 0].double().cpu().numpy()
    i = j = 0
    for m, n in zip(q_len, k_len):
        s = a * d * key[j:j + n] * scale
        see = np.arange(n)[None] <= np.arange(m)[:, None] + (n - m) if causal else np.ones((m, n), bool)
        x = np.where(see, s[None], -np.inf)
        top = x.max(-1, keepdims=True)
        p = (x == top) & see
        count = p.sum(-1)
        share = torch.from_numpy(p / np.maximum(count, 1)[:, None]).cuda()
        vv = v[j:j + n].double().repeat_interleave(H // Hk, 1)
        o, mag = (torch.einsum("ij,jhd->ihd", share, x).cpu().numpy() for x in (vv, vv.abs()))
        slack = (n * 2.0 ** -22 + 16 * 2.0 ** -24) * mag
        live = count > 0
        err = np.abs(got[i:i + m] - o) - slack - HALF[dtype] * (np.abs(o) + slack)
        assert (err[live] <= 0).all(), (float(np.nanmax(err[live])), got[i:i + m][live][0, 0, :3], o[live][0, 0, :3])
        assert (got[i:i + m][~live] == 0).all() and (got_lse[i:i + m][~live] == -np.inf).all()
        want = top[live] + np.log(count[live])[:, None]
        assert (np.abs(got_lse[i:i + m][live] - want) <= 2.0 ** -21 * (1 + np.abs(want))).all()
        i, j = i + m, j + n


# Rows of a few queries, one tile, more than one, and enough tiles for two a block; the keys of each in one piece.
WHOLE = [([1], [250], 4, 2), ([40], [250], 4, 2), ([250], [255], 2, 2), ([200] * 20, [200 + 7 * i for i in range(20)], 8, 8)]


@pytest.mark.parametrize("q_len,k_len,H,Hk", WHOLE, ids=["few", "tile", "tiles", "pairs"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("power,sign,order,by,causal", [
    (10, 1, (1, 2, 3), "values", False), (9, -1, (3, 2, 1), "scale", True), (20, 1, (1, 3, 2), "values", True),
    (31, 1, (1,), "values", False), (31, -1, (2, 1), "scale", False), (32, 1, (1, 2, 3), "values", True),
    (34, 1, (1,), "values", False), (34, -1, (1, 2), "values", True), (37, 1, (3, 1, 2), "scale", False),
    (40, 1, (1, 2), "values", True), (40, -1, (3, 2, 1), "scale", False), (100, 1, (1, 2), "scale", True)])
def test_scores_beyond_the_exponent(M, q_len, k_len, H, Hk, d, dtype, power, sign, order, by, causal):
    check(M, q_len, k_len, H, Hk, d, dtype, power, sign, order, by, causal)


# Key axes that are cut: chunks of different lengths, and rows (causal) that see a part of their last chunk.
CUT = [([1], [5000], 4, 2), ([3, 1], [2600, 9001], 4, 1), ([40], [5000], 4, 2), ([300], [9001], 2, 2), ([17, 250], [700, 12000], 2, 1)]


@pytest.mark.parametrize("q_len,k_len,H,Hk", CUT, ids=["one", "few", "tile", "tiles", "uneven"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [72, 128])
@pytest.mark.parametrize("power,sign,order,by,causal", [
    (10, 1, (1,), "values", False), (16, -1, (1,), "scale", True), (20, 1, (1, 3, 2), "values", True), (24, -1, (1,), "values", False),
    (31, 1, (1,), "scale", True), (34, 1, (1, 2), "values", False), (40, -1, (2, 1), "scale", True), (100, 1, (1,), "scale", False)])
def test_chunks_are_joined_by_their_sums(M, q_len, k_len, H, Hk, d, dtype, power, sign, order, by, causal):
    """The same score everywhere: a chunk weighs what its number of keys says, at any score."""
    check(M, q_len, k_len, H, Hk, d, dtype, power, sign, order, by, causal, drift=2.0)
