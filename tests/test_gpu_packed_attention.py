"""Head norms with rotation and attention over packed sequences, on the GPU against plain 64-bit results.

Tolerances.  fp32 sums of n terms in any order (rounding, or truncating as the tensor core adds) are off by at most
n 2^-23 times the sum of the magnitudes.

Norm and rotation: the sum of squares is off by dim 2^-23 of itself, its root by half of that, and the root, the
division, two products, the two products and the sum of the rotation add a rounding of 2^-24 each: in all
(dim / 2 + 8) 2^-23 (|a| + |b|) for a turned pair (a, b), and the result's rounding.

Attention: a score in base 2 is off by e = (dim + 2) 2^-23 scale log2(e) sum |q k|, the exponential's argument by
another 2^-23 of the largest |score|, the exponential by 2^-22 of itself; p and the sum of p change alike by at most
those in nats, so o changes by twice as much times sum p |v|.  Sums over n keys add n 2^-22, rescaling and joining some
16 roundings, p's own rounding to bf16 2^-8, each times sum p |v|; the result's rounding is 2^-8 (bf16) or 2^-24.
The log of the sum changes by the scores' error, p's and the sum's in nats.
"""
import math

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


def f64(t):
    return t.detach().double().cpu().numpy()


def heads(seed, T, H, d, dtype, extra=0, pad=0):
    """[T, H, d] values inside a wider buffer: `extra` heads more per token, `pad` values more per head."""
    g = torch.Generator().manual_seed(seed)
    buf = torch.randn(T, H + extra, d + pad, generator=g).to(TYPES[dtype]).cuda()
    return buf[:, extra:, :d]


# --- norm and rotation ---------------------------------------------------------


def rotated(x, w, table, pos, eps, pairs):
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    slack = np.abs(y)
    if table is not None:
        P = table.shape[1]
        c, s = table[pos][:, None, :, 0], table[pos][:, None, :, 1]
        ia = slice(0, 2 * P, 2) if pairs else slice(0, P)
        ib = slice(1, 2 * P, 2) if pairs else slice(P, 2 * P)
        a, b = y[..., ia].copy(), y[..., ib].copy()
        y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
        slack[..., ia] = slack[..., ib] = np.abs(a) + np.abs(b)
    return y, slack


QK = [(1, 12, 12, 64, 64), (3, 1, 1, 1, 0), (5, 2, 1, 3, 2), (7, 4, 2, 72, 72), (130, 16, 16, 72, 36), (65, 20, 4, 128, 96),
      (33, 3, 3, 100, 50), (9, 2, 2, 512, 512), (6, 1, 1, 511, 254), (1000, 6, 2, 80, 80), (2, 40, 8, 96, 0), (300, 5, 5, 24, 24)]


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["fused", "odd", "contiguous"])
@pytest.mark.parametrize("T,H,Hk,d,rot", QK)
def test_norm_and_rotation(M, T, H, Hk, d, rot, dtype, layout, pairs):
    g = torch.Generator().manual_seed(T + d)
    pad = 3 if layout == "odd" else 0
    buf = torch.randn(T, H + 2 * Hk, d + pad, generator=g).to(TYPES[dtype]).cuda()
    q, k = buf[:, :H, :d], buf[:, H:H + Hk, :d]
    if layout == "contiguous":
        q, k = q.contiguous(), k.contiguous()
    table = pos = None
    n_pos = 50
    if rot:
        table = M.rope_table(torch.arange(n_pos), rot).cuda()
        pos = torch.randint(0, n_pos, (T,), generator=g).to(torch.int32)
    wq, wk = (1 + 0.3 * torch.randn(2, d, generator=g)).cuda()
    args = dict(table=table, pos=None if pos is None else pos.cuda(), eps=1e-5, pairs=pairs)
    got = M.qk_norm_rope(q, k, q_weight=wq, k_weight=wk, **args)
    for x, w, y in ((q, wq, got[0]), (k, wk, got[1])):
        want, slack = rotated(f64(x), f64(w), None if table is None else f64(table), None if pos is None else pos.numpy(),
                              1e-5, pairs)
        slack = (d / 2 + 8) * 2.0 ** -23 * slack
        assert (np.abs(f64(y) - want) <= slack + HALF[dtype] * (np.abs(want) + slack)).all()
    # Without weights; in place, the rest of the buffer as it was.
    plain = M.qk_norm_rope(q, k, **args)
    whole = buf.clone()
    q2, k2 = (whole[:, :H, :d], whole[:, H:H + Hk, :d])
    M.qk_norm_rope(q2, k2, q_out=q2, k_out=k2, **args)
    assert torch.equal(q2, plain[0]) and torch.equal(k2, plain[1])
    q2.copy_(q)
    k2.copy_(k)
    assert torch.equal(whole, buf)
    only, none = M.qk_norm_rope(q, None, **args)
    assert none is None and torch.equal(only, plain[0])


def test_positions_outside_the_table_are_left_out(M):
    q = heads(1, 6, 2, 32, "bf16")
    table = M.rope_table(torch.arange(4), 32).cuda()
    pos = torch.tensor([0, -1, 3, 4, 2 ** 31 - 1, 1], dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 5.0)
    M.qk_norm_rope(q, None, table, pos=pos, q_out=out)
    assert bool((out[[1, 3, 4]] == 5).all()) and not bool((out[[0, 2, 5]] == 5).any())
    out.fill_(5.0)
    M.qk_norm_rope(q, None, table, q_out=out)  # the tokens' numbers: 4 and 5 are outside
    assert bool((out[4:] == 5).all()) and not bool((out[:4] == 5).any())


def test_norm_of_zero_huge_and_odd_rows(M):
    x = torch.zeros(4, 1, 64, device="cuda")
    x[1] = 1e-30
    x[2] = 1e18
    x[3, 0, 3] = float("nan")
    y, _ = M.qk_norm_rope(x, None, eps=1e-6)
    assert bool((y[0] == 0).all()) and torch.allclose(y[2], torch.ones(1, 64, device="cuda")) and bool(y[3].isnan().all())
    z, _ = M.qk_norm_rope(torch.zeros(1, 1, 8, device="cuda"), None, eps=0.0)
    assert bool(z.isnan().all())  # 0 / 0, as the formula has it


def test_rope_table_of_far_positions(M):
    pos = torch.tensor([[0, 0], [1, 2], [1_000_003, 123_456_789]])
    t = M.rope_table(pos, (8, 4), theta=500.0)
    assert t.shape == (3, 6, 2) and t.dtype == torch.float32
    for r in range(3):
        want = [(int(pos[r, 0]), 500.0 ** (-2 * i / 8)) for i in range(4)] + [(int(pos[r, 1]), 500.0 ** (-2 * i / 4)) for i in range(2)]
        for i, (p, f) in enumerate(want):
            # The angle in 64 bits is off by 2 x 2^-53 of itself, up to 1.3e8: below 3e-8; fp32 rounds by 2^-24.
            assert abs(float(t[r, i, 0]) - math.cos(p * f)) < 1.2e-7 and abs(float(t[r, i, 1]) - math.sin(p * f)) < 1.2e-7


# --- attention -------------------------------------------------------------------


def offsets(lengths, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(lengths)]), dtype=torch.int32, device="cuda")


def attend(q, k, v, causal, scale):
    """One sequence in 64 bits: o, lse, and the two factors of the tolerance: of the scores (in nats) and sum p |v|."""
    Lq, H, d = q.shape
    Lk, Hk, _ = k.shape
    if Lk == 0:
        z = np.zeros((Lq, H))
        return np.zeros_like(q), z - np.inf, z, np.zeros_like(q)
    kk, vv = np.repeat(k, H // Hk, 1), np.repeat(v, H // Hk, 1)
    s = np.einsum("ihd,jhd->hij", q, kk) * scale
    mag = np.einsum("ihd,jhd->hij", np.abs(q), np.abs(kk)) * scale
    see = np.arange(Lk)[None] <= np.arange(Lq)[:, None] + (Lk - Lq) if causal else np.ones((Lq, Lk), bool)
    s = np.where(see, s, -np.inf)
    m = np.max(s, -1, keepdims=True)
    p = np.exp(s - np.where(np.isfinite(m), m, 0.0))
    l = p.sum(-1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (np.log(l) + np.where(np.isfinite(m), m, 0.0))[..., 0]
    p = p / np.where(l > 0, l, 1.0)
    top = np.where(see, mag, 0.0).max(-1)
    e = (d + 2) * 2.0 ** -23 * top + 2.0 ** -23 * np.where(see, np.abs(s), 0.0).max(-1) + 2.0 ** -22
    o = np.einsum("hij,jhd->ihd", p, vv)
    return o, lse.T, e.T, np.einsum("hij,jhd->ihd", p, np.abs(vv))


def check(M, q, k, v, q_len, k_len, causal=False, scale=None, first=(0, 0), given=True, **kw):
    dtype = "bf16" if q.dtype == torch.bfloat16 else "f32"
    if given:
        kw.update(q_offsets=offsets(q_len, first[0]), k_offsets=offsets(k_len, first[1]))
    out, lse = M.attention(q, k, v, causal=causal, scale=scale, lse=True, **kw)
    got, got_lse = f64(out), f64(lse)
    q6, k6, v6 = f64(q), f64(k), f64(v)
    i, j = first
    if given:
        assert (got[:i] == 0).all() and (got_lse[:i] == -np.inf).all()
    for m, n in zip(q_len, k_len):
        o, l, e, pv = attend(q6[i:i + m], k6[j:j + n], v6[j:j + n], causal, scale or q.shape[2] ** -0.5)
        slack = (2 * e[..., None] + (n * 2.0 ** -22 + 16 * 2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0.0))) * pv
        err = np.abs(got[i:i + m] - o)
        tol = slack + HALF[dtype] * (np.abs(o) + slack)
        assert (err <= tol).all(), (float((err - tol).max()), np.argwhere(err > tol)[:3] + [[i, 0, 0]])
        dead = l == -np.inf
        assert (got_lse[i:i + m][dead] == -np.inf).all()
        diff = np.abs(got_lse[i:i + m][~dead] - l[~dead])
        assert (diff <= 2 * e[~dead] + n * 2.0 ** -22 + 2.0 ** -22 * (1 + np.abs(l[~dead]))).all()
        i, j = i + m, j + n
    if given:
        assert (got[i:] == 0).all() and (got_lse[i:] == -np.inf).all()
    return out


def qkv(seed, Tq, Tk, H, Hk, d, dtype):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(Tq, H, d, generator=g).to(TYPES[dtype]).cuda()
    kv = torch.randn(Tk, 2, Hk, d, generator=g).to(TYPES[dtype]).cuda()
    return q, kv[:, 0], kv[:, 1]


# query lengths, key lengths, heads, key heads, dim
SEQS = [
    ([1], [1], 1, 1, 64), ([1], [0], 2, 1, 64), ([0, 3, 0], [2, 5, 0], 2, 2, 72), ([5, 1, 7], [5, 1, 7], 4, 2, 128),
    ([129], [129], 2, 2, 64), ([200, 56], [200, 56], 6, 2, 80), ([128, 128], [128, 128], 2, 1, 96), ([255], [257], 3, 1, 72),
    ([40, 3, 300], [300, 3, 40], 4, 4, 64), ([1, 1, 1, 1], [77, 1, 500, 129], 8, 1, 128), ([2, 3], [600, 33], 8, 2, 72),
    ([17, 16, 15], [1000, 63, 64], 5, 5, 128), ([260], [700], 8, 2, 128), ([31], [2100], 12, 4, 64), ([513], [513], 1, 1, 128),
    ([64, 0, 65, 127, 1], [64, 9, 65, 127, 128], 7, 1, 80),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("q_len,k_len,H,Hk,d", SEQS)
def test_attention(M, q_len, k_len, H, Hk, d, causal, dtype):
    q, k, v = qkv(d + H, sum(q_len), sum(k_len), H, Hk, d, dtype)
    check(M, q, k, v, q_len, k_len, causal)
    check(M, q, k, v, q_len, k_len, causal, max_q=max(q_len))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,d", [(1, 1, 1), (3, 1, 5), (2, 2, 8), (4, 2, 40), (2, 1, 100), (2, 1, 160), (1, 1, 256), (130, 1, 64)])
def test_attention_of_other_heads(M, H, Hk, d, dtype):
    q, k, v = qkv(d, 70, 90, H, Hk, d, dtype)
    check(M, q, k, v, [30, 40], [50, 40], True)
    check(M, q[:2], k, v, [1, 1], [50, 40], True, max_q=1)


@pytest.mark.parametrize("H,Hk,d", [(17, 1, 64), (48, 1, 72), (96, 1, 128), (128, 2, 64), (128, 1, 80), (100, 4, 96)])
def test_large_groups(M, H, Hk, d):
    """Tiles of one to seven queries with all of their heads, full and with rows to spare."""
    q, k, v = qkv(H, 30, 300, H, Hk, d, "bf16")
    check(M, q, k, v, [9, 1, 20], [9, 130, 161], True)
    check(M, q[:2], k, v, [1, 1], [1, 299], True, max_q=1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
def test_equal_lengths_need_no_offsets(M, causal, dtype):
    q, k, v = qkv(3, 4 * 65, 4 * 130, 4, 2, 72, dtype)
    check(M, q, k, v, [65] * 4, [130] * 4, causal, given=False, n_seqs=4)
    one = check(M, q, k, v, [65] * 4, [130] * 4, causal)
    assert torch.equal(one, M.attention(q, k, v, k_offsets=offsets([130] * 4), causal=causal))
    q, k, v = qkv(4, 6, 6 * 4000, 4, 1, 128, dtype)
    check(M, q, k, v, [1] * 6, [4000] * 6, causal, given=False, n_seqs=6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q_len,first", [([100, 30], (7, 11)), ([1, 1], (3, 5))])
def test_tokens_of_no_sequence(M, q_len, first, dtype):
    """Tokens before the first and behind the last sequence, full of NaN: nothing of theirs is read into a row."""
    k_len = [90, 333]
    q, k, v = qkv(5, sum(q_len) + first[0] + 9, sum(k_len) + first[1] + 300, 4, 2, 64, dtype)
    for t, n, lengths in ((q, first[0], q_len), (k, first[1], k_len), (v, first[1], k_len)):
        t[:n] = float("nan")
        t[n + sum(lengths):] = float("nan")
    check(M, q, k, v, q_len, k_len, True, first=first)
    kept = torch.full_like(q, 5.0)
    M.attention(q, k, v, q_offsets=offsets(q_len, first[0]), k_offsets=offsets(k_len, first[1]), causal=True, out=kept)
    used = slice(first[0], first[0] + sum(q_len))
    assert bool((kept[:used.start] == 5).all()) and bool((kept[used.stop:] == 5).all()) and bool(kept[used].isfinite().all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,q_n", [(40, 40), (200, 200), (1500, 1), (1500, 90)])
def test_values_of_other_sequences_stay_there(M, n, q_n, dtype):
    """NaN and infinities in one sequence's keys and values do not reach its neighbours."""
    q, k, v = qkv(6, 3 * q_n, 3 * n, 4, 2, 64, dtype)
    k[n:2 * n], v[n:2 * n] = float("inf"), float("nan")
    out = M.attention(q, k, v, q_offsets=offsets([q_n] * 3), k_offsets=offsets([n] * 3), max_q=q_n)
    assert bool(out[:q_n].isfinite().all()) and bool(out[2 * q_n:].isfinite().all()) and bool(out[q_n:2 * q_n].isnan().all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q_n,n", [(300, 300), (1, 3000), (2, 40)])
def test_large_scores(M, q_n, n, dtype):
    """Scores in the hundreds, and a maximum that rises along the keys: one or two keys take all of a row."""
    q, k, v = qkv(7, q_n, n, 2, 2, 64, dtype)
    k.mul_(torch.linspace(0.1, 40, n, device="cuda")[:, None, None].to(k.dtype))
    check(M, q, k, v, [q_n], [n], True, scale=0.7)
    check(M, q, k.flip(0).contiguous(), v, [q_n], [n], False, scale=0.7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q_n,n", [(200, 260), (1, 2600)])
def test_layouts(M, q_n, n, dtype):
    """Heads first, parts of a fused projection, odd strides, results in place: the same values each time."""
    d = 72
    q, k, v = qkv(8, q_n, n, 4, 2, d, dtype)
    want = check(M, q, k, v, [q_n], [n], True)

    def moved(x, how):
        T, H, _ = x.shape
        if how == "heads":
            return x.permute(1, 0, 2).contiguous().permute(1, 0, 2)
        buf = torch.full((T, H + 3, d + (8 if how == "wide" else 3)), float("nan"), dtype=x.dtype, device="cuda")
        y = buf[:, 1:H + 1, :d]
        y.copy_(x)
        return y

    for how in ("heads", "wide", "odd"):
        got = check(M, moved(q, how), moved(k, how), moved(v, how), [q_n], [n], True)
        assert how == "odd" or torch.equal(got, want)
    own = moved(q, "wide")
    got = M.attention(own, k, v, causal=True, out=own, n_seqs=1)
    assert got is own and torch.equal(own, want)
    fused = torch.cat([q, q, q], 1)
    M.attention(fused[:, 4:8], k, v, causal=True, out=fused[:, 4:8])
    assert torch.equal(fused[:, 4:8], want) and torch.equal(fused[:, :4], q) and torch.equal(fused[:, 8:], q)


def test_long_key_axis(M):
    """65536 keys for 1, 20 and 200 queries: the axis is cut and joined."""
    for q_n in (1, 20, 200):
        q, k, v = qkv(9, q_n, 65536, 4, 2, 64, "bf16")
        check(M, q, k, v, [q_n], [65536], True, given=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_queries_behind_max_q_are_left(M, dtype):
    q, k, v = qkv(10, 50, 400, 2, 1, 64, dtype)
    out = torch.full_like(q, 5.0)
    M.attention(q, k, v, q_offsets=offsets([30, 20]), k_offsets=offsets([100, 300]), max_q=12, out=out)
    full = M.attention(q, k, v, q_offsets=offsets([30, 20]), k_offsets=offsets([100, 300]))
    done = [*range(12), *range(30, 42)]
    left = [t for t in range(50) if t not in done]
    assert bool((out[left] == 5).all())
    # The same formula by another kernel (bf16: p rounded against another maximum).
    assert torch.allclose(out[done].float(), full[done].float(), atol=4 * HALF[dtype] + 1e-5)


@pytest.mark.parametrize("bad", [[-5, 20, 10, 60], [0, 70, 30, 1000], [40, 0, 0, 40], [-2 ** 31, 2 ** 31 - 1, 0, 5]])
@pytest.mark.parametrize("n", [40, 1])
def test_offsets_that_are_wrong_stay_inside(M, bad, n):
    """Offsets out of range or order: clamped, and nothing outside the tensors is touched."""
    q, k, v = qkv(11, 60, 60, 2, 1, 64, "bf16")
    off = torch.tensor(bad, dtype=torch.int32, device="cuda")
    buf = torch.full((80, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    M.attention(q, k, v, q_offsets=off, k_offsets=off, out=buf[10:70], max_q=n)
    torch.cuda.synchronize()
    assert bool((buf[:10] == 5).all()) and bool((buf[70:] == 5).all()) and not bool(buf.isnan().any())


def test_many_sequences(M):
    lengths = np.random.default_rng(1).integers(0, 9, 3000).tolist()
    T = sum(lengths)
    q, k, v = qkv(12, T, T, 2, 1, 64, "bf16")
    got = M.attention(q, k, v, q_offsets=offsets(lengths), k_offsets=offsets(lengths), causal=True, max_q=8)
    i = 0
    q6, k6, v6 = f64(q), f64(k), f64(v)
    for m in lengths:
        o, _, e, pv = attend(q6[i:i + m], k6[i:i + m], v6[i:i + m], True, 0.125)
        slack = (2 * e[..., None] + 2.0 ** -8 + 2.0 ** -18) * pv
        assert (np.abs(f64(got[i:i + m]) - o) <= slack + 2.0 ** -8 * (np.abs(o) + slack)).all()
        i += m


@pytest.mark.parametrize("q_n", [1, 300])
def test_attention_captured_twice_and_side_by_side(M, q_n):
    """Two graphs of different inputs replayed one after another and on two streams at once."""
    sets = [qkv(20 + i, q_n, 5000, 4, 2, 128, "bf16") for i in range(2)]
    want = [M.attention(*s, causal=True) for s in sets]
    graphs, outs = [], []
    for s in sets:
        M.attention(*s, causal=True)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(M.attention(*s, causal=True))
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    streams = [torch.cuda.Stream() for _ in range(2)]
    res = []
    for st, s in zip(streams, sets):
        for _ in range(5):
            last = M.attention(*s, causal=True, stream=st.cuda_stream)
        res.append(last)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(res, want))


@pytest.mark.parametrize("q_n", [1, 200])
def test_keys_beyond_32_bits(M, q_n):
    """Tokens 16400 values apart: the last keys lie 2.4e9 values into their buffer."""
    n, stride = 147_000, 16_400
    q, k, v = qkv(30, q_n, n, 1, 1, 64, "bf16")
    buf = torch.empty(n * stride, dtype=torch.bfloat16, device="cuda")
    kf, vf = (buf.as_strided((n, 1, 64), (stride, 64, 1), at) for at in (0, 8192))
    kf.copy_(k)
    vf.copy_(v)
    off = [1000, n - 1000 - 300, 300]
    args = dict(q_offsets=offsets([0, 0, q_n]), k_offsets=offsets(off), causal=True)
    assert torch.equal(M.attention(q, kf, vf, **args), M.attention(q, k, v, **args))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q_n", [1, 40])
def test_one_key_head_expanded(M, q_n, dtype):
    """Heads and tokens that share their memory (stride 0)."""
    q, k, v = qkv(31, q_n, 700, 4, 1, 64, dtype)
    want = check(M, q, k, v, [q_n], [700], True)
    got = check(M, q, k.expand(-1, 4, -1), v.expand(-1, 4, -1), [q_n], [700], True)
    assert got.shape == want.shape
    check(M, q[:1].expand(q_n, -1, -1), k, v, [q_n], [700])
    check(M, q, k[:1].expand(700, -1, -1), v, [q_n], [700])


def test_two_host_threads_at_once(M):
    """Two threads, each with its stream and its inputs: cut and whole key axes, sorts and rows, side by side."""
    import threading

    def work(seed, stream):
        q, k, v = qkv(seed, 1 + 200 * seed, 4000 + seed, 4, 2, 128, "bf16")
        ids = torch.randint(0, 16, (5000, 2), dtype=torch.int32, generator=torch.Generator().manual_seed(seed)).cuda()
        x = torch.randn(5000, 72, generator=torch.Generator().manual_seed(seed)).cuda()
        torch.cuda.synchronize()

        def run():
            plan = M.expert_sort(ids, 16, stream=stream.cuda_stream)
            return (M.attention(q, k, v, causal=True, stream=stream.cuda_stream), M.expert_rows(x, plan, stream=stream.cuda_stream),
                    plan.place)

        first = run()
        stream.synchronize()
        for _ in range(20):
            again = run()
            stream.synchronize()
            if not all(torch.equal(a, b) for a, b in zip(first, again)):
                bad.append(seed)

    bad = []
    threads = [threading.Thread(target=work, args=(i, torch.cuda.Stream())) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
