"""8-bit rows at the edges of their formats, sizes and streams, against the float64 oracle (tolerances: see
tests/test_gpu_q8.py)."""
import numpy as np
import pytest
import torch

from oracle import q8 as O
from test_gpu_q8 import HALF, M, TYPES, VALUES, activations, exps, f64, filled, ints  # noqa: F401  (M: a fixture)

pytestmark = pytest.mark.gpu


# --- combine: infinities -----------------------------------------------------

@pytest.mark.parametrize("k", [1, 2, 3, 5, 6, 7, 8, 9, 10, 13, 16])
@pytest.mark.parametrize("unaligned", [0, 1])
def test_combine_keeps_infinities(M, k, unaligned):
    """An e5m2 infinity in a token's first or last slot reaches its own value with its sign and nothing else, in a
    call of few tokens and in one of many, which agree bit for bit."""
    D, T, few = 264, 2000, 20
    c, h = filled(M, 5, 50, D, "e5m2")
    for row, at, byte, v in ((0, 3, 0x7c, np.inf), (1, 130, 0xfc, -np.inf), (2, 263, 0x7c, np.inf)):
        c.q.view(torch.uint8)[row, at] = byte
        h[row, at] = v
    rng = np.random.default_rng(k)
    rows = rng.integers(3, 50, (T, k)).astype(np.int32)
    rows[::4, 0], rows[1::4, k - 1], rows[2::4, k // 2] = 0, 1, 2
    w = rng.uniform(0.1, 1, (T, k)).astype(np.float32)
    x = activations(7, T, D + unaligned, "bf16")[:, unaligned:]
    rt, wt = torch.from_numpy(rows).cuda(), torch.from_numpy(w).cuda()
    out, norms = M.q8_combine(c, rt, wt, x=x, norms=True)
    want, wn = O.combine(h, rows, w.astype(np.float64), f64(x))
    inf = np.isinf(want)
    np.testing.assert_array_equal(f64(out)[inf], want[inf])
    big, _ = O.combine(np.abs(h), rows, w, np.abs(f64(x)))
    err = (k + 3) * 2.0 ** -23 * big[~inf]
    assert (np.abs(f64(out)[~inf] - want[~inf]) <= err + HALF["bf16"] * (np.abs(want[~inf]) + err)).all()
    np.testing.assert_array_equal(np.isinf(f64(norms)), np.isinf(wn))
    small, small_n = M.q8_combine(c, rt[:few], wt[:few], x=x[:few], norms=True)
    assert torch.equal(small, out[:few])
    np.testing.assert_array_equal(np.isinf(f64(small_n)), np.isinf(wn[:few]))


# --- results on a stream that is not the current one -------------------------

def held_back(side):
    """The current stream busy for a while (a tenth of a second), `side` free."""
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    return side.cuda_stream


@pytest.mark.parametrize("dtype", [torch.float8_e4m3fn, torch.float8_e5m2])
def test_product_on_another_stream_keeps_its_rows(M, dtype):
    """Nothing of a product's own result is filled on the current stream after the product has run on another."""
    a, _ = filled(M, 1, 300, 256, "e4m3")
    b, _ = filled(M, 2, 500, 256, "e4m3")
    want = M.q8_matmul(a, b, dtype=dtype)
    side = torch.cuda.Stream()
    got = M.q8_matmul(a, b, dtype=dtype, stream=held_back(side))
    torch.cuda.synchronize()
    assert torch.equal(got.q.view(torch.uint8), want.q.view(torch.uint8)) and torch.equal(got.scale, want.scale)


@pytest.mark.parametrize("call", ["read", "combine", "norms", "matmul"])
def test_results_on_another_stream_have_memory_of_their_own(M, call):
    """Memory that the current stream has freed but may still write is not given to a result of another stream."""
    a, _ = filled(M, 1, 1024, 512, "e4m3")
    b, _ = filled(M, 2, 512, 512, "e4m3")
    rows = torch.arange(1024, dtype=torch.int32, device="cuda")[:, None].expand(1024, 8).contiguous()
    calls = dict(read=lambda s: M.q8_read(a, dtype=torch.float32, stream=s),
                 combine=lambda s: M.q8_combine(a, rows, dtype=torch.float32, stream=s),
                 norms=lambda s: M.q8_combine(a, rows, norms=True, stream=s)[1],
                 matmul=lambda s: M.q8_matmul(a, b, dtype=torch.float32, stream=s))
    want = calls[call](0).clone()
    side = torch.cuda.Stream()
    torch.empty_like(want).fill_(5.0)  # loads the fill's kernel, which would wait for the stream
    s = held_back(side)
    stale = torch.empty_like(want)
    stale.fill_(5.0)  # runs once the current stream is free again
    del stale
    got = calls[call](s)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


# --- rows that a product does not write --------------------------------------

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.float8_e4m3fn])
@pytest.mark.parametrize("by", ["offsets", "dst"])
def test_a_new_result_has_zeros_where_nothing_is_written(M, dtype, by):
    a, _ = filled(M, 1, 200, 256, "e4m3")
    b, _ = filled(M, 2, 2 * 128, 256, "e4m3")
    if by == "offsets":  # rows before, between and behind the groups' ones: 10..49 and 50..119 have one
        kw, b2, live = dict(offsets=ints([10, 50, 120])), b, range(10, 120)
    else:
        b2 = M.Q8(b.q[:128], b.scale[:128])
        kw, live = dict(dst=ints([r if r % 3 else -1 for r in range(200)])), [r for r in range(200) if r % 3]
    stale = torch.full((200, 128), 7.0, device="cuda")  # what such a result's memory may have held
    del stale
    stale = torch.full((200, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    del stale
    got = M.q8_matmul(a, b2, dtype=dtype, **kw)
    v = M.q8_read(got, dtype=torch.float32) if isinstance(got, M.Q8) else got.float()
    rest = torch.ones(200, dtype=torch.bool)
    rest[list(live)] = False
    assert bool((v[rest.cuda()] == 0).all()) and bool((v[~rest.cuda()] != 0).any(1).all())


# --- combine: scales at the ends of their range ------------------------------

@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", [1, 2, 5, 9, 16])
@pytest.mark.parametrize("T", [30, 2000])
def test_combine_weights_meet_values_not_scales(M, T, k, dtype, fmt):
    """Scale bytes from 0 to 254 under weights from 0 to 2048: w h where w x scale would pass fp32's range (2^127 x 2,
    2^118 x 2048) or lose digits among its subnormals, and zeros in such blocks stay zeros.
    Each fp32 operation is off by 2^-24 of its result or by half of the least subnormal, 2^-150."""
    D, R = 200, 400
    rng = np.random.default_rng(T + k)
    c = M.q8_empty(R, D, TYPES[fmt])
    v = torch.from_numpy(rng.standard_normal((R, D)).astype(np.float32) / 16).clamp(-0.25, 0.25).to(TYPES[fmt])
    c.q.copy_(v)
    c.q.view(torch.uint8)[:, ::3] = 0
    kinds = np.array([0, 1, 3, 20, 100, 127, 140, 240, 245, 254])
    e = kinds[rng.integers(0, len(kinds) - 3, (R, 2))]
    e[:40] = rng.choice(kinds[-3:], (40, 2))  # the first rows are huge
    c.scale.copy_(torch.from_numpy(e.astype(np.uint8)))
    h = O.dequantise(f64(c.q), e - 127)
    assert np.isfinite(h.astype(np.float32)).all()
    rows = rng.integers(40, R, (T, k)).astype(np.int32)
    rows[::2, k // 2] = rng.integers(0, 40, len(rows[::2]))  # one huge row at most in a token
    w = rng.choice(np.array([0, 1e-20, 1e-3, 0.3, 1.7], np.float32), (T, k))
    small = np.abs(h).max(1)[rows] < 2.0 ** 116
    w = np.where(small & (rng.random((T, k)) < 0.3), np.float32(2048), w)
    w[::4, k // 2] = 2.0
    out = M.q8_combine(c, torch.from_numpy(rows).cuda(), torch.from_numpy(w).cuda(), dtype=VALUES[dtype])
    want, _ = O.combine(h, rows, w.astype(np.float64))
    big, _ = O.combine(np.abs(h), rows, w.astype(np.float64))
    assert (np.abs(want) < 2.0 ** 127).all()
    err = (k + 3) * 2.0 ** -23 * big + k * 2.0 ** -149
    bound = err + HALF[dtype] * (np.abs(want) + err) + (2.0 ** -134 if dtype == "bf16" else 2.0 ** -150)
    assert (np.abs(f64(out) - want) <= bound).all()


# --- GELU --------------------------------------------------------------------

@pytest.mark.parametrize("act", ["gelu", "gelu_tanh"])
def test_gelu_is_as_exact_as_fp32_functions_make_it(M, act):
    """The product's GELU against float64, beside the same formula in fp32 with the library's erf and tanh.

    Bounds, in units of u = 2^-24, for z (1 + h) / 2 = |z| / 2 x |h| + z / 2, rounded once (u |result|).
    erf, |h| = 1 - 2^-g: the fit 0.04 u, g's three last roundings 3 ln2 g 2^-g u <= 1.6 u, 2^x 2.9 2^-g u <= 2.9 u, |h|'s
    rounding 0.5 u: 5.1 u of h, so 2.6 u + 1 u of |z|; for z < -2, where 2^-g < 0.05, 0.04 + 0.5 + 0.15 + 0.5 = 1.2 u,
    0.6 u + 0.05 u.
    tanh, |h| = 1 - 2t: the exponent's roundings and constants 4 u ln2 w 2 t (1 - t) <= 1.8 u, 2^x 2.9 u 2 t (1 - t) <=
    1.5 u, four more on t 5 u 2t <= 5 u, 0.5 u: 8.8 u, so 4.4 u + 1 u of |z|; for z < -2 (t < 0.023) 0.7 + 0.2 + 0.3 +
    0.5 = 1.7 u, 0.9 u + 0.05 u.
    On the mean no more than a quarter above the fp32 formula for |z| > 1/2, and below twice it near 0, where the
    result's own rounding no longer covers the two functions' difference."""
    n = 1 << 17
    g = torch.Generator().manual_seed(5)
    near = (2 * torch.rand(n // 2, generator=g) - 1) * torch.exp2(torch.randint(-10, 1, (n // 2,), generator=g).float())
    z = torch.cat([14 * torch.rand(n // 2, generator=g) - 7, near]).cuda()
    a, b = M.q8_write(torch.zeros(1, 1, device="cuda"), M.q8_empty(1, 1)), M.q8_empty(n, 1)
    got = f64(M.q8_matmul(a, b, bias=z[None], act=act, dtype=torch.float32))[0]
    if act == "gelu":
        plain = 0.5 * z * (1 + torch.erf(z * 0.7071067811865476))
    else:
        plain = 0.5 * z * (1 + torch.tanh(0.7978845608028654 * (z + 0.044715 * z * z * z)))
    z64 = f64(z)
    if act == "gelu":  # 1 + erf and 1 + tanh cancel in float64 as well
        from scipy.special import erfc
        want = 0.5 * z64 * erfc(-z64 / np.sqrt(2))
    else:
        want = z64 / (1 + np.exp(-2 * np.sqrt(2 / np.pi) * (z64 + 0.044715 * z64 ** 3)))
    u = 2.0 ** -24 * np.abs(z64)
    err, err_plain = np.abs(got - want) / u, np.abs(f64(plain) - want) / u
    low = z64 < -2
    assert err.max() <= (3.6 if act == "gelu" else 5.4) and err[low].max() <= (0.65 if act == "gelu" else 0.95)
    rms = lambda v: np.sqrt((v * v).mean())  # noqa: E731
    for lo, hi, most in ((-7, -4, 1.25), (-4, -2, 1.25), (-2, -0.5, 1.25), (-0.5, 0.5, 2), (0.5, 2, 1.25), (2, 7, 1.25)):
        at = (z64 >= lo) & (z64 < hi)
        assert rms(err[at]) <= most * rms(err_plain[at]), (lo, hi)
