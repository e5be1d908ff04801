"""8-bit rows on the GPU against the float64 oracle.

Tolerances.  Quantising is exact arithmetic and one rounding: outputs equal the
oracle's.  Reading back is exact in fp32, and in bf16 away from its subnormals.
A sum of n products in fp32 (any order, each addition rounded or truncated) is
off by at most n 2^-23 times the sum of the magnitudes; GELU has slope below
1.13 and is evaluated within 8 x 2^-24 |z|; a result in bf16 / fp32 is off by
2^-8 / 2^-24 of itself, one in 8 bits by half a step of the scale it carries:
2^-4 (e4m3) or 2^-3 (e5m2) of itself, or half of the least subnormal.
"""
import numpy as np
import pytest
import torch

from oracle import q8 as O

pytestmark = pytest.mark.gpu

TYPES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
VALUES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24, "e4m3": 2.0 ** -4, "e5m2": 2.0 ** -3}


@pytest.fixture(scope="module")
def M():
    from paper_2606_15615_gb300 import moeca
    return moeca


def f64(t):
    return t.detach().double().cpu().numpy()


def exps(scale):
    return scale.cpu().numpy().astype(np.int64) - 127


def activations(seed, rows, width, dtype="f32"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, width, generator=g) * torch.exp(torch.randn(rows, 1, generator=g)) \
        * torch.exp(torch.randn(1, width, generator=g))
    return x.to(VALUES[dtype]).cuda()


def filled(M, seed, rows, width, fmt):
    """A cache of quantised rows, its padding full of NaN bytes and stray scales, and its float64 value."""
    c = M.q8_empty(rows, width, TYPES[fmt])
    q, e = O.quantise(f64(activations(seed, rows, width)), fmt)
    c.q.untyped_storage().fill_(0x7f)
    c.scale.untyped_storage().fill_(0xff)
    c.q.copy_(torch.from_numpy(q).to(torch.float32).to(TYPES[fmt]))
    c.scale.copy_(torch.from_numpy((e + 127).astype(np.uint8)))
    return c, O.dequantise(q, e)


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def same(cache, x, fmt, rows=None):
    """The cache's rows hold x's quantised rows, bit for bit (NaN for NaN)."""
    q, e = O.quantise(f64(x), fmt)
    got, ge = f64(cache.q), exps(cache.scale)
    if rows is not None:
        got, ge = got[rows], ge[rows]
    np.testing.assert_array_equal(ge, e)
    np.testing.assert_array_equal(got, q)


# --- write -------------------------------------------------------------------

WIDTHS = [(1, 1), (2, 127), (3, 128), (5, 129), (7, 1152), (33, 1000), (300, 2560), (4, 4099), (2000, 384), (65, 17)]


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,width", WIDTHS)
def test_write(M, rows, width, dtype, fmt):
    x = activations(rows, rows, width, dtype)
    c = M.q8_empty(rows, width, TYPES[fmt])
    c.q.untyped_storage().fill_(0x55)
    c.scale.untyped_storage().fill_(0x55)
    assert M.q8_write(x, c) is c
    same(c, x, fmt)
    pad = c.q.view(torch.uint8).as_strided((rows, c.q.stride(0) if rows > 1 else width), (c.q.stride(0), 1))[:, width:]
    assert bool((pad == 0x55).all())
    nb = c.scale.shape[1]
    spad = c.scale.as_strided((rows, c.scale.stride(0) if rows > 1 else nb), (c.scale.stride(0), 1))[:, nb:]
    assert bool((spad == 0x55).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_write_special_values(M, dtype, fmt):
    """Zero blocks, NaN, infinities, borders of the scale, the largest and smallest magnitudes."""
    most = O.FORMATS[fmt][0]
    x = torch.zeros(24, 256)
    g = torch.Generator().manual_seed(4)
    x[4:] = torch.randn(20, 256, generator=g)
    x[1, 3], x[2, 4], x[3, 200] = float("nan"), float("inf"), -float("inf")
    x[4, 5], x[5, 6], x[6, 7] = float("nan"), float("-inf"), float("inf")
    x[7] = float("nan")
    x[8] = float("inf")
    for r, v in enumerate([most, most * 2 ** 7, most * 2 ** -40, 3.0e38, -3.38e38, 1e-38, 1e-40, 2.0 ** -133, 1.7, 1.76,
                           most * (1 + 2 ** -7), most * 2 ** -120]):
        x[9 + r, :128] *= abs(v) / 8
        x[9 + r, 17] = v
    x[21] = x[21] * 1e-39
    x[22, :128] = torch.logspace(-60, 0, 128, base=2.0)
    x = x.to(VALUES[dtype]).cuda()
    c = M.q8_empty(24, 256, TYPES[fmt])
    M.q8_write(x, c)
    same(c, x, fmt)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("base,stride", [(0, 1408), (1, 1301), (3, 1290), (8, 1304), (4, 1300)])
def test_write_from_strided_rows(M, dtype, base, stride):
    buf = activations(9, 1, 40 * stride + 16, dtype)[0]
    x = buf.as_strided((37, 1290), (stride, 1), base)
    c = M.q8_empty(37, 1290)
    M.q8_write(x, c)
    same(c, x, "e4m3")


def test_write_lists(M):
    """src and dst lists, entries out of range, a device count; other rows keep what they hold."""
    x = activations(1, 20, 300, "bf16")
    lib = 1 << 30
    src = ints([3, 0, -1, 20, 5, 19, 7, 7, 2, lib])
    dst = ints([9, 0, 1, 2, -1, 15, 16, 4, 5, 6])
    for count, live in [(None, [(3, 9), (0, 0), (19, 15), (7, 4), (2, 5)]), (6, [(3, 9), (0, 0), (19, 15)]), (0, []),
                        (-4, []), (1, [(3, 9)]), (lib, [(3, 9), (0, 0), (19, 15), (7, 4), (2, 5)])]:
        c, before = filled(M, 2, 16, 300, "e4m3")
        q0, s0 = c.q.view(torch.uint8).clone(), c.scale.clone()
        M.q8_write(x, c, src=src, dst=dst, count=None if count is None else ints([count]))
        for s, d in live:
            same(c, x[s:s + 1], "e4m3", [d])
        rest = [r for r in range(16) if r not in [d for _, d in live]]
        assert torch.equal(c.q.view(torch.uint8)[rest], q0[rest]) and torch.equal(c.scale[rest], s0[rest])


def test_write_one_sided_lists(M):
    x = activations(5, 50, 129)
    c = M.q8_empty(12, 129)
    M.q8_write(x, c, src=ints(list(range(40, 28, -1))))
    same(c, x[torch.arange(40, 28, -1)], "e4m3")
    c = M.q8_empty(60, 129)
    M.q8_write(x, c, dst=ints(list(range(59, 9, -1))))
    same(c, x, "e4m3", list(range(59, 9, -1)))


# --- read --------------------------------------------------------------------

@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,width", WIDTHS)
def test_read(M, rows, width, dtype, fmt):
    c, h = filled(M, 7, rows, width, fmt)
    got = M.q8_read(c, dtype=VALUES[dtype])
    assert got.dtype == VALUES[dtype]
    np.testing.assert_array_equal(f64(got), h)
    at = ([rows - 1, 0, -1, rows, 0, 1 << 30, -(1 << 31)] * 60)[:401]
    out = torch.full((401, width + 3), 5.0, dtype=VALUES[dtype], device="cuda")
    assert M.q8_read(c, ints(at), out=out[:, 1:width + 1]).data_ptr() == out[:, 1:].data_ptr()
    want = np.array([h[i] if 0 <= i < rows else np.zeros(width) for i in at])
    np.testing.assert_array_equal(f64(out[:, 1:width + 1]), want)
    assert bool((out[:, 0] == 5).all()) and bool((out[:, width + 1:] == 5).all())


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_read_every_byte_and_scale(M, fmt):
    """All 256 bytes under each scale that fp32 can hold; 255 is NaN."""
    c = M.q8_empty(256, 256, TYPES[fmt])
    c.q.view(torch.uint8).copy_(torch.arange(256, dtype=torch.uint8).expand(256, 256))
    c.scale.copy_(torch.arange(256, dtype=torch.uint8)[:, None].expand(256, 2))
    got = f64(M.q8_read(c, dtype=torch.float32))
    v = f64(c.q[0])
    with np.errstate(over="ignore"):
        want = np.where(np.arange(256)[:, None] == 255, np.nan, v * np.ldexp(1.0, np.arange(256) - 127)[:, None])
        want = want.astype(np.float32).astype(np.float64)
    np.testing.assert_array_equal(got, want)
    assert (np.signbit(got) == np.signbit(want))[~np.isnan(want)].all()


# --- combine -----------------------------------------------------------------

COMBINE = [(1, 1, 1, 1), (1, 2, 1152, 1), (2, 3, 129, 1), (7, 2, 1000, 7), (300, 2, 1152, 100), (310, 3, 2560, 31),
           (64, 8, 384, 64), (333, 9, 1003, 37), (320, 16, 200, 5), (305, 5, 127, 61), (400, 1, 768, 40), (303, 4, 264, 101)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("T,k,D,seq", COMBINE)
def test_combine(M, T, k, D, seq, fmt, dtype):
    rng = np.random.default_rng(T + k)
    R = T * k + 3
    c, h = filled(M, 3, R, D, fmt)
    rows = rng.permutation(R)[:T * k].reshape(T, k).astype(np.int32)
    rows[rng.random((T, k)) < 0.15] = rng.choice([-1, R, 1 << 30, -(1 << 31)])
    rows[T // 2] = -1  # a token with nothing cached
    w = rng.standard_normal((T, k)).astype(np.float32)
    x = activations(11, T, D, dtype)
    gate = torch.from_numpy(rng.standard_normal((T // seq, D)).astype(np.float32)).cuda()
    wt, rt = torch.from_numpy(w).cuda(), torch.from_numpy(rows).cuda()
    for kw in (dict(weights=wt, x=x, gate=gate, norms=True), dict(weights=wt, x=x), dict(norms=True, dtype=x.dtype),
               dict(gate=gate, weights=wt, dtype=x.dtype)):
        has = {n: n in kw for n in ("weights", "x", "gate")}
        got = M.q8_combine(c, rt, **kw)
        out, norms = got if "norms" in kw else (got, None)
        want, wn = O.combine(h, rows, w.astype(np.float64) if has["weights"] else None, f64(x) if has["x"] else None,
                             f64(gate) if has["gate"] else None, seq)
        big, _ = O.combine(np.abs(h), rows, np.abs(w) if has["weights"] else None, np.abs(f64(x)) if has["x"] else None,
                           np.abs(f64(gate)) if has["gate"] else None, seq)
        assert out.dtype == x.dtype
        bound = (k + 3) * 2.0 ** -23 * big + HALF[dtype] * (np.abs(want) + (k + 3) * 2.0 ** -23 * big)
        assert (np.abs(f64(out) - want) <= bound).all()
        if norms is not None:
            assert (np.abs(f64(norms) - wn) <= (D + 4) * 2.0 ** -24 * wn).all()


def test_combine_in_place_and_unaligned(M):
    c, h = filled(M, 3, 700, 130, "e4m3")
    rows = torch.randint(0, 700, (350, 2), dtype=torch.int32, device="cuda")
    buf = activations(1, 350, 141)
    x = buf[:, 5:135]
    want, _ = O.combine(h, rows.cpu().numpy(), None, f64(x))
    left, right = buf[:, :5].clone(), buf[:, 135:].clone()
    out = M.q8_combine(c, rows, x=x, out=x)
    assert out is x
    np.testing.assert_allclose(f64(x), want, rtol=2 ** -20, atol=1e-4)
    assert torch.equal(buf[:, :5], left) and torch.equal(buf[:, 135:], right)


def test_an_empty_slot_takes_no_weight(M):
    """A weight of NaN or infinity on a slot that holds nothing changes nothing; NaN rows stay in their tokens."""
    c, h = filled(M, 3, 8, 256, "e5m2")
    c.q.view(torch.uint8)[2] = 0x7f
    x = activations(2, 3, 256)
    rows = ints([[0, -1], [99, -7], [2, 1]])
    w = torch.tensor([[0.5, float("nan")], [float("inf"), 1.0], [1.0, 1.0]], device="cuda")
    out, norms = M.q8_combine(c, rows, w, x=x, norms=True)
    np.testing.assert_allclose(f64(out[0]), f64(x[0]) + 0.5 * h[0], rtol=2 ** -22, atol=1e-5)
    assert torch.equal(out[1], x[1]) and bool(out[2].isnan().all())
    assert norms[0, 1] == 0 and norms[1].tolist() == [0, 0] and bool(norms[2, 0].isnan()) and norms[2, 1] > 0


# --- matmul ------------------------------------------------------------------

def check_rows(got, scale, z, err, fmt):
    """8-bit rows `got` (float64 grid values) with scale exponents against results z known within err."""
    n, width = z.shape
    step = np.ldexp(1.0, scale)[:, np.arange(width) // O.BLOCK]
    most, _, least, _ = O.FORMATS[fmt]
    digits = O.FORMATS[fmt][1]
    half = np.maximum(HALF[fmt] * (np.abs(z) + err), step * 2.0 ** (least - digits - 1))
    assert (np.abs(got * step - z) <= err + half).all()
    for b in range(scale.shape[1]):  # the scale holds the block's largest value, and half of it would not
        s = slice(b * O.BLOCK, (b + 1) * O.BLOCK)
        top, off = np.abs(z[:, s]).max(1), err[:, s].max(1)
        sc = np.ldexp(1.0, scale[:, b])
        assert (top <= most * sc + off).all()
        assert ((top + off >= most * sc / 2) | (scale[:, b] == -127) | (top <= off)).all()


def run_matmul(M, sizes, N, K, a_fmt="e4m3", b_fmt="e4m3", out="bf16", act="none", bias=False, dst=False, lead=0, tail=0,
               seed=0):
    """One product against the oracle; `lead` / `tail` rows of a stand before / behind the groups."""
    rng = np.random.default_rng(seed + 1)
    G, rows = len(sizes), lead + sum(sizes) + tail
    a, av = filled(M, seed + 2, rows, K, a_fmt)
    b, bv = filled(M, seed + 3, G * N, K, b_fmt)
    off = lead + np.concatenate([[0], np.cumsum(sizes)])
    bi = rng.standard_normal((G, N)).astype(np.float32) if bias else None
    bt = torch.from_numpy(bi).cuda() if bias else None
    out_rows = rows + 5 if dst else rows
    to = np.arange(rows)
    if dst:
        to = rng.permutation(out_rows)[:rows]
        to[rng.random(rows) < 0.1] = rng.choice([-1, out_rows, 1 << 30])
    if out in TYPES:
        o, _ = filled(M, seed + 4, out_rows, N, out)
        before = (o.q.view(torch.uint8).clone(), o.scale.clone())
    else:
        o = torch.full((out_rows, N), 7.0, dtype=VALUES[out], device="cuda")
    use_off = not (G == 1 and lead == 0 and tail == 0)
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    r = M.q8_matmul(a, b, offsets=ints(off.tolist()) if use_off else None, bias=bt, act=act,
                    dst=ints(to.tolist()) if dst else None, out=o, status=status)
    assert r is o and status.tolist() == [0, 0]
    z, done, big = O.matmul(av, bv, off, N, bi, act)
    err = 1.13 * (K + 2) * 2.0 ** -23 * big + 2.0 ** -21 * np.abs(z)
    at = to[done]
    live = (at >= 0) & (at < out_rows)
    z, err, at = z[done][live], err[done][live], at[live]
    rest = np.setdiff1d(np.arange(out_rows), at)
    if out in TYPES:
        check_rows(f64(o.q)[at], exps(o.scale)[at], z, err, out)
        assert torch.equal(o.q.view(torch.uint8)[rest], before[0][rest]) and torch.equal(o.scale[rest], before[1][rest])
        if out_rows > 1:  # the bytes past the rows' widths stay as they were
            pad = o.q.view(torch.uint8).as_strided((out_rows, o.q.stride(0)), (o.q.stride(0), 1))[:, N:]
            spad = o.scale.as_strided((out_rows, o.scale.stride(0)), (o.scale.stride(0), 1))[:, o.scale.shape[1]:]
            assert bool((pad == 0x7f).all()) and bool((spad == 0xff).all())
    else:
        assert (np.abs(f64(o)[at] - z) <= err + HALF[out] * (np.abs(z) + err)).all()
        assert bool((o[rest] == 7).all())


SHAPES = [  # rows of each group, columns, inner
    ([1], 1, 1), ([1], 128, 128), ([2], 130, 127), ([5], 77, 129), ([1], 1152, 1152), ([8], 300, 1000), ([9], 264, 520),
    ([33], 256, 64), ([64], 1000, 513), ([128], 384, 384), ([200], 129, 640), ([257], 513, 1024), ([700], 768, 256),
    ([1, 1], 200, 300), ([1, 0, 3, 0], 96, 130), ([0, 0, 0], 64, 64), ([31, 32, 33, 1, 64], 256, 1152),
    ([130, 0, 300, 7], 250, 700), ([3] * 40, 64, 200), ([193, 385, 96], 640, 2000),
    ([3, 40], 20, 70001),
]


@pytest.mark.parametrize("sizes,N,K", SHAPES, ids=str)
def test_matmul_shapes(M, sizes, N, K):
    run_matmul(M, sizes, N, K)
    run_matmul(M, sizes, N, K, out="e4m3", act="gelu", bias=True, dst=True)
    run_matmul(M, sizes, N, K, out="f32", a_fmt="e5m2", bias=True, lead=3, tail=6)


@pytest.mark.parametrize("a_fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("b_fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("out", ["bf16", "f32", "e4m3", "e5m2"])
@pytest.mark.parametrize("act", ["none", "gelu", "gelu_tanh"])
def test_matmul_types(M, a_fmt, b_fmt, out, act):
    run_matmul(M, [70, 3, 129], 300, 400, a_fmt, b_fmt, out, act, bias=True)
    run_matmul(M, [2, 0, 3], 300, 400, a_fmt, b_fmt, out, act, dst=True)
    run_matmul(M, [130], 256, 4700, a_fmt, b_fmt, out, act)


@pytest.mark.parametrize("rows", [2, 200])
def test_matmul_scales_far_apart(M, rows):
    """Block scales from 2^-30 to 2^30 within a row: each block counts with its own."""
    K, N = 1300, 160
    a, av = filled(M, 1, rows, K, "e4m3")
    b, bv = filled(M, 2, N, K, "e4m3")
    rng = np.random.default_rng(0)
    ea, eb = rng.integers(-30, 31, a.scale.shape), rng.integers(-30, 31, b.scale.shape)
    for c, e in ((a, ea), (b, eb)):
        c.scale.copy_(torch.from_numpy((e + 127).astype(np.uint8)))
    av, bv = O.dequantise(f64(a.q), ea), O.dequantise(f64(b.q), eb)
    out = M.q8_matmul(a, b, dtype=torch.float32)
    z, _, big = O.matmul(av, bv, [0, rows], N)
    assert (np.abs(f64(out) - z) <= (K + 2) * 2.0 ** -23 * big + 2.0 ** -24 * np.abs(z)).all()


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh"])
def test_matmul_activation_far_out(M, act):
    """GELU from -40 to 40: within 8 x 2^-24 |z| of the function, zero where 1 + tanh and 1 + erf vanish in fp32; an
    8-bit block of such values has the scale of zeros."""
    z = torch.linspace(-40, 40, 641, device="cuda")
    a = M.q8_write(torch.zeros(1, 1, device="cuda"), M.q8_empty(1, 1))
    b = M.q8_empty(641, 1)
    got = f64(M.q8_matmul(a, b, bias=z[None], act=act, dtype=torch.float32))[0]
    z64 = f64(z)
    assert (np.abs(got - O.gelu(z64, act == "gelu_tanh")) <= 2.0 ** -21 * np.abs(z64)).all()
    assert (got[z64 < -6.5] == 0).all() and (got[z64 > 6.5] == z64[z64 > 6.5]).all()
    low = torch.full((1, 130), -9.0, device="cuda")
    low[0, 0] = 1.0
    q = M.q8_matmul(a, M.q8_empty(130, 1), bias=low, act=act, dtype=torch.float8_e5m2)
    assert exps(q.scale).tolist() == [[-16, 0]] and bool((q.q[:, 1:].float() == 0).all())


@pytest.mark.parametrize("rows", [3, 150])
@pytest.mark.parametrize("ea,eb", [(-70, -62), (-70, -70), (61, 60), (62, 62)])
def test_matmul_tiny_and_huge_results(M, rows, ea, eb):
    """Results among fp32's subnormals keep their digits; past its largest value they are infinite, NaN in e4m3."""
    a, _ = filled(M, 1, rows, 256, "e4m3")
    b, _ = filled(M, 2, 96, 256, "e4m3")
    for c, e in ((a, ea), (b, eb)):
        c.scale.copy_(torch.full(c.scale.shape, 127 + e, dtype=torch.uint8))
    z, _, big = O.matmul(O.dequantise(f64(a.q), exps(a.scale)), O.dequantise(f64(b.q), exps(b.scale)), [0, rows], 96)
    err = 258 * 2.0 ** -23 * big + 2.0 ** -148  # and a few steps of the subnormals
    got = f64(M.q8_matmul(a, b, dtype=torch.float32))
    most = float(np.finfo(np.float32).max)
    over = np.abs(z) > most * (1 + 2.0 ** -10)
    fine = (np.abs(z) < most * (1 - 2.0 ** -10)) & (big < most)
    assert np.isinf(got[over]).all() and (np.abs(got[fine] - z[fine]) <= err[fine]).all()
    q = M.q8_matmul(a, b, dtype=torch.float8_e4m3fn)
    if over.any():
        assert np.isnan(f64(q.q)[over]).all()
        assert not np.isnan(f64(q.q)[fine]).any()
    else:
        check_rows(f64(q.q), exps(q.scale), z, err, "e4m3")


@pytest.mark.parametrize("rows", [3, 150])
def test_matmul_non_finite_rows_stay_apart(M, rows):
    """A row of NaN, a NaN scale and an infinity reach their own results only."""
    a, av = filled(M, 1, rows, 260, "e5m2")
    b, bv = filled(M, 2, 140, 260, "e4m3")
    a.q.view(torch.uint8)[1] = 0x7f
    a.scale[2, 1] = 255
    b.q.view(torch.uint8)[139, 5] = 0x7f
    out = M.q8_matmul(a, b, dtype=torch.float32)
    q = M.q8_matmul(a, b, dtype=torch.float8_e4m3fn)
    assert bool(out[1:3].isnan().all()) and bool(out[:, 139].isnan().all())
    keep = [r for r in range(rows) if r not in (1, 2)]
    z, _, big = O.matmul(av, bv, [0, rows], 140)
    assert (np.abs(f64(out)[keep, :139] - z[keep, :139]) <= 262 * 2.0 ** -23 * big[keep, :139]).all()
    v = f64(M.q8_read(q, dtype=torch.float32))
    assert np.isnan(v[1:3]).all() and np.isnan(v[:, 139]).all() and np.isfinite(v[keep][:, :139]).all()


@pytest.mark.parametrize("rows", [4, 300])
def test_matmul_bad_offsets(M, rows):
    """Offsets past the rows are clamped, a group that ends before it starts is empty."""
    N, K = 72, 256
    a, av = filled(M, 1, rows, K, "e4m3")
    b, bv = filled(M, 2, 4 * N, K, "e4m3")
    for off in ([-5, 2, 1, 3, 1 << 30], [2, 2, 2, 2, 2], [rows, 0, 0, 0, 2], [0, 0, -3, rows + 9, rows]):
        out = torch.full((rows, N), 7.0, device="cuda")
        M.q8_matmul(a, b, offsets=ints(off), out=out)
        cl = np.clip(off, 0, rows)
        claims = np.zeros(rows, int)
        for g in range(4):
            claims[cl[g]:cl[g + 1]] += 1
        z, done, big = O.matmul(av, bv, off, N)
        one = claims == 1
        assert (np.abs(f64(out)[one] - z[one]) <= (K + 2) * 2.0 ** -23 * big[one] + 2.0 ** -24 * np.abs(z[one])).all()
        assert bool((out[torch.from_numpy(claims == 0).cuda()] == 7).all())


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [3, 140])
def test_matmul_into_strided_rows(M, out, rows):
    a, av = filled(M, 1, rows, 256, "e4m3")
    b, bv = filled(M, 2, 131, 256, "e4m3")
    buf = torch.full((rows, 151), 7.0, dtype=VALUES[out], device="cuda")
    M.q8_matmul(a, b, out=buf[:, 9:140])
    z, _, big = O.matmul(av, bv, [0, rows], 131)
    err = 258 * 2.0 ** -23 * big
    assert (np.abs(f64(buf[:, 9:140]) - z) <= err + HALF[out] * (np.abs(z) + err)).all()
    assert bool((buf[:, :9] == 7).all()) and bool((buf[:, 140:] == 7).all())


# --- together ----------------------------------------------------------------

def expert_layer(M, s):
    """The layer's branches at 8 bits: rows gathered and quantised by list, both expert products, the branch outputs
    written into their cache slots, Eq. 8."""
    M.q8_write(s["x"], s["rows8"], src=s["token"])
    M.q8_matmul(s["rows8"], s["w1"], offsets=s["offsets"], act="gelu_tanh", out=s["hidden"])
    M.q8_matmul(s["hidden"], s["w2"], offsets=s["offsets"], dst=s["slot"], out=s["cache"])
    return M.q8_combine(s["cache"], s["slot_rows"], s["weight"], x=s["x"], norms=True)


def layer_state(M, seed, T=150, k=2, E=4, D=256, F=520):
    rng = np.random.default_rng(seed)
    experts = np.stack([rng.permutation(E)[:k] for _ in range(T)])
    order = np.argsort(experts.reshape(-1), kind="stable")  # branches, one expert's after another's
    s = dict(x=activations(seed, T, D), token=ints((order // k).tolist()), slot=ints(order.tolist()),
             offsets=ints(np.concatenate([[0], np.cumsum(np.bincount(experts.reshape(-1), minlength=E))]).tolist()),
             slot_rows=torch.arange(T * k, dtype=torch.int32, device="cuda").view(T, k),
             weight=torch.from_numpy(rng.random((T, k)).astype(np.float32)).cuda(),
             w1f=activations(seed + 1, E * F, D) / 16, w2f=activations(seed + 2, E * D, F) / 16,
             rows8=M.q8_empty(T * k, D), hidden=M.q8_empty(T * k, F), cache=M.q8_empty(T * k, D, torch.float8_e5m2))
    s["w1"], s["w2"] = M.q8_write(s["w1f"], M.q8_empty(E * F, D)), M.q8_write(s["w2f"], M.q8_empty(E * D, F))
    s["experts"], s["dims"] = experts, (T, k, E, D, F)
    return s


def test_expert_layer_runs_together(M):
    s = layer_state(M, 3)
    out, norms = expert_layer(M, s)
    T, k, E, D, F = s["dims"]
    # Each stage against the oracle on the stage's own stored inputs.
    xq, xe = O.quantise(f64(s["x"])[f64(s["token"]).astype(int)], "e4m3")
    np.testing.assert_array_equal(f64(s["rows8"].q), xq)
    off = s["offsets"].cpu().numpy()
    w1, w2 = O.dequantise(f64(s["w1"].q), exps(s["w1"].scale)), O.dequantise(f64(s["w2"].q), exps(s["w2"].scale))
    z, done, big = O.matmul(O.dequantise(xq, xe), w1, off, F, act="gelu_tanh")
    assert done.all()
    check_rows(f64(s["hidden"].q), exps(s["hidden"].scale), z, 1.13 * (D + 2) * 2.0 ** -23 * big + 2.0 ** -21 * np.abs(z), "e4m3")
    hid = O.dequantise(f64(s["hidden"].q), exps(s["hidden"].scale))
    z, _, big = O.matmul(hid, w2, off, D)
    slot = s["slot"].cpu().numpy()
    check_rows(f64(s["cache"].q)[slot], exps(s["cache"].scale)[slot], z, (F + 2) * 2.0 ** -23 * big, "e5m2")
    h = O.dequantise(f64(s["cache"].q), exps(s["cache"].scale))
    want, wn = O.combine(h, s["slot_rows"].cpu().numpy(), f64(s["weight"]), f64(s["x"]))
    np.testing.assert_allclose(f64(out), want, rtol=2 ** -20, atol=2 ** -20 * np.abs(want).max())
    np.testing.assert_allclose(f64(norms), wn, rtol=2 ** -14)
    # And against the layer in float64 without 8-bit storage: roundings of 2^-4 (e4m3) and 2^-3 (e5m2) at most in
    # four places, independent of one another, stay within their sum.
    x = f64(s["x"])
    w1, w2 = f64(s["w1f"]).reshape(E, F, D), f64(s["w2f"]).reshape(E, D, F)
    full = x.copy()
    for e in range(E):
        t, p = np.nonzero(s["experts"] == e)
        full[t] += f64(s["weight"])[t, p][:, None] * (O.gelu(x[t] @ w1[e].T, True) @ w2[e].T)
    rel = np.linalg.norm(f64(out) - full) / np.linalg.norm(full - x)
    assert rel < 4 * 2.0 ** -4 + 2.0 ** -3


def test_graph_replays_follow_their_inputs(M):
    s = layer_state(M, 3)
    want0 = [t.clone() for t in expert_layer(M, s)]
    x1 = activations(77, *s["x"].shape)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        expert_layer(M, s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            got = expert_layer(M, s)
    torch.cuda.current_stream().wait_stream(side)
    g.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, want0))
    x0 = s["x"].clone()
    s["x"].copy_(x1)
    g.replay()
    first = [t.clone() for t in got]
    eager = expert_layer(M, s)
    assert all(torch.equal(a, b) for a, b in zip(first, eager)) and not torch.equal(first[0], want0[0])
    s["x"].copy_(x0)
    g.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, want0))


def test_two_streams_at_once(M):
    """Calls on two streams share nothing: each gives the bits it gives alone."""
    states = [layer_state(M, 5, T=600, D=512, F=1024), layer_state(M, 6, T=500, E=8, D=384, F=640)]
    alone = [[t.clone() for t in expert_layer(M, s)] for s in states]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in states]
    for _ in range(20):
        got = []
        for s, st in zip(states, streams):
            with torch.cuda.stream(st):
                got.append(expert_layer(M, s))
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_two_host_threads_at_once(M):
    """Host threads that call at the same time, each on its own stream, get the bits of calls alone."""
    import threading
    states = [layer_state(M, 7, T=300, D=256, F=520), layer_state(M, 8, T=260, E=8, D=384, F=640)]
    alone = [[t.clone() for t in expert_layer(M, s)] for s in states]
    torch.cuda.synchronize()
    wrong = []

    def work(s, want):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(25):
                got = expert_layer(M, s)
                stream.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want)):
                    wrong.append(1)

    threads = [threading.Thread(target=work, args=p) for p in zip(states, alone)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_repeats_give_the_same_bits(M):
    a, _ = filled(M, 1, 777, 1500, "e4m3")
    b, _ = filled(M, 2, 3 * 500, 1500, "e4m3")
    off = ints([0, 100, 101, 777])
    first = M.q8_matmul(a, b, off, dtype=torch.float32)
    for _ in range(5):
        assert torch.equal(M.q8_matmul(a, b, off, dtype=torch.float32), first)
    for n in (1, 4, 8):
        part = M.Q8(a.q[:n], a.scale[:n])
        one = M.q8_matmul(part, M.Q8(b.q[:500], b.scale[:500]), dtype=torch.float32)
        assert torch.equal(one, M.q8_matmul(part, M.Q8(b.q[:500], b.scale[:500]), dtype=torch.float32))


# --- sizes and paths at the edges --------------------------------------------

@pytest.mark.parametrize("T,k,D", [(400, 9, 2600), (310, 16, 9000), (305, 2, 30001), (320, 3, 8), (5000, 2, 24)])
@pytest.mark.parametrize("off", [0, 1])
def test_combine_wide_and_narrow_rows(M, T, k, D, off):
    """Rows that fit no shared-memory buffer, and many tokens of a few values; aligned and not."""
    rng = np.random.default_rng(D)
    c, h = filled(M, 5, 700, D, "e4m3")
    rows = rng.integers(-2, 700, (T, k)).astype(np.int32)
    w = rng.standard_normal((T, k)).astype(np.float32)
    x = activations(3, T, D + off, "bf16")[:, off:]
    out = torch.full((T, D + 3 * off), 9.0, dtype=torch.bfloat16, device="cuda")
    got, norms = M.q8_combine(c, torch.from_numpy(rows).cuda(), torch.from_numpy(w).cuda(), x=x,
                              out=out[:, 2 * off:2 * off + D], norms=True)
    want, wn = O.combine(h, rows, w, f64(x))
    big, _ = O.combine(np.abs(h), rows, np.abs(w), np.abs(f64(x)))
    err = (k + 3) * 2.0 ** -23 * big
    assert (np.abs(f64(got) - want) <= err + HALF["bf16"] * (np.abs(want) + err)).all()
    assert (np.abs(f64(norms) - wn) <= (D + 4) * 2.0 ** -24 * wn).all()
    assert bool((out[:, :2 * off] == 9).all()) and bool((out[:, 2 * off + D:] == 9).all())


def test_offsets_past_32_bits(M):
    """Rows whose bytes lie past 2^32: written, read back, combined, multiplied, scattered."""
    rows, D = 4_200_000, 1024
    c = M.Q8(torch.empty((rows, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn),
             torch.empty((rows, 8), dtype=torch.uint8, device="cuda"))
    at = [rows - 1, 5, rows - 400, 4_194_304, 4_194_303, 17]
    x = activations(1, 6, D, "bf16")
    M.q8_write(x, c, dst=ints(at))
    same(c, x, "e4m3", at)
    q, e = O.quantise(f64(x), "e4m3")
    h = O.dequantise(q, e)
    np.testing.assert_array_equal(f64(M.q8_read(c, ints(at), dtype=torch.float32)), h)
    for many in (1, 60):  # both forms of the kernel
        got = M.q8_combine(c, ints([at] * many), dtype=torch.float32)
        np.testing.assert_allclose(f64(got), np.repeat(h.sum(0)[None], many, 0), rtol=2 ** -20, atol=2 ** -18 * np.abs(h).max())
    got = M.q8_read(c, ints(at * 60), dtype=torch.float32)
    np.testing.assert_array_equal(f64(got), np.tile(h, (60, 1)))
    b, bv = filled(M, 2, 1024, D, "e4m3")
    small = M.q8_write(x, M.q8_empty(6, D))
    z, _, big = O.matmul(h, bv, [0, 6], 1024)
    check = lambda v: (np.abs(v - z) <= (D + 2) * 2.0 ** -23 * big + HALF["bf16"] * np.abs(z)).all()  # noqa: E731
    tail = M.Q8(c.q[rows - 400:], c.scale[rows - 400:])  # a's own rows far into memory
    a_all = M.q8_matmul(tail, b, dtype=torch.float32)
    assert check(np.stack([f64(a_all[399]), f64(M.q8_matmul(small, b, dtype=torch.float32))[1], f64(a_all[0]),
                           *[f64(M.q8_matmul(small, b, dtype=torch.float32))[i] for i in (3, 4, 5)]]))
    out = c.q.view(torch.bfloat16)[:, :512]  # 8.6 GB seen as bf16 rows of half a width
    b2 = M.Q8(b.q[:512], b.scale[:512])
    M.q8_matmul(small, b2, dst=ints(at), out=out)
    assert (np.abs(f64(out[torch.tensor(at)]) - z[:, :512]) <= (D + 2) * 2.0 ** -23 * big[:, :512]
            + HALF["bf16"] * (np.abs(z[:, :512]) + 1e-30)).all()


def test_matmul_many_groups_and_tiles(M):
    """512 groups, most of a single row, one large; every tile width of a group's rows."""
    rng = np.random.default_rng(0)
    sizes = rng.integers(0, 3, 511).tolist() + [900]
    run_matmul(M, sizes, 40, 96)
    run_matmul(M, list(range(1, 60, 3)) + [100, 150, 223, 224, 225, 230, 448, 449], 130, 160, out="e4m3", bias=True)


def test_first_call_of_a_process_may_be_captured(M):
    """A captured call needs no eager one before it."""
    import subprocess
    import sys
    from pathlib import Path
    code = """
import torch
from paper_2606_15615_gb300 import moeca as M
x = torch.randn(40, 256, device="cuda")
rows8, out8, big = M.q8_empty(40, 256), M.q8_empty(40, 128), M.q8_empty(700, 256)
w = M.q8_empty(128, 256)
rows = torch.zeros(600, 2, dtype=torch.int32, device="cuda")
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    M.q8_write(x, rows8)
    M.q8_write(torch.ones_like(x), w, src=torch.zeros(128, dtype=torch.int32, device="cuda"))
    M.q8_matmul(rows8, w, out=out8)
    y = M.q8_read(out8, dtype=torch.float32)
    z = M.q8_combine(rows8, rows, dtype=torch.float32)
g.replay()
torch.cuda.synchronize()
want = M.q8_read(rows8, dtype=torch.float32)
assert torch.allclose(y, want.sum(1, keepdim=True).expand(-1, 128), rtol=0.07, atol=1e-3)
assert torch.allclose(z, 2 * want[:1].expand(600, -1))
"""
    root = Path(__file__).resolve().parents[1]
    subprocess.run([sys.executable, "-c", code], check=True, cwd=root, timeout=300)


def test_stack_snapshot_in_8_bits(M):
    """A stack's state with its branch outputs in 8 bits: half the bytes, and a resumed trajectory whose reused
    branches are off by the format's rounding."""
    from paper_2606_15615_gb300 import workloads as W
    T, D, E, k, F = 256, 128, 8, 2, 256
    w = W.tiny_layer(41, T, D, E, k, F, dtype="bf16", wscale=0.05)[0]
    cfg = M.moeca_config_default(n_layers=1, hidden=D, ffn=F, n_experts=E, top_k=k, max_tokens=T, tau0=0.75)
    x = torch.randn(T, D, device="cuda").bfloat16()
    x2 = (x.float() + 0.05 * torch.randn_like(x.float())).bfloat16()
    s = M.Stack(cfg, [w])
    s.step(x, 1)
    exact, small = s.get_state(0), s.get_state(0, q8=torch.float8_e4m3fn)
    assert isinstance(small["cache_h"], M.Q8) and small["cache_h"].q.shape == (T * k, D)
    same(small["cache_h"], exact["cache_h"].reshape(T * k, D), "e4m3")
    assert torch.equal(small["cache_norm"], exact["cache_norm"]) and torch.equal(small["ema"], exact["ema"])
    want = s.step(x2, 1)
    s.set_state(0, small)
    back = s.get_state(0)
    h = M.q8_read(small["cache_h"]).view(T, k, D)
    assert torch.equal(back["cache_h"], h) and torch.equal(back["cache_e"], exact["cache_e"])
    got = s.step(x2, 1)
    st = s.stats()
    assert st["device_status"] == 0 and st["reused"] > 0
    # Decisions read norms and weights, which are exact: only reused rows differ, by at most half a step of each.
    tr = s.get_trace(0, T)
    reused = (tr["recompute"] == 0).double()
    bound = (reused * tr["route_w"].double()).sum(1, keepdim=True) * 2.0 ** -4 * exact["cache_h"].double().abs().amax((1, 2))[:, None]
    assert bool(((got.double() - want.double()).abs() <= bound + 2.0 ** -7 * want.double().abs()).all())
    s.close()
