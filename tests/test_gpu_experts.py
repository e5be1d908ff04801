"""Tokens sorted by expert and back, with gradients, on the GPU against plain 64-bit results.

Tolerances.  The sort and the copies are exact.  A sum of n products in fp32 in any order is off by at most
n 2^-23 times the sum of the magnitudes, a product rounded to fp32 by 2^-24 of itself; a result in bf16 / fp32 by
2^-8 / 2^-24 of itself (bf16: or half its least subnormal, 2^-134).
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


def ids(seed, T, k, E, empty=0.0, skew=0.0):
    rng = np.random.default_rng(seed)
    p = np.exp(skew * rng.standard_normal(E))
    x = rng.choice(E, size=(T, k), p=p / p.sum())
    bad = rng.choice([-1, -7, E, E + 5, 2 ** 31 - 1, -2 ** 31], size=(T, k))
    return np.where(rng.random((T, k)) < empty, bad, x).astype(np.int32)


def sorted_plan(x, E):
    flat = x.reshape(-1)
    keep = np.flatnonzero((flat >= 0) & (flat < E))
    slot = keep[np.argsort(flat[keep], kind="stable")]
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[keep], minlength=E))])
    place = np.full(flat.size, -1)
    place[slot] = np.arange(slot.size)
    full = np.full(flat.size, -1)
    full[:slot.size] = slot
    return offsets, place.reshape(x.shape), full, np.where(full >= 0, full // x.shape[1], -1)


def check_plan(plan, x, E):
    for got, want, name in zip(plan, sorted_plan(x, E), ("offsets", "place", "slot", "token")):
        np.testing.assert_array_equal(got.cpu().numpy(), want, err_msg=name)


SORTS = [(0, 2, 4), (1, 1, 1), (1, 2, 16), (3, 16, 5), (31, 1, 7), (32, 1, 512), (33, 2, 512), (257, 3, 37), (1024, 8, 64),
         (4096, 2, 16), (4097, 2, 16), (4096, 3, 400), (8193, 1, 2), (20011, 3, 129), (32768, 8, 64), (70001, 5, 512)]


@pytest.mark.parametrize("empty", [0.0, 0.3, 1.0])
@pytest.mark.parametrize("T,k,E", SORTS)
def test_sort(M, T, k, E, empty):
    x = ids(T + E, T, k, E, empty, skew=1.0)
    check_plan(M.expert_sort(torch.from_numpy(x).cuda(), E), x, E)


@pytest.mark.parametrize("T,k", [(5000, 1), (9000, 2), (300_000, 1)])
def test_sort_of_one_expert(M, T, k):
    x = np.full((T, k), 6, np.int32)
    check_plan(M.expert_sort(torch.from_numpy(x).cuda(), 9), x, 9)


def test_sort_writes_given_lists_only(M):
    x = ids(1, 700, 3, 20, 0.2)
    buf = torch.full((4, 4000), -77, dtype=torch.int32, device="cuda")
    plan = M.ExpertPlan(buf[0, 8:29], buf[1, 8:2108].view(700, 3), buf[2, 8:2108], buf[3, 8:2108])
    assert M.expert_sort(torch.from_numpy(x).cuda(), 20, plan=plan) is plan
    check_plan(plan, x, 20)
    assert bool((buf[:, :8] == -77).all()) and bool((buf[0, 29:] == -77).all()) and bool((buf[1:, 2108:] == -77).all())


def values(seed, n, width, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, width, generator=g) * torch.exp(torch.randn(n, 1, generator=g)) * scale
    return x.to(TYPES[dtype]).cuda()


def strided(x, pad, base, fill=7.0):
    """x's values in rows `pad` values further apart, from value `base` of a buffer on; and that buffer."""
    n, width = x.shape
    buf = torch.full((base + n * (width + pad) + 16,), fill, dtype=x.dtype, device="cuda")
    v = buf.as_strided((n, width), (width + pad, 1), base)
    v.copy_(x)
    return v, buf


def f64(t):
    return t.detach().double().cpu().numpy()


def close(got, want, slack, dtype):
    err = np.abs(f64(got) - want)
    tol = slack + HALF[dtype] * (np.abs(want) + slack) + 2.0 ** -134
    assert (err <= tol).all(), float((err - tol).max())


# tokens, slots, experts, width, share of branches that are not sorted
ROWS = [(1, 1, 1, 1, 0.0), (1, 2, 16, 1152, 0.0), (2, 3, 4, 7, 0.5), (5, 16, 9, 130, 0.3), (64, 2, 4, 8, 0.0), (33, 4, 8, 1001, 0.2),
        (300, 2, 16, 768, 0.0), (257, 5, 37, 1000, 1.0), (1000, 8, 64, 65, 0.1), (41, 1, 3, 5000, 0.2), (2050, 2, 16, 1152, 0.0)]
LAYOUTS = [(0, 0), (8, 0), (3, 1), (1, 3), (0, 5)]


@pytest.mark.parametrize("pad,base", LAYOUTS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,E,D,empty", ROWS)
def test_rows(M, T, k, E, D, empty, dtype, pad, base):
    e = ids(T + D, T, k, E, empty)
    plan = M.expert_sort(torch.from_numpy(e).cuda(), E)
    x, _ = strided(values(D, T, D, dtype), pad, base)
    used = int(plan.offsets[-1])
    token = plan.token[:used].long()
    want = x[token]
    new = M.expert_rows(x, plan)
    assert new.shape == (T * k, D) and torch.equal(new[:used], want) and bool((new[used:] == 0).all())
    out, buf = strided(torch.full((T * k, D), 3.0, dtype=TYPES[dtype], device="cuda"), pad, (base * 3) % 7)
    before = buf.clone()
    assert M.expert_rows(x, plan, out=out) is out
    assert torch.equal(out[:used], want)
    out.copy_(torch.full_like(out, 3.0))
    assert torch.equal(buf, before)  # rows behind the last and what lies between rows


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_take_any_values(M, dtype):
    x = values(1, 40, 24, dtype)
    x[3, 5], x[4, 6], x[5] = float("nan"), float("inf"), -float("inf")
    plan = M.expert_sort(torch.arange(40, dtype=torch.int32, device="cuda")[:, None] % 3, 3)
    got = M.expert_rows(x, plan)
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(got.view(bits), x[plan.token.long()].view(bits))


@pytest.mark.parametrize("pad,base", LAYOUTS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,E,D,empty", ROWS)
def test_combine_and_gradients(M, T, k, E, D, empty, dtype, pad, base):
    e = ids(T + D + 1, T, k, E, empty)
    plan = M.expert_sort(torch.from_numpy(e).cuda(), E)
    used = int(plan.offsets[-1])
    place = plan.place.cpu().numpy()
    live = place >= 0
    rows = values(D + 1, T * k, D, dtype)
    rows[used:] = float("nan")  # behind the last row nothing is read
    rows, _ = strided(rows, pad, base)
    x, _ = strided(values(D + 2, T, D, dtype), pad, base)
    w = torch.randn(T, k, generator=torch.Generator().manual_seed(D)).cuda()
    w64 = f64(w)
    h = np.where(live[..., None], f64(rows)[np.maximum(place, 0)], 0.0)
    terms = w64[..., None] * h
    want = terms.sum(1)
    slack = (k + 1) * 2.0 ** -23 * (np.abs(terms).sum(1) + np.abs(f64(x)))
    close(M.expert_combine(rows, plan, w, x=x), f64(x) + want, slack, dtype)
    close(M.expert_combine(rows, plan, w), want, slack, dtype)
    close(M.expert_combine(rows, plan), h.sum(1), k * 2.0 ** -23 * np.abs(h).sum(1), dtype)
    own = x.clone()
    M.expert_combine(rows, plan, w, x=own, out=own)  # in place
    close(own, f64(x) + want, slack, dtype)
    out, buf = strided(x, pad, (base + 1) % 4)
    left = buf.clone()
    M.expert_combine(rows, plan, w, x=out, out=out)
    close(out, f64(x) + want, slack, dtype)
    out.copy_(x)
    assert torch.equal(buf, left)
    # Gradients.
    dy = x
    drows, dw = M.expert_combine_grad(dy, rows, plan, w)
    token = np.maximum(plan.token.cpu().numpy(), 0)
    slot = np.maximum(plan.slot.cpu().numpy(), 0)
    want_rows = np.where((np.arange(T * k) < used)[:, None], w64.reshape(-1)[slot][:, None] * f64(dy)[token], 0.0)
    close(drows, want_rows, 2.0 ** -24 * np.abs(want_rows), dtype)
    prod = f64(dy)[:, None] * h
    assert (np.abs(f64(dw) - prod.sum(-1)) <= (D + 1) * 2.0 ** -23 * np.abs(prod).sum(-1)).all()
    given, buf = strided(torch.full((T * k, D), 3.0, dtype=TYPES[dtype], device="cuda"), pad, (base * 3) % 5)
    left = buf.clone()
    got, none = M.expert_combine_grad(dy, rows, plan, w, drows=given, dweights=False)
    assert got is given and none is None
    close(given[:used], want_rows[:used], 2.0 ** -24 * np.abs(want_rows[:used]), dtype)
    given.copy_(torch.full_like(given, 3.0))
    assert torch.equal(buf, left)
    drows[used:] = float("nan")
    g = np.where(live[..., None], f64(drows)[np.maximum(place, 0)], 0.0)
    close(M.expert_rows_grad(drows, plan), g.sum(1), k * 2.0 ** -23 * np.abs(g).sum(1), dtype)


def test_empty_slots_add_nothing_whatever_their_weight(M):
    plan = M.expert_sort(torch.tensor([[0, -1], [-1, -1], [5, 1]], dtype=torch.int32, device="cuda"), 3)
    rows = torch.ones(6, 16, device="cuda")
    rows[2:] = float("nan")
    w = torch.tensor([[2.0, float("nan")], [float("inf"), float("nan")], [float("inf"), 3.0]], device="cuda")
    y = M.expert_combine(rows, plan, w)
    assert torch.equal(y[:, 0].cpu(), torch.tensor([2.0, 0.0, 3.0]))
    _, dw = M.expert_combine_grad(torch.ones(3, 16, device="cuda"), rows, plan, w)
    assert torch.equal(dw.cpu(), torch.tensor([[16.0, 0.0], [0.0, 0.0], [0.0, 16.0]]))


def test_gradients_agree_with_differences(M):
    """L = sum(c * combine(rows(x) * 1.5, w, x)): the calls' gradients against central differences of the calls."""
    T, k, E, D = 7, 3, 4, 12
    g = torch.Generator().manual_seed(3)
    plan = M.expert_sort(torch.from_numpy(ids(3, T, k, E, 0.2)).cuda(), E)
    x, c = (torch.randn(T, D, generator=g).cuda() for _ in range(2))
    w = torch.randn(T, k, generator=g).cuda()

    def loss(x, w):
        return float((c.double() * M.expert_combine(1.5 * M.expert_rows(x, plan), plan, w, x=x).double()).sum())

    rows = 1.5 * M.expert_rows(x, plan)
    drows, dw = M.expert_combine_grad(c, rows, plan, w)
    dx = c + M.expert_rows_grad(1.5 * drows, plan)
    h = 2.0 ** -6
    # L is linear in x and in w: the difference's own error is the roundings of L, below 200 terms of 10 x 2^-23 each.
    tol = 200 * 10 * 2.0 ** -23 / h
    for i in range(T):
        for j in range(k):
            e = torch.zeros_like(w)
            e[i, j] = h
            assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * h) - float(dw[i, j])) < tol
        for j in range(0, D, 5):
            e = torch.zeros_like(x)
            e[i, j] = h
            assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * h) - float(dx[i, j])) < tol


def test_captured_and_on_another_stream(M):
    T, k, E, D = 3000, 4, 32, 256
    a, b = (torch.from_numpy(ids(s, T, k, E, 0.1)).cuda() for s in (1, 2))
    x, w = values(1, T, D, "bf16"), torch.rand(T, k, device="cuda")

    def run(e):
        plan = M.expert_sort(e, E)
        rows = M.expert_rows(x, plan)
        y = M.expert_combine(rows, plan, w, x=x)
        return (*plan, rows, y, *M.expert_combine_grad(y, rows, plan, w))

    want = run(b)
    torch.cuda.synchronize()
    e = a.clone()
    graph = torch.cuda.CUDAGraph()
    run(e)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = run(e)
    e.copy_(b)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for u, v in zip(got, want):
        assert torch.equal(u, v)
    s = torch.cuda.Stream()
    raw = s.cuda_stream
    plan = M.expert_sort(b, E, stream=raw)
    rows = M.expert_rows(x, plan, stream=raw)
    y = M.expert_combine(rows, plan, w, x=x, stream=raw)
    drows, dw = M.expert_combine_grad(y, rows, plan, w, stream=raw)
    s.synchronize()
    for u, v in zip((*plan, rows, y, drows, dw), want):
        assert torch.equal(u, v)


def test_results_repeat(M):
    T, k, E, D = 20000, 6, 100, 200
    e = torch.from_numpy(ids(5, T, k, E, 0.1, skew=2.0)).cuda()
    x, w = values(2, T, D, "f32"), torch.rand(T, k, device="cuda")
    first = None
    for _ in range(4):
        plan = M.expert_sort(e, E)
        rows = M.expert_rows(x, plan)
        now = (*plan, rows, M.expert_combine(rows, plan, w), *M.expert_combine_grad(x, rows, plan, w))
        first = first or now
        assert all(torch.equal(u, v) for u, v in zip(first, now))


def test_rows_beyond_32_bits(M):
    """Rows 16400 values apart: the last lie 2.4e9 values into their buffer."""
    T, D, stride = 147_000, 24, 16_400
    e = torch.from_numpy(ids(9, T, 1, 3)).cuda()
    plan = M.expert_sort(e, 3)
    x, w = values(3, T, D, "bf16"), torch.rand(T, 1, device="cuda")
    want = M.expert_rows(x, plan)
    buf = torch.empty(T * stride, dtype=torch.bfloat16, device="cuda")
    far = buf.as_strided((T, D), (stride, 1), 0)
    assert torch.equal(M.expert_rows(x, plan, out=far), want)
    assert torch.equal(M.expert_combine(far, plan, w), M.expert_combine(want, plan, w))
    got, want = M.expert_combine_grad(x, far, plan, w), M.expert_combine_grad(x, want, plan, w)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    far.copy_(x)
    assert torch.equal(M.expert_rows(far, plan), M.expert_rows(x, plan))
