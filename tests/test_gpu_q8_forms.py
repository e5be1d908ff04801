"""Both forms of the 8-bit combine's kernel (staged in shared memory, direct), at sizes taken from the rule that
chooses between them, against the float64 oracle (tolerances: see tests/test_gpu_q8.py)."""
import threading

import numpy as np
import pytest
import torch

from oracle import q8 as O
from test_gpu_q8 import (HALF, M, TYPES, VALUES, activations, expert_layer, f64, filled, ints,  # noqa: F401
                         layer_state)

pytestmark = pytest.mark.gpu


def first_staged(M, k, width, dtype, residual=True, aligned=True):
    """The fewest tokens whose combine is staged on this device."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    staged = lambda T: M.moeca_probe_q8_staged(sms, T, k, width, M.MOECA_BF16 if dtype == "bf16" else M.MOECA_F32,  # noqa: E731
                                               residual, aligned)
    T = next((T for T in range(1, 16 * sms) if staged(T)), None)
    assert T is not None and all(staged(T + i) for i in (1, 7, 1000)) and not staged(1)
    return T


@pytest.fixture(scope="module")
def cache(M):
    """400 rows of each format and width, and their values."""
    made = {}

    def get(fmt, width):
        if (fmt, width) not in made:
            made[fmt, width] = filled(M, 3, 400, width, fmt)
        return made[fmt, width]
    return get


def slots(seed, T, k, R=400):
    """Lists of rows, some out of range, one token's all; and weights, also on what holds nothing."""
    rng = np.random.default_rng(seed)
    rows = rng.integers(0, R, (T, k)).astype(np.int32)
    rows[rng.random((T, k)) < 0.15] = rng.choice([-1, R, 1 << 30, -(1 << 31)])
    rows[T // 2] = -1
    return rows, rng.standard_normal((T, k)).astype(np.float32)


def check(got, h, rows, w, x, gate, seq, dtype):
    out, norms = got
    k, D = rows.shape[1], h.shape[1]
    want, wn = O.combine(h, rows, w, x, gate, seq)
    big, _ = O.combine(np.abs(h), rows, None if w is None else np.abs(w), None if x is None else np.abs(x),
                       None if gate is None else np.abs(gate), seq)
    err = (k + 3) * 2.0 ** -23 * big
    assert (np.abs(f64(out) - want) <= err + HALF[dtype] * (np.abs(want) + err)).all()
    assert (np.abs(f64(norms) - wn) <= (D + 4) * 2.0 ** -24 * wn).all()


@pytest.mark.parametrize("k", range(1, 17))
@pytest.mark.parametrize("D,unaligned", [(1152, 0), (1000, 0), (264, 4), (129, 1), (8, 0)])
def test_combine_on_both_sides_of_the_rule(M, cache, k, D, unaligned):
    """The last direct and the first staged count of tokens and some more: weights, residual and gate or not, in both
    types; the tokens that both calls have come out the same."""
    fmt, dtype = ("e4m3", "e5m2")[k % 2], ("bf16", "f32")[(k + D) % 2]
    c, h = cache(fmt, D)
    edge = first_staged(M, k, D, dtype, aligned=not unaligned)
    T = edge + 77
    rows, w = slots(k + D, T, k)
    seq = 31
    buf = activations(11, T, D + 2 * unaligned, dtype)
    x = buf[:, unaligned:unaligned + D]
    gate = torch.randn(-(-T // seq), D, generator=torch.Generator().manual_seed(k)).cuda()
    rt, wt = torch.from_numpy(rows).cuda(), torch.from_numpy(w).cuda()

    def run(n, weights, residual, gated):
        out = torch.full((n, D + 2 * unaligned), 9.0, dtype=VALUES[dtype], device="cuda")
        tokens = n // seq * seq if gated else n  # whole groups of the gate
        got = M.q8_combine(c, rt[:tokens], wt[:tokens] if weights else None, x=x[:tokens] if residual else None,
                           gate=gate[:tokens // seq] if gated else None, norms=True,
                           out=out[:tokens, unaligned:unaligned + D])
        assert bool((out[:, :unaligned] == 9).all()) and bool((out[:, unaligned + D:] == 9).all())
        assert bool((out[tokens:] == 9).all())
        return got

    for weights, residual, gated in ((1, 1, 1), (1, 1, 0), (0, 0, 1), (0, 0, 0)):
        many, few = run(T, weights, residual, gated), run(edge - 1, weights, residual, gated)
        n = len(many[0])
        check(many, h, rows[:n], w[:n].astype(np.float64) if weights else None, f64(x[:n]) if residual else None,
              f64(gate[:n // seq]) if gated else None, seq, dtype)
        assert torch.equal(few[0], many[0][:len(few[0])])
        check(few, h, rows[:len(few[0])], w[:len(few[0])].astype(np.float64) if weights else None,
              f64(x[:len(few[0])]) if residual else None, f64(gate[:len(few[0]) // seq]) if gated else None, seq, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k,D,at", [(2, 1152, 0), (2, 130, 5), (1, 1001, 1), (3, 2560, 0), (8, 200, 3)])
def test_combine_in_place_when_staged(M, cache, k, D, at, dtype):
    c, h = cache("e4m3", D)
    T = first_staged(M, k, D, dtype, aligned=at == 0) + 400
    rows, w = slots(k, T, k)
    buf = activations(1, T, D + 2 * at, dtype)
    x = buf[:, at:at + D]
    before, x64 = buf.clone(), f64(x)
    got = M.q8_combine(c, torch.from_numpy(rows).cuda(), torch.from_numpy(w).cuda(), x=x, out=x, norms=True)
    assert got[0] is x
    check(got, h, rows, w.astype(np.float64), x64, None, 1, dtype)
    assert torch.equal(buf[:, :at], before[:, :at]) and torch.equal(buf[:, at + D:], before[:, at + D:])


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,at", [(1152, 0), (1000, 0), (384, 8), (1153, 1), (129, 3), (17, 0), (1, 0)])
def test_reads_when_staged(M, cache, D, at, dtype, fmt):
    """By list, entries out of range, into rows that do not start at 16 bytes; and the whole cache."""
    c, h = cache(fmt, D)
    n = first_staged(M, 1, D, dtype, residual=False, aligned=at * (2 if dtype == "bf16" else 4) % 16 == 0 and D % 8 == 0) + 900
    rows = np.random.default_rng(D).integers(-40, 440, n).astype(np.int32)
    rows[5:9] = 1 << 30, -(1 << 31), 400, -1
    want = np.where(((rows >= 0) & (rows < 400))[:, None], h[np.clip(rows, 0, 399)], 0.0)
    out = torch.full((n, D + 2 * at), 5.0, dtype=VALUES[dtype], device="cuda")
    M.q8_read(c, torch.from_numpy(rows).cuda(), out=out[:, at:at + D])
    np.testing.assert_array_equal(f64(out[:, at:at + D]), want)
    assert bool((out[:, :at] == 5).all()) and bool((out[:, at + D:] == 5).all())
    whole, hw = filled(M, 4, n, D, fmt)
    np.testing.assert_array_equal(f64(M.q8_read(whole, dtype=VALUES[dtype])), hw)


@pytest.mark.parametrize("x_at,out_at", [(0, 1), (1, 0), (3, 2), (4, 4)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_staged_rows_of_unlike_alignment(M, cache, x_at, out_at, dtype):
    """x and out that start at different bytes, with strides that move the start from row to row."""
    D, k = 333, 3
    c, h = cache("e5m2", D)
    T = first_staged(M, k, D, dtype, aligned=False) + 50
    rows, w = slots(8, T, k)
    x = activations(2, T, D + 5, dtype)[:, x_at:x_at + D]
    out = torch.full((T, D + 7), 9.0, dtype=VALUES[dtype], device="cuda")
    got = M.q8_combine(c, torch.from_numpy(rows).cuda(), torch.from_numpy(w).cuda(), x=x, out=out[:, out_at:out_at + D],
                       norms=True)
    check(got, h, rows, w.astype(np.float64), f64(x), None, 1, dtype)
    assert bool((out[:, :out_at] == 9).all()) and bool((out[:, out_at + D:] == 9).all())


def test_staged_offsets_past_32_bits(M):
    """Rows, residual and result whose bytes lie past 2^32, read by the staged form."""
    R, D, k = 4_200_000, 1024, 2
    c = M.Q8(torch.empty((R, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn),
             torch.empty((R, 8), dtype=torch.uint8, device="cuda"))
    at = [R - 1, 5, R - 400, 4_194_304, 4_194_303, 17]
    src = activations(1, 6, D, "bf16")
    M.q8_write(src, c, dst=ints(at))
    h = O.dequantise(*O.quantise(f64(src), "e4m3"))
    T = first_staged(M, k, D, "f32") + 300
    pick = np.random.default_rng(0).integers(0, 6, (T, k))
    rows = ints(np.array(at)[pick].tolist())
    stride = (1 << 32) // T // 4 // 4 * 4 + 4096  # so that x and out pass 2^32 bytes
    x = torch.empty(T * stride, device="cuda").as_strided((T, D), (stride, 1))
    x.copy_(activations(2, T, D))
    want, _ = O.combine(h, pick, None, f64(x))
    out = torch.empty(T * stride, device="cuda").as_strided((T, D), (stride, 1))
    got = M.q8_combine(c, rows, x=x, out=out)
    big, _ = O.combine(np.abs(h), pick, None, np.abs(f64(x)))
    assert (np.abs(f64(got) - want) <= (k + 4) * 2.0 ** -23 * big).all()
    one = first_staged(M, 1, D, "f32", residual=False) + 300
    pick = np.random.default_rng(1).integers(0, 6, one)
    np.testing.assert_array_equal(f64(M.q8_read(c, ints(np.array(at)[pick].tolist()), dtype=torch.float32)), h[pick])


# --- the whole layer with a staged combine -----------------------------------

@pytest.fixture(scope="module")
def layers(M):
    """Two expert layers of so many tokens that their combine is staged."""
    made = [layer_state(M, 15, T=first_staged(M, 2, 512, "f32") + 300, D=512, F=640),
            layer_state(M, 16, T=first_staged(M, 2, 384, "f32") + 101, E=8, D=384, F=520)]
    return made, [[t.clone() for t in expert_layer(M, s)] for s in made]


def test_staged_layer_matches_its_stored_stages(M, layers):
    for s, (out, norms) in zip(*layers):
        h = M.q8_read(s["cache"], dtype=torch.float32)
        want, wn = O.combine(f64(h), s["slot_rows"].cpu().numpy(), f64(s["weight"]), f64(s["x"]))
        big, _ = O.combine(np.abs(f64(h)), s["slot_rows"].cpu().numpy(), f64(s["weight"]), np.abs(f64(s["x"])))
        assert (np.abs(f64(out) - want) <= 6 * 2.0 ** -23 * big).all()
        assert (np.abs(f64(norms) - wn) <= (h.shape[1] + 4) * 2.0 ** -24 * wn).all()


def test_staged_layer_in_a_graph(M, layers):
    s, want = layers[0][0], layers[1][0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        expert_layer(M, s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            got = expert_layer(M, s)
    torch.cuda.current_stream().wait_stream(side)
    x0 = s["x"].clone()
    for x in (x0, activations(77, *x0.shape), x0):
        s["x"].copy_(x)
        g.replay()
        replayed = [t.clone() for t in got]
        eager = expert_layer(M, s)
        assert all(torch.equal(a, b) for a, b in zip(replayed, eager))
    assert all(torch.equal(a, b) for a, b in zip(replayed, want))


def test_staged_layers_on_two_streams_and_threads(M, layers):
    states, alone = layers
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in states]
    for _ in range(20):
        got = []
        for s, st in zip(states, streams):
            with torch.cuda.stream(st):
                got.append(expert_layer(M, s))
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for a, b in zip(alone, got) for x, y in zip(a, b))
    wrong = []

    def work(s, want, stream):
        with torch.cuda.stream(stream):
            for _ in range(25):
                got = expert_layer(M, s)
                stream.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want)):
                    wrong.append(1)

    threads = [threading.Thread(target=work, args=p) for p in zip(states, alone, streams)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
