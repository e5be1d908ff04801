"""Limits of the packed attention's arguments, checked on the host: no GPU, and nothing is launched."""
import math

import pytest

from paper_2606_15615_gb300 import build

A = 1 << 20  # device addresses that are never read: megabytes apart


@pytest.fixture(scope="module")
def M():
    build.build()
    from paper_2606_15615_gb300 import moeca
    return moeca


def args(M, n_queries=0, n_keys=50, n_seqs=1, H=4, Hk=2, d=64, dtype=None, max_q=0, causal=1, offsets=False, scale=0.125):
    h = M.moeca_heads
    return M.moeca_attention_args(
        h(16 * A, H * d, d, H), h(1 << 40, 2 * Hk * d, d, Hk), h((1 << 40) + 2 * Hk * d, 2 * Hk * d, d, Hk), h(1 << 41, H * d, d, H),
        A if offsets else None, 2 * A if offsets else None, None, 1 << 42, None, n_queries, n_keys, n_seqs, max_q,
        M.MOECA_BF16 if dtype is None else dtype, d, causal, 0, scale)


@pytest.mark.parametrize("scale", [2.36e38, 3e38, 3.4e38, math.inf, math.nan, 0.0, -1e-3])
def test_scales_without_a_finite_base_2_form_are_refused(M, scale):
    with pytest.raises(M.MoecaError, match="scale") as e:
        M.moeca_attention(args(M, scale=scale))
    assert e.value.status == M.MOECA_ERR_INVALID_ARG and M.moeca_attention_workspace(args(M, scale=scale)) == -1


@pytest.mark.parametrize("scale", [2.35e38, 1.0, 1e-45])
def test_scales_up_to_the_largest_are_taken(M, scale):
    M.moeca_attention(args(M, scale=scale))
    assert M.moeca_attention_workspace(args(M, scale=scale)) == 0


@pytest.mark.parametrize("clear", [-1, 3, 1 << 30])
def test_what_clear_may_be(M, clear):
    bad = args(M)
    bad.clear = clear
    with pytest.raises(M.MoecaError, match="clear"):
        M.moeca_attention(bad)
    for good in (0, 1, 2):
        bad.clear = good
        M.moeca_attention(bad)


@pytest.mark.parametrize("clear", [-1, 4, 1 << 30])
def test_what_the_norm_may_clear(M, clear):
    h = M.moeca_heads
    bad = M.moeca_qk_norm_rope_args(h(16 * A, 512, 64, 4), h(17 * A, 512, 64, 2), h(18 * A, 256, 64, 4), h(19 * A, 128, 64, 2), A, 2 * A,
                                    3 * A, 4 * A, 50, M.MOECA_BF16, 0, 64, 64, 0, 1e-6, clear)
    with pytest.raises(M.MoecaError, match="clear"):
        M.moeca_qk_norm_rope(bad)
    for good in range(4):
        bad.clear = good
        M.moeca_qk_norm_rope(bad)


# Sizes and the form they reach: (queries, keys, sequences, heads, key heads, dim, max_q), form, whether keys are cut.
FORMS = [((1, 300, 1, 4, 2, 64, 0), "ROWS", False), ((1, 65536, 1, 4, 4, 128, 0), "ROWS", True), ((16, 300, 1, 2, 2, 64, 0), "ROWS", False),
         ((17, 300, 1, 2, 2, 64, 0), "TILE", False), ((128, 128, 1, 1, 1, 72, 0), "TILE", False), ((64, 32768, 1, 8, 8, 128, 0), "TILE", True),
         ((4096, 4096, 16, 16, 16, 72, 256), "TILES", False), ((16384, 16384, 5, 32, 8, 128, 6000), "TILES", False),
         ((512, 40448, 16, 32, 2, 64, 32), "TILE", True), ((400, 4096, 4, 20, 20, 128, 200), "TILE", False),
         ((800, 20000, 40, 2, 2, 64, 20), "TILE", True), ((300, 9001, 1, 2, 2, 64, 0), "TILES", True), ((300, 300, 1, 2, 2, 130, 0), "CORES", True), ((40, 40, 1, 2, 2, 36, 0), "CORES", False)]


@pytest.mark.parametrize("size,form,cut", FORMS, ids=str)
def test_forms(M, size, form, cut):
    n, m, seqs, H, Hk, d, max_q = size
    a = args(M, n, m, seqs, H, Hk, d, max_q=max_q, offsets=True)
    got, chunk = M.moeca_probe_attention_form(a)
    assert got == getattr(M, "MOECA_ATTENTION_FORM_" + form) and (chunk > 0) == cut
    assert (M.moeca_attention_workspace(a) > 0) == cut
    assert M.moeca_probe_attention_form(args(M, n, m, seqs, H, Hk, d, max_q=max_q, offsets=True, dtype=M.MOECA_F32))[0] == 0


def test_form_refusals(M):
    for bad in (args(M), args(M, 1, d=257), args(M, 1, scale=-1.0), args(M, (1 << 30) + 1)):
        with pytest.raises(M.MoecaError):
            M.moeca_probe_attention_form(bad)


def parts(M, layout, H, T, d, parts=3):
    """q, k, v of one fused buffer: which strides a token and a head have, and how far apart the parts are."""
    token, head, part = {"token, part, head": (parts * H * d, d, H * d), "token, head, part": (parts * H * d, parts * d, d),
                         "head, token, part": (parts * d, parts * T * d, d), "head, part, token": (d, parts * T * d, T * d),
                         "part, token, head": (H * d, d, T * H * d)}[layout]
    return [M.moeca_heads(A + 2 * p * part, token, head, H) for p in range(parts)]


@pytest.mark.parametrize("layout", ["token, part, head", "token, head, part", "head, token, part", "head, part, token", "part, token, head"])
@pytest.mark.parametrize("H,d", [(4, 64), (5, 72), (4, 33)])
def test_parts_of_a_fused_buffer_do_not_overlap(M, layout, H, d):
    """Results over the queries of a fused buffer in any order of its axes: refused for its size alone, which is
    looked at last; a value too far, and it meets its neighbour."""
    T = 1 << 29
    q, k, v = parts(M, layout, H, T, d)
    a = args(M, T, T, H=H, Hk=H, d=d)
    a.q, a.k, a.v, a.out, a.workspace = q, k, v, q, None
    with pytest.raises(M.MoecaError) as e:
        M.moeca_attention(a)
    assert e.value.status == M.MOECA_ERR_UNSUPPORTED
    for near in (k, v):
        a.out = M.moeca_heads(near.data - 2, q.token_stride, q.head_stride, H)
        with pytest.raises(M.MoecaError, match="overlaps") as e:
            M.moeca_attention(a)
        assert e.value.status == M.MOECA_ERR_INVALID_ARG
