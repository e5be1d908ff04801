"""Expert sort, its way back, head norms and packed attention check their arguments on the host: every refusal here
comes before any launch (no GPU), and so do calls with nothing to do."""
import ctypes
import shutil
import subprocess
from pathlib import Path

import pytest

from paper_2606_15615_gb300 import build

ROOT = Path(__file__).resolve().parents[1]


@pytest.fixture(scope="module")
def M():
    build.build()
    from paper_2606_15615_gb300 import moeca
    return moeca


A = 1 << 20  # device addresses that are never read: megabytes apart


def refused(M, call, args, status=None):
    with pytest.raises(M.MoecaError) as e:
        call(args)
    assert e.value.status == (M.MOECA_ERR_INVALID_ARG if status is None else status) and str(e.value).split(": ", 1)[1]


def with_fields(args, **kw):
    for k, v in kw.items():
        target = args
        *path, last = k.split("__")
        for p in path:
            target = getattr(target, p)
        setattr(target, last, v)
    return args


def sort_args(M, **kw):
    return with_fields(M.moeca_expert_sort_args(A, 100, 2, 8, 2 * A, 3 * A, 4 * A, 5 * A, 6 * A), **kw)


@pytest.mark.parametrize("bad", [
    dict(n_tokens=-1), dict(n_slots=0), dict(n_slots=17), dict(n_experts=0), dict(n_experts=513), dict(experts=None),
    dict(offsets=None), dict(place=None), dict(experts=A + 2), dict(offsets=2 * A + 1), dict(place=3 * A + 3),
    dict(slot=4 * A + 2), dict(token=5 * A + 1), dict(n_tokens=10_000, workspace=None), dict(workspace=6 * A + 2),
    dict(place=A), dict(slot=3 * A + 400), dict(token=4 * A), dict(offsets=A + 796), dict(n_tokens=(1 << 30) // 2 + 1),
    dict(n_tokens=10_000, workspace=4 * A)], ids=str)
def test_sort_refusals(M, bad):
    refused(M, M.moeca_expert_sort, sort_args(M, **bad))


def test_sort_workspace(M):
    assert M.moeca_expert_sort_workspace(1, 1, 1) == 0 == M.moeca_expert_sort_workspace(0, 16, 512)
    assert 0 < M.moeca_expert_sort_workspace(32768, 8, 64) <= 32768 * 8
    assert M.moeca_expert_sort_workspace(1 << 26, 16, 512) > 0
    for bad in ((-1, 1, 1), (1, 0, 1), (1, 17, 1), (1, 1, 0), (1, 1, 513), ((1 << 26) + 1, 16, 1)):
        assert M.moeca_expert_sort_workspace(*bad) == -1


def rows_args(M, **kw):
    return with_fields(M.moeca_expert_rows_args(A, 64, 2 * A, 64, 8, 3 * A, 4 * A, M.MOECA_BF16, 4, 2, 64), **kw)


COMMON = [dict(dtype=2), dict(n_tokens=-1), dict(n_slots=0), dict(n_slots=17), dict(width=0), dict(width=(1 << 20) + 1),
          dict(n_rows=-1), dict(n_rows=1 << 31), dict(place=None), dict(place=3 * A + 2)]


@pytest.mark.parametrize("bad", COMMON + [
    dict(x=None), dict(x=A + 1), dict(x_stride=63), dict(rows=None), dict(rows=2 * A + 1), dict(rows_stride=63),
    dict(count=4 * A + 2), dict(rows=A + 400), dict(rows=3 * A), dict(rows=4 * A), dict(rows_stride=1 << 62)], ids=str)
def test_rows_refusals(M, bad):
    refused(M, M.moeca_expert_rows, rows_args(M, **bad))


def back_args(M, **kw):
    return with_fields(M.moeca_expert_combine_args(2 * A, 64, 8, 3 * A, 4 * A, A, 64, 5 * A, 64, M.MOECA_BF16, 4, 2, 64), **kw)


@pytest.mark.parametrize("bad", COMMON + [
    dict(x=A + 1), dict(x_stride=63), dict(rows=None), dict(rows=2 * A + 1), dict(rows_stride=63), dict(out=None),
    dict(out=5 * A + 1), dict(out_stride=60), dict(weights=4 * A + 2), dict(out=2 * A), dict(out=3 * A), dict(out=4 * A),
    dict(out=A + 16), dict(out=A, out_stride=72)], ids=str)
def test_combine_refusals(M, bad):
    refused(M, M.moeca_expert_combine, back_args(M, **bad))


def grad_args(M, **kw):
    return with_fields(M.moeca_expert_combine_grad_args(A, 64, 2 * A, 64, 8, 3 * A, 4 * A, 5 * A, 6 * A, 64, 7 * A, M.MOECA_BF16, 4,
                                                        2, 64), **kw)


@pytest.mark.parametrize("bad", COMMON + [
    dict(dout=None), dict(dout=A + 1), dict(dout_stride=63), dict(rows=None), dict(rows=2 * A + 1), dict(rows_stride=63),
    dict(drows=6 * A + 1), dict(drows_stride=63), dict(weights=4 * A + 1), dict(dweights=7 * A + 2), dict(count=5 * A + 2),
    dict(drows=A), dict(drows=2 * A + 128), dict(dweights=3 * A), dict(dweights=4 * A), dict(drows=5 * A), dict(dweights=6 * A)],
    ids=str)
def test_gradient_refusals(M, bad):
    refused(M, M.moeca_expert_combine_grad, grad_args(M, **bad))


def test_nothing_to_do(M):
    M.moeca_expert_rows(rows_args(M, n_rows=0, rows=None))
    M.moeca_expert_rows(rows_args(M, n_tokens=0, x=None, place=None, count=None))
    M.moeca_expert_combine(back_args(M, n_tokens=0, out=None, place=None))
    M.moeca_expert_combine_grad(grad_args(M, drows=None, dweights=None))
    M.moeca_expert_combine_grad(grad_args(M, n_tokens=0, count=None, dout=None, place=None))
    M.moeca_qk_norm_rope(qk_args(M, n_tokens=0))
    M.moeca_attention(attention_args(M, n_queries=0, q_offsets=None))


def qk_args(M, **kw):
    h = M.moeca_heads
    return with_fields(M.moeca_qk_norm_rope_args(
        h(16 * A, 512, 64, 4), h(17 * A, 512, 64, 2), h(18 * A, 256, 64, 4), h(19 * A, 128, 64, 2), A, 2 * A, 3 * A, 4 * A, 50,
        M.MOECA_BF16, 10, 64, 64, 0, 1e-6), **kw)


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(n_tokens=-1), dict(dim=0), dict(dim=513), dict(rot=-2), dict(rot=63), dict(rot=66), dict(pairs=2),
    dict(eps=-1.0), dict(eps=float("nan")), dict(n_positions=-1), dict(n_positions=1 << 31), dict(q__data=None),
    dict(q__data=16 * A + 1), dict(q__heads=0), dict(q__heads=-1), dict(k__heads=3), dict(q_out__heads=3), dict(q__token_stride=-1),
    dict(q__token_stride=1 << 41), dict(k__head_stride=-64), dict(q_out__token_stride=255), dict(q_out__head_stride=63),
    dict(table=None), dict(table=3 * A + 4), dict(pos=4 * A + 2), dict(q_weight=A + 1), dict(k_weight=2 * A + 2),
    dict(q_out__data=16 * A + 2), dict(q_out__data=17 * A), dict(k_out__data=16 * A), dict(k_out__data=18 * A + 64),
    dict(q_out__data=3 * A), dict(q_out__data=4 * A), dict(k_out__data=A), dict(q_out__data=16 * A, q_out__token_stride=512 + 64)],
    ids=str)
def test_norm_refusals(M, bad):
    refused(M, M.moeca_qk_norm_rope, qk_args(M, **bad))


def attention_args(M, **kw):
    h = M.moeca_heads
    return with_fields(M.moeca_attention_args(
        h(16 * A, 256, 64, 4), h(17 * A, 256, 64, 2), h(17 * A + 256, 256, 64, 2), h(18 * A, 256, 64, 4), A, 2 * A, 3 * A, 4 * A,
        5 * A, 40, 50, 3, 0, M.MOECA_BF16, 64, 1, 0, 0.125), **kw)


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(dim=0), dict(dim=257), dict(n_seqs=0), dict(n_seqs=(1 << 20) + 1), dict(n_queries=-1), dict(n_keys=-1),
    dict(max_q=-1), dict(q_offsets=None), dict(k_offsets=None), dict(q__heads=3, out__heads=3), dict(q__heads=0), dict(k__heads=0),
    dict(v__heads=1), dict(out__heads=2), dict(causal=2), dict(clear=-1), dict(scale=0.0), dict(scale=-1.0),
    dict(scale=float("nan")), dict(scale=float("inf")), dict(q__data=None), dict(k__data=None), dict(v__data=17 * A + 257),
    dict(out__data=None), dict(out__token_stride=64), dict(q_offsets=A + 2), dict(k_offsets=2 * A + 1), dict(lse=3 * A + 2),
    dict(status=5 * A + 1), dict(out__data=16 * A + 2), dict(out__data=17 * A), dict(out__data=A), dict(out__data=2 * A),
    dict(out__data=3 * A), dict(lse=17 * A), dict(status=16 * A), dict(lse=A), dict(status=3 * A + 4),
    dict(out__data=16 * A, out__head_stride=128, out__token_stride=512)], ids=str)
def test_attention_refusals(M, bad):
    refused(M, M.moeca_attention, attention_args(M, **bad))


def test_attention_needs_its_workspace(M):
    long = dict(n_queries=3, q_offsets=None, n_keys=1 << 18, k__data=64 * A, v__data=64 * A + 256, max_q=1)
    size = M.moeca_attention_workspace(attention_args(M, **long))
    assert 0 < size <= 1 << 30
    refused(M, M.moeca_attention, attention_args(M, workspace=None, **long))
    refused(M, M.moeca_attention, attention_args(M, workspace=4 * A + 8, **long))
    refused(M, M.moeca_attention, attention_args(M, workspace=65 * A, **long))  # inside k
    refused(M, M.moeca_attention, attention_args(M, workspace=18 * A - size // 2 // 16 * 16, **long))
    assert M.moeca_attention_workspace(attention_args(M)) == 0
    assert M.moeca_attention_workspace(attention_args(M, dim=0)) == -1


def test_sizes_beyond_a_launch(M):
    assert M.moeca_attention_workspace(attention_args(M, n_keys=(1 << 30) + 1)) == -1
    refused(M, M.moeca_attention, attention_args(M, n_keys=(1 << 30) + 1, k__data=1 << 50, v__data=(1 << 50) + 256),
            M.MOECA_ERR_UNSUPPORTED)


def test_parts_of_one_buffer_are_no_overlap(M):
    """A fused projection's parts in place: refused only where they meet."""
    import paper_2606_15615_gb300.moeca as m
    h = m.moeca_heads
    base = 16 * A
    q, k = h(base, 8 * 64, 64, 4), h(base + 4 * 64 * 2, 8 * 64, 64, 2)
    args = qk_args(m, n_tokens=0)
    args.q, args.k, args.q_out, args.k_out = q, k, q, k
    args.n_tokens = 10
    args.k_out = h(base + 4 * 64 * 2 - 128, 8 * 64, 64, 2)
    with pytest.raises(m.MoecaError, match="overlaps"):
        M.moeca_qk_norm_rope(args)
    args.k_out, args.pos = k, base + 6 * 64 * 2  # between the parts, but inside their range
    with pytest.raises(m.MoecaError, match="overlaps"):
        M.moeca_qk_norm_rope(args)
    args.pos, args.q_weight = 4 * A, A + 1
    with pytest.raises(m.MoecaError, match="aligned"):
        M.moeca_qk_norm_rope(args)


def test_struct_layouts_match_the_headers(M, tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "moeca_experts.h"', '#include "moeca_attention.h"',
             "int main(void) {"]
    expect = []
    for name in ("moeca_expert_sort_args", "moeca_expert_rows_args", "moeca_expert_combine_args", "moeca_expert_combine_grad_args",
                 "moeca_heads", "moeca_qk_norm_rope_args", "moeca_attention_args"):
        py = getattr(M, name)
        lines.append(f'  printf("%zu\\n", sizeof({name}));')
        expect.append(ctypes.sizeof(py))
        for field, _ in py._fields_:
            lines.append(f'  printf("%zu\\n", offsetof({name}, {field}));')
            expect.append(getattr(py, field).offset)
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    exe = tmp_path / "layout"
    subprocess.run([cc, "-std=c11", f"-I{ROOT / 'include'}", str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == expect


def test_python_refusals(M):
    """Tensors that are not on the GPU, or of a wrong shape or type, raise ValueError."""
    import torch
    i = torch.zeros(4, 2, dtype=torch.int32)
    x = torch.zeros(4, 8)
    plan = M.ExpertPlan(torch.zeros(4, dtype=torch.int32), i, torch.zeros(8, dtype=torch.int32), torch.zeros(8, dtype=torch.int32))
    h = torch.zeros(4, 2, 8)
    for call in (lambda: M.expert_sort(i.long(), 3), lambda: M.expert_sort(i[0], 3), lambda: M.expert_sort(i, 0),
                 lambda: M.expert_sort(i, 513), lambda: M.expert_sort(i, 3), lambda: M.expert_rows(x, plan),
                 lambda: M.expert_rows(x[:3], plan), lambda: M.expert_rows(x.double(), plan), lambda: M.expert_rows(x.T, plan),
                 lambda: M.expert_combine(x, plan, weights=x), lambda: M.expert_combine(x, plan, x=x[:2]),
                 lambda: M.expert_combine_grad(x[:2], x, plan), lambda: M.qk_norm_rope(h, h), lambda: M.qk_norm_rope(h.half(), h),
                 lambda: M.qk_norm_rope(h, h[:, :, :4]), lambda: M.qk_norm_rope(x, None), lambda: M.qk_norm_rope(h, None, x),
                 lambda: M.attention(h, h, h[:2]), lambda: M.attention(h, h[..., :4], h), lambda: M.attention(h, h, h),
                 lambda: M.attention(h, h, h, q_offsets=i[0], n_seqs=7), lambda: M.rope_table(torch.zeros(3, 2), [4]),
                 lambda: M.rope_table(torch.zeros(3), 5)):
        with pytest.raises((ValueError, M.MoecaError)):
            call()
