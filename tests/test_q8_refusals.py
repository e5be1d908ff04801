"""8-bit row calls check their arguments on the host: every refusal here comes before any launch (no GPU)."""
import ctypes

import pytest

from paper_2606_15615_gb300 import build


@pytest.fixture(scope="module")
def M():
    build.build()
    from paper_2606_15615_gb300 import moeca
    return moeca


A = 1 << 20  # device addresses that are never read: megabytes apart


def rows(M, at, n=4, width=200, q_stride=208, scale_stride=4, fmt=2, **kw):
    r = M.moeca_q8_rows(at * A, at * A + A // 2, n, q_stride, scale_stride, width, fmt)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


BAD_ROWS = [dict(fmt=1), dict(fmt=4), dict(width=0), dict(width=209), dict(q_stride=200), dict(q_stride=192),
            dict(scale_stride=3), dict(scale_stride=0), dict(n=-1), dict(n=1 << 31), dict(q=None), dict(scale=None),
            dict(q=16 * A + 8), dict(scale=16 * A + 2), dict(width=(1 << 20) + 1, q_stride=1 << 21, scale_stride=1 << 14),
            dict(q_stride=1 << 62)]


def refused(M, call, args):
    with pytest.raises(M.MoecaError) as e:
        call(args)
    assert e.value.status == M.MOECA_ERR_INVALID_ARG and str(e.value).split(": ", 1)[1]


def write_args(M, cache=None, **kw):
    a = M.moeca_q8_write_args(cache or rows(M, 16), 1 * A, 4, 200, M.MOECA_BF16, 4, 2 * A, 3 * A, 4 * A)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("bad", BAD_ROWS, ids=str)
def test_bad_rows_are_refused_everywhere(M, bad):
    r = rows(M, 16, **bad)
    refused(M, M.moeca_q8_write, write_args(M, r))
    refused(M, M.moeca_q8_read, M.moeca_q8_read_args(r, A, 200, M.MOECA_F32, 1, 2 * A))
    refused(M, M.moeca_q8_combine, combine_args(M, r))
    for at in ("a", "b"):
        args = matmul_args(M)
        setattr(args, at, r)
        refused(M, M.moeca_q8_matmul, args)
    if bad != dict(fmt=1):  # bf16 rows are an output
        refused(M, M.moeca_q8_matmul, matmul_args(M, out=r))


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(n=-1), dict(x=None), dict(x=A + 1), dict(x_stride=199), dict(x_rows=-1), dict(src=None, n=5),
    dict(dst=None, n=5), dict(src=2 * A + 1), dict(dst=3 * A + 2), dict(count=4 * A + 1), dict(x=16 * A + 16),
    dict(x=16 * A + A // 2), dict(dst=16 * A), dict(x_stride=1 << 62)], ids=str)
def test_write_refusals(M, bad):
    refused(M, M.moeca_q8_write, write_args(M, **bad))


@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(n=-1), dict(out=None), dict(out=A + 2), dict(out_stride=199), dict(rows=2 * A + 1),
    dict(rows=None, n=5), dict(out=16 * A), dict(out=2 * A)], ids=str)
def test_read_refusals(M, bad):
    a = M.moeca_q8_read_args(rows(M, 16), A, 200, M.MOECA_F32, 4, 2 * A)
    for k, v in bad.items():
        setattr(a, k, v)
    refused(M, M.moeca_q8_read, a)


def combine_args(M, cache=None, **kw):
    a = M.moeca_q8_combine_args(cache or rows(M, 16), 2 * A, 3 * A, 4 * A, 200, 5 * A, 200, 6 * A, 200, 7 * A,
                                M.MOECA_BF16, 4, 2, 2)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(n_tokens=-1), dict(n_slots=0), dict(n_slots=17), dict(rows=None), dict(rows=2 * A + 1),
    dict(out=None), dict(out=6 * A + 1), dict(out_stride=100), dict(x=4 * A + 1), dict(x_stride=199), dict(seq=0),
    dict(gate=5 * A + 2), dict(gate_stride=10), dict(weights=3 * A + 2), dict(norms=7 * A + 2), dict(out=4 * A + 16),
    dict(out=4 * A, x_stride=208), dict(norms=6 * A), dict(out=16 * A), dict(norms=2 * A), dict(out=5 * A)], ids=str)
def test_combine_refusals(M, bad):
    refused(M, M.moeca_q8_combine, combine_args(M, **bad))


def matmul_args(M, **kw):
    a = M.moeca_q8_matmul_args(rows(M, 8), rows(M, 9, n=2 * 72), rows(M, 10, width=72, q_stride=80), 2 * A, 3 * A,
                               4 * A, 5 * A, 2, 72, 0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("bad", [
    dict(n_groups=0), dict(n_groups=1025), dict(n_groups=3), dict(n_cols=0), dict(n_cols=71), dict(offsets=None),
    dict(act=3), dict(act=-1), dict(offsets=2 * A + 1), dict(bias=3 * A + 2), dict(dst=4 * A + 1), dict(status=5 * A + 2),
    dict(status=8 * A), dict(dst=10 * A), dict(bias=10 * A)], ids=str)
def test_matmul_refusals(M, bad):
    refused(M, M.moeca_q8_matmul, matmul_args(M, **bad))


def test_matmul_output_refusals(M):
    for out in (rows(M, 10, width=71, q_stride=80), rows(M, 8, width=72, q_stride=80), rows(M, 9, width=72, q_stride=80),
                rows(M, 10, width=72, q_stride=80, fmt=5), rows(M, 10, width=72, q_stride=143, fmt=1),
                rows(M, 10, width=72, q_stride=142, fmt=1), rows(M, 10, width=72, q_stride=284, fmt=0),
                rows(M, 10, width=72, q_stride=144, fmt=1, q=10 * A + 1)):
        refused(M, M.moeca_q8_matmul, matmul_args(M, out=out))
    refused(M, M.moeca_q8_matmul, matmul_args(M, a=rows(M, 8, width=201)))
    refused(M, M.moeca_q8_matmul, matmul_args(M, dst=None, out=rows(M, 10, n=3, width=72, q_stride=80)))
    assert M.LIB.moeca_q8_matmul(None, None) == M.LIB.moeca_q8_combine(None, None) == -1
    assert M.LIB.moeca_q8_write(None, None) == M.LIB.moeca_q8_read(None, None) == -1


def test_products_too_large_to_count_are_unsupported(M):
    far = 1 << 20  # 2^40 bytes
    wide = rows(M, 2 * far, n=1 << 30, width=1 << 12, q_stride=1 << 12, scale_stride=32)
    for args in (matmul_args(M, a=rows(M, far, n=(1 << 30) + 1)),
                 matmul_args(M, a=rows(M, far, n=1 << 30), b=rows(M, 9, n=1 << 12), n_groups=1, n_cols=1 << 12, out=wide)):
        with pytest.raises(M.MoecaError) as e:
            M.moeca_q8_matmul(args)
        assert e.value.status == M.MOECA_ERR_UNSUPPORTED


def test_empty_calls_launch_nothing(M):
    """No rows: OK without a device."""
    M.moeca_q8_write(write_args(M, n=0))
    M.moeca_q8_write(write_args(M, x_rows=0, x=None, n=3))
    M.moeca_q8_read(M.moeca_q8_read_args(rows(M, 16), None, 200, M.MOECA_F32, 0, None))
    M.moeca_q8_combine(combine_args(M, n_tokens=0, rows=None, out=None, x=None))
    M.moeca_q8_matmul(matmul_args(M, a=rows(M, 8, n=0, q=None, scale=None)))


def test_binding_refusals(M):
    """The torch calls check types, shapes and devices before they ask for a device."""
    torch = pytest.importorskip("torch")
    cache = M.q8_empty(4, 200, device="cpu")
    assert cache.q.shape == (4, 200) and cache.q.stride() == (208, 1) and cache.scale.shape == (4, 2)
    assert (M.q8_read.__doc__ and cache.scale.stride() == (4, 1))
    x = torch.zeros(4, 200)
    i32 = torch.zeros(4, dtype=torch.int32)
    bad = [lambda: M.q8_write(x, cache),                                        # no CUDA device
           lambda: M.q8_write(x.half(), cache), lambda: M.q8_write(x[:, :100], cache),
           lambda: M.q8_write(x, cache, dst=i32.long()), lambda: M.q8_write(x, cache, src=i32[:2], dst=i32),
           lambda: M.q8_write(x, cache, count=i32), lambda: M.q8_write(x.T, cache),
           lambda: M.q8_write(x, M.Q8(cache.q.view(torch.uint8), cache.scale)),
           lambda: M.q8_write(x, M.Q8(cache.q, cache.scale[:, :1])),
           lambda: M.q8_write(x, M.Q8(cache.q, cache.scale[:3])),
           lambda: M.q8_read(cache, dtype=torch.float16), lambda: M.q8_read(cache, i32.view(2, 2)),
           lambda: M.q8_read(cache, out=x[:3]), lambda: M.q8_read(cache, dtype=torch.bfloat16, out=x),
           lambda: M.q8_combine(cache, i32), lambda: M.q8_combine(cache, i32.view(4, 1), x=x[:2]),
           lambda: M.q8_combine(cache, i32.view(4, 1), x=x, out=x.bfloat16()),
           lambda: M.q8_combine(cache, i32.view(4, 1), gate=x[:3]),
           lambda: M.q8_combine(cache, i32.view(4, 1), weights=x),
           lambda: M.q8_matmul(cache, cache, offsets=i32[:1]), lambda: M.q8_matmul(cache, cache, offsets=i32),
           lambda: M.q8_matmul(cache, cache, act="relu"), lambda: M.q8_matmul(cache, cache, dtype=torch.float16),
           lambda: M.q8_matmul(cache, cache, out=x), lambda: M.q8_matmul(cache, cache, bias=x)]
    for f in bad:
        with pytest.raises(ValueError):
            f()


def test_struct_layouts_match_the_header(M, tmp_path):
    import shutil
    import subprocess
    from pathlib import Path
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    names = ["moeca_q8_rows", "moeca_q8_write_args", "moeca_q8_read_args", "moeca_q8_combine_args", "moeca_q8_matmul_args"]
    lines, expect = ['#include <stdio.h>', '#include <stddef.h>', '#include "moeca_q8.h"', "int main(void) {"], []
    for n in names:
        py = getattr(M, n)
        lines.append(f'  printf("%zu\\n", sizeof({n}));')
        expect.append(ctypes.sizeof(py))
        for f, _ in py._fields_:
            lines.append(f'  printf("%zu\\n", offsetof({n}, {f}));')
            expect.append(getattr(py, f).offset)
    src, exe = tmp_path / "l.c", tmp_path / "l"
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    subprocess.run([cc, "-std=c11", f"-I{Path(__file__).resolve().parents[1] / 'include'}", str(src), "-o", str(exe)], check=True)
    assert [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()] == expect
