"""Sizes that the 8-bit product refuses because its tiles could not be counted (no GPU: refused before any launch)."""
import pytest

from test_q8_refusals import M, matmul_args, refused, rows, write_args  # noqa: F401  (M: a fixture)

FAR = 1 << 20  # 2^40 bytes apart


@pytest.mark.parametrize("groups,n_rows,cols", [(512, 1 << 24, 1 << 15), (512, 1 << 20, 1 << 19), (63, 1 << 29, 1 << 12)])
def test_rows_claimed_again_and_again_are_counted(M, groups, n_rows, cols):
    """Offsets 0, rows, 0, rows, .. make every second group claim all rows: more tiles than 32 bits can count, although
    each row counted once they are few."""
    wide = -(-cols // 256)
    assert (n_rows / 16 + groups) * wide <= 1 << 30
    assert (groups + 1) // 2 * (n_rows // 224) * wide > (1 << 30)
    args = matmul_args(M, a=rows(M, FAR, n=n_rows, width=16, q_stride=16),
                       b=rows(M, 2 * FAR, n=groups * cols, width=16, q_stride=16),
                       out=rows(M, 3 * FAR, n=8, width=cols, q_stride=cols, scale_stride=cols // 128, scale=4 * FAR << 20), n_groups=groups,
                       n_cols=cols, offsets=8 * FAR << 20, dst=9 * FAR << 20, bias=None, status=None)
    with pytest.raises(M.MoecaError) as e:
        M.moeca_q8_matmul(args)
    assert e.value.status == M.MOECA_ERR_UNSUPPORTED


def test_columns_of_wider_rows_end_with_their_own_bytes(M):
    """The last row of a block of columns ends where its bytes do, not a stride after its start: what lies there is
    another buffer.  No rows are asked for, so that nothing is launched; one byte less is an overlap."""
    at, stride, width = 16 << 20, 2048, 200
    end, s_end = at + 3 * stride + 208, at + (1 << 19) + 3 * 16 + 4

    def cache():
        return rows(M, 16, n=4, width=width, q_stride=stride, scale_stride=16)

    for behind in (end, s_end):
        M.moeca_q8_write(write_args(M, cache(), n=0, x=behind))
        refused(M, M.moeca_q8_write, write_args(M, cache(), n=0, x=behind - 4))
    b = rows(M, 16, n=4, width=width, q_stride=stride, scale_stride=16)
    for q in (end, s_end // 16 * 16 + 16):
        M.moeca_q8_matmul(matmul_args(M, a=rows(M, 8, n=0), b=b, n_groups=1, n_cols=4, out=rows(
            M, 1, n=2, width=4, q_stride=16, q=q), status=None))
    refused(M, M.moeca_q8_matmul, matmul_args(M, a=rows(M, 8, n=0), b=b, n_groups=1, n_cols=4,
                                              out=rows(M, 1, n=2, width=4, q_stride=16, q=end - 16), status=None))
