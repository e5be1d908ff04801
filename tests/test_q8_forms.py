"""The rule that chooses the 8-bit combine's form (no GPU)."""
import pytest

from test_q8_refusals import M  # noqa: F401  (a fixture)


def test_the_rule_follows_tokens_width_and_device(M):
    staged = M.moeca_probe_q8_staged
    for dtype in (M.MOECA_F32, M.MOECA_BF16):
        for k, width in ((1, 8), (2, 1152), (8, 1152), (16, 1024)):
            for sms in (100, 152):
                first = next(T for T in range(1, 16 * sms) if staged(sms, T, k, width, dtype))
                assert first % sms == 1 and first > sms  # as many tokens as direct blocks run at once are direct
                assert staged(sms, 1 << 30, k, width, dtype) and not staged(sms, first - 1, k, width, dtype)
        assert not staged(152, 1 << 30, 2, 1 << 20, dtype) and not staged(152, 1 << 30, 16, 9000, dtype)
    for bad in ((0, 1, 1, 8, 0), (152, -1, 1, 8, 0), (152, 1, 0, 8, 0), (152, 1, 17, 8, 0), (152, 1, 1, 0, 0),
                (152, 1, 1, 8, 2)):
        with pytest.raises(M.MoecaError):
            staged(*bad)
