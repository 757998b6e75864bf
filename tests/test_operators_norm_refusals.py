"""CPU: what layer norm refuses beside tests/test_more_operators_refusals.py, and the workspace that it asks for."""
import ctypes as C

import pytest

from paper_1710_06952_amd import binding as B

NOWHERE = 1 << 20                                        # an aligned address that is never read


@pytest.mark.parametrize("eps", [1e39, 3.5e38, 2.0 ** 128, 1e300, 2.0 ** -127])
def test_eps_that_32_bits_do_not_hold(eps):
    """It would be infinity there, and 1 / sqrt of it 0; subnormal ones are 0 to the instruction."""
    L = B.lib()
    o = B.LayerNorm(B.TYPE_F32, B.TYPE_F32, 4, 16, NOWHERE, 16, NOWHERE, NOWHERE, eps, None, 0)
    assert L.adpsgd_layer_norm_forward(C.byref(o), NOWHERE, NOWHERE, None) == B.ERR_ARG
    assert "eps" in L.adpsgd_last_error(None).decode()
    for fine in (2.0 ** -126, 3.4e38):                   # refused for its missing result, behind the check of eps
        o.eps = fine
        assert L.adpsgd_layer_norm_forward(C.byref(o), None, NOWHERE, None) == B.ERR_ARG
        assert "y is NULL" in L.adpsgd_last_error(None).decode()


@pytest.mark.parametrize("kind,least", [(B.TYPE_BF16, 16_384 + 8), (B.TYPE_F16, 16_384 + 8), (B.TYPE_F32, 8192 + 4)])
def test_the_workspace_of_long_rows_is_small_beside_them(kind, least):
    """Rows in passes: strips for the columns' sums are as many as fill the chip beside n / 256 blocks across, 8 bytes a column each: 2048 blocks of 256 columns
    (4 MiB), and one strip where n is more than that."""
    L = B.lib()
    for n in (least, 32_768, 70_001, 1 << 18, 1 << 20, 1 << 24):
        for rows in (1, 2, 33, 512, 2000, 100_000, 5_000_000):
            if rows * n > 1 << 43:
                continue
            got = L.adpsgd_layer_norm_workspace_bytes(kind, rows, n)
            assert 8 * n <= got <= max(8 * 256 * 2048, 8 * n)
            assert got <= 8 * n * rows and got % (8 * n) == 0
