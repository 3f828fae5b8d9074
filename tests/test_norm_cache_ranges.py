"""Numbers that the library's types do not hold: refused on the host (no GPU here)."""
import pytest

from test_block_devices import BF, HERE, I32, Rows
from test_norm_cache_refusals import INV, L, P, _holders, parts  # noqa: F401


@pytest.mark.parametrize("base", [2 ** 31, 2 ** 32 + 1, -2 ** 31 - 1])
def test_a_base_of_positions_beyond_32_bits(parts, base):  # noqa: F811
    """2^32 + 1 is not 1."""
    holders, c = _holders(parts, HERE)
    rows, ids = Rows((3, 32), BF), Rows((3,), I32)
    with pytest.raises(ValueError, match="pos_base"):
        c.append(0, rows, rows, ids, ids, pos_base=base)
    assert c._append.made == 0
    for fine in (1, 0, -2 ** 31, 2 ** 31 - 1):
        c.append(0, rows, rows, ids, ids, pos_base=fine)
    assert c._append.made == 4


def test_scales_that_f32_does_not_hold(L):  # noqa: F811
    """(they would make 0 times infinity, NaN)"""
    fwd = lambda a=1.0, b=1.0, eps=1e-6: L.ps_residual_norm_fwd(4, 64, 0, 3, P, 64, P, 64, P, P, P, a, b, eps, P, 64, P, 64, None)  # noqa: E731
    bwd = lambda a=1.0, b=1.0, eps=1e-6: L.ps_residual_norm_bwd(4, 64, 0, 3, P, 64, P, 64, P, 64, P, 64, P, P, P, a, b, eps, P, 64,  # noqa: E731
                                                                P, 64, P, P, P, 0, P, 1 << 24, None)
    for call in (fwd, bwd):
        for bad in (dict(a=1e39), dict(a=-1e300), dict(b=1e39), dict(eps=1e39)):
            assert call(**bad) == INV, bad
    need = L.ps_paged_decode_workspace_size(64)
    for scale in (1e39, -1e39, 3e38):
        assert L.ps_paged_decode(2, 4, 2, 64, 0, P, 256, P, P, 16, 16, P, 8, P, 0, scale, P, 256, None, P, need, None) == INV, scale
