"""Numbers that the library's types do not hold: refused on the host (no GPU here)."""
import pytest

from test_block_devices import BF, HERE, I32, Rows
from test_norm_cache_refusals import _holders, parts  # noqa: F401


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
