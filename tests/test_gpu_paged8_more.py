"""The paged cache of 8-bit floating point where its kernels can go wrong by how a call is cut, and at the ends of its ranges."""
import pytest

from paged8_lines import line
from test_gpu_paged8 import Pair, attend, in_blocks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("diff", [False, True])
def test_units_of_every_number_of_pieces(diff):
    """Blocks cut into 5 to 11 pieces, among them 6 and 11: their last pieces have no neighbour at a level between two at which they have one."""
    lengths = [32 * (95 + 4 * s) + 7 for s in range(33)]
    rows = [16] * 33
    assert in_blocks(1, 16, rows, lengths, diff)
    pieces = line(1, 16, rows, lengths, 16, -(-max(lengths) // 64) * 64)[1]
    assert {5, 6, 7, 8, 9, 10, 11} <= set(pieces)
    c = Pair(1, 64, 33, -(-max(lengths) // 64), seed=41).filled(lengths)
    attend(c, 16, rows, lengths, diff=diff)
