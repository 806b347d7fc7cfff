"""The scratch of the vocabulary calls at the sizes' limits."""
import pytest

import paper_2607_24434_amd as de

# The largest number of rows for a vocabulary: rows * ceil(V / 4096) < 2^24, at most 2^20.
LIMITS = [(1, 1 << 20), (61440, 1 << 20), (65536, (1 << 20) - 1), (65537, 986895), (1 << 20, 65535),
          (1 << 30, 63)]


@pytest.mark.parametrize("V,rows", LIMITS)
def test_no_scratch_for_sizes_that_the_calls_refuse(V, rows):
    assert rows * -(-V // 4096) < 1 << 24
    assert de.de_scores_workspace_bytes(rows, V, 0) > 0
    more = rows + 1
    assert more > 1 << 20 or more * -(-V // 4096) >= 1 << 24
    assert de.de_scores_workspace_bytes(more, V, 0) == 0
    with pytest.raises(de.DEError):
        de.scores_workspace(more, V, device="cpu")
