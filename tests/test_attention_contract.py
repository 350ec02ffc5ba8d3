"""What the attention calls promise that shows without a GPU."""
import pytest

pytest.importorskip("torch")


def test_workspace_of_values_that_would_be_rejected():
    import paper_2505_07239_amd as comet
    size = lambda m, ld, d: comet.workspace_bytes(comet.OP_VALUES, m, ld, d, 0)
    assert size(8, 20000, 64) >= 3 * 8 * 64 * 8
    for m, ld, d in ((8, 20001, 64), (8, 20000, 63), (8, 20000, 0), (8, 20000, -2), (8, 20000, 4098), (8, 1 << 24, 64), (8, 0, 64),
                     (8, -2, 64), (-1, 20000, 64), (1 << 31, 20000, 64)):
        assert size(m, ld, d) == 0, (m, ld, d)
