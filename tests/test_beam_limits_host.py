"""The largest calls of q4kv_beam_select: refused in front of a launch that its grid does not fit."""
import pytest

from paper_2603_04428_amd import binding as b
from tests.test_device_tables_host import err, select


@pytest.mark.parametrize("rows,fits", [(2 ** 26 - 4, True), (2 ** 26 - 3, False), (2 ** 26 - 2, False), (2 ** 26 - 1, False), (2 ** 26, False)])
def test_spans_of_all_rows(rows, fits):
    """One span to a row of one token; four spans are a workgroup of 256 threads, and a grid holds 2^32 - 1."""
    need = b.lib().q4kv_beam_select_workspace_bytes(0, 1, rows, 1)
    assert (need > 0) == fits
    if not fits:
        assert "fewer groups" in err()
        assert select(rows=rows, vocab=1, stride=1, out=1, bytes=1 << 40) == -3 and "fewer groups" in err()
    assert ((rows + 3) // 4 * 256 < 2 ** 32) == fits
