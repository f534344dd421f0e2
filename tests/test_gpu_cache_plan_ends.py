"""dd_cache_plan at the end of 32-bit positions: tables long enough for more tokens than a position can name."""
import numpy as np
import pytest

from paper_2609_04010_amd import _lib as dd
from tests.gpu_util import dev_i32, say, torch_or_skip

pytestmark = pytest.mark.gpu

P, HELD = 256, 1 << 23


def _plan(torch, T, n_new):
    ld = HELD + 16
    cc, m = dd.cache_config(16, P, 1, 64), dd.CacheMap.empty(1, T, ld)
    m.block_table[0, HELD - 1] = 5
    free, n_free, err = dev_i32(torch, np.arange(16)), dev_i32(torch, [8]), dev_i32(torch, [0])
    length = dev_i32(torch, [2 ** 31 - 9])
    say("plan of", T, "rows,", n_new, "new tokens")
    dd.cache_plan(cc, m, length, dev_i32(torch, [n_new]), dev_i32(torch, [HELD]), free, n_free, n_free, dev_err=err)
    return m, int(n_free.item()), int(err.item())


@pytest.mark.parametrize("T", [64, 9000])          # one launch, and the rows in a second one
def test_positions_that_pass_31_bits_do_not_fit(T):
    torch = torch_or_skip()
    m, n_free, err = _plan(torch, T, 9)
    assert err == dd.DD_DEVERR_CACHE and n_free == 8
    assert int(m.kv_len.item()) == 2 ** 31 - 9 and int(m.held.item()) == HELD and m.row_start.tolist() == [0, 0]
    for x in (m.row_seq, m.row_pos, m.slots):
        assert bool((x == -1).all())
    assert int((m.block_table != -1).sum()) == 1


@pytest.mark.parametrize("T", [64, 9000])
def test_the_last_position(T):
    torch = torch_or_skip()
    m, n_free, err = _plan(torch, T, 8)
    assert err == 0 and n_free == 8 and int(m.kv_len.item()) == 2 ** 31 - 1 and m.row_start.tolist() == [0, 8]
    assert m.row_pos[:8].tolist() == list(range(2 ** 31 - 9, 2 ** 31 - 1)) and m.slots[:8].tolist() == list(range(6 * P - 9, 6 * P - 1))
    assert bool((m.row_seq[8:] == -1).all()) and bool((m.slots[8:] == -1).all())
