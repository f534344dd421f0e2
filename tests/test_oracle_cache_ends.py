"""The oracle's plan at the end of 32-bit positions."""
import numpy as np

from oracle import cache as oc


def test_positions_that_pass_31_bits_do_not_fit():
    held = 1 << 23
    for n, err in ((8, False), (9, True)):
        table = np.full((1, held + 16), -1, np.int32)
        table[0, held - 1] = 5
        w = oc.plan(16, 256, held + 16, 64, np.array([2 ** 31 - 9]), np.array([n]), np.array([held]), table, np.arange(16), 8)
        assert w["err"] == err and int(w["kv_len"][0]) == 2 ** 31 - (9 if err else 1)
        assert (w["slots"] >= 0).sum() == (0 if err else 8)
