"""Pins of the cached context's oracle: the e4m3 numbers against torch's conversion, scales against their
definition, plans by their invariants, attention and edits on cases with known answers."""
import math

import numpy as np
import pytest

from oracle import cache as oc


def test_e4m3_codes_match_torch():
    torch = pytest.importorskip("torch")
    val = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.isnan(val), np.isnan(oc.e4m3_values()))
    assert np.array_equal(val[~np.isnan(val)], oc.e4m3_values()[~np.isnan(val)])
    rng = np.random.default_rng(0)
    pos = oc.e4m3_values()[:127]
    x = np.concatenate([pos, (pos[1:] + pos[:-1]) / 2, rng.uniform(-448, 448, 4000), 2.0 ** rng.uniform(-12, 8, 4000),
                        [0.0, -0.0, math.inf, -math.inf, math.nan]]).astype(np.float32)
    x = np.concatenate([x, -x])
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    got = oc.encode(x)
    nan = ~np.isfinite(x)
    assert np.array_equal(got[~nan], want[~nan]) and ((got[nan] & 127) == 127).all()


@pytest.mark.parametrize("a,e", [(448.0, 0), (448.0001, 1), (449.0, 1), (224.0, -1), (1.75, -8), (1.7500001, -7), (2.0, -7),
                                 (0.0, -100), (1e-45, -100), (3.4028234e38, 120)])
def test_scale_exponent(a, e):
    assert oc.scale_exponent(a) == e
    assert a <= 448 * 2.0 ** e


def test_plan_walks_a_batch_through_its_life():
    """Admit, decode, reject, end: blocks are conserved, no block is held twice, slots follow positions."""
    rng = np.random.default_rng(1)
    n_blocks, P, S, ld = 24, 32, 4, 6
    table, held, length = np.full((S, ld), -1), np.zeros(S, int), np.zeros(S, int)
    free, n_free = rng.permutation(n_blocks), n_blocks
    for step in range(60):
        n_new = rng.integers(0, 40, S)
        n_new[rng.random(S) < 0.2] = -1
        n_new = np.where((length + n_new > ld * P) | (rng.random(S) < 0.1), -1, n_new)
        o = oc.plan(n_blocks, P, ld, 256, length, n_new, held, table, free, n_free)
        assert not o["err"]
        table, held, free, n_free = o["table"], o["held"], o["free"], o["n_free"]
        owned = [b for s in range(S) for b in table[s, :held[s]]]
        assert sorted(owned + list(free[:n_free])) == list(range(n_blocks))
        live = o["row_seq"] >= 0
        assert live.sum() == np.maximum(n_new, 0).sum() and len(set(o["slots"][live])) == live.sum()
        assert np.array_equal(o["kv_len"], np.where(n_new < 0, 0, length + n_new))
        length = o["kv_len"] - np.minimum(o["kv_len"], rng.integers(0, 9, S))     # some tokens are rejected


def test_plan_does_nothing_where_it_does_not_fit():
    free = np.arange(4)
    o = oc.plan(4, 32, 8, 64, [0, 0], [64, 65], [0, 0], np.full((2, 8), -1), free, 4)     # 2 + 3 blocks of 4
    assert o["err"] and o["n_free"] == 4 and (o["held"] == 0).all() and (o["slots"] == -1).all()


def test_append_and_gather_return_what_was_written():
    rng = np.random.default_rng(2)
    P, H, dh = 32, 2, 32
    codes, scales = np.zeros((4, H, 2 * P * dh), np.uint8), np.ones((4, H, 2))
    k, v = rng.normal(size=(40, H, dh)), rng.normal(size=(40, H, dh))
    slots = np.concatenate([2 * P + np.arange(32), 1 * P + np.arange(8)])
    c, s = oc.append(codes, scales, P, k, v, [0, 40], slots)
    gk, gv = oc.gather(c, s, P, dh, [2, 1], 40)
    assert np.abs(gk - k).max() <= np.abs(k).max() * 2.0 ** -4 and np.abs(gv - v).max() <= np.abs(v).max() * 2.0 ** -4
    # eight more tokens, larger ones: the block's scale grows and the older codes are rounded again, exactly
    # where they stay normal numbers
    c2, s2 = oc.append(c, s, P, 64 * k[:8], 64 * v[:8], [0, 8], 1 * P + 8 + np.arange(8))
    assert (s2[1] > s[1]).all() and np.array_equal(s2[2], s[2])
    gk2, _ = oc.gather(c2, s2, P, dh, [2, 1], 48)
    big = np.abs(gk[32:40]) >= 2.0 ** -6 * s2[1, :, 0][None, :, None]
    assert np.array_equal(gk2[32:40][big], gk[32:40][big]) and np.array_equal(gk2[:32], gk[:32])


def test_attention_by_hand():
    q = np.zeros((2, 1, 32))
    k = np.zeros((3, 1, 32))
    v = np.arange(3)[:, None, None] * np.ones((3, 1, 32))
    out = oc.attention(q, k, v, 1, True, 1.0)
    assert np.allclose(out[0], 0.5) and np.allclose(out[1], 1.0)
    assert (oc.attention(q, k[:0], v[:0], 0, False, 1.0) == 0).all()


def test_edit_by_hand():
    l = np.array([[2.0, -2.0, 1.0, 0.5]])
    out = oc.edit(l, [0], history=[[0, 1, 1, 9, -1]], repetition=[2.0], presence=[0.5], frequency=[0.25],
                  bias=[[(2, 1.0), (3, 5.0), (2, 7.0)]], allow=[np.array([1, 1, 1, 0], bool)])
    assert np.array_equal(out, [[1.0 - 0.75, -4.0 - 1.0, 8.0, -math.inf]])
    assert np.array_equal(oc.edit(l, [0], history=[[0]], hist_len=[-1], presence=[1.0]), l)
