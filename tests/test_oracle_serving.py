"""Pins of the oracle's tokens under settings, forks and compactions."""
import numpy as np
import pytest

from oracle import serving as so


def test_choices_of_a_small_row():
    l = np.log(np.array([0.1, 0.4, 0.2, 0.2, 0.1]))
    assert so.choose(l)[0].tolist() == [1, 2, 3, 0, 4]
    assert so.choose(l, top_k=3)[0].tolist() == [1, 2, 3]
    assert so.choose(l, top_p=0.39)[0].tolist() == [1]
    assert so.choose(l, top_p=0.41)[0].tolist() == [1, 2]
    assert so.choose(l, top_p=0.0)[0].tolist() == [1]
    assert so.choose(l, min_p=0.49)[0].tolist() == [1, 2, 3]
    assert so.choose(l, min_p=0.51)[0].tolist() == [1]
    # top-p counts what the others leave: 0.4 of 0.8, 0.6 of 0.8
    assert so.choose(l, top_k=3, top_p=0.6)[0].tolist() == [1, 2]
    assert so.choose(l, temperature=0)[0].tolist() == [1]
    # a temperature of one half squares the weights: 16 4 4 1 1
    assert so.choose(l, temperature=0.5, top_p=16.1 / 26)[0].tolist() == [1, 2]


def test_draws_have_the_shares():
    rng = np.random.default_rng(0)
    l = rng.normal(size=40) * 2
    l[5] = -np.inf
    order, w, _ = so.choose(l, 0.8, 20, 0.95, 0.01)
    n = 200000
    words = (np.arange(n, dtype=np.uint64) * (2 ** 32 // n)).tolist()      # evenly spread
    got = np.bincount([so.token(l, x, temperature=0.8, top_k=20, top_p=0.95, min_p=0.01)[0] for x in words[::50]], minlength=40)
    share = w / w.sum()
    assert set(np.nonzero(got)[0]) <= set(order.tolist())
    assert np.abs(got[order] / got.sum() - share).max() < 2 / (n / 50) * 2
    z, logp, kept, _ = so.token(l, 2 ** 31, temperature=0.8, top_k=20, top_p=0.95, min_p=0.01)
    assert kept == len(order) and abs(logp - np.log(share[order.tolist().index(z)])) < 1e-12


@pytest.mark.parametrize("seed", range(30))
def test_forks_keep_contents_and_blocks(seed):
    """Contents are followed token by token: after the moves, every sequence reads its source's first tokens, no block that a
    sequence appends into belongs to another one, and no block is lost or held and free at once."""
    rng = np.random.default_rng(seed)
    P, nb, ld, S = 4, 60, 6, 5
    perm = rng.permutation(nb)
    held = rng.integers(0, ld + 1, S)
    table = np.full((S, ld), -1)
    at = 0
    for s in range(S):
        table[s, :held[s]] = perm[at:at + held[s]]
        at += held[s]
    ln = [int(rng.integers(max(0, h * P - 5), h * P + 1)) for h in held]
    free = np.concatenate([perm[at:], np.full(at, -1)])
    n_free = nb - at
    tok = {(int(table[s, i // P]), i % P): (s, i) for s in range(S) for i in range(ln[s])}
    want = [[(s, i) for i in range(ln[s])] for s in range(S)]
    for _ in range(4):
        n_to = int(rng.integers(1, 9))
        src = rng.integers(-1, len(held), n_to)
        keep = np.array([rng.integers(max(0, ln[q] - 6), ln[q] + 1) if q >= 0 else 0 for q in src])
        f = so.fork(nb, P, table, held, ln, src, keep, free, n_free, ld)
        assert not f["err"]
        for a, b in f["moves"]:
            for o in range(P):
                tok[b, o] = tok.get((a, o))
        want = [want[q][:k] if q >= 0 else [] for q, k in zip(src, keep)]
        for s, r in enumerate(f["rows"]):
            assert [tok[r[i // P], i % P] for i in range(f["kv_len"][s])] == want[s]
            if f["kv_len"][s] % P:
                assert sum(x == r[-1] for t in f["rows"] for x in t) == 1
        now = {b for r in f["rows"] for b in r}
        assert sorted(list(now) + list(f["free"][:f["n_free"]])) == list(range(nb))
        table = np.full((n_to, ld), -1)
        for s, r in enumerate(f["rows"]):
            table[s, :len(r)] = r
        held, ln, free, n_free = f["held"], f["kv_len"], np.array(f["free"]), f["n_free"]
    c = so.compact(nb, table, held)
    for a, b in c["moves"]:
        for o in range(P):
            tok[b, o] = tok.get((a, o))
    for s, r in enumerate(c["rows"]):
        assert [tok[r[i // P], i % P] for i in range(ln[s])] == want[s]
    now = {b for r in c["rows"] for b in r}
    assert now == set(range(len(now))) and sorted(c["free"] + list(now)) == list(range(nb))


def test_forks_that_do_nothing():
    a = dict(n_blocks=4, P=4, table=[[0, 1], [2, -1]], held=[2, 1], seq_len=[7, 4], src=[0, 0], keep=[7, 7], free=[3, -1, -1, -1], n_free=1, ld_to=2)
    assert not so.fork(**a)["err"]
    for k, v in (("n_free", 5), ("keep", [7, 8]), ("src", [0, 2]), ("src", [-2, 0]), ("ld_to", 1), ("seq_len", [9, 4]), ("held", [2, 2]),
                 ("held", [3, 1])):
        assert so.fork(**dict(a, **{k: v}))["err"], k
    # the ended sequence's block is what the second continuation takes
    f = so.fork(**dict(a, n_free=0))
    assert f["moves"] == [(1, 2)] and f["n_free"] == 0
    assert so.fork(**dict(a, n_free=0, src=[0, 0, 1], keep=[7, 7, 3]))["err"]
