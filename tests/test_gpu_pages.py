"""dd_cache_fork, dd_cache_compact and dd_cache_copy against the oracle, and continuations of a prompt through the
denoiser's cached pass."""
import numpy as np
import pytest

import workloads
from oracle import serving as so
from paper_2609_04010_amd import _lib as dd
from tests.gpu_util import dev_i32, say, torch_or_skip

pytestmark = pytest.mark.gpu


def pool(rng, S, nb, P, ld, most=None, share=False):
    """(table, held, lengths, free, n_free) of S sequences with up to `most` blocks each."""
    held = rng.integers(0, (most or ld) + 1, S)
    while held.sum() > nb:
        held = held // 2
    perm = rng.permutation(nb)
    table, at = np.full((S, ld), -1), 0
    for s in range(S):
        table[s, :held[s]] = perm[at:at + held[s]]
        at += held[s]
    if share:
        for s in range(S):
            if s % 4:
                n = min(held[s], held[s - s % 4]) // 2
                table[s, :n] = table[s - s % 4, :n]
    used = {int(b) for s in range(S) for b in table[s, :held[s]]}
    free = [b for b in perm.tolist() if b not in used]
    lens = np.array([rng.integers(max(0, h * P - P), h * P + 1) for h in held], dtype=np.int64) if S else np.zeros(0, int)
    return table, held, lens, np.array(free + [-1] * (nb - len(free))), len(free)


class Pages:
    def __init__(self, torch, cc, S_to, ld_to, T=1):
        self.torch, self.cc = torch, cc
        self.to = dd.CacheMap.empty(S_to, T, ld_to)
        self.to.held.fill_(-9)
        self.to.kv_len.fill_(-9)
        self.n_out, self.n_moves, self.err = dev_i32(torch, [-9]), dev_i32(torch, [-9]), dev_i32(torch, [0])
        self.moves = dev_i32(torch, np.full((S_to, 2), -9))

    def fork(self, c, src, keep, ws=None, n_free=None):
        torch, cc, to = self.torch, self.cc, self.to
        n_in = dev_i32(torch, [c[4]]) if n_free is None else n_free
        table, held, lens, free, n_free = c
        S = len(held)
        m = dd.CacheMap.empty(S, 1, table.shape[1])
        m.block_table.copy_(dev_i32(torch, table))
        m.held.copy_(dev_i32(torch, held))
        self.free = dev_i32(torch, free)
        ws = torch.full((dd.cache_fork_workspace_bytes(cc, S, to.S),), 255, dtype=torch.uint8, device="cuda") if ws is None else ws
        dd.cache_fork(cc, m, to, dev_i32(torch, lens), dev_i32(torch, src), self.free, n_in, self.n_out, self.moves,
                      self.n_moves, ws, keep=None if keep is None else dev_i32(torch, keep), dev_err=self.err)
        assert np.array_equal(m.block_table.cpu().numpy(), table) and np.array_equal(m.held.cpu().numpy(), held)

    def same(self, w, before):
        """The call's outputs are the oracle's."""
        t, moves = self.to.block_table.cpu().numpy(), self.moves.cpu().numpy()
        assert (int(self.err.item()) == dd.DD_DEVERR_CACHE) == w["err"]
        assert self.to.held.tolist() == w["held"] and self.to.kv_len.tolist() == w["kv_len"]
        for s, r in enumerate(w["rows"]):
            assert t[s, :len(r)].tolist() == r and (t[s, len(r):] == -1).all(), s
        n = len(w["moves"])
        assert int(self.n_moves.item()) == n and [tuple(x) for x in moves[:n].tolist()] == w["moves"] and (moves[n:] == -9).all()
        assert int(self.n_out.item()) == w["n_free"]
        assert self.free.tolist() == [int(b) for b in (before[3] if w["err"] and not n else w["free"])]


FORK = [  # sequences, new ones, blocks, P, entries per row of both tables
    (1, 1, 1, 32, 1, 1), (1, 16, 40, 64, 16, 16), (5, 5, 60, 32, 9, 9), (3, 40, 300, 128, 70, 70), (64, 64, 700, 64, 8, 8),
    (200, 150, 9000, 32, 30, 33), (65, 1, 16500, 256, 200, 190), (1000, 1024, 30000, 32, 25, 25), (7, 300, 8192, 64, 300, 300),
    (4, 4, 8193, 64, 2000, 2000), (0, 3, 10, 32, 4, 4), (5, 0, 30, 32, 4, 4),
    (128, 128, 3000, 32, 8, 8), (129, 100, 3000, 64, 8, 8), (100, 129, 3000, 64, 8, 8), (8193, 300, 20000, 32, 3, 3), (600, 8200, 9000, 32, 3, 5)]


@pytest.mark.parametrize("S,to,nb,P,ld,ld_to", FORK)
@pytest.mark.parametrize("how", ["all", "some", "one"])
def test_forks_against_oracle(S, to, nb, P, ld, ld_to, how):
    torch = torch_or_skip()
    rng = np.random.default_rng(S * 1000 + to + nb)
    c = pool(rng, S, nb, P, ld, most=min(ld, ld_to, max(1, nb // max(1, S))), share=how == "some")
    src = rng.integers(0, S, to) if S else np.full(to, -1)
    if how == "some":
        src[rng.random(to) < 0.3] = -1
        keep = np.array([rng.integers(0, c[2][q] + 1) if q >= 0 else -77 for q in src], dtype=np.int64)
    elif how == "one" and S:
        src[:] = S // 2
        keep = np.full(to, c[2][S // 2])
        keep[1::3] = np.maximum(0, keep[1::3] - 1)
    else:
        keep = None
    cc = dd.cache_config(nb, P, 1, 32)
    p = Pages(torch, cc, to, ld_to)
    say("fork", S, to, nb, P, how)
    p.fork(c, src, keep)
    w = so.fork(nb, P, c[0], c[1], c[2], src, keep, c[3], c[4], ld_to)
    p.same(w, c)


BAD = [dict(held=(1, -1)), dict(held=(1, 7)), dict(lens=(0, -1)), dict(lens=(2, 10 ** 6)), dict(src=(0, -2)), dict(src=(3, 4)), dict(keep=(1, -1)),
       dict(keep=(2, 10 ** 6)), dict(table=(0, 50)), dict(table=(0, -1)), dict(table=(3, 2 ** 31 - 1)), dict(table=(3, -2 ** 31)), dict(n_free=-1),
       dict(n_free=51), dict(n_free=0)]


@pytest.mark.parametrize("bad", BAD, ids=[f"{k}-{v}" for b in BAD for k, v in b.items()])
def test_forks_that_do_not_fit(bad):
    torch = torch_or_skip()
    rng = np.random.default_rng(3)
    table, held, lens, free, n_free = pool(rng, 4, 50, 32, 6)
    held[:] = 6
    table[:] = np.arange(24).reshape(4, 6)
    lens[:] = [170, 192, 161, 180]
    free[:], n_free = np.concatenate([np.arange(24, 50), np.full(24, -1)]), 26
    src, keep = np.array([0, 0, 1, 2, 2, 3]), np.array([170, 169, 33, 1, 160, 64])
    if "n_free" in bad and bad["n_free"] == 0:
        src[:], keep[:] = 0, 161                     # nothing ends but the others' blocks: too few if they stay
        src[1:4] = [1, 2, 3]
        keep[:] = [161, 192, 161, 180, 161, 161]
    c = dict(table=table.reshape(-1), held=held, lens=lens, src=src, keep=keep)
    for k, v in bad.items():
        if k == "n_free":
            n_free = v
        else:
            c[k][v[0]] = v[1]
    cc = dd.cache_config(50, 32, 1, 32)
    p = Pages(torch, cc, 6, 6)
    state = (table, held, lens, free, n_free)
    p.fork(state, src, keep)
    w = so.fork(50, 32, table, held, lens, src, keep, free, n_free, 6)
    assert w["err"] and int(p.err.item()) == dd.DD_DEVERR_CACHE
    assert p.to.held.tolist() == [0] * 6 and p.to.kv_len.tolist() == [0] * 6 and int(p.n_moves.item()) == 0
    assert int(p.n_out.item()) == n_free and p.free.tolist() == free.tolist()


@pytest.mark.parametrize("S", [16, 300, 20000])
def test_the_stack_and_its_height_in_place(S):
    """n_free_out may be n_free: workgroups that begin late still see the height before the call."""
    torch = torch_or_skip()
    rng = np.random.default_rng(S)
    nb, P, ld = 3 * S, 32, 2
    c = pool(rng, S, nb, P, ld)
    src = rng.integers(0, S, S)
    w = so.fork(nb, P, c[0], c[1], c[2], src, None, c[3], c[4], ld)
    p = Pages(torch, dd.cache_config(nb, P, 1, 32), S, ld)
    p.n_out.fill_(c[4])
    p.fork(c, src, None, n_free=p.n_out)
    p.same(w, c)


def test_a_stack_with_a_wrong_number():
    torch = torch_or_skip()
    table, held, lens = np.array([[2, 3]]), np.array([2]), np.array([40])
    for wrong in (-1, 8):
        free = np.array([0, wrong, -1, -1, -1, -1, -1, -1])
        p = Pages(torch, dd.cache_config(8, 32, 1, 32), 2, 2)
        p.fork((table, held, lens, free, 2), np.array([0, 0]), None)
        assert int(p.err.item()) == dd.DD_DEVERR_CACHE and p.to.block_table.tolist() == [[2, 3], [2, wrong]] and int(p.n_out.item()) == 1


COMPACT = [(1, 1, 32, 1), (5, 60, 32, 9), (64, 2000, 64, 8), (300, 9000, 32, 30), (2, 8192, 64, 100), (1000, 40000, 32, 20), (4, 30, 32, 6), (0, 40, 32, 3), (128, 8000, 32, 9),
           (129, 8000, 32, 9), (4000, 30000, 32, 6)]


@pytest.mark.parametrize("S,nb,P,ld", COMPACT)
@pytest.mark.parametrize("place", ["new", "same"])
@pytest.mark.parametrize("share", [False, True])
def test_compactions_against_oracle(S, nb, P, ld, place, share):
    torch = torch_or_skip()
    rng = np.random.default_rng(S + nb)
    table, held, _, free, _ = pool(rng, S, nb, P, ld, share=share)
    cc = dd.cache_config(nb, P, 1, 32)
    m = dd.CacheMap.empty(S, 1, ld)
    m.block_table.copy_(dev_i32(torch, table))
    m.held.copy_(dev_i32(torch, held))
    out = m.block_table if place == "same" else torch.full_like(m.block_table, -1)
    f, n_out, n_moves, err = dev_i32(torch, np.full(nb, -9)), dev_i32(torch, [-9]), dev_i32(torch, [-9]), dev_i32(torch, [0])
    moves = dev_i32(torch, np.full((max(1, nb // 2), 2), -9))
    ws = torch.full((dd.cache_compact_workspace_bytes(cc),), 255, dtype=torch.uint8, device="cuda")
    say("compact", S, nb, P, place)
    dd.cache_compact(cc, m, out, f, n_out, moves, n_moves, ws, dev_err=err)
    w = so.compact(nb, table, held)
    n, nf = len(w["moves"]), len(w["free"])
    got = out.cpu().numpy()
    assert int(err.item()) == 0 and int(n_out.item()) == nf and int(n_moves.item()) == n
    assert f.tolist() == w["free"] + [-9] * (nb - nf)
    assert [tuple(x) for x in moves[:n].tolist()] == w["moves"] and (moves[n:] == -9).all()
    for s in range(S):
        assert got[s, :held[s]].tolist() == w["rows"][s] and (got[s, held[s]:] == -1).all()


@pytest.mark.parametrize("where,value", [("held", -1), ("held", 7), ("table", -1), ("table", 50)])
def test_compactions_that_do_not_fit(where, value):
    torch = torch_or_skip()
    rng = np.random.default_rng(1)
    table, held, _, _, _ = pool(rng, 4, 50, 32, 6)
    held[:] = 6
    table[:] = rng.permutation(50)[:24].reshape(4, 6)
    (held if where == "held" else table[2])[2] = value
    cc = dd.cache_config(50, 32, 1, 32)
    m = dd.CacheMap.empty(4, 1, 6)
    m.block_table.copy_(dev_i32(torch, table))
    m.held.copy_(dev_i32(torch, held))
    out, f = torch.full_like(m.block_table, -5), dev_i32(torch, np.arange(50))
    n_out, n_moves, err, moves = dev_i32(torch, [3]), dev_i32(torch, [4]), dev_i32(torch, [0]), dev_i32(torch, np.full((25, 2), -9))
    ws = torch.zeros(dd.cache_compact_workspace_bytes(cc), dtype=torch.uint8, device="cuda")
    dd.cache_compact(cc, m, out, f, n_out, moves, n_moves, ws, dev_err=err)
    assert int(err.item()) == dd.DD_DEVERR_CACHE and int(n_out.item()) == 3 and int(n_moves.item()) == 0
    assert f.tolist() == list(range(50)) and (moves == -9).all()
    for s in range(4):
        n = held[s] if 0 <= held[s] <= 6 else 0
        assert out[s].tolist() == table[s, :n].tolist() + [-5] * (6 - n)


@pytest.mark.parametrize("layers,heads,dh,P,nb,n", [(1, 1, 32, 32, 2, 1), (3, 2, 64, 64, 40, 13), (2, 5, 128, 256, 30, 15), (24, 12, 64, 64, 9, 4),
                                                    (1, 1, 32, 32, 5000, 2500)])
def test_copies(layers, heads, dh, P, nb, n):
    """Every byte of the listed blocks and no other; entries past the count, past the list and out of range are left out."""
    torch = torch_or_skip()
    rng = np.random.default_rng(nb)
    cc = dd.cache_config(nb, P, heads, dh)
    codes, scales = dd.cache_tensors(cc, layers=layers)
    g = torch.Generator(device="cuda").manual_seed(nb)
    codes.copy_(torch.randint(0, 256, codes.shape, generator=g, device="cuda", dtype=torch.uint8))
    scales.copy_(torch.rand(scales.shape, generator=g, device="cuda"))
    perm = rng.permutation(nb)
    moves = np.full((n + 3, 2), 0)
    moves[:n] = np.stack([perm[:n], perm[n:2 * n]], 1)
    err = dev_i32(torch, [0])
    for count, bad in ((0, None), (n, None), (n + 99, (-1, nb)), (n - 1, (nb, 0)), (-5, None)):
        c, s = codes.clone(), scales.clone()
        mv = moves.copy()
        if bad is not None:
            mv[n:] = bad
            if count < n:
                mv[0] = bad
        a, b = torch.from_numpy(mv[:max(0, min(count, n)), 0]).cuda(), torch.from_numpy(mv[:max(0, min(count, n)), 1]).cuda()
        if bad is not None and count < n:
            a, b = a[1:], b[1:]
        wc, wsc = c.clone(), s.clone()
        wc[:, b], wsc[:, b] = c[:, a], s[:, a]
        err.zero_()
        dd.cache_copy(cc, c, s, dev_i32(torch, mv), dev_i32(torch, [count]), layers=layers, dev_err=err)
        assert torch.equal(c, wc) and torch.equal(s, wsc), count
        assert (int(err.item()) == dd.DD_DEVERR_CACHE) == (bad is not None and (count > n or count > 0))


def test_a_pool_of_many_ranges():
    """More ranges than CUs: as few parts as one."""
    torch = torch_or_skip()
    rng = np.random.default_rng(2)
    S, nb, P, ld = 90, 2_200_000, 32, 40
    c = pool(rng, S, nb, P, ld)
    cc = dd.cache_config(nb, P, 1, 32)
    src = rng.integers(0, S, 70)
    p = Pages(torch, cc, 70, ld)
    p.fork(c, src, None)
    p.same(so.fork(nb, P, c[0], c[1], c[2], src, None, c[3], c[4], ld), c)
    w = so.compact(nb, c[0], c[1])
    m = dd.CacheMap.empty(S, 1, ld)
    m.block_table.copy_(dev_i32(torch, c[0]))
    m.held.copy_(dev_i32(torch, c[1]))
    f, n_out, n_moves, moves = dev_i32(torch, np.zeros(nb)), dev_i32(torch, [0]), dev_i32(torch, [0]), dev_i32(torch, np.zeros((nb // 2, 2)))
    dd.cache_compact(cc, m, m.block_table, f, n_out, moves, n_moves, torch.full((dd.cache_compact_workspace_bytes(cc),), 255, dtype=torch.uint8,
                                                                                 device="cuda"))
    n = len(w["moves"])
    assert int(n_moves.item()) == n and [tuple(x) for x in moves[:n].tolist()] == w["moves"]
    assert f[:int(n_out.item())].tolist() == w["free"]
    got = m.block_table.cpu().numpy()
    assert all(got[s, :c[1][s]].tolist() == w["rows"][s] for s in range(S))


def test_copies_past_32_bits():
    torch = torch_or_skip()
    cc = dd.cache_config(600, 256, 8, 128)
    codes, scales = dd.cache_tensors(cc, layers=9)                       # 2.8 GB
    codes[8, 500] = 77
    codes[0, 3] = 5
    scales[8, 500] = 2.0
    moves = dev_i32(torch, [[500, 599], [3, 4]])
    dd.cache_copy(cc, codes, scales, moves, dev_i32(torch, [2]), layers=9)
    assert (codes[8, 599] == 77).all() and (scales[8, 599] == 2).all() and (codes[0, 4] == 5).all() and (codes[:8, 599] == 0).all()
    assert int((codes != 0).sum()) == 4 * codes[0, 0].numel()


def test_continuations_of_prompts_through_the_denoiser():
    """Three prompts in a pool: forked (all and parts), every continuation adds tokens drawn from its truncated logits, some end, the pool
    is put in order, and another pass runs.  Every pass's logits are those, bit for bit, of a second program that keeps a
    copy of each context in blocks of its own."""
    torch = torch_or_skip()
    cfg = workloads.model_cfg(2, n_layers=2, vocab=300, max_len=256)
    V, P, ld, nb, T = 300, 32, 8, 60, 160
    ldl = int(dd.logits_ld(V))
    params = torch.zeros(dd.param_bytes(cfg), dtype=torch.uint8, device="cuda")
    dd.init_params(cfg, params, seed=3)
    H = cfg["n_heads"]
    rng = np.random.default_rng(6)

    class Program:
        def __init__(self):
            self.cc = dd.cache_config(nb, P, H, 64)
            self.codes, self.scales = dd.cache_tensors(self.cc, layers=2)
            self.free, self.n_free = dev_i32(torch, np.random.default_rng(1).permutation(nb)), dev_i32(torch, [nb])

        def start(self, S):
            self.m = dd.CacheMap.empty(S, T, ld)
            self.length = dev_i32(torch, np.zeros(S))

        def step(self, n_new, z):
            m = self.m
            ws = torch.zeros(dd.cached_workspace_bytes(cfg, self.cc, m.S, T, T, 256), dtype=torch.uint8, device="cuda")
            err = ws[:4].view(torch.int32)
            dd.cache_plan(self.cc, m, self.length, dev_i32(torch, n_new), m.held, self.free, self.n_free, self.n_free, dev_err=err)
            logits = torch.zeros((T, ldl), dtype=torch.bfloat16, device="cuda")
            dd.denoise_forward_cached(cfg, params, z, 1.0, self.cc, self.codes, self.scales, m, logits, ldl, ws, T, 256)
            assert dd.read_device_error(err) == 0
            self.length = m.kv_len.clone()
            return logits

    a, b = Program(), Program()
    a.start(3)
    b.start(3)
    n0 = [70, 33, 32]
    z = dev_i32(torch, rng.integers(0, V, T))
    la, lb = a.step(n0, z), b.step(n0, z)
    assert torch.equal(la[:135], lb[:135])
    hist = [z.tolist()[:70], z.tolist()[70:103], z.tolist()[103:135]]
    for src, keep, new in (([0, 0, 0, 1, 2, 2], [70, 70, 65, 33, 32, 32], [3, 1, 40, 2, 5, 1]), ([1, 1, 3, 3, 5, 0, 2], None, [1, 2, 1, 1, 1, 3, 6])):
        S = len(src)
        # the program with shared blocks
        old, a.m = a.m, dd.CacheMap.empty(S, T, ld)
        moves, n_moves, err = dev_i32(torch, np.zeros((S, 2))), dev_i32(torch, [0]), dev_i32(torch, [0])
        ws = torch.empty(dd.cache_fork_workspace_bytes(a.cc, old.S, S), dtype=torch.uint8, device="cuda")
        dd.cache_fork(a.cc, old, a.m, a.length, dev_i32(torch, src), a.free, a.n_free, a.n_free, moves, n_moves, ws,
                      keep=None if keep is None else dev_i32(torch, keep), dev_err=err)
        dd.cache_copy(a.cc, a.codes, a.scales, moves, n_moves, layers=2, dev_err=err)
        a.length = a.m.kv_len.clone()
        if keep is None:                             # the pool in order, then the same again
            mv2 = dev_i32(torch, np.zeros((nb // 2, 2)))
            ws2 = torch.empty(dd.cache_compact_workspace_bytes(a.cc), dtype=torch.uint8, device="cuda")
            dd.cache_compact(a.cc, a.m, a.m.block_table, a.free, a.n_free, mv2, n_moves, ws2, dev_err=err)
            dd.cache_copy(a.cc, a.codes, a.scales, mv2, n_moves, layers=2, dev_err=err)
            used = a.m.block_table[a.m.block_table >= 0]
            say("moves of the compaction", int(n_moves.item()), "blocks in use", len(set(used.tolist())))
            assert int(used.max().item()) + 1 == len(set(used.tolist())) == nb - int(a.n_free.item())
        assert int(err.item()) == 0
        # the other one copies whole contexts into blocks of their own
        kl = [len(hist[q]) if keep is None else keep[i] for i, q in enumerate(src)]
        tb, held = b.m.block_table.cpu().numpy(), [-(-k // P) for k in kl]
        fresh = [x for x in range(nb) if x not in set(tb[tb >= 0].tolist())]
        c2, s2 = b.codes.clone(), b.scales.clone()
        table = np.full((S, ld), -1)
        at = iter(np.random.default_rng(2).permutation(nb).tolist())
        for i, q in enumerate(src):
            for j in range(held[i]):
                table[i, j] = next(at)
                c2[:, table[i, j]], s2[:, table[i, j]] = b.codes[:, tb[q, j]], b.scales[:, tb[q, j]]
        b.codes, b.scales = c2, s2
        free = [x for x in range(nb) if x not in set(table[table >= 0].tolist())]
        b.start(S)
        b.m.block_table.copy_(dev_i32(torch, table))
        b.m.held.copy_(dev_i32(torch, held))
        b.length = dev_i32(torch, kl)
        b.free, b.n_free = dev_i32(torch, free + [-1] * (nb - len(free))), dev_i32(torch, [len(free)])
        del fresh
        # the first new token of each is drawn from its source's last row, under settings of its own
        z = rng.integers(0, V, T)
        rows = np.cumsum([0] + n0)[1:] - 1
        t = torch.tensor(rng.uniform(0.5, 2, S), dtype=torch.float32, device="cuda")
        k = dev_i32(torch, rng.integers(1, 40, S))
        first = dev_i32(torch, np.zeros(S))
        ids = dev_i32(torch, [rows[q] for q in src])
        dd.token_sample(la, "bf16", ldl, T, V, first, S, row_ids=ids, temperature=t, top_k=k, top_p=torch.full((S,), 0.9, device="cuda"), seed=5,
                        dev_err=err)
        start = np.cumsum([0] + new)
        zd = dev_i32(torch, z)
        zd[torch.from_numpy(start[:-1]).cuda()] = first
        n = int(start[-1])
        la, lb = a.step(new, zd), b.step(new, zd)
        assert torch.equal(la[:n], lb[:n]) and la[:n, :V].isfinite().all()
        z = zd.tolist()
        hist = [hist[q][:kl[i]] + z[start[i]:start[i + 1]] for i, q in enumerate(src)]
        assert a.length.tolist() == [len(h) for h in hist] == b.length.tolist()
        n0 = new


def test_fork_and_copy_captured():
    """Replays of a captured fork, copy and compaction equal the eager calls on the same tables."""
    torch = torch_or_skip()
    rng = np.random.default_rng(9)
    S, nb, P, ld = 50, 900, 32, 12
    cc = dd.cache_config(nb, P, 2, 32)
    codes, scales = dd.cache_tensors(cc)
    m = dd.CacheMap.empty(S, 1, ld)
    seq, src, free, n_free = (dev_i32(torch, np.zeros(n)) for n in (S, S, nb, 1))
    wf = torch.empty(dd.cache_fork_workspace_bytes(cc, S, S), dtype=torch.uint8, device="cuda")
    wc = torch.empty(dd.cache_compact_workspace_bytes(cc), dtype=torch.uint8, device="cuda")

    def outs():
        z = lambda *n: dev_i32(torch, np.full(n, -1))   # noqa: E731
        return dict(to=dd.CacheMap.empty(S, 1, ld), free=z(nb), n_out=z(1), moves=z(S, 2), n_moves=z(1), t2=z(S, ld), f2=z(nb), n2=z(1),
                    mv2=z(nb // 2, 2), nm2=z(1), codes=codes.clone(), scales=scales.clone())

    def call(o):
        o["free"].copy_(free)
        o["codes"].copy_(codes)
        dd.cache_fork(cc, m, o["to"], seq, src, o["free"], n_free, o["n_out"], o["moves"], o["n_moves"], wf)
        dd.cache_copy(cc, o["codes"], o["scales"], o["moves"], o["n_moves"])
        dd.cache_compact(cc, o["to"], o["t2"], o["f2"], o["n2"], o["mv2"], o["nm2"], wc)

    def fill():
        c = pool(rng, S, nb, P, ld)
        for x, v in ((m.block_table, c[0]), (m.held, c[1]), (seq, c[2]), (free, c[3]), (n_free, [c[4]]), (src, rng.integers(-1, S, S))):
            x.copy_(dev_i32(torch, v))
        codes.copy_(torch.randint(0, 255, codes.shape, device="cuda", dtype=torch.uint8))

    a, b = outs(), outs()
    fill()
    call(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(a)
    for _ in range(4):
        fill()
        graph.replay()
        call(b)
        torch.cuda.synchronize()
        for k in a:
            if k == "to":
                assert torch.equal(a[k].held, b[k].held) and torch.equal(a[k].kv_len, b[k].kv_len)
                live = torch.arange(ld, device="cuda") < a[k].held[:, None]
                assert torch.equal(a[k].block_table[live], b[k].block_table[live])
            elif k in ("free", "f2"):
                n = int((a["n_out"] if k == "free" else a["n2"]).item())
                assert torch.equal(a[k][:n], b[k][:n])
            elif k in ("moves", "mv2"):
                n = int((a["n_moves"] if k == "moves" else a["nm2"]).item())
                assert torch.equal(a[k][:n], b[k][:n])
            elif k == "t2":
                assert torch.equal(a[k][live], b[k][live])
            else:
                assert torch.equal(a[k], b[k]), k
