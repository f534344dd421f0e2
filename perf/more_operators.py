"""Operators of serving with several continuations per request, as cases that can be timed and compared.

Kinds (the public entry points of paper_2609_04010_amd._lib, and their plain forms in elementary torch
operations):
  sample     token_sample: a token per draw from rows of logits, with temperature, min-p, top-k and top-p
  truncate   logits_truncate: the same choice of classes as an edit of the logits, for draws and verifications that follow
  fork       cache_fork: block tables of continuations from those of the contexts that they continue
  copy       cache_copy: the blocks that a fork or a compaction lists, in every layer of the cache
  compact    cache_compact: the blocks in use to the lowest numbers of the pool

Classes are ordered by falling logit, the lowest index first among equal ones.  With w = exp((l - max l) / temperature),
min-p keeps w >= min_p, top-k the first k of those, top-p the shortest beginning of these whose weights add up to at least
top_p times their sum.  The token is the first kept class at which the running sum of w exceeds u times the kept sum,
u = (word + 1/2) 2^-32.

Inputs are synthetic and made on the GPU from the seed.
"""
import math

import numpy as np
import torch

own = False

GPT2S_VOCAB = 50257


def listed():
    return [
        # one token each for a handful of requests, usual settings: latency
        dict(name="sample decode S8", kind="sample", dtype="bf16", vocab=GPT2S_VOCAB, draws=8, per=1, stride=1, uses="tkp",
             shape="peaked", banned=0.0, ended=0.0),
        # a full serving batch, every request with settings of its own; each one's last row of a pass of four rows
        dict(name="sample serving S512", kind="sample", dtype="bf16", vocab=GPT2S_VOCAB, draws=512, per=1, stride=4, uses="tgkpm",
             shape="mixed", banned=0.0, ended=0.05),
        # the first tokens of 32 continuations of each of 16 prompts, fp32, flat rows, top-p alone
        dict(name="sample forks fp32", kind="sample", dtype="fp32", vocab=GPT2S_VOCAB, draws=512, per=32, stride=1, uses="tp",
             shape="flat", banned=0.0, ended=0.0),
        # target rows of one small verification: 4 requests of 16 rows
        dict(name="truncate verify S4", kind="truncate", dtype="bf16", vocab=GPT2S_VOCAB, S=4, rows_per_seq=16, uses="tkp",
             shape="peaked", banned=0.0),
        # every row of a large pass, settings per request
        dict(name="truncate posterior S256", kind="truncate", dtype="bf16", vocab=GPT2S_VOCAB, S=256, rows_per_seq=16,
             uses="tgkpm", shape="mixed", banned=0.0),
        # another vocabulary of odd size, fp32, rows that a mask has been over
        dict(name="truncate odd fp32", kind="truncate", dtype="fp32", vocab=32003, S=37, rows_per_seq=9, uses="tpm",
             shape="flat", banned=0.3),
        # a prompt's context goes to sixteen continuations: latency
        dict(name="fork one prompt S16", kind="fork", S=1, S_to=16, ctx=1000, block=64, back=0, mode="one", shared=False, ended=0.0),
        # all continuations of a full batch chosen anew, some tokens dropped, some requests ended
        dict(name="fork resample S1024", kind="fork", S=1024, S_to=1024, ctx=4096, block=64, back=16, mode="resample",
             shared=True, ended=0.05),
        # the partly filled blocks of sixteen continuations, 12 layers
        dict(name="copy continuations S16", kind="copy", layers=12, heads=12, dh=64, block=64, moves=16),
        # a pool that is put in order: a thousand blocks of 12 layers
        dict(name="copy pool 1024", kind="copy", layers=12, heads=12, dh=64, block=64, moves=1024),
        # a small pool, half in use
        dict(name="compact S16", kind="compact", S=16, ctx=1000, block=64, shared=False, room=2.0),
        # a large pool of short blocks whose sequences share prompts
        dict(name="compact S1024", kind="compact", S=1024, ctx=4096, block=32, shared=True, room=1.5),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: vocabularies 32..131072, 1..4096 rows, both types, every mix of settings; 1..1024 sequences of 1..8192
    tokens in blocks of 32..256; 1..1024 blocks copied in 1..24 layers."""
    kind = rng.choice(["sample", "sample", "sample", "truncate", "truncate", "truncate", "fork", "fork", "copy", "copy", "compact"])
    block = rng.choice([32, 64, 64, 128, 256])
    if kind in ("sample", "truncate"):
        dtype = "bf16" if rng.random() < 0.7 else "fp32"
        vocab = rng.choice([GPT2S_VOCAB, GPT2S_VOCAB, _log_int(rng, 32, GPT2S_VOCAB), _log_int(rng, 1024, 131072)])
        most = 4096 * GPT2S_VOCAB // vocab // (1 if dtype == "bf16" else 2)
        uses = "t" * (rng.random() < 0.9) + "g" * (rng.random() < 0.2) + "k" * (rng.random() < 0.5) + "p" * (rng.random() < 0.6) + "m" * (rng.random() < 0.3)
        case = dict(kind=kind, dtype=dtype, vocab=vocab, uses=uses, shape=rng.choice(["peaked", "mixed", "flat"]),
                    banned=rng.choice([0.0, 0.0, 0.3, 0.9]))
        if kind == "truncate":
            per = rng.choice([1, 16, _log_int(rng, 1, 64)])
            return dict(case, S=_log_int(rng, 1, max(1, min(1024, most, 4096) // per)), rows_per_seq=per)
        per = rng.choice([1, 1, 1, rng.randint(2, 32)])
        stride = 1 if per > 1 else rng.choice([1, 1, rng.randint(2, 16)])
        rows = _log_int(rng, 1, max(1, min(1024, most // 4) // (stride * per)))
        return dict(case, draws=rows * per, per=per, stride=stride, ended=rng.choice([0.0, 0.0, 0.1]))
    if kind == "copy":
        layers = rng.choice([1, 12, 24])
        heads, dh = rng.choice([(2, 32), (12, 64), (16, 64), (8, 128), (2, 128)])
        most = 1024 * 12 * 12 * 64 * 64 // (layers * heads * dh * block)
        return dict(kind=kind, layers=layers, heads=heads, dh=dh, block=block, moves=_log_int(rng, 1, max(1, min(1024, most))))
    ctx = _log_int(rng, 1, 8192)
    S = _log_int(rng, 1, max(1, min(1024, 1024 * 4096 // 32 // (ctx // block + 1))))
    if kind == "compact":
        return dict(kind=kind, S=S, ctx=ctx, block=block, shared=rng.random() < 0.5, room=rng.choice([1.0, 1.5, 3.0]))
    one = rng.random() < 0.3
    to = S if rng.random() < 0.5 else _log_int(rng, 1, max(1, min(1024, 1024 * 4096 // 64 // (ctx // block + 1))))
    return dict(kind=kind, S=S, S_to=to, ctx=ctx, block=block, back=rng.choice([0, 1, 16, 300]), mode="one" if one else "resample",
                shared=rng.random() < 0.5, ended=rng.choice([0.0, 0.05, 0.3]))


# ------------------------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _i32(x):
    return x.to(torch.int32)


def _ints(g, lo, hi, n):
    """n whole numbers in [lo, hi]."""
    return torch.randint(int(lo), int(hi) + 1, (n,), generator=g, device="cuda")


def _rand(g, *n):
    return torch.rand(n, generator=g, device="cuda")


def _exp2(e):
    """2^e in fp32 for whole numbers e, -126 <= e <= 127, from its bits."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _logits(case, rows, g):
    """Rows of a language model's logits: a broad body, and in peaked rows a few classes that stand out; banned classes
    are -inf, as masks leave them."""
    V = case["vocab"]
    ld = (V + 63) // 64 * 64
    out = torch.empty((rows, ld), dtype=torch.bfloat16 if case["dtype"] == "bf16" else torch.float32, device="cuda")
    for r in range(0, rows, 1024):
        n = min(1024, rows - r)
        x = torch.randn((n, ld), generator=g, device="cuda").mul_(2.5)
        if case["shape"] != "flat":
            at = torch.randint(0, V, (n, 12), generator=g, device="cuda")
            up = 4.0 + 10.0 * _rand(g, n, 12)
            if case["shape"] == "mixed":
                up = torch.where(_rand(g, n, 1) < 0.5, up, torch.zeros_like(up))
            x.scatter_add_(1, at, up)
        if case["banned"]:
            ban = _rand(g, n, ld) < case["banned"]
            ban[:, 0] = False
            x.masked_fill_(ban, -math.inf)
        out[r:r + n] = x.to(out.dtype)
    return out, ld


def _settings(case, n, g):
    """Temperature, top-k, top-p and min-p of n requests, some of which do without; None for what the program does not use."""
    uses, st = case["uses"], dict(temperature=None, top_k=None, top_p=None, min_p=None)
    off = lambda share: _rand(g, n) < share   # noqa: E731
    if "t" in uses:
        t = 0.5 + _rand(g, n)
        st["temperature"] = torch.where(off(0.1), torch.zeros_like(t), t) if "g" in uses else t
    if "k" in uses:
        k = torch.exp(math.log(min(1000, case["vocab"])) * _rand(g, n))
        st["top_k"] = _i32(torch.where(off(0.2), torch.zeros_like(k), k).floor())
    if "p" in uses:
        p = 0.5 + 0.499 * _rand(g, n)
        st["top_p"] = torch.where(off(0.2), torch.ones_like(p), p)
    if "m" in uses:
        m = 0.2 * _rand(g, n).square()
        st["min_p"] = torch.where(off(0.2), torch.zeros_like(m), m)
    return st


def _contexts(case, g):
    """Block tables of S sequences over a pool, and the stack of its free blocks.  Shared: sequences in groups of eight
    hold the first one's blocks of half their prompts."""
    S, P, ctx = case["S"], case["block"], case["ctx"]
    lens = _ints(g, (ctx + 1) // 2, ctx, S)
    lens[0] = ctx
    held = (lens + P - 1) // P
    ld = -(-ctx // P)
    n_blocks = int(S * ld * case.get("room", 1.0)) + case.get("S_to", 0) + 1
    perm = torch.randperm(n_blocks, generator=g, device="cuda")
    j = torch.arange(ld, device="cuda")
    s = torch.arange(S, device="cuda")
    owner = s[:, None].expand(S, ld)
    if case["shared"]:
        head = s // 8 * 8
        common = torch.minimum(lens, lens[head]) // (2 * P)
        owner = torch.where(j < common[:, None], head[:, None], owner)
    table = torch.where(j < held[:, None], perm[owner * ld + j], torch.full_like(owner, -1))
    used = torch.zeros(n_blocks + 1, dtype=torch.bool, device="cuda").index_fill_(0, table.reshape(-1) % (n_blocks + 1), True)[:-1]
    k = torch.randperm(n_blocks, generator=g, device="cuda")
    k = k[torch.argsort(used[k].to(torch.int8), stable=True)]        # the free ones first, in random order
    n_free = (~used).sum().reshape(1)
    free = torch.where(torch.arange(n_blocks, device="cuda") < n_free, k, torch.full_like(k, -1))
    return dict(n_blocks=n_blocks, ld=ld, table=_i32(table).contiguous(), held=_i32(held), kv_len=_i32(lens), free=_i32(free),
                n_free=_i32(n_free))


def _empty(*n):
    return torch.zeros(n, dtype=torch.int32, device="cuda")


def _map(S, table, held, kv_len):
    """The program's map of a pass; the row maps are not looked at here."""
    from paper_2609_04010_amd import _lib as dd
    return dd.CacheMap(table, held, kv_len, _empty(S + 1), _empty(1), _empty(1), _empty(1))


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    st = dict(case=case)
    if kind == "sample":
        n, per, stride = case["draws"], case["per"], case["stride"]
        rows = n // per * stride
        logits, ld = _logits(case, rows, g)
        at = torch.arange(n, device="cuda") // per * stride + stride - 1
        at = torch.where(_rand(g, n) < case["ended"], torch.full_like(at, -1), at)
        words = torch.randint(-2**31, 2**31, (n,), generator=g, device="cuda", dtype=torch.int64)
        st.update(logits=logits, ld=ld, rows=rows, n=n, row_ids=_i32(at), words=_i32(words), z=_empty(n), kept=_empty(n),
                  logp=torch.zeros(n, device="cuda"), **_settings(case, n // per, g))
        return st
    if kind == "truncate":
        rows = case["S"] * case["rows_per_seq"]
        logits, ld = _logits(case, rows, g)
        st.update(logits=logits, ld=ld, rows=rows, out=torch.zeros_like(logits), kept=_empty(rows), **_settings(case, case["S"], g))
        return st
    if kind == "copy":
        m, layers, heads, dh, P = case["moves"], case["layers"], case["heads"], case["dh"], case["block"]
        n_blocks = 2 * m + m // 2 + 1
        codes = torch.empty((layers, n_blocks, heads, 2 * P * dh), dtype=torch.uint8, device="cuda")
        x = torch.randn((min(n_blocks * layers, 512), heads, 2 * P * dh), generator=g, device="cuda").mul_(100.0).clamp_(-448, 448)
        x = x.to(torch.float8_e4m3fn).view(torch.uint8)
        torch.index_select(x, 0, torch.randint(0, x.shape[0], (layers * n_blocks,), generator=g, device="cuda"),
                           out=codes.view(-1, heads, 2 * P * dh))
        scales = _exp2(torch.randint(-8, -5, (layers, n_blocks, heads, 2), generator=g, device="cuda"))
        perm = torch.randperm(n_blocks, generator=g, device="cuda")
        moves = torch.full((m + m // 4 + 1, 2), -1, device="cuda")   # a program has room for more than a pass needs
        moves[:m, 0], moves[:m, 1] = perm[:m], perm[m:2 * m]
        st.update(n_blocks=n_blocks, codes=codes, scales=scales, moves=_i32(moves).contiguous(),
                  n_moves=torch.full((1,), m, dtype=torch.int32, device="cuda"))
        if own:
            from paper_2609_04010_amd import _lib as dd
            st["cc"] = dd.cache_config(n_blocks, P, heads, dh)
        return st
    c = _contexts(case, g)
    S, ld, n_blocks = case["S"], c["ld"], c["n_blocks"]
    if kind == "compact":
        st.update(c, to_table=torch.full_like(c["table"], -1), free=_empty(n_blocks), n_free_out=_empty(1),
                  moves=_empty(n_blocks // 2 + 1, 2), n_moves=_empty(1))
        if own:
            from paper_2609_04010_amd import _lib as dd
            st["cc"] = dd.cache_config(n_blocks, case["block"], 1, 64)
            st["map"] = _map(S, c["table"], c["held"], c["kv_len"])
            st["ws"] = torch.empty(max(256, dd.cache_compact_workspace_bytes(st["cc"])), dtype=torch.uint8, device="cuda")
        return st
    to = case["S_to"]
    src = torch.zeros(to, dtype=torch.int64, device="cuda")
    if case["mode"] == "resample":                                    # good ones are chosen several times
        src = (S * _rand(g, to).square()).long().clamp(max=S - 1)
    src[1:] = torch.where(_rand(g, to - 1) < case["ended"], torch.full_like(src[1:], -1), src[1:])
    lens = c["kv_len"].long()[src.clamp(min=0)]
    keep = (lens - _ints(g, 0, case["back"], to)).clamp(min=0)
    st.update(c, src=_i32(src), keep=_i32(torch.where(src >= 0, keep, torch.zeros_like(keep))),
              to_table=torch.full((to, ld), -1, dtype=torch.int32, device="cuda"), to_held=_empty(to), to_kv=_empty(to),
              n_free_out=_empty(1), moves=_empty(to, 2), n_moves=_empty(1))
    if own:
        from paper_2609_04010_amd import _lib as dd
        st["cc"] = dd.cache_config(n_blocks, case["block"], 1, 64)
        st["map"] = _map(S, c["table"], c["held"], c["kv_len"])
        st["to"] = _map(to, st["to_table"], st["to_held"], st["to_kv"])
        st["ws"] = torch.empty(max(256, dd.cache_fork_workspace_bytes(st["cc"], S, to)), dtype=torch.uint8, device="cuda")
    return st


# ------------------------------------------------------------------------------------ plain forms

def _at(x, seq, off):
    """Each row's setting [rows][1] in 64 bits; `off` where there is none."""
    if x is None:
        return torch.full((seq.shape[0], 1), off, dtype=torch.float64, device="cuda")
    return x.double()[seq][:, None]


def _kept_plain(l, st, seq):
    """Order of the classes, (l - max l) / temperature and weight in that order (0 for what is not kept), and how many
    are kept, of rows l in 64 bits."""
    t, p, m = _at(st["temperature"], seq, 1.0), _at(st["top_p"], seq, 1.0), _at(st["min_p"], seq, 0.0)
    k = _at(st["top_k"], seq, 0)
    s, order = torch.sort(l, dim=1, descending=True, stable=True)
    rank = torch.arange(l.shape[1], device="cuda")
    x = (s - s[:, :1]) / torch.where(t > 0, t, torch.ones_like(t))
    w = x.exp()
    alive = (s > -math.inf) & (w >= m) & ((rank < k) | (k <= 0)) & ((t > 0) | (rank < 1))
    w = w * alive
    cum = w.cumsum(1)
    alive &= (cum - w < p * cum[:, -1:]) | (p >= 1) | (rank < 1)
    return order, x, w * alive, alive


def _sample_plain(st):
    V, per = st["case"]["vocab"], st["case"]["per"]
    at = st["row_ids"].long()
    live = at >= 0
    seq = torch.arange(st["n"], device="cuda") // per
    order, x, w, alive = _kept_plain(st["logits"][:, :V].double()[at.clamp(min=0)], st, seq)
    kept = alive.sum(1)
    cum = w.cumsum(1)
    u = ((st["words"].long() & 0xFFFFFFFF).double() + 0.5) * 2.0 ** -32
    pos = (cum <= u[:, None] * cum[:, -1:]).sum(1)
    pos = torch.minimum(pos, kept - 1)[:, None]
    logp = (x.gather(1, pos) - cum[:, -1:].log())[:, 0]
    st["z"].copy_(torch.where(live, _i32(order.gather(1, pos)[:, 0]), st["z"]))
    st["kept"].copy_(torch.where(live, _i32(kept), st["kept"]))
    st["logp"].copy_(torch.where(live, logp.float(), st["logp"]))
    return dict(z=st["z"], kept=st["kept"], logp=st["logp"])


def _truncate_plain(st):
    V = st["case"]["vocab"]
    seq = torch.arange(st["rows"], device="cuda") // st["case"]["rows_per_seq"]
    l = st["logits"][:, :V]
    order, _, _, alive = _kept_plain(l.double(), st, seq)
    stays = torch.zeros_like(alive).scatter_(1, order, alive)
    t = _at(st["temperature"], seq, 1.0).float()
    x = l.float() / torch.where(t > 0, t, torch.ones_like(t))
    st["out"][:, :V] = x.masked_fill_(~stays, -math.inf).to(st["out"].dtype)
    st["kept"].copy_(_i32(alive.sum(1)))
    return dict(out=st["out"], kept=st["kept"])


def _held_marks(table, held, n_blocks):
    """Which blocks stand in the held entries of a table; entry n_blocks takes what is not held."""
    live = torch.arange(table.shape[1], device="cuda") < held[:, None]
    at = torch.where(live, table, torch.full_like(table, n_blocks))
    return torch.zeros(n_blocks + 1, dtype=torch.bool, device="cuda").index_fill_(0, at.reshape(-1), True)[:-1]


def _fork_plain(st):
    P, S, to, ld, nb = st["case"]["block"], st["case"]["S"], st["case"]["S_to"], st["ld"], st["n_blocks"]
    table, held, src, keep, n_free = (st[k].long() for k in ("table", "held", "src", "keep", "n_free"))
    n = (keep + P - 1) // P
    j, s = torch.arange(ld, device="cuda"), torch.arange(to, device="cuda")
    live = j < n[:, None]
    t = table[src.clamp(min=0)]
    at = torch.where(live, t, torch.full_like(t, nb))
    # the sequence whose block it stays: any that holds it whole, else the first of those whose last block it is
    part = (keep % P != 0) & (n > 0)
    last = part[:, None] & (j == n[:, None] - 1)
    claim = torch.where(last, s[:, None], torch.full_like(t, -1))
    owner = torch.full((nb + 1,), to, device="cuda").scatter_reduce_(0, at.reshape(-1), claim.reshape(-1), "amin")
    mine = at.gather(1, (n - 1).clamp(min=0)[:, None])[:, 0]
    copies = part & (owner[mine] != s)
    now = owner[:-1] < to
    freed = _held_marks(table, held, nb) & ~now
    top = n_free + freed.sum()
    place = torch.where(freed, n_free + freed.long().cumsum(0) - 1, torch.full_like(owner[:-1], nb))
    free = torch.cat([st["free"].long(), n_free]).scatter_(0, place, torch.arange(nb, device="cuda"))[:-1]
    rank = copies.long().cumsum(0) - 1
    fresh = free[(top - 1 - rank).clamp(0, nb - 1)]
    t = torch.where(last & copies[:, None], fresh[:, None], t)
    row = torch.where(copies, rank, torch.full_like(rank, to))
    moves = torch.cat([st["moves"].long(), torch.zeros((1, 2), dtype=torch.int64, device="cuda")])
    moves = moves.scatter_(0, row[:, None].expand(to, 2), torch.stack([mine, fresh], 1))[:-1]
    return dict(table=_i32(torch.where(live, t, st["to_table"].long())), held=_i32(n), kv_len=_i32(keep), free=_i32(free),
                n_free=_i32(top - copies.sum()), moves=_i32(moves), n_moves=_i32(copies.sum().reshape(1)))


def _copy_plain(st):
    codes, scales, m, nb = st["codes"], st["scales"], st["moves"].long(), st["n_blocks"]
    live = torch.arange(m.shape[0], device="cuda") < st["n_moves"]
    # entries that do not count copy the first one again
    a, b = (torch.where(live, m[:, k], m[0, k]) for k in (0, 1))
    codes[:, b] = codes[:, a]
    scales[:, b] = scales[:, a]
    return dict(codes=codes.view(torch.float8_e4m3fn), scales=scales)


def _compact_plain(st):
    table, held, nb = st["table"].long(), st["held"].long(), st["n_blocks"]
    used = _held_marks(table, held, nb)
    n = used.sum()
    k = torch.arange(nb, device="cuda")
    leave, hole = used & (k >= n), ~used & (k < n)
    rows = st["moves"].shape[0]
    no = torch.full_like(k, rows)
    frm = torch.zeros(rows + 1, dtype=torch.int64, device="cuda").scatter_(0, torch.where(leave, leave.long().cumsum(0) - 1, no), k)
    to = torch.zeros(rows + 1, dtype=torch.int64, device="cuda").scatter_(0, torch.where(hole, hole.long().cumsum(0) - 1, no), k)
    counts = (torch.arange(rows, device="cuda") < leave.sum())[:, None]
    moves = torch.where(counts, torch.stack([frm, to], 1)[:-1], st["moves"].long())
    name = torch.where(leave, to[(leave.long().cumsum(0) - 1).clamp(min=0)], k)
    live = torch.arange(table.shape[1], device="cuda") < held[:, None]
    new = torch.where(live, name[table.clamp(min=0)], st["to_table"].long())
    free = torch.where(k < nb - n, nb - 1 - k, st["free"].long())
    return dict(table=_i32(new), free=_i32(free), n_free=_i32((nb - n).reshape(1)), moves=_i32(moves),
                n_moves=_i32(leave.sum().reshape(1)))


# ------------------------------------------------------------------------------------ one pass

def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        return {"sample": _sample_plain, "truncate": _truncate_plain, "fork": _fork_plain, "copy": _copy_plain,
                "compact": _compact_plain}[kind](st)
    from paper_2609_04010_amd import _lib as dd
    if kind == "sample":
        dd.token_sample(st["logits"], case["dtype"], st["ld"], st["rows"], case["vocab"], st["z"], st["n"], row_ids=st["row_ids"],
                        draws_per_seq=case["per"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"],
                        min_p=st["min_p"], noise_words=st["words"], logp=st["logp"], n_kept=st["kept"])
        return dict(z=st["z"], kept=st["kept"], logp=st["logp"])
    if kind == "truncate":
        dd.logits_truncate(st["logits"], case["dtype"], st["ld"], st["rows"], case["vocab"], st["out"], case["rows_per_seq"],
                           temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"],
                           n_kept=st["kept"])
        return dict(out=st["out"], kept=st["kept"])
    if kind == "fork":
        dd.cache_fork(st["cc"], st["map"], st["to"], st["kv_len"], st["src"], st["free"], st["n_free"], st["n_free_out"],
                      st["moves"], st["n_moves"], st["ws"], keep=st["keep"])
        return dict(table=st["to_table"], held=st["to_held"], kv_len=st["to_kv"], free=st["free"], n_free=st["n_free_out"],
                    moves=st["moves"], n_moves=st["n_moves"])
    if kind == "copy":
        dd.cache_copy(st["cc"], st["codes"], st["scales"], st["moves"], st["n_moves"], layers=case["layers"])
        return dict(codes=st["codes"].view(torch.float8_e4m3fn), scales=st["scales"])
    dd.cache_compact(st["cc"], st["map"], st["to_table"], st["free"], st["n_free_out"], st["moves"], st["n_moves"], st["ws"])
    return dict(table=st["to_table"], free=st["free"], n_free=st["n_free_out"], moves=st["moves"], n_moves=st["n_moves"])


def work(case):
    kind = case["kind"]
    es = 2 if case.get("dtype") == "bf16" else 4
    if kind == "sample":
        n = case["draws"]
        return {"bytes": n / case["per"] * (1 - case["ended"]) * case["vocab"] * es + 20 * n + 16 * n / case["per"], "flops": 0}
    if kind == "truncate":
        rows = case["S"] * case["rows_per_seq"]
        return {"bytes": 2 * rows * case["vocab"] * es + 4 * rows + 16 * case["S"], "flops": 0}
    if kind == "copy":
        return {"bytes": 2 * case["moves"] * case["layers"] * case["heads"] * (2 * case["block"] * case["dh"] + 8), "flops": 0}
    entries = case["S"] * (0.75 * case["ctx"] / case["block"] + 0.5)
    if kind == "compact":
        n_blocks = case["S"] * -(-case["ctx"] // case["block"]) * case["room"]
        return {"bytes": 4 * (2 * entries + case["S"]) + 4 * max(0.0, n_blocks - entries), "flops": 0}
    to = case["S_to"] * (1 - case["ended"])
    return {"bytes": 4 * (entries + 2 * case["S"] + to * (0.75 * case["ctx"] / case["block"] + 0.5) * 2 + 5 * case["S_to"]), "flops": 0}


# ------------------------------------------------------------------------------------ in 64 bits

def _host(x):
    return None if x is None else x.double().cpu().numpy()


def _exact_row(l, t, k, p, m):
    """Classes that stay, in order, and their weights, of one row."""
    order = np.lexsort((np.arange(l.size), -l))
    order = order[np.isfinite(l[order])]
    if t == 0:
        return order[:1], np.ones(1)
    w = np.exp((l[order] - l[order[0]]) / t)
    n = int(np.searchsorted(-w, -m, side="right")) if m > 0 else w.size
    if k > 0:
        n = min(n, int(k))
    if p < 1:
        # the shortest beginning whose weights reach p times the sum
        n = min(n, 1 + int(np.searchsorted(np.cumsum(w[:n]), p * math.fsum(w[:n]), side="left")))
    return order[:n], w[:n]


def _exact_choice(st, r, s, V):
    t, k, p, m = (float(x[s]) if x is not None else off for x, off in
                  ((st["t"], 1.0), (st["k"], 0.0), (st["p"], 1.0), (st["m"], 0.0)))
    return (t, *_exact_row(st["logits"][r, :V].double().cpu().numpy(), t, k, p, m))


def exact(case, seed):
    kind = case["kind"]
    if kind in ("fork", "compact"):
        return None
    if kind == "copy":
        if case["layers"] * case["moves"] * case["heads"] * case["block"] * case["dh"] > 2 ** 27:
            return None
        st = prepare(case, seed)
        val, sc = st["codes"].view(torch.float8_e4m3fn).double(), st["scales"].double()
        for a, b in st["moves"][:int(st["n_moves"])].tolist():
            val[:, b] = val[:, a].clone()
            sc[:, b] = sc[:, a].clone()
        return dict(codes=val, scales=sc)
    rows = case["draws"] if kind == "sample" else case["S"] * case["rows_per_seq"]
    if rows * case["vocab"] > 3 * 10 ** 7:
        return None
    st = prepare(case, seed)
    V = case["vocab"]
    st.update(t=_host(st["temperature"]), k=_host(st["top_k"]), p=_host(st["top_p"]), m=_host(st["min_p"]))
    if kind == "truncate":
        out = st["out"].double()
        for r in range(rows):
            t, stay, _ = _exact_choice(st, r, r // case["rows_per_seq"], V)
            l = st["logits"][r, :V].double()
            at = torch.from_numpy(stay).cuda()
            out[r, :V] = -math.inf
            out[r, at] = l[at] / (t if t > 0 else 1.0)
        return dict(out=out, kept=None)
    logp = torch.zeros(rows, dtype=torch.float64)
    ids, words = st["row_ids"].tolist(), st["words"].tolist()
    for i in range(rows):
        if ids[i] >= 0:
            _, stay, w = _exact_choice(st, ids[i], i // case["per"], V)
            c = np.cumsum(w)
            u = ((words[i] & 0xFFFFFFFF) + 0.5) / 2.0 ** 32
            j = min(int(np.searchsorted(c, u * c[-1], side="right")), w.size - 1)
            logp[i] = math.log(w[j] / c[-1])
    return dict(z=None, kept=None, logp=logp)
