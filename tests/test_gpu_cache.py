"""The cached context on the GPU (dd_cache_plan, dd_cache_append, dd_cache_attention) against the float64
oracle: plans and codes exactly, attention within bounds that follow from its roundings."""
import numpy as np
import pytest

from oracle import cache as oc
from paper_2609_04010_amd import _lib as dd
from tests.gpu_util import dev_i32, say, torch_or_skip

pytestmark = pytest.mark.gpu


def _cpu(t):
    return t.cpu().numpy()


# ---------------------------------------------------------------- plan

def _plan_gpu(torch, n_blocks, P, T, length, n_new, held, table, free, n_free, alias=False):
    S, ld = table.shape
    cc = dd.cache_config(n_blocks, P, 1, 64)
    m = dd.CacheMap.empty(S, T, ld)
    m.block_table.copy_(dev_i32(torch, table))
    fr, nf, err = dev_i32(torch, free), dev_i32(torch, [n_free]), dev_i32(torch, [0])
    ln, hd, nn = dev_i32(torch, length), dev_i32(torch, held), dev_i32(torch, n_new)
    if alias:                       # the arrays in place: held and lengths of the map itself, one counter
        m.held.copy_(hd)
        m.kv_len.copy_(ln)
        ln, hd, nout = m.kv_len, m.held, nf
    else:
        nout = dev_i32(torch, [-7])
    dd.cache_plan(cc, m, ln, nn, hd, fr, nf, nout, dev_err=err)
    return dict(table=_cpu(m.block_table), free=_cpu(fr), kv_len=_cpu(m.kv_len), held=_cpu(m.held), row_start=_cpu(m.row_start),
                row_seq=_cpu(m.row_seq), row_pos=_cpu(m.row_pos), slots=_cpu(m.slots), n_free=int(nout.item())), int(err.item())


def _same_plan(got, err, want):
    assert bool(err) == want["err"] and err in (0, dd.DD_DEVERR_CACHE)
    for k in got:
        assert np.array_equal(got[k], want[k]), k


@pytest.mark.parametrize("S,new,ctx,P,ld,T", [(1, 1, 0, 32, 1, 1), (3, 5, 40, 32, 4, 20), (1024, 3, 200, 64, 8, 4000),
                                              (1025, 2, 90, 32, 6, 2100), (2500, 9, 300, 128, 5, 24000),
                                              (70, 400, 0, 256, 4, 30000)])
@pytest.mark.parametrize("alias", [False, True])
def test_plan_equals_oracle(S, new, ctx, P, ld, T, alias):
    torch = torch_or_skip()
    rng = np.random.default_rng(S * 7 + new)
    n_blocks = S * ld
    length = rng.integers(0, ctx + 1, S)
    n_new = rng.integers(0, new + 1, S)
    n_new[rng.random(S) < 0.1] = -1
    held = np.minimum(ld, -(-length // P) + (rng.random(S) < 0.2))
    perm = rng.permutation(n_blocks)
    table, used = np.full((S, ld), -1), 0
    for s in range(S):
        table[s, :held[s]] = perm[used:used + held[s]]
        used += held[s]
    free = np.concatenate([perm[used:], np.full(used, -1)])
    args = (length, n_new, held, table, free, n_blocks - used)
    want = oc.plan(n_blocks, P, ld, T, *args)
    got, err = _plan_gpu(torch, n_blocks, P, T, *args, alias=alias)
    say(f"plan S {S}: rows {want['row_start'][-1]} of {T}, free {args[-1]} -> {want['n_free']}")
    assert not want["err"]
    _same_plan(got, err, want)


@pytest.mark.parametrize("what", ["blocks", "rows", "table", "length", "n_new", "held", "n_free", "double"])
def test_plan_that_does_not_fit_changes_nothing(what):
    torch = torch_or_skip()
    n_blocks, P, S, ld, T = 12, 32, 3, 4, 64
    length, n_new, held = np.array([30, 0, 64]), np.array([10, 3, 1]), np.array([1, 0, 2])
    table = np.full((S, ld), -1)
    table[0, 0], table[2, :2] = 0, [1, 2]
    free, n_free = np.concatenate([np.arange(3, 12), [-1] * 3]), 9
    if what == "blocks":
        n_free = 1
    elif what == "rows":
        n_new[1] = 60
    elif what == "table":
        n_new[2] = 65
    elif what == "length":
        length[0] = 33
    elif what == "n_new":
        n_new[1] = -2
    elif what == "held":
        held[1] = 5
    elif what == "n_free":
        n_free = 13
    else:                           # blocks given back twice
        n_free, n_new = 12, np.array([-1, 3, 1])
    args = (length, n_new, held, table, free, n_free)
    want = oc.plan(n_blocks, P, ld, T, *args)
    assert want["err"]
    got, err = _plan_gpu(torch, n_blocks, P, T, *args)
    _same_plan(got, err, want)


@pytest.mark.parametrize("T", [64, 9000])
def test_plan_reports_block_numbers_out_of_range(T):
    torch = torch_or_skip()
    length, n_new, held = np.array([30, 0, 64]), np.array([10, 3, -1]), np.array([1, 0, 2])
    table = np.full((3, 4), -1)
    table[0, 0], table[2, :2] = 77, [1, 2]                    # the partly filled block of sequence 0 is none
    args = (length, n_new, held, table, np.concatenate([np.arange(3, 12), [-1] * 3]), 9)
    want = oc.plan(12, 32, 4, T, *args)
    got, err = _plan_gpu(torch, 12, 32, T, *args)
    assert want["err"] and (want["slots"][:2] == -1).all() and want["slots"][2] >= 0
    _same_plan(got, err, want)


def test_plan_of_no_sequences():
    torch = torch_or_skip()
    cc = dd.cache_config(4, 32, 1, 64)
    m = dd.CacheMap.empty(0, 5, 2)
    m.row_start.fill_(9)
    free, nf, no, z = dev_i32(torch, [0, 1, 2, 3]), dev_i32(torch, [4]), dev_i32(torch, [0]), dev_i32(torch, [])
    dd.cache_plan(cc, m, z, z, z, free, nf, no)
    assert int(no.item()) == 4 and int(m.row_start.item()) == 0 and (_cpu(m.slots) == -1).all()


# ---------------------------------------------------------------- append

def _tables(rng, lens, news, P, ld, n_blocks, pad=0):
    """Map arrays of sequences with lens cached and news new tokens, blocks in random order."""
    S = len(lens)
    T = int(sum(news)) + pad
    perm = rng.permutation(n_blocks)
    table = np.full((S, ld), -1)
    used, start, seq, pos, slots = 0, [0], np.full(T, -1), np.full(T, -1), np.full(T, -1)
    for s in range(S):
        nb = -(-(lens[s] + news[s]) // P)
        table[s, :nb] = perm[used:used + nb]
        used += nb
        for i in range(news[s]):
            r, p = start[-1] + i, lens[s] + i
            seq[r], pos[r], slots[r] = s, p, table[s, p // P] * P + p % P
        start.append(start[-1] + news[s])
    return dict(table=table, kv=np.array(lens) + np.array(news), start=np.array(start), seq=seq, pos=pos, slots=slots, T=T)


def _map(torch, t):
    S, ld = t["table"].shape
    d = lambda x: dev_i32(torch, x)   # noqa: E731
    return dd.CacheMap(d(t["table"]).reshape(S, ld), d(np.full(S, ld)), d(t["kv"]), d(t["start"]), d(t["seq"]), d(t["pos"]), d(t["slots"]))


def _pow2(torch, rng, shape, lo=-9, hi=3):
    return torch.from_numpy(2.0 ** rng.integers(lo, hi, shape).astype(np.float64)).float().cuda()


APPEND = [  # lens, news, heads, dh, block, padding rows
    ([0], [1], 1, 32, 32, 0), ([0, 31, 32, 33], [1, 1, 1, 1], 2, 64, 32, 3), ([5, 0, 40], [70, 64, 0], 3, 64, 64, 2),
    ([100, 128, 1], [300, 128, 27], 2, 128, 128, 0), ([17, 255, 256], [250, 2, 600], 2, 128, 256, 5),
    ([200], [1000], 2, 32, 256, 1), (list(range(40)), [3] * 40, 12, 64, 64, 0),
    (list(range(300)), [1] * 300, 1, 32, 64, 3), ([31, 0, 63] * 20, [2, 0, 3] * 20, 3, 64, 32, 0),
    ([7] * 299 + [0], [4] * 299 + [70], 1, 64, 32, 0)]


@pytest.mark.parametrize("lens,news,H,dh,P,pad", APPEND)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append_equals_oracle(lens, news, H, dh, P, pad, dtype):
    torch = torch_or_skip()
    rng = np.random.default_rng(sum(lens) + dh + P)
    nb = int(sum(-(-(a + b) // P) for a, b in zip(lens, news))) + 3
    t = _tables(rng, lens, news, P, -(-max(a + b for a, b in zip(lens, news)) // P), nb, pad)
    m, cc = _map(torch, t), dd.cache_config(nb, P, H, dh)
    codes = torch.from_numpy(rng.integers(0, 256, (nb, H, 2 * P * dh)).astype(np.uint8)).cuda()
    scales = _pow2(torch, rng, (nb, H, 2))
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    # sizes that make some scales grow and others stay; a few values that are not finite; rows of zeros
    x = rng.normal(size=(t["T"], 3, H, dh)) * 2.0 ** rng.integers(-6, 8, (t["T"], 1, H, 1))
    x[rng.random(x.shape) < 0.002] = np.inf
    x[rng.random(x.shape) < 0.002] = -np.inf
    x[rng.random(x.shape) < 0.002] = np.nan
    x[::7] = 0.0
    qkv = torch.from_numpy(x).to(tdt).reshape(t["T"], -1).cuda()
    k, v = qkv[:, H * dh:2 * H * dh], qkv[:, 2 * H * dh:]
    f = lambda y: y.double().cpu().numpy().reshape(-1, H, dh)   # noqa: E731
    wc, ws = oc.append(_cpu(codes), _cpu(scales), P, f(k), f(v), t["start"], t["slots"])
    err = dev_i32(torch, [0])
    dd.cache_append(cc, codes, scales, m, k, v, dev_err=err)
    gc, gs = _cpu(codes), _cpu(scales)
    assert int(err.item()) == 0
    assert np.array_equal(gs, ws), "scales"
    a, b = oc.decode(gc), oc.decode(wc)
    bad = ~((a == b) | (np.isnan(a) & np.isnan(b)))
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5])
    dd.cache_append(cc, codes, scales, m, k, v)          # the same again changes nothing
    assert np.array_equal(_cpu(scales), gs)
    c = oc.decode(_cpu(codes))
    assert ((c == a) | (np.isnan(c) & np.isnan(a))).all()


@pytest.mark.parametrize("big", [0.0, 1e-42, 1e-30, 2.0 ** -92, 3.0e38])
def test_append_at_the_ends_of_the_scales(big):
    torch = torch_or_skip()
    rng = np.random.default_rng(5)
    H, dh, P = 1, 64, 32
    t = _tables(rng, [0], [40], P, 2, 4)
    cc, m = dd.cache_config(4, P, H, dh), _map(torch, t)
    codes, scales = dd.cache_tensors(cc)
    k = torch.from_numpy(rng.uniform(-1, 1, (40, H * dh)) * big).float().cuda()
    wc, ws = oc.append(_cpu(codes), _cpu(scales), P, k.double().cpu().numpy().reshape(-1, H, dh),
                       k.double().cpu().numpy().reshape(-1, H, dh), t["start"], t["slots"])
    dd.cache_append(cc, codes, scales, m, k, k)
    assert np.array_equal(_cpu(scales), ws) and np.array_equal(oc.decode(_cpu(codes)), oc.decode(wc))


def test_append_leaves_out_rows_of_no_place():
    torch = torch_or_skip()
    rng = np.random.default_rng(6)
    H, dh, P = 2, 64, 32
    t = _tables(rng, [0, 0], [32, 32], P, 1, 2)
    t["slots"][32:] = 2 * P + np.arange(32)              # a block that the pool does not have
    cc, m = dd.cache_config(2, P, H, dh), _map(torch, t)
    codes, scales = dd.cache_tensors(cc)
    k = torch.randn((64, H * dh), device="cuda")
    err = dev_i32(torch, [0])
    dd.cache_append(cc, codes, scales, m, k, k, dev_err=err)
    b = int(t["table"][0, 0])
    assert int(err.item()) == dd.DD_DEVERR_CACHE
    assert int(codes[1 - b].count_nonzero()) == 0 and int(codes[b].count_nonzero()) > 0


# ---------------------------------------------------------------- attention

def _attention_case(torch, rng, lens, news, hq, hkv, dh, P, dtype, pad, spare=2, wide=0):
    """A pool whose unused places hold NaN codes and random bytes, and rows q in columns of wider rows."""
    nb = int(sum(-(-(a + b) // P) for a, b in zip(lens, news))) + spare
    t = _tables(rng, lens, news, P, max(1, -(-max(a + b for a, b in zip(lens, news)) // P)), nb, pad)
    codes = rng.integers(0, 256, (nb, hkv, 2 * P * dh)).astype(np.uint8)
    scales = 2.0 ** rng.integers(-9, -6, (nb, hkv, 2)).astype(np.float64)
    vi = oc.v_index(P, dh)
    for s in range(len(lens)):
        L = t["kv"][s]
        for j in range(-(-L // P)):
            b, n = t["table"][s, j], min(P, L - j * P)
            fill = lambda: oc.encode(np.clip(rng.normal(size=(hkv, n, dh)) * 100, -448, 448))   # noqa: E731
            codes[b][:, np.arange(P * dh).reshape(P, dh)[:n]] = fill()
            codes[b][:, P * dh + vi[:n]] = fill()
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = torch.from_numpy(rng.normal(size=(t["T"], hq * dh + wide)) * 2).to(tdt).cuda()
    return t, codes, scales, q


def _attend(torch, t, codes, scales, q, hq, hkv, dh, P, pattern, out=None, err=None, max_new=None, max_kv=None):
    cc = dd.cache_config(codes.shape[0], P, hkv, dh)
    news = np.diff(t["start"])
    max_new, max_kv = max_new or max(1, int(news.max())), max_kv or max(1, int(t["kv"].max()))
    S, T = len(news), t["T"]
    n = dd.cache_attention_workspace_bytes(cc, S, T, hq, max_new, max_kv)
    ws = torch.full((max(n, 256),), 255, dtype=torch.uint8, device="cuda")      # NaN wherever nothing is written
    out = torch.full((T, hq * dh), -7.0, dtype=q.dtype, device="cuda") if out is None else out
    c, s = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).float().cuda()
    dd.cache_attention(cc, c, s, _map(torch, t), q, out, hq, max_new, max_kv, ws, pattern=pattern, dev_err=err)
    return out, n


def _check(torch, t, codes, scales, q, out, hq, hkv, dh, P, pattern, rows=None):
    """Rows against the oracle.  Roundings counted: products of dh terms in fp32 put the scores off by at most
    (dh + 8) 2^-24 scale sum |q||k|, twice that relative in p; p itself 2^-8 (bf16) or the pieces' 2^-22 with
    exp2's and the sums' (L + 16) 2^-23; the result half a step."""
    bf = q.dtype == torch.bfloat16
    scale = dh ** -0.5
    q64 = q.double().cpu().numpy()[:, :hq * dh].reshape(-1, hq, dh)
    got = out.double().cpu().numpy()[:, :hq * dh].reshape(-1, hq, dh)
    worst = 0.0
    for s in range(len(t["kv"])):
        r0, r1, L = t["start"][s], t["start"][s + 1], int(t["kv"][s])
        if r0 == r1:
            continue
        k, v = oc.gather(codes, scales, P, dh, t["table"][s, :-(-L // P)], L) if L else (np.zeros((0, hkv, dh)),) * 2
        want = oc.attention(q64[r0:r1], k, v, L - (r1 - r0), pattern == "causal", scale)
        mass = oc.attention(q64[r0:r1], k, np.abs(v), L - (r1 - r0), pattern == "causal", scale)
        g = hq // hkv
        A = max([float((np.abs(q64[r0:r1, h]) @ np.abs(k[:, h // g]).T).max()) for h in range(hq)], default=0.0) * scale if L else 0.0
        rel = 2 * (dh + 8) * 2.0 ** -24 * A + (L + 16) * 2.0 ** -23 + (2.0 ** -8 if bf else 2.0 ** -22)
        tol = np.abs(want) * (2.0 ** -8 if bf else 2.0 ** -24) + mass * rel
        x = got[r0:r1]
        assert np.array_equal(np.isnan(x), np.isnan(want)), (s, np.argwhere(np.isnan(x) != np.isnan(want))[:5])
        ok = ~np.isnan(want)
        d = np.abs(x - want)[ok]
        worst = max(worst, float((d / np.maximum(tol[ok], 1e-30)).max(initial=0.0)))
        assert (d <= tol[ok]).all(), (s, float(d.max()), worst)
    assert (got[t["start"][-1]:] == -7).all()            # padding rows stay as they were
    return worst


ATTEND = [  # lens, news, query heads, key heads, dh, block, padding rows
    ([0], [1], 1, 1, 64, 32, 0), ([0, 31, 32, 33, 63, 64], [1] * 6, 2, 2, 64, 32, 1),
    ([1000], [1], 12, 12, 64, 64, 0), ([2000, 3, 700], [16, 16, 16], 4, 4, 64, 64, 0),
    ([5, 90, 300, 0], [7, 0, 1, 40], 8, 2, 128, 128, 3), ([70, 200], [33, 5], 6, 2, 32, 32, 2),
    ([100, 17], [130, 64], 3, 3, 64, 256, 0), ([300], [257], 16, 2, 128, 64, 0), ([4100], [3], 15, 5, 64, 32, 0),
    ([0, 0], [40, 70], 2, 1, 32, 64, 0),
    # enough heads for one, two and four wavefronts per column tile, and for whole sequences of more than 64 blocks
    ([40], [70], 2100, 2100, 32, 32, 0), ([40], [70], 600, 600, 64, 32, 0), ([40], [70], 600, 600, 128, 32, 0),
    ([400], [33], 150, 150, 32, 32, 0), ([900], [33], 150, 150, 64, 32, 2), ([2500], [1], 130, 130, 32, 32, 1)]


@pytest.mark.parametrize("lens,news,hq,hkv,dh,P,pad", ATTEND)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("pattern", ["causal", "bidirectional"])
def test_attention_against_oracle(lens, news, hq, hkv, dh, P, pad, dtype, pattern):
    torch = torch_or_skip()
    rng = np.random.default_rng(sum(lens) + sum(news) + dh)
    t, codes, scales, q = _attention_case(torch, rng, lens, news, hq, hkv, dh, P, dtype, pad)
    err = dev_i32(torch, [0])
    out, n = _attend(torch, t, codes, scales, q, hq, hkv, dh, P, pattern, err=err)
    worst = _check(torch, t, codes, scales, q, out, hq, hkv, dh, P, pattern)
    say(f"attention {lens} + {news} {hq}/{hkv} x {dh} {dtype} {pattern}: ws {n}, worst {worst:.3f} of the bound")
    assert int(err.item()) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_of_strided_rows(dtype):
    """q as columns of packed rows and out with wider rows: what stands beside the columns stays."""
    torch = torch_or_skip()
    rng = np.random.default_rng(8)
    hq, hkv, dh, P = 4, 2, 64, 64
    t, codes, scales, q = _attention_case(torch, rng, [200, 31], [5, 9], hq, hkv, dh, P, dtype, 2, wide=64)
    big = torch.full((t["T"], hq * dh + 32), -7.0, dtype=q.dtype, device="cuda")
    out, _ = _attend(torch, t, codes, scales, q[:, :hq * dh], hq, hkv, dh, P, "causal", out=big[:, :hq * dh])
    _check(torch, t, codes, scales, q, out, hq, hkv, dh, P, "causal")
    assert (big[:, hq * dh:] == -7).all()


@pytest.mark.parametrize("new,hkv,ctx", [(3, 2, 45), (40, 2, 45), (100, 2, 45), (35, 150, 900), (35, 150, 400), (35, 150, 45)])
@pytest.mark.parametrize("where", ["key", "value"])
def test_attention_nan_reaches_the_rows_that_see_it(where, new, hkv, ctx):
    """A NaN key (value) of a new token: rows before it are untouched, it and later rows are NaN (in that feature)."""
    torch = torch_or_skip()
    rng = np.random.default_rng(9)
    hq, dh, P = hkv, 64, 32
    t, codes, scales, q = _attention_case(torch, rng, [ctx], [new], hq, hkv, dh, P, "bf16", 0)
    at = ctx + new // 2
    b, o = t["table"][0, at // P], at % P
    if where == "key":
        codes[b][1, o * dh + 9] = 0x7F
    else:
        codes[b][1, P * dh + oc.v_index(P, dh)[o, 9]] = 0xFF
    out, _ = _attend(torch, t, codes, scales, q, hq, hkv, dh, P, "causal")
    _check(torch, t, codes, scales, q, out, hq, hkv, dh, P, "causal")
    n = torch.isnan(out).reshape(-1, hq, dh)
    assert not n[:new // 2].any() and not n[:, 0].any()
    assert n[new // 2:, 1].all() if where == "key" else n[new // 2:, 1, 9].all() and int(n.sum()) == new - new // 2


def test_attention_rows_that_see_nothing_are_zero():
    torch = torch_or_skip()
    rng = np.random.default_rng(10)
    hq, hkv, dh, P = 2, 1, 64, 32
    t, codes, scales, q = _attention_case(torch, rng, [0, 0], [6, 5], hq, hkv, dh, P, "bf16", 0)
    t["kv"] = np.array([4, 0])                # two of the first sequence's six rows stand before its first token
    for pattern in ("causal", "bidirectional"):
        out, _ = _attend(torch, t, codes, scales, q, hq, hkv, dh, P, pattern)
        _check(torch, t, codes, scales, q, out, hq, hkv, dh, P, pattern)
        assert (out[6:] == 0).all() and (pattern != "causal" or (out[:2] == 0).all())


def test_attention_blocks_out_of_range_are_not_seen():
    torch = torch_or_skip()
    rng = np.random.default_rng(11)
    hq, hkv, dh, P = 2, 2, 64, 32
    t, codes, scales, q = _attention_case(torch, rng, [100], [4], hq, hkv, dh, P, "fp32", 0)
    whole = t["table"].copy()
    keep = np.concatenate([np.arange(32), np.arange(64, 104)])
    for bad in (-1, codes.shape[0], 2 ** 31 - 1):
        t["table"] = whole.copy()
        t["table"][0, 1] = bad
        err = dev_i32(torch, [0])
        out, _ = _attend(torch, t, codes, scales, q, hq, hkv, dh, P, "bidirectional", err=err)
        k, v = oc.gather(codes, scales, P, dh, whole[0], 104)
        want = oc.attention(q.double().cpu().numpy().reshape(4, hq, dh), k[keep], v[keep], 0, False, dh ** -0.5)
        assert int(err.item()) == dd.DD_DEVERR_CACHE
        # fp32: the bound of _check with |s| below 40 and |v| below 4
        assert np.abs(out.double().cpu().numpy().reshape(4, hq, dh) - want).max() < 4 * (2 * 72 * 2.0 ** -24 * 40 + 2.0 ** -16)


def test_attention_bounds_that_do_not_hold_are_reported():
    torch = torch_or_skip()
    rng = np.random.default_rng(12)
    hq, hkv, dh, P = 2, 2, 64, 32
    t, codes, scales, q = _attention_case(torch, rng, [100, 10], [4, 2], hq, hkv, dh, P, "bf16", 0)
    err = dev_i32(torch, [0])
    out, _ = _attend(torch, t, codes, scales, q, hq, hkv, dh, P, "causal", err=err, max_new=3)
    assert int(err.item()) == dd.DD_DEVERR_CACHE and (out[3] == -7).all() and (out[:3] != -7).any() and (out[4:] != -7).any()
    err.zero_()
    cut = dict(t, kv=np.array([64, 12]), table=t["table"])
    out, _ = _attend(torch, t, codes, scales, q, hq, hkv, dh, P, "bidirectional", err=err, max_kv=64)
    _check(torch, cut, codes, scales, q, out, hq, hkv, dh, P, "bidirectional")
    assert int(err.item()) == dd.DD_DEVERR_CACHE


def test_pool_beyond_32_bit_offsets():
    """Blocks whose codes lie more than 2^32 bytes into the pool: append, then attend."""
    torch = torch_or_skip()
    rng = np.random.default_rng(13)
    H, dh, P = 2, 64, 64
    nb = (1 << 32) // (H * 2 * P * dh) + 40
    t = _tables(rng, [0], [150], P, 3, 3)
    t["table"] += nb - 3
    t["slots"] += (nb - 3) * P
    cc, m = dd.cache_config(nb, P, H, dh), _map(torch, t)
    codes = torch.empty((nb, H, 2 * P * dh), dtype=torch.uint8, device="cuda")
    codes[-3:] = 0
    codes[:40] = 0
    scales = torch.zeros((nb, H, 2), device="cuda")
    qkv = torch.from_numpy(rng.normal(size=(150, 3 * H * dh))).bfloat16().cuda()
    q, k, v = qkv[:, :H * dh], qkv[:, H * dh:2 * H * dh], qkv[:, 2 * H * dh:]
    dd.cache_append(cc, codes, scales, m, k, v)
    assert int(codes[:40].count_nonzero()) == 0
    out = torch.full((150, H * dh), -7.0, dtype=torch.bfloat16, device="cuda")
    n = dd.cache_attention_workspace_bytes(cc, 1, 150, H, 150, 150)
    ws = torch.empty(max(256, n), dtype=torch.uint8, device="cuda")
    dd.cache_attention(cc, codes, scales, m, q, out, H, 150, 150, ws)
    small = dict(t, table=t["table"] - (nb - 3))
    _check(torch, small, _cpu(codes[-3:]), _cpu(scales[-3:]).astype(np.float64), q, out, H, H, dh, P, "causal")


def test_attention_is_the_same_from_call_to_call_and_in_a_graph():
    """Bit-equal outputs on another stream and from a captured graph that is replayed with other contents."""
    torch = torch_or_skip()
    rng = np.random.default_rng(14)
    hq, hkv, dh, P = 12, 12, 64, 64
    t, codes, scales, q = _attention_case(torch, rng, [900, 40, 1500], [16, 16, 16], hq, hkv, dh, P, "bf16", 0)
    cc, m = dd.cache_config(codes.shape[0], P, hkv, dh), _map(torch, t)
    c, s = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).float().cuda()
    n = dd.cache_attention_workspace_bytes(cc, 3, 48, hq, 16, 1516)
    assert n > 0
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    k = torch.randn((48, hq * dh), device="cuda").bfloat16()

    def step(qq, out, w):
        dd.cache_append(cc, c, s, m, k, k)
        dd.cache_attention(cc, c, s, m, qq, out, hq, 16, 1516, w)
    a, b = torch.zeros_like(q), torch.zeros_like(q)
    step(q, a, ws[0])
    step(q, b, ws[0])
    assert torch.equal(a, b)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        step(q, b.zero_(), ws[1])
    torch.cuda.synchronize()
    assert torch.equal(a, b)
    qs, os_ = q.clone(), torch.zeros_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(qs, os_, ws[1])
    for i in range(3):
        x = torch.from_numpy(rng.normal(size=tuple(q.shape))).bfloat16().cuda()
        qs.copy_(x)
        os_.zero_()
        g.replay()
        step(x, a, ws[0])
        torch.cuda.synchronize()
        assert torch.equal(a, os_), i


def test_binding_refuses_tensors_that_do_not_fit():
    torch = torch_or_skip()
    cc, m = dd.cache_config(4, 32, 2, 64), dd.CacheMap.empty(2, 8, 2)
    codes, scales = dd.cache_tensors(cc)
    x = torch.zeros((8, 128), device="cuda")
    z = dev_i32(torch, [0, 0])
    bad = [(TypeError, lambda: dd.cache_append(cc, codes, scales, m, x, x.bfloat16())),
           (TypeError, lambda: dd.cache_append(cc, codes, scales, m, x.half(), x.half())),
           (ValueError, lambda: dd.cache_append(cc, codes, scales, m, x[:7], x)),
           (ValueError, lambda: dd.cache_append(cc, codes, scales, m, x[:, :120], x[:, :120])),
           (ValueError, lambda: dd.cache_append(cc, codes, scales, m, x, torch.zeros((8, 256), device="cuda"))),
           (ValueError, lambda: dd.cache_append(cc, codes, scales, m, x[:1].expand(8, 128), x[:1].expand(8, 128))),
           (ValueError, lambda: dd.cache_append(cc, codes, scales, m, x.t(), x.t())),
           (ValueError, lambda: dd.cache_append(cc, codes, scales, m, x.cpu(), x.cpu())),
           (ValueError, lambda: dd.cache_append(cc, codes[:3], scales, m, x, x)),
           (TypeError, lambda: dd.cache_append(cc, codes, scales.double(), m, x, x)),
           (ValueError, lambda: dd.cache_attention(cc, codes, scales, m, x, x[:, :64].contiguous(), 2, 4, 64)),
           (dd.DDError, lambda: dd.cache_attention(cc, codes, scales, m, x, x.clone(), 2, 4, 65)),
           (KeyError, lambda: dd.cache_attention(cc, codes, scales, m, x, x.clone(), 2, 4, 64, pattern="none")),
           (ValueError, lambda: dd.cache_plan(cc, m, z[:1], z, z, dev_i32(torch, [0] * 4), z, z)),
           (TypeError, lambda: dd.cache_plan(cc, m, z.long(), z, z, dev_i32(torch, [0] * 4), z, z)),
           (ValueError, lambda: dd.logits_edit(x, "fp32", 128, 8, 100, x, history=z)),
           (ValueError, lambda: dd.logits_edit(x, "fp32", 128, 8, 100, x, bias_ids=z[None])),
           (ValueError, lambda: dd.logits_edit(x, "fp32", 128, 9, 100, x)),
           (ValueError, lambda: dd.logits_edit(x, "fp32", 128, 8, 100, x, hist_len=z)),
           (TypeError, lambda: dd.logits_edit(x, "bf16", 128, 8, 100, x))]
    for i, (what, call) in enumerate(bad):
        with pytest.raises(what):
            call()
            pytest.fail(f"call {i} was not refused")
