"""dd_token_sample and dd_logits_truncate against the float64 oracle."""
import numpy as np
import pytest

from oracle import philox, serving as so
from paper_2609_04010_amd import _lib as dd
from tests.gpu_util import dev_i32, dev_words, logits_dev, round_to_dtype, say, torch_or_skip

pytestmark = pytest.mark.gpu

OFF = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
NAMES = tuple(OFF)


def margin_ok(margin, V):
    """Weights are multiples of 2^-f, f = min(46, 62 - ceil(log2 V)): each of V is at most half a step off, a running sum by V of
    those, and the bound that it is compared with as much again; exponentials and products in float64 add V 2^-52 on each side."""
    f = min(46, 62 - int(np.ceil(np.log2(max(V, 2)))))
    return margin > 2 * V * 2.0 ** -(f + 1) + 2 * V * 2.0 ** -52


def settings(torch, rows, keep):
    """Device arrays of a list of settings, those named in `keep` alone (the others have to be off)."""
    out = {}
    for k in keep:
        v = [r[k] for r in rows]
        out[k] = dev_i32(torch, v) if k == "top_k" else torch.tensor(v, dtype=torch.float32, device="cuda")
    return out


def f32(x):
    return float(np.float32(x))


def check(torch, l, dtype, per_row, words, keep=NAMES, ld=None, sure=0.98):
    """Draws and truncated rows of every row of l (already rounded to dtype) against the oracle."""
    R, V = l.shape
    ld = ld or int(dd.logits_ld(V))
    per_row = [{k: (int(v) if k == "top_k" else f32(v)) for k, v in s.items()} for s in per_row]
    x = logits_dev(torch, l, dtype, ld)
    if ld > V:
        x[:, V:] = 50.0                              # (nothing reads what stands behind a row)
    a = settings(torch, per_row, keep)
    z, kept, kept2, err = dev_i32(torch, [-9] * R), dev_i32(torch, [-9] * R), dev_i32(torch, [-9] * R), dev_i32(torch, [0])
    logp = torch.full((R,), 7.0, device="cuda")
    out = torch.full_like(x, -7.0)
    dd.token_sample(x, dtype, ld, R, V, z, R, noise_words=dev_words(torch, words), logp=logp, n_kept=kept, dev_err=err, **a)
    dd.logits_truncate(x, dtype, ld, R, V, out, n_kept=kept2, dev_err=err, **a)
    assert int(err.item()) == 0
    o = out.double().cpu().numpy()
    assert (o[:, V:] == -7).all()
    z, kept, logp, same = z.tolist(), kept.tolist(), logp.double().tolist(), torch.equal(kept, kept2)
    assert same
    clear, largest = 0, float(torch.finfo(x.dtype).max)
    for r in range(R):
        wz, wl, wn, margin = so.token(l[r], words[r], **per_row[r])
        wo, _, m2 = so.truncate(l[r], largest, **per_row[r])
        if margin_ok(m2, V):
            assert kept[r] == wn, (r, kept[r], wn, per_row[r])
            fin = np.isfinite(wo)
            assert np.array_equal(fin, np.isfinite(o[r, :V])), r
            # one division in fp32, one rounding to the type
            tol = np.abs(wo[fin]) * (2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0)) + 1e-38
            assert (np.abs(o[r, :V][fin] - wo[fin]) <= tol).all(), r
        if margin_ok(margin, V):
            clear += 1
            assert z[r] == wz, (r, z[r], wz, per_row[r])
            # (l - max) / temperature exact to 2^-52, the sum to V 2^-47 of at least 1, one rounding to fp32
            assert abs(logp[r] - wl) <= abs(wl) * 2.0 ** -23 + V * 2.0 ** -45 + 1e-14, (r, logp[r], wl)
    say("rows", R, "V", V, dtype, "clear", clear)
    # (words 0 and 2^32 - 1 are 2^-33 of the sum away from its ends, which for sums near 1 is less than the bound for V > 8192)
    assert clear >= sure * (R - 2)
    dd.logits_truncate(x, dtype, ld, R, V, x, **a)   # in place
    assert torch.equal(x[:, :V], out[:, :V]) and (ld == V or (x[:, V:] == 50).all())


def draw_settings(rng, R, V):
    pick = lambda off, f: off if rng.random() < 0.3 else f()   # noqa: E731
    return [dict(temperature=pick(1.0, lambda: rng.choice([0.0, 0.3, 0.7, 1.3, 3.0])), top_k=pick(0, lambda: int(rng.integers(-1, V + 3))),
                 top_p=pick(1.0, lambda: rng.choice([0.0, 0.1, 0.5, 0.9, 0.99, 1.5])), min_p=pick(0.0, lambda: rng.choice([1e-6, 0.01, 0.3, 1.0])))
            for _ in range(R)]


def words_of(rng, R):
    w = rng.integers(0, 2 ** 32, R, dtype=np.uint64)
    w[:2] = [0, 2 ** 32 - 1][:R]
    return w


SIZES = [(1, 3), (2, 5), (31, 40), (64, 40), (65, 40), (300, 60), (2047, 40), (4096, 30), (8193, 30), (20000, 16), (50257, 24),
         (65537, 6), (140001, 4)]


@pytest.mark.parametrize("V,R", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_draws_and_rows_against_oracle(V, R, dtype):
    torch = torch_or_skip()
    rng = np.random.default_rng(V)
    l = round_to_dtype(rng.normal(size=(R, V)) * rng.choice([0.2, 2.5, 8.0], (R, 1)), dtype)
    l[rng.random(l.shape) < 0.1] = -np.inf
    l[:, rng.integers(0, V)] = 1.0
    check(torch, l, dtype, draw_settings(rng, R, V), words_of(rng, R))


@pytest.mark.parametrize("keep", [(), ("temperature",), ("top_k",), ("top_p",), ("min_p",), ("temperature", "top_p"), ("top_k", "top_p"),
                                  ("temperature", "top_k", "min_p")])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_some_settings_alone(keep, dtype):
    torch = torch_or_skip()
    rng = np.random.default_rng(len(keep))
    R, V = 12, 5003
    s = [{k: (v if k in keep else OFF[k]) for k, v in x.items()} for x in draw_settings(rng, R, V)]
    check(torch, round_to_dtype(rng.normal(size=(R, V)) * 3, dtype), dtype, s, words_of(rng, R), keep)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [7, 200, 5000, 50257])
def test_ties_and_extremes(V, dtype):
    """Rows of one value, of two, of the type's ends, of values next to each other, of both zeros, of one finite class."""
    torch = torch_or_skip()
    rng = np.random.default_rng(V)
    big = float(torch.finfo(torch.bfloat16 if dtype == "bf16" else torch.float32).max)
    step = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -23
    rows = [np.zeros(V), np.full(V, -3.0), rng.choice([1.0, 2.0], V), rng.choice([big, -big], V), rng.choice([0.0, -big], V),
            1.0 + step * rng.integers(0, 9, V), rng.choice([0.0, -0.0], V), np.where(np.arange(V) == V // 2, 5.0, -np.inf),
            rng.choice([1e-38, -1e-38, 0.0], V), rng.choice([-big, -np.inf, big / 2], V), -np.arange(V) * 1.0, rng.normal(size=V) * 1e-6,
            np.where(rng.random(V) < 0.5, -1e9, rng.normal(size=V)), rng.normal(size=V) * 1e4]
    rows[4][V // 3] = 0.0
    rows[9][-1] = -big
    l = round_to_dtype(np.stack(rows), dtype)
    R = len(rows)
    some = [dict(OFF), dict(OFF, top_k=V // 2), dict(OFF, top_p=0.63), dict(OFF, temperature=1e-30), dict(OFF, temperature=1e30, top_p=0.4),
            dict(OFF, min_p=1.0), dict(OFF, temperature=0.0), dict(temperature=0.7, top_k=max(1, V // 3), top_p=0.7, min_p=0.01)]
    for s in some:
        say("settings", s)
        check(torch, l, dtype, [s] * R, words_of(rng, R), sure=0.5)


def test_rows_and_settings_that_allow_nothing():
    torch = torch_or_skip()
    V, ld, R = 500, 512, 12
    rng = np.random.default_rng(0)
    l = rng.normal(size=(R, V)).astype(np.float32)
    l[1, 7], l[2, 499], l[3] = np.nan, np.inf, -np.inf
    x = logits_dev(torch, l, "fp32", ld)
    s = [dict(OFF) for _ in range(R)]
    for r, kv in ((5, dict(temperature=-1.0)), (6, dict(temperature=np.nan)), (7, dict(temperature=np.inf)), (8, dict(top_p=-0.1)),
                  (9, dict(top_p=np.nan)), (10, dict(min_p=1.5)), (11, dict(min_p=np.nan))):
        s[r].update(kv)
    words = words_of(rng, R)
    for bad, bit in (((1, 2, 3), dd.DD_DEVERR_LOGITS), ((5, 6, 7, 8, 9, 10, 11), dd.DD_DEVERR_SAMPLING)):
        at = [0, *bad, 4]
        a = settings(torch, [s[r] for r in at], NAMES)
        y = x[at].contiguous()
        z, n, err = dev_i32(torch, [-9] * len(at)), dev_i32(torch, [-9] * len(at)), dev_i32(torch, [0])
        logp, out = torch.zeros(len(at), device="cuda"), torch.full_like(y, 3.0)
        dd.token_sample(y, "fp32", ld, len(at), V, z, len(at), noise_words=dev_words(torch, words[at]), logp=logp, n_kept=n, dev_err=err, **a)
        assert int(err.item()) == bit
        err.zero_()
        dd.logits_truncate(y, "fp32", ld, len(at), V, out, n_kept=n, dev_err=err, **a)
        assert int(err.item()) == bit
        assert z.tolist()[1:-1] == [0] * len(bad) and n.tolist()[1:-1] == [0] * len(bad) and logp[1:-1].isnan().all()
        assert torch.equal(torch.nan_to_num(out[1:-1, :V]), torch.nan_to_num(y[1:-1, :V])) and (out[:, V:] == 3).all()
        for i in (0, len(at) - 1):
            assert z[i].item() == so.token(l[at[i]].astype(np.float64), words[at[i]])[0] and n[i].item() == V and logp[i].isfinite()


def test_rows_by_number():
    """One row for several draws, rows left out, numbers out of range, settings shared by draws, Philox noise."""
    torch = torch_or_skip()
    V, ld, R, n, per = 700, 704, 9, 20, 3
    rng = np.random.default_rng(4)
    l = round_to_dtype(rng.normal(size=(R, V)) * 2, "bf16")
    x = logits_dev(torch, l, "bf16", ld)
    ids = rng.integers(0, R, n)
    ids[[3, 11]] = -1
    s = [dict(temperature=f32(rng.uniform(0.5, 2)), top_k=int(rng.integers(0, 50)), top_p=f32(rng.uniform(0.5, 1)), min_p=0.0) for _ in range(7)]
    z, kept, err = dev_i32(torch, [-9] * n), dev_i32(torch, [-9] * n), dev_i32(torch, [0])
    logp = torch.full((n,), 7.0, device="cuda")
    a = settings(torch, s, NAMES)
    dd.token_sample(x, "bf16", ld, R, V, z, n, row_ids=dev_i32(torch, ids), draws_per_seq=per, seed=77, step=5, row0=1000, logp=logp, n_kept=kept,
                    dev_err=err, **a)
    assert int(err.item()) == 0
    for i in range(n):
        if ids[i] < 0:
            assert z[i].item() == -9 and kept[i].item() == -9 and logp[i].item() == 7
            continue
        word = int(philox.philox_scalar((0, 1000 + i, 5, 6), (77, 0))[0])
        wz, _, wn, margin = so.token(l[ids[i]], word, **s[i // per])
        assert not margin_ok(margin, V) or (z[i].item(), kept[i].item()) == (wz, wn)
    ids[[5, 6]] = [R, -2]
    z2 = torch.full_like(z, -9)
    dd.token_sample(x, "bf16", ld, R, V, z2, n, row_ids=dev_i32(torch, ids), draws_per_seq=per, seed=77, step=5, row0=1000, dev_err=err, **a)
    assert int(err.item()) == dd.DD_DEVERR_SAMPLING
    z[5] = z[6] = -9
    assert torch.equal(z, z2)


def test_more_draws_than_workgroups():
    """Rows of few classes, many more than the grid is wide, equal the same rows one call each."""
    torch = torch_or_skip()
    V, ld, R = 33, 40, 5000
    rng = np.random.default_rng(8)
    l = round_to_dtype(rng.normal(size=(R, V)), "fp32")
    check(torch, l, "fp32", draw_settings(rng, R, V), words_of(rng, R), ld=ld)


def test_more_draws_than_a_grid_holds():
    """4.2 million rows of 5 classes equal their halves."""
    torch = torch_or_skip()
    V, ld, R = 5, 8, 2 ** 22 + 5
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((R, ld), generator=g, device="cuda").bfloat16()
    a, h = dict(seed=4), R // 2
    z, z2, n, n2 = (torch.zeros(R, dtype=torch.int32, device="cuda") for _ in range(4))
    p, out, out2 = torch.full((R,), 0.8, device="cuda"), torch.full_like(x, 3.0), torch.full_like(x, 3.0)
    dd.token_sample(x, "bf16", ld, R, V, z, R, top_p=p, n_kept=n, **a)
    dd.logits_truncate(x, "bf16", ld, R, V, out, top_p=p)
    for i, k in ((0, h), (h, R - h)):
        dd.token_sample(x[i:], "bf16", ld, k, V, z2[i:], k, top_p=p[i:], n_kept=n2[i:], row0=i, **a)
        dd.logits_truncate(x[i:], "bf16", ld, k, V, out2[i:], top_p=p[i:])
    assert torch.equal(z, z2) and torch.equal(n, n2) and torch.equal(out, out2)


def test_rows_past_32_bits():
    """Row offsets beyond 2^31 numbers."""
    torch = torch_or_skip()
    V, ld, R = 50257, 50304, 43000
    x = torch.zeros((R, ld), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    at = torch.randint(0, V, (R,), generator=g, device="cuda")
    x.scatter_(1, at[:, None], 30.0)
    z, n = dev_i32(torch, np.zeros(R)), dev_i32(torch, np.zeros(R))
    p = torch.full((R,), 0.9, device="cuda")
    dd.token_sample(x, "bf16", ld, R, V, z, R, top_p=p, n_kept=n, seed=3)
    assert torch.equal(z, at.int()) and (n == 1).all()
    dd.logits_truncate(x, "bf16", ld, R, V, x, top_p=p)
    assert ((x[:, :V] == 30).sum(1) == 1).all() and int(x[:, :V].isinf().sum()) == R * (V - 1)


def test_on_another_stream_and_captured():
    """Replays of a captured call equal the eager one, with new logits and words in place."""
    torch = torch_or_skip()
    V, ld, R = 5000, 5056, 70
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.empty((R, ld), device="cuda")
    words = torch.empty(R, dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(1)
    a = settings(torch, draw_settings(rng, R, V), NAMES)
    z, z2, out, out2 = dev_i32(torch, np.zeros(R)), dev_i32(torch, np.zeros(R)), torch.zeros_like(x), torch.zeros_like(x)

    def fill():
        x.copy_(torch.randn((R, ld), generator=g, device="cuda") * 3)
        words.copy_(torch.randint(-2**31, 2**31, (R,), generator=g, device="cuda", dtype=torch.int64).int())

    def call(z, out):
        dd.token_sample(x, "fp32", ld, R, V, z, R, noise_words=words, **a)
        dd.logits_truncate(x, "fp32", ld, R, V, out, **a)

    fill()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call(z2, out2)
    torch.cuda.current_stream().wait_stream(s)
    call(z, out)
    assert torch.equal(z, z2) and torch.equal(out, out2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(z, out)
    for _ in range(4):
        fill()
        graph.replay()
        call(z2, out2)
        torch.cuda.synchronize()
        assert torch.equal(z, z2) and torch.equal(out, out2)


def test_truncated_rows_in_the_draws_that_follow():
    """Rows truncated, then the posterior's draw and a verification: tokens that stay alone, and a draft from the truncated draft
    row is accepted where target and draft are the same."""
    torch = torch_or_skip()
    V, ld, S, B = 1000, 1024, 40, 4
    g = torch.Generator(device="cuda").manual_seed(5)
    p = (torch.randn((S * B, ld), generator=g, device="cuda") * 2).bfloat16()
    k = torch.full((S,), 13, dtype=torch.int32, device="cuda")
    t = torch.full((S,), 0.7, device="cuda")
    q = torch.empty_like(p)
    n, err = dev_i32(torch, np.zeros(S * B)), dev_i32(torch, [0])
    dd.logits_truncate(p, "bf16", ld, S * B, V, q, B, temperature=t, top_k=k, n_kept=n, dev_err=err)
    assert (n == 13).all()
    zt, zs = torch.full((S * B,), V, dtype=torch.int32, device="cuda"), dev_i32(torch, np.zeros(S * B))
    dd.posterior_sample("mask", q, "bf16", ld, S * B, V, zt, 0.0, 1.0, zs, seed=3, dev_err=err)
    assert q.gather(1, zs.long()[:, None]).isfinite().all()
    draft = dev_i32(torch, np.zeros(S * (B - 1))).view(S, B - 1)
    draft.copy_(zs.view(S, B)[:, :B - 1])
    qd = q.view(S, B, ld)[:, :B - 1].contiguous()
    n_out, z_out = dev_i32(torch, np.zeros(S)), dev_i32(torch, np.zeros(S))
    ws = torch.empty(dd.spec_verify_workspace_bytes(S, B), dtype=torch.uint8, device="cuda")
    dd.spec_verify(q, qd, "bf16", ld, S, B, V, draft, n_out, z_out, ws, seed=9, dev_err=err)
    last = q.view(S, B, ld)[:, B - 1]
    assert int(err.item()) == 0 and (n_out == B).all() and last.gather(1, z_out.long()[:, None]).isfinite().all()


@pytest.mark.parametrize("V,dtype", [(v, "bf16") for v in (2048, 2049, 8192, 16384, 16385, 32768, 32769, 53248, 53249, 57344, 57345, 65536, 131072, 131073)] +
                         [(4096, "fp32"), (4097, "fp32")])
def test_sizes_at_which_another_kernel_begins(V, dtype):
    torch = torch_or_skip()
    rng = np.random.default_rng(V)
    R = 5
    l = round_to_dtype(rng.normal(size=(R, V)) * np.array([0.2, 1.0, 3.0, 8.0, 3.0])[:, None], dtype)
    l[4, rng.random(V) < 0.5] = -np.inf
    l[:, 0], l[:, V - 1] = 3.0, 3.5
    check(torch, l, dtype, [dict(OFF, top_p=0.8), dict(OFF, top_k=V // 3, temperature=1.5), dict(OFF, top_k=40, top_p=0.9),
                            dict(OFF, min_p=0.001), dict(OFF)], words_of(rng, R), sure=0.6)


@pytest.mark.parametrize("V,dtype", [(1500, "bf16"), (5000, "bf16"), (12000, "bf16"), (30000, "bf16"), (50257, "bf16"), (55000, "bf16"), (140000, "bf16"),
                                     (3000, "fp32"), (9000, "fp32"), (20000, "fp32")])
def test_many_rows_equal_few(V, dtype):
    """A call of more rows than CUs equals calls of some of them, bit for bit: sums do not depend on the kernel."""
    torch = torch_or_skip()
    rng = np.random.default_rng(V)
    R, part, ld = 2 * torch.cuda.get_device_properties(0).multi_processor_count + 77, 97, int(dd.logits_ld(V))
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn((R, ld), generator=g, device="cuda") * torch.rand((R, 1), generator=g, device="cuda") * 6
    x[torch.rand((R, ld), generator=g, device="cuda") < 0.05] = -np.inf
    x[:, V // 2] = 1.0
    x = x.bfloat16() if dtype == "bf16" else x
    s, words = draw_settings(rng, R, V), words_of(rng, R)
    got = []
    for step in (R, part):
        z, n, n2, err = (dev_i32(torch, np.full(k, -9)) for k in (R, R, R, 1))
        err.zero_()
        logp, out = torch.zeros(R, device="cuda"), torch.full_like(x, 3.0)
        for i in range(0, R, step):
            j = min(R, i + step)
            a = settings(torch, s[i:j], NAMES)
            dd.token_sample(x[i:j], dtype, ld, j - i, V, z[i:j], j - i, noise_words=dev_words(torch, words[i:j]), logp=logp[i:j], n_kept=n[i:j],
                            dev_err=err, **a)
            dd.logits_truncate(x[i:j], dtype, ld, j - i, V, out[i:j], n_kept=n2[i:j], dev_err=err, **a)
        assert int(err.item()) == 0 and torch.equal(n, n2)
        got.append((z, n, logp, out))
    for u, v in zip(*got):
        assert torch.equal(u, v)


@pytest.mark.parametrize("V,dtype", [(3000, "fp32"), (9000, "fp32"), (132000, "bf16")])
def test_draws_of_one_row_equal_single_ones(V, dtype):
    """Runs of draws from one row, also across rows left out, numbers out of range, rows that allow nothing, greedy draws and
    settings of which some do not hold, equal the same draws in calls of few."""
    torch = torch_or_skip()
    rng = np.random.default_rng(V)
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    R, per, ld = 12, 7, int(dd.logits_ld(V))
    n = 7 * cus + 5
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn((R, ld), generator=g, device="cuda") * 3
    x[3, 5], x[4] = np.nan, -np.inf
    x = x.bfloat16() if dtype == "bf16" else x
    ids = np.repeat(rng.integers(0, R, n // 50 + 1), 50)[:n]
    ids[rng.random(n) < 0.05] = -1
    ids[[40, 41, 300]] = [R, -2, 2 ** 31 - 1]
    S = -(-n // per)
    s = draw_settings(rng, S, V)
    s[9]["temperature"], s[20]["top_p"], s[21]["min_p"] = -1.0, -0.5, 2.0
    words = words_of(rng, n)
    got = []
    step = per * (cus // per)
    for most in (n, step):
        z, kept, err = dev_i32(torch, np.full(n, -9)), dev_i32(torch, np.full(n, -9)), dev_i32(torch, [0])
        logp = torch.full((n,), 7.0, device="cuda")
        for i in range(0, n, most):
            j = min(n, i + most)
            dd.token_sample(x, dtype, ld, R, V, z[i:j], j - i, row_ids=dev_i32(torch, ids[i:j]), draws_per_seq=per,
                            noise_words=dev_words(torch, words[i:j]), logp=logp[i:j], n_kept=kept[i:j], dev_err=err,
                            **settings(torch, s[i // per:-(-j // per)], NAMES))
        assert int(err.item()) == dd.DD_DEVERR_SAMPLING | dd.DD_DEVERR_LOGITS
        got.append((z, kept, torch.nan_to_num(logp, nan=-77.0)))
    for u, v in zip(*got):
        assert torch.equal(u, v)
    assert (got[0][0][dev_i32(torch, ids) == -1] == -9).all() and len(set(got[0][0].tolist())) > 100


@pytest.mark.parametrize("V,R,dtype", [(985, 6, "fp32"), (3000, 600, "fp32"), (9000, 6, "fp32"), (9000, 300, "fp32"), (140000, 3, "bf16")])
def test_a_bin_that_is_cut_again(V, R, dtype):
    """Five values under a temperature that puts all in one bin.  The zeros before the first of the largest fall into the part
    of the numbers just above them, which is cut again: what is listed then ends where that part ends."""
    torch = torch_or_skip()
    rng = np.random.default_rng(V)
    l = rng.choice([1.0, 1e-40, 0.0, -1e-40, -1.0], V)
    l[:9], l[9] = 0.0, 1.0
    l = np.tile(round_to_dtype(l[None], dtype), (R, 1))
    up, t = int((l[0] > 0).sum()), f32(1e11)
    at = np.concatenate([np.arange(up - 4, up + 14), rng.integers(1, V, R)])[:R] if R > 20 else up + np.arange(R)
    # the at-th class in order, as all weights are next to 1; and at classes
    words = np.floor((at + 0.5) / V * 2.0 ** 32).astype(np.uint64)
    check(torch, l, dtype, [dict(OFF, temperature=t)] * R, words, sure=1.0)
    check(torch, l, dtype, [dict(OFF, temperature=t, top_k=int(k)) for k in at], words, sure=0.9)
    check(torch, l, dtype, [dict(OFF, temperature=t, top_p=float(k) / V) for k in at], words, sure=0.9)


@pytest.mark.parametrize("R", [6, 600])
def test_a_bin_that_reaches_the_lowest_numbers(R):
    """Numbers that weigh nothing stand in one bin down to the type's lowest: its last part would end past 64 bits."""
    torch = torch_or_skip()
    V = 2100
    rng = np.random.default_rng(5)
    l = np.sign(rng.normal(size=V)) * 10.0 ** rng.uniform(-40, 37, V)
    l[rng.permutation(V)[:100]] = -2.0 ** 127 * rng.uniform(1, 1.99, 100)
    l = np.tile(round_to_dtype(l[None], "fp32"), (R, 1))
    k = V - np.array([1, 2, 30, 60, 95, 100]) if R == 6 else V - np.arange(R) // 3
    check(torch, l, "fp32", [dict(OFF, top_k=int(x)) for x in k], words_of(rng, R), sure=1.0)


@pytest.mark.parametrize("V,dtype", [(33, "fp32"), (33, "bf16"), (6000, "fp32"), (6000, "bf16")])
def test_rows_one_call_each(V, dtype):
    """Rows of one call equal, bit for bit, the same rows in calls of their own."""
    torch = torch_or_skip()
    rng = np.random.default_rng(V)
    R, ld = 600, int(dd.logits_ld(V))
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn((R, ld), generator=g, device="cuda") * 4
    x = x.bfloat16() if dtype == "bf16" else x
    a = settings(torch, draw_settings(rng, R, V), NAMES)
    words = dev_words(torch, words_of(rng, R))
    got = []
    for k in (R, 1):
        z, n, n2, err = (dev_i32(torch, np.full(m, -9)) for m in (R, R, R, 1))
        err.zero_()
        logp, out = torch.zeros(R, device="cuda"), torch.full_like(x, 3.0)
        for i in range(0, R, k):
            s = {name: t[i:i + k] for name, t in a.items()}
            dd.token_sample(x[i:i + k], dtype, ld, k, V, z[i:i + k], k, noise_words=words[i:i + k], logp=logp[i:i + k], n_kept=n[i:i + k], dev_err=err, **s)
            dd.logits_truncate(x[i:i + k], dtype, ld, k, V, out[i:i + k], n_kept=n2[i:i + k], dev_err=err, **s)
        assert int(err.item()) == 0 and torch.equal(n, n2)
        got.append((z, n, logp, out))
    for u, v in zip(*got):
        assert torch.equal(u, v)


@pytest.mark.parametrize("V", [985, 9000, 50257])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_settings_at_their_ends(V, dtype):
    """Smallest and largest temperatures, shares next to 0 and 1, counts around a workgroup's threads."""
    torch = torch_or_skip()
    rng = np.random.default_rng(V)
    under = 1 - 2.0 ** -24
    some = [dict(temperature=t) for t in (1e-44, 1e-30, 3e38)] + [dict(top_p=p) for p in (0.0, 1e-30, under, np.inf)] + \
        [dict(min_p=m) for m in (1e-45, 1e-10, under)] + [dict(top_k=k) for k in (1, 255, 256, 257, 511, 512, 513, 1024, 1025, V - 1, V, 2 ** 31 - 1, -2 ** 31)] + \
        [dict(temperature=1e20, top_k=V // 2, top_p=0.5), dict(temperature=1e-3, top_k=V - 1), dict(temperature=0.01, top_k=700, top_p=under, min_p=1e-30)]
    some = [dict(OFF, **s) for s in some]
    R = len(some)
    l = round_to_dtype(rng.normal(size=(R, V)) * rng.choice([0.5, 3.0, 40.0], (R, 1)), dtype)
    l[rng.random(l.shape) < 0.1] = -np.inf
    l[:, V // 2] = 1.0
    check(torch, l, dtype, some, rng.integers(2 ** 28, 2 ** 32 - 2 ** 28, R, dtype=np.uint64), sure=0.9)
