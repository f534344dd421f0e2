"""dd_logits_edit against the float64 oracle, and edited logits in the draws that follow."""
import numpy as np
import pytest

from oracle import cache as oc
from paper_2609_04010_amd import _lib as dd
from tests.gpu_util import dev_i32, logits_dev, round_to_dtype, say, torch_or_skip

pytestmark = pytest.mark.gpu


def _case(rng, S, per, V, H, nb, na, grow, rows=None):
    rows = rows or S * per
    c = dict(history=rng.integers(-2, V + 3, (S, H)), seq=np.arange(rows) // per)
    c["history"][:, ::3] = rng.integers(0, max(1, V // 50) + 1, c["history"][:, ::3].shape)    # tokens that repeat
    c["hist_len"] = np.array([min(H, H // 2 + m % per) if grow else H for m in range(rows)])
    if rows > 3:
        c["hist_len"][[1, 3]] = [-1, H + 50]
    c["repetition"] = rng.uniform(0.7, 1.6, S).astype(np.float32)
    c["presence"] = rng.uniform(-0.5, 0.5, S).astype(np.float32)
    c["frequency"] = rng.uniform(0, 0.3, S).astype(np.float32)
    c["bias_ids"] = rng.integers(-1, V + 1, (S, nb))
    if nb > 2:
        c["bias_ids"][:, 2] = c["bias_ids"][:, 0]                                             # an id listed twice
    c["bias_values"] = rng.normal(size=(S, nb)).astype(np.float32) * 3
    c["allow"] = rng.integers(0, 2 ** 32, (na, (V + 31) // 32), dtype=np.uint64).astype(np.uint32)
    c["allow_id"] = rng.integers(-1, max(na, 1), rows)
    return c


def _args(torch, c, keep):
    f = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()   # noqa: E731
    a = {}
    for k in keep:
        a[k] = f(c[k].view(np.int32)) if k == "allow" else f(c[k]) if c[k].dtype == np.float32 else dev_i32(torch, c[k])
    return a


def _oracle(c, keep, l):
    a = {k: c[k] for k in keep if k in ("history", "hist_len", "repetition", "presence", "frequency", "allow_id")}
    if "bias_ids" in keep:
        a["bias"] = [[(int(i), float(x)) for i, x in zip(ids, xs)] for ids, xs in zip(c["bias_ids"], c["bias_values"])]
    if "allow" in keep:
        V = l.shape[1]
        a["allow"] = [np.array([m[v // 32] >> np.uint32(v % 32) & 1 for v in range(V)], bool) for m in c["allow"]]
    return oc.edit(l, c["seq"], **a)


ALL = ("history", "hist_len", "repetition", "presence", "frequency", "bias_ids", "bias_values", "allow", "allow_id")
EDIT = [  # sequences, rows each, V, history, biases, masks, histories that grow
    (1, 1, 1, 1, 1, 1, False), (3, 5, 37, 20, 3, 2, True), (2, 17, 4096, 300, 40, 3, True),
    (4, 3, 4097, 1000, 7, 1, False), (2, 20, 12345, 64, 300, 4, True), (5, 1, 8190, 33, 0, 2, False),
    (700, 16, 300, 40, 5, 3, True), (9, 64, 9000, 90, 2, 3, True)]   # several rows per workgroup


@pytest.mark.parametrize("S,per,V,H,nb,na,grow", EDIT)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("keep", [ALL, ("history", "presence"), ("bias_ids", "bias_values"), ("allow",), ()])
def test_edit_against_oracle(S, per, V, H, nb, na, grow, dtype, keep):
    torch = torch_or_skip()
    rng = np.random.default_rng(V + H)
    c = _case(rng, S, per, V, H, nb, na, grow)
    rows, ld = S * per, int(dd.logits_ld(V))
    l = round_to_dtype(rng.normal(size=(rows, V)) * 3, dtype)
    l[rng.random(l.shape) < 0.01] = -np.inf
    l[rng.random(l.shape) < 0.001] = np.nan
    x = logits_dev(torch, l, dtype, ld)
    if ld > V:
        x[:, V:] = 5
    out, err = torch.full_like(x, -7.0), dev_i32(torch, [0])
    a = _args(torch, c, keep)
    dd.logits_edit(x, dtype, ld, rows, V, out, per, dev_err=err, **a)
    want = _oracle(c, keep, l)
    got = out.double().cpu().numpy()
    assert (got[:, V:] == -7).all() and int(err.item()) == 0
    got = got[:, :V]
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got == -np.inf, want == -np.inf)
    fin = np.isfinite(want)
    # at most six roundings of fp32 on the way (1 / repetition, its product, count * frequency, + presence, the difference,
    # + bias), each half a step of no more than the largest term, then one to the type
    term = np.abs(np.where(np.isfinite(l), l, 0)) * 1.6 + 0.5 + 0.3 * H + 16
    tol = np.abs(np.where(fin, want, 0)) * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) + 6 * 2.0 ** -24 * term
    d = np.abs(np.where(fin, got, 0) - np.where(fin, want, 0))
    assert (d <= tol).all(), float((d / tol).max())
    dd.logits_edit(x, dtype, ld, rows, V, x, per, **a)                    # in place
    assert torch.equal(torch.nan_to_num(x[:, :V].float()), torch.nan_to_num(out[:, :V].float()))
    assert ld == V or (x[:, V:] == 5).all()


@pytest.mark.parametrize("steps", [[3, 3, 3, 3], [0, 70, 0, 5], [5, -2, 9, 1], [64, 64, 65, 1]])
def test_edit_of_histories_that_jump(steps):
    """Rows edited together whose histories grow by much, shrink, or stand still, between rows that pass."""
    torch = torch_or_skip()
    rng = np.random.default_rng(17)
    S, per, V, H = 600, 16, 300, 1100
    c = _case(rng, S, per, V, H, 3, 1, False)
    c["history"] = rng.integers(0, 40, (S, H))
    n = np.cumsum(np.resize(steps, per)) + 5
    c["hist_len"] = np.tile(n, S)
    c["hist_len"][::7] = -1
    l = round_to_dtype(rng.normal(size=(S * per, V)) * 3, "fp32")
    x, out = logits_dev(torch, l, "fp32", 304), dev_i32(torch, [0])
    out, err = torch.zeros_like(x), out
    keep = ("history", "hist_len", "repetition", "presence", "frequency", "bias_ids", "bias_values")
    dd.logits_edit(x, "fp32", 304, S * per, V, out, per, dev_err=err, **_args(torch, c, keep))
    want = _oracle(c, keep, l)
    got = out[:, :V].double().cpu().numpy()
    assert int(err.item()) == 0
    term = np.abs(l) * 1.6 + 0.5 + 0.3 * H + 16               # as in test_edit_against_oracle
    assert (np.abs(got - want) <= np.abs(want) * 2.0 ** -24 + 6 * 2.0 ** -24 * term).all()


def test_edit_of_more_rows_than_the_grid_is_high():
    """More than 64 rows in each workgroup; whole numbers and halves, so nothing is rounded."""
    torch = torch_or_skip()
    rows, V, per, H, na = 65535 * 66 + 5, 5, 1000, 4, 7
    ld, S = int(dd.logits_ld(V)), -(-rows // per)
    g = torch.Generator(device="cuda").manual_seed(3)
    draw = lambda lo, hi, *shape: torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)   # noqa: E731
    x = draw(-8, 9, rows, ld).to(torch.bfloat16)
    history, hist_len = draw(0, V, S, H), draw(-1, H + 1, rows)
    allow, allow_id = draw(0, 2 ** V, na, 1), draw(-1, na, rows)
    presence = torch.full((S,), 0.5, device="cuda")
    say("edit rows", rows)
    out = torch.empty_like(x)
    dd.logits_edit(x, "bf16", ld, rows, V, out, per, history=history, hist_len=hist_len, presence=presence, allow=allow,
                   allow_id=allow_id)
    seq = torch.arange(rows, device="cuda") // per
    bits = (allow >> torch.arange(V, device="cuda", dtype=torch.int32)) & 1
    want = x[:, :V].float()
    named = torch.zeros_like(want, dtype=torch.bool)
    for i in range(H):
        named |= (history[seq, i, None] == torch.arange(V, device="cuda")) & (hist_len > i)[:, None]
    want = want - 0.5 * named
    shut = (bits[allow_id.clamp(min=0).long()] == 0) & (allow_id >= 0)[:, None] & (hist_len >= 0)[:, None]
    want = torch.where(shut, torch.full_like(want, -np.inf), want)
    assert torch.equal(out[:, :V].float(), want)


def test_edit_of_rows_past_the_last_whole_sequence_and_bad_mask_numbers():
    torch = torch_or_skip()
    rng = np.random.default_rng(3)
    S, per, V = 3, 4, 100
    c = _case(rng, S, per, V, 9, 2, 2, False, rows=10)                    # the third sequence has two rows
    l = round_to_dtype(rng.normal(size=(10, V)), "fp32")
    x, err = logits_dev(torch, l, "fp32", 128), dev_i32(torch, [0])
    c["allow_id"][4:6] = [2, -5]
    out = torch.zeros_like(x)
    dd.logits_edit(x, "fp32", 128, 10, V, out, per, dev_err=err, **_args(torch, c, ALL))
    assert int(err.item()) == dd.DD_DEVERR_MASK
    c["allow_id"][4:6] = -1
    want = _oracle(c, ALL, l)
    got = out[:, :V].double().cpu().numpy()
    assert np.array_equal(np.isfinite(got), np.isfinite(want))
    fin = np.isfinite(want)
    assert np.abs(got[fin] - want[fin]).max() <= 2.0 ** -20 * 8


def test_a_row_that_allows_nothing_is_reported_by_the_draw():
    """Edits, then the posterior's draw: allowed classes only; a row whose mask allows none keeps its token and sets
    the logits bit."""
    torch = torch_or_skip()
    V, rows, ld = 300, 64, 320
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn((rows, ld), generator=g, device="cuda").bfloat16()
    allow = np.zeros((2, 10), np.uint32)
    allow[0, 3] = 0xF0                                                    # classes 100 .. 103
    ids = np.zeros(rows, int)
    ids[7] = 1
    z = torch.full((rows,), V, dtype=torch.int32, device="cuda")
    zs, err = torch.empty_like(z), dev_i32(torch, [0])
    dd.logits_edit(x, "bf16", ld, rows, V, x, rows, allow=dev_i32(torch, allow.view(np.int32)), allow_id=dev_i32(torch, ids))
    dd.posterior_sample("mask", x, "bf16", ld, rows, V, z, 0.0, 1.0, zs, seed=3, dev_err=err)
    got = zs.cpu().numpy()
    say("drawn", sorted(set(got.tolist())))
    assert int(err.item()) == dd.DD_DEVERR_LOGITS and got[7] == V
    assert set(np.delete(got, 7).tolist()) <= {100, 101, 102, 103}
