"""dd_logits_edit on requests at their start: histories that begin empty and grow row by row, beside many biases."""
import numpy as np
import pytest

from paper_2609_04010_amd import _lib as dd
from tests.gpu_util import dev_i32, logits_dev, round_to_dtype, say, torch_or_skip
from tests.test_gpu_edit import _args, _case, _oracle

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("S,per,V,nb", [
    (700, 16, 300, 250),         # a workgroup's rows within one sequence
    (650, 20, 300, 250),         # a new request first in its group, behind one with a longer history
    (1200, 6, 300, 250),         # two requests in one group
    (300, 16, 2048 + 700, 2000)])   # two pieces, biases over several rounds of a workgroup's threads
def test_edit_of_histories_that_start_empty(dtype, S, per, V, nb):
    """Lengths 0, 1, 2, .. of each request, several rows per workgroup, more biased classes in a piece than a wavefront
    has lanes."""
    torch = torch_or_skip()
    rng = np.random.default_rng(S + V)
    H = per
    c = _case(rng, S, per, V, H, nb, 1, False)
    c["history"] = rng.integers(0, V, (S, H))                      # mostly classes without a bias of their own
    c["hist_len"] = np.tile(np.arange(per), S)
    c["hist_len"][5::11 * per] = -1
    c["bias_ids"] = np.stack([rng.permutation(V)[:nb] for _ in range(S)])
    keep = ("history", "hist_len", "repetition", "presence", "frequency", "bias_ids", "bias_values")
    rows, ld = S * per, int(dd.logits_ld(V))
    l = round_to_dtype(rng.normal(size=(rows, V)) * 3, dtype)
    x, err = logits_dev(torch, l, dtype, ld), dev_i32(torch, [0])
    out = torch.full_like(x, -7.0)
    say("edit", dtype, "rows", rows, "of", V, "biases", nb)
    dd.logits_edit(x, dtype, ld, rows, V, out, per, dev_err=err, **_args(torch, c, keep))
    want = _oracle(c, keep, l)
    got = out[:, :V].double().cpu().numpy()
    assert int(err.item()) == 0
    # the roundings of test_edit_against_oracle: six of fp32 of no more than the largest term, one to the type
    term = np.abs(l) * 1.6 + 0.5 + 0.3 * H + 16
    tol = np.abs(want) * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) + 6 * 2.0 ** -24 * term
    d = np.abs(got - want)
    assert (d <= tol).all(), float((d / tol).max())
