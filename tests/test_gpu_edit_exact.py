"""The repetition penalty of dd_logits_edit is a division, rounded once: equal to fp32 division, not near it."""
import numpy as np
import pytest

from paper_2609_04010_amd import _lib as dd
from tests.gpu_util import dev_i32, logits_dev, round_to_dtype, say, torch_or_skip

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("S,per,V", [(5, 3, 1000), (300, 16, 2500)])
def test_repetition_is_divided_by(dtype, S, per, V):
    torch = torch_or_skip()
    rng = np.random.default_rng(V)
    rows, ld = S * per, int(dd.logits_ld(V))
    l = round_to_dtype(rng.normal(size=(rows, V)) * 5, dtype)
    l[:, ::17] = 0.0
    l[:, 1::19] = -np.inf
    l[:, 2::23] = np.inf
    rep = rng.uniform(0.5, 2.0, S).astype(np.float32)
    rep[0] = 1e-39                                       # 1 / rep is beyond fp32, l / rep of a small l is not
    l[:per] = round_to_dtype(rng.uniform(-1e-3, 1e-3, (per, V)), dtype)
    x = logits_dev(torch, l, dtype, ld)
    say("edit", dtype, rows, V)
    dd.logits_edit(x, dtype, ld, rows, V, x, per, history=dev_i32(torch, np.tile(np.arange(V), (S, 1))),
                   repetition=torch.from_numpy(rep).cuda())
    f, r = l.astype(np.float32), np.repeat(rep, per)[:, None]
    with np.errstate(over="ignore"):
        want = np.where(f > 0, f / r, f * r)             # numpy's fp32 division and product: each rounded once
    want = round_to_dtype(want, dtype)
    got = x[:, :V].double().cpu().numpy()
    assert np.array_equal(got, want), (int((got != want).sum()), np.argwhere(got != want)[:5])
