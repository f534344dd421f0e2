"""Attention over caches whose scales stand at the ends of their range: finite values, however large, give finite
results, and what stands in places behind the last token does not show."""
import numpy as np
import pytest

from oracle import cache as oc
from paper_2609_04010_amd import _lib as dd
from tests.gpu_util import dev_i32, say, torch_or_skip
from tests.test_gpu_cache import _attend, _attention_case, _check

pytestmark = pytest.mark.gpu

SHAPES = [([100, 0, 33], [7, 40, 1], 4, 2, 64, 32),            # whole sequences
          ([4000], [1], 2, 2, 64, 64),                        # cut into pieces
          ([370], [33], 150, 150, 128, 64), ([20], [40], 2100, 2100, 32, 32)]   # two wavefronts per tile, and one


def _case(torch, shape, dtype, e, most, stale):
    """Value codes up to `most` with scale 2^e; `stale` in all other places of the sequences' blocks."""
    lens, news, hq, hkv, dh, P = shape
    rng = np.random.default_rng(len(lens) + dh)
    t, codes, scales, q = _attention_case(torch, rng, lens, news, hq, hkv, dh, P, dtype, 0)
    vi = oc.v_index(P, dh)
    for s in range(len(lens)):
        L = int(t["kv"][s])
        for j in range(-(-L // P)):
            b, n = t["table"][s, j], min(P, L - j * P)
            codes[b][:, P * dh + vi[n:]] = stale
            codes[b][:, P * dh + vi[:n]] = oc.encode(np.clip(rng.normal(size=(hkv, n, dh)) * most / 4, -most, most))
    scales[:, :, 1] = 2.0 ** e
    return t, codes, scales, q


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("e,most,stale", [(120, 64, 0x7E), (119, 128, 0xFE), (112, 448, 0x7E), (-100, 448, 0x7E), (-100, 2, 0xFE)])
def test_values_at_the_ends_of_the_scales(shape, dtype, e, most, stale):
    """Values up to 2^126 (2^121 from codes of 448), or down to 2^-109; behind the last token codes of 448, which at the
    largest scale no fp32 number holds."""
    torch = torch_or_skip()
    lens, news, hq, hkv, dh, P = shape
    t, codes, scales, q = _case(torch, shape, dtype, e, most, stale)
    q = q / 64                                            # many tokens with a share each
    say("attention", shape, dtype, "scale 2^", e)
    err = dev_i32(torch, [0])
    for pattern in ("causal", "bidirectional") if hq < 10 else ("causal",):
        out, _ = _attend(torch, t, codes, scales, q, hq, hkv, dh, P, pattern, err=err)
        worst = _check(torch, t, codes, scales, q, out, hq, hkv, dh, P, pattern)
        say(pattern, "worst", worst, "of the bound")
    assert int(err.item()) == 0


def test_fp32_rows_of_large_values_through_append():
    """Values of 3e38 appended and attended to by queries of zero: the mean of the stored values."""
    torch = torch_or_skip()
    H, dh, P, L = 2, 64, 64, 200
    cc, m = dd.cache_config(4, P, H, dh), dd.CacheMap.empty(1, L, 4)
    free, z = dev_i32(torch, np.arange(4)), dev_i32(torch, [0])
    dd.cache_plan(cc, m, z, dev_i32(torch, [L]), z, free, dev_i32(torch, [4]), dev_i32(torch, [0]))
    codes, scales = dd.cache_tensors(cc)
    k = torch.ones((L, H * dh), device="cuda")
    v = torch.full((L, H * dh), 3.0e38, device="cuda")
    v[1::2] = -2.5e38
    dd.cache_append(cc, codes, scales, m, k, v)
    out = torch.zeros_like(k)
    n = dd.cache_attention_workspace_bytes(cc, 1, L, H, L, L)
    ws = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
    dd.cache_attention(cc, codes, scales, m, torch.zeros_like(k), out, H, L, L, ws, pattern="bidirectional")
    # codes of 3e38 and -2.5e38 at scale 2^120: 225.7 -> 224 and 188.08 -> 192; as many of each
    want = (224.0 - 192.0) / 2 * 2.0 ** 120
    got = out.double().cpu().numpy()
    # sums of 200 exact terms in fp32, the product with 1 / 200, the result: at most 200 + 3 half steps of the terms' mass
    assert np.abs(got - want).max() <= 203 * 2.0 ** -24 * 208.0 * 2.0 ** 120, np.abs(got - want).max()
