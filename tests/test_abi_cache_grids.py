"""Sizes of the cached context's calls at the largest launch that the runtime takes (2^32 - 1 work-items); no GPU needed: refused
calls end before any launch, and for sizes that fit only the workspace is asked."""
import pytest

import workloads
from paper_2609_04010_amd import _lib as dd
from tests.test_abi_cache import _append, _attend, _cache, _cached, _map


def _bytes(S, T, max_new, max_kv=256, block=64):
    c = _cache(n_kv_heads=12, n_blocks=100, block=block)
    return dd.cached_workspace_bytes(workloads.model_cfg(2), c, S, T, max_new, max_kv)


def test_attention_with_a_loose_bound_on_new_rows():
    """1024 sequences, 32 heads of 128, the pass's row count as bound on each: 2^24 workgroups of 256 work-items."""
    c, m = _cache(n_kv_heads=32, head_dim=128), _map(S=1024, T=65536)
    args = dict(heads=32, ldq=4096, ldo=4096)
    assert _attend(c, m, max_new=65536, **args) == 6 and _attend(c, m, max_new=65536, pattern=0, **args) == 6


def test_attention_at_the_limit():
    """One row each of S sequences, 12 heads: 12 S workgroups of 256 work-items."""
    fits = ((1 << 24) - 1) // 12 // 8 * 8 - 8
    assert _bytes(fits, 1 << 20, 1) > 0
    assert _bytes(fits + 16, 1 << 20, 1) == 0
    m = _map(S=fits + 16, T=1 << 20)
    assert _attend(_cache(n_kv_heads=12), m, heads=12, ldq=768, ldo=768, max_new=1) == 6


def test_append_at_the_limit():
    """One row each of S sequences: a workgroup per row and four heads' keys or values."""
    c = _cache(n_kv_heads=8192)
    rows = (1 << 24) // 4096
    ld = 8192 * 64
    assert _append(c, _map(S=rows, T=rows), ld=ld) == 6
    # many rows of few sequences: a workgroup per touched block, head and kind
    assert _append(c, _map(S=1, T=64 * 1022), ld=ld) == 6


def test_append_of_many_short_sequences_still_fits():
    """2^19 sequences of one token, 12 heads: six workgroups each, four heads' keys or values in one."""
    assert _bytes(1 << 19, 1 << 19, 1) > 0


@pytest.mark.parametrize("T,ok", [((1 << 26) - 4, True), ((1 << 26) - 3, False), (1 << 27, False)])
def test_rows_of_the_denoiser(T, ok):
    assert (_bytes(1, T, 16, block=256) > 0) == ok
    if not ok:
        assert _cached(c=_cache(n_kv_heads=12, block=256), m=_map(T=T), wsb=1 << 62) == 6
