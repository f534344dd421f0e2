"""Refusals of the cached context's and the logit edits' entry points (no GPU needed: each call fails its
validation, or has nothing to do, before any launch; the pointers are never followed)."""
import ctypes

import pytest

from paper_2609_04010_amd import _lib as dd

P = ctypes.c_void_p
FAKE = 0x10000
REF = ctypes.byref


def _cache(**kw):
    a = dict(n_blocks=8, block=64, n_kv_heads=2, head_dim=64)
    a.update(kw)
    return dd.DDCache(**a)


def _map(**kw):
    a = dict(S=2, T=8, ld_table=4, block_table=FAKE, held=FAKE, kv_len=FAKE, row_start=FAKE, row_seq=FAKE, row_pos=FAKE,
             slots=FAKE)
    a.update(kw)
    return dd.DDCacheMap(**a)


def _plan(c, m, **kw):
    a = dict(seq_len=FAKE, n_new=FAKE, held=FAKE, free=FAKE, n_free=FAKE, n_free_out=FAKE)
    a.update(kw)
    return dd.lib().dd_cache_plan(REF(c) if c else None, REF(m) if m else None, a["seq_len"], a["n_new"], a["held"],
                                  a["free"], a["n_free"], a["n_free_out"], None, None)


def _append(c, m, **kw):
    a = dict(codes=FAKE, scales=FAKE, k=FAKE, v=FAKE, dtype=0, ld=128)
    a.update(kw)
    return dd.lib().dd_cache_append(REF(c), a["codes"], a["scales"], REF(m), a["k"], a["v"], a["dtype"], a["ld"], None, None)


def _attend(c, m, **kw):
    a = dict(codes=FAKE, scales=FAKE, q=FAKE, ldq=256, out=FAKE, ldo=256, dtype=0, heads=4, pattern=1, scale=0.125,
             max_new=4, max_kv=256, ws=None, wsb=0)
    a.update(kw)
    return dd.lib().dd_cache_attention(REF(c), a["codes"], a["scales"], REF(m), a["q"], a["ldq"], a["out"], a["ldo"],
                                       a["dtype"], a["heads"], a["pattern"], a["scale"], a["max_new"], a["max_kv"],
                                       a["ws"], a["wsb"], None, None)


BAD_CACHE = [(dict(n_blocks=0), 1), (dict(n_blocks=-3), 1), (dict(n_kv_heads=0), 1), (dict(block=16), 6), (dict(block=48), 6),
             (dict(block=512), 6), (dict(head_dim=16), 6), (dict(head_dim=96), 6), (dict(n_blocks=1 << 25, block=64), 6)]


@pytest.mark.parametrize("kw,status", BAD_CACHE)
def test_caches_that_are_refused(kw, status):
    c = _cache(**kw)
    assert _plan(c, _map()) == status and _append(c, _map()) == status and _attend(c, _map()) == status
    assert dd.cache_attention_workspace_bytes(c, 2, 8, 4, 4, 256) == 0


BAD_MAP = [dict(S=-1), dict(T=-1), dict(ld_table=0), dict(row_start=None), dict(block_table=None), dict(kv_len=None),
           dict(held=None), dict(row_seq=None), dict(slots=None), dict(row_pos=None)]


@pytest.mark.parametrize("kw", BAD_MAP)
def test_maps_that_are_refused(kw):
    m = _map(**kw)
    assert _plan(_cache(), m) == 1 and _append(_cache(), m) == 1 and _attend(_cache(), m) == 1


@pytest.mark.parametrize("kw", [dict(S=(1 << 24) + 1), dict(T=(1 << 30) + 1), dict(ld_table=(1 << 26) + 1)])
def test_maps_that_are_too_large(kw):
    m = _map(**kw)
    assert _plan(_cache(), m) == 6 and _append(_cache(), m) == 6 and _attend(_cache(), m) == 6


@pytest.mark.parametrize("name", ["seq_len", "n_new", "held", "free", "n_free", "n_free_out"])
def test_plan_refuses_null(name):
    assert _plan(_cache(), _map(), **{name: None}) == 1
    assert _plan(None, _map()) == 1 and _plan(_cache(), None) == 1


@pytest.mark.parametrize("kw,status", [(dict(dtype=2), 3), (dict(ld=(1 << 21) + 8), 6), (dict(ld=127), 2), (dict(ld=132), 2), (dict(ld=126, dtype=1), 2),
                                       (dict(codes=None), 1), (dict(scales=None), 1), (dict(k=None), 1), (dict(v=None), 1),
                                       (dict(k=FAKE + 8), 1), (dict(codes=FAKE + 4), 1), (dict(scales=FAKE + 4), 1)])
def test_append_refusals(kw, status):
    assert _append(_cache(), _map(), **kw) == status


def test_nothing_to_do_is_done():
    for m in (_map(S=0, block_table=None, held=None, kv_len=None), _map(T=0, row_seq=None, row_pos=None, slots=None)):
        assert _append(_cache(), m, codes=None, scales=None, k=None, v=None) == 0
        assert _attend(_cache(), m, codes=None, scales=None, q=None, out=None) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=7), 3), (dict(heads=0), 1), (dict(heads=3), 2), (dict(pattern=2), 6), (dict(pattern=9), 6), (dict(scale=0.0), 1),
    (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(max_new=0), 1), (dict(max_kv=0), 1),
    (dict(max_kv=257), 2), (dict(ldq=255), 2), (dict(ldq=260), 2), (dict(ldo=248), 2), (dict(q=None), 1), (dict(out=None), 1),
    (dict(codes=None), 1), (dict(q=FAKE + 2), 1), (dict(out=FAKE + 8), 1), (dict(ws=FAKE, wsb=16), 4), (dict(ws=None, wsb=1 << 40), 1),
    (dict(ws=FAKE + 64, wsb=1 << 40), 1), (dict(max_kv=(1 << 30) + 1), 6), (dict(max_new=1 << 30), 6)])
def test_attention_refusals(kw, status):
    m = _map(ld_table=4 if kw.get("wsb", 0) == 0 else 64)
    if kw.get("wsb", 0):
        kw = dict(kw, max_kv=4096)              # long enough to be cut: a workspace is needed
    assert _attend(_cache(), m, **kw) == status


def test_attention_workspace_grows_with_what_is_cut():
    c = _cache(n_blocks=1000)
    n = [dd.cache_attention_workspace_bytes(c, 1, 1, 4, 1, kv) for kv in (64, 4096, 32768)]
    assert n[0] == 0 < n[1] <= n[2] and n[1] % 256 == 0
    assert dd.cache_attention_workspace_bytes(c, 0, 0, 4, 1, 64) == 0
    assert dd.cache_attention_workspace_bytes(c, 1, 1, 3, 1, 64) == 0


def _edit(e=None, **kw):
    a = dict(logits=FAKE, dtype=0, ld=64, rows=4, V=32, out=FAKE, per=2)
    a.update(kw)
    return dd.lib().dd_logits_edit(a["logits"], a["dtype"], a["ld"], a["rows"], a["V"], a["out"], a["per"],
                                   REF(dd.DDLogitsEdits(**(e or {}))) if e != "null" else None, None, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=5), 3), (dict(V=0), 1), (dict(rows=-1), 1), (dict(per=0), 1), (dict(ld=31), 2), (dict(ld=36), 2),
    (dict(V=(1 << 24) + 1, ld=1 << 25), 6), (dict(rows=(1 << 30) + 1), 6), (dict(logits=None), 1), (dict(out=None), 1), (dict(out=FAKE + 8), 1),
    (dict(e="null"), 1), (dict(e=dict(ld_history=-1)), 1), (dict(e=dict(n_bias=-1)), 1), (dict(e=dict(bias_ids=FAKE)), 1),
    (dict(e=dict(bias_values=FAKE)), 1), (dict(e=dict(allow_id=FAKE)), 1), (dict(e=dict(allow=FAKE, ld_allow=1, n_allow=0)), 2),
    (dict(e=dict(allow=FAKE, ld_allow=0, n_allow=1)), 2), (dict(e=dict(n_allow=-1)), 1)])
def test_edit_refusals(kw, status):
    assert _edit(**kw) == status


def test_edit_of_no_rows():
    assert _edit(rows=0, logits=None, out=None) == 0


def test_map_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    z = torch.zeros((2, 4), dtype=torch.int32)
    with pytest.raises(ValueError):
        dd.CacheMap(z, z[:, 0], z[:, 0], z[0], z[0], z[0], z[0])


def _cached(cfg=None, c=None, m=None, **kw):
    import workloads
    cfg = dd.make_config(dict(workloads.model_cfg(2), **(cfg or {})))
    a = dict(params=FAKE, z=FAKE, alpha=1.0, codes=FAKE, scales=FAKE, pattern=1, max_new=4, max_kv=256, gate=None, logits=FAKE,
             ld=50304, ws=FAKE, wsb=1 << 40)
    a.update(kw)
    return dd.lib().dd_denoise_forward_cached(
        REF(cfg), a["params"], a["z"], a["alpha"], REF(c or _cache(n_kv_heads=12)), a["codes"], a["scales"], REF(m or _map()),
        a["pattern"], a["max_new"], a["max_kv"], a["gate"], a["logits"], a["ld"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(cfg=dict(d_model=770)), 1), (dict(cfg=dict(n_heads=24)), 6), (dict(c=_cache(n_kv_heads=6)), 2),
    (dict(c=_cache(n_kv_heads=12, head_dim=32)), 2), (dict(c=_cache(n_kv_heads=12, block=40)), 6), (dict(m=_map(S=-1)), 1),
    (dict(alpha=1.5), 1), (dict(pattern=0, codes=None), 1), (dict(pattern=3), 6), (dict(max_kv=257), 2), (dict(max_kv=1025), 2),
    (dict(max_new=0), 1), (dict(gate=FAKE), 1), (dict(ld=50000), 2), (dict(ld=50257), 2), (dict(params=None), 1), (dict(z=None), 1),
    (dict(scales=None), 1), (dict(logits=None), 1), (dict(ws=None), 1), (dict(ws=FAKE + 16), 1), (dict(logits=FAKE + 8), 1),
    (dict(scales=FAKE + 4), 1), (dict(wsb=1000), 4)])
def test_cached_forward_refusals(kw, status):
    assert _cached(**kw) == status


def test_cached_workspace():
    import workloads
    cfg, c = workloads.model_cfg(2), _cache(n_kv_heads=12, n_blocks=100)
    n = dd.cached_workspace_bytes(cfg, c, 4, 64, 16, 1024)
    assert n >= dd.workspace_bytes(cfg, 1, 64) + dd.cache_attention_workspace_bytes(c, 4, 64, 12, 16, 1024)
    assert dd.cached_workspace_bytes(cfg, c, 4, 64, 16, 1025) == 0      # beyond max_len
    assert _cached(m=_map(T=0, row_seq=None, row_pos=None, slots=None), logits=None, ws=None) == 0
