"""Refusals of the sampling calls and of the calls on blocks between passes (no GPU needed: each fails its validation, or has
nothing to do, before any launch; the pointers are never followed)."""
import ctypes

import pytest

from paper_2609_04010_amd import _lib as dd

FAKE = 0x10000
REF = ctypes.byref


def _sample(**kw):
    a = dict(logits=FAKE, dtype=0, ld=64, rows=4, V=32, ids=None, n=4, per=1, how=dd.DDSampling(), z=FAKE)
    a.update(kw)
    return dd.lib().dd_token_sample(a["logits"], a["dtype"], a["ld"], a["rows"], a["V"], a["ids"], a["n"], a["per"],
                                    REF(a["how"]) if a["how"] else None, None, 0, 0, 0, a["z"], None, None, None, None)


def _truncate(**kw):
    a = dict(logits=FAKE, dtype=0, ld=64, rows=4, V=32, out=FAKE, per=1, how=dd.DDSampling())
    a.update(kw)
    return dd.lib().dd_logits_truncate(a["logits"], a["dtype"], a["ld"], a["rows"], a["V"], a["out"], a["per"],
                                       REF(a["how"]) if a["how"] else None, None, None, None)


BOTH = [(dict(dtype=2), 3), (dict(V=0), 1), (dict(rows=-1), 1), (dict(per=0), 1), (dict(ld=31), 2), (dict(ld=36), 2),
        (dict(V=(1 << 24) + 1, ld=1 << 25), 6), (dict(rows=(1 << 30) + 1), 6), (dict(logits=None), 1), (dict(logits=FAKE + 8), 1), (dict(how=None), 1)]


@pytest.mark.parametrize("kw,status", BOTH)
def test_refusals_of_both(kw, status):
    assert _sample(**kw) == status and _truncate(**kw) == status


@pytest.mark.parametrize("kw,status", [(dict(n=-1), 1), (dict(n=(1 << 30) + 1, ids=FAKE), 1), (dict(n=5), 2), (dict(z=None), 1), (dict(rows=0, n=1), 2)])
def test_sample_refusals(kw, status):
    assert _sample(**kw) == status


@pytest.mark.parametrize("kw,status", [(dict(out=None), 1), (dict(out=FAKE + 4), 1)])
def test_truncate_refusals(kw, status):
    assert _truncate(**kw) == status


def test_nothing_to_draw():
    assert _sample(n=0, logits=None, z=None) == 0 and _sample(n=0, rows=0) == 0 and _truncate(rows=0, logits=None, out=None) == 0


def _cache(**kw):
    a = dict(n_blocks=8, block=64, n_kv_heads=2, head_dim=64)
    a.update(kw)
    return dd.DDCache(**a)


def _map(table=FAKE, held=FAKE, kv_len=FAKE, **kw):
    a = dict(S=2, T=0, ld_table=4, block_table=table, held=held, kv_len=kv_len)
    a.update(kw)
    return dd.DDCacheMap(**a)


def _new(**kw):
    return _map(**dict(dict(table=FAKE + 0x1000, held=FAKE + 0x1000, kv_len=FAKE + 0x1000), **kw))


def _fork(c=None, m=None, to=None, **kw):
    a = dict(seq=FAKE, src=FAKE, free=FAKE, n_free=FAKE, n_out=FAKE, moves=FAKE, n_moves=FAKE, ws=FAKE, wsb=1 << 30)
    a.update(kw)
    return dd.lib().dd_cache_fork(REF(c or _cache()), REF(m or _map()), REF(to or _new()), a["seq"], a["src"], None, a["free"], a["n_free"], a["n_out"],
                                  a["moves"], a["n_moves"], a["ws"], a["wsb"], None, None)


def _compact(c=None, m=None, **kw):
    a = dict(out=FAKE, free=FAKE, n_out=FAKE, moves=FAKE, n_moves=FAKE, ws=FAKE, wsb=1 << 30)
    a.update(kw)
    return dd.lib().dd_cache_compact(REF(c or _cache()), REF(m or _map()), a["out"], a["free"], a["n_out"], a["moves"], a["n_moves"], a["ws"], a["wsb"],
                                     None, None)


def _copy(c=None, **kw):
    a = dict(codes=FAKE, scales=FAKE, layers=2, moves=FAKE, n=FAKE, most=3)
    a.update(kw)
    return dd.lib().dd_cache_copy(REF(c or _cache()), a["codes"], a["scales"], a["layers"], a["moves"], a["n"], a["most"], None, None)


@pytest.mark.parametrize("kw,status", [(dict(n_blocks=0), 1), (dict(block=48), 6), (dict(head_dim=16), 6), (dict(n_kv_heads=0), 1),
                                       (dict(n_blocks=1 << 25, block=64), 6)])
def test_caches_that_are_refused(kw, status):
    c = _cache(**kw)
    assert _fork(c) == status and _compact(c) == status and _copy(c) == status
    assert dd.cache_fork_workspace_bytes(c, 2, 2) == 0 and dd.cache_compact_workspace_bytes(c) == 0


@pytest.mark.parametrize("kw,status", [(dict(S=-1), 1), (dict(ld_table=0), 1), (dict(table=None), 1), (dict(held=None), 1), (dict(kv_len=None), 1),
                                       (dict(S=(1 << 16) + 1), 6), (dict(ld_table=(1 << 26) + 1), 6)])
def test_maps_that_are_refused(kw, status):
    assert _fork(m=_map(**kw)) == status and _fork(to=_new(**kw)) == status and _compact(m=_map(**kw)) == status


@pytest.mark.parametrize("kw,status", [(dict(seq=None), 1), (dict(src=None), 1), (dict(free=None), 1), (dict(n_free=None), 1), (dict(n_out=None), 1),
                                       (dict(moves=None), 1), (dict(n_moves=None), 1), (dict(ws=None), 1), (dict(ws=FAKE + 16), 1), (dict(wsb=100), 4),
                                       (dict(to=_new(table=FAKE)), 1), (dict(to=_new(held=FAKE)), 1), (dict(to=_new(kv_len=FAKE)), 1),
                                       (dict(seq=FAKE + 0x1000), 1)])
def test_fork_refusals(kw, status):
    assert _fork(**kw) == status


@pytest.mark.parametrize("kw,status", [(dict(out=None), 1), (dict(free=None), 1), (dict(n_out=None), 1), (dict(moves=None), 1), (dict(n_moves=None), 1),
                                       (dict(ws=None), 1), (dict(ws=FAKE + 64), 1), (dict(wsb=100), 4)])
def test_compact_refusals(kw, status):
    assert _compact(**kw) == status


@pytest.mark.parametrize("kw,status", [(dict(layers=-1), 1), (dict(most=-1), 1), (dict(layers=(1 << 16) + 1), 6), (dict(codes=None), 1), (dict(scales=None), 1),
                                       (dict(moves=None), 1), (dict(n=None), 1), (dict(codes=FAKE + 8), 1), (dict(scales=FAKE + 4), 1)])
def test_copy_refusals(kw, status):
    assert _copy(**kw) == status


def test_nothing_to_copy():
    assert _copy(layers=0, codes=None) == 0 and _copy(most=0, moves=None) == 0
    assert _copy(_cache(n_blocks=1, block=256, n_kv_heads=16384, head_dim=128), layers=1 << 11) == 6


def test_workspaces_grow():
    n = [dd.cache_fork_workspace_bytes(_cache(n_blocks=nb), 4, s) for nb, s in ((8, 1), (80000, 1), (80000, 5000))]
    assert 0 < n[0] < n[1] < n[2] and n[2] % 256 == 0
    assert dd.cache_fork_workspace_bytes(_cache(), 4, -1) == 0 and dd.cache_fork_workspace_bytes(_cache(), (1 << 16) + 1, 4) == 0
    assert 0 < dd.cache_compact_workspace_bytes(_cache()) < dd.cache_compact_workspace_bytes(_cache(n_blocks=80000))


def test_the_binding_refuses_host_tensors_and_short_ones():
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("the GPU tests cover the binding there")
    with pytest.raises(Exception):
        dd.token_sample(torch.zeros(4, 64), "fp32", 64, 4, 32, torch.zeros(4, dtype=torch.int32), 4)
