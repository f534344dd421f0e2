"""dd_denoise_forward_cached against the oracle, and the operators of a serving program together: requests that
enter, verify drafted blocks under edited logits, keep what was accepted, end and give their blocks back."""
import numpy as np
import pytest

import workloads
from oracle import cache as oc, forward as oforward, masks, params as oparams, verify as overify
from paper_2609_04010_amd import _lib as dd
from tests.gpu_util import GAP, dev_i32, logits_dev, say, torch_or_skip

pytestmark = pytest.mark.gpu

# the forward pass's bars (fp32: 1e-4): the oracle reads the GPU's own cache, so nothing else is rounded
LOGIT_TOL = {"bf16": 5e-2, "fp32": 1e-4}


class Server:
    """A program that keeps a pool, tables and lengths; every array of the GPU's is the call's own output."""

    def __init__(self, torch, cfg, seed, S, T, n_blocks, P, ld_table):
        self.torch, self.cfg, self.S, self.T, self.P, self.ld = torch, cfg, S, T, P, ld_table
        self.params_host = oparams.split_storage(cfg, workloads.host_params(cfg, seed, oparams.specs(cfg)))
        blob = dd.pack_params(cfg, oparams.storage_tensors(cfg, self.params_host))
        self.params = torch.zeros(blob.size, dtype=torch.uint8, device="cuda")
        dd.init_params(cfg, self.params, host_blob=blob)
        H = cfg["n_heads"]
        self.cc = dd.cache_config(n_blocks, P, H, cfg["d_model"] // H)
        self.codes, self.scales = dd.cache_tensors(self.cc, layers=cfg["n_layers"])
        self.codes.fill_(0x7F)                                   # NaN wherever nothing was written
        self.m = dd.CacheMap.empty(S, T, ld_table)
        self.length = dev_i32(torch, np.zeros(S))
        self.free, self.n_free = dev_i32(torch, np.random.default_rng(seed).permutation(n_blocks)), dev_i32(torch, [n_blocks])
        self.ldl = int(dd.logits_ld(cfg["vocab"]))
        tdt = torch.bfloat16 if cfg["dtype"] == "bf16" else torch.float32
        self.logits = torch.zeros((T, self.ldl), dtype=tdt, device="cuda")
        self.max_kv = min(ld_table * P, cfg["max_len"])
        self.ws = torch.full((dd.cached_workspace_bytes(cfg, self.cc, S, T, T, self.max_kv),), 255, dtype=torch.uint8, device="cuda")
        dd.workspace_reset(self.ws)

    def plan(self, n_new):
        before = [x.cpu().numpy() for x in (self.length, self.m.held, self.m.block_table, self.free)]
        nf = int(self.n_free.item())
        dd.cache_plan(self.cc, self.m, self.length, dev_i32(self.torch, n_new), self.m.held, self.free, self.n_free, self.n_free,
                      dev_err=self.ws[:4].view(self.torch.int32))
        w = oc.plan(self.cc.n_blocks, self.P, self.ld, self.T, before[0], n_new, before[1], before[2], before[3], nf)
        g = dict(kv_len=self.m.kv_len, held=self.m.held, table=self.m.block_table, free=self.free, row_start=self.m.row_start,
                 row_seq=self.m.row_seq, row_pos=self.m.row_pos, slots=self.m.slots)
        assert not w["err"] and int(self.n_free.item()) == w["n_free"]
        for k, x in g.items():
            assert np.array_equal(x.cpu().numpy(), w[k]), k
        return w

    def forward(self, z, alpha, pattern="causal", gate=None):
        """One pass; returns the logits and checks them, and the cache that it leaves, against the oracle."""
        cfg, w = self.cfg, {k: getattr(self.m, k).cpu().numpy() for k in ("kv_len", "row_start", "block_table", "slots")}
        c0, s0 = self.codes.cpu().numpy(), self.scales.cpu().numpy().astype(np.float64)
        dd.denoise_forward_cached(cfg, self.params, dev_i32(self.torch, z), alpha, self.cc, self.codes, self.scales, self.m,
                                  self.logits, self.ldl, self.ws, self.T, self.max_kv, pattern=pattern,
                                  lora_gate=None if gate is None else dev_i32(self.torch, gate))
        assert dd.read_device_error(self.ws[:4].view(self.torch.int32)) == 0
        c1, s1 = self.codes.cpu().numpy(), self.scales.cpu().numpy().astype(np.float64)
        ref, kvs = oc.forward_cached(cfg, self.params_host, np.asarray(z), alpha, c1, s1, self.P, w["block_table"], w["kv_len"],
                                     w["row_start"], pattern == "causal", gate)
        n = int(w["row_start"][-1])
        got = self.logits[:, :cfg["vocab"]].double().cpu().numpy()
        err = float(np.abs(got[:n] - ref[:n]).max())
        say(f"pass of {n} rows, lengths {w['kv_len'].tolist()}: max |dlogit| = {err:.3e} (std {ref[:n].std():.3f})")
        assert err <= LOGIT_TOL[cfg["dtype"]]
        if cfg["dtype"] == "fp32":
            # the codes are those of the oracle's keys and values but where fp32 stands on the other side of a
            # border: then the neighbouring code, and rarely
            for l, (k, v) in enumerate(kvs):
                wc, wsc = oc.append(c0[l], s0[l], self.P, k, v, w["row_start"], w["slots"])
                assert np.array_equal(wsc, s1[l])
                a, b = oc.decode(c1[l]), oc.decode(wc)
                same = (a == b) | (np.isnan(a) & np.isnan(b))
                assert same.mean() > 0.999 and (np.abs(a - b)[~same] <= np.maximum(np.abs(b)[~same] / 8, 2.0 ** -9)).all()
        return got


def _tiny(**over):
    return workloads.model_cfg(1, max_len=160, **over)


@pytest.mark.parametrize("cfg", [_tiny(), _tiny(norm="rms", lora_rank=16, lora_alpha=32.0), _tiny(time_cond=False, prior="uniform"),
                                 workloads.model_cfg(2, n_layers=2, vocab=300, max_len=256),
                                 workloads.model_cfg(2, n_layers=2, vocab=300, max_len=256, norm="rms", lora_rank=64, lora_alpha=128.0)],
                         ids=["fp32", "fp32-lora", "fp32-uniform", "bf16", "bf16-lora"])
def test_cached_passes_against_oracle(cfg):
    """Prompts of odd lengths, a second pass with one row each, a block that sees itself whole, padding rows."""
    torch = torch_or_skip()
    rng = np.random.default_rng(4)
    sv = Server(torch, cfg, 11, S=3, T=150, n_blocks=16, P=32, ld_table=5)
    V = cfg["vocab"]
    gate = (lambda n: rng.integers(0, 2, n)) if cfg.get("lora_rank") else (lambda n: None)
    toks = lambda: np.where(np.arange(150) < n, rng.integers(0, V, 150), -5)   # noqa: E731
    for n_new, alpha, pattern in (([33, 1, 70], 1.0, "causal"), ([1, 1, 1], 1.0, "causal"), ([16, 0, 9], 0.4, "bidirectional"),
                                  ([0, 100, 40], 0.9, "causal")):
        w = sv.plan(np.array(n_new))
        n = int(w["row_start"][-1])
        sv.forward(toks(), alpha, pattern, gate(150))
        sv.length.copy_(sv.m.kv_len)


def test_one_pass_is_the_uncached_forward_but_for_the_cache_rounding():
    """A whole sequence in one pass, fp32: the logits of dd_denoise_forward_ex (causal) up to what rounding keys and
    values to 8 bits changes, which the oracle shows on its own side."""
    torch = torch_or_skip()
    cfg = _tiny()
    rng = np.random.default_rng(5)
    L, V = 90, cfg["vocab"]
    sv = Server(torch, cfg, 12, S=1, T=L, n_blocks=4, P=32, ld_table=3)
    z = rng.integers(0, V, L)
    sv.plan(np.array([L]))
    got = sv.forward(z, 0.7)
    ref = oforward.forward(cfg, sv.params_host, z[None], 0.7, vis=masks.causal(L))[0]
    c, s = sv.codes.cpu().numpy(), sv.scales.cpu().numpy().astype(np.float64)
    mine, _ = oc.forward_cached(cfg, sv.params_host, z, 0.7, c, s, 32, sv.m.block_table.cpu().numpy(), [L], [0, L])
    say(f"rounding of the cache moves logits by {np.abs(mine - ref).max():.3e} of std {ref.std():.3f}")
    assert np.abs((got - ref) - (mine - ref)).max() <= 1e-4
    assert np.corrcoef(got.ravel(), ref.ravel())[0, 1] > 0.99


def test_serving_loop():
    """Requests enter with prompts, verify drafted blocks under penalties and masks, keep what is accepted, and end;
    every call's result is the oracle's."""
    torch = torch_or_skip()
    cfg = _tiny()
    rng = np.random.default_rng(6)
    S, B, V, T = 4, 5, cfg["vocab"], 128
    sv = Server(torch, cfg, 13, S, T, n_blocks=14, P=32, ld_table=5)
    text = [list(rng.integers(0, V, n)) for n in (40, 3, 66, 0)]      # the last slot stays empty at first
    live = np.array([True, True, True, False])
    H = 160
    allow = rng.integers(0, 2 ** 32, (2, (V + 31) // 32), dtype=np.uint64).astype(np.uint32) | np.uint32(0xFFFF)
    rep = rng.uniform(1.0, 1.4, S).astype(np.float32)
    pres, freq = rng.uniform(0, 0.3, S).astype(np.float32), rng.uniform(0, 0.1, S).astype(np.float32)
    f32 = lambda x: torch.from_numpy(x).cuda()   # noqa: E731
    emitted = 0
    for step in range(8):
        if step == 4:                                                # one request ends, another one enters
            text[0], live[0] = [], False
            text[3], live[3] = list(rng.integers(0, V, 20)), True
        cached = sv.length.cpu().numpy()
        # the tokens a request's pass runs on: what the cache lacks of its text, then the drafted ones
        fresh = [text[s][cached[s]:] if live[s] else [] for s in range(S)]
        draft = rng.integers(0, V, (S, B - 1))
        n_new = np.array([len(fresh[s]) + B - 1 if live[s] else -1 for s in range(S)])
        w = sv.plan(n_new)
        z = np.full(T, -9)
        for s in range(S):
            if live[s]:
                z[w["row_start"][s]:w["row_start"][s + 1]] = fresh[s] + list(draft[s])
        got = sv.forward(z, 1.0)
        # the last B rows of each request are its block's target logits
        ids = [s for s in range(S) if live[s]]
        pick = np.concatenate([np.arange(w["row_start"][s + 1] - B, w["row_start"][s + 1]) for s in ids])
        n = len(ids)
        p = sv.logits[torch.from_numpy(pick).cuda()].contiguous()
        hist = np.full((n, H), -1)
        for i, s in enumerate(ids):
            h = text[s] + list(draft[s])
            hist[i, :len(h)] = h
        hl = np.array([len(text[s]) + i for s in ids for i in range(B)])
        aid = rng.integers(-1, 2, n * B)
        dd.logits_edit(p, "fp32", sv.ldl, n * B, V, p, B, history=dev_i32(torch, hist), hist_len=dev_i32(torch, hl),
                       repetition=f32(rep[ids]), presence=f32(pres[ids]), frequency=f32(freq[ids]),
                       allow=dev_i32(torch, allow.view(np.int32)), allow_id=dev_i32(torch, aid))
        ok = [np.array([m[v // 32] >> np.uint32(v % 32) & 1 for v in range(V)], bool) for m in allow]
        want = oc.edit(got[pick], np.arange(n * B) // B, history=hist, hist_len=hl, repetition=rep[ids], presence=pres[ids],
                       frequency=freq[ids], allow=ok, allow_id=aid)
        pl = p[:, :V].double().cpu().numpy()
        fin = np.isfinite(want)
        assert np.array_equal(fin, np.isfinite(pl)) and np.abs(pl[fin] - want[fin]).max() <= 2.0 ** -20 * 16
        ql = rng.normal(size=(n, B - 1, V))
        ql += np.where(np.isfinite(pl.reshape(n, B, V)[:, :-1]), pl.reshape(n, B, V)[:, :-1], 0)
        ql = ql.astype(np.float32).astype(np.float64)
        q = logits_dev(torch, ql.reshape(n * (B - 1), V), "fp32", sv.ldl)
        no, zo, err = dev_i32(torch, np.zeros(n)), dev_i32(torch, np.zeros(n)), dev_i32(torch, [0])
        vw = torch.zeros(dd.spec_verify_workspace_bytes(n, B), dtype=torch.uint8, device="cuda")
        dd.spec_verify(p, q, "fp32", sv.ldl, n, B, V, dev_i32(torch, draft[ids]), no, zo, vw, seed=77, step=step, dev_err=err)
        assert int(err.item()) == 0
        with np.errstate(divide="ignore", invalid="ignore"):
            rn, rz, marg, gaps = overify.spec_verify(pl.reshape(n, B, V), ql, draft[ids], overify.PhiloxVerifyNoise(77, step))
        gn, gz = no.cpu().numpy(), zo.cpu().numpy()
        clear = np.abs(marg).min(axis=1) > 1e-4
        assert np.array_equal(gn[clear], rn[clear])
        sure = clear & (gn == rn) & (gaps.min(axis=1) > GAP)
        assert np.array_equal(gz[sure], rz[sure])
        keep = cached.copy()
        for i, s in enumerate(ids):
            acc = list(draft[s][:gn[i] - 1])
            if aid[i * B + gn[i] - 1] >= 0:
                assert ok[aid[i * B + gn[i] - 1]][gz[i]], "a token that its row's mask does not allow"
            text[s] = text[s] + acc + [int(gz[i])]
            keep[s] = len(text[s]) - 1                               # all but the token just drawn is in the cache
            emitted += len(acc) + 1
        keep[[s for s in range(S) if not live[s]]] = 0
        sv.length.copy_(dev_i32(torch, keep))
    say(f"{emitted} tokens in 8 passes; {int(sv.n_free.item())} of {sv.cc.n_blocks} blocks free")
    assert int(sv.n_free.item()) + int(sv.m.held.sum().item()) == sv.cc.n_blocks


def test_cached_forward_in_a_graph():
    """A verification pass captured once and replayed with other tokens and lengths equals the eager passes."""
    torch = torch_or_skip()
    cfg = workloads.model_cfg(2, n_layers=2, vocab=300, max_len=256)
    rng = np.random.default_rng(7)
    a, b = (Server(torch, cfg, 14, S=2, T=40, n_blocks=12, P=32, ld_table=6) for _ in range(2))
    z0 = dev_i32(torch, rng.integers(0, 300, 40))

    def step(sv, z, n_new):
        dd.cache_plan(sv.cc, sv.m, sv.length, n_new, sv.m.held, sv.free, sv.n_free, sv.n_free)
        dd.denoise_forward_cached(cfg, sv.params, z, 1.0, sv.cc, sv.codes, sv.scales, sv.m, sv.logits, sv.ldl, sv.ws, 40, sv.max_kv)
        sv.length.copy_(sv.m.kv_len)
    n_new = dev_i32(torch, [20, 11])
    for sv in (a, b):
        step(sv, z0, n_new)
    zs, ns = z0.clone(), n_new.clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(b, zs, ns)
    for n in ([5, 16], [1, 0], [16, 3], [7, 24]):
        z = dev_i32(torch, rng.integers(0, 300, 40))
        zs.copy_(z)
        ns.copy_(dev_i32(torch, n))
        g.replay()
        step(a, z, dev_i32(torch, n))
        torch.cuda.synchronize()
        k = sum(n)
        assert torch.equal(a.logits[:k], b.logits[:k]) and torch.equal(a.m.kv_len, b.m.kv_len)
        assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    assert dd.read_device_error(b.ws[:4].view(torch.int32)) == 0


def test_profiler_counts_the_launches():
    torch = torch_or_skip()
    cfg = workloads.model_cfg(2, n_layers=2, vocab=300, max_len=256)
    sv = Server(torch, cfg, 15, S=1, T=20, n_blocks=4, P=32, ld_table=3)
    z = dev_i32(torch, np.arange(20))
    dd.profile_begin(200, ["cache_plan", "cache_append", "cache_attention", "logits_edit"])
    try:
        dd.cache_plan(sv.cc, sv.m, sv.length, dev_i32(torch, [20]), sv.m.held, sv.free, sv.n_free, sv.n_free)
        dd.denoise_forward_cached(cfg, sv.params, z, 1.0, sv.cc, sv.codes, sv.scales, sv.m, sv.logits, sv.ldl, sv.ws, 20, sv.max_kv)
        dd.logits_edit(sv.logits, "bf16", sv.ldl, 20, 300, sv.logits)
    finally:
        dd.profile_end()
    got = dd.profile_read()
    say(got)
    assert {k: v[0] for k, v in got.items()} == {"cache_plan": 1, "cache_append": 2, "cache_attention": 2, "logits_edit": 1}
    assert all(v[1] > 0 for v in got.values())
