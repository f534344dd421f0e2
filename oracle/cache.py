"""The cached context of a serving pass, and edits of logits, in float64.

Written from the definitions: block tables by walking the sequences, the 8-bit cache by the table of the
256 e4m3 numbers, attention by a softmax per row, edits by one class after the other.
"""
import math

import numpy as np

E_MIN, E_MAX = -100, 120


def e4m3_values():
    """The 256 numbers: sign, 4 exponent bits of bias 7, 3 mantissa bits; 0x7F and 0xFF are NaN."""
    out = np.zeros(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        x = math.ldexp(1 + m / 8, e - 7) if e else math.ldexp(m / 8, -6)
        out[c] = math.nan if c & 127 == 127 else -x if c & 128 else x
    return out


_VAL = e4m3_values()
_POS = _VAL[:127]          # ascending


def encode(x):
    """Codes of the nearest e4m3 numbers, ties to the even code; |x| <= 448 or not finite (NaN codes)."""
    x = np.asarray(x, dtype=np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    hi = np.clip(np.searchsorted(_POS, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _POS[hi] - a, a - _POS[lo]
    c = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    c = np.where(_POS[hi] == a, hi, c)
    c = np.where(np.isfinite(x), c, 127)
    return (c + np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def decode(codes):
    return _VAL[np.asarray(codes, dtype=np.uint8)]


def plan(n_blocks, P, ld_table, T, seq_len, n_new, held, table, free, n_free):
    """dd_cache_plan; returns a dict of the arrays it writes, with "err" True where nothing was done."""
    S = len(seq_len)
    table, free = np.array(table), np.array(free)
    fit = 0 <= n_free <= n_blocks
    need, give = [], 0
    for s in range(S):
        if n_new[s] < -1 or seq_len[s] < 0 or not 0 <= held[s] <= ld_table or seq_len[s] > held[s] * P:
            fit = False
            need.append(0)
        elif n_new[s] == -1:
            give += held[s]
            need.append(0)
        else:
            total = seq_len[s] + n_new[s]
            fit = fit and total <= min(ld_table * P, 2 ** 31 - 1)
            need.append(max(0, -(-total // P) - held[s]))
    rows = sum(max(0, int(n)) for n in n_new)
    fit = fit and rows <= T and n_free + give <= n_blocks and sum(need) <= n_free + give
    out = dict(table=table, free=free, row_seq=np.full(T, -1), row_pos=np.full(T, -1), slots=np.full(T, -1))
    if not fit:
        out.update(err=True, kv_len=np.array(seq_len), held=np.array(held), row_start=np.zeros(S + 1, int), n_free=n_free)
        return out
    top = n_free
    for s in range(S):
        if n_new[s] == -1:
            for j in range(held[s]):
                free[top] = table[s, j]
                top += 1
    err = False
    kv, hold, start, r = [], [], [0], 0
    for s in range(S):
        if n_new[s] == -1:
            kv.append(0)
            hold.append(0)
        else:
            for j in range(need[s]):
                top -= 1
                table[s, held[s] + j] = free[top]
            kv.append(seq_len[s] + n_new[s])
            hold.append(held[s] + need[s])
            for i in range(n_new[s]):
                pos = seq_len[s] + i
                b = table[s, pos // P]
                out["row_seq"][r], out["row_pos"][r] = s, pos
                if 0 <= b < n_blocks:
                    out["slots"][r] = b * P + pos % P
                else:
                    err = True
                r += 1
        start.append(r)
    out.update(err=err, kv_len=np.array(kv, int), held=np.array(hold, int), row_start=np.array(start), n_free=top)
    return out


def v_index(P, dh):
    """Where feature f of the token at place o stands among a block's value codes: index [P][dh]."""
    o, f = np.arange(P)[:, None], np.arange(dh)[None, :]
    return o // 32 * 32 * dh + f * 32 + o % 32


def scale_exponent(a):
    """The smallest e with a <= 448 * 2^e, clamped."""
    if a == 0:
        return E_MIN
    e = math.frexp(a)[1] - 10
    while a > math.ldexp(448.0, e):
        e += 1
    return min(max(e, E_MIN), E_MAX)


def append(codes, scales, P, k, v, row_start, slots):
    """dd_cache_append on copies: codes uint8 [n_blocks, H, 2 P dh], scales [n_blocks, H, 2], k and v
    [T, H, dh]; returns (codes, scales)."""
    codes, scales = codes.copy(), scales.astype(np.float64).copy()
    H, dh = k.shape[1], k.shape[2]
    vi = v_index(P, dh)
    for s in range(len(row_start) - 1):
        r = row_start[s]
        while r < row_start[s + 1]:
            if slots[r] < 0:
                r += 1
                continue
            b, off = slots[r] // P, slots[r] % P
            n = min(P - off, row_start[s + 1] - r)
            for h in range(H):
                for w, x in enumerate((k[r:r + n, h], v[r:r + n, h])):
                    x = np.asarray(x, dtype=np.float64)
                    fin = np.isfinite(x)
                    e = scale_exponent(np.abs(x[fin]).max() if fin.any() else 0.0)
                    body = codes[b, h, w * P * dh:(w + 1) * P * dh]
                    at = np.arange(P * dh).reshape(P, dh) if w == 0 else vi
                    if off:
                        old = math.frexp(scales[b, h, w])[1] - 1
                        if e > old:
                            body[:] = encode(decode(body) * 2.0 ** (old - e))
                        e = max(e, old)
                    body[at[off:off + n]] = encode(x * 2.0 ** -e)
                    scales[b, h, w] = 2.0 ** e
            r += n
    return codes, scales


def gather(codes, scales, P, dh, blocks, L):
    """Keys and values [L, H, dh] of the first L tokens in these blocks."""
    vi = v_index(P, dh)
    k = np.concatenate([decode(codes[b][:, :P * dh]).reshape(-1, P, dh) * scales[b][:, :1, None] for b in blocks], 1)
    v = np.concatenate([decode(codes[b][:, P * dh:])[:, vi] * scales[b][:, 1:, None] for b in blocks], 1)
    return k.transpose(1, 0, 2)[:L], v.transpose(1, 0, 2)[:L]


def attention(q, k, v, first, causal, scale):
    """Rows q [n, Hq, dh] at positions first .. over keys and values [L, Hkv, dh]; zeros where nothing is visible.
    NaN keys and values count for the rows that see them alone."""
    n, Hq, dh = q.shape
    L, Hkv = k.shape[0], k.shape[1]
    out = np.zeros((n, Hq, dh))
    for i in range(n):
        see = min(max(first + i + 1, 0), L) if causal else L
        if see == 0:
            continue
        for h in range(Hq):
            kh = h // (Hq // Hkv)
            w = k[:see, kh] @ q[i, h] * scale
            m = np.max(w[~np.isnan(w)], initial=-np.inf)
            p = np.exp(w - m)
            out[i, h] = (p @ v[:see, kh]) / p.sum()
    return out


def edit(l, seq, history=None, hist_len=None, repetition=None, presence=None, frequency=None, bias=None, allow=None,
         allow_id=None):
    """Rows l [rows, V] of sequence seq[m]; history [n_seq] lists, bias [n_seq] lists of (id, value), allow [n_allow]
    boolean masks over the classes."""
    l = np.array(l, dtype=np.float64)
    rows, V = l.shape
    for m in range(rows):
        s = seq[m]
        n = None if hist_len is None else int(hist_len[m])
        if n is not None and n < 0:
            continue
        h = [] if history is None else list(history[s])[:n]
        rep = 1.0 if repetition is None else float(repetition[s])
        pre = 0.0 if presence is None else float(presence[s])
        fre = 0.0 if frequency is None else float(frequency[s])
        count = {}
        for t in h:
            if 0 <= t < V:
                count[int(t)] = count.get(int(t), 0) + 1
        for t, c in count.items():
            x = l[m, t]
            l[m, t] = (x / rep if x > 0 else x * rep) - (pre + c * fre)
        for t, x in ({} if bias is None else {int(t): x for t, x in bias[s]}).items():
            if 0 <= t < V:
                l[m, t] += x
        if allow is not None:
            a = 0 if allow_id is None else int(allow_id[m])
            if 0 <= a < len(allow):
                l[m, ~allow[a]] = -np.inf
    return l


def forward_cached(cfg, P, z, alpha_t, codes, scales, block, table, kv_len, row_start, causal=True, gate=None):
    """The denoiser on rows z [T] over caches that already hold the rows' own keys and values: codes uint8
    [layers, n_blocks, H, 2 block dh], scales [layers, n_blocks, H, 2].  Returns the logits [T, V] (zero rows of
    padding) and every layer's keys and values [T, H, dh] before their rounding."""
    from . import forward as fw
    T, d, H = len(z), cfg["d_model"], cfg["n_heads"]
    dh, S = d // H, len(kv_len)
    pos, live = np.zeros(T, int), np.zeros(T, bool)
    for s in range(S):
        n = row_start[s + 1] - row_start[s]
        pos[row_start[s]:row_start[s + 1]] = kv_len[s] - n + np.arange(n)
        live[row_start[s]:row_start[s + 1]] = True
    g = np.ones(T) if gate is None else np.asarray(gate, dtype=np.float64)
    h = P["tok_emb"][np.where(live, z, 0)] + P["pos_emb"][pos]
    if cfg.get("time_cond", True):
        h = h + fw.time_embedding(alpha_t, d)[None]
    kvs = []
    for l in range(cfg["n_layers"]):
        p = lambda n: P[f"l{l}.{n}"]   # noqa: E731
        proj = lambda name, a: fw.projection(cfg, P, l, name, a[None], g)[0]   # noqa: E731
        qkv = proj("qkv", fw.normalise(cfg, h, p("ln1_g"), p("ln1_b"))).reshape(T, 3, H, dh)
        kvs.append((qkv[:, 1], qkv[:, 2]))
        o = np.zeros((T, H, dh))
        for s in range(S):
            r0, r1, L = row_start[s], row_start[s + 1], int(kv_len[s])
            if r1 > r0:
                k, v = gather(codes[l], scales[l], block, dh, table[s][:-(-L // block)], L)
                o[r0:r1] = attention(qkv[r0:r1, 0], k, v, L - (r1 - r0), causal, dh ** -0.5)
        h = h + proj("o", o.reshape(T, d))
        a = fw.normalise(cfg, h, p("ln2_g"), p("ln2_b"))
        h = h + proj("2", fw.gelu_tanh(proj("1", a)))
    out = fw.normalise(cfg, h, P["lnf_g"], P["lnf_b"]) @ P["w_out"].T
    out[~live] = 0
    return out, kvs
