// Attention of a pass's rows over the 8-bit cache.
//
// The rows of one sequence that share a key head (rows x query heads per key head) are the columns of
// its products; a wavefront owns 32 columns and walks tiles of 32 tokens:
//   S^T = K Q^T   v_mfma_f32_32x32x16_bf16, first operand K, second the wavefront's Q, held in registers.
//   O^T += V^T P^T  first operand V, second the probabilities as they leave the first product.
// e4m3 numbers times a power of two are exact in bf16, so the codes become operands with
// v_cvt_scalef32_pk_bf16_fp8, which also applies the block's scale; nothing else is done per cached number.
// A lane's column of S^T (and of O^T) is one query: maximum, sum and rescaling stay in the lane, with one
// exchange between lane and lane ^ 32 per tile for the maximum.
//
// Operand layout.  Row m = 8 i + 4 g + j of the 32 x 32 result is register 4 i + j of half g (lane >> 5).
// The lane that loads key row m takes token 16 g + 4 i + j of the tile, so half g ends with tokens
// 16 g .. 16 g + 15 in register order, which are the 16 consecutive bytes of V (tokens innermost in
// the cache) that the half loads for each feature: no shuffle, transposition or LDS between the products.
// The head dimension enters K Q^T in the order that 16-byte loads give: load i of half g holds features
// 32 i + 16 g .. + 15, steps 2 i and 2 i + 1.
//
// fp32 rows: q (and the probabilities) are taken as the sum of three bf16 numbers of 8 bits each, which is
// exact, one product each.
//
// A workgroup is four wavefronts: KW of them share a column tile and take every KW-th tile of tokens, their
// results meet in LDS; 4 / KW column tiles side by side.  Long caches are cut into pieces of `chunk` tokens
// over workgroups whose partial results cache_attn_join_kernel adds.
#include <math.h>

#include <algorithm>

#include "cache.h"
#include "mfma.h"

namespace dd {

// eight codes as a bf16 operand, times the scale (a power of two)
DD_DEV bf16x8 cvt8(uint32_t lo, uint32_t hi, float scale) {
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    const auto b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const auto c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    const auto d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
DD_DEV bf16x8 half8(const uint4& u, int h, float scale) {
    return h ? cvt8(u.z, u.w, scale) : cvt8(u.x, u.y, scale);
}
DD_DEV f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// x as NS bf16 numbers: one, rounded to nearest even; or three of 8 bits each, whose sum is x
template <int NS> DD_DEV void split8(const float (&x)[8], bf16x8 (&o)[NS]) {
    uint32_t u[NS][4];
    if constexpr (NS == 1) {
#pragma unroll
        for (int e = 0; e < 4; ++e) u[0][e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t h[3][2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float v = x[2 * e + k];
                const bool fin = fabsf(v) < INFINITY;
                h[0][k] = v != v ? 0x7FC00000u : __float_as_uint(v) & 0xFFFF0000u;
                const float r = fin ? v - __uint_as_float(h[0][k]) : 0.f;
                h[1][k] = __float_as_uint(r) & 0xFFFF0000u;
                h[2][k] = __float_as_uint(r - __uint_as_float(h[1][k])) & 0xFFFF0000u;
            }
#pragma unroll
            for (int p = 0; p < 3; ++p) u[p][e] = h[p][0] >> 16 | h[p][1];
        }
    }
#pragma unroll
    for (int p = 0; p < NS; ++p) o[p] = __builtin_bit_cast(bf16x8, u32x4{u[p][0], u[p][1], u[p][2], u[p][3]});
}

DD_DEV int wave_min_int(int v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = min(v, __shfl_xor(v, o, 64));
    return __builtin_amdgcn_readfirstlane(v);
}
DD_DEV int wave_max_int(int v) { return -wave_min_int(-v); }

template <typename T> DD_DEV void store4(T* p, float4 v);
template <> DD_DEV void store4<bf16_t>(bf16_t* p, float4 v) {
    *(uint2*)p = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
}
template <> DD_DEV void store4<float>(float* p, float4 v) { *(float4*)p = v; }

DD_DEV float4 scaled(float4 v, float f) { return make_float4(v.x * f, v.y * f, v.z * f, v.w * f); }

template <typename T, int DH, int KW>
__global__ __launch_bounds__(256) void cache_attn_kernel(CacheAttnArgs a) {
    constexpr int CW = 4 / KW, NS = sizeof(T) == 4 ? 3 : 1, KS = DH / 16, MT = DH / 32;
    const int lane = threadIdx.x & 63, g = lane >> 5, ln = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kw = wave % KW, cw = wave / KW;

    // workgroup -> (sequence, key head, piece, column tiles): the column tiles of a piece, which read the
    // same tokens, are 8 apart in launch order, so that one XCD's L2 serves them
    const int ntile = (int)((a.max_new * (int64_t)a.G + 32 * CW - 1) / (32 * CW));
    const int slot = blockIdx.x >> 3;
    const int group = slot / ntile * 8 + (blockIdx.x & 7), ct = ntile - 1 - slot % ntile;   // the longest first
    if (group >= a.S * a.c.H * a.nsplit) return;
    const int piece = group % a.nsplit, sh = group / a.nsplit, h = sh % a.c.H, s = sh / a.c.H;

    const int kv = a.kv_len[s], most = (int)min((int64_t)a.max_kv, (int64_t)a.ld_table * a.c.P);
    const int L = min(max(kv, 0), most);
    const int r0 = min(max(a.row_start[s], 0), a.T), r1 = min(max(a.row_start[s + 1], r0), a.T);
    const int n = min(r1 - r0, a.max_new);
    if (a.err && threadIdx.x == 0 && h == 0 && piece == 0 && ct == 0 &&
        (kv < 0 || kv > most || r1 - r0 > a.max_new))
        atomicOr(a.err, DD_DEVERR_CACHE);
    const int cols = n * a.G;
    const int k0 = piece * a.chunk;
    if (ct * CW * 32 >= cols || (piece > 0 && k0 >= L)) return;
    const bool whole = L <= a.chunk;   // the sequence has this piece alone

    // this lane's column: row of the sequence and query head, and how many tokens it sees
    const int col = (ct * CW + cw) * 32 + ln;
    const bool real = col < cols;
    const int i = real ? col / a.G : 0, head = h * a.G + (real ? col % a.G : 0);
    int lim = L;
    if (real && a.causal) lim = min(max(kv - (r1 - r0) + i + 1, 0), L);
    const int lo = wave_min_int(lim), hi = wave_max_int(real ? lim : 0);

    bf16x8 q[KS][NS];
#pragma unroll
    for (int st = 0; st < KS; ++st) {
        float x[8] = {};
        if (real) {
            const T* p = (const T*)a.q + (int64_t)(r0 + i) * a.ldq + (int64_t)head * DH + (st >> 1) * 32 + g * 16 + (st & 1) * 8;
            if constexpr (NS == 1) {
                const uint4 u = *(const uint4*)p;
                q[st][0] = __builtin_bit_cast(bf16x8, u);
                continue;
            } else {
                const float4 y = ((const float4*)p)[0], z = ((const float4*)p)[1];
                x[0] = y.x; x[1] = y.y; x[2] = y.z; x[3] = y.w;
                x[4] = z.x; x[5] = z.y; x[6] = z.z; x[7] = z.w;
            }
        }
        split8<NS>(x, q[st]);
    }

    f32x16 o[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) o[mt] = f32x16{};
    float m = -INFINITY, l = 0.f;

    const int k1 = min(k0 + a.chunk, hi), nt = k1 > k0 ? (k1 - k0 + 31) >> 5 : 0;
    // block numbers and scales of 64 blocks from block bw on, one per lane (-1: not to be read)
    int bw = 0, id = -1;
    float2 sc = make_float2(0.f, 0.f);
    auto window = [&](int first) {
        bw = first;
        id = -1;
        const int b = first + lane;
        if ((int64_t)b << a.c.log2p < L) {
            id = a.table[(int64_t)s * a.ld_table + b];
            if (id < 0 || id >= a.c.n_blocks) {
                if (a.err) atomicOr(a.err, DD_DEVERR_CACHE);
                id = -1;
            }
        }
        if (id >= 0) sc = *(const float2*)(a.scales + ((int64_t)id * a.c.H + h) * 2);
    };
    struct Tile {
        uint4 k[DH / 32], v[MT];
        float ks, vs;
        bool ok;
    };
    const int krow = 16 * (ln >> 2 & 1) + 4 * (ln >> 3) + (ln & 3);   // the token whose key this lane loads
    auto fetch = [&](int t, Tile& x) {
        const int key0 = k0 + 32 * t, b = key0 >> a.c.log2p;
        if (b - bw >= 64) window(b);
        const int blk = __builtin_amdgcn_readlane(id, b - bw);
        x.ok = blk >= 0;
        if (!x.ok) return;
        x.ks = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sc.x), b - bw));
        x.vs = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sc.y), b - bw));
        const uint8_t* p = a.codes + cache_slab(a.c, DH, blk, h) + (int64_t)(key0 & (a.c.P - 1)) * DH;
        const uint8_t* pv = p + (int64_t)a.c.P * DH;
#pragma unroll
        for (int e = 0; e < DH / 32; ++e) x.k[e] = *(const uint4*)(p + krow * DH + e * 32 + g * 16);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) x.v[mt] = *(const uint4*)(pv + (mt * 32 + ln) * 32 + g * 16);
    };

    window(k0 >> a.c.log2p);
    Tile cur, nxt;
    if (kw < nt) fetch(kw, cur);
    for (int t = kw; t < nt; t += KW) {
        nxt.ok = false;
        if (t + KW < nt) fetch(t + KW, nxt);
        if (cur.ok) {
            f32x16 sT = {};
#pragma unroll
            for (int st = 0; st < KS; ++st) {
                const bf16x8 kf = half8(cur.k[st >> 1], st & 1, cur.ks);
#pragma unroll
                for (int p = NS - 1; p >= 0; --p) sT = mfma32(kf, q[st][p], sT);
            }
            const int key0 = k0 + 32 * t + 16 * g;
            const bool edge = k0 + 32 * t + 32 > lo;   // some column does not see the whole tile
            if (edge) {
#pragma unroll
                for (int r = 0; r < 16; ++r) sT[r] = key0 + r < lim ? sT[r] : -INFINITY;
            }
            float tm = sT[0];
#pragma unroll
            for (int r = 1; r < 16; ++r) tm = fmaxf(tm, sT[r]);
            tm = fmaxf(tm, __shfl_xor(tm, 32, 64)) * a.scale_log2;
            // the reference moves only where a score passes it by 2^8: sums stay far inside fp32
            if (__any(tm > m + 8.f)) {
                const float mn = fmaxf(m, tm), f = mn == m ? 1.f : __builtin_amdgcn_exp2f(m - mn);
                m = mn;
                l *= f;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[mt][r] *= f;
            }
            const float ref = m == -INFINITY ? 0.f : m;
            float p[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                p[r] = __builtin_amdgcn_exp2f(fmaf(sT[r], a.scale_log2, -ref));
                l += p[r];
            }
            if (edge) {
                // NaN codes in places that not every column sees (or nobody: beyond the sequence's end)
                // would reach every column as 0 * NaN: they leave V, and the columns that see one get it back
                uint32_t any = 0;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const uint4& u = cur.v[mt];
                    any |= ((u.x & 0x7F7F7F7Fu) + 0x01010101u) | ((u.y & 0x7F7F7F7Fu) + 0x01010101u) |
                           ((u.z & 0x7F7F7F7Fu) + 0x01010101u) | ((u.w & 0x7F7F7F7Fu) + 0x01010101u);
                }
                if (__any((any & 0x80808080u) != 0)) {
                    float see[16];
#pragma unroll
                    for (int r = 0; r < 16; ++r) see[r] = key0 + r < lim ? 1.f : 0.f;
                    bf16x8 sb[2][1];
                    split8<1>(*(const float(*)[8])see, sb[0]);
                    split8<1>(*(const float(*)[8])(see + 8), sb[1]);
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        uint32_t u[4] = {cur.v[mt].x, cur.v[mt].y, cur.v[mt].z, cur.v[mt].w}, w[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t b = (((u[e] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7;
                            u[e] &= ~(b * 0xFFu);
                            w[e] = b * 0x38u;   // 1.0
                        }
                        cur.v[mt] = make_uint4(u[0], u[1], u[2], u[3]);
                        f32x16 cnt = {};
                        cnt = mfma32(cvt8(w[0], w[1], 1.f), sb[0][0], cnt);
                        cnt = mfma32(cvt8(w[2], w[3], 1.f), sb[1][0], cnt);
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[mt][r] += cnt[r] > 0.f ? NAN : 0.f;
                    }
                }
            }
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = p[8 * st + e];
                bf16x8 pf[NS];
                split8<NS>(x, pf);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const bf16x8 vf = half8(cur.v[mt], st, cur.vs);
#pragma unroll
                    for (int e = NS - 1; e >= 0; --e) o[mt] = mfma32(vf, pf[e], o[mt]);
                }
            }
        }
        cur = nxt;
    }
    l += __shfl_xor(l, 32, 64);

    // four consecutive features of a column, normalised into out or, of a cut sequence, as they are
    auto put = [&](int row, int hd, int d, float4 v, float sum) {
        if (whole) {
            store4<T>((T*)a.out + (int64_t)row * a.ldo + (int64_t)hd * DH + d, scaled(v, sum == 0.f ? 0.f : 1.f / sum));
        } else {
            *(float4*)(a.part + (((int64_t)row * a.Hq + hd) * a.nsplit + piece) * DH + d) = v;
        }
    };
    auto put_ml = [&](int row, int hd, float mx, float sum) {
        float* ml = a.part + (int64_t)a.T * a.Hq * a.nsplit * DH;
        *(float2*)(ml + (((int64_t)row * a.Hq + hd) * a.nsplit + piece) * 2) = make_float2(mx, sum);
    };
    if constexpr (KW == 1) {
        if (!real) return;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                put(r0 + i, head, mt * 32 + 2 * r + 4 * g, make_float4(o[mt][r], o[mt][r + 1], o[mt][r + 2], o[mt][r + 3]), l);
        if (!whole && g == 0) put_ml(r0 + i, head, m, l);
    } else {
        // the KW results of a column tile meet in LDS, 32 features at a time
        constexpr int LDC = 36;   // floats per column: 16-byte rows whose starts fall on different banks
        __shared__ float so[4][32][LDC];
        __shared__ float sml[4][32][2];
        if (g == 0) {
            sml[wave][ln][0] = m;
            sml[wave][ln][1] = l;
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            if (mt) __syncthreads();
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *(float4*)&so[wave][ln][2 * r + 4 * g] = make_float4(o[mt][r], o[mt][r + 1], o[mt][r + 2], o[mt][r + 3]);
            __syncthreads();
#pragma unroll
            for (int c = 0; c < CW; ++c) {
                const int cl = threadIdx.x >> 3, d = (threadIdx.x & 7) * 4, cc = (ct * CW + c) * 32 + cl;
                if (cc >= cols) continue;
                float mx = -INFINITY, sum = 0.f;
#pragma unroll
                for (int k = 0; k < KW; ++k) mx = fmaxf(mx, sml[c * KW + k][cl][0]);
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int k = 0; k < KW; ++k) {
                    const float mk = sml[c * KW + k][cl][0], f = mk == mx ? 1.f : __builtin_amdgcn_exp2f(mk - mx);
                    const float4 y = *(const float4*)&so[c * KW + k][cl][d];
                    sum += sml[c * KW + k][cl][1] * f;
                    v.x += y.x * f; v.y += y.y * f; v.z += y.z * f; v.w += y.w * f;
                }
                const int row = r0 + cc / a.G, hd = h * a.G + cc % a.G;
                put(row, hd, mt * 32 + d, v, sum);
                if (!whole && mt == 0 && d == 0) put_ml(row, hd, mx, sum);
            }
        }
    }
}

// Adds the pieces of cut sequences: one wavefront per (row of a sequence, query head); lanes first hold one
// piece's maximum and sum each (at most 64), then DH / 64 features.
template <typename T, int DH>
__global__ __launch_bounds__(256) void cache_attn_join_kernel(CacheAttnArgs a) {
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int64_t per = (int64_t)a.max_new * a.Hq;
    const int s = (int)(item / per), i = (int)(item % per / a.Hq), head = (int)(item % a.Hq);
    if (s >= a.S) return;
    const int most = (int)min((int64_t)a.max_kv, (int64_t)a.ld_table * a.c.P);
    const int L = min(max(a.kv_len[s], 0), most), np = (L + a.chunk - 1) / a.chunk;
    const int r0 = min(max(a.row_start[s], 0), a.T), r1 = min(max(a.row_start[s + 1], r0), a.T);
    if (np < 2 || i >= r1 - r0) return;
    const int64_t at = ((int64_t)(r0 + i) * a.Hq + head) * a.nsplit;
    const float* part = a.part + at * DH;
    const float2* ml = (const float2*)(a.part + (int64_t)a.T * a.Hq * a.nsplit * DH) + at;
    const float2 x = lane < np ? ml[lane] : make_float2(-INFINITY, 0.f);
    const float mx = wave_max(x.x), f = x.x == mx ? 1.f : __builtin_amdgcn_exp2f(x.x - mx);
    const float sum = wave_sum(x.y * f);
    constexpr int N = DH < 64 ? 1 : DH / 64;
    float v[N] = {};
    if (lane * N < DH)
        for (int p = 0; p < np; ++p) {
            const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), p));
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] += w * part[(int64_t)p * DH + lane * N + e];
        }
    if (lane * N >= DH) return;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    T* out = (T*)a.out + (int64_t)(r0 + i) * a.ldo + (int64_t)head * DH + lane * N;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        if constexpr (sizeof(T) == 2) out[e] = f32_to_bf16(v[e] * inv);
        else out[e] = v[e] * inv;
    }
}

CacheAttnPlan cache_attn_plan(int32_t S, int32_t T, int32_t Hkv, int32_t Hq, int dh, int32_t max_new, int32_t max_kv) {
    CacheAttnPlan p;
    const int64_t cols = (int64_t)max_new * (Hq / Hkv);
    p.kw = cols <= 32 ? 4 : cols <= 64 ? 2 : 1;
    const int64_t wgs = std::max<int64_t>(1, (int64_t)S * Hkv * ceil_div(cols, 32 * (4 / p.kw)));
    const int64_t want = std::min<int64_t>(64, std::max<int64_t>(1, ceil_div(2048, wgs)));
    const int64_t unit = 32 * p.kw;
    const int64_t chunk = std::max<int64_t>(2 * unit, ceil_div(ceil_div(max_kv, want), unit) * unit);
    p.chunk = (int)std::min<int64_t>(chunk, ceil_div(max_kv, unit) * unit);
    p.nsplit = (int)ceil_div(max_kv, p.chunk);
    p.ws = p.nsplit == 1 ? 0 : ((size_t)T * Hq * p.nsplit * (dh + 2) * sizeof(float) + 255) & ~(size_t)255;
    return p;
}

template <typename T, int DH>
static void launch_cache_attn_t(const CacheAttnArgs& a, int kw, hipStream_t s) {
    const int64_t groups = (int64_t)a.S * a.c.H * a.nsplit;
    const int64_t tiles = ceil_div((int64_t)a.max_new * a.G, 32 * (4 / kw));
    const dim3 grid((unsigned)(ceil_div(groups, 8) * 8 * tiles));
    {
        ProfScope ps(KC_CACHE_ATTN, s);
        if (kw == 4) launch_k((cache_attn_kernel<T, DH, 4>), grid, dim3(256), 0, s, a);
        else if (kw == 2) launch_k((cache_attn_kernel<T, DH, 2>), grid, dim3(256), 0, s, a);
        else launch_k((cache_attn_kernel<T, DH, 1>), grid, dim3(256), 0, s, a);
    }
    if (a.nsplit > 1) {
        ProfScope ps(KC_CACHE_ATTN, s);
        launch_k((cache_attn_join_kernel<T, DH>), dim3((unsigned)ceil_div((int64_t)a.S * a.max_new * a.Hq, 4)), dim3(256), 0, s, a);
    }
}

dd_status launch_cache_attn(int dtype, const CacheAttnArgs& a, int kw, hipStream_t s) {
    switch (a.dh) {
#define X(d)                                                          \
    case d:                                                           \
        if (dtype == DD_BF16) launch_cache_attn_t<bf16_t, d>(a, kw, s); \
        else launch_cache_attn_t<float, d>(a, kw, s);                 \
        break;
        X(32) X(64) X(128)
#undef X
    }
    return launch_status("cache_attention");
}

}  // namespace dd
