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
// exact, one product each.  bf16 rows: the probabilities are rounded to bf16 for the product with V (their sum is not):
// another bf16 number of theirs would cost another product, and the result is rounded to bf16 in any case.  0.0020 off
// the 64-bit result (in norm), where fp32 probabilities give 0.0017.
//
// KW wavefronts of a workgroup share a column tile and take every KW-th tile of tokens; their results meet in
// LDS.  Where that leaves CUs idle, long caches are cut into pieces of `chunk` tokens over workgroups whose
// partial results cache_attn_join_kernel adds.
//
// Bound: few columns per key head, by the bytes of the cache (32 rows, 8 heads of 128, 16384 to 32768 tokens:
// 1.61 GB in 301 us, 5.4 TB/s, where reading such blocks and nothing else reaches 6.0; 64 x 16 rows, 12 heads of 64,
// 2048 to 4112 tokens: 307 MB in 60 us, 5.1 TB/s); many columns, by the vector instructions between the products
// (about 590 cycles per 32 x 32 tile, 256 of matrix instructions: prompts of 4 x 2048 rows, 64 GFLOP in 97 us).  Times
// here and below are those of calls that follow each other.
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

// maximum of a lane and the one 32 from it, in both
DD_DEV float max_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Values enter the products times 2^-16 and the result leaves times 2^16.  Scales go up to 2^120: as they stand, codes of
// 256 and more would be infinite in bf16 (and, in places behind the last token, 0 * inf), and sums of 2^8 times a value, or
// of many values, pass fp32's end before the division.  With it every code is finite, a sum of weights
// may reach 2^16 at the largest value (2^32 at 2^112), and the smallest code, 2^-109, is 2^-125, still a normal number.
constexpr float V_DOWN = 0x1p-16f, V_UP = 0x1p16f;

// KW wavefronts share a column tile, CW column tiles side by side, NB tiles of tokens in a wavefront's registers
// (NB - 1 ahead of the one in work).
template <typename T, int DH, int KW, int CW, int NB>
__global__ __launch_bounds__(64 * KW * CW) void cache_attn_kernel(CacheAttnArgs a) {
    constexpr int NS = sizeof(T) == 4 ? 3 : 1, KS = DH / 16, MT = DH / 32;
    constexpr int WC = 32 * CW;   // columns of a workgroup
    const int lane = threadIdx.x & 63, g = lane >> 5, ln = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kw = wave % KW, cw = wave / KW;

    // workgroup -> (sequence, key head, piece, column tiles): an XCD (every eighth workgroup) has all column
    // tiles of a piece, which read the same tokens; the last tiles, which see most, start first
    const int ntile = (int)((a.max_new * (int64_t)a.G + WC - 1) / WC);
    const int groups = a.S * a.c.H * a.nsplit, gx = (groups + 7) >> 3;
    const int slot = blockIdx.x >> 3;
    const int group = slot % gx * 8 + (blockIdx.x & 7), ct = ntile - 1 - slot / gx;
    if (group >= groups) return;
    // (pieces outermost: the XCDs share every piece's workgroups, of which the last ones may have nothing to do)
    const int nsh = a.S * a.c.H, piece = group / nsh, sh = group - piece * nsh, s = sh / a.c.H, h = sh - s * a.c.H;

    // block numbers and scales of 64 blocks from block bw on, one per lane (-1: not to be read); the table may be
    // read before the length is known
    const int k0 = piece * a.chunk;
    int bw = k0 >> a.c.log2p, id = -1;
    float2 sc = make_float2(0.f, 0.f);
    if (bw + lane < a.ld_table) id = a.table[(int64_t)s * a.ld_table + bw + lane];

    const int kv = a.kv_len[s], most = (int)min((int64_t)a.max_kv, (int64_t)a.ld_table * a.c.P);
    const int L = min(max(kv, 0), most);
    const int r0 = min(max(a.row_start[s], 0), a.T), r1 = min(max(a.row_start[s + 1], r0), a.T);
    const int n = min(r1 - r0, a.max_new);
    if (a.err && threadIdx.x == 0 && h == 0 && piece == 0 && ct == 0 &&
        (kv < 0 || kv > most || r1 - r0 > a.max_new))
        atomicOr(a.err, DD_DEVERR_CACHE);
    const int cols = n * a.G;
    if (ct * WC >= cols || (piece > 0 && k0 >= L)) return;
    const bool whole = L <= a.chunk;   // the sequence has this piece alone

    auto scales = [&]() {
        const bool in = (int64_t)(bw + lane) << a.c.log2p < L;
        if (in && (id < 0 || id >= a.c.n_blocks) && a.err) atomicOr(a.err, DD_DEVERR_CACHE);
        if (!in || id < 0 || id >= a.c.n_blocks) id = -1;
        if (id >= 0) sc = *(const float2*)(a.scales + ((int64_t)id * a.c.H + h) * 2);
    };
    scales();

    // this lane's column: row of the sequence and query head, and how many tokens it sees
    const int col = (ct * CW + cw) * 32 + ln;
    const bool real = col < cols;
    const int i = real ? col / a.G : 0, row = r0 + i, head = h * a.G + (real ? col - i * a.G : 0);
    int lim = L;
    if (real && a.causal) lim = min(max(kv - (r1 - r0) + i + 1, 0), L);
    bf16x8 q[KS][NS];
#pragma unroll
    for (int st = 0; st < KS; ++st) {
        float x[8] = {};
        if (real) {
            const T* p = (const T*)a.q + (int64_t)row * a.ldq + (int64_t)head * DH + (st >> 1) * 32 + g * 16 + (st & 1) * 8;
            if constexpr (NS == 1) {
                q[st][0] = __builtin_bit_cast(bf16x8, *(const uint4*)p);
                continue;
            } else {
                const float4 y = ((const float4*)p)[0], z = ((const float4*)p)[1];
                x[0] = y.x; x[1] = y.y; x[2] = y.z; x[3] = y.w;
                x[4] = z.x; x[5] = z.y; x[6] = z.z; x[7] = z.w;
            }
        }
        split8<NS>(x, q[st]);
    }
    const int lo = wave_min_int(lim), hi = wave_max_int(real ? lim : 0);

    f32x16 o[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) o[mt] = f32x16{};
    float m = -INFINITY, l = 0.f;

    struct Tile {
        uint4 k[MT], v[MT];
    };
    const int krow = 16 * (ln >> 2 & 1) + 4 * (ln >> 3) + (ln & 3);   // the token whose key this lane loads
    const int koff = krow * DH + g * 16, voff = ln * 32 + g * 16;
    // loads the tile of 32 tokens from key0 on (block 0's places where its block is not to be read)
    auto fetch = [&](int key0, Tile& x) {
        const int blk = max(__builtin_amdgcn_readlane(id, (key0 >> a.c.log2p) - bw), 0);
        const uint8_t* p = a.codes + cache_slab(a.c, DH, blk, h) + (int64_t)(key0 & (a.c.P - 1)) * DH;
        const uint8_t* pv = p + (int64_t)a.c.P * DH;
#pragma unroll
        for (int e = 0; e < MT; ++e) x.k[e] = *(const uint4*)(p + koff + e * 32);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) x.v[mt] = *(const uint4*)(pv + voff + mt * 1024);
    };

    auto work = [&](int tile0, Tile& x) {
        const int b = (tile0 >> a.c.log2p) - bw;
        if (__builtin_amdgcn_readlane(id, b) < 0) return;
        const float ks = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sc.x), b));
        const float vs = V_DOWN * __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sc.y), b));
        f32x16 sT = {};
#pragma unroll
        for (int st = 0; st < KS; ++st) {
            const bf16x8 kf = half8(x.k[st >> 1], st & 1, ks);
#pragma unroll
            for (int p = NS - 1; p >= 0; --p) sT = mfma32(kf, q[st][p], sT);
        }
        const int key0 = tile0 + 16 * g;
        if (tile0 + 32 > lo) {   // some column does not see the whole tile
#pragma unroll
            for (int r = 0; r < 16; ++r) sT[r] = key0 + r < lim ? sT[r] : -INFINITY;
            // NaN codes in places that not every column sees (or nobody: beyond the sequence's end)
            // would reach every column as 0 * NaN: they leave V, and the columns that see one get it back
            uint32_t any = 0;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const uint4& u = x.v[mt];
                any |= ((u.x & 0x7F7F7F7Fu) + 0x01010101u) | ((u.y & 0x7F7F7F7Fu) + 0x01010101u) |
                       ((u.z & 0x7F7F7F7Fu) + 0x01010101u) | ((u.w & 0x7F7F7F7Fu) + 0x01010101u);
            }
            if (__any((any & 0x80808080u) != 0)) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    uint32_t u[4] = {x.v[mt].x, x.v[mt].y, x.v[mt].z, x.v[mt].w}, w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t nan = (((u[e] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7;
                        u[e] &= ~(nan * 0xFFu);
                        w[e] = nan * 0x38u;   // 1.0
                    }
                    x.v[mt] = make_uint4(u[0], u[1], u[2], u[3]);
                    f32x16 cnt = {};
#pragma unroll
                    for (int st = 0; st < 2; ++st) {
                        float see[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) see[e] = key0 + 8 * st + e < lim ? 1.f : 0.f;
                        bf16x8 sb[1];
                        split8<1>(see, sb);
                        cnt = mfma32(cvt8(w[2 * st], w[2 * st + 1], 1.f), sb[0], cnt);
                    }
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[mt][r] += cnt[r] > 0.f ? NAN : 0.f;
                }
            }
        }
        float tm = sT[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) tm = fmaxf(tm, sT[r]);
        tm = max_halves(tm) * a.scale_log2;
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
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p[e] = __builtin_amdgcn_exp2f(fmaf(sT[8 * st + e], a.scale_log2, -ref));
                l += p[e];
            }
            bf16x8 pf[NS];
            split8<NS>(p, pf);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const bf16x8 vf = half8(x.v[mt], st, vs);
#pragma unroll
                for (int e = NS - 1; e >= 0; --e) o[mt] = mfma32(vf, pf[e], o[mt]);
            }
        }
    };

    // Tiles of a window of 64 blocks: this wavefront takes every KW-th.  Loads run NB - 1 tiles ahead and are
    // issued on every path (past the window's end its last tile again), so that the wait for a tile's
    // registers counts the younger loads and does not drain them.
    const int k1 = min(k0 + a.chunk, hi);
    for (int w0 = k0; w0 < k1;) {
        const int w1 = (int)min((int64_t)k1, (int64_t)(bw + 64) << a.c.log2p);
        const int last = w0 + ((w1 - w0 - 1) & ~31);
        const int t0 = w0 + 32 * kw;
        if (t0 <= last) {
            Tile tile[NB];
#pragma unroll
            for (int b = 0; b < NB - 1; ++b) fetch(min(t0 + 32 * KW * b, last), tile[b]);
            for (int t = t0; t <= last; t += 32 * KW * NB) {
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const int tb = t + 32 * KW * b;
                    fetch(min(tb + 32 * KW * (NB - 1), last), tile[(b + NB - 1) % NB]);
                    if (tb <= last) work(tb, tile[b]);
                }
            }
        }
        w0 = w1;
        if (w0 < k1) {
            bw = w0 >> a.c.log2p;
            id = -1;
            if (bw + lane < a.ld_table) id = a.table[(int64_t)s * a.ld_table + bw + lane];
            scales();
        }
    }
    l += __shfl_xor(l, 32, 64);

    // four consecutive features of a column, normalised into out or, of a cut sequence, as they are
    auto put = [&](int rw, int hd, int d, float4 v, float sum) {
        if (whole) {
            store4<T>((T*)a.out + (int64_t)rw * a.ldo + (int64_t)hd * DH + d, scaled(v, sum == 0.f ? 0.f : V_UP / sum));
        } else {
            *(float4*)(a.part + (((int64_t)rw * a.Hq + hd) * a.nsplit + piece) * DH + d) = v;
        }
    };
    auto put_ml = [&](int rw, int hd, float mx, float sum) {
        float* ml = a.part + (int64_t)a.T * a.Hq * a.nsplit * DH;
        *(float2*)(ml + (((int64_t)rw * a.Hq + hd) * a.nsplit + piece) * 2) = make_float2(mx, sum);
    };
    if constexpr (KW == 1) {
        if (!real) return;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                put(row, head, mt * 32 + 2 * r + 4 * g, make_float4(o[mt][r], o[mt][r + 1], o[mt][r + 2], o[mt][r + 3]), l);
        if (!whole && g == 0) put_ml(row, head, m, l);
    } else {
        // The KW results of a column tile meet in LDS: all features at once where the columns are few, else 32
        // at a time.
        constexpr int NT = 64 * KW * CW, LDC = 36, LDA = DH + 4;   // floats per column, 16-byte rows on different banks
        constexpr int FEW = CW == 1 ? 32 * LDC / LDA : 0;
        __shared__ __attribute__((aligned(16))) float so[KW * CW][32 * LDC];
        __shared__ float sml[KW * CW][32][2];
        if (g == 0) {
            sml[wave][ln][0] = m;
            sml[wave][ln][1] = l;
        }
        auto join = [&](int c, int cl, int ld, int dl, int d) {   // column cl of tile c, four features from d on
            const int cc = (ct * CW + c) * 32 + cl;
            if (cc >= cols) return;
            float mx = -INFINITY, sum = 0.f;
#pragma unroll
            for (int k = 0; k < KW; ++k) mx = fmaxf(mx, sml[c * KW + k][cl][0]);
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < KW; ++k) {
                const float mk = sml[c * KW + k][cl][0], f = mk == mx ? 1.f : __builtin_amdgcn_exp2f(mk - mx);
                const float4 y = *(const float4*)&so[c * KW + k][cl * ld + dl];
                sum += sml[c * KW + k][cl][1] * f;
                v.x += y.x * f; v.y += y.y * f; v.z += y.z * f; v.w += y.w * f;
            }
            const int j = cc / a.G, rw = r0 + j, hd = h * a.G + cc - j * a.G;
            put(rw, hd, d, v, sum);
            if (!whole && d == 0) put_ml(rw, hd, mx, sum);
        };
        const int here = min(cols - ct * WC, WC);
        if (here <= FEW) {
            if (real) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int r = 0; r < 16; r += 4)
                        *(float4*)&so[wave][ln * LDA + mt * 32 + 2 * r + 4 * g] =
                            make_float4(o[mt][r], o[mt][r + 1], o[mt][r + 2], o[mt][r + 3]);
            }
            __syncthreads();
            for (int e = threadIdx.x; e < here * (DH / 4); e += NT) join(0, e / (DH / 4), LDA, e % (DH / 4) * 4, e % (DH / 4) * 4);
            return;
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            if (mt) __syncthreads();
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *(float4*)&so[wave][ln * LDC + 2 * r + 4 * g] = make_float4(o[mt][r], o[mt][r + 1], o[mt][r + 2], o[mt][r + 3]);
            __syncthreads();
            for (int e = threadIdx.x; e < 256 * CW; e += NT) join(e >> 8, e >> 3 & 31, LDC, (e & 7) * 4, mt * 32 + (e & 7) * 4);
        }
    }
}

// Adds the pieces of cut sequences: one wavefront per (row of a sequence, query head).  Each lane holds one
// piece's maximum and sum (at most 64 pieces); DH / 4 lanes then hold four features each of one piece, 256 / DH
// pieces side by side.
template <typename T, int DH>
__global__ __launch_bounds__(256) void cache_attn_join_kernel(CacheAttnArgs a) {
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int64_t per = (int64_t)a.max_new * a.Hq;
    const int s = (int)(item / per), rem = (int)(item - s * per), i = rem / a.Hq, head = rem - i * a.Hq;
    if (s >= a.S) return;
    const int most = (int)min((int64_t)a.max_kv, (int64_t)a.ld_table * a.c.P);
    const int L = min(max(a.kv_len[s], 0), most), np = (L + a.chunk - 1) / a.chunk;
    const int r0 = min(max(a.row_start[s], 0), a.T), r1 = min(max(a.row_start[s + 1], r0), a.T);
    if (np < 2 || i >= r1 - r0) return;
    const int64_t at = ((int64_t)(r0 + i) * a.Hq + head) * a.nsplit;
    const float* part = a.part + at * DH;
    const float2* ml = (const float2*)(a.part + (int64_t)a.T * a.Hq * a.nsplit * DH) + at;
    constexpr int FL = DH / 4, PP = 64 / FL;
    const int f4 = lane % FL, pg = lane / FL;
    const float2 x = lane < np ? ml[lane] : make_float2(-INFINITY, 0.f);
    const float mx = wave_max(x.x), f = x.x == mx ? 1.f : __builtin_amdgcn_exp2f(x.x - mx);
    const float sum = wave_sum(x.y * f);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int p = pg; p < np; p += PP) {
        const float mp = ml[p].x, w = mp == mx ? 1.f : __builtin_amdgcn_exp2f(mp - mx);
        const float4 y = *(const float4*)(part + (int64_t)p * DH + f4 * 4);
        v.x += w * y.x; v.y += w * y.y; v.z += w * y.z; v.w += w * y.w;
    }
#pragma unroll
    for (int d = FL; d < 64; d <<= 1) {
        v.x += __shfl_xor(v.x, d, 64);
        v.y += __shfl_xor(v.y, d, 64);
        v.z += __shfl_xor(v.z, d, 64);
        v.w += __shfl_xor(v.w, d, 64);
    }
    if (pg == 0)
        store4<T>((T*)a.out + (int64_t)(r0 + i) * a.ldo + (int64_t)head * DH + f4 * 4, scaled(v, sum == 0.f ? 0.f : V_UP / sum));
}

// Shapes of a workgroup: wavefronts that share a column tile, column tiles side by side.
struct AttnShape {
    int kw, cw;
};
static constexpr AttnShape SHAPES[] = {{8, 1}, {4, 1}, {2, 2}, {1, 4}};

// Wavefronts per column tile: as many as leave some six wavefronts per SIMD in all (three of the larger ones of
// head dimension 128), since a tile's chain of loads, products and exponentials wants others beside it; but where the
// column tiles alone give every CU work, at least six tiles of tokens each (the first loads and the meeting in
// LDS cost about as much as two).  Measured, us, with 8 | 4 | 2 | 1: causal prompts of 4 x 2048 rows, 12 heads, over
// 4096 tokens - | 109 | 100 | 105; 2048 column tiles of head dimension 128 over 1500 tokens - | 72 | 65 | 61; 768 tiles
// (64 x 16 rows, 12 heads, 4096 tokens) 56 | 56 | 59 | -; 768 tiles over 1024 tokens 21 | 18 | 19 | -; 320 tiles
// (2 x 300 rows, 16 heads, 900 tokens) 13 | 10 | 12 | 20; 192 tiles (8 x 40 rows, 12 heads, 4096 tokens)
// 18 | 20 | 22 | 33.
// Pieces: cutting a sequence costs the partial results' way through memory and a second launch (768 tiles:
// 56 us whole, 73 in two), so it is done only while the workgroups are fewer than half the CUs, for pieces of 1024
// tokens and more (1 row, 8 heads, 32768 tokens: 20 us in 16 pieces, 27 in 8; 12 heads, 1001 tokens: 7.1 us whole,
// 8.2 in four).
CacheAttnPlan cache_attn_plan(int32_t S, int32_t T, int32_t Hkv, int32_t Hq, int dh, int32_t max_new, int32_t max_kv) {
    CacheAttnPlan p;
    const int64_t cols = (int64_t)max_new * (Hq / Hkv), per = std::max<int64_t>(1, (int64_t)S * Hkv);
    const int64_t tiles = std::max<int64_t>(1, per * ceil_div(cols, 32));
    int64_t waves = (dh > 64 ? 3200 : 6400) / tiles;
    if (tiles > 256) waves = std::min(waves, ceil_div(max_kv, 32) / 6);
    p.shape = waves >= 8 ? 0 : waves >= 4 ? 1 : waves >= 2 ? 2 : 3;
    const AttnShape sh = SHAPES[p.shape];
    p.threads = 64 * sh.kw * sh.cw;
    p.tiles = ceil_div(cols, 32 * sh.cw);
    const int64_t wgs = per * p.tiles;
    int64_t chunk = ceil_div(max_kv, 32) * 32;
    if (wgs < 128) chunk = std::min(chunk, std::max<int64_t>(1024, ceil_div(max_kv, ceil_div(256, wgs))));
    chunk = std::max<int64_t>(ceil_div(chunk, 32) * 32, ceil_div(ceil_div(max_kv, 64), 32) * 32);   // at most 64 pieces
    p.chunk = (int)chunk;
    p.nsplit = (int)ceil_div(max_kv, p.chunk);
    p.ws = p.nsplit == 1 ? 0 : ((size_t)T * Hq * p.nsplit * (dh + 2) * sizeof(float) + 255) & ~(size_t)255;
    return p;
}

template <typename T, int DH, int I>
static void launch_shape(const CacheAttnArgs& a, dim3 grid, hipStream_t s) {
    constexpr AttnShape h = SHAPES[I];
    launch_k((cache_attn_kernel<T, DH, h.kw, h.cw, 2>), grid, dim3(64 * h.kw * h.cw), 0, s, a);
}

template <typename T, int DH>
static void launch_cache_attn_t(const CacheAttnArgs& a, const CacheAttnPlan& p, hipStream_t s) {
    const int64_t groups = (int64_t)a.S * a.c.H * a.nsplit;
    const dim3 grid((unsigned)(ceil_div(groups, 8) * 8 * p.tiles));
    {
        ProfScope ps(KC_CACHE_ATTN, s);
        switch (p.shape) {
            case 0: launch_shape<T, DH, 0>(a, grid, s); break;
            case 1: launch_shape<T, DH, 1>(a, grid, s); break;
            case 2: launch_shape<T, DH, 2>(a, grid, s); break;
            default: launch_shape<T, DH, 3>(a, grid, s); break;
        }
    }
    if (a.nsplit > 1) {
        ProfScope ps(KC_CACHE_ATTN, s);
        launch_k((cache_attn_join_kernel<T, DH>), dim3((unsigned)ceil_div((int64_t)a.S * a.max_new * a.Hq, 4)), dim3(256), 0, s, a);
    }
}

dd_status launch_cache_attn(int dtype, const CacheAttnArgs& a, const CacheAttnPlan& p, hipStream_t s) {
    switch (a.dh) {
#define X(d)                                                          \
    case d:                                                           \
        if (dtype == DD_BF16) launch_cache_attn_t<bf16_t, d>(a, p, s); \
        else launch_cache_attn_t<float, d>(a, p, s);                  \
        break;
        X(32) X(64) X(128)
#undef X
    }
    return launch_status("cache_attention");
}

}  // namespace dd
