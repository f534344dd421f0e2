// The cache of a serving pass: block tables and row maps from request lengths, and new keys and values
// rounded into the 8-bit cache.
#include <algorithm>

#include "cache.h"

namespace dd {

// ---------------------------------------------------------------- block tables and row maps
//
// With fin_s = [n_new_s = -1], total_s = fin_s ? 0 : len_s + n_new_s:
//   rel_s = fin_s ? held_s : 0,  need_s = fin_s ? 0 : max(0, ceil(total_s / P) - held_s)
// everything is an exclusive prefix sum of n_new, need and rel over the sequences.  One workgroup of
// 1024 threads walks the sequences 1024 at a time: once for the totals (whether the pass fits, before
// anything is written), once for the blocks given back (only if there are any), once for rows and
// blocks taken.  Inside such a piece the items (blocks, rows) are spread over the threads, which find
// their sequence by bisection of the prefix sums in LDS.  Bound by latency: a chain of two loads, a few
// scans and the stores.
constexpr int PT = 1024;           // threads, and sequences of a piece

struct PlanLds {
    int32_t rows[PT + 1], need[PT + 1], rel[PT + 1];   // exclusive prefix sums of the piece
    int32_t len[PT], held[PT];
    int32_t wsum[3][PT / 64];
    long long tot[3];
    int bad;
};

// piece-wide exclusive prefix sums of x (their total in .[PT] of each array)
DD_DEV void plan_scan(PlanLds& sm, int32_t (&x)[3], int tid) {
    const int lane = tid & 63, w = tid >> 6;
    int32_t inc[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        inc[k] = x[k];
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int32_t up = __shfl_up(inc[k], o, 64);
            if (lane >= o) inc[k] += up;
        }
        if (lane == 63) sm.wsum[k][w] = inc[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        int32_t before = 0;
        for (int i = 0; i < w; ++i) before += sm.wsum[k][i];
        int32_t* out = k == 0 ? sm.rows : k == 1 ? sm.need : sm.rel;
        out[tid] = before + inc[k] - x[k];
        if (tid == PT - 1) out[PT] = before + inc[k];
    }
    __syncthreads();
}

// last i with a[i] <= v, for a[0] <= v < a[PT]
DD_DEV int plan_find(const int32_t* a, int32_t v) {
    int lo = 0, hi = PT;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a[mid] <= v) lo = mid;
        else hi = mid;
    }
    return lo;
}

DD_DEV int32_t plan_slot(const PlanArgs& a, int32_t block, int32_t pos) {
    if (block >= 0 && block < a.c.n_blocks) return block * a.c.P + (pos & (a.c.P - 1));
    if (a.err) atomicOr(a.err, DD_DEVERR_CACHE);
    return -1;
}

// ROWS: the row maps are written here as well (else by cache_rows_kernel)
template <bool ROWS>
__global__ __launch_bounds__(PT) void cache_plan_kernel(PlanArgs a) {
    __shared__ PlanLds sm;
    const int tid = threadIdx.x, P1 = a.c.P - 1, lp = a.c.log2p;
    const int32_t n_free = *a.n_free;
    // a sequence's numbers; false where they are no plan's
    auto load = [&](int s, int32_t& len, int32_t& held, int32_t& add, int32_t& need, int32_t& rel) -> bool {
        len = a.seq_len[s];
        held = a.held[s];
        const int32_t n = a.n_new[s];
        const int64_t total = (int64_t)len + n;
        add = need = rel = 0;
        if (n < -1 || held < 0 || held > a.ld_table || len < 0 || len > (int64_t)held * a.c.P) return false;
        if (n == -1) {
            rel = held;
            return true;
        }
        if (total > (int64_t)a.ld_table * a.c.P) return false;
        add = n;
        need = max(0, (int32_t)((total + P1) >> lp) - held);
        return true;
    };

    if (tid == 0) {
        sm.tot[0] = sm.tot[1] = sm.tot[2] = 0;
        sm.bad = n_free < 0 || n_free > a.c.n_blocks;
    }
    __syncthreads();
    {
        long long t[3] = {0, 0, 0};
        bool bad = false;
        for (int s = tid; s < a.S; s += PT) {
            int32_t len, held, x[3];
            bad |= !load(s, len, held, x[0], x[1], x[2]);
#pragma unroll
            for (int k = 0; k < 3; ++k) t[k] += x[k];
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) {
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) t[k] += __shfl_xor(t[k], o, 64);
            if ((tid & 63) == 0 && t[k]) atomicAdd((unsigned long long*)&sm.tot[k], (unsigned long long)t[k]);
        }
        if (bad) sm.bad = 1;
    }
    __syncthreads();
    const long long rows = sm.tot[0], needs = sm.tot[1], rels = sm.tot[2];
    const bool ok = !sm.bad && rows <= a.T && n_free + rels <= a.c.n_blocks && needs <= n_free + rels;
    if (!ok) {
        if (tid == 0) {
            if (a.err) atomicOr(a.err, DD_DEVERR_CACHE);
            *a.n_free_out = n_free;
            a.row_start[a.S] = 0;
        }
        for (int s = tid; s < a.S; s += PT) {
            a.kv_len[s] = a.seq_len[s];
            a.held_out[s] = a.held[s];
            a.row_start[s] = 0;
        }
        if (ROWS)
            for (int r = tid; r < a.T; r += PT) a.row_seq[r] = a.row_pos[r] = a.slots[r] = -1;
        return;
    }
    const int32_t top = n_free + (int32_t)rels;   // the stack's height once the ended sequences' blocks are on it
    if (rels > 0) {
        int32_t base = n_free;
        for (int s0 = 0; s0 < a.S; s0 += PT) {
            const int s = s0 + tid;
            int32_t len = 0, held = 0, x[3] = {0, 0, 0};
            if (s < a.S) load(s, len, held, x[0], x[1], x[2]);
            plan_scan(sm, x, tid);
            const int32_t n = sm.rel[PT];
            for (int32_t i = tid; i < n; i += PT) {
                const int q = plan_find(sm.rel, i);
                const int32_t b = a.table[(int64_t)(s0 + q) * a.ld_table + (i - sm.rel[q])];
                a.free_blocks[base + i] = b;
                if ((b < 0 || b >= a.c.n_blocks) && a.err) atomicOr(a.err, DD_DEVERR_CACHE);
            }
            base += n;
            __syncthreads();
        }
    }
    int32_t row0 = 0, taken = 0;
    for (int s0 = 0; s0 < a.S; s0 += PT) {
        const int s = s0 + tid;
        int32_t len = 0, held = 0, x[3] = {0, 0, 0};
        if (s < a.S) load(s, len, held, x[0], x[1], x[2]);
        sm.len[tid] = len;
        sm.held[tid] = held;
        plan_scan(sm, x, tid);
        if (s < a.S) {
            const bool fin = a.n_new[s] == -1;
            a.row_start[s] = row0 + sm.rows[tid];
            a.kv_len[s] = fin ? 0 : len + x[0];
            a.held_out[s] = fin ? 0 : held + x[1];
        }
        const int32_t need = sm.need[PT], nrow = sm.rows[PT];
        for (int32_t i = tid; i < need; i += PT) {
            const int q = plan_find(sm.need, i);
            a.table[(int64_t)(s0 + q) * a.ld_table + sm.held[q] + (i - sm.need[q])] = a.free_blocks[top - 1 - (taken + i)];
        }
        if (ROWS) {
            __syncthreads();   // the table entries just written
            for (int32_t i = tid; i < nrow; i += PT) {
                const int q = plan_find(sm.rows, i);
                const int32_t pos = sm.len[q] + (i - sm.rows[q]);
                a.row_seq[row0 + i] = s0 + q;
                a.row_pos[row0 + i] = pos;
                a.slots[row0 + i] = plan_slot(a, a.table[(int64_t)(s0 + q) * a.ld_table + (pos >> lp)], pos);
            }
        }
        row0 += nrow;
        taken += need;
        __syncthreads();
    }
    if (tid == 0) {
        a.row_start[a.S] = row0;
        *a.n_free_out = top - taken;
    }
    if (ROWS)
        for (int r = row0 + tid; r < a.T; r += PT) a.row_seq[r] = a.row_pos[r] = a.slots[r] = -1;
}

// Row maps of many rows, one thread each, from the arrays that cache_plan_kernel wrote.
__global__ __launch_bounds__(256) void cache_rows_kernel(PlanArgs a) {
    const int r = blockIdx.x * 256 + threadIdx.x;
    if (r >= a.T) return;
    if (r >= a.row_start[a.S]) {
        a.row_seq[r] = a.row_pos[r] = a.slots[r] = -1;
        return;
    }
    int lo = 0, hi = a.S;   // row_start[lo] <= r < row_start[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.row_start[mid] <= r) lo = mid;
        else hi = mid;
    }
    const int32_t pos = a.kv_len[lo] - (a.row_start[lo + 1] - r);
    a.row_seq[r] = lo;
    a.row_pos[r] = pos;
    a.slots[r] = plan_slot(a, a.table[(int64_t)lo * a.ld_table + (pos >> a.c.log2p)], pos);
}

constexpr int PLAN_ROWS = 8192;   // rows up to which one launch does all

dd_status launch_cache_plan(const PlanArgs& a, hipStream_t s) {
    ProfScope ps(KC_CACHE_PLAN, s);
    if (a.T <= PLAN_ROWS) {
        launch_k(cache_plan_kernel<true>, dim3(1), dim3(PT), 0, s, a);
        return launch_status("cache_plan");
    }
    launch_k(cache_plan_kernel<false>, dim3(1), dim3(PT), 0, s, a);
    ProfScope pr(KC_CACHE_PLAN, s);
    launch_k(cache_rows_kernel, dim3((unsigned)ceil_div(a.T, 256)), dim3(256), 0, s, a);
    return launch_status("cache_plan");
}

// ---------------------------------------------------------------- append
//
// A unit of work is one (block, head, keys or values) that a sequence's rows fall into: the workgroup
// takes the largest finite |x| of its rows (at most P dh numbers), fixes the scale from its exponent and
// mantissa bits, and writes the codes.  The unit's first row (the "leader": the first place of a block,
// or the sequence's first row) stands for it; a workgroup looks for leaders among rows_per_wg rows and
// does their units in turn.  Each of its four wavefronts owns slabs of 32 tokens, held in registers
// between the maximum and the codes, so the rows are read once.
//
// Keys: a lane holds 8 features of a token (16-byte loads of bf16) and stores 8 codes.  Values: a lane
// holds 2 features of TPL tokens that are neighbours in the cache's [dh][32] slab and stores TPL codes at
// a time; a slab whose places are not all new is read, changed and written back in the same lanes.

template <typename T> DD_DEV void load8(const T* p, float (&x)[8]);
template <> DD_DEV void load8<bf16_t>(const bf16_t* p, float (&x)[8]) {
    const uint4 u = *(const uint4*)p;
    x[0] = bf16_lo(u.x); x[1] = bf16_hi(u.x); x[2] = bf16_lo(u.y); x[3] = bf16_hi(u.y);
    x[4] = bf16_lo(u.z); x[5] = bf16_hi(u.z); x[6] = bf16_lo(u.w); x[7] = bf16_hi(u.w);
}
template <> DD_DEV void load8<float>(const float* p, float (&x)[8]) {
    const float4 a = ((const float4*)p)[0], b = ((const float4*)p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
template <typename T> DD_DEV float2 load2(const T* p);
template <> DD_DEV float2 load2<bf16_t>(const bf16_t* p) {
    const uint32_t u = *(const uint32_t*)p;
    return make_float2(bf16_lo(u), bf16_hi(u));
}
template <> DD_DEV float2 load2<float>(const float* p) { return *(const float2*)p; }

// largest |x| over finite x, as bits (of non-negative floats, which order like their bits)
DD_DEV uint32_t amax_bits(uint32_t m, float x) {
    const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
    return b < 0x7F800000u ? max(m, b) : m;
}

// the smallest e with a <= 448 2^e = 1.75 2^(e + 8), clamped: a's own exponent less 8, one more where its
// mantissa is above 1.75 (subnormal a lies far below the clamp)
DD_DEV int scale_exp(uint32_t a) {
    const int e = (int)(a >> 23) - 127 - 8 + ((a & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return min(max(e, CACHE_EMIN), CACHE_EMAX);
}

// four codes, multiplied by f (a power of two <= 1) and rounded again
DD_DEV uint32_t rescale4(uint32_t c, float f) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
    return enc_fp8x4(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
}

// One unit: rows r .. r + n - 1 at places off .. off + n - 1 of the block whose codes (keys or values) start
// at `body` and whose scale is *scale.
template <typename T, int DH, bool VALUES>
DD_DEV void append_unit(const T* x, int64_t ld, int n, int off, int P, uint8_t* body, float* scale, uint32_t* red) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    constexpr int LPT = VALUES ? DH / 2 : DH / 8;        // lanes per token
    constexpr int TG = 64 / LPT;                         // tokens side by side
    constexpr int TPL = 32 / TG;                         // tokens of a slab per lane
    constexpr int NF = VALUES ? 2 : 8;                   // features per lane
    const int f = lane % LPT * NF, tg = lane / LPT;
    // token of the slab: keys TG apart (a store covers whole rows), values neighbours
    auto tok = [&](int i) { return VALUES ? tg * TPL + i : i * TG + tg; };
    const int end = off + n;
    float v[2][TPL][NF] = {};   // P <= 256: at most two slabs per wavefront
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int t0 = (w + 4 * j) * 32;
        if (t0 >= end || t0 + 32 <= off) continue;
#pragma unroll
        for (int i = 0; i < TPL; ++i) {
            const int t = t0 + tok(i);
            if (t >= off && t < end) {
                const T* p = x + (int64_t)(t - off) * ld + f;
                if constexpr (VALUES) {
                    const float2 y = load2<T>(p);
                    v[j][i][0] = y.x;
                    v[j][i][1] = y.y;
                } else {
                    load8<T>(p, v[j][i]);
                }
            }
#pragma unroll
            for (int e = 0; e < NF; ++e) m = amax_bits(m, v[j][i][e]);
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
    __syncthreads();   // the last unit's readers are done with red and with *scale
    if (lane == 0) red[w] = m;
    const float s_old = off > 0 ? *scale : 0.f;
    __syncthreads();
    m = max(max(red[0], red[1]), max(red[2], red[3]));
    int e = scale_exp(m);
    float again = 1.f;   // what the block's other codes are multiplied by
    if (off > 0) {
        const int eo = min(max((int)(__float_as_uint(s_old) >> 23 & 255u) - 127, CACHE_EMIN), CACHE_EMAX);
        if (e > eo) again = pow2i(max(eo - e, -126));
        e = max(e, eo);
    }
    if (threadIdx.x == 0) *scale = pow2i(e);
    const float inv = pow2i(-e);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int t0 = (w + 4 * j) * 32;
        const bool fresh = t0 < end && t0 + 32 > off;    // has new places
        if (t0 >= P || (!fresh && again == 1.f)) continue;
        if constexpr (!VALUES) {
#pragma unroll
            for (int i = 0; i < TPL; ++i) {
                const int t = t0 + tok(i);
                uint2* p = (uint2*)(body + (int64_t)t * DH + f);
                if (t >= off && t < end) {
                    const auto& y = v[j][i];
                    *p = make_uint2(enc_fp8x4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv),
                                    enc_fp8x4(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv));
                } else if (again != 1.f) {
                    const uint2 c = *p;
                    *p = make_uint2(rescale4(c.x, again), rescale4(c.y, again));
                }
            }
        } else {
            const int a0 = t0 + tg * TPL;                // this lane's first token
            const bool whole = a0 >= off && a0 + TPL <= end;
#pragma unroll
            for (int e2 = 0; e2 < 2; ++e2) {
                uint32_t* p = (uint32_t*)(body + (int64_t)t0 * DH + (f + e2) * 32 + tg * TPL);
                uint32_t c[TPL / 4];
                if (!whole) {
                    if constexpr (TPL == 8) {
                        const uint2 u = *(const uint2*)p;
                        c[0] = u.x; c[1] = u.y;
                    } else {
#pragma unroll
                        for (int i = 0; i < TPL / 16; ++i) {
                            const uint4 u = ((const uint4*)p)[i];
                            c[4 * i] = u.x; c[4 * i + 1] = u.y; c[4 * i + 2] = u.z; c[4 * i + 3] = u.w;
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < TPL / 4; ++i) {
                    const uint32_t nw = enc_fp8x4(v[j][4 * i][e2] * inv, v[j][4 * i + 1][e2] * inv,
                                                  v[j][4 * i + 2][e2] * inv, v[j][4 * i + 3][e2] * inv);
                    if (whole) {
                        c[i] = nw;
                    } else {
                        const uint32_t od = again != 1.f ? rescale4(c[i], again) : c[i];
                        uint32_t y = 0;
#pragma unroll
                        for (int b = 0; b < 4; ++b) {
                            const int t = a0 + 4 * i + b;
                            y |= (t >= off && t < end ? nw : od) & (0xFFu << (8 * b));
                        }
                        c[i] = y;
                    }
                }
                if constexpr (TPL == 8) {
                    *(uint2*)p = make_uint2(c[0], c[1]);
                } else {
#pragma unroll
                    for (int i = 0; i < TPL / 16; ++i)
                        ((uint4*)p)[i] = make_uint4(c[4 * i], c[4 * i + 1], c[4 * i + 2], c[4 * i + 3]);
                }
            }
        }
    }
}

template <typename T, int DH>
__global__ __launch_bounds__(256) void cache_append_kernel(AppendArgs a) {
    __shared__ uint32_t red[4];
    const int lane = threadIdx.x & 63;
    const int h = blockIdx.y >> 1, values = blockIdx.y & 1;
    const int r0 = blockIdx.x * a.rows_per_wg;
    // lane i looks at row r0 + i: its slot, and how many rows of its block it leads (0: none)
    int slot = -1, n = 0;
    if (lane < a.rows_per_wg && r0 + lane < a.T) {
        const int r = r0 + lane;
        slot = a.slots[r];
        const int s = a.row_seq[r];
        if (slot >= 0 && s >= 0 && s < a.S && slot < a.c.n_blocks * a.c.P) {
            const int off = slot & (a.c.P - 1);
            if (off == 0 || r == a.row_start[s]) n = min(min(a.row_start[s + 1], a.T) - r, a.c.P - off);
        } else if ((slot >= 0 || s >= 0) && a.err && blockIdx.y == 0 && threadIdx.x < 64) {
            atomicOr(a.err, DD_DEVERR_CACHE);
        }
    }
    uint64_t todo = __ballot(n > 0);
    while (todo) {
        const int i = __ffsll((unsigned long long)todo) - 1;
        todo &= todo - 1;
        const int sl = __builtin_amdgcn_readlane(slot, i), cnt = __builtin_amdgcn_readlane(n, i);
        const int64_t block = sl >> a.c.log2p;
        uint8_t* body = a.codes + cache_slab(a.c, DH, block, h) + (values ? (int64_t)a.c.P * DH : 0);
        float* scale = a.scales + (block * a.c.H + h) * 2 + values;
        const T* x = (const T*)(values ? a.v : a.k) + (int64_t)(r0 + i) * a.ld + (int64_t)h * DH;
        if (values) append_unit<T, DH, true>(x, a.ld, cnt, sl & (a.c.P - 1), a.c.P, body, scale, red);
        else append_unit<T, DH, false>(x, a.ld, cnt, sl & (a.c.P - 1), a.c.P, body, scale, red);
    }
}

dd_status launch_cache_append(int dtype, const AppendArgs& args, hipStream_t s) {
    AppendArgs a = args;
    // rows per workgroup: enough workgroups to fill the CUs twice over with units of few rows, no more
    // than 32 rows (the smallest block) so that prompts spread over all units
    const int64_t units = (int64_t)a.T * 2 * a.c.H;
    a.rows_per_wg = (int)std::min<int64_t>(32, std::max<int64_t>(1, units / 4096));
    ProfScope ps(KC_CACHE_APPEND, s);
    const dim3 grid((unsigned)ceil_div(a.T, a.rows_per_wg), 2 * a.c.H);
#define X(T, d)                                                                    \
    if (a.dh == d) {                                                               \
        launch_k((cache_append_kernel<T, d>), grid, dim3(256), 0, s, a);           \
        return launch_status("cache_append");                                      \
    }
    if (dtype == DD_BF16) { X(bf16_t, 32) X(bf16_t, 64) X(bf16_t, 128) }
    else { X(float, 32) X(float, 64) X(float, 128) }
#undef X
    set_error("cache_append: head_dim %d", a.dh);
    return DD_E_UNSUPPORTED;
}

}  // namespace dd
