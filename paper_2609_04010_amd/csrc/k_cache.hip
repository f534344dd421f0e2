// The cache of a serving pass: block tables and row maps from request lengths, and new keys and values
// rounded into the 8-bit cache.
#include <algorithm>

#include "cache.h"

namespace dd {

// Wavefront sum of whole numbers (the lane moves of wave_sum_dpp).
template <int CTRL, int ROWS> DD_DEV int dpp_add_int(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false); }
DD_DEV int wave_sum_int(int v) {
    v = dpp_add_int<0xB1, 0xF>(v);
    v = dpp_add_int<0x4E, 0xF>(v);
    v = dpp_add_int<0x141, 0xF>(v);
    v = dpp_add_int<0x140, 0xF>(v);
    v = dpp_add_int<0x142, 0xA>(v);
    v = dpp_add_int<0x143, 0xC>(v);
    return __builtin_amdgcn_readlane(v, 63);
}

// ---------------------------------------------------------------- block tables and row maps
//
// With fin_s = [n_new_s = -1], total_s = fin_s ? 0 : len_s + n_new_s:
//   rel_s = fin_s ? held_s : 0,  need_s = fin_s ? 0 : max(0, ceil(total_s / P) - held_s)
// everything is an exclusive prefix sum of n_new, need and rel over the sequences.  One workgroup of
// 1024 threads walks the sequences 1024 at a time: once for the totals (whether the pass fits, before
// anything is written), once for the blocks given back (only if there are any), once for rows and
// blocks taken.  Inside such a piece the items (blocks, rows) are spread over the threads, which find
// their sequence by bisection of the prefix sums in LDS.  Bound by latency: a chain of two or three loads, a few
// scans and the stores, 6.0 us for 16 sequences of one token, 14.1 us (with the rows' own launch) for 1024
// sequences of 16 drafted tokens, some prompts and some ends, 65536 rows.
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
        const int32_t before = wave_sum_int(lane < w ? sm.wsum[k][lane & (PT / 64 - 1)] : 0);
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
    auto load = [&](int s, int32_t& len, int32_t& held, int32_t (&x)[3], bool& fin) -> bool {
        len = a.seq_len[s];
        held = a.held[s];
        const int32_t n = a.n_new[s];
        const int64_t total = (int64_t)len + n;
        x[0] = x[1] = x[2] = 0;   // rows, blocks lacked, blocks given back
        fin = n == -1;
        if (n < -1 || held < 0 || held > a.ld_table || len < 0 || len > (int64_t)held * a.c.P) return false;
        if (fin) {
            x[2] = held;
            return true;
        }
        if (total > min((int64_t)a.ld_table * a.c.P, (int64_t)INT32_MAX)) return false;   // (a table may reach past 32-bit positions)
        x[0] = n;
        x[1] = max(0, (int32_t)((total + P1) >> lp) - held);
        return true;
    };

    // the first piece's numbers stay in registers: usually there is no other
    int32_t len0 = 0, held0 = 0, x0[3] = {0, 0, 0};
    bool fin0 = false, bad = tid < a.S && !load(tid, len0, held0, x0, fin0);
    if (tid == 0) {
        sm.tot[0] = sm.tot[1] = sm.tot[2] = 0;
        sm.bad = n_free < 0 || n_free > a.c.n_blocks;
    }
    __syncthreads();
    {
        long long t[3] = {x0[0], x0[1], x0[2]};
        for (int s = tid + PT; s < a.S; s += PT) {
            int32_t len, held, x[3];
            bool fin;
            bad |= !load(s, len, held, x, fin);
#pragma unroll
            for (int k = 0; k < 3; ++k) t[k] += x[k];
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            if (a.S <= PT) {   // sums of 64 halves fit 32 bits
                t[k] = ((long long)wave_sum_int(x0[k] >> 16) << 16) + wave_sum_int(x0[k] & 0xFFFF);
            } else {
#pragma unroll
                for (int o = 32; o > 0; o >>= 1) t[k] += __shfl_xor(t[k], o, 64);
            }
            if ((tid & 63) == 0 && t[k]) atomicAdd((unsigned long long*)&sm.tot[k], (unsigned long long)t[k]);
        }
        if (bad) sm.bad = 1;
    }
    __syncthreads();
    // a piece's numbers: of the first piece from the registers
    auto reload = [&](int s0, int32_t& len, int32_t& held, int32_t (&x)[3]) -> bool {
        len = held = x[0] = x[1] = x[2] = 0;
        bool fin = false;
        if (s0 == 0) {
            len = len0; held = held0; fin = fin0;
            x[0] = x0[0]; x[1] = x0[1]; x[2] = x0[2];
        } else if (s0 + tid < a.S) {
            load(s0 + tid, len, held, x, fin);
        }
        return fin;
    };
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
            int32_t len, held, x[3];
            reload(s0, len, held, x);
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
        int32_t len, held, x[3];
        const bool fin = reload(s0, len, held, x);
        sm.len[tid] = len;
        sm.held[tid] = held;
        if (a.S <= PT && rels > 0) __syncthreads();   // the sums of the blocks given back stand
        else plan_scan(sm, x, tid);
        if (s < a.S) {
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

// rows up to which one launch does all: 4096 rows 8.3 us against 9.1 in two, 8192 rows 11.8 against 10.0
constexpr int PLAN_ROWS = 4096;

dd_status launch_cache_plan(const PlanArgs& a, hipStream_t s) {
    const bool rows = a.T <= PLAN_ROWS;
    {
        ProfScope ps(KC_CACHE_PLAN, s);
        if (rows) launch_k(cache_plan_kernel<true>, dim3(1), dim3(PT), 0, s, a);
        else launch_k(cache_plan_kernel<false>, dim3(1), dim3(PT), 0, s, a);
    }
    if (rows) return launch_status("cache_plan");
    ProfScope ps(KC_CACHE_PLAN, s);
    launch_k(cache_rows_kernel, dim3((unsigned)ceil_div(a.T, 256)), dim3(256), 0, s, a);
    return launch_status("cache_plan");
}

// ---------------------------------------------------------------- append
//
// A unit of work is one (block, head, keys or values) that a sequence's rows fall into: take the largest finite
// |x| of its rows (at most P dh numbers), fix the scale from its exponent and mantissa bits, write the codes.
// Sequence s touches ceil((o_s + n_s) / P) blocks, o_s the place of its first new token; a wavefront finds its
// unit by a prefix sum of those over the lanes, 64 sequences at a time, so the grid has about as many
// units as there are (T / P + 2 S at most) and hardly a workgroup without work.  (A workgroup that only finds that it
// has nothing to do still costs about a microsecond of its CU: with one per row, 256 x 16 rows took 107 us.)
//
// Slabs of 32 tokens stay in registers between the maximum and the codes, so the rows are read once; W
// wavefronts share a unit's slabs: one where sequences add few tokens (then the four wavefronts of a workgroup
// have units of their own and nothing waits at a barrier), four for prompts.
//
// Keys: a lane holds 8 features of a token (16-byte loads of bf16) and stores 8 codes.  Values: a lane
// holds 2 features of TPL tokens that are neighbours in the cache's [dh][32] slab and stores TPL codes at
// a time; a slab whose places are not all new is read, changed and written back in the same lanes.

// N neighbouring numbers of a row as they stand in memory, and one of them as fp32
template <typename T, int N> struct Raw {
    uint32_t w[N * sizeof(T) / 4];
    DD_DEV void load(const T* p) {
        constexpr int W = N * sizeof(T) / 4;
        if constexpr (W == 1) {
            w[0] = *(const uint32_t*)p;
        } else if constexpr (W == 2) {
            const uint2 u = *(const uint2*)p;
            w[0] = u.x; w[1] = u.y;
        } else {
#pragma unroll
            for (int i = 0; i < W; i += 4) {
                const uint4 u = *(const uint4*)((const uint32_t*)p + i);
                w[i] = u.x; w[i + 1] = u.y; w[i + 2] = u.z; w[i + 3] = u.w;
            }
        }
    }
    DD_DEV float operator[](int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        else return e & 1 ? bf16_hi(w[e / 2]) : bf16_lo(w[e / 2]);
    }
};

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

// the lowest n bytes (none for n <= 0, all for n >= 4)
DD_DEV uint32_t low_bytes(int n) { return n <= 0 ? 0u : 0xFFFFFFFFu >> (32 - 8 * min(n, 4)); }

// One unit: n rows from x on at places off .. off + n - 1 of the block whose codes (keys or values) start at
// `body` and whose scale is *scale, by W wavefronts of which this is number w.
template <typename T, int DH, bool VALUES, int W>
DD_DEV void append_unit(const T* x, int64_t ld, int n, int off, int P, uint8_t* body, float* scale, int w, uint32_t* red) {
    const int lane = threadIdx.x & 63;
    constexpr int LPT = VALUES ? DH / 2 : DH / 8;        // lanes per token
    constexpr int TG = 64 / LPT;                         // tokens side by side
    constexpr int TPL = 32 / TG;                         // tokens of a slab per lane
    constexpr int NF = VALUES ? 2 : 8;                   // features per lane
    const int f = lane % LPT * NF, tg = lane / LPT;
    // token of the slab: keys TG apart (a store covers whole rows), values neighbours
    auto tok = [&](int i) { return VALUES ? tg * TPL + i : i * TG + tg; };
    const int end = off + n, first = off >> 5, slabs = ((end + 31) >> 5) - first;   // the slabs with new places
    const float s_old = off > 0 ? *scale : 0.f;
    const uint32_t ldb = (uint32_t)ld * sizeof(T);   // (256 rows of at most 2^21 numbers: below 2^32)
    Raw<T, NF> v[2][TPL];
    uint32_t old[2][2][TPL / 4];   // values: the codes that stand where this lane will write
    // All loads of two slabs at once; places that are not new take a neighbouring row, which changes no maximum and
    // is not stored.
    auto load = [&](int j0) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int sl = j0 + w + W * j, t0 = (first + sl) * 32;
            if (sl >= slabs) continue;
#pragma unroll
            for (int i = 0; i < TPL; ++i) v[j][i].load((const T*)((const char*)x + (uint32_t)(min(max(t0 + tok(i), off), end - 1) - off) * ldb) + f);
            if (VALUES && (t0 < off || t0 + 32 > end)) {
#pragma unroll
                for (int e2 = 0; e2 < 2; ++e2) {
                    const uint32_t* p = (const uint32_t*)(body + (int64_t)t0 * DH + (f + e2) * 32 + tg * TPL);
                    if constexpr (TPL == 8) {
                        const uint2 u = *(const uint2*)p;
                        old[j][e2][0] = u.x; old[j][e2][1] = u.y;
                    } else {
#pragma unroll
                        for (int i = 0; i < TPL / 16; ++i) {
                            const uint4 u = ((const uint4*)p)[i];
                            old[j][e2][4 * i] = u.x; old[j][e2][4 * i + 1] = u.y;
                            old[j][e2][4 * i + 2] = u.z; old[j][e2][4 * i + 3] = u.w;
                        }
                    }
                }
            }
        }
    };
    uint32_t m = 0;
    for (int j0 = 0; j0 < slabs; j0 += 2 * W) {
        load(j0);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (j0 + w + W * j >= slabs) continue;
#pragma unroll
            for (int i = 0; i < TPL; ++i)
#pragma unroll
                for (int e = 0; e < NF; ++e) m = amax_bits(m, v[j][i][e]);
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
    if constexpr (W > 1) {
        if (lane == 0) red[w] = m;
        __syncthreads();   // (also: every wavefront has read *scale)
#pragma unroll
        for (int i = 0; i < W; ++i) m = max(m, red[i]);
    }
    int e = scale_exp(m);
    float again = 1.f;   // what the block's other codes are multiplied by
    if (off > 0) {
        const int eo = min(max((int)(__float_as_uint(s_old) >> 23 & 255u) - 127, CACHE_EMIN), CACHE_EMAX);
        if (e > eo) again = pow2i(max(eo - e, -126));
        e = max(e, eo);
    }
    if (w == 0 && lane == 0) *scale = pow2i(e);
    const float inv = pow2i(-e);
    auto encode = [&](int j0) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int sl = j0 + w + W * j, t0 = (first + sl) * 32;
            if (sl >= slabs) continue;
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
                if (again == 1.f && (a0 + TPL <= off || a0 >= end)) continue;
#pragma unroll
                for (int e2 = 0; e2 < 2; ++e2) {
                    uint32_t* p = (uint32_t*)(body + (int64_t)t0 * DH + (f + e2) * 32 + tg * TPL);
                    uint32_t c[TPL / 4];
#pragma unroll
                    for (int i = 0; i < TPL / 4; ++i) {
                        const uint32_t nw = enc_fp8x4(v[j][4 * i][e2] * inv, v[j][4 * i + 1][e2] * inv,
                                                      v[j][4 * i + 2][e2] * inv, v[j][4 * i + 3][e2] * inv);
                        if (whole) {
                            c[i] = nw;
                        } else {
                            const uint32_t od = again != 1.f ? rescale4(old[j][e2][i], again) : old[j][e2][i];
                            const uint32_t in = low_bytes(end - (a0 + 4 * i)) & ~low_bytes(off - (a0 + 4 * i));
                            c[i] = (nw & in) | (od & ~in);
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
    };
    if (slabs <= 2 * W) {
        encode(0);
    } else {
        for (int j0 = 0; j0 < slabs; j0 += 2 * W) {
            load(j0);
            encode(j0);
        }
    }
    if (again != 1.f)   // slabs without new places
        for (int sl = w; sl < P >> 5; sl += W)
            if (sl < first || sl >= first + slabs)
                for (int i = lane; i < 2 * DH; i += 64) {
                    uint4* p = (uint4*)(body + (int64_t)sl * 32 * DH) + i;
                    const uint4 c = *p;
                    *p = make_uint4(rescale4(c.x, again), rescale4(c.y, again), rescale4(c.z, again), rescale4(c.w, again));
                }
}

// The u-th touched block of the pass: its sequence and which of the sequence's touched blocks it is.  false: there
// are not so many.  256 sequences' loads at a time; only the 64 that u falls into are scanned.
DD_DEV bool append_find(const AppendArgs& a, int u, int lane, int& seq, int& j, int& off, int& r0, int& n) {
    for (int s0 = 0; s0 < a.S; s0 += 256) {
        int b[4], e[4], o[4], nb[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int s = min(s0 + 64 * c + lane, a.S - 1);
            b[c] = a.row_start[s];
            e[c] = a.row_start[s + 1];
            o[c] = a.kv_len[s];
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            b[c] = min(max(b[c], 0), a.T);
            e[c] = min(max(e[c], b[c]), a.T);
            o[c] = (o[c] - (e[c] - b[c])) & (a.c.P - 1);
            nb[c] = e[c] > b[c] && s0 + 64 * c + lane < a.S ? (o[c] + (e[c] - b[c]) + a.c.P - 1) >> a.c.log2p : 0;
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int total = wave_sum_int(nb[c]);
            if (u < total) {
                int inc = nb[c];
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const int up = __shfl_up(inc, d, 64);
                    if (lane >= d) inc += up;
                }
                const int at = __popcll(__ballot(inc <= u));   // the first lane whose sum passes u
                seq = s0 + 64 * c + at;
                j = u - (__builtin_amdgcn_readlane(inc, at) - __builtin_amdgcn_readlane(nb[c], at));
                off = __builtin_amdgcn_readlane(o[c], at);
                r0 = __builtin_amdgcn_readlane(b[c], at);
                n = __builtin_amdgcn_readlane(e[c], at) - r0;
                return true;
            }
            u -= total;
        }
    }
    return false;
}

template <typename T, int DH, int W>
__global__ __launch_bounds__(256) void cache_append_kernel(AppendArgs a) {
    __shared__ uint32_t red[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // head and kind run fastest: workgroups that run together read whole rows
    const int per = W == 4 ? 2 * a.c.H : (2 * a.c.H + 3) / 4, unit = blockIdx.x / per;
    const int hk = W == 4 ? blockIdx.x - unit * per : (blockIdx.x - unit * per) * 4 + wave;
    if (W == 1 && hk >= 2 * a.c.H) return;
    const int values = hk >= a.c.H, h = values ? hk - a.c.H : hk;
    int off, r, n, slot;
    bool bad;
    if (a.by_row) {
        // a unit per row: the first row of a block, or of its sequence, does the block
        r = unit;
        slot = a.slots[r];
        const int seq = a.row_seq[r];
        if (slot < 0 && seq < 0) return;   // padding
        bad = slot < 0 || slot >= a.c.n_blocks * a.c.P || seq < 0 || seq >= a.S;
        off = slot & (a.c.P - 1);
        n = 0;
        if (!bad) {
            if (off != 0 && a.row_start[seq] != r) return;
            n = min(a.row_start[seq + 1], a.T) - r;
            bad = n <= 0;
        }
    } else {
        int seq, j;
        if (!append_find(a, unit, lane, seq, j, off, r, n)) return;
        if (j > 0) {   // rows and places of the sequence's j-th touched block
            const int skip = (j << a.c.log2p) - off;
            r += skip;
            n -= skip;
            off = 0;
        }
        slot = a.slots[r];
        bad = slot < 0 || slot >= a.c.n_blocks * a.c.P || (slot & (a.c.P - 1)) != off || a.row_seq[r] != seq;
    }
    if (bad) {
        if (a.err && threadIdx.x == 0) atomicOr(a.err, DD_DEVERR_CACHE);
        return;
    }
    n = min(n, a.c.P - off);
    const int64_t block = slot >> a.c.log2p;
    uint8_t* body = a.codes + cache_slab(a.c, DH, block, h) + (values ? (int64_t)a.c.P * DH : 0);
    float* scale = a.scales + (block * a.c.H + h) * 2 + values;
    const T* x = (const T*)(values ? a.v : a.k) + (int64_t)r * a.ld + (int64_t)h * DH;
    const int w = W == 4 ? wave : 0;
    if (values) append_unit<T, DH, true, W>(x, a.ld, n, off, a.c.P, body, scale, w, red);
    else append_unit<T, DH, false, W>(x, a.ld, n, off, a.c.P, body, scale, w, red);
}

AppendGrid cache_append_grid(int32_t S, int32_t T, int32_t P, int32_t H) {
    AppendGrid g;
    // with at most two rows per sequence on average nearly every row is a unit of its own, and needs no search
    g.by_row = T <= 2 * (int64_t)S;
    const int64_t units = g.by_row ? T : std::min<int64_t>(T, T / P + 2 * (int64_t)S);
    // sequences that add 32 rows or more on average: four wavefronts per unit
    g.wide = T >= 32 * (int64_t)S;
    g.wgs = units * (g.wide ? 2 * H : (2 * H + 3) / 4);
    return g;
}

dd_status launch_cache_append(int dtype, const AppendArgs& args, hipStream_t s) {
    AppendArgs a = args;
    ProfScope ps(KC_CACHE_APPEND, s);
    const AppendGrid g = cache_append_grid(a.S, a.T, a.c.P, a.c.H);
    a.by_row = g.by_row;
    const dim3 grid((unsigned)g.wgs);
#define X(T, d)                                                                          \
    if (a.dh == d) {                                                                     \
        if (g.wide) launch_k((cache_append_kernel<T, d, 4>), grid, dim3(256), 0, s, a);    \
        else launch_k((cache_append_kernel<T, d, 1>), grid, dim3(256), 0, s, a);         \
        return launch_status("cache_append");                                            \
    }
    if (dtype == DD_BF16) { X(bf16_t, 32) X(bf16_t, 64) X(bf16_t, 128) }
    else { X(float, 32) X(float, 64) X(float, 128) }
#undef X
    set_error("cache_append: head_dim %d", a.dh);
    return DD_E_UNSUPPORTED;
}

}  // namespace dd
