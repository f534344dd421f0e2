// A token per row of logits, or the row with the classes that stay, under temperature, min-p, top-k and top-p.
//
// Classes in order: falling logit l, the lowest index first among equal ones; w = exp((l - max) / temperature).  What
// stays is a beginning of that order (min-p cuts it at a value, top-k at a count, top-p at a sum of weights), and the draw is
// the first class at which the running sum exceeds u times the sum of what stays: every step but min-p asks for
// the first class at which a running sum (of ones, or of weights) reaches a bound.  That is answered without sorting:
// a histogram of counts and weights over NB bins of equal width in l, its prefix sums, the bin where the bound lies, and the
// classes of that bin one by one (a bin of more than 64 is cut again by its numbers' bits and indices).
//
// Sums of weights are whole numbers, multiples of 2^-46 (the exponential is taken in 64 bits and rounded once), so that neither the
// order of the atomics nor the cut into bins shows, and no border moves by more than 2^-47 per class.
#include <float.h>
#include <math.h>

#include <algorithm>

#include "elem.h"
#include "kernels.h"
#include "rng.h"

namespace dd {

namespace {

// smaller first: the order of classes by value (-0 is 0)
DD_DEV uint32_t value_key(float l) {
    const uint32_t u = __float_as_uint(l + 0.f);
    return ~(u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u));
}
DD_DEV float key_value(uint32_t k) {
    const uint32_t u = ~k;
    return __uint_as_float(u ^ ((u >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
// the place in the whole order
DD_DEV uint64_t place(float l, int v) { return ((uint64_t)value_key(l) << 32) | (uint32_t)v; }

constexpr int TAB = 64;      // 2^(-j / TAB)
constexpr int LIST = 64;     // classes of a bin that are ordered one by one
constexpr int EQUALS = 256;  // equal numbers that are

template <int NT>
struct SampleLds {
    static constexpr int NB = 2 * NT, NW = NT / 64;
    double tab[TAB];
    uint64_t w1[NB], w2[NB];    // weights of the bins, then their inclusive prefix sums; of the row, of a bin that is cut again
    uint32_t c1[NB], c2[NB];    // counts, likewise
    uint64_t list[LIST];
    uint64_t lo[NW], hi[NW];
    float mx[NW], mn[NW];
    uint64_t wsum[NW];
    uint32_t csum[NW];
    int bad[NW];
    // what a search found
    uint64_t base_w, in_w, at;
    uint32_t base_c, in_c;
    int bin, listed;
};

// what a row's weights and bins are made of
struct RowScale {
    float top, least, per;   // largest logit; smallest that min-p leaves; bins per unit of l
    double turn;             // TAB log2(e) / temperature
    int frac;                // weights are multiples of 2^-frac
    bool weigh;              // sums of weights are needed
};

// 2^(-j / TAB), from its series (25 terms, each factor below ln 2)
struct PowerTable {
    double v[TAB];
    constexpr PowerTable() : v() {
        for (int j = 0; j < TAB; ++j) {
            const double x = -0.69314718055994530942 * j / TAB;
            double e = 1.0;
            for (int n = 25; n > 0; --n) e = 1.0 + e * x / n;
            v[j] = e;
        }
    }
};
__constant__ PowerTable power_table = PowerTable();

// w 2^frac, rounded.  With t = turn (top - l) = n + f, |f| <= 1/2: w = 2^-(n / TAB) 2^(-f / TAB), the first factor from the
// table and an exponent, the second from the first six terms of its series (the next is below 4e-17).
DD_DEV uint64_t weight(const RowScale& s, const double* tab, float l) {
    const double t = fmin(s.turn * ((double)s.top - (double)l), 64.0 * TAB);
    const double n = rint(t), x = (n - t) * (0.69314718055994530942 / TAB);
    const int k = (int)n;
    double e = fma(x, 1.0 / 120.0, 1.0 / 24.0);
    e = fma(x, e, 1.0 / 6.0);
    e = fma(x, e, 0.5);
    e = fma(x, e, 1.0);
    e = fma(x, e, 1.0);
    e = ldexp(e * tab[k & (TAB - 1)], s.frac - (k / TAB));
    return (uint64_t)__double_as_longlong(e + 0x1p52) - 0x4330000000000000ull;
}

// l / t, rounded to nearest, from y = 1 / t rounded to nearest: a quotient within two steps, then twice corrected by what
// it leaves.  For |l| in [2^-100, 2^90] and t in [2^-30, 2^30] (below, within a step).
DD_DEV float quotient(float l, float t, float y) {
    float q = l * y;
    q = fmaf(fmaf(-q, t, l), y, q);
    return fmaf(fmaf(-q, t, l), y, q);
}
DD_DEV bool quotient_fits(float t, float a, float b) {
    return t >= 0x1p-30f && t <= 0x1p30f && fabsf(a) < 0x1p90f && fabsf(b) < 0x1p90f;
}

DD_DEV int bin_of(const RowScale& s, float l, int last) { return (int)fminf((s.top - l) * s.per, (float)last); }

// inclusive prefix sums of c and w over the bins, in place
template <int NT>
DD_DEV void scan_bins(SampleLds<NT>& sm, uint32_t* c, uint64_t* w, bool weigh) {
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    uint32_t c0 = c[2 * tid], c1 = c0 + c[2 * tid + 1], cs = c1;
    uint64_t w0 = weigh ? w[2 * tid] : 0, w1 = w0 + (weigh ? w[2 * tid + 1] : 0), ws = w1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t cu = __shfl_up(cs, o, 64);
        const uint64_t wu = __shfl_up(ws, o, 64);
        if (lane >= o) {
            cs += cu;
            ws += wu;
        }
    }
    if (lane == 63) {
        sm.csum[wv] = cs;
        sm.wsum[wv] = ws;
    }
    __syncthreads();
    uint32_t cb = cs - c1;
    uint64_t wb = ws - w1;
    for (int i = 0; i < wv; ++i) {
        cb += sm.csum[i];
        wb += sm.wsum[i];
    }
    c[2 * tid] = cb + c0;
    c[2 * tid + 1] = cb + c1;
    w[2 * tid] = wb + w0;
    w[2 * tid + 1] = wb + w1;
    __syncthreads();
}

// the bin in which the running count (COUNT) or weight reaches t, t >= 1 and no more than all bins together hold
template <int NT>
DD_DEV void find_bin(SampleLds<NT>& sm, const uint32_t* c, const uint64_t* w, bool count, uint64_t t) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int b = 2 * threadIdx.x + k;
        const uint32_t ce = b ? c[b - 1] : 0;
        const uint64_t we = b ? w[b - 1] : 0;
        if (count ? (ce < t && t <= c[b]) : (we < t && t <= w[b])) {
            sm.bin = b;
            sm.base_c = ce;
            sm.base_w = we;
            sm.in_c = c[b] - ce;
        }
    }
    __syncthreads();
}

// T: logits; NT: threads; RES: 16-byte chunks of a row that a thread keeps in registers (0: read again for each pass);
// DRAW: a token per draw (else: the row with what stays)
template <typename T, int NT, int RES, bool DRAW>
__global__ __launch_bounds__(NT) void sample_kernel(SampleArgs a) {
    using L = SampleLds<NT>;
    constexpr int E = Elem<T>::E, NB = L::NB, NW = L::NW;
    __shared__ L sm;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int chunks = RES > 0 ? RES : (a.V + NT * E - 1) / (NT * E);
    if (tid < TAB) sm.tab[tid] = power_table.v[tid];
    for (int i = blockIdx.x; i < a.n; i += gridDim.x) {
        int r = i;
        if (DRAW && a.row_ids) {
            r = a.row_ids[i];
            if (r < 0 || r >= a.rows) {
                if (r != -1 && tid == 0 && a.err) atomicOr(a.err, DD_DEVERR_SAMPLING);
                continue;
            }
        }
        const T* row = (const T*)a.logits + (int64_t)r * a.ld;
        const int s = i / a.per;
        const float t = a.temperature ? a.temperature[s] : 1.f, p = a.top_p ? a.top_p[s] : 1.f, m = a.min_p ? a.min_p[s] : 0.f;
        const int k = a.top_k ? a.top_k[s] : 0;
        auto chunk = [&](int c) -> uint4 {
            const int v = (c * NT + tid) * E;
            if (v >= a.V) return Elem<T>::NEG_INF4;
            uint4 u = *(const uint4*)(row + v);
            if (v + E > a.V) Elem<T>::clip(u, a.V - v);
            return u;
        };
        uint4 reg[RES > 0 ? RES : 1];
        if constexpr (RES > 0) {
#pragma unroll
            for (int c = 0; c < RES; ++c) reg[c] = chunk(c);
        }
        auto each = [&](auto&& f) {   // f(logit, class) for this thread's classes
            if constexpr (RES > 0) {
#pragma unroll
                for (int c = 0; c < RES; ++c)
#pragma unroll
                    for (int e = 0; e < E; ++e) f(Elem<T>::get(reg[c], e), (c * NT + tid) * E + e);
            } else {
                for (int c = 0; c < chunks; ++c) {
                    const uint4 u = chunk(c);
#pragma unroll
                    for (int e = 0; e < E; ++e) f(Elem<T>::get(u, e), (c * NT + tid) * E + e);
                }
            }
        };

        // largest and smallest finite logit, and whether there is anything that allows no choice
        RowScale q;
        {
            float mx = -INFINITY, mn = INFINITY;
            bool nan = false;
            each([&](float l, int) {
                mx = fmaxf(mx, l);
                nan |= l != l;
                if (l > -INFINITY) mn = fminf(mn, l);
            });
            for (int o = 32; o > 0; o >>= 1) {
                mx = fmaxf(mx, __shfl_xor(mx, o, 64));
                mn = fminf(mn, __shfl_xor(mn, o, 64));
            }
            nan = __any(nan);
            __syncthreads();   // the last row's results
            if (lane == 0) {
                sm.mx[wv] = mx;
                sm.mn[wv] = mn;
                sm.bad[wv] = nan;
            }
            for (int b = tid; b < NB; b += NT) {
                sm.c1[b] = 0;
                sm.w1[b] = 0;
            }
            __syncthreads();
            for (int x = 0; x < NW; ++x) {
                mx = fmaxf(mx, sm.mx[x]);
                mn = fminf(mn, sm.mn[x]);
                nan |= sm.bad[x] != 0;
            }
            const bool settings = t >= 0.f && t < INFINITY && p >= 0.f && m >= 0.f && m <= 1.f;   // (false for NaN)
            if (nan || mx == INFINITY || mx == -INFINITY || !settings) {
                if (tid == 0) {
                    if (a.err) atomicOr(a.err, settings ? DD_DEVERR_LOGITS : DD_DEVERR_SAMPLING);
                    if (a.kept) a.kept[i] = 0;
                    if (DRAW) {
                        a.z[i] = 0;
                        if (a.logp) a.logp[i] = NAN;
                    }
                }
                if (!DRAW && a.out != a.logits) {
                    T* out = (T*)a.out + (int64_t)r * a.ld;
                    for (int v = tid; v < a.V; v += NT) out[v] = row[v];
                }
                continue;
            }
            q.top = mx;
            const float reach = fminf(mx - mn, 32.f * t);
            q.per = reach > 0.f ? fminf(NB / reach, 1e37f) : 0.f;
            q.turn = TAB * 1.4426950408889634 / (double)t;
            q.frac = a.frac;
            q.least = -FLT_MAX;
            if (m > 0.f && t > 0.f) {   // w >= m where l >= top + t log m
                const double b = (double)mx + (double)t * log((double)m);
                if (b > -FLT_MAX) {
                    q.least = (float)b;
                    if ((double)q.least < b) q.least = key_value(value_key(q.least) - 1);   // the next number above
                }
            }
        }
        uint64_t cut = ~0ull, kept_w = 0;   // the last place that stays, and the sums up to there
        uint32_t kept_c = 0;
        if (t == 0.f || k == 1) {
            if (tid == 0) sm.bin = INT_MAX;
            __syncthreads();
            int v = INT_MAX;
            each([&](float l, int c) { if (l == q.top) v = min(v, c); });
            for (int o = 32; o > 0; o >>= 1) v = min(v, __shfl_xor(v, o, 64));
            if (lane == 0) atomicMin(&sm.bin, v);
            __syncthreads();
            cut = place(q.top, sm.bin);
            kept_c = 1;
            if (DRAW) {
                if (tid == 0) {
                    a.z[i] = sm.bin;
                    if (a.logp) a.logp[i] = 0.f;
                    if (a.kept) a.kept[i] = 1;
                }
                continue;
            }
        } else if (DRAW || k > 0 || p < 1.f || a.kept) {
            q.weigh = DRAW || p < 1.f;
            each([&](float l, int) {
                if (l >= q.least) {
                    const int b = bin_of(q, l, NB - 1);
                    atomicAdd(&sm.c1[b], 1u);
                    if (q.weigh) atomicAdd((unsigned long long*)&sm.w1[b], (unsigned long long)weight(q, sm.tab, l));
                }
            });
            __syncthreads();
            scan_bins<NT>(sm, sm.c1, sm.w1, q.weigh);
            kept_c = sm.c1[NB - 1];
            kept_w = sm.w1[NB - 1];
            // the first class at which the running count or weight reaches bound: its place in sm.at, the sums with it in
            // sm.base_c and sm.base_w
            auto search = [&](bool count, uint64_t bound) {
                find_bin<NT>(sm, sm.c1, sm.w1, count, bound);
                const int b1 = sm.bin;
                uint32_t base_c = sm.base_c, n = sm.in_c;
                uint64_t base_w = sm.base_w, lo = 0, hi = ~0ull;
                auto mine = [&](float l, int v, uint64_t& c) {
                    if (!(l >= q.least) || bin_of(q, l, NB - 1) != b1) return false;
                    c = place(l, v);
                    return c >= lo && c <= hi;
                };
                while (n > LIST) {
                    uint64_t first = ~0ull, last = 0;
                    each([&](float l, int v) {
                        uint64_t c;
                        if (mine(l, v, c)) {
                            first = first < c ? first : c;
                            last = last > c ? last : c;
                        }
                    });
                    for (int o = 32; o > 0; o >>= 1) {
                        const uint64_t f = __shfl_xor(first, o, 64), g = __shfl_xor(last, o, 64);
                        first = first < f ? first : f;
                        last = last > g ? last : g;
                    }
                    if (lane == 0) {
                        sm.lo[wv] = first;
                        sm.hi[wv] = last;
                    }
                    for (int b = tid; b < NB; b += NT) {
                        sm.c2[b] = 0;
                        sm.w2[b] = 0;
                    }
                    __syncthreads();
                    for (int x = 0; x < NW; ++x) {
                        first = first < sm.lo[x] ? first : sm.lo[x];
                        last = last > sm.hi[x] ? last : sm.hi[x];
                    }
                    int shift = 0;
                    while (((last - first) >> shift) >= NB) ++shift;
                    each([&](float l, int v) {
                        uint64_t c;
                        if (mine(l, v, c)) {
                            const int b = (int)((c - first) >> shift);
                            atomicAdd(&sm.c2[b], 1u);
                            if (q.weigh) atomicAdd((unsigned long long*)&sm.w2[b], (unsigned long long)weight(q, sm.tab, l));
                        }
                    });
                    __syncthreads();
                    scan_bins<NT>(sm, sm.c2, sm.w2, q.weigh);
                    find_bin<NT>(sm, sm.c2, sm.w2, count, bound - (count ? (uint64_t)base_c : base_w));
                    base_c += sm.base_c;
                    base_w += sm.base_w;
                    n = sm.in_c;
                    lo = first + ((uint64_t)sm.bin << shift);
                    hi = lo + ((1ull << shift) - 1);
                    __syncthreads();
                }
                if (tid == 0) sm.listed = 0;
                __syncthreads();
                each([&](float l, int v) {
                    uint64_t c;
                    if (mine(l, v, c)) sm.list[atomicAdd(&sm.listed, 1)] = c;
                });
                __syncthreads();
                if (tid < 64) {
                    const uint64_t c = tid < (int)n ? sm.list[tid] : ~0ull;
                    const uint64_t w = tid < (int)n && q.weigh ? weight(q, sm.tab, key_value((uint32_t)(c >> 32))) : 0;
                    uint32_t cs = base_c;
                    uint64_t ws = base_w;
                    for (int j = 0; j < (int)n; ++j) {
                        const uint64_t cj = __shfl(c, j, 64), wj = __shfl(w, j, 64);
                        if (cj <= c) {
                            ++cs;
                            ws += wj;
                        }
                    }
                    if (tid < (int)n && (count ? cs == bound : (ws >= bound && ws - w < bound))) {
                        sm.at = c;
                        sm.base_c = cs;
                        sm.base_w = ws;
                    }
                }
                __syncthreads();
            };
            if (k > 0 && (uint32_t)k < kept_c) {
                search(true, (uint64_t)k);
                cut = sm.at;
                kept_c = sm.base_c;
                kept_w = sm.base_w;
                __syncthreads();
            }
            if (p < 1.f) {
                const uint64_t bound = (uint64_t)ceil((double)p * (double)kept_w);
                search(false, bound > 0 ? bound : 1);
                cut = sm.at;
                kept_c = sm.base_c;
                kept_w = sm.base_w;
                __syncthreads();
            }
            if (DRAW) {
                const uint32_t word = a.noise ? a.noise[i] : counter_word(a.seed, STREAM_TOKEN, a.step, a.row0 + (uint32_t)i, 0);
                const double u = ((double)word + 0.5) * 0x1p-32;
                search(false, (uint64_t)(u * (double)kept_w) + 1);
                if (tid == 0) {
                    const double x = ((double)key_value((uint32_t)(sm.at >> 32)) - (double)q.top) / (double)t;
                    a.z[i] = (int32_t)(uint32_t)sm.at;
                    if (a.logp) a.logp[i] = (float)(x - log(ldexp((double)kept_w, -q.frac)));
                    if (a.kept) a.kept[i] = (int32_t)kept_c;
                }
                continue;
            }
        }
        if constexpr (!DRAW) {
            if (a.kept && tid == 0) a.kept[i] = (int32_t)kept_c;
            T* out = (T*)a.out + (int64_t)r * a.ld;
            const float last = key_value((uint32_t)(cut >> 32));
            const int last_v = (int)(uint32_t)cut;
            const bool all = cut == ~0ull;
            const float largest = sizeof(T) == 2 ? 0x1.FEp127f : FLT_MAX;   // (quotients do not become infinite)
            auto edit = [&](float l, int v) {
                const bool stays = l >= q.least && (all || l > last || (l == last && v <= last_v));
                return stays ? (t == 0.f ? l : fminf(fmaxf(l / t, -largest), largest)) : -INFINITY;
            };
            auto store = [&](int c, const uint4& u) {
                const int v = (c * NT + tid) * E;
                if (v >= a.V) return;
                float x[E];
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] = edit(Elem<T>::get(u, e), v + e);
                if (v + E <= a.V) {
                    if constexpr (sizeof(T) == 2)
                        *(uint4*)(out + v) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
                    else
                        *(float4*)(out + v) = make_float4(x[0], x[1], x[2], x[3]);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        if (v + e >= a.V) continue;
                        if constexpr (sizeof(T) == 2) out[v + e] = f32_to_bf16(x[e]);
                        else out[v + e] = x[e];
                    }
                }
            };
            if constexpr (RES > 0) {
#pragma unroll
                for (int c = 0; c < RES; ++c) store(c, reg[c]);
            } else {
                for (int c = 0; c < chunks; ++c) store(c, chunk(c));
            }
        }
    }
}

// ---------------------------------------------------------------- bf16 rows
//
// A bf16 number's 16 bits, as a signed whole number that orders like it (k = +-magnitude), are a bin of their own: equal
// numbers are all that a bin holds, so a count gives its weight, the exponential is taken once per bin, and a bound
// inside a bin is a division away.  A window of keys stands in LDS: MAGS magnitudes of either sign below the largest that can matter (weights
// below e^-34 round to 0), with the numbers nearer to 0 in one bin between them, whose weights are summed one by one (few:
// the window spans 16 binades).  Where a bound falls among those, or among numbers below the window (top-k alone can ask for
// them), the next window is counted.  Two packed numbers are handled at a time.
typedef __attribute__((ext_vector_type(2))) short s16x2;
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;

constexpr int KMAX = 0x7F7F, KINF = 0x7F80;                      // keys of the largest number and of infinity

DD_DEV s16x2 keys_of(uint32_t w) {
    const s16x2 sign = __builtin_bit_cast(s16x2, w) >> (short)15;
    const uint32_t m = (w & 0x7FFF7FFFu) ^ __builtin_bit_cast(uint32_t, sign);
    return __builtin_bit_cast(s16x2, m) - sign;
}
DD_DEV float key_float(int k) { return __uint_as_float((uint32_t)(k < 0 ? 0x8000 - k : k) << 16); }

// a value that all lanes have alike, where the compiler knows it; lane x's value
DD_DEV int same(int v) { return __builtin_amdgcn_readfirstlane(v); }
DD_DEV uint32_t same(uint32_t v) { return (uint32_t)same((int)v); }
DD_DEV uint64_t same(uint64_t v) { return ((uint64_t)same((uint32_t)(v >> 32)) << 32) | same((uint32_t)v); }
DD_DEV uint32_t of_lane(uint32_t v, int x) { return (uint32_t)__builtin_amdgcn_readlane((int)v, x); }
DD_DEV uint64_t of_lane(uint64_t v, int x) { return ((uint64_t)of_lane((uint32_t)(v >> 32), x) << 32) | of_lane((uint32_t)v, x); }

// inclusive prefix sums over the lanes: shifts within rows of 16, then the last lanes of rows into those behind them
template <int CTRL, int ROWS> DD_DEV uint32_t moved(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, true);
}
template <int CTRL, int ROWS> DD_DEV void scan_step(uint32_t& c, uint64_t& w) {
    c += moved<CTRL, ROWS>(c);
    w += ((uint64_t)moved<CTRL, ROWS>((uint32_t)(w >> 32)) << 32) | moved<CTRL, ROWS>((uint32_t)w);
}
DD_DEV void wave_scan(uint32_t& c, uint64_t& w) {
    scan_step<0x111, 0xF>(c, w);
    scan_step<0x112, 0xF>(c, w);
    scan_step<0x114, 0xF>(c, w);
    scan_step<0x118, 0xF>(c, w);
    scan_step<0x142, 0xA>(c, w);
    scan_step<0x143, 0xC>(c, w);
}
DD_DEV uint32_t wave_scan(uint32_t c) {
    c += moved<0x111, 0xF>(c);
    c += moved<0x112, 0xF>(c);
    c += moved<0x114, 0xF>(c);
    c += moved<0x118, 0xF>(c);
    c += moved<0x142, 0xA>(c);
    c += moved<0x143, 0xC>(c);
    return c;
}

// The window that is counted: MAGS magnitudes up to `max`, of either sign, and the keys that count.  Bins: positive, near 0,
// negative, one to spare.
template <int MAGS>
struct Window {
    static constexpr int ZERO = MAGS, BINS = 2 * MAGS + 2;
    int max, lo, hi;
    DD_DEV int min() const { return max - MAGS + 1; }
    DD_DEV int key(int bin) const { return bin < ZERO ? max - bin : bin == ZERO ? 0 : -(bin - ZERO - 1 + min()); }
};

template <int NT, int CH>
struct KeyLds {
    static constexpr int NW = NT / 64;
    using Win = Window<NT < 512 ? 2047 : 4095>;      // (a wider one is cleared and summed longer: not for short rows)
    double tab[TAB];
    uint32_t hist[Win::BINS + 64];       // counts; numbers outside the window go behind them, lane by lane
    // bins in groups of 256: weights of four neighbours and those before them in their group; of a group.  Counts likewise
    static constexpr int GROUPS = Win::BINS / 256;
    uint64_t pw[Win::BINS / 4], tw[GROUPS];
    uint32_t pc[Win::BINS / 4], tc[GROUPS];
    int hi[NW], lo[NW], kth[NW];
    uint64_t zero_w;
    uint32_t zero_c, below;
    __attribute__((aligned(16))) int list[EQUALS];
    int listed;                      // classes of equal numbers, where they are few
    uint32_t cell[CH * NW];          // equal numbers per chunk and wavefront
    // what wavefront 0 decided: count this window (or, `ask`, the numbers below it), or the j-th of the numbers of key `last`
    Win next;
    int again, ask, last, pick, at;
    uint32_t j, n;
};

template <int NT, int CH, bool DRAW>
__global__ __launch_bounds__(NT, 4) void sample_keys_kernel(SampleArgs a) {
    using L = KeyLds<NT, CH>;
    using Win = typename L::Win;
    constexpr int NW = L::NW, MAGS = Win::ZERO, ZERO = Win::ZERO, KBINS = Win::BINS, GROUPS = L::GROUPS;
    __shared__ __attribute__((aligned(16))) L sm;
    const int tid = threadIdx.x, lane = tid & 63, wv = same(tid >> 6);
    const int i = blockIdx.x;
    int r = i;
    if (DRAW && a.row_ids) {
        r = a.row_ids[i];
        if (r < 0 || r >= a.rows) {
            if (r != -1 && tid == 0 && a.err) atomicOr(a.err, DD_DEVERR_SAMPLING);
            return;
        }
    }
    const bf16_t* row = (const bf16_t*)a.logits + (int64_t)r * a.ld;
    s16x2 key[CH * 4];
    {
        uint4 u[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int v = (c * NT + tid) * 8;
            u[c] = Elem<bf16_t>::NEG_INF4;
            if (v < a.V) u[c] = *(const uint4*)(row + v);
        }
        if (tid < TAB) sm.tab[tid] = power_table.v[tid];
        static_assert(NT >= EQUALS, "a thread for each");
        if (tid < EQUALS) sm.list[tid] = INT_MAX;
#pragma unroll
        for (int b = 0; b < KBINS / 4 / NT; ++b) ((uint4*)sm.hist)[b * NT + tid] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int v = (c * NT + tid) * 8;
            if (v < a.V && v + 8 > a.V) Elem<bf16_t>::clip(u[c], a.V - v);
            key[4 * c] = keys_of(u[c].x);
            key[4 * c + 1] = keys_of(u[c].y);
            key[4 * c + 2] = keys_of(u[c].z);
            key[4 * c + 3] = keys_of(u[c].w);
        }
    }
    const int set = i / a.per;
    const float t = a.temperature ? a.temperature[set] : 1.f, p = a.top_p ? a.top_p[set] : 1.f, m = a.min_p ? a.min_p[set] : 0.f;
    const int k = a.top_k ? a.top_k[set] : 0;
    // largest and smallest key (NaN stands beyond the infinities)
    int kx, kn, kmin = -KMAX;    // kmin: the smallest that counts
    {
        s16x2 x = key[0], n = key[0];
#pragma unroll
        for (int w = 1; w < CH * 4; ++w) {
            x = __builtin_elementwise_max(x, key[w]);
            n = __builtin_elementwise_min(n, key[w]);
        }
        kx = max((int)x[0], (int)x[1]);
        kn = min((int)n[0], (int)n[1]);
        // top-k: the ceil(k / NW)-th largest of a wavefront's lanes' largest numbers; as many numbers reach the smallest of
        // those of all wavefronts as k at least, and what is smaller need not be counted
        int kth = -KINF;
        if (k > 1 && k <= NT) {
            const int rank = (k + NW - 1) / NW;
            int lo = -KINF - 1, hi = KINF + 255;       // (above lo: rank lanes or more; above hi: fewer)
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (__popcll(__ballot(kx > mid)) >= rank) lo = mid;
                else hi = mid;
            }
            kth = hi;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            kx = max(kx, __shfl_xor(kx, o, 64));
            kn = min(kn, __shfl_xor(kn, o, 64));
        }
        if (lane == 0) {
            sm.hi[wv] = kx;
            sm.lo[wv] = kn;
            sm.kth[wv] = kth;
        }
        if (tid == 0) {
            sm.listed = 0;
            sm.zero_c = sm.below = 0;
            sm.zero_w = 0;
        }
        __syncthreads();
        kx = sm.hi[lane & (NW - 1)];
        kn = sm.lo[lane & (NW - 1)];
        kth = sm.kth[lane & (NW - 1)];
#pragma unroll
        for (int o = NW / 2; o > 0; o >>= 1) {
            kx = max(kx, __shfl_xor(kx, o, 64));
            kn = min(kn, __shfl_xor(kn, o, 64));
            kth = min(kth, __shfl_xor(kth, o, 64));
        }
        kx = same(kx);
        kn = same(kn);
        kmin = max(kmin, same(kth));
    }
    const bool settings = t >= 0.f && t < INFINITY && p >= 0.f && m >= 0.f && m <= 1.f;   // (false for NaN)
    if (kx >= KINF || kx <= -KINF || kn < -KINF || !settings) {
        if (tid == 0) {
            if (a.err) atomicOr(a.err, settings ? DD_DEVERR_LOGITS : DD_DEVERR_SAMPLING);
            if (a.kept) a.kept[i] = 0;
            if (DRAW) {
                a.z[i] = 0;
                if (a.logp) a.logp[i] = NAN;
            }
        }
        if (!DRAW && a.out != a.logits) {
            bf16_t* out = (bf16_t*)a.out + (int64_t)r * a.ld;
            for (int v = tid; v < a.V; v += NT) out[v] = row[v];
        }
        return;
    }
    const float top = key_float(kx);
    const RowScale q = {top, 0.f, 0.f, TAB * 1.4426950408889634 / (double)t, a.frac, DRAW || p < 1.f};
    const bool few = kmin > -KMAX;       // (top-k has said so: most numbers do not count)
    int mags;                    // the largest magnitude that can matter
    {
        float b = top - 34.f * t;
        if (kn > -KINF) b = fmaxf(b, key_float(kn));
        if (m > 0.f && t > 0.f) {          // w >= m where l >= top + t log m
            const double e = (double)top + (double)t * log((double)m);
            if (e > -FLT_MAX) {
                float f = (float)e;
                if ((double)f < e) f = key_value(value_key(f) - 1);    // the next number above
                const uint32_t u = __float_as_uint(f);
                kmin = max(kmin, same((int32_t)u < 0 ? -(int)((u & 0x7FFFFFFFu) >> 16) : (int)((u + 0xFFFFu) >> 16)));
            }
        }
        b = fmaxf(b, key_float(kmin));
        mags = min(KMAX, (int)((__float_as_uint(b) & 0x7FFFFFFFu) >> 16) + 1);
        mags = same(max(max(mags, kx < 0 ? -kx : kx), MAGS));
    }
    int last = kmin, pick = 0;           // key of the last that stays (or of the draw); whether the j-th of them is looked for
    uint32_t j = 1, n = INT_MAX, kept_c = 1;     // n: how many there are (or more)
    uint64_t kept_w = 0;
    if (t == 0.f || k == 1) {
        last = kx;
        pick = 1;
    } else if (!q.weigh && k <= 0) {
        if (a.kept) {                    // what min-p leaves
            uint32_t x = 0;
#pragma unroll
            for (int y = 0; y < CH * 4; ++y) x += (uint32_t)((int)key[y][0] >= kmin) + (uint32_t)((int)key[y][1] >= kmin);
            x = wave_scan(x);
            if (lane == 63) atomicAdd(&sm.below, x);
            __syncthreads();
            kept_c = sm.below;
        }
    } else {
        Win win = {mags, kmin, KMAX};
        // of wavefront 0: sums before the window; top-k, top-p and draw done; what is looked for
        uint32_t base_c = 0, main_c = 0;
        uint64_t base_w = 0, bound = 0;
        int step = 0;
        bool have = false, count = false, main = true;
        int below = -1;                  // numbers below the main window, once they are counted
        for (;;) {
            // (what a pass makes of the keys is not to be kept for the next: there are too many)
#pragma unroll
            for (int x = 0; x < CH * 4; ++x) asm volatile("" : "+v"(key[x]));
            {
                const u16x2 hi = (u16x2)(unsigned short)win.max, mid = (u16x2)(unsigned short)ZERO;
                const u16x2 sh = (u16x2)(unsigned short)(win.max + win.min() - (MAGS + 1)), out = (u16x2)(unsigned short)(KBINS + lane);
#pragma unroll
                for (int x = 0; x < CH * 4; ++x) {
                    if (few && !__any(max((int)key[x][0], (int)key[x][1]) >= kmin)) continue;
                    const u16x2 d = hi - __builtin_bit_cast(u16x2, key[x]);
                    u16x2 b = __builtin_elementwise_min(d, __builtin_elementwise_max(mid, __builtin_elementwise_sub_sat(d, sh)));
                    b = __builtin_elementwise_min(b, out);
                    atomicAdd(&sm.hist[b[0]], 1u);
                    atomicAdd(&sm.hist[b[1]], 1u);
                }
            }
            __syncthreads();
            const bool near = win.min() > 1 && same(sm.hist[ZERO]) != 0;       // (from magnitude 1 on, zeros are alone in their bin)
            if (near) {
#pragma unroll
                for (int x = 0; x < CH * 4; ++x) asm volatile("" : "+v"(key[x]));
                uint32_t zc = 0;
                uint64_t zw = 0;
                const int lo = max(win.lo, 1 - win.min()), hi = min(win.hi, win.min() - 1);
                const u16x2 from = (u16x2)(unsigned short)(short)lo;
#pragma unroll
                for (int half = 0; half < CH; half += 8) {
                    uint64_t some = 0;
#pragma unroll
                    for (int y = half; y < CH && y < half + 8; ++y) {
                        u16x2 x = __builtin_bit_cast(u16x2, key[4 * y]) - from;
#pragma unroll
                        for (int z = 1; z < 4; ++z) x = __builtin_elementwise_min(x, __builtin_bit_cast(u16x2, key[4 * y + z]) - from);
                        if (lo > hi || min(x[0], x[1]) > hi - lo) continue;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int f = key[4 * y + e / 2][e & 1];
                            some |= (uint64_t)(f >= lo && f <= hi) << (8 * (y - half) + e);
                        }
                    }
                    zc += __popcll(some);
                    if (q.weigh)
#pragma unroll 1
                        for (; some; some &= some - 1) {
                            const int x = __builtin_ctzll(some) + 8 * half;
                            zw += weight(q, sm.tab, bf16_to_f32(row[((x >> 3) * NT + tid) * 8 + (x & 7)]));
                        }
                }
                if (zc) {
                    atomicAdd(&sm.zero_c, zc);
                    atomicAdd((unsigned long long*)&sm.zero_w, (unsigned long long)zw);
                }
                __syncthreads();
            }
            // count and weight of a bin, and the weight of one of its numbers
            auto bin_sums = [&](int bin, uint32_t n, uint32_t& c, uint64_t& w) -> uint64_t {
                const int f = win.key(bin);
                c = f < win.lo || f > win.hi || bin == KBINS - 1 ? 0 : n;
                const uint64_t one = q.weigh ? weight(q, sm.tab, key_float(f)) : 0;
                w = c * one;
                if (near && bin == ZERO) {
                    c = sm.zero_c;
                    w = sm.zero_w;
                }
                return one;
            };
            // (every wavefront a group of each part of the bins: most numbers stand in few of them)
#pragma unroll 1
            for (int g = wv; g < GROUPS; g += NW) {
                const int b = (g * 64 + lane) * 4;
                const uint4 n = *(const uint4*)&sm.hist[b];
                if (!__any((n.x | n.y | n.z | n.w) != 0)) {
                    if (lane == 0) {
                        sm.tc[g] = 0;
                        sm.tw[g] = 0;
                    }
                    continue;
                }
                uint32_t c, c_sum = 0;
                uint64_t w, w_sum = 0;
                bin_sums(b, n.x, c, w);
                c_sum += c, w_sum += w;
                bin_sums(b + 1, n.y, c, w);
                c_sum += c, w_sum += w;
                bin_sums(b + 2, n.z, c, w);
                c_sum += c, w_sum += w;
                bin_sums(b + 3, n.w, c, w);
                c_sum += c, w_sum += w;
                wave_scan(c_sum, w_sum);
                sm.pc[g * 64 + lane] = c_sum;
                sm.pw[g * 64 + lane] = w_sum;
                if (lane == 63) {
                    sm.tc[g] = c_sum;
                    sm.tw[g] = w_sum;
                }
            }
            __syncthreads();
            if (wv == 0) {
                static_assert(GROUPS <= 64, "a group per lane");
                uint32_t ic = lane < GROUPS ? sm.tc[lane & (GROUPS - 1)] : 0;
                uint64_t iw = lane < GROUPS ? sm.tw[lane & (GROUPS - 1)] : 0;
                wave_scan(ic, iw);
                const uint32_t all_c = base_c + of_lane(ic, 63);
                const uint64_t all_w = base_w + of_lane(iw, 63);
                int again = 0, ask = 0;
                if (main && step == 0 && !have) {
                    main_c = all_c;
                    kept_c = all_c + (uint32_t)max(below, 0);
                    kept_w = all_w;
                }
                for (;;) {
                    if (!have) {                       // the main window is the one that stands
                        if (step == 0) {
                            const bool further = kn < -win.max && kmin < -win.max;      // numbers below the window
                            if (k > 0 && (uint32_t)k < kept_c) {
                                count = have = true;
                                bound = (uint32_t)k;
                            } else if (further && below < 0 && (k > 0 || (a.kept && p >= 1.f))) {
                                ask = 1;
                                break;
                            }
                            step = 1;
                            if (have && kept_c > main_c && (uint32_t)k > main_c) {      // it is below the window
                                base_c = main_c;
                                base_w = all_w;
                                main = false;
                                again = 1;
                                win.hi = -win.max - 1;
                                win.max = min(win.max + MAGS, KMAX);
                                break;
                            }
                        }
                        if (!have && step == 1) {
                            step = 2;
                            if (p < 1.f) {
                                bound = same((uint64_t)ceil((double)p * (double)kept_w));
                                bound = bound > 0 ? bound : 1;
                                count = false;
                                have = true;
                            }
                        }
                        if (!have) {
                            if (!DRAW) break;
                            step = 3;
                            const uint32_t word = a.noise ? a.noise[i] : counter_word(a.seed, STREAM_TOKEN, a.step, a.row0 + (uint32_t)i, 0);
                            bound = same((uint64_t)(((double)word + 0.5) * 0x1p-32 * (double)kept_w) + 1);
                            count = false;
                            have = true;
                        }
                    }
                    if (count && bound > all_c) {      // further down
                        base_c = all_c;
                        base_w = all_w;
                        again = 1;
                        win.hi = -win.max - 1;
                        win.max = min(win.max + MAGS, KMAX);
                        break;
                    }
                    // the group, four neighbours and bin where the running count or weight reaches the bound
                    auto reached = [&](uint32_t c, uint64_t w) { return count ? c >= bound : w >= bound; };
                    const int x = __builtin_ctzll(__ballot(reached(base_c + ic, base_w + iw)));
                    uint32_t before_c = base_c + (x ? of_lane(ic, x - 1) : 0);
                    uint64_t before_w = base_w + (x ? of_lane(iw, x - 1) : 0);
                    const uint32_t lc = sm.pc[x * 64 + lane];
                    const uint64_t lw = sm.pw[x * 64 + lane];
                    const int y = __builtin_ctzll(__ballot(reached(before_c + lc, before_w + lw)));
                    before_c += y ? of_lane(lc, y - 1) : 0;
                    before_w += y ? of_lane(lw, y - 1) : 0;
                    const int bin0 = (x * 64 + y) * 4;
                    uint32_t bc, sc;
                    uint64_t bw, sw;
                    const uint64_t b1 = bin_sums(bin0 + (lane & 3), sm.hist[bin0 + (lane & 3)], bc, bw);
                    sc = bc, sw = bw;
                    scan_step<0x111, 0xF>(sc, sw);     // (of lanes 0 to 3; the others are not looked at)
                    scan_step<0x112, 0xF>(sc, sw);
                    const int z = __builtin_ctzll(__ballot(reached(before_c + sc, before_w + sw)));
                    before_c += z ? of_lane(sc, z - 1) : 0;
                    before_w += z ? of_lane(sw, z - 1) : 0;
                    const uint32_t in_c = of_lane(bc, z);
                    if (bin0 + z == ZERO && win.min() > 1) {       // among the numbers nearer to 0
                        base_c = before_c;
                        base_w = before_w;
                        main = false;
                        again = 1;
                        win.lo = max(win.lo, 1 - win.min());
                        win.hi = min(win.hi, win.min() - 1);
                        win.max = max(win.min() - 1, MAGS);
                        break;
                    }
                    last = win.key(bin0 + z);
                    const uint64_t one = of_lane(b1, z);
                    if (count) {
                        j = (uint32_t)(bound - before_c);
                    } else {                           // the first j of them whose weights reach the bound
                        const uint64_t lack = bound - before_w;
                        j = same((uint32_t)((double)lack / (double)one));
                        while (j * one < lack) ++j;
                        while (j > 1 && (j - 1) * one >= lack) --j;
                    }
                    pick = j < in_c || step == 3;
                    n = in_c;
                    if (step == 3) break;
                    kept_c = before_c + j;
                    kept_w = before_w + j * one;
                    have = false;
                    if (!DRAW && (step == 2 || p >= 1.f)) break;
                    if (!main) {
                        main = true;
                        again = 1;
                        win = {mags, kmin, KMAX};
                        base_c = 0;
                        base_w = 0;
                        break;
                    }
                }
                if (lane == 0) {
                    sm.again = again;
                    sm.ask = ask;
                    sm.next = win;
                    sm.last = last;
                    sm.pick = pick;
                    sm.j = j;
                    sm.n = n;
                }
            }
            __syncthreads();
            if (same(sm.ask)) {
                // numbers below the window
                uint32_t x = 0;
#pragma unroll
                for (int y = 0; y < CH * 4; ++y)
#pragma unroll
                    for (int e = 0; e < 2; ++e) x += key[y][e] >= kmin && key[y][e] < -win.max;
                if (x) atomicAdd(&sm.below, x);
                __syncthreads();
                below = same((int)sm.below);
            } else if (!same(sm.again)) {
                break;
            }
            win.max = same(sm.next.max);
            win.lo = same(sm.next.lo);
            win.hi = same(sm.next.hi);
            __syncthreads();
#pragma unroll
            for (int b = 0; b < KBINS / 4 / NT; ++b) ((uint4*)sm.hist)[b * NT + tid] = make_uint4(0u, 0u, 0u, 0u);
            if (tid == 0) {
                sm.zero_c = 0;
                sm.zero_w = 0;
            }
            __syncthreads();
        }
        last = same(sm.last);
        pick = same(sm.pick);
        j = same(sm.j);
        n = same(sm.n);
    }
    // the j-th number equal to `last`, in the order of classes
    int last_v = INT_MAX;
    if (pick) {
        const u16x2 is = (u16x2)(unsigned short)(short)last;
        if (n <= EQUALS) {           // all of them, and those before each counted
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                u16x2 d = __builtin_bit_cast(u16x2, key[4 * c]) ^ is;
#pragma unroll
                for (int y = 1; y < 4; ++y) d = __builtin_elementwise_min(d, __builtin_bit_cast(u16x2, key[4 * c + y]) ^ is);
                if (d[0] != 0 && d[1] != 0) continue;
                uint32_t x = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) x |= (uint32_t)((int)key[4 * c + e / 2][e & 1] == last) << e;
                int to = atomicAdd(&sm.listed, __popc(x));
                for (; x; x &= x - 1) sm.list[to++] = (c * NT + tid) * 8 + __builtin_ctz(x);
            }
            __syncthreads();
            if (tid < (int)n) {
                const int v = sm.list[tid];
                uint32_t before = 0;
                for (int x = 0; x < (int)n; x += 16) {       // (behind them stands INT_MAX)
                    int4 y[4];
#pragma unroll
                    for (int z = 0; z < 4; ++z) y[z] = *(const int4*)&sm.list[x + 4 * z];
#pragma unroll
                    for (int z = 0; z < 4; ++z) before += (y[z].x < v) + (y[z].y < v) + (y[z].z < v) + (y[z].w < v);
                }
                if (before == j - 1) sm.at = v;
            }
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                u16x2 d = (u16x2)(unsigned short)0;        // how many are not equal
#pragma unroll
                for (int y = 0; y < 4; ++y) d += __builtin_elementwise_min(__builtin_bit_cast(u16x2, key[4 * c + y]) ^ is, (u16x2)(unsigned short)1);
                uint32_t x = 8 - d[0] - d[1];
                if (__ballot(x != 0)) x = wave_scan(x);
                if (lane == 63) sm.cell[c * NW + wv] = x;
            }
            __syncthreads();
            // the cell of the j-th: each lane sums PER neighbours
            constexpr int PER = (CH * NW + 63) / 64;
            uint32_t cells[PER], sum = 0;
#pragma unroll
            for (int x = 0; x < PER; ++x) {
                cells[x] = lane * PER + x < CH * NW ? sm.cell[lane * PER + x] : 0;
                sum += cells[x];
            }
            const uint32_t inc = wave_scan(sum);
            const int owner = __builtin_ctzll(__ballot(inc >= j));     // (j is at most their number)
            uint32_t before = of_lane(inc - sum, owner);
            int at = owner * PER;
#pragma unroll
            for (int x = 0; x < PER - 1; ++x) {
                const uint32_t y = of_lane(cells[x], owner);
                if (at == owner * PER + x && before + y < j) {
                    before += y;
                    ++at;
                }
            }
            if (at % NW == wv) {
                // (from memory again: registers have no numbers)
                const int v = (at / NW * NT + tid) * 8;
                const uint4 u = v < a.V ? *(const uint4*)(row + v) : Elem<bf16_t>::NEG_INF4;
                uint32_t x = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t w = e < 2 ? u.x : e < 4 ? u.y : e < 6 ? u.z : u.w;
                    x |= (uint32_t)(v + e < a.V && (int)keys_of(w)[e & 1] == last) << e;
                }
                const uint32_t mine = __popc(x), up = wave_scan(mine), want = j - before;
                if (up - mine < want && want <= up) {
                    for (uint32_t f = want - (up - mine); f > 1; --f) x &= x - 1;
                    sm.at = v + __builtin_ctz(x);
                }
            }
        }
        __syncthreads();
        last_v = same(sm.at);
    }
    if (tid == 0) {
        if (a.kept) a.kept[i] = (int32_t)kept_c;
        if (DRAW) {
            a.z[i] = last_v;
            if (a.logp) {
                const bool first = t == 0.f || k == 1;
                a.logp[i] = first ? 0.f : (float)(((double)key_float(last) - (double)top) / (double)t - log(ldexp((double)kept_w, -a.frac)));
            }
        }
    }
    if constexpr (!DRAW) {
        bf16_t* out = (bf16_t*)a.out + (int64_t)r * a.ld;
        constexpr float largest = 0x1.FEp127f;     // (quotients do not become infinite)
        const bool divide = t != 1.f && t != 0.f, fast = quotient_fits(t, top, key_float(last));
        const float rt = 1.f / t;
        uint32_t some = 0;                         // chunks in which something stays
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            s16x2 x = key[4 * c];
#pragma unroll
            for (int y = 1; y < 4; ++y) x = __builtin_elementwise_max(x, key[4 * c + y]);
            some |= (uint32_t)(max((int)x[0], (int)x[1]) >= last) << c;
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int v = (c * NT + tid) * 8;
            if (v >= a.V) continue;
            uint4 o = Elem<bf16_t>::NEG_INF4;
            if (some >> c & 1) {
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int g = key[4 * c + e / 2][e & 1];
                    float l = key_float(g);
                    if (divide) l = fast ? quotient(l, t, rt) : fminf(fmaxf(l / t, -largest), largest);
                    f[e] = g > last || (g == last && v + e <= last_v) ? l : -INFINITY;
                }
                o = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
            }
            if (v + 8 <= a.V) {
                *(uint4*)(out + v) = o;
            } else {
                const uint32_t w[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (v + e < a.V) out[v + e] = (bf16_t)(w[e / 2] >> (16 * (e & 1)));
            }
        }
    }
}

}  // namespace

template <bool DRAW>
static void launch_sample_keys(const SampleArgs& a, hipStream_t s) {
    auto go = [&](auto kernel, int threads) { launch_k(kernel, dim3((unsigned)a.n), dim3(threads), 0, s, a); };
    // A row's time is that of its phases one behind the other: with a CU for each row it ends sooner in 1024 threads; where
    // rows wait for CUs, two of 512 threads on a CU do less work each.
    const bool few = a.n <= num_cus();
    if (a.V <= 2048) go(sample_keys_kernel<256, 1, DRAW>, 256);
    else if (a.V <= 8192) go(sample_keys_kernel<256, 4, DRAW>, 256);
    else if (a.V <= 16384) go(sample_keys_kernel<512, 4, DRAW>, 512);
    else if (a.V <= 32768) go(sample_keys_kernel<512, 8, DRAW>, 512);
    else if (a.V <= 57344 && few) go(sample_keys_kernel<1024, 7, DRAW>, 1024);
    else if (a.V <= 53248) go(sample_keys_kernel<512, 13, DRAW>, 512);
    else if (a.V <= 65536) go(sample_keys_kernel<512, 16, DRAW>, 512);
    else go(sample_keys_kernel<1024, 16, DRAW>, 1024);
}

template <typename T, bool DRAW>
static void launch_sample_t(const SampleArgs& a, hipStream_t s) {
    if constexpr (sizeof(T) == 2) {
        if (a.V <= 131072 && grid_fits(a.n, 1024)) return launch_sample_keys<DRAW>(a, s);
    }
    const dim3 grid((unsigned)std::min<int64_t>(a.n, 2 * num_cus()));
    launch_k((sample_kernel<T, 1024, 0, DRAW>), grid, dim3(1024), 0, s, a);
}

dd_status launch_sample(const SampleArgs& args, int dtype, bool draw, hipStream_t s) {
    SampleArgs a = args;
    // V weights of at most 1 have to fit 62 bits
    int lg = 0;
    while ((1 << lg) < a.V) ++lg;
    a.frac = std::min(46, 62 - lg);
    ProfScope ps(draw ? KC_TOKEN_SAMPLE : KC_LOGITS_TRUNCATE, s);
    if (dtype == DD_BF16) draw ? launch_sample_t<bf16_t, true>(a, s) : launch_sample_t<bf16_t, false>(a, s);
    else draw ? launch_sample_t<float, true>(a, s) : launch_sample_t<float, false>(a, s);
    return launch_status(draw ? "token_sample" : "logits_truncate");
}

}  // namespace dd
