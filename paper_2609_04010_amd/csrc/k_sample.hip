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

constexpr int TAB = 256;     // 2^(-j / TAB)
constexpr int LIST = 64;     // classes of a bin that are ordered one by one

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

// w 2^frac, rounded.  With t = turn (top - l) = n + f, |f| <= 1/2: w = 2^-(n / TAB) 2^(-f / TAB), the first factor from the
// table and an exponent, the second from the first five terms of its series (the next is below 4e-17).
DD_DEV uint64_t weight(const RowScale& s, const double* tab, float l) {
    const double t = fmin(s.turn * ((double)s.top - (double)l), 64.0 * TAB);
    const double n = rint(t), x = (n - t) * (0.69314718055994530942 / TAB);
    const int k = (int)n;
    double e = fma(x, 1.0 / 24.0, 1.0 / 6.0);
    e = fma(x, e, 0.5);
    e = fma(x, e, 1.0);
    e = fma(x, e, 1.0);
    e = ldexp(e * tab[k & (TAB - 1)], s.frac - (k / TAB));
    return (uint64_t)__double_as_longlong(e + 0x1p52) - 0x4330000000000000ull;
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
    for (int j = tid; j < TAB; j += NT) sm.tab[j] = exp2(-(double)j / TAB);
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

}  // namespace

template <typename T, bool DRAW>
static void launch_sample_t(const SampleArgs& a, hipStream_t s) {
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
