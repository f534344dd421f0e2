// A token per row of logits, or the row with the classes that stay, under temperature, min-p, top-k and top-p.
//
// Classes in order: falling logit l, the lowest index first among equal ones; w = exp((l - max) / temperature).  What
// stays is a beginning of that order (min-p cuts it at a value, top-k at a count, top-p at a sum of weights), and the draw is
// the first class at which the running sum exceeds u times the sum of what stays: every step but min-p asks for
// the first class at which a running sum (of ones, or of weights) reaches a bound.  That is answered without sorting: counts
// and weights of a histogram's bins, in falling order of l, their prefix sums, the bin where the bound lies, and the
// classes of that bin one by one.  bf16 rows of up to 131072 classes have a kernel of their own: their numbers are few.
//
// Sums of weights are whole numbers, multiples of 2^-46 (coarser where 2^16 classes of weight 1 would pass 62 bits; the
// exponential is taken in 64 bits and rounded once), so that neither the order of the atomics nor the cut into bins shows, and
// no border moves by more than half of that per class.
//
// A row is one workgroup's: its phases (largest number, histogram, sums, search) follow each other, so a call of few rows is
// bound by latency, and one of many by the instructions of the histogram and the search, not by reading the row.
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
constexpr int EQUALS = 256;  // equal numbers that are ordered one by one (more are counted)

// what a row's weights are made of
struct RowScale {
    float top, least;        // largest logit; smallest that counts
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

// ---------------------------------------------------------------- bf16 rows
//
// A bf16 number's 16 bits, as a signed whole number that orders like it (k = +-magnitude), are a bin of their own: equal
// numbers are all that a bin holds, so a count gives its weight, the exponential is taken once per bin, and a bound
// inside a bin is a division away.  A window of keys stands in LDS: MAGS magnitudes of either sign below the largest that can
// matter (weights below e^-34 round to 0), with the numbers nearer to 0 in one bin between them, whose weights are summed one by one (few:
// the window spans 16 binades, 32 in 512 threads and more).  Where a bound falls among those, or among numbers below the window (top-k
// alone can ask for them), the next window is counted.  Two packed numbers are handled at a time, and the row stays in registers; at
// their limit of 128, draws spill 2 registers with 8 chunks per thread, 5 with 13 and up to 19 with 16.
//
// Rows of 50257 classes under temperature, top-k and top-p: 8 in 16 to 19 us, 512 in 31 to 34 (of a row's 24 there, two on a CU: 7 for the
// loads, 3 for the largest, 7 for counting, 2.5 each for the sums and the search, 1.2 for the class); 4096 truncated in 175 (4.7 TB/s read and
// written; 284 with a division per number, all numbers counted, and rows written number by number).
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
    const RowScale q = {top, 0.f, TAB * 1.4426950408889634 / (double)t, a.frac, DRAW || p < 1.f};
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
                            const bool further = kn < -win.max && kmin < -win.max;      // numbers below the window, or -inf
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
                // numbers below the window.  (Where only -inf stands there, also behind the last class, the window is counted again
                // for nothing: 512 draws under temperature alone take 39.8 us with n_kept, and 26.7 without)
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
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int v = (c * NT + tid) * 8;
            if (v >= a.V) continue;
            uint4 o = Elem<bf16_t>::NEG_INF4;
            s16x2 x = key[4 * c];
#pragma unroll
            for (int y = 1; y < 4; ++y) x = __builtin_elementwise_max(x, key[4 * c + y]);
            if (max((int)x[0], (int)x[1]) >= last) {
                // keys above `under` stay; with equal ones up to last_v: whole chunks of them, or one by one
                const bool split = v <= last_v && last_v < v + 7;
                const s16x2 under = (s16x2)(short)(v > last_v ? last : last - 1);
                uint32_t w[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const s16x2 g = key[4 * c + y], sign = g >> (short)15;
                    // the number's bits, from its key
                    uint32_t l = __builtin_bit_cast(uint32_t, (s16x2)((g ^ sign) - sign)) | (__builtin_bit_cast(uint32_t, sign) & 0x80008000u);
                    if (divide) {
                        const float lo = bf16_lo(l), hi = bf16_hi(l);
                        l = fast ? pack_bf16x2(quotient(lo, t, rt), quotient(hi, t, rt))
                                 : pack_bf16x2(fminf(fmaxf(lo / t, -largest), largest), fminf(fmaxf(hi / t, -largest), largest));
                    }
                    const uint32_t stays = __builtin_bit_cast(uint32_t, (s16x2)(__builtin_elementwise_sub_sat(under, g) >> (short)15));
                    w[y] = (l & stays) | (0xFF80FF80u & ~stays);
                }
                if (split)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if ((int)key[4 * c + e / 2][e & 1] == last && v + e > last_v)
                            w[e / 2] = e & 1 ? (w[e / 2] & 0xFFFFu) | 0xFF800000u : (w[e / 2] & 0xFFFF0000u) | 0xFF80u;
                o = make_uint4(w[0], w[1], w[2], w[3]);
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

// ---------------------------------------------------------------- fp32 rows, and bf16 rows of very many classes
//
// Every pass reads the row again, from L2 after the first.  (With the row in registers, 52 of them, the compiler keeps
// the rest in scratch memory: 512 draws from 16 rows of 50257 took 81 us, and take 54 to 66 with the rows' values.)  Bins are steps of the exponential's
// table, so a number's bin falls out of its weight; numbers that weigh nothing share the last one.  A bin holds different numbers: those
// of the bin where a bound lies are listed with their weights, and each sums those before it; where they are too many for that, their
// places are cut into parts first, with three readings of the row number by number (512 draws of 50257 classes: 354 us at a temperature that
// puts all in one bin, 65 at 1).  Draws that follow each
// other from one row under the same settings share all but the last step.  A truncated row is
// written while its last bin is listed, unless that is in place: 333 rows of 32003 take 48 us, and 51 with a pass of its own.
template <int NT>
struct StreamLds {
    static constexpr int NW = NT / 64;
    static constexpr int LOG = NT >= 512 ? 0 : 2;              // steps of the table per bin: 2^LOG
    static constexpr int BINS = 4096 >> LOG, PARTS = NT;       // bins, and parts that one of them is cut into
    static constexpr int CANDS = NT / 2;                       // numbers of a bin and its edges that are ordered one by one
    double tab[TAB];
    // of the bins; numbers that do not count go behind them, lane by lane
    uint64_t w1[BINS + 64], w2[PARTS];
    uint32_t c1[BINS + 64], c2[PARTS];
    uint64_t place[CANDS], w[CANDS];
    float value[CANDS];
    int id[CANDS];
    uint64_t lo[NW], hi[NW], wsum[NW];
    uint32_t csum[NW];
    float mx[NW], kth[NW];
    uint32_t big[NW];
    uint64_t before_w, in_w, at;
    uint32_t before_c, in_c, count;
    int bin, listed;
};

// sums before this thread's share and in all, of shares c and w
template <int NT, typename L>
DD_DEV void block_scan(L& sm, uint32_t c, uint64_t w, uint32_t& c_at, uint64_t& w_at, uint32_t& c_all, uint64_t& w_all) {
    constexpr int NW = NT / 64;
    const int lane = threadIdx.x & 63, wv = same((int)threadIdx.x >> 6);
    uint32_t ci = c;
    uint64_t wi = w;
    wave_scan(ci, wi);
    if (lane == 63) {
        sm.csum[wv] = ci;
        sm.wsum[wv] = wi;
    }
    __syncthreads();
    uint32_t ct = lane < NW ? sm.csum[lane & (NW - 1)] : 0;
    uint64_t wt = lane < NW ? sm.wsum[lane & (NW - 1)] : 0;
    const uint32_t c0 = ct;
    const uint64_t w0 = wt;
    wave_scan(ct, wt);
    c_all = of_lane(ct, 63);
    w_all = of_lane(wt, 63);
    c_at = ci - c + of_lane(ct, wv) - of_lane(c0, wv);
    w_at = wi - w + of_lane(wt, wv) - of_lane(w0, wv);
}

template <typename T, int NT, bool DRAW>
__global__ __launch_bounds__(NT, 4) void sample_stream_kernel(SampleArgs a) {
    using L = StreamLds<NT>;
    constexpr int E = Elem<T>::E, NW = L::NW, BINS = L::BINS, PARTS = L::PARTS, CANDS = L::CANDS, PER = BINS / NT;
    __shared__ __attribute__((aligned(16))) L sm;
    const int tid = threadIdx.x, lane = tid & 63, wv = same(tid >> 6);
    const int chunks = (a.V + NT * E - 1) / (NT * E);
    if (tid < TAB) sm.tab[tid] = power_table.v[tid];
    // of the row whose sums stand in LDS
    int have_row = -1, have_set = -1, state = 0;      // state: 0 the first class alone, 1 no choice, 2 sums
    RowScale q = {};
    float t = 1.f;
    bool weigh = false, counted = false;
    uint64_t kept_w = 0, cut = ~0ull, w_at = 0, w_sum = 0;
    uint32_t kept_c = 0, c_at = 0, c_sum = 0;
    const int i0 = blockIdx.x * a.chunk, i1 = min(i0 + a.chunk, a.n);
    for (int i = i0; i < i1; ++i) {
        int r = i;
        if (DRAW && a.row_ids) {
            r = a.row_ids[i];
            if (r < 0 || r >= a.rows) {
                if (r != -1 && tid == 0 && a.err) atomicOr(a.err, DD_DEVERR_SAMPLING);
                continue;
            }
        }
        const int set = i / a.per;
        const T* row = (const T*)a.logits + (int64_t)r * a.ld;
        // f(numbers, class of the first) for each chunk; what stands behind the row is -inf
        auto each_chunk = [&](auto&& f) {
            constexpr int AHEAD = 4;       // chunks whose loads are under way together
            for (int c0 = 0; c0 < chunks; c0 += AHEAD) {
                const bool whole = (c0 + AHEAD) * NT * E <= a.V;
                uint4 u[AHEAD];
#pragma unroll
                for (int c = 0; c < AHEAD; ++c)      // (no branch between the loads; ld is a multiple of 8: in bounds)
                    u[c] = *(const uint4*)(row + min(((c0 + c) * NT + tid) * E, (a.V - 1) & ~(E - 1)));
#pragma unroll
                for (int c = 0; c < AHEAD; ++c) {
                    const int v = ((c0 + c) * NT + tid) * E;
                    if (c0 + c >= chunks) break;
                    if (!whole) {
                        if (v >= a.V) u[c] = Elem<T>::NEG_INF4;
                        else if (v + E > a.V) Elem<T>::clip(u[c], a.V - v);
                    }
                    float x[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] = Elem<T>::get(u[c], e);
                    f(x, v);
                }
            }
        };
        // bin and weight of a number: of t = turn (top - x) the nearest whole step, from the last bits of t + 1.5 2^52, and as in weight()
        auto weight_of = [&](float x, int& bin) -> uint64_t {
            const double u = fmin(((double)q.top - (double)x) * q.turn, (double)(64 * TAB - 1));
            const double m = u + 0x1.8p52, f = (m - 0x1.8p52) - u;
            const int n = (int)(uint32_t)__double_as_longlong(m);
            constexpr double s = 0.69314718055994530942 / TAB;
            double e = fma(f, s * s * s * s * s / 120.0, s * s * s * s / 24.0);
            e = fma(f, e, s * s * s / 6.0);
            e = fma(f, e, s * s / 2.0);
            e = fma(f, e, s);
            e = fma(f, e, 1.0);
            e = ldexp(e * sm.tab[n & (TAB - 1)], q.frac - n / TAB);
            bin = n >> L::LOG;
            return (uint64_t)__double_as_longlong(e + 0x1p52) - 0x4330000000000000ull;
        };
        static_assert(BINS << L::LOG == 64 * TAB, "bins end where weights do");
        uint64_t at = 0;
        int step = 2;                      // top-k, top-p, draw
        int k = 0;
        float p = 1.f;
        if (r != have_row || set != have_set) {
            have_row = r;
            have_set = set;
            t = a.temperature ? a.temperature[set] : 1.f;
            p = a.top_p ? a.top_p[set] : 1.f;
            const float m = a.min_p ? a.min_p[set] : 0.f;
            k = a.top_k ? a.top_k[set] : 0;
            float mx = -INFINITY, kth = -INFINITY;
            uint32_t big = 0;              // NaN stands above infinity
            each_chunk([&](const float (&x)[E], int) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    mx = fmaxf(mx, x[e]);
                    big = max(big, __float_as_uint(x[e]) & 0x7FFFFFFFu);
                }
            });
            if (k > 1 && k <= NT) {        // (as for bf16 rows)
                const int rank = (k + NW - 1) / NW;
                const uint32_t mine = ~value_key(mx);
                uint32_t found = 0;
                for (int b = 31; b >= 0; --b)
                    if (__popcll(__ballot(mine >= (found | 1u << b))) >= rank) found |= 1u << b;
                kth = key_value(~found);
            }
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) {
                mx = fmaxf(mx, __shfl_xor(mx, o, 64));
                big = max(big, (uint32_t)__shfl_xor((int)big, o, 64));
            }
            __syncthreads();               // the last row's sums
            if (lane == 0) {
                sm.mx[wv] = mx;
                sm.kth[wv] = kth;
                sm.big[wv] = big;
            }
            for (int b = tid; b < BINS / 2; b += NT) ((uint4*)sm.w1)[b] = make_uint4(0u, 0u, 0u, 0u);
            for (int b = tid; b < BINS / 4; b += NT) ((uint4*)sm.c1)[b] = make_uint4(0u, 0u, 0u, 0u);
            __syncthreads();
            mx = sm.mx[lane & (NW - 1)];
            kth = sm.kth[lane & (NW - 1)];
            big = sm.big[lane & (NW - 1)];
#pragma unroll
            for (int o = NW / 2; o > 0; o >>= 1) {
                mx = fmaxf(mx, __shfl_xor(mx, o, 64));
                kth = fminf(kth, __shfl_xor(kth, o, 64));
                big = max(big, (uint32_t)__shfl_xor((int)big, o, 64));
            }
            mx = __int_as_float(same(__float_as_int(mx)));
            kth = __int_as_float(same(__float_as_int(kth)));
            big = same(big);
            const bool settings = t >= 0.f && t < INFINITY && p >= 0.f && m >= 0.f && m <= 1.f;   // (false for NaN)
            if (big > 0x7F800000u || mx == INFINITY || mx == -INFINITY || !settings) {
                state = 1;
                if (tid == 0 && a.err) atomicOr(a.err, settings ? DD_DEVERR_LOGITS : DD_DEVERR_SAMPLING);
            } else {
                state = t == 0.f || k == 1 ? 0 : 2;
                q = {mx, fmaxf(kth, -FLT_MAX), TAB * 1.4426950408889634 / (double)t, a.frac, true};
                if (m > 0.f && t > 0.f) {  // w >= m where l >= top + t log m
                    const double b = (double)mx + (double)t * log((double)m);
                    if (b > -FLT_MAX) {
                        float f = (float)b;
                        if ((double)f < b) f = key_value(value_key(f) - 1);     // the next number above
                        q.least = fmaxf(q.least, f);
                    }
                }
                cut = ~0ull;
                kept_c = 0;
                counted = false;
                if (state == 0) {          // the lowest index of the largest number
                    if (tid == 0) sm.bin = INT_MAX;
                    __syncthreads();
                    int v = INT_MAX;
                    each_chunk([&](const float (&x)[E], int at) {
#pragma unroll
                        for (int e = E - 1; e >= 0; --e)
                            if (x[e] == mx) v = min(v, at + e);
                    });
                    if (v != INT_MAX) atomicMin(&sm.bin, v);
                    __syncthreads();
                    cut = place(mx, same(sm.bin));
                    kept_c = 1;
                    counted = true;
                }
                weigh = DRAW || p < 1.f;
                if (state == 2 && (weigh || k > 0)) {
                    const bool few = kth > -INFINITY;
                    each_chunk([&](const float (&x)[E], int) {
                        bool any = false;
#pragma unroll
                        for (int e = 0; e < E; ++e) any |= x[e] >= q.least;
                        if (few && !__any(any)) return;
#pragma unroll
                        for (int h = 0; h < E; h += 4) {
                            int bin[4];
                            uint64_t w[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                w[e] = weight_of(x[h + e], bin[e]);
                                bin[e] = x[h + e] >= q.least ? bin[e] : BINS + lane;
                            }
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                if (weigh) atomicAdd((unsigned long long*)&sm.w1[bin[e]], (unsigned long long)w[e]);
                                if (k > 0) atomicAdd(&sm.c1[bin[e]], 1u);
                            }
                        }
                    });
                    __syncthreads();
                    c_sum = 0;
                    w_sum = 0;
#pragma unroll
                    for (int b = 0; b < PER; ++b) {
                        c_sum += sm.c1[tid * PER + b];
                        w_sum += sm.w1[tid * PER + b];
                    }
                    block_scan<NT>(sm, c_sum, w_sum, c_at, w_at, kept_c, kept_w);
                    step = 0;
                }
            }
        }
        if (state == 1) {
            if (tid == 0) {
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
        // a chunk of the truncated row: f(number, class) says what stays
        const bool divide = t != 1.f && t != 0.f;
        const float rt = 1.f / t;
        constexpr float largest = sizeof(T) == 2 ? 0x1.FEp127f : FLT_MAX;   // (quotients do not become infinite)
        float edge = state == 2 ? q.least : q.top;   // nothing below it stays
        bool written = false;
        uint32_t stay_n = 0;
        auto over_t = [&](float x) {
            return quotient_fits(t, q.top, edge) ? quotient(x, t, rt) : fminf(fmaxf(x / t, -largest), largest);
        };
        auto put = [&](const float (&x)[E], int v, auto&& f) {
            T* out = (T*)a.out + (int64_t)r * a.ld;
            if (v >= a.V) return;
            float y[E];
            bool any = false;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const bool in = f(x[e], v + e);
                stay_n += in;
                any |= in;
                y[e] = in ? x[e] : -INFINITY;
            }
            if (divide && any)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float z = over_t(x[e]);
                    y[e] = y[e] == -INFINITY ? y[e] : z;
                }
            if (v + E <= a.V) {
                if constexpr (sizeof(T) == 2)
                    *(uint4*)(out + v) = make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
                else
                    *(float4*)(out + v) = make_float4(y[0], y[1], y[2], y[3]);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if (v + e >= a.V) continue;
                    if constexpr (sizeof(T) == 2) out[v + e] = f32_to_bf16(y[e]);
                    else out[v + e] = y[e];
                }
            }
        };
        if (state == 2 && (DRAW || step == 0)) {
            for (; step < (DRAW ? 3 : 2); ++step) {
                bool count = false;
                uint64_t bound = 0;
                if (step == 0) {
                    if (!(k > 0 && (uint32_t)k < kept_c)) continue;
                    count = true;
                    bound = (uint32_t)k;
                } else if (step == 1) {
                    if (!(p < 1.f)) continue;
                    bound = same((uint64_t)ceil((double)p * (double)kept_w));
                    bound = bound > 0 ? bound : 1;
                } else {
                    const uint32_t word = a.noise ? a.noise[i] : counter_word(a.seed, STREAM_TOKEN, a.step, a.row0 + (uint32_t)i, 0);
                    bound = same((uint64_t)(((double)word + 0.5) * 0x1p-32 * (double)kept_w) + 1);
                }
                // the bin where the running count or weight reaches the bound
                if (count ? c_at < bound && bound <= c_at + c_sum : w_at < bound && bound <= w_at + w_sum) {
                    uint32_t c = c_at;
                    uint64_t w = w_at;
#pragma unroll 1
                    for (int b = tid * PER;; ++b) {
                        const uint32_t c0 = sm.c1[b];
                        const uint64_t w0 = sm.w1[b];
                        if (count ? bound <= c + c0 : bound <= w + w0) {
                            sm.bin = b;
                            sm.before_c = c;
                            sm.before_w = w;
                            sm.listed = 0;
                            break;
                        }
                        c += c0;
                        w += w0;
                    }
                }
                __syncthreads();
                const int bin1 = same(sm.bin);
                uint32_t base_c = same(sm.before_c);
                uint64_t base_w = same(sm.before_w);
                // numbers that may stand in that bin: a quarter of a step more at either side
                const int n0 = bin1 << L::LOG, n1 = n0 + (1 << L::LOG) - 1;
                const float from = bin1 == BINS - 1 ? -FLT_MAX : (float)fmax((double)q.top - ((double)n1 + 0.75) / q.turn, -FLT_MAX);
                const float upto = bin1 == 0 ? q.top : (float)fmax((double)q.top - ((double)n0 - 0.75) / q.turn, -FLT_MAX);
                const float low = fmaxf(from, q.least), high = fmaxf(upto, low);
                edge = low;
                // the last pass but for the bin's numbers: what is larger stays.  (Not in place: the bin may have to be read again)
                const bool ahead = !DRAW && a.out != a.logits && (step == 1 || !(p < 1.f));
                // (a draw's pass counts what stays, if that is asked for and top-k has not said it)
                const bool tally = step == 2 && a.kept && !counted;
                const float last = key_value((uint32_t)(cut >> 32));
                uint32_t stay = 0;
                each_chunk([&](const float (&x)[E], int v) {
                    bool in[E], any = false;
                    if constexpr (!DRAW)
                        if (ahead) put(x, v, [&](float x, int) { return x > high; });
                    if (tally)
#pragma unroll
                        for (int e = 0; e < E; ++e)
                            stay += x[e] >= q.least && (cut == ~0ull || x[e] > last || (x[e] == last && v + e <= (int)(uint32_t)cut));
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        in[e] = __builtin_amdgcn_fmed3f(x[e], low, high) == x[e];
                        any |= in[e];
                    }
                    if (!__any(any)) return;
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (in[e]) {
                            const int y = atomicAdd(&sm.listed, 1);
                            if (y < CANDS) {
                                sm.value[y] = x[e];
                                sm.id[y] = v + e;
                            }
                        }
                });
                if (tally) {
                    stay = wave_scan(stay);
                    if (lane == 63) sm.csum[wv] = stay;
                }
                __syncthreads();
                if (tally) {
                    kept_c = 0;
                    for (int x = 0; x < NW; ++x) kept_c += same(sm.csum[x]);
                    counted = true;
                }
                int n = same(sm.listed);
                const bool few = n <= CANDS;
                if (few) {
                    if (tid < n) {
                        int bin;
                        const uint64_t w = weight_of(sm.value[tid], bin);
                        sm.place[tid] = bin == bin1 ? place(sm.value[tid], sm.id[tid]) : ~0ull;
                        sm.w[tid] = bin == bin1 && weigh ? w : 0;
                    }
                } else {
                    // too many: their places in PARTS parts, and those of the part where the bound lies, until they are few
                    uint64_t lo = 0, hi = ~0ull;
                    auto each = [&](auto&& f) {         // f(place, weight)
#pragma unroll 1
                        for (int v = tid; v < a.V; v += NT) {
                            const float x = Elem<T>::load1(row, v);
                            if (!(x >= low && x <= high)) continue;
                            int bin;
                            const uint64_t w = weight_of(x, bin), at = place(x, v);
                            if (bin == bin1 && at >= lo && at <= hi) f(at, w);
                        }
                    };
                    do {
                        uint64_t first = ~0ull, past = 0;
                        each([&](uint64_t at, uint64_t) {
                            first = first < at ? first : at;
                            past = past > at ? past : at;
                        });
                        for (int o = 32; o > 0; o >>= 1) {
                            const uint64_t f = __shfl_xor(first, o, 64), g = __shfl_xor(past, o, 64);
                            first = first < f ? first : f;
                            past = past > g ? past : g;
                        }
                        if (lane == 0) {
                            sm.lo[wv] = first;
                            sm.hi[wv] = past;
                        }
                        sm.c2[tid] = 0;
                        sm.w2[tid] = 0;
                        __syncthreads();
                        for (int x = 0; x < NW; ++x) {
                            first = first < sm.lo[x] ? first : sm.lo[x];
                            past = past > sm.hi[x] ? past : sm.hi[x];
                        }
                        first = same(first);
                        past = same(past);
                        int shift = 0;
                        while (((past - first) >> shift) >= PARTS) ++shift;
                        each([&](uint64_t at, uint64_t w) {
                            const int b = (int)((at - first) >> shift);
                            atomicAdd(&sm.c2[b], 1u);
                            if (weigh) atomicAdd((unsigned long long*)&sm.w2[b], (unsigned long long)w);
                        });
                        __syncthreads();
                        const uint32_t c = sm.c2[tid];
                        const uint64_t w = sm.w2[tid];
                        uint32_t ca, call;
                        uint64_t wa, wall;
                        block_scan<NT>(sm, c, w, ca, wa, call, wall);
                        ca += base_c;
                        wa += base_w;
                        if (count ? ca < bound && bound <= ca + c : wa < bound && bound <= wa + w) {
                            sm.bin = tid;
                            sm.before_c = ca;
                            sm.before_w = wa;
                            sm.in_c = c;
                            sm.listed = 0;
                        }
                        __syncthreads();
                        base_c = same(sm.before_c);
                        base_w = same(sm.before_w);
                        n = (int)same(sm.in_c);
                        lo = first + ((uint64_t)same(sm.bin) << shift);
                        // (no further than the range that was cut: a part's end lies past the last one's, and past 64 bits)
                        const uint64_t width = (1ull << shift) - 1;
                        hi = past - lo < width ? past : lo + width;
                        __syncthreads();
                    } while (n > CANDS);
                    each([&](uint64_t at, uint64_t w) {
                        const int x = atomicAdd(&sm.listed, 1);
                        sm.place[x] = at;
                        sm.w[x] = weigh ? w : 0;
                    });
                }
                __syncthreads();
                if (tid < n) {
                    const uint64_t mine = sm.place[tid], own = sm.w[tid];
                    uint32_t cs = base_c;
                    uint64_t ws = base_w;
#pragma unroll 4
                    for (int x = 0; x < n; ++x) {
                        const bool in = sm.place[x] <= mine;
                        cs += in;
                        ws += in ? sm.w[x] : 0;
                    }
                    if (mine != ~0ull && (count ? cs == bound : ws >= bound && ws - own < bound)) {
                        sm.at = mine;
                        sm.before_c = cs;
                        sm.before_w = ws;
                    }
                }
                __syncthreads();
                at = same(sm.at);
                if (!DRAW && ahead) {
                    written = few;
                    if (!few) {
                        stay_n = 0;
                    } else if (tid < n && place(sm.value[tid], sm.id[tid]) <= at) {
                        const float y = divide ? over_t(sm.value[tid]) : sm.value[tid];
                        T* out = (T*)a.out + (int64_t)r * a.ld + sm.id[tid];
                        if constexpr (sizeof(T) == 2) *out = f32_to_bf16(y);
                        else *out = y;
                        ++stay_n;
                    }
                }
                if (step < 2) {
                    cut = at;
                    kept_w = same(sm.before_w);
                    kept_c = same(sm.before_c);
                    counted = count;
                }
                __syncthreads();
            }
        }
        const float last = key_value((uint32_t)(cut >> 32));
        const int last_v = (int)(uint32_t)cut;
        const bool all = cut == ~0ull;
        auto stays = [&](float x, int v) { return x >= q.least && (all || x > last || (x == last && v <= last_v)); };
        if (DRAW && tid == 0) {
            if (a.kept) a.kept[i] = (int32_t)kept_c;
            if (state == 0) at = cut;
            a.z[i] = (int32_t)(uint32_t)at;
            if (a.logp) {
                const double x = ((double)key_value((uint32_t)(at >> 32)) - (double)q.top) / (double)t;
                a.logp[i] = state == 0 ? 0.f : (float)(x - log(ldexp((double)kept_w, -q.frac)));
            }
        }
        if constexpr (!DRAW) {
            if (!written) each_chunk([&](const float (&x)[E], int v) { put(x, v, stays); });
            if (a.kept) {
                const uint32_t n = wave_scan(stay_n);
                if (tid == 0) sm.count = 0;
                __syncthreads();
                if (lane == 63) atomicAdd(&sm.count, n);
                __syncthreads();
                if (tid == 0) a.kept[i] = (int32_t)sm.count;
            }
        }
    }
}

}  // namespace

template <bool DRAW>
static void launch_sample_keys(const SampleArgs& a, hipStream_t s) {
    auto go = [&](auto kernel, int threads) { launch_k(kernel, dim3((unsigned)a.n), dim3(threads), 0, s, a); };
    // A CU holds 1024 such threads, in one workgroup or several: a row ends soonest in many threads, and many rows cost least in
    // few each (a wavefront's share of the search is the same for any).  At up to a CU, up to two and more rows per CU, draws
    // under top-p: 32000 classes, 200 rows 14.0 us in 1024 threads and 15.1 in 512, 300 rows 24.1 and 19.7; 8000 classes, 500 rows 13.8
    // in 512 and 14.7 in 256, 700 rows 19.8 and 17.0; 16000 classes, 500 rows 16.2 and 17.7, 1024 rows 28.4 and 24.4;
    // 50257 classes, 200 rows 17.9 in 1024 and 18.7 in 512, 300 rows 31.6 and 24.7.  Between 32769 and 53248 classes a row pays for
    // all chunks: 33000, 40000 and 50257 under top-k too, 200 rows 22.8, 23.1 and 24.7, 300 rows 29.2, 28.5 and 31.0.
    const int cus = num_cus();
    const bool few = a.n <= cus, some = a.n <= 2 * (int64_t)cus;
    if (a.V <= 2048) go(sample_keys_kernel<256, 1, DRAW>, 256);
    else if (a.V <= 8192 && some) go(sample_keys_kernel<512, 2, DRAW>, 512);
    else if (a.V <= 8192) go(sample_keys_kernel<256, 4, DRAW>, 256);
    else if (a.V <= 16384 && some) go(sample_keys_kernel<512, 4, DRAW>, 512);
    else if (a.V <= 16384) go(sample_keys_kernel<256, 8, DRAW>, 256);
    else if (a.V <= 32768 && few) go(sample_keys_kernel<1024, 4, DRAW>, 1024);
    else if (a.V <= 32768) go(sample_keys_kernel<512, 8, DRAW>, 512);
    else if (a.V <= 57344 && few) go(sample_keys_kernel<1024, 7, DRAW>, 1024);
    else if (a.V <= 53248) go(sample_keys_kernel<512, 13, DRAW>, 512);
    else if (a.V <= 65536) go(sample_keys_kernel<512, 16, DRAW>, 512);
    else go(sample_keys_kernel<1024, 16, DRAW>, 1024);
}

template <typename T, bool DRAW>
static void launch_sample_t(const SampleArgs& args, hipStream_t s) {
    SampleArgs a = args;
    if constexpr (sizeof(T) == 2) {
        if (a.V <= 131072 && grid_fits(a.n, 1024)) return launch_sample_keys<DRAW>(a, s);
    }
    // Draws that share settings, and may share a row, are one workgroup's as far as every CU has one.  (Where they do not, that
    // costs: 4096 draws from as many rows of 32000 take 512 us with 16 draws to a setting, and 317 with one.)
    a.chunk = DRAW && a.per > 1 && a.row_ids ? (int)std::max<int64_t>(1, a.n / num_cus()) : 1;
    if (!grid_fits(ceil_div(a.n, a.chunk), 1024)) a.chunk = 1024;
    auto go = [&](auto kernel, int threads) { launch_k(kernel, dim3((unsigned)ceil_div(a.n, a.chunk)), dim3(threads), 0, s, a); };
    // As above: draws from 4000 classes, 200 rows 12.4 us in 256 threads and 13.3 in 512; from 16000, 300 rows 29.3 and 27.3, 700
    // rows 38.3 and 42.4; from 32000, 200 rows 31.5 in 512 and 26.2 in 1024, 300 rows 42.3 and 48.9, 2048 rows 159.7 in 256 and 164.3
    // in 512 (within the noise).
    const int64_t groups = ceil_div(a.n, a.chunk), cus = num_cus();
    if (a.V <= 4096 || (a.V <= 16384 && groups > 2 * cus)) return go(sample_stream_kernel<T, 256, DRAW>, 256);
    if (groups > cus) return go(sample_stream_kernel<T, 512, DRAW>, 512);
    go(sample_stream_kernel<T, 1024, DRAW>, 1024);
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
