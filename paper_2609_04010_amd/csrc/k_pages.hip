// Blocks of the cached context between passes: contexts that go on in several sequences, blocks copied, a pool put in
// order.
//
// Fork and compaction ask, for every block of the pool, which sequences hold it.  Launch 1 cuts the pool into ranges of
// RB blocks, one workgroup each: every workgroup walks all tables and keeps what falls into its range in LDS, so
// nothing has to be cleared first and no atomics leave the CU; it leaves a bit per block and a count per range.  Launch 2
// ranks blocks by those counts and the bits, and writes tables, stack and moves.
#include <algorithm>

#include "cache.h"

namespace dd {

namespace {

constexpr int RB = PAGE_RANGE;      // blocks of a range
constexpr int RW = RB / 32;         // words of its bits
constexpr int MT = 1024;            // threads of launch 1
constexpr int AT = 256;             // threads of launch 2
static_assert(RW == AT, "a thread per word of a range");

// f(block, row, j, length) for entry j < length of every row; head(row, source, length) says where a row stands in
// the table.  A wavefront takes whole rows, the heads of 64 at once and the first entries of four.
template <int NT, typename Head, typename F>
DD_DEV void walk(const int32_t* table, int64_t ld, int rows, Head&& head, F&& f) {
    constexpr int W = NT / 64;
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    for (int base = wv; base < rows; base += 64 * W) {
        int src = 0, len = 0;
        if (base + lane * W < rows) head(base + lane * W, src, len);
        for (int g = 0; g < 64 && base + g * W < rows; g += 4) {
            const int32_t* p[4];
            int n[4], b[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                n[u] = __builtin_amdgcn_readlane(len, g + u);
                p[u] = table + (int64_t)__builtin_amdgcn_readlane(src, g + u) * ld;
                b[u] = lane < n[u] ? p[u][lane] : 0;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int row = base + (g + u) * W;
                if (lane < n[u]) f(b[u], row, lane, n[u]);
#pragma unroll 4
                for (int j = lane + 64; j < n[u]; j += 64) f(p[u][j], row, j, n[u]);
            }
        }
    }
}

// where row s of the new tables comes from, and how many entries it has; false where that is no fork's
DD_DEV bool fork_head(const ForkArgs& a, int s, int& src, int& len, int& keep) {
    src = a.src[s];
    len = keep = 0;
    if (src == -1) {
        src = 0;
        return true;
    }
    if (src < -1 || src >= a.S) {
        src = 0;
        return false;
    }
    const int have = a.seq_len[src], held = a.held[src];
    const int want = a.keep ? a.keep[s] : have;
    if (want < 0 || want > have || held < 0 || held > a.ld_table || have > (int64_t)held * a.c.P) return false;
    const int n = (int)(((int64_t)want + a.c.P - 1) >> a.c.log2p);
    if (n > a.ld_to) return false;
    len = n;
    keep = want;
    return true;
}
DD_DEV bool held_ok(const int32_t* held, int ld, int q, int& len) {
    len = held[q];
    if (len >= 0 && len <= ld) return true;
    len = 0;
    return false;
}

// sum over the workgroup, for every thread
template <int NT> DD_DEV int block_sum(int v, int* red) {
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
    for (int i = 0; i < NT / 64; ++i) v += red[i];
    return v;
}
// exclusive prefix sum of v over the workgroup
template <int NT> DD_DEV int block_before(int v, int* red) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    int inc = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(inc, o, 64);
        if (lane >= o) inc += up;
    }
    __syncthreads();
    if (lane == 63) red[wv] = inc;
    __syncthreads();
    for (int i = 0; i < wv; ++i) inc += red[i];
    return inc - v;
}

// the place of the r-th set bit of w, r below their number
DD_DEV int nth_bit(uint32_t w, int r) {
    while (r-- > 0) w &= w - 1;
    return __builtin_ctz(w);
}

// ---------------------------------------------------------------- fork
//
// Row s of the new tables is the first ceil(keep_s / P) entries of row src_s of the old ones.  A block is freed if an old
// row holds it and no new one.  owner[b]: -1 where a new row holds b whole, else the first sequence whose partly filled last
// block it is; the other sequences of that kind take a fresh block, and a move for its contents.
__global__ __launch_bounds__(MT) void fork_mark_kernel(ForkArgs a) {
    __shared__ int32_t owner[RB];
    __shared__ uint32_t old[RW];
    __shared__ int red[MT / 64], bad;
    const int tid = threadIdx.x, b0 = blockIdx.x * RB;
    const bool first = blockIdx.x == 0;
    for (int i = tid; i < RB; i += MT) owner[i] = INT32_MAX;
    if (tid < RW) old[tid] = 0;
    if (tid == 0) bad = 0;
    __syncthreads();
    walk<MT>(a.table, a.ld_table, a.S,
             [&](int q, int& src, int& len) {
                 src = q;
                 bool ok = held_ok(a.held, a.ld_table, q, len);
                 if (first) {
                     const int have = a.seq_len[q];
                     ok = ok && have >= 0 && have <= (int64_t)len * a.c.P;
                 }
                 if (!ok) bad = 1;
             },
             [&](int b, int, int, int) {
                 if (b < 0 || b >= a.c.n_blocks) bad = 1;
                 const uint32_t x = (uint32_t)b - (uint32_t)b0;
                 if (x < RB) atomicOr(&old[x >> 5], 1u << (x & 31));
             });
    walk<MT>(a.table, a.ld_table, a.S_to,
             [&](int s, int& src, int& len) {
                 int keep;
                 if (!fork_head(a, s, src, len, keep)) bad = 1;
             },
             [&](int b, int s, int j, int n) {
                 const uint32_t x = (uint32_t)b - (uint32_t)b0;
                 if (x >= RB) return;
                 int who = -1;
                 if (j == n - 1 && ((a.keep ? a.keep[s] : a.seq_len[a.src[s]]) & (a.c.P - 1))) who = s;   // partly filled
                 atomicMin(&owner[x], who);
             });
    __syncthreads();
    int n = 0;
    if (tid < RW) {
        uint32_t w = old[tid];
        for (uint32_t x = w; x; x &= x - 1) {
            const int k = __builtin_ctz(x);
            if (owner[tid * 32 + k] != INT32_MAX) w &= ~(1u << k);
        }
        n = __popc(w);
        if (b0 + tid * 32 < a.c.n_blocks) a.freed[blockIdx.x * RW + tid] = w;
    }
    n = block_sum<MT>(n, red);
    if (tid == 0) {
        a.counts[blockIdx.x] = n;
        if (first) *a.bad = bad;
    }
    for (int s = tid; s < a.S_to; s += MT) {
        int src, len, keep, b = -1;
        fork_head(a, s, src, len, keep);
        const bool part = len > 0 && (keep & (a.c.P - 1));
        if (part) b = a.table[(int64_t)src * a.ld_table + len - 1];
        const uint32_t x = (uint32_t)b - (uint32_t)b0;
        if (part && x < RB) a.copies[s] = owner[x] != s;
        if (first && (!part || b < 0 || b >= a.c.n_blocks)) a.copies[s] = 0;
    }
}

// the r-th freed block in ascending order, by a wavefront
DD_DEV int nth_freed(const ForkArgs& a, int r) {
    const int lane = threadIdx.x & 63;
    int t = 0;
    for (int n; r >= (n = a.counts[t]); ++t) r -= n;
    const uint32_t* w = a.freed + (int64_t)t * RW;
    const int words = min(RW, (int)(((int64_t)a.c.n_blocks + 31) / 32 - (int64_t)t * RW));
    for (int k = 0;; k += 64) {      // (ends: r is below the range's count)
        const uint32_t x = k + lane < words ? w[k + lane] : 0;
        const int c = __popc(x);
        int inc = c;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int up = __shfl_up(inc, o, 64);
            if (lane >= o) inc += up;
        }
        const uint64_t hit = __ballot(inc > r);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            const int before = __shfl(inc - c, l, 64);
            return (t * RW + k + l) * 32 + nth_bit((uint32_t)__shfl((int)x, l, 64), r - before);
        }
        r -= __shfl(inc, 63, 64);
    }
}

__global__ __launch_bounds__(AT) void fork_apply_kernel(ForkArgs a) {
    __shared__ int red[AT / 64];
    constexpr int W = AT / 64;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int s0 = blockIdx.x * W;                 // sequences of this workgroup, one per wavefront
    const int32_t n_free = *a.n_free;
    int before = 0, all = 0, freed = 0;
    for (int s = tid; s < a.S_to; s += AT) {
        const int c = a.copies[s];
        all += c;
        before += s < s0 ? c : 0;
    }
    for (int t = tid; t < a.ranges; t += AT) freed += a.counts[t];
    all = block_sum<AT>(all, red);
    before = block_sum<AT>(before, red);
    freed = block_sum<AT>(freed, red);
    const bool ok = !*a.bad && n_free >= 0 && n_free <= a.c.n_blocks && (int64_t)n_free + freed <= a.c.n_blocks &&
                    all <= (int64_t)n_free + freed;
    if (blockIdx.x == 0 && tid == 0) {
        if (!ok && a.err) atomicOr(a.err, DD_DEVERR_CACHE);
        *a.n_free_out = ok ? n_free + freed - all : n_free;
        *a.n_moves = ok ? all : 0;
    }
    const int s = s0 + wv;
    if (s < a.S_to) {
        int src = 0, len = 0, keep = 0;
        if (ok) fork_head(a, s, src, len, keep);
        if (lane == 0) {
            a.to_held[s] = len;
            a.to_len[s] = keep;
        }
        const int32_t* from = a.table + (int64_t)src * a.ld_table;
        int32_t* to = a.to_table + (int64_t)s * a.ld_to;
        const bool copy = ok && a.copies[s];
        for (int j = lane; j < len - copy; j += 64) to[j] = from[j];
        if (copy) {
            int rank = before;
            for (int i = 0; i < wv; ++i) rank += a.copies[s0 + i];
            // the top of the stack once the freed blocks are on it
            const int at = n_free + freed - 1 - rank;
            const int b = at < n_free ? a.free_blocks[at] : nth_freed(a, at - n_free);
            if (lane == 0) {
                to[len - 1] = b;
                a.moves[2 * rank] = from[len - 1];
                a.moves[2 * rank + 1] = b;
                if ((b < 0 || b >= a.c.n_blocks) && a.err) atomicOr(a.err, DD_DEVERR_CACHE);
            }
        }
    }
    if (!ok) return;
    // the freed blocks of a range, one word per thread
    int base = n_free, done = 0;
    for (int t = blockIdx.x; t < a.ranges; t += gridDim.x) {
        int sum = 0;
        for (int x = done + tid; x < t; x += AT) sum += a.counts[x];
        base += block_sum<AT>(sum, red);
        done = t;
        const int64_t word = (int64_t)t * RW + tid;
        uint32_t x = word * 32 < a.c.n_blocks ? a.freed[word] : 0;
        int i = base + block_before<AT>(__popc(x), red);
        for (; x; x &= x - 1) a.free_blocks[i++] = (int32_t)(word * 32) + __builtin_ctz(x);
    }
}

// ---------------------------------------------------------------- compaction
//
// n blocks are in use.  The i-th used block >= n moves to the i-th number below n that is not used.
__global__ __launch_bounds__(MT) void compact_mark_kernel(CompactArgs a) {
    __shared__ uint32_t used[RW];
    __shared__ int red[MT / 64], bad;
    const int tid = threadIdx.x, b0 = blockIdx.x * RB;
    if (tid < RW) used[tid] = 0;
    if (tid == 0) bad = 0;
    __syncthreads();
    walk<MT>(a.table, a.ld_table, a.S,
             [&](int q, int& src, int& len) {
                 src = q;
                 if (!held_ok(a.held, a.ld_table, q, len)) bad = 1;
             },
             [&](int b, int, int, int) {
                 if (b < 0 || b >= a.c.n_blocks) bad = 1;
                 const uint32_t x = (uint32_t)b - (uint32_t)b0;
                 if (x < RB) atomicOr(&used[x >> 5], 1u << (x & 31));
             });
    __syncthreads();
    const int c = tid < RW ? __popc(used[tid]) : 0;
    const int before = block_before<MT>(c, red);
    if (tid < RW && b0 + tid * 32 < a.c.n_blocks) {
        a.used[blockIdx.x * RW + tid] = used[tid];
        a.before[blockIdx.x * RW + tid] = before;
    }
    if (tid == RW - 1) {
        a.counts[blockIdx.x] = before + c;
        if (blockIdx.x == 0) *a.bad = bad;
    }
}

__global__ __launch_bounds__(AT) void compact_apply_kernel(CompactArgs a) {
    __shared__ int32_t start[PAGE_RANGES];         // used blocks before each range
    __shared__ int red[AT / 64];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    int n = 0;
    for (int t0 = 0; t0 < a.ranges; t0 += AT) {
        const int c = t0 + tid < a.ranges ? a.counts[t0 + tid] : 0;
        const int before = n + block_before<AT>(c, red);
        if (t0 + tid < a.ranges) start[t0 + tid] = before;
        n += block_sum<AT>(c, red);
    }
    __syncthreads();
    const int nb = a.c.n_blocks;
    const bool ok = !*a.bad;
    auto used_before = [&](int b) {                // used blocks below b < nb
        return start[b / RB] + a.before[b >> 5] + __popc(a.used[b >> 5] & ((1u << (b & 31)) - 1u));
    };
    const int low = n < nb ? used_before(n) : n;   // used blocks below n: they stay
    auto hole = [&](int r) {                       // the r-th number below n that is not used
        int lo = 0, hi = (n - 1) >> 5;             // the last word that fewer or as many as r free numbers stand before
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (mid * 32 - (start[mid / RW] + a.before[mid]) <= r) lo = mid;
            else hi = mid - 1;
        }
        return lo * 32 + nth_bit(~a.used[lo], r - (lo * 32 - (start[lo / RW] + a.before[lo])));
    };
    const int gw = blockIdx.x * (AT / 64) + wv, waves = gridDim.x * (AT / 64);
    for (int q = gw; q < a.S; q += waves) {
        int len;
        held_ok(a.held, a.ld_table, q, len);
        const int32_t* from = a.table + (int64_t)q * a.ld_table;
        int32_t* to = a.to_table + (int64_t)q * a.ld_table;
        for (int j = lane; j < len; j += 64) {
            const int b = from[j];
            to[j] = ok && b >= n ? hole(used_before(b) - low) : b;
        }
    }
    if (blockIdx.x == 0 && tid == 0) {
        if (ok) {
            *a.n_free_out = nb - n;
            *a.n_moves = n - low;
        } else {
            *a.n_moves = 0;
            if (a.err) atomicOr(a.err, DD_DEVERR_CACHE);
        }
    }
    if (!ok) return;
    const int64_t step = (int64_t)gridDim.x * AT, at = (int64_t)blockIdx.x * AT + tid;
    for (int64_t i = at; i < nb - n; i += step) a.free_blocks[i] = (int32_t)(nb - 1 - i);
    for (int64_t b = n + at; b < nb; b += step)
        if (a.used[b >> 5] >> (b & 31) & 1) {
            const int r = used_before((int)b) - low;
            a.moves[2 * r] = (int32_t)b;
            a.moves[2 * r + 1] = hole(r);
        }
}

// ---------------------------------------------------------------- copy
//
// A block's codes of all heads stand one behind the other, H 2 P dh bytes, and so do its scales.  A workgroup copies a piece of
// one block in one layer.
constexpr int CT = 256, CL = 4;           // threads, 16-byte loads of each
constexpr int PIECE = CT * CL * 16;

__global__ __launch_bounds__(CT) void copy_kernel(CopyArgs a) {
    const int tid = threadIdx.x;
    const uint32_t pieces = (uint32_t)((a.slab + PIECE - 1) / PIECE), per = pieces * (uint32_t)a.layers;
    const int n_moves = min(*a.n_moves, a.max_moves);
    for (int64_t unit = blockIdx.x; unit < (int64_t)n_moves * per; unit += gridDim.x) {
        const int move = (int)(unit / per);
        const uint32_t in = (uint32_t)(unit - (int64_t)move * per), layer = in / pieces, piece = in - layer * pieces;
        const int from = a.moves[2 * move], to = a.moves[2 * move + 1];
        if ((uint32_t)from >= (uint32_t)a.n_blocks || (uint32_t)to >= (uint32_t)a.n_blocks) {
            if (tid == 0 && in == 0 && a.err) atomicOr(a.err, DD_DEVERR_CACHE);
            continue;
        }
        const int64_t lay = (int64_t)layer * a.n_blocks;
        const uint8_t* src = a.codes + (lay + from) * a.slab;
        uint8_t* dst = a.codes + (lay + to) * a.slab;
        const int64_t at = (int64_t)piece * PIECE + tid * 16;
        uint4 u[CL];
#pragma unroll
        for (int k = 0; k < CL; ++k)
            if (at + k * CT * 16 < a.slab) u[k] = *(const uint4*)(src + at + k * CT * 16);
#pragma unroll
        for (int k = 0; k < CL; ++k)
            if (at + k * CT * 16 < a.slab) *(uint4*)(dst + at + k * CT * 16) = u[k];
        if (piece == 0) {
            const float2* ss = (const float2*)a.scales + (lay + from) * a.heads;
            float2* sd = (float2*)a.scales + (lay + to) * a.heads;
            for (int h = tid; h < a.heads; h += CT) sd[h] = ss[h];
        }
    }
}

}  // namespace

dd_status launch_cache_fork(const ForkArgs& a, hipStream_t s) {
    {
        ProfScope ps(KC_CACHE_FORK, s);
        launch_k(fork_mark_kernel, dim3((unsigned)a.ranges), dim3(MT), 0, s, a);
    }
    ProfScope ps(KC_CACHE_FORK, s);
    launch_k(fork_apply_kernel, dim3((unsigned)std::max<int64_t>(1, ceil_div(a.S_to, AT / 64))), dim3(AT), 0, s, a);
    return launch_status("cache_fork");
}

dd_status launch_cache_compact(const CompactArgs& a, hipStream_t s) {
    {
        ProfScope ps(KC_CACHE_COMPACT, s);
        launch_k(compact_mark_kernel, dim3((unsigned)a.ranges), dim3(MT), 0, s, a);
    }
    ProfScope ps(KC_CACHE_COMPACT, s);
    const int64_t wgs = std::max(ceil_div(a.S, AT / 64), ceil_div(a.c.n_blocks, 4 * AT));
    launch_k(compact_apply_kernel, dim3((unsigned)std::min<int64_t>(1024, wgs)), dim3(AT), 0, s, a);
    return launch_status("cache_compact");
}

dd_status launch_cache_copy(const CopyArgs& a, hipStream_t s) {
    const double units = (double)ceil_div(a.slab, PIECE) * a.max_moves * a.layers;
    ProfScope ps(KC_CACHE_COPY, s);
    launch_k(copy_kernel, dim3((unsigned)std::min<double>(units, 8 * num_cus())), dim3(CT), 0, s, a);
    return launch_status("cache_copy");
}

}  // namespace dd
