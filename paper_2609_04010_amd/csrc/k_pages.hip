// Blocks of the cached context between passes: contexts that go on in several sequences, blocks copied, a pool put in
// order.
//
// Fork and compaction ask, for every block of the pool, which sequences hold it.  The pool is cut into ranges of RB blocks and
// the sequences into up to page_parts() parts: a workgroup of the first launch walks the tables of one part and keeps what falls
// into one range as bits in LDS, so nothing has to be cleared first and no atomics leave the CU.  The second launch joins
// the parts of each range and counts; the others rank blocks by those counts and write tables, stack and moves.  Bound by
// latency and launches: a pool of one range and few sequences is one launch.
#include <algorithm>

#include "cache.h"

namespace dd {

namespace {

constexpr int RB = PAGE_RANGE;      // blocks of a range
constexpr int RW = RB / 32;         // words of its bits
constexpr int MT = 1024;            // threads of the launches that look at ranges
constexpr int AT = 256;             // threads of the others
static_assert(RW == AT, "a thread per word of a range");
constexpr int ONE_LAUNCH = 128;     // sequences up to which one workgroup does everything for a pool of one range
constexpr int FREE_WORD = 63;       // of the first 64 words of a fork's workspace: the stack's height before it
constexpr int SOURCES = 8192;       // old rows up to which LDS holds how much of them stays

// f(block, j, head) for entry j < head.len of the rows part, part + parts, .. (block -1 behind that: no branch per lane); head(row)
// says how long a row is, and what else f wants to know.  A wavefront takes whole rows: the heads of 64 at once, then 256
// entries at a time.  Short code on purpose: each wavefront passes here a few times only, and fetching the instructions is
// most of that (32 rows on their way together, unrolled, took 17 us for 1024 rows of 128 and 25
// ranges in 8 parts; this takes 7, in 10).
struct Head {
    int len, whole;
};
template <int NT, typename H, typename F>
DD_DEV void walk(const int32_t* table, int64_t ld, int all, int part, int parts, H&& head, F&& f) {
    constexpr int W = NT / 64;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rows = (all - part + parts - 1) / parts;
#pragma unroll 1
    for (int base = wv; base < rows; base += 64 * W) {
        Head mine = {0, 0};
        if (base + lane * W < rows) mine = head((base + lane * W) * parts + part);
#pragma unroll 1
        for (int g = 0; g < 64 && base + g * W < rows; ++g) {
            const Head h = {__builtin_amdgcn_readlane(mine.len, g), __builtin_amdgcn_readlane(mine.whole, g)};
            const int32_t* p = table + ((int64_t)(base + g * W) * parts + part) * ld;
#pragma unroll 1
            for (int j0 = lane; j0 - lane < h.len; j0 += 256) {
                int b[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) b[u] = p[min(j0 + 64 * u, h.len - 1)];
#pragma unroll
                for (int u = 0; u < 4; ++u) f(j0 + 64 * u < h.len ? b[u] : -1, j0 + 64 * u, h);
            }
        }
    }
}
// whether an entry is out of range: entries of -1 that stand in a table are told from those behind a row by their place
DD_DEV bool wrong(int b, int j, const Head& h, int n_blocks) { return (uint32_t)b >= (uint32_t)n_blocks && j < h.len; }

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
// block it is; the other sequences of that kind take a fresh block, and a move for its contents.  What is held whole of an old row
// is a beginning of it, the longest that any new row asks for: the new rows are not walked.  1024
// rows of 65 entries, 9 ranges: 6 us with 28 parts, 12 with 8, 19 with one.
struct ForkLds {
    int32_t owner[RB];
    uint32_t old[RW], whole[RW], part[RW];      // held by an old row; whole by a new one; as a new one's partly filled last
    int32_t most[SOURCES];                      // whole blocks of an old row that new rows hold
    int red[MT / 64], bad;
    // in one launch, read once: where new rows come from, their last blocks, and what the phases hand on
    int32_t src[ONE_LAUNCH], len[ONE_LAUNCH], keep[ONE_LAUNCH], last[ONE_LAUNCH], copies[ONE_LAUNCH];
};

template <bool ONE> DD_DEV void fork_mark(const ForkArgs& a, ForkLds& sm, int range, int part) {
    const int tid = threadIdx.x, b0 = range * RB;
    const bool first = range == 0, fits = a.S <= SOURCES;
    for (int i = tid; i < (fits ? a.S : 0); i += MT) sm.most[i] = 0;
    if (tid < RW) sm.old[tid] = sm.whole[tid] = 0;
    if (tid == 0) sm.bad = 0;
    __syncthreads();
    bool bad = false;
    for (int s = tid; s < a.S_to; s += MT) {
        int src, len, keep;
        bad |= !fork_head(a, s, src, len, keep);
        const int n = keep >> a.c.log2p;
        if (fits && n > 0) atomicMax(&sm.most[src], n);
        if constexpr (ONE) {
            sm.src[s] = src;
            sm.len[s] = len;
            sm.keep[s] = keep;
            sm.last[s] = keep & (a.c.P - 1) ? a.table[(int64_t)src * a.ld_table + len - 1] : -1;
        }
    }
    __syncthreads();
    walk<MT>(a.table, a.ld_table, a.S, part, a.parts,
             [&](int q) {
                 int len;
                 bad |= !held_ok(a.held, a.ld_table, q, len);
                 if (first) {
                     const int have = a.seq_len[q];
                     bad |= have < 0 || have > (int64_t)len * a.c.P;
                 }
                 return Head{len, fits ? sm.most[q] : 0};
             },
             [&](int b, int j, const Head& h) {
                 if (first) bad |= wrong(b, j, h, a.c.n_blocks);      // (one range's workgroups look)
                 const uint32_t x = (uint32_t)b - (uint32_t)b0;
                 if (x < RB) {
                     atomicOr(&sm.old[x >> 5], 1u << (x & 31));
                     if (j < h.whole) atomicOr(&sm.whole[x >> 5], 1u << (x & 31));
                 }
             });
    if (!fits) {                         // the new rows one by one
        for (int s = part + a.parts * (tid >> 6); s < a.S_to; s += a.parts * (MT / 64)) {
            int src, len, keep;
            fork_head(a, s, src, len, keep);
            for (int j = tid & 63; j < keep >> a.c.log2p; j += 64) {
                const uint32_t x = (uint32_t)a.table[(int64_t)src * a.ld_table + j] - (uint32_t)b0;
                if (x < RB) atomicOr(&sm.whole[x >> 5], 1u << (x & 31));
            }
        }
    }
    if (bad) sm.bad = 1;
    __syncthreads();
    if constexpr (ONE) return;
    const int64_t word = (int64_t)range * RW + tid, words = ((int64_t)a.c.n_blocks + 31) / 32;
    if (tid < RW && word < words) {
        a.old[part * words + word] = sm.old[tid];
        a.whole[part * words + word] = sm.whole[tid];
    }
    if (first && tid == 0) a.bad[part] = sm.bad;
}

// the parts together: which blocks of the range are freed, and which sequences take a fresh block for one of it
template <bool ONE> DD_DEV void fork_join(const ForkArgs& a, ForkLds& sm, int range) {
    const int tid = threadIdx.x, b0 = range * RB;
    const int64_t word = (int64_t)range * RW + tid, words = ((int64_t)a.c.n_blocks + 31) / 32;
    for (int i = tid; i < RB; i += MT) sm.owner[i] = INT32_MAX;
    if (tid < RW) {
        if constexpr (!ONE) {
            uint32_t old = 0, whole = 0;
#pragma unroll 8
            for (int k = 0; k < a.parts; ++k) {
                old |= word < words ? a.old[k * words + word] : 0;
                whole |= word < words ? a.whole[k * words + word] : 0;
            }
            sm.old[tid] = old;
            sm.whole[tid] = whole;
        }
        sm.part[tid] = 0;
    }
    const bool bad = ONE ? (__syncthreads(), false) : __syncthreads_or(tid < a.parts && a.bad[tid]);
    // the partly filled last block of a sequence, -1 without
    auto last_block = [&](int s) -> int {
        if constexpr (ONE) return sm.last[s];
        int src, len, keep;
        fork_head(a, s, src, len, keep);
        return keep & (a.c.P - 1) ? a.table[(int64_t)src * a.ld_table + len - 1] : -1;
    };
    auto set = [&](int s, int copy) {
        if constexpr (ONE) sm.copies[s] = copy;
        else a.copies[s] = copy;
    };
    int mine = -1;                       // this thread's first sequence's
    for (int s = tid; s < a.S_to; s += MT) {
        const int b = last_block(s);
        const uint32_t x = (uint32_t)b - (uint32_t)b0;
        if (range == 0 && (uint32_t)b >= (uint32_t)a.c.n_blocks) set(s, 0);
        if (s == tid) mine = b;
        if (x >= RB || b >= a.c.n_blocks) continue;
        atomicMin(&sm.owner[x], s);
        atomicOr(&sm.part[x >> 5], 1u << (x & 31));
    }
    __syncthreads();
    for (int s = tid; s < a.S_to; s += MT) {
        const int b = s == tid ? mine : last_block(s);
        const uint32_t x = (uint32_t)b - (uint32_t)b0;
        if (x < RB && b < a.c.n_blocks) set(s, (sm.whole[x >> 5] >> (x & 31) & 1) || sm.owner[x] != s);
    }
    uint32_t w = tid < RW ? sm.old[tid] & ~sm.whole[tid] & ~sm.part[tid] : 0;
    if (tid < RW && word < words) a.freed[word] = w;
    const int n = block_sum<MT>(__popc(w), sm.red);
    if (tid == 0) a.counts[range] = n;
    if (!ONE && range == 0 && tid == 0) {
        a.bad[0] = bad;
        a.bad[FREE_WORD] = *a.n_free;    // (the next launch may write n_free_out in its place)
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

// NT threads; workgroup wg of `wgs`
template <int NT, bool ONE>
DD_DEV void fork_apply(const ForkArgs& a, ForkLds* sm, int* red, int wg, int wgs) {
    constexpr int W = NT / 64;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int s0 = wg * W;                         // sequences of this workgroup, one per wavefront
    const int32_t n_free = ONE ? *a.n_free : a.bad[FREE_WORD];
    const int bad = ONE ? sm->bad : a.bad[0];
    auto copies = [&](int s) -> int {
        if constexpr (ONE) return sm->copies[s];
        else return a.copies[s];
    };
    int before = 0, all = 0, freed = 0;
    for (int s = tid; s < a.S_to; s += NT) {
        const int c = copies(s);
        all += c;
        before += s < s0 ? c : 0;
    }
    for (int t = tid; t < a.ranges; t += NT) freed += a.counts[t];
    all = block_sum<NT>(all, red);
    before = block_sum<NT>(before, red);
    freed = block_sum<NT>(freed, red);
    const bool ok = !bad && n_free >= 0 && n_free <= a.c.n_blocks && (int64_t)n_free + freed <= a.c.n_blocks &&
                    all <= (int64_t)n_free + freed;
    if (wg == 0 && tid == 0) {
        if (!ok && a.err) atomicOr(a.err, DD_DEVERR_CACHE);
        *a.n_free_out = ok ? n_free + freed - all : n_free;
        *a.n_moves = ok ? all : 0;
    }
    for (int s1 = s0; s1 < a.S_to; s1 += wgs * W) {      // (one pass where there are as many workgroups as that)
        const int s = s1 + wv;
        if (s < a.S_to) {
            int src = 0, len = 0, keep = 0;
            if (ok) {
                if constexpr (ONE) {
                    src = sm->src[s];
                    len = sm->len[s];
                    keep = sm->keep[s];
                } else {
                    fork_head(a, s, src, len, keep);
                }
            }
            if (lane == 0) {
                a.to_held[s] = len;
                a.to_len[s] = keep;
            }
            const int32_t* from = a.table + (int64_t)src * a.ld_table;
            int32_t* to = a.to_table + (int64_t)s * a.ld_to;
            const bool copy = ok && copies(s);
            for (int j = lane; j < len - copy; j += 64) to[j] = from[j];
            if (copy) {
                int rank = before;
                for (int i = s1; i < s; ++i) rank += copies(i);
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
        if (s1 + wgs * W < a.S_to) {
            int c = 0;
            for (int i = s1 + tid; i < min(s1 + wgs * W, a.S_to); i += NT) c += copies(i);
            before += block_sum<NT>(c, red);
        }
    }
    if (!ok) return;
    // the freed blocks of a range, one word per thread
    int base = n_free, done = 0;
    for (int t = wg; t < a.ranges; t += wgs) {
        int sum = 0;
        for (int x = done + tid; x < t; x += NT) sum += a.counts[x];
        base += block_sum<NT>(sum, red);
        done = t;
        const int64_t word = (int64_t)t * RW + tid;
        uint32_t x = tid < RW && word * 32 < a.c.n_blocks ? a.freed[word] : 0;
        int i = base + block_before<NT>(__popc(x), red);
        for (; x; x &= x - 1) a.free_blocks[i++] = (int32_t)(word * 32) + __builtin_ctz(x);
    }
}

__global__ __launch_bounds__(MT) void fork_mark_kernel(ForkArgs a) {
    __shared__ ForkLds sm;
    fork_mark<false>(a, sm, blockIdx.x, blockIdx.y);
}
__global__ __launch_bounds__(MT) void fork_join_kernel(ForkArgs a) {
    __shared__ ForkLds sm;
    fork_join<false>(a, sm, blockIdx.x);
}
__global__ __launch_bounds__(AT) void fork_apply_kernel(ForkArgs a) {
    __shared__ int red[AT / 64];
    fork_apply<AT, false>(a, nullptr, red, blockIdx.x, gridDim.x);
}
// all of it for a pool of one range and few sequences, in one launch that hands on in LDS (through memory: 11 us and not 8.5 for
// one prompt to 16 continuations)
__global__ __launch_bounds__(MT) void fork_kernel(ForkArgs a) {
    __shared__ ForkLds sm;
    fork_mark<true>(a, sm, 0, 0);
    fork_join<true>(a, sm, 0);
    __threadfence_block();
    __syncthreads();
    fork_apply<MT, true>(a, &sm, sm.red, 0, 1);
}

// ---------------------------------------------------------------- compaction
//
// n blocks are in use.  The i-th used block >= n moves to the i-th number below n that is not used.  With used(b) blocks in use below
// b, block b >= n is number used(b) - used(n) of those that move, and an unused number h < n is number h - used(h) of those
// that they move to: each writes its half of a move, and the tables look theirs up.
struct CompactLds {
    uint32_t used[RW];
    int32_t start[PAGE_RANGES];         // used blocks before each range
    int red[MT / 64], bad;
};

DD_DEV void compact_mark(const CompactArgs& a, CompactLds& sm, int range, int part) {
    const int tid = threadIdx.x, b0 = range * RB;
    if (tid < RW) sm.used[tid] = 0;
    if (tid == 0) sm.bad = 0;
    __syncthreads();
    bool bad = false;
    walk<MT>(a.table, a.ld_table, a.S, part, a.parts,
             [&](int q) {
                 int len;
                 bad |= !held_ok(a.held, a.ld_table, q, len);
                 return Head{len, 0};
             },
             [&](int b, int j, const Head& h) {
                 if (range == 0) bad |= wrong(b, j, h, a.c.n_blocks);
                 const uint32_t x = (uint32_t)b - (uint32_t)b0;
                 if (x < RB) atomicOr(&sm.used[x >> 5], 1u << (x & 31));
             });
    if (bad) sm.bad = 1;
    __syncthreads();
    const int64_t word = (int64_t)range * RW + tid, words = ((int64_t)a.c.n_blocks + 31) / 32;
    if (tid < RW && word < words) a.used[part * words + word] = sm.used[tid];
    if (range == 0 && tid == 0) a.bad[part] = sm.bad;
}

// the parts together, into the first one's bits
DD_DEV void compact_join(const CompactArgs& a, CompactLds& sm, int range) {
    const int tid = threadIdx.x;
    const int64_t word = (int64_t)range * RW + tid, words = ((int64_t)a.c.n_blocks + 31) / 32;
    uint32_t x = 0;
    if (tid < RW && word < words)
#pragma unroll 8
        for (int k = 0; k < a.parts; ++k) x |= a.used[k * words + word];
    const bool bad = __syncthreads_or(tid < a.parts && a.bad[tid]);
    const int before = block_before<MT>(__popc(x), sm.red);
    if (tid < RW && word < words) {
        a.used[word] = x;
        a.before[word] = before;
    }
    if (tid == RW - 1) a.counts[range] = before + __popc(x);
    if (range == 0 && tid == 0) a.bad[0] = bad;
}

// used blocks before each range into start; their number
template <int NT>
DD_DEV int compact_starts(const CompactArgs& a, int32_t* start, int* red) {
    int n = 0;
    for (int t0 = 0; t0 < a.ranges; t0 += NT) {
        const int t = t0 + threadIdx.x, c = t < a.ranges ? a.counts[t] : 0;
        const int before = n + block_before<NT>(c, red);
        if (t < a.ranges) start[t] = before;
        n += block_sum<NT>(c, red);
    }
    __syncthreads();
    return n;
}
DD_DEV int used_before(const CompactArgs& a, const int32_t* start, int b) {      // b below n_blocks
    return start[b / RB] + a.before[b >> 5] + __popc(a.used[b >> 5] & ((1u << (b & 31)) - 1u));
}

// the moves and the stack
template <int NT>
DD_DEV void compact_moves(const CompactArgs& a, const int32_t* start, int n, int wg, int wgs) {
    const int nb = a.c.n_blocks;
    const int low = n < nb ? used_before(a, start, n) : n;     // used blocks below n: they stay
    const bool ok = !a.bad[0];
    if (wg == 0 && threadIdx.x == 0) {
        *a.n_moves = ok ? n - low : 0;
        if (ok) *a.n_free_out = nb - n;
        else if (a.err) atomicOr(a.err, DD_DEVERR_CACHE);
    }
    if (!ok) return;
    for (int64_t i = (int64_t)wg * NT + threadIdx.x; i < nb; i += (int64_t)wgs * NT) {
        const int b = (int)i;
        if (i < nb - n) a.free_blocks[i] = nb - 1 - b;
        const bool in = a.used[b >> 5] >> (b & 31) & 1;
        if (in == (b < n)) continue;
        const int u = used_before(a, start, b);
        if (in) a.moves[2 * (u - low)] = b;
        else a.moves[2 * (b - u) + 1] = b;
    }
}

// the tables under the new numbers
template <int NT>
DD_DEV void compact_tables(const CompactArgs& a, const int32_t* start, int n, int wg, int wgs) {
    const int lane = threadIdx.x & 63, nb = a.c.n_blocks;
    const int low = n < nb ? used_before(a, start, n) : n;
    const bool ok = !a.bad[0];
    for (int q = wg * (NT / 64) + (threadIdx.x >> 6); q < a.S; q += wgs * (NT / 64)) {
        int len;
        held_ok(a.held, a.ld_table, q, len);
        const int32_t* from = a.table + (int64_t)q * a.ld_table;
        int32_t* to = a.to_table + (int64_t)q * a.ld_table;
        for (int j = lane; j < len; j += 64) {
            const int b = from[j];
            to[j] = ok && b >= n ? a.moves[2 * (used_before(a, start, b) - low) + 1] : b;
        }
    }
}

__global__ __launch_bounds__(MT) void compact_mark_kernel(CompactArgs a) {
    __shared__ CompactLds sm;
    compact_mark(a, sm, blockIdx.x, blockIdx.y);
}
__global__ __launch_bounds__(MT) void compact_join_kernel(CompactArgs a) {
    __shared__ CompactLds sm;
    compact_join(a, sm, blockIdx.x);
}
__global__ __launch_bounds__(AT) void compact_moves_kernel(CompactArgs a) {
    __shared__ int32_t start[PAGE_RANGES];
    __shared__ int red[AT / 64];
    compact_moves<AT>(a, start, compact_starts<AT>(a, start, red), blockIdx.x, gridDim.x);
}
__global__ __launch_bounds__(AT) void compact_tables_kernel(CompactArgs a) {
    __shared__ int32_t start[PAGE_RANGES];
    __shared__ int red[AT / 64];
    compact_tables<AT>(a, start, compact_starts<AT>(a, start, red), blockIdx.x, gridDim.x);
}
// all of it for a pool of one range and few sequences: one launch
__global__ __launch_bounds__(MT) void compact_kernel(CompactArgs a) {
    __shared__ CompactLds sm;
    compact_mark(a, sm, 0, 0);
    __threadfence_block();
    __syncthreads();
    compact_join(a, sm, 0);
    __threadfence_block();
    __syncthreads();
    const int n = compact_starts<MT>(a, sm.start, sm.red);
    compact_moves<MT>(a, sm.start, n, 0, 1);
    __threadfence_block();
    __syncthreads();
    compact_tables<MT>(a, sm.start, n, 0, 1);
}

// ---------------------------------------------------------------- copy
//
// A block's codes of all heads stand one behind the other, H 2 P dh bytes, and so do its scales.  A workgroup copies a piece of
// one block in one layer, 16 bytes per thread, and takes another while there are any: how many moves there are, only the
// device knows.  Bound by the memory: 4.9 TB/s read and written at 1024 moves of 98304 bytes in 12 layers, 494 us; 16 of them
// take 7.7 on the same 38 MB again and again, which the last-level cache keeps, and 11.5 on those of 12 pools in turn.  One load per thread and many short workgroups: two or four loads per thread cost the small copy 9 us, and the large
// one 5.  16 workgroups per CU and not as many as there are pieces: 484 us at 64 per CU, but an empty list would pay for those.
constexpr int CT = 512;
constexpr int PIECE = CT * 16;

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
        if (at < a.slab) *(uint4*)(dst + at) = *(const uint4*)(src + at);
        if (piece == 0) {
            const float2* ss = (const float2*)a.scales + (lay + from) * a.heads;
            float2* sd = (float2*)a.scales + (lay + to) * a.heads;
            for (int h = tid; h < a.heads; h += CT) sd[h] = ss[h];
        }
    }
}

}  // namespace

// ONE_LAUNCH: 16 sequences compact in 7 us, and took 9 in three launches.  Sequences of a part: two for a wavefront.
constexpr int PER_PART = 2 * MT / 64;

static int parts_for(int ranges, int32_t S) { return std::max(1, std::min(page_parts(ranges), S / PER_PART)); }

dd_status launch_cache_fork(const ForkArgs& args, hipStream_t s) {
    ForkArgs a = args;
    auto go = [&](auto kernel, dim3 grid, int threads) {
        ProfScope ps(KC_CACHE_FORK, s);
        launch_k(kernel, grid, dim3(threads), 0, s, a);
    };
    if (a.ranges == 1 && a.S <= ONE_LAUNCH && a.S_to <= ONE_LAUNCH) {
        a.parts = 1;
        go(fork_kernel, dim3(1), MT);
        return launch_status("cache_fork");
    }
    a.parts = parts_for(a.ranges, a.S);
    // (The last launch has a wavefront per new sequence; each workgroup sums the copies of all, and together they push the freed
    // blocks of all ranges.  Both show at the ends: 1024 sequences of 512 tokens into 65536 take 513 us, 16384 of 4096 into 4 take 994.)
    go(fork_mark_kernel, dim3((unsigned)a.ranges, (unsigned)a.parts), MT);
    go(fork_join_kernel, dim3((unsigned)a.ranges), MT);
    go(fork_apply_kernel, dim3((unsigned)std::max<int64_t>(1, ceil_div(a.S_to, AT / 64))), AT);
    return launch_status("cache_fork");
}

dd_status launch_cache_compact(const CompactArgs& args, hipStream_t s) {
    CompactArgs a = args;
    auto go = [&](auto kernel, dim3 grid, int threads) {
        ProfScope ps(KC_CACHE_COMPACT, s);
        launch_k(kernel, grid, dim3(threads), 0, s, a);
    };
    if (a.ranges == 1 && a.S <= ONE_LAUNCH) {
        a.parts = 1;
        go(compact_kernel, dim3(1), MT);
        return launch_status("cache_compact");
    }
    a.parts = parts_for(a.ranges, a.S);
    go(compact_mark_kernel, dim3((unsigned)a.ranges, (unsigned)a.parts), MT);
    go(compact_join_kernel, dim3((unsigned)a.ranges), MT);
    go(compact_moves_kernel, dim3((unsigned)std::min<int64_t>(1024, ceil_div(a.c.n_blocks, AT))), AT);
    go(compact_tables_kernel, dim3((unsigned)std::min<int64_t>(1024, std::max<int64_t>(1, ceil_div(a.S, AT / 64)))), AT);
    return launch_status("cache_compact");
}

dd_status launch_cache_copy(const CopyArgs& a, hipStream_t s) {
    const double units = (double)ceil_div(a.slab, PIECE) * a.max_moves * a.layers;
    ProfScope ps(KC_CACHE_COPY, s);
    launch_k(copy_kernel, dim3((unsigned)std::min<double>(units, 16 * num_cus())), dim3(CT), 0, s, a);
    return launch_status("cache_copy");
}

}  // namespace dd
