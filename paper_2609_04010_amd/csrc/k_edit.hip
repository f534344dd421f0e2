// Penalties for repeated tokens, biases and allowed-token masks on rows of logits.
//
// A workgroup owns a piece of EC classes and walks rows_per_wg rows, R at a time.  In LDS stand the counts of the
// history's tokens and the biases of its classes, and a list of the classes that have either (whole numbers, so the
// order of the atomics does not show).  The rows' pieces pass through LDS as they are in memory: there the listed
// classes are edited, one per thread whatever rows they belong to, and every thread takes its 16 bytes back,
// applies the mask to the packed numbers and stores them.  Rows of one sequence share their counts: a longer
// history adds its new entries (those that only some of the rows edited together have are compared one by one), a
// shorter one (or another sequence) begins again.
//
// Bound by the memory traffic of the logits: 16384 rows of 50257 bf16 take 0.61 ms with every kind of edit (0.59 to
// 0.61 with any one kind, a copy 0.67 ms), 5.4 TB/s.  2048 classes and 4 rows at a time (8 rows: the same time, twice
// the LDS; 4096 classes: 3 % slower).  No row waits for its own history length or mask number: the lanes read those
// of 64 rows at once (read row by row, 0.77 ms).
#include <algorithm>

#include "cache.h"
#include "elem.h"

namespace dd {

constexpr int EC = 2048;   // classes of a workgroup
constexpr int ET = 256;
constexpr int MORE = 64;   // entries by which the histories of rows edited together may differ

template <typename T> DD_DEV void store_one(T* p, float x);
template <> DD_DEV void store_one<bf16_t>(bf16_t* p, float x) { *p = f32_to_bf16(x); }
template <> DD_DEV void store_one<float>(float* p, float x) { *p = x; }

// -inf where a bit of ok is clear
template <typename T> DD_DEV void mask_chunk(uint4& u, uint32_t ok) {
    uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        uint32_t keep;
        if constexpr (sizeof(T) == 2) {
            const uint32_t lo = (uint32_t)((int32_t)(ok << (31 - 2 * k)) >> 31), hi = (uint32_t)((int32_t)(ok << (30 - 2 * k)) >> 31);
            keep = (lo & 0xFFFFu) | (hi & 0xFFFF0000u);
            w[k] = (w[k] & keep) | (0xFF80FF80u & ~keep);
        } else {
            keep = (uint32_t)((int32_t)(ok << (31 - k)) >> 31);
            w[k] = (w[k] & keep) | (0xFF800000u & ~keep);
        }
    }
    u = make_uint4(w[0], w[1], w[2], w[3]);
}

// R: rows at a time
template <typename T, int R>
__global__ __launch_bounds__(ET) void logits_edit_kernel(EditArgs a) {
    constexpr int E = Elem<T>::E, NC = EC / (ET * E);   // chunks per thread and row
    __shared__ __attribute__((aligned(16))) T piece[R][EC];
    __shared__ __attribute__((aligned(16))) uint32_t count[EC];     // how often the class stands in the history
    __shared__ __attribute__((aligned(16))) uint32_t bias[EC];      // its bias (while they are gathered: 1 + the last entry
                                                                    // of the bias list that names it)
    __shared__ uint32_t some[EC / 32];                              // classes with either,
    __shared__ uint16_t list[EC];                                   // and the same as a list
    __shared__ int listed;
    __shared__ uint16_t extra[MORE];                                // classes of the entries that only later rows of a run have
    __shared__ int entries[R];                                      // the rows' history lengths
    const int tid = threadIdx.x;
    const int v0 = blockIdx.x * EC, nv = min(EC, a.V - v0);
    const int m0 = blockIdx.y * a.rows_per_wg, m1 = min(m0 + a.rows_per_wg, a.rows);
    const bool biased = a.e.bias_ids != nullptr && a.e.n_bias > 0;
    const bool lists = a.e.ld_history > 0 || biased;   // some class may need its logit changed
    int seq = -1, have = 0;   // sequence whose tables stand in LDS, entries counted
    float rep = 1.f, pres = 0.f, freq = 0.f;
    // history lengths (negative: the row goes through as it is) and mask numbers of 64 rows, one per lane: no row
    // waits for its own
    int lens = 0, masks = 0;
    auto window = [&](int g) {
        const int m = min(g + (tid & 63), m1 - 1);
        const int64_t n = a.e.hist_len ? a.e.hist_len[m] : a.e.ld_history;
        lens = (int)(n < a.e.ld_history ? n : a.e.ld_history);
        masks = a.e.allow_id ? a.e.allow_id[m] : 0;
    };
    auto length = [&](int m) { return __builtin_amdgcn_readlane(lens, (m - m0) & 63); };
    auto add = [&](uint32_t v) {   // class v of this piece into the list
        const uint32_t bit = 1u << (v & 31u);
        if (!(atomicOr(&some[v >> 5], bit) & bit)) list[atomicAdd(&listed, 1)] = (uint16_t)v;
    };
    for (int g = m0; g < m1; g += R) {
        const int nr = min(R, m1 - g);
        if (((g - m0) & 63) == 0) window(g);
        uint4 u[R][NC];
        uint32_t ok[R][NC];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const T* in = (const T*)a.logits + (int64_t)min(g + r, m1 - 1) * a.ld + v0;   // (no branch between the loads)
#pragma unroll
            for (int k = 0; k < NC; ++k)   // (ld is a multiple of 8: in bounds)
                u[r][k] = *(const uint4*)(in + min((k * ET + tid) * E, (nv - 1) & ~(E - 1)));
        }
        if (a.e.allow) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int m = min(g + r, m1 - 1), id = __builtin_amdgcn_readlane(masks, (m - m0) & 63), len = length(m);
                const bool in = id >= 0 && id < a.e.n_allow, every = !in || len < 0;
                if (!in && id != -1 && len >= 0 && a.err && tid == 0 && blockIdx.x == 0) atomicOr(a.err, DD_DEVERR_MASK);
                const uint32_t* allow = a.e.allow + (in ? (int64_t)id * a.e.ld_allow : 0);
#pragma unroll
                for (int k = 0; k < NC; ++k) {
                    const int v = v0 + min((k * ET + tid) * E, (nv - 1) & ~(E - 1));
                    ok[r][k] = (allow[v >> 5] | (every ? 0xFFFFFFFFu : 0u)) >> (v & 31);
                }
            }
        }
        if (lists) {
            const int mine = __shfl(lens, (g - m0 + tid) & 63, 64);
            if (tid < nr) entries[tid] = mine;
            // rows r .. q - 1 at a time whose histories are the first one's with a few more entries each
            for (int r = 0; r < nr;) {
                const int s = (g + r) / a.per, n = length(g + r);
                int q = r + 1, last = n;
                for (; q < nr && n >= 0 && (g + q) / a.per == s; ++q) {
                    const int t = length(g + q);
                    if (t < last || t - n > MORE) break;
                    last = t;
                }
                const int more = last - n;
                if (n >= 0 && (s != seq || n < have)) {
                    __syncthreads();         // the last rows' edits
                    for (int i = tid; i < EC / 4; i += ET) {
                        ((uint4*)count)[i] = make_uint4(0u, 0u, 0u, 0u);
                        ((uint4*)bias)[i] = make_uint4(0u, 0u, 0u, 0u);
                    }
                    if (tid < EC / 32) some[tid] = 0u;
                    if (tid == 0) listed = 0;
                    __syncthreads();
                    if (biased) {
                        for (int i = tid; i < a.e.n_bias; i += ET) {
                            const uint32_t v = (uint32_t)a.e.bias_ids[(int64_t)s * a.e.n_bias + i] - (uint32_t)v0;
                            if (v < (uint32_t)nv) {
                                atomicMax(&bias[v], (uint32_t)i + 1u);
                                add(v);
                            }
                        }
                        __syncthreads();
                        for (int i = tid, e = listed; i < e; i += ET) {
                            const int c = list[i];
                            bias[c] = __float_as_uint(a.e.bias_values[(int64_t)s * a.e.n_bias + (bias[c] - 1u)]);
                        }
                    }
                    rep = a.e.repetition ? a.e.repetition[s] : 1.f;
                    pres = a.e.presence ? a.e.presence[s] : 0.f;
                    freq = a.e.frequency ? a.e.frequency[s] : 0.f;
                    seq = s;
                    have = 0;
                }
                if (n > have) {
                    __syncthreads();         // the last rows' edits, the biases
                    for (int i = have + tid; i < n; i += ET) {
                        const uint32_t v = (uint32_t)a.e.history[(int64_t)s * a.e.ld_history + i] - (uint32_t)v0;
                        if (v < (uint32_t)nv) {
                            atomicAdd(&count[v], 1u);
                            add(v);
                        }
                    }
                    have = n;
                }
                if (more > 0) {
                    if (r > 0 || n == 0) __syncthreads();   // the last rows' edits; the biases, where no entry was counted
                    if (tid < more) {
                        const uint32_t v = (uint32_t)a.e.history[(int64_t)s * a.e.ld_history + n + tid] - (uint32_t)v0;
                        extra[tid] = (uint16_t)(v < (uint32_t)nv ? v : EC);
                        if (v < (uint32_t)nv) add(v);
                    }
                }
                if (r == 0) {
#pragma unroll
                    for (int i = 0; i < R; ++i)
#pragma unroll
                        for (int k = 0; k < NC; ++k) *(uint4*)&piece[i][(k * ET + tid) * E] = u[i][k];
                }
                __syncthreads();
                const int nl = n >= 0 ? listed : 0;
                for (int i = tid; i < nl * (q - r); i += ET) {
                    const int x = i / nl, c = list[i - x * nl];
                    T* p = &piece[r + x][c];
                    float y = Elem<T>::load1(p, 0);
                    uint32_t k = count[c];
                    if (more > 0)
                        for (int e = 0, t = entries[r + x] - n; e < t; ++e) k += extra[e] == c;
                    if (k) y = (y > 0.f ? y / rep : y * rep) - (pres + (float)k * freq);
                    store_one<T>(p, y + __uint_as_float(bias[c]));
                }
                if (more > 0) {
                    __syncthreads();
                    if (tid < more && extra[tid] < EC) atomicAdd(&count[extra[tid]], 1u);
                    have = last;
                }
                r = q;
            }
            __syncthreads();
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r >= nr) continue;
            T* out = (T*)a.out + (int64_t)(g + r) * a.ld + v0;
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                const int c = (k * ET + tid) * E;
                if (c >= nv) continue;
                uint4 x = u[r][k];
                if (lists) x = *(const uint4*)&piece[r][c];
                if (a.e.allow) mask_chunk<T>(x, ok[r][k]);
                if (c + E <= nv) {
                    *(uint4*)(out + c) = x;
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (c + e < nv) store_one<T>(out + c + e, Elem<T>::get(x, e));
                }
            }
        }
    }
}

template <typename T>
static void launch_edit_t(const EditArgs& a, dim3 grid, hipStream_t s) {
    constexpr int R = 4 * Elem<T>::E * ET / EC;   // 64 bytes in flight per thread
    if (a.rows_per_wg == 1) launch_k((logits_edit_kernel<T, 1>), grid, dim3(ET), 0, s, a);
    else if (a.rows_per_wg == 2) launch_k((logits_edit_kernel<T, 2>), grid, dim3(ET), 0, s, a);
    else launch_k((logits_edit_kernel<T, R>), grid, dim3(ET), 0, s, a);
}

dd_status launch_edit(const EditArgs& args, int dtype, hipStream_t s) {
    EditArgs a = args;
    const int64_t pieces = ceil_div(a.V, EC);
    // Rows of one sequence share their counts in a workgroup, as far as three workgroups per CU remain (64 rows: 8.7 us with
    // one each, 7.9 with two, 11.1 with eight; 4096 rows whose histories grow: 404 with one each, 183 with sixteen).
    a.rows_per_wg = (int)std::min<int64_t>(std::min<int64_t>(16, a.per), std::max<int64_t>(1, a.rows * pieces / 800));
    while (a.rows_per_wg & (a.rows_per_wg - 1)) a.rows_per_wg &= a.rows_per_wg - 1;   // whole groups of R
    if (ceil_div(a.rows, a.rows_per_wg) > 65535) a.rows_per_wg = (int)ceil_div(a.rows, 65535);
    const dim3 grid((unsigned)pieces, (unsigned)ceil_div(a.rows, a.rows_per_wg));
    ProfScope ps(KC_LOGITS_EDIT, s);
    if (dtype == DD_BF16) launch_edit_t<bf16_t>(a, grid, s);
    else launch_edit_t<float>(a, grid, s);
    return launch_status("logits_edit");
}

}  // namespace dd
