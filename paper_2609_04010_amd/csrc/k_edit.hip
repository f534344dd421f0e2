// Penalties for repeated tokens, biases and allowed-token masks on rows of logits.
//
// A workgroup owns a piece of EC classes and walks rows_per_wg rows: the counts of the history's tokens and
// the biases of its classes stand in LDS (whole numbers, so the order of the atomics does not show), and each
// row's piece is read, edited and written in one pass.  Rows of one sequence share their counts: a longer
// history adds its new entries, a shorter one (or another sequence) begins again.  Bound by the memory
// traffic of the logits.
#include <math.h>

#include <algorithm>

#include "cache.h"
#include "elem.h"

namespace dd {

constexpr int EC = 4096;   // classes of a workgroup: 32 KB of LDS, five workgroups per CU
constexpr int ET = 256;

template <typename T> DD_DEV void store_chunk(T* p, const float (&x)[Elem<T>::E]);
template <> DD_DEV void store_chunk<bf16_t>(bf16_t* p, const float (&x)[8]) {
    *(uint4*)p = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}
template <> DD_DEV void store_chunk<float>(float* p, const float (&x)[4]) { *(float4*)p = make_float4(x[0], x[1], x[2], x[3]); }
template <typename T> DD_DEV void store_one(T* p, float x);
template <> DD_DEV void store_one<bf16_t>(bf16_t* p, float x) { *p = f32_to_bf16(x); }
template <> DD_DEV void store_one<float>(float* p, float x) { *p = x; }

template <typename T>
__global__ __launch_bounds__(ET) void logits_edit_kernel(EditArgs a) {
    constexpr int E = Elem<T>::E;
    __shared__ __attribute__((aligned(16))) uint32_t count[EC];   // how often the class stands in the history
    __shared__ __attribute__((aligned(16))) uint32_t bias[EC];    // 1 + the last entry of the bias list that names it
    const int tid = threadIdx.x;
    const int v0 = blockIdx.x * EC, nv = min(EC, a.V - v0);
    const int m0 = blockIdx.y * a.rows_per_wg, m1 = min(m0 + a.rows_per_wg, a.rows);
    const bool hist = a.e.history || a.e.hist_len, biased = a.e.bias_ids != nullptr && a.e.n_bias > 0;
    int seq = -1, have = 0;   // sequence whose tables stand in LDS, entries counted
    float rep = 1.f, pres = 0.f, freq = 0.f;
    for (int m = m0; m < m1; ++m) {
        const int s = m / a.per;
        int len = 0;
        if (hist) {
            const int64_t n = a.e.hist_len ? a.e.hist_len[m] : a.e.ld_history;
            len = (int)(n < a.e.ld_history ? n : a.e.ld_history);
        }
        const bool pass = len < 0;   // the row goes through as it is
        if (!pass && (s != seq || len < have)) {
            __syncthreads();         // the last row's readers
            for (int i = tid; i < EC / 4; i += ET) {
                ((uint4*)count)[i] = make_uint4(0u, 0u, 0u, 0u);
                if (s != seq) ((uint4*)bias)[i] = make_uint4(0u, 0u, 0u, 0u);
            }
            __syncthreads();
            if (s != seq && biased)
                for (int i = tid; i < a.e.n_bias; i += ET) {
                    const uint32_t v = (uint32_t)a.e.bias_ids[(int64_t)s * a.e.n_bias + i] - (uint32_t)v0;
                    if (v < (uint32_t)nv) atomicMax(&bias[v], (uint32_t)i + 1u);
                }
            if (s != seq) {
                rep = a.e.repetition ? a.e.repetition[s] : 1.f;
                pres = a.e.presence ? a.e.presence[s] : 0.f;
                freq = a.e.frequency ? a.e.frequency[s] : 0.f;
            }
            seq = s;
            have = 0;
            if (len == 0) __syncthreads();
        }
        if (!pass && len > have) {
            __syncthreads();
            for (int i = have + tid; i < len; i += ET) {
                const uint32_t v = (uint32_t)a.e.history[(int64_t)s * a.e.ld_history + i] - (uint32_t)v0;
                if (v < (uint32_t)nv) atomicAdd(&count[v], 1u);
            }
            have = len;
            __syncthreads();
        }
        const uint32_t* allow = nullptr;
        if (!pass && a.e.allow) {
            const int id = a.e.allow_id ? a.e.allow_id[m] : 0;
            if (id >= 0 && id < a.e.n_allow) allow = a.e.allow + (int64_t)id * a.e.ld_allow;
            else if (id != -1 && a.err && tid == 0 && blockIdx.x == 0) atomicOr(a.err, DD_DEVERR_MASK);
        }
        const T* in = (const T*)a.logits + (int64_t)m * a.ld + v0;
        T* out = (T*)a.out + (int64_t)m * a.ld + v0;
        for (int c = tid * E; c < nv; c += ET * E) {
            const uint4 u = *(const uint4*)(in + c);   // ld is a multiple of 8: in bounds
            float x[E];
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = Elem<T>::get(u, e);
            if (!pass) {
                uint32_t n[E], b[E];
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const uint4 k = *(const uint4*)&count[c + e], w = *(const uint4*)&bias[c + e];
                    n[e] = k.x; n[e + 1] = k.y; n[e + 2] = k.z; n[e + 3] = k.w;
                    b[e] = w.x; b[e + 1] = w.y; b[e + 2] = w.z; b[e + 3] = w.w;
                }
                uint32_t ok = 0xFFu;
                if (allow) ok = allow[(v0 + c) >> 5] >> ((v0 + c) & 31);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if (n[e]) x[e] = (x[e] > 0.f ? x[e] / rep : x[e] * rep) - (pres + (float)n[e] * freq);
                    if (b[e]) x[e] += a.e.bias_values[(int64_t)s * a.e.n_bias + (b[e] - 1u)];
                    if (!(ok >> e & 1u)) x[e] = -INFINITY;
                }
            }
            if (c + E <= nv) {
                store_chunk<T>(out + c, x);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (c + e < nv) store_one<T>(out + c + e, x[e]);
            }
        }
    }
}

dd_status launch_edit(const EditArgs& args, int dtype, hipStream_t s) {
    EditArgs a = args;
    const int64_t pieces = ceil_div(a.V, EC);
    // rows of one sequence share their counts in a workgroup, as far as 4096 workgroups (16 per CU) remain
    a.rows_per_wg = (int)std::min<int64_t>(16, std::max<int64_t>(1, a.rows * pieces / 4096));
    a.rows_per_wg = (int)std::min<int64_t>(a.rows_per_wg, a.per);
    if (ceil_div(a.rows, a.rows_per_wg) > 65535) a.rows_per_wg = (int)ceil_div(a.rows, 65535);
    const dim3 grid((unsigned)pieces, (unsigned)ceil_div(a.rows, a.rows_per_wg));
    ProfScope ps(KC_LOGITS_EDIT, s);
    if (dtype == DD_BF16) launch_k(logits_edit_kernel<bf16_t>, grid, dim3(ET), 0, s, a);
    else launch_k(logits_edit_kernel<float>, grid, dim3(ET), 0, s, a);
    return launch_status("logits_edit");
}

}  // namespace dd
