// Attention over mixed sets by position: capped or biased logits, rows that a rule hides, and the weight that every row receives.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "vxl_mfma.h"
#include "vxl_mixed.h"

namespace vxl {

namespace {

// The rule as the kernels take it.  Logits are kept in units of log 2: y = x log2(e).
struct Rule {
    float c2;                  // scale log2(e)
    float cap_in, cap2;        // scale / softcap, softcap log2(e); cap2 == 0: no cap
    int causal, window, n_always;
    const float* slopes;
    const int32_t *q_pos, *row_pos;
};

// Rows that a token sees: positions lo .. hi and 0 .. na - 1.  A padding token: none.  (Without positions every row of the set has
// position 0 and every token sees it.)
struct Span {
    int lo, hi;
    unsigned na;
};
__device__ __forceinline__ Span span_of(const Rule& r, int pq) {
    if (!r.q_pos) return {0, 0, 0u};
    if (pq < 0) return {1, 0, 0u};
    return {r.window ? max(pq - r.window + 1, 0) : 0, r.causal ? pq : INT32_MAX, (unsigned)r.n_always};
}
__device__ __forceinline__ bool sees(const Span& s, int pk) { return (pk >= s.lo && pk <= s.hi) || (unsigned)pk < s.na; }

// Sets as the kernels see them.
struct Sets {
    const void *q, *k, *v;
    const int32_t* len;
    int T, n_q, n_kv, cap;
};

// ------------------------------------------------------------------------------------------
// Row by row: one wave, a key per lane for the logits and a column per lane for O, in fp32, over the rows that the token sees and no
// others.  The cross-check of the matrix-core kernels.
// ------------------------------------------------------------------------------------------
template <typename T, int D>
__device__ __forceinline__ float dot_row(const float* q, const T* k) {
    constexpr int VEC = 16 / sizeof(T);
    float a = 0.f;
#pragma unroll 4
    for (int d = 0; d < D; d += VEC) {
        T x[VEC];
        *(uint4*)x = *(const uint4*)(k + d);
#pragma unroll
        for (int j = 0; j < VEC; ++j) a = fmaf(q[d + j], as_float(x[j]), a);
    }
    return a;
}

__device__ __forceinline__ float exact_logit(const Rule& r, float dot, float slope2, int pq, int pk) {
    float y = r.cap2 > 0.f ? r.cap2 * tanhf(dot * r.cap_in) : dot * r.c2;
    if (slope2 != 0.f) y = fmaf(-slope2, (float)abs(pq - pk), y);
    return y;
}

template <typename T, int D>
__device__ __forceinline__ void exact_row(const Rule& r, const float* q, const T* k, const T* v, const int32_t* pos, int lo, int hi, int pq,
                                          float slope2, float& m, float& l, float (&acc)[D / 64]) {
    const int lane = threadIdx.x & 63;
    const Span span = span_of(r, pq);
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int x = 0; x < D / 64; ++x) acc[x] = 0.f;
    for (int base = lo; base < hi; base += 64) {
        const int row = base + lane;
        const int pk = row < hi ? (pos ? pos[row] : 0) : -1;
        float y = -INFINITY;
        if (sees(span, pk)) y = exact_logit(r, dot_row<T, D>(q, k + (size_t)row * D), slope2, pq, pk);
        float m_new = y;
        for (int o = 32; o > 0; o >>= 1) m_new = fmaxf(m_new, __shfl_xor(m_new, o));
        m_new = fmaxf(m_new, m);
        const float ref = m_new == -INFINITY ? 0.f : m_new, alpha = exp2f(m - ref), p = exp2f(y - ref);
        float sum = p;
        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
        m = m_new;
        l = l * alpha + sum;
#pragma unroll
        for (int x = 0; x < D / 64; ++x) acc[x] = acc[x] == 0.f ? 0.f : acc[x] * alpha;
        for (int j = 0; j < 64; ++j) {
            const float pj = __shfl(p, j);
            if (pj == 0.f) continue;
            const T* vr = v + (size_t)(base + j) * D;
#pragma unroll
            for (int x = 0; x < D / 64; ++x) acc[x] = fmaf(pj, as_float(vr[lane + 64 * x]), acc[x]);
        }
    }
}

__device__ __forceinline__ float slope_of(const Rule& r, int h) { return r.slopes ? r.slopes[h] * kLog2e : 0.f; }

template <bool F32, int D>
__global__ __launch_bounds__(256) void simple_attend_kernel(Sets s, Rule r, void* O, float* LSE, float* lse2, long long n_rows) {
    using T = typename Storage<F32>::T;
    __shared__ __attribute__((aligned(16))) float q_lds[4][D];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long row = (long long)folded_id() * 4 + wave;   // (query, token, head)
    if (row >= n_rows) return;
    const int h = (int)(row % s.n_q), t = (int)(row / s.n_q % s.T), b = (int)(row / s.n_q / s.T), group = s.n_q / s.n_kv, g = h / group;
#pragma unroll
    for (int x = 0; x < D / 64; ++x) q_lds[wave][lane + 64 * x] = as_float(((const T*)s.q)[row * D + lane + 64 * x]);
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    const int len = min(max(s.len[b], 0), s.cap), pq = r.q_pos ? r.q_pos[b * s.T + t] : 0;
    const size_t set = ((size_t)b * s.n_kv + g) * s.cap;
    float m, l, acc[D / 64];
    exact_row<T, D>(r, q_lds[wave], (const T*)s.k + set * D, (const T*)s.v + set * D, r.row_pos ? r.row_pos + set : nullptr, 0, len, pq,
                    slope_of(r, h), m, l, acc);
#pragma unroll
    for (int x = 0; x < D / 64; ++x) store_as((T*)O + row * D + lane + 64 * x, l == 0.f ? 0.f : acc[x] / l);
    if (lane == 0) {
        const float y = l == 0.f ? -INFINITY : m + log2f(l);
        if (LSE) LSE[row] = y * kLn2;
        lse2[(((size_t)b * s.n_kv + g) * s.T + t) * group + h % group] = y;
    }
}

// Weights: a row of the set per lane, which goes over the query rows of its KV head in order.
template <bool F32, int D>
__global__ __launch_bounds__(256) void simple_weights_kernel(Sets s, Rule r, const float* lse2, const float* weight, float* weight_out) {
    using T = typename Storage<F32>::T;
    __shared__ __attribute__((aligned(16))) float q_lds[D];
    const int g = blockIdx.y % s.n_kv, b = blockIdx.y / s.n_kv, group = s.n_q / s.n_kv;
    const int len = min(max(s.len[b], 0), s.cap);
    if ((int)blockIdx.x * 256 >= len) return;
    const int row = blockIdx.x * 256 + threadIdx.x;
    const size_t set = ((size_t)b * s.n_kv + g) * s.cap;
    const int pk = row < len ? (r.row_pos ? r.row_pos[set + row] : 0) : -1;
    const T* k = (const T*)s.k + (set + min(row, len - 1)) * D;
    float w = 0.f;
    for (int t = 0; t < s.T; ++t) {
        const int pq = r.q_pos ? r.q_pos[b * s.T + t] : 0;
        const Span span = span_of(r, pq);
        for (int hg = 0; hg < group; ++hg) {
            const size_t q_row = ((size_t)b * s.T + t) * s.n_q + g * group + hg;
            __syncthreads();
            if (threadIdx.x < D) q_lds[threadIdx.x] = as_float(((const T*)s.q)[q_row * D + threadIdx.x]);
            __syncthreads();
            const float lse = lse2[(((size_t)b * s.n_kv + g) * s.T + t) * group + hg];
            if (lse == -INFINITY || !sees(span, pk)) continue;
            w += exp2f(exact_logit(r, dot_row<T, D>(q_lds, k), slope_of(r, g * group + hg), pq, pk) - lse);
        }
    }
    if (row < len) weight_out[set + row] = (weight ? weight[set + row] : 0.f) + w;
}

}  // namespace

MixedPlan mixed_plan(const vxl_attn_desc* d, int batch, int T, int l_cap) {
    MixedPlan p{};
    const long long rows = (long long)(d->n_q_heads / d->n_kv_heads) * T, units = (long long)batch * d->n_kv_heads;
    p.fits = units <= 65535 && rows <= 1 << 30;
    if (!p.fits) return p;
    p.lse2 = 0;
    p.total = align_up((size_t)units * rows * sizeof(float), 256);
    return p;
}

vxl_status launch_mixed_attend(const MixedPlan& p, const MixedCall& c, bool force_simple, hipStream_t s) {
    const vxl_attn_desc* d = c.d;
    const vxl_score_rule none{};
    const vxl_score_rule& u = c.rule ? *c.rule : none;
    const Rule rule{c.scale * kLog2e, u.softcap > 0.f ? c.scale / u.softcap : 0.f, u.softcap * kLog2e, u.causal, u.window, u.n_always, u.slopes,
                    c.q_pos, c.row_pos};
    const Sets sets{c.Qd, c.Kmix, c.Vmix, c.mix_len, c.T, d->n_q_heads, d->n_kv_heads, c.l_cap};
    const long long n_rows = (long long)c.batch * c.T * d->n_q_heads;
    float* lse2 = (float*)(c.ws + p.lse2);
    return by_storage(d, [&](auto f32, auto dim) {
        hipLaunchKernelGGL((simple_attend_kernel<f32, dim>), folded_grid((n_rows + 3) / 4), dim3(256), 0, s, sets, rule, c.O, c.LSE, lse2, n_rows);
        vxl_status st = mixed_launched();
        if (st != VXL_OK || !c.weight_out) return st;
        hipLaunchKernelGGL((simple_weights_kernel<f32, dim>), dim3((c.l_cap + 255) / 256, c.batch * d->n_kv_heads), dim3(256), 0, s, sets, rule,
                           lse2, c.weight, c.weight_out);
        return mixed_launched();
    });
}

}  // namespace vxl
