// Attention over mixed sets by position: capped or biased logits, rows that a rule hides, and the weight that every row receives.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <limits>
#include <type_traits>

#include "vxl_mfma.h"
#include "vxl_mixed.h"

namespace vxl {

namespace {

// The rule as the kernels take it.  Logits are kept in units of log 2: y = x log2(e).
struct Rule {
    float c2;                  // scale log2(e)
    float cap_in, cap2;        // scale / softcap, softcap log2(e); cap2 == 0: no cap
    float cap_few, cap_k[3];   // (cap_logits) below which products the series holds, its coefficients,
    float cap_exp, cap_m2;     // 2 log2(e) scale / softcap, -2 cap2
    int causal, window, n_always;
    const float* slopes;
    const int32_t *q_pos, *row_pos;
};

// Rows that a token sees: positions lo .. lo + width - 1 and 0 .. na - 1.  A padding token: none.  (Without positions every row of the set
// has position 0 and every token sees it.)
struct Span {
    int lo;
    unsigned width, na;
    __device__ __forceinline__ int hi() const { return (int)((unsigned)lo + width - 1u); }       // (of one that is not empty)
};
__device__ __forceinline__ Span span_of(const Rule& r, int pq) {
    if (!r.q_pos) return {0, 1u, 0u};
    if (pq < 0) return {0, 0u, 0u};
    const int lo = r.window ? max(pq - r.window + 1, 0) : 0, hi = r.causal ? pq : INT32_MAX;
    return {lo, (unsigned)hi - (unsigned)lo + 1u, (unsigned)r.n_always};
}
// (A negative position is 2^31 or more as it is and with lo taken off.)
__device__ __forceinline__ bool sees(const Span& s, int pk) { return ((unsigned)pk - (unsigned)s.lo < s.width) | ((unsigned)pk < s.na); }
// A logit, or -inf where it is hidden; FIRST: there may be an na.  Selections one after the other: comparisons that are joined go through
// scalar registers and wait for them.
template <bool FIRST>
__device__ __forceinline__ float shown(const Span& s, int pk, float y) {
    float z = (unsigned)pk - (unsigned)s.lo < s.width ? y : -INFINITY;
    if constexpr (FIRST) z = (unsigned)pk < s.na ? y : z;
    return z;
}

// Sets as the kernels see them.
struct Sets {
    const void *q, *k, *v;
    const int32_t* len;
    int T, n_q, n_kv, cap;
};

// ------------------------------------------------------------------------------------------
// Row by row: one wave, a key per lane for the logits and a column per lane for O, in fp32, over the rows that the token sees and no
// others.  The cross-check of the matrix-core kernels, and what makes a row again that they cannot (exact_row).
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

// (rows [lo, hi), `width` <= 64 of every `step`)
template <typename T, int D>
__device__ __forceinline__ void exact_row(const Rule& r, const float* q, const T* k, const T* v, const int32_t* pos, int lo, int hi, int width,
                                          int step, int pq, float slope2, float& m, float& l, float (&acc)[D / 64]) {
    const int lane = threadIdx.x & 63;
    const Span span = span_of(r, pq);
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int x = 0; x < D / 64; ++x) acc[x] = 0.f;
    for (int base = lo; base < hi; base += step) {
        const int row = base + lane;
        const int pk = row < hi && lane < width ? (pos ? pos[row] : 0) : -1;
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
        for (int j = 0; j < width; ++j) {
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
    exact_row<T, D>(r, q_lds[wave], (const T*)s.k + set * D, (const T*)s.v + set * D, r.row_pos ? r.row_pos + set : nullptr, 0, len, 64, 64, pq,
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

// ------------------------------------------------------------------------------------------
// Many stacked query rows (rho = t * G + head of the group): 32 per wave, NW waves per workgroup; the 64-key tiles of the workgroup's split
// stream through a ring of four LDS stages by direct loads, two tiles ahead of the arithmetic, as in the plain decode's ring, whose
// products and layouts these are.  What a rule adds:
//   * The positions of a tile come with it, by one wave's load.  A lane has a key's; against the range of positions that the wave's 32 rows
//     see, a ballot each tells a tile that none sees (skipped), one that all see (nothing more) and one that needs a test per element;
//     only then, and for a bias, a lane reads the positions of its elements.
//   * The second product takes its weights in bf16, as the plain decode's does (each off by 2^-8 of it at most, what the rounding of a
//     value or of a result is; the fp32 instruction has a 1/16 of the rate).  Sums are of the weights as they are, so that LSE and row
//     weights have fp32's error.
//   * A value that is not a number reaches rows that do not see it, 0 * inf: a row whose result is none is made again by exact_row.
// Bound by the matrix instructions, and with a cap by the vector ones.  In replayed graphs (boxes differ by some 5 %), 2,048 tokens of 28
// heads on 4 over 18,688 rows, 519 GFLOP of products: 540 us, 0.96 PFLOP/s where a library product of 8192^3 reaches 1.24; 64 tokens over
// 23,872 rows, with the merge of the splits: 43 us, capped 48 (52 by the exponential).  128 and 256 rows a workgroup: see ring_plan.
// ------------------------------------------------------------------------------------------
constexpr float kLowest = -std::numeric_limits<float>::max();

template <int D, int NW>
struct RingCfg {
    static constexpr int NS = 4, ROWS = 32 * NW, TILE = kKeyTile * D, STAGE = 2 * TILE;        // elements
    static constexpr int PPR = D / 8, RPI = 64 / PPR, IPW = kKeyTile / RPI / NW;               // pieces of a row; rows, loads of a wave
    static constexpr int POS_AT = NS * STAGE * 2, LDS_BYTES = POS_AT + NS * kKeyTile * 4;      // bytes: the positions behind the stages
};

// What kernels that cut the keys leave for the merge: unnormalised O, and per row the reference (base 2) and the sum.
struct Partials {
    float* o;                  // [unit][split][rows][D]
    float2* ml;                // [unit][split][rows]
};

// Workgroups that read the same keys are neighbours on one XCD (workgroups go to the XCDs in turn): grid.x = XCDs.
__device__ __forceinline__ bool place(int units, int n_split, int n_rtile, int* unit, int* split, int* rtile) {
    const unsigned all = (unsigned)(units * n_split * n_rtile), each = (all + gridDim.x - 1) / gridDim.x;
    const unsigned own = blockIdx.z * gridDim.y + blockIdx.y, id = blockIdx.x * each + own;
    if (own >= each || id >= all) return false;
    *rtile = (int)(id % n_rtile);
    *split = (int)(id / n_rtile % n_split);
    *unit = (int)(id / n_rtile / n_split);
    return true;
}

// The positions that the 32 rows of a wave see, at most and at least.
struct Reach {
    Span most, least;
    __device__ __forceinline__ void of(const Span& s) {
        int lo = s.width ? s.lo : INT32_MAX, hi = s.width ? s.hi() : -1, lo_most = lo, hi_least = hi;
        unsigned na = s.na, na_least = s.na;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            lo = min(lo, __shfl_xor(lo, o));
            hi = max(hi, __shfl_xor(hi, o));
            na = max(na, (unsigned)__shfl_xor((int)na, o));
            lo_most = max(lo_most, __shfl_xor(lo_most, o));
            hi_least = min(hi_least, __shfl_xor(hi_least, o));
            na_least = min(na_least, (unsigned)__shfl_xor((int)na_least, o));
        }
        most = {lo, hi >= lo ? (unsigned)hi - (unsigned)lo + 1u : 0u, na};
        least = {lo_most, hi_least >= lo_most ? (unsigned)hi_least - (unsigned)lo_most + 1u : 0u, na_least};
    }
};

// From products s to softcap tanh(u), u = s scale / softcap, in units of log 2; one decision for the wave's elements that are seen.  What
// the others are has no part in it: in a tile seen in part, where some element is not small, largest_seen(x), the largest magnitude of a
// lane's seen ones, decides (64 tokens over 23,872 rows, all tiles in part: 4 % more with a cap of 50, 14 % with one of 5).
//   * All |u| < 1/8, as with caps of 30 and more: the odd series to u^7 (the next term is 1.3e-9 of it there) in the product itself, its
//     coefficients with the powers of scale / softcap in them, so that u is not made.
//   * Else 1 - 2 / (e^2|u| + 1) with the sign of s, off by 4 roundings of the cap at most: the exponential, the sum and the quotient by one
//     each of less than the cap, the argument by less than half a one.  That is the error of LSE and row weights too: 9e-6 at most of a
//     logit below a quarter of a cap of 50, where an fp32 tanh has 2e-6.
// The series to u^13 for all |u| < 0.4 is no faster, and both with a selection, exact to a rounding of the result, took 63 us where the
// exponential took 48 (the ring alone, 64 tokens over 23,872 rows, a cap of 5).
template <int N, typename F>
__device__ __forceinline__ void cap_logits(float (&x)[N], const Rule& r, bool all_seen, F&& largest_seen) {
    float top = 0.f;                                          // (NaN is NaN either way)
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, fabsf(x[i]));
    bool small = __builtin_amdgcn_ballot_w64(!(top < r.cap_few)) == 0;
    if (!small && !all_seen) small = __builtin_amdgcn_ballot_w64(!(largest_seen(x) < r.cap_few)) == 0;
    if (small) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float z = x[i] * x[i], y = x[i] * r.c2;
            x[i] = fmaf(y, z * fmaf(fmaf(r.cap_k[2], z, r.cap_k[1]), z, r.cap_k[0]), y);     // (y z may be no number: z is up to 2^108)
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float q = __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(fabsf(x[i] * r.cap_exp)) + 1.f);
            x[i] = copysignf(fmaf(r.cap_m2, q, r.cap2), x[i]);
            if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);               // (four at a time: all at once need more registers than there are)
        }
    }
}

// Of a token's products with 32 keys, as a lane has them, the largest magnitude of those with keys of a position that it sees.
__device__ __forceinline__ float largest_of(const Span& span, int n_always, const int32_t* pos, int hi, const float (&x)[16]) {
    auto of = [&](auto first) __attribute__((always_inline)) {
        float top = 0.f;
#pragma unroll
        for (int rq = 0; rq < 4; ++rq) {
            const int4 p4 = *(const int4*)(pos + rq * 8 + hi * 4);
            const int p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, shown<first>(span, p[i], fabsf(x[rq * 4 + i])));
        }
        return top;
    };
    return n_always > 0 ? of(std::true_type{}) : of(std::false_type{});
}

template <int D, int NW, bool POS>
__global__ __launch_bounds__(64 * NW, 2) void attend_ring_kernel(Sets s, Rule r, Partials part, uint16_t* __restrict__ O, float* __restrict__ LSE,
                                                                 float* __restrict__ lse2, int units, int n_split, int n_rtile) {
    using C = RingCfg<D, NW>;
    extern __shared__ __attribute__((aligned(16))) uint16_t lds[];
    __shared__ __attribute__((aligned(16))) float q_lds[NW][D];          // (of rows made again)
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
    const int lane = threadIdx.x & 63, l32 = lane & 31, hi = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int unit, split, rtile;
    if (!place(units, n_split, n_rtile, &unit, &split, &rtile)) return;
    const int g = unit % s.n_kv, b = unit / s.n_kv, group = s.n_q / s.n_kv, n_rows = group * s.T;
    const int len = __builtin_amdgcn_readfirstlane(min(max(s.len[b], 0), s.cap));
    // the split's tiles: an even share of the set's
    const int tiles = (len + kKeyTile - 1) / kKeyTile, share = tiles / n_split, more = tiles % n_split;
    const int tile0 = split * share + min(split, more), n_t = share + (split < more ? 1 : 0);
    const int k_lo = tile0 * kKeyTile, k_hi = min((tile0 + n_t) * kKeyTile, len);
    const int wrow0 = rtile * C::ROWS + wave * 32;
    const bool wave_active = wrow0 < n_rows;                  // (waves without rows only help with the loads)
    const size_t set = (size_t)unit * s.cap;
    const uint16_t *kset = (const uint16_t*)s.k + set * D, *vset = (const uint16_t*)s.v + set * D;
    const char *kbase = (const char*)(kset + (size_t)k_lo * D), *vbase = (const char*)(vset + (size_t)k_lo * D);
    const int32_t* pos = POS ? r.row_pos + set : nullptr;
    const int r_in = lane / C::PPR, pp = lane % C::PPR;

    // Tile t -> stage t % NS; rows past the end of the split are its last row (masked, and V a value that counts).
    auto issue = [&](int t) __attribute__((always_inline)) {
        const int row0 = t * kKeyTile, rlim = min(kKeyTile - 1, k_hi - k_lo - 1 - row0);
        const char *kb = kbase + (size_t)row0 * (D * 2), *vb = vbase + (size_t)row0 * (D * 2);
        const uint32_t st = lds_base + (uint32_t)(t % C::NS) * (C::STAGE * 2);
#pragma unroll
        for (int i = 0; i < C::IPW; ++i) {
            const int slot = wave + i * NW, row = slot * C::RPI + r_in;
            const int kp = pp ^ ((row / (16 / C::PPR)) & (C::PPR - 1));
            constexpr int CPR = D * 2 / 64, RPL = D == 128 ? 1 : 2;
            const int vp = (((pp >> 2) ^ ((row / RPL) & (CPR - 1))) << 2) | (pp & 3);
            const uint32_t roff = (uint32_t)min(row, rlim) * (D * 2);
            dma16(kb, roff + kp * 16, st + slot * 1024);
            dma16(vb, roff + vp * 16, st + C::TILE * 2 + slot * 1024);
        }
        if (POS && wave == 0)
            dma4(pos + k_lo + row0, (uint32_t)min(lane, rlim) * 4, lds_base + C::POS_AT + (uint32_t)(t % C::NS) * (kKeyTile * 4));
    };
    if (n_t > 0) {
        issue(0);
        issue(min(1, n_t - 1));
    }
    const int rho = min(wrow0 + l32, n_rows - 1), tok = rho / group, h = g * group + rho % group;
    bf16x8 qreg[1][D / 16];
    {
        const uint4* src = (const uint4*)((const uint16_t*)s.q + (((size_t)b * s.T + tok) * s.n_q + h) * D);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) qreg[0][ks] = __builtin_bit_cast(bf16x8, src[ks * 2 + hi]);
    }
    const int pq = POS ? r.q_pos[b * s.T + tok] : 0;
    const Span span = span_of(r, pq);
    Reach reach;
    reach.of(span);
    const float slope2 = POS ? slope_of(r, h) : 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {                     // complete here: no load that the compiler counts is outstanding behind
        typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
        asm volatile("" :: "v"(__builtin_bit_cast(u32x4, qreg[0][ks])));
    }
    asm volatile("" :: "v"(pq), "v"(slope2));
    __builtin_amdgcn_sched_barrier(0);

    f32x16 o[1][D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) o[0][db] = zero16();
    const bool capped = r.cap2 > 0.f, biased = POS && r.slopes;
    const float cu = capped || biased ? 1.f : r.c2, unit_of = capped ? 1.f : r.c2;       // units of log 2 of x below; of what a bias is put to
    float m_run = -INFINITY, mc_run = kLowest, l_run = 0.f;

    auto process = [&](int ti) __attribute__((always_inline)) {
        if (!wave_active) return;
        const int left = k_hi - k_lo - ti * kKeyTile;
        bool partial = left < kKeyTile;
        const int32_t* tile_pos = (const int32_t*)((const char*)lds + C::POS_AT) + (ti % C::NS) * kKeyTile;
        if constexpr (POS) {
            const int pk = lane < left ? tile_pos[lane] : -1;
            if (__builtin_amdgcn_ballot_w64(sees(reach.most, pk)) == 0) return;
            partial = ~__builtin_amdgcn_ballot_w64(sees(reach.least, pk)) != 0;
        }
        const uint16_t* kt = lds + (ti % C::NS) * C::STAGE;
        f32x16 x[1][2];
        if constexpr (NW == 4) qk_tile_ahead<D, 1>(kt, qreg, l32, hi, x);
        else qk_tile<D, 1>(kt, qreg, l32, hi, x);
        if (capped) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                float c[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) c[i] = x[0][kb][i];
                cap_logits(c, r, !POS || !partial, [&](const float (&y)[16]) __attribute__((always_inline)) {
                    return largest_of(span, r.n_always, tile_pos + kb * 32, hi, y);
                });
#pragma unroll
                for (int i = 0; i < 16; ++i) x[0][kb][i] = c[i];
            }
        }
        if constexpr (POS) {
            auto by_position = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int rq = 0; rq < 4; ++rq) {
                        const int4 p4 = *(const int4*)(tile_pos + kb * 32 + rq * 8 + hi * 4);
                        const int p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[0][kb][rq * 4 + i] = f(x[0][kb][rq * 4 + i], p[i], acc_key(kb, rq * 4 + i, hi));
                    }
            };
            if (biased) by_position([&](float y, int p, int) { return fmaf(-slope2, (float)abs(pq - p), y * unit_of); });
            if (partial) {
                if (r.n_always > 0) by_position([&](float y, int p, int) { return shown<true>(span, p, y); });
                else by_position([&](float y, int p, int) { return shown<false>(span, p, y); });
                if (left < kKeyTile) by_position([&](float y, int, int key) { return key < left ? y : -INFINITY; });
            }
        } else if (partial) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[0][kb][i] = acc_key(kb, i, hi) < left ? x[0][kb][i] : -INFINITY;
        }
        // The reference is raised, and sums and O rescaled, only when a logit is more than 2^8 above it.
        float top = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, x[0][kb][i]);
        if (__builtin_amdgcn_ballot_w64(fmaf(top, cu, -mc_run) > 8.f) != 0) {
            const float m_new = fmaxf(m_run, fmaxf(top, __shfl_xor(top, 32)));
            const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m_run - m_new) * cu);
            l_run *= alpha;
            m_run = m_new;
            mc_run = fmaxf(m_new * cu, kLowest);
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[0][db][i] *= alpha;
        }
        bf16x8 pb[1][2][2];
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float p = __builtin_amdgcn_exp2f(fmaf(x[0][kb][i], cu, -mc_run));
                sum[i & 1] += p;
                pb[0][kb][i >> 3][i & 7] = (__bf16)p;
            }
        l_run += sum[0] + sum[1];
        if constexpr (NW == 4) pv_tile_ahead<D, 2>(kt + C::TILE, pb, lane, o);
        else pv_tile<D, 1>(kt + C::TILE, pb, lane, o);
    };
    for (int t0 = 0; t0 < n_t; t0 += 2) {
        wait_vmcnt<0>();                                      // this wave's parts of tiles t0, t0 + 1 have landed
        __builtin_amdgcn_s_barrier();                         // ... and everyone's; the other two stages are free
        issue(min(t0 + 2, n_t - 1));
        process(t0);
        issue(min(t0 + 3, n_t - 1));
        if (t0 + 1 < n_t) process(t0 + 1);
    }
    wait_vmcnt<0>();                                          // drain the refills before the wave ends

    if (!wave_active) return;
    const float l = l_run + __shfl_xor(l_run, 32);
    bool odd = false;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) odd |= !(fabsf(o[0][db][i]) < INFINITY);
    const bool there = wrow0 + l32 < n_rows;
    unsigned long long again = __builtin_amdgcn_ballot_w64(odd && there);
    again = (again | again >> 32) & 0xffffffffull;
    const size_t part_row0 = ((size_t)unit * n_split + split) * n_rows;
    if (there && !(again >> l32 & 1)) {
        const size_t out = ((size_t)b * s.T + tok) * s.n_q + h;
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int rq = 0; rq < 4; ++rq) {
                const int d = db * 32 + rq * 8 + hi * 4;
                const float v[4] = {o[0][db][rq * 4], o[0][db][rq * 4 + 1], o[0][db][rq * 4 + 2], o[0][db][rq * 4 + 3]};
                if (n_split > 1) {
                    *(float4*)(part.o + (part_row0 + rho) * D + d) = make_float4(v[0], v[1], v[2], v[3]);
                } else {
                    __attribute__((aligned(8))) const uint16_t x[4] = {f32_to_bf16(v[0] * inv), f32_to_bf16(v[1] * inv), f32_to_bf16(v[2] * inv),
                                                                       f32_to_bf16(v[3] * inv)};
                    *(uint2*)(O + out * D + d) = *(const uint2*)x;
                }
            }
        if (hi == 0) {
            if (n_split > 1) {
                part.ml[part_row0 + rho] = make_float2(l == 0.f ? -INFINITY : mc_run, l);
            } else {
                const float y = l == 0.f ? -INFINITY : mc_run + __builtin_amdgcn_logf(l);
                if (LSE) LSE[out] = y * kLn2;
                lse2[(size_t)unit * n_rows + rho] = y;
            }
        }
    }
    if (again == 0) return;
    float* q_row = q_lds[wave];
    while (again) {                                           // (uniform)
        const int row = wrow0 + __builtin_ctzll(again);
        again &= again - 1;
        const int t = row / group, hq = g * group + row % group;
        const size_t out = ((size_t)b * s.T + t) * s.n_q + hq;
        __builtin_amdgcn_wave_barrier();
        for (int x = lane; x < D; x += 64) q_row[x] = as_float(((const uint16_t*)s.q)[out * D + x]);
        __builtin_amdgcn_wave_barrier();
        float m, l2, acc[D / 64];
        exact_row<uint16_t, D>(r, q_row, kset, vset, r.row_pos ? r.row_pos + set : nullptr, k_lo, k_hi, 64, 64,
                               r.q_pos ? r.q_pos[b * s.T + t] : 0, slope_of(r, hq), m, l2, acc);
#pragma unroll
        for (int x = 0; x < D / 64; ++x) {
            if (n_split > 1) part.o[(part_row0 + row) * D + lane + 64 * x] = acc[x];
            else O[out * D + lane + 64 * x] = f32_to_bf16(l2 == 0.f ? 0.f : acc[x] / l2);
        }
        if (lane == 0) {
            if (n_split > 1) {
                part.ml[part_row0 + row] = make_float2(m, l2);
            } else {
                const float y = l2 == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(l2);
                if (LSE) LSE[out] = y * kLn2;
                lse2[(size_t)unit * n_rows + row] = y;
            }
        }
    }
}

// Of a part with reference and sum ml, against a reference: its weight in the whole, 0 if it has none, whatever it holds (and then nothing
// of it is added); 1 if its sum is not a number, which the whole then is not either.
__device__ __forceinline__ float part_weight(float2 ml, float ref) {
    return ml.y == 0.f ? 0.f : ml.y != ml.y ? 1.f : __builtin_amdgcn_exp2f(ml.x - ref);
}
__device__ __forceinline__ float add_part(float f, float x, float sum) { return f == 0.f ? sum : fmaf(f, x, sum); }

// ------------------------------------------------------------------------------------------
// At most 32 stacked query rows, the generated tokens: bound by memory, or by latency.  Every wave walks 32-key tiles of its own, in turn
// with the other waves of all splits, from two pairs of LDS areas filled by direct loads and counted by hand; the waves' (reference, sum,
// O) are merged through LDS.  The logits, in units of log 2, are kept in the workspace (4 bytes per query row and key beside 4 D of key and
// value), so that the weights need no second pass over the keys: -inf where the row is not seen, kLowest for a seen one of -inf.
// One token of eight queries, 28 heads on 4 of D = 128, sets of up to 18,177 rows, 120,138 together: 50 us for 252 MB of keys, values and
// numbers of rows, 5.0 TB/s, the rate of a copy (4.9); of one query and 4,097 rows 7.0, launch and three dependent trips to memory.
// ------------------------------------------------------------------------------------------
constexpr int kStepTile = 32, kStepWaves = 4, kStepRows = 32;

template <int D>
struct StepCfg {
    static constexpr int TILE = kStepTile * D, AREA = 2 * 2 * TILE;               // elements: of a tile, of a wave's two pairs
    static constexpr int POS_AT = kStepWaves * AREA * 2, LDS_BYTES = POS_AT + kStepWaves * 2 * 64 * 4;
    static constexpr int PPR = D / 8, RPI = 64 / PPR, NL = kStepTile / RPI;       // pieces of a row; rows, loads of a tile
};

// The weights of a set of which one workgroup had all keys and query rows, from its waves' logits (complete and in the L2 since their wait
// for all that was under way); lse: +inf for a row that weighs nothing.
template <int THREADS>
__device__ __forceinline__ void weigh_set(const float* logits, int stride, int n_rows, int len, const float* lse, const float* weight,
                                          float* weight_out) {
    wait_vmcnt<0>();
    __syncthreads();
    auto weigh = [&](int key, auto most) __attribute__((always_inline)) {          // (all logits requested together)
        float x[most], w = 0.f;
#pragma unroll
        for (int row = 0; row < most; ++row) x[row] = logits[(size_t)min(row, n_rows - 1) * stride + key];
#pragma unroll
        for (int row = 0; row < most; ++row)
            w += __builtin_amdgcn_exp2f(x[row] == -INFINITY || row >= n_rows ? -INFINITY : x[row] - lse[min(row, n_rows - 1)]);
        weight_out[key] = (weight ? weight[key] : 0.f) + w;
    };
    for (int key = threadIdx.x; key < len; key += THREADS) {
        if (n_rows <= 8) weigh(key, std::integral_constant<int, 8>{});
        else weigh(key, std::integral_constant<int, kStepRows>{});
    }
}

template <int D, bool POS, bool ONCE>
__global__ __launch_bounds__(64 * kStepWaves, 2) void attend_step_kernel(Sets s, Rule r, Partials part, uint16_t* __restrict__ O,
                                                                         float* __restrict__ LSE, float* logits, int stride, int n_split,
                                                                         const float* weight, float* weight_out) {
    using C = StepCfg<D>;
    constexpr int NW = kStepWaves, TK = kStepTile, PPR = C::PPR, NL = C::NL;
    extern __shared__ __attribute__((aligned(16))) uint16_t lds[];
    __shared__ float2 stats[NW][kStepRows];
    __shared__ float lse_lds[kStepRows];
    __shared__ __attribute__((aligned(16))) float q_lds[NW][D];                   // (of rows made again)
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int split = blockIdx.x, unit = blockIdx.y, g = unit % s.n_kv, b = unit / s.n_kv, group = s.n_q / s.n_kv, n_rows = group * s.T;
    const size_t set = (size_t)unit * s.cap;
    const uint16_t *kset = (const uint16_t*)s.k + set * D, *vset = (const uint16_t*)s.v + set * D;
    const int32_t* pos = POS ? r.row_pos + set : nullptr;
    uint16_t* const area = lds + wave * C::AREA;
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
    const uint32_t lds_w = lds_base + wave * (C::AREA * 2), lds_pos = lds_base + C::POS_AT + wave * (2 * 64 * 4);
    const int tile0 = split * NW + wave, every = n_split * NW;                    // the wave's tiles: tile0, tile0 + every, ...
    const int r_in = lane / PPR, pp = lane % PPR;

    // `rows`: rows that may be read, the capacity for the first request, which does not wait for the length
    auto request = [&](int tile, int buf, int rows) __attribute__((always_inline)) {
        const int key0 = tile * TK, rlim = min(TK - 1, rows - 1 - key0);
        const char *kb = (const char*)(kset + (size_t)key0 * D), *vb = (const char*)(vset + (size_t)key0 * D);
#pragma unroll
        for (int x = 0; x < NL; ++x) {
            const int row = x * C::RPI + r_in;
            const int kp = pp ^ ((row / (16 / PPR)) & (PPR - 1));
            constexpr int CPR = D * 2 / 64, RPL = D == 128 ? 1 : 2;
            const int vp = (((pp >> 2) ^ ((row / RPL) & (CPR - 1))) << 2) | (pp & 3);
            const uint32_t kdst = lds_w + (uint32_t)buf * (4 * C::TILE) + x * 1024, roff = (uint32_t)min(row, rlim) * (D * 2);
            dma16_as<ONCE>(kb, roff + kp * 16, kdst);
            dma16_as<ONCE>(vb, roff + vp * 16, kdst + 2 * C::TILE);
        }
        if constexpr (POS) dma4(pos + key0, (uint32_t)min(lane, rlim) * 4, lds_pos + buf * 256);
    };
    constexpr int LOADS = 2 * NL + (POS ? 1 : 0);
    if (tile0 * TK < s.cap) request(tile0, 0, s.cap);

    const int rho = min(l32, n_rows - 1), tok = rho / group, h = g * group + rho % group;
    bf16x8 qreg[1][D / 16];
    {
        const uint4* src = (const uint4*)((const uint16_t*)s.q + (((size_t)b * s.T + tok) * s.n_q + h) * D);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) qreg[0][ks] = __builtin_bit_cast(bf16x8, src[ks * 2 + hi]);
    }
    const int pq = POS ? r.q_pos[b * s.T + tok] : 0;
    const float slope2 = POS ? slope_of(r, h) : 0.f;
    const int len = min(max(s.len[b], 0), s.cap);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {                     // complete here, with the older request of the first tile
        typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
        asm volatile("" :: "v"(__builtin_bit_cast(u32x4, qreg[0][ks])));
    }
    asm volatile("" :: "v"(pq), "v"(slope2), "v"(len));
    wait_vmcnt<0>();
    const Span span = span_of(r, pq);
    Reach reach;
    if (s.T == 1) reach.most = reach.least = span;            // (all rows are one token's)
    else reach.of(span);
    const int n_tiles = (len + TK - 1) / TK, n = tile0 < n_tiles ? (n_tiles - tile0 + every - 1) / every : 0;
    // Rows past the length may hold anything (0 * NaN): the one tile that straddles it is fetched again, its rows the last one.
    if (n > 0 && tile0 * TK + TK > len) {
        request(tile0, 0, len);
        wait_vmcnt<0>();
    }
    f32x16 o[1][D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) o[0][db] = zero16();
    const bool capped = r.cap2 > 0.f, biased = POS && r.slopes;
    const float cu = capped || biased ? 1.f : r.c2, unit_of = capped ? 1.f : r.c2;       // units of log 2 of y below; of what a bias is put to
    float m_run = -INFINITY, mc_run = kLowest, l_run = 0.f;
    float* const kept = logits ? logits + ((size_t)unit * n_rows + rho) * stride : nullptr;

    if (n > 1) request(tile0 + every, 1, len);
    for (int i = 0; i < n; ++i) {
        const int tile = tile0 + i * every, left = len - tile * TK;
        if (i >= 1) {
            const bool more = i + 1 < n;
            if (more) request(tile + every, (i + 1) & 1, len);
            if (more) wait_vmcnt<LOADS>(); else wait_vmcnt<0>();                 // tile i has landed
        }
        __builtin_amdgcn_wave_barrier();
        const uint16_t *kt = area + (i & 1) * 2 * C::TILE, *vt = kt + C::TILE;
        const int32_t* tile_pos = (const int32_t*)((const char*)lds + C::POS_AT) + (wave * 2 + (i & 1)) * 64;
        bool all = left >= TK;                                // all rows see all keys
        if constexpr (POS) {
            const int pk = l32 < left ? tile_pos[l32] : -1;
            if (__builtin_amdgcn_ballot_w64(sees(reach.most, pk)) == 0) {
                if (kept && l32 < n_rows)
#pragma unroll
                    for (int jq = 0; jq < 4; ++jq)
                        *(float4*)(kept + tile * TK + jq * 8 + hi * 4) = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
                continue;
            }
            all &= ~__builtin_amdgcn_ballot_w64(sees(reach.least, pk)) == 0;
        }
        f32x16 x[1][1];
        qk_tile<D, 1, 1>(kt, qreg, l32, hi, x);
        float y[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) y[j] = x[0][0][j];
        if (capped)
            cap_logits(y, r, !POS || all, [&](const float (&z)[16]) __attribute__((always_inline)) {
                return largest_of(span, r.n_always, tile_pos, hi, z);
            });
        if (biased) {
#pragma unroll
            for (int j = 0; j < 16; ++j) y[j] = fmaf(-slope2, (float)abs(pq - tile_pos[acc_key(0, j, hi)]), y[j] * unit_of);
        }
        auto keep = [&](const float (&v)[16]) __attribute__((always_inline)) {
            if (kept && l32 < n_rows)
#pragma unroll
                for (int jq = 0; jq < 4; ++jq)
                    *(float4*)(kept + tile * TK + jq * 8 + hi * 4) = make_float4(v[jq * 4], v[jq * 4 + 1], v[jq * 4 + 2], v[jq * 4 + 3]);
        };
        auto kept_as = [&](float z) { return z * cu == -INFINITY ? kLowest : z * cu; };
        float v[16];
        if (all) {
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = kept_as(y[j]);
        } else {
#pragma unroll
            for (int jq = 0; jq < 4; ++jq) {
                int p[4] = {0, 0, 0, 0};
                if constexpr (POS) {
                    const int4 p4 = *(const int4*)(tile_pos + jq * 8 + hi * 4);
                    p[0] = p4.x; p[1] = p4.y; p[2] = p4.z; p[3] = p4.w;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = jq * 4 + e, pk = acc_key(0, j, hi) < left ? p[e] : -1;
                    v[j] = shown<true>(span, pk, kept_as(y[j]));
                    y[j] = shown<true>(span, pk, y[j]);
                }
            }
        }
        keep(v);
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 16; ++j) top = fmaxf(top, y[j]);
        if (__builtin_amdgcn_ballot_w64(fmaf(top, cu, -mc_run) > 8.f) != 0) {
            const float m_new = fmaxf(m_run, fmaxf(top, __shfl_xor(top, 32)));
            const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m_run - m_new) * cu);
            l_run *= alpha;
            m_run = m_new;
            mc_run = fmaxf(m_new * cu, kLowest);
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[0][db][j] *= alpha;
        }
        bf16x8 pb[1][1][2];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float p = __builtin_amdgcn_exp2f(fmaf(y[j], cu, -mc_run));
            l_run += p;
            pb[0][0][j >> 3][j & 7] = (__bf16)p;
        }
        pv_tile<D, 1, 1>(vt, pb, lane, o);
        __builtin_amdgcn_wave_barrier();
    }
    wait_vmcnt<0>();                                           // (a wave without tiles: its request of the first one)

    // ---- merge the waves: 16-byte piece c of a row lies at c ^ row (mod the pieces) of the wave's area, which is free now ----
    static_assert(kStepRows * D * 4 <= C::AREA * 2, "the merge fits a wave's area");
    constexpr int PPR4 = D / 4;
    float* red = (float*)area;
    const float l = l_run + __shfl_xor(l_run, 32);
    bool odd = false;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int j = 0; j < 16; ++j) odd |= !(fabsf(o[0][db][j]) < INFINITY);
    unsigned long long again = __builtin_amdgcn_ballot_w64(odd && l32 < n_rows);
    again = (again | again >> 32) & 0xffffffffull;
    if (l32 < n_rows && !(again >> l32 & 1)) {
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int rq = 0; rq < 4; ++rq)
                *(float4*)(red + (l32 * PPR4 + ((db * 8 + rq * 2 + hi) ^ (l32 & (PPR4 - 1)))) * 4) =
                    make_float4(o[0][db][rq * 4], o[0][db][rq * 4 + 1], o[0][db][rq * 4 + 2], o[0][db][rq * 4 + 3]);
        if (hi == 0) stats[wave][l32] = make_float2(l == 0.f ? -INFINITY : mc_run, l);
    }
    while (again) {                                            // (uniform in the wave)
        const int row = __builtin_ctzll(again);
        again &= again - 1;
        const int t = row / group, hq = g * group + row % group;
        __builtin_amdgcn_wave_barrier();
        for (int x = lane; x < D; x += 64) q_lds[wave][x] = as_float(((const uint16_t*)s.q)[(((size_t)b * s.T + t) * s.n_q + hq) * D + x]);
        __builtin_amdgcn_wave_barrier();
        float m, l2, acc[D / 64];
        exact_row<uint16_t, D>(r, q_lds[wave], kset, vset, r.row_pos ? r.row_pos + set : nullptr, tile0 * TK, len, TK, every * TK,
                               r.q_pos ? r.q_pos[b * s.T + t] : 0, slope_of(r, hq), m, l2, acc);
#pragma unroll
        for (int x = 0; x < D / 64; ++x) {
            const int d = lane + 64 * x;
            red[(row * PPR4 + ((d >> 2) ^ (row & (PPR4 - 1)))) * 4 + (d & 3)] = acc[x];
        }
        if (lane == 0) stats[wave][row] = make_float2(m, l2);
    }
    __syncthreads();
    const size_t part_row0 = ((size_t)unit * n_split + split) * n_rows;
    constexpr int ITEMS = kStepRows * PPR4 / (64 * NW);       // pieces of a thread at most: all read before any is worked on
    float2 st[ITEMS][NW];
    float4 v[ITEMS][NW];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        if (i * 64 * NW >= n_rows * PPR4) break;
        const int e = min(i * 64 * NW + tid, n_rows * PPR4 - 1), row = e / PPR4, c = e % PPR4;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            st[i][w] = stats[w][row];
            v[i][w] = *(const float4*)((const float*)(lds + w * C::AREA) + (row * PPR4 + (c ^ (row & (PPR4 - 1)))) * 4);
        }
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int e = i * 64 * NW + tid, row = e / PPR4, c = e % PPR4;
        if (e >= n_rows * PPR4) break;
        float M = -INFINITY, L = 0.f, a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) M = fmaxf(M, st[i][w].x);
        const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = part_weight(st[i][w], ref);
            L = add_part(f, st[i][w].y, L);
            a[0] = add_part(f, v[i][w].x, a[0]); a[1] = add_part(f, v[i][w].y, a[1]);
            a[2] = add_part(f, v[i][w].z, a[2]); a[3] = add_part(f, v[i][w].w, a[3]);
        }
        if (n_split > 1) {
            if (c == 0) part.ml[part_row0 + row] = make_float2(M, L);
            *(float4*)(part.o + (part_row0 + row) * D + c * 4) = make_float4(a[0], a[1], a[2], a[3]);
        } else {
            const size_t out = ((size_t)b * s.T + row / group) * s.n_q + g * group + row % group;
            __attribute__((aligned(8))) uint16_t z[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) z[j] = f32_to_bf16(L == 0.f ? 0.f : a[j] / L);
            *(uint2*)(O + out * D + c * 4) = *(const uint2*)z;
            if (c == 0) {
                const float y = M + __builtin_amdgcn_logf(L);
                if (LSE) LSE[out] = L == 0.f ? -INFINITY : y * kLn2;
                lse_lds[row] = L == 0.f ? INFINITY : y;       // (weighs nothing)
            }
        }
    }
    if (n_split > 1 || !logits) return;
    // One workgroup had all keys: the weights too.
    weigh_set<64 * NW>(logits + (size_t)unit * n_rows * stride, stride, n_rows, len, lse_lds, weight ? weight + set : nullptr, weight_out + set);
}

// The merge of the splits of one query row by a workgroup: SG groups of D / 4 lanes take every SG-th split, six requested together, and are
// folded through LDS in their order.
template <bool F32, int D>
struct MergeArea {
    static constexpr int NV = D / 4, SG = 256 / NV;
    __attribute__((aligned(16))) float red[SG][D];
    float2 stat[SG];
};
template <bool F32, int D>
__device__ __forceinline__ void merge_row(MergeArea<F32, D>& area, const Partials& part, typename Storage<F32>::T* O, float* LSE, float* lse2,
                                          int T, int n_q, int n_kv, int n_split, long long id) {
    constexpr int NV = D / 4, SG = 256 / NV, U = 6;
    const int group = n_q / n_kv, n_rows = T * group, sg = threadIdx.x / NV, d = threadIdx.x % NV * 4;
    const int rho = (int)(id % n_rows);
    const long long unit = id / n_rows;
    const int g = (int)(unit % n_kv), b = (int)(unit / n_kv);
    const size_t base = (size_t)unit * n_split * n_rows + rho;
    float M = -INFINITY, L = 0.f, a[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = sg; s0 < n_split; s0 += U * SG) {
        float2 ml[U];
        float4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const size_t at = base + (size_t)min(s0 + u * SG, n_split - 1) * n_rows;
            ml[u] = part.ml[at];
            v[u] = *(const float4*)(part.o + at * D + d);
        }
        float m_new = M;
#pragma unroll
        for (int u = 0; u < U; ++u) m_new = fmaxf(m_new, ml[u].x);
        const float ref = m_new == -INFINITY ? 0.f : m_new, f0 = part_weight(make_float2(M, L), ref);
        M = m_new;
        L *= f0;
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] = f0 == 0.f ? 0.f : a[j] * f0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float f = s0 + u * SG < n_split ? part_weight(ml[u], ref) : 0.f;
            L = add_part(f, ml[u].y, L);
            a[0] = add_part(f, v[u].x, a[0]); a[1] = add_part(f, v[u].y, a[1]); a[2] = add_part(f, v[u].z, a[2]); a[3] = add_part(f, v[u].w, a[3]);
        }
    }
    *(float4*)&area.red[sg][d] = make_float4(a[0], a[1], a[2], a[3]);
    if (d == 0) area.stat[sg] = make_float2(M, L);
    __syncthreads();
    if (threadIdx.x >= D) return;                             // a column each
    M = -INFINITY;
#pragma unroll
    for (int i = 0; i < SG; ++i) M = fmaxf(M, area.stat[i].x);
    const float ref = M == -INFINITY ? 0.f : M;
    float sum = 0.f;
    L = 0.f;
#pragma unroll
    for (int i = 0; i < SG; ++i) {
        const float f = part_weight(area.stat[i], ref);
        L = add_part(f, area.stat[i].y, L);
        sum = add_part(f, area.red[i][threadIdx.x], sum);
    }
    const size_t row = ((size_t)b * T + rho / group) * n_q + g * group + rho % group;
    store_as(O + row * D + threadIdx.x, L == 0.f ? 0.f : sum / L);
    if (threadIdx.x == 0) {
        const float y = L == 0.f ? -INFINITY : M + __builtin_amdgcn_logf(L);
        if (LSE) LSE[row] = y * kLn2;
        if (lse2) lse2[id] = y;
    }
}

template <bool F32, int D>
__global__ __launch_bounds__(256) void attend_merge_kernel(Partials part, typename Storage<F32>::T* __restrict__ O, float* __restrict__ LSE,
                                                           float* __restrict__ lse2, int T, int n_q, int n_kv, int n_split, long long all) {
    __shared__ MergeArea<F32, D> area;
    const long long id = folded_id();
    if (id < all) merge_row<F32, D>(area, part, O, LSE, lse2, T, n_q, n_kv, n_split, id);
}

// What follows on the kernels that keep their logits: the first n_merge workgroups merge the splits of a query row, the others add up the
// weights of 1,024 rows of a set, each with the LSE of its (at most R) query rows made from the splits' sums again.  One launch instead of
// two, and neither part waits for the other.  4.5 us behind a token over 4,097 rows (a launch and two trips to memory), 7.2 behind eight
// over 18,177.  R = 8, 16, 32 for the registers that the logits wait in.
template <bool F32, int D, int R>
__global__ __launch_bounds__(256) void attend_finish_kernel(Partials part, typename Storage<F32>::T* __restrict__ O, float* __restrict__ LSE,
                                                            const float* __restrict__ logits, const int32_t* __restrict__ mix_len,
                                                            const float* weight, float* weight_out, int T, int n_q, int n_kv, int cap, int stride,
                                                            int n_split, int n_merge, int n_blocks, long long all) {
    __shared__ MergeArea<F32, D> area;
    __shared__ float2 ml_lds[4][R];
    __shared__ float lse_lds[R];
    long long id = folded_id();
    if (id >= all) return;
    if (id < n_merge) {
        merge_row<F32, D>(area, part, O, LSE, nullptr, T, n_q, n_kv, n_split, id);
        return;
    }
    id -= n_merge;
    const int unit = (int)(id / n_blocks), key0 = (int)(id % n_blocks) * 1024, key = key0 + (int)threadIdx.x * 4, n_rows = n_q / n_kv * T;
    const size_t set = (size_t)unit * cap;
    // Everything is requested before anything is waited for: logits and weights of rows up to the capacity, whatever the length.
    const float* y = logits + (size_t)unit * n_rows * stride + min(key, stride - 4);
    float4 rows[R];
    float w_in[4];
#pragma unroll
    for (int i = 0; i < R; ++i) rows[i] = *(const float4*)(y + (size_t)min(i, n_rows - 1) * stride);
#pragma unroll
    for (int j = 0; j < 4; ++j) w_in[j] = weight ? weight[set + min(key + j, cap - 1)] : 0.f;
    // LSE of the query rows: every (256 / R)-th split by each of R threads, four requested together, joined over the lanes and waves.
    constexpr int SG = 256 / R, U = 4;
    const int row = threadIdx.x % R, sg = threadIdx.x / R;
    const float2* ml = part.ml + (size_t)unit * n_split * n_rows + min(row, n_rows - 1);
    float2 sum = make_float2(-INFINITY, 0.f);
    auto join = [](float2 a, float2 b) __attribute__((always_inline)) {
        const float M = fmaxf(a.x, b.x), ref = M == -INFINITY ? 0.f : M;
        return make_float2(M, add_part(part_weight(a, ref), a.y, add_part(part_weight(b, ref), b.y, 0.f)));
    };
    for (int s0 = sg; s0 < n_split; s0 += U * SG) {
        float2 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = ml[(size_t)min(s0 + u * SG, n_split - 1) * n_rows];
#pragma unroll
        for (int u = 0; u < U; ++u) sum = join(sum, s0 + u * SG < n_split ? v[u] : make_float2(-INFINITY, 0.f));
    }
    const int len = min(max(mix_len[unit / n_kv], 0), cap);
    if (key0 >= len) return;
#pragma unroll
    for (int o = R; o < 64; o <<= 1) sum = join(sum, make_float2(__shfl_xor(sum.x, o), __shfl_xor(sum.y, o)));
    if (threadIdx.x % 64 < R) ml_lds[threadIdx.x / 64][row] = sum;
    __syncthreads();
    if (threadIdx.x < R) {
        sum = join(join(ml_lds[0][row], ml_lds[1][row]), join(ml_lds[2][row], ml_lds[3][row]));
        lse_lds[row] = sum.y == 0.f || row >= n_rows ? INFINITY : sum.x + __builtin_amdgcn_logf(sum.y);          // (weighs nothing)
    }
    __syncthreads();
    float w[4] = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](float4 v, float lse) __attribute__((always_inline)) {
        const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] += __builtin_amdgcn_exp2f(x[j] == -INFINITY ? -INFINITY : x[j] - lse);
    };
#pragma unroll
    for (int i = 0; i < R; ++i) add(rows[i], lse_lds[i]);     // (behind the last row: it again, weighing nothing)
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (key + j < len) weight_out[set + key + j] = w_in[j] + w[j];
}

// ------------------------------------------------------------------------------------------
// The weights of the rows where there are many query rows: the logits once more, against the LSE.  A wave keeps 64 keys in registers as the
// operand of the first product and goes over query rows, 64 at a time from a ring of four LDS stages, which direct loads fill three tiles
// ahead for the four waves of a workgroup (counted by hand); a lane's sums are of its elements of the tiles, folded over the lanes at the
// end.  Query rows are cut into n_part parts where keys alone do not fill the chip, whose sums a last kernel adds in order.
// Bound by the vector instructions, an exponential and a sum per element beside one product where the ring has two.  What the pass adds to
// a call in replayed graphs: 14,336 query rows and 18,688 rows of 4 KV heads 312 us, 0.83 PFLOP/s (under a profiler, 12 launches, 355 at
// least); 448 and 23,872 26, capped 32 (41 by the exponential).  Each wave fed from memory by itself, without the ring: 39 where it took
// 30.  Logits kept for this instead of made again would be 4 bytes an element both ways: 171 MB, 70 us, for the 448.
// ------------------------------------------------------------------------------------------
// Lanes whose bit N is set keep the upper half of their elements and take their partner's, the others the lower half.
template <int N>
__device__ __forceinline__ void fold(const float (&from)[2 * N], float (&to)[N], int lane) {
    const bool upper = lane & N;
#pragma unroll
    for (int j = 0; j < N; ++j) to[j] = (upper ? from[j + N] : from[j]) + __shfl_xor(upper ? from[j] : from[j + N], N);
}

constexpr int kWeightWaves = 4, kWeightKeys = 64 * kWeightWaves, kWeightRows = 64;

template <int D>
struct WeightsCfg {
    static constexpr int NS = 4, TILE = kWeightRows * D, PPR = D / 8, RPI = 64 / PPR, IPW = kWeightRows / RPI / kWeightWaves;   // as the ring's
    static constexpr int LOADS = IPW + 1;                     // of a wave and tile: its rows, and one of LSE, position and slope
    static constexpr int INFO_AT = NS * TILE * 2, LDS_BYTES = INFO_AT + NS * kWeightWaves * 64 * 4;
};

template <int D, bool POS>
__global__ __launch_bounds__(64 * kWeightWaves, 2) void attend_weights_kernel(Sets s, Rule r, const float* __restrict__ lse2, const float* weight,
                                                                              float* weight_out, float* __restrict__ part_w, int units, int n_part) {
    using C = WeightsCfg<D>;
    struct Row {               // of a query row, as a lane needs it
        float lse, slope2;     // (lse +inf: weighs nothing)
        Span span;
        int pq;
    };
    extern __shared__ __attribute__((aligned(16))) uint16_t lds[];
    __shared__ __attribute__((aligned(16))) int32_t pos_lds[POS ? kWeightWaves : 1][64];
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // The last rows of a set first: new ones, which later tokens see and earlier ones do not, take longest.
    const unsigned id = folded_id(), pairs = (unsigned)(units * n_part);
    const int unit = (int)(id % pairs) / n_part, part = (int)(id % pairs) % n_part, g = unit % s.n_kv, b = unit / s.n_kv;
    const int group = s.n_q / s.n_kv, n_rows = group * s.T, len = min(max(s.len[b], 0), s.cap);
    const int block = (len + kWeightKeys - 1) / kWeightKeys - 1 - (int)(id / pairs);
    if (block < 0) return;
    const size_t set = (size_t)unit * s.cap;
    const int key0 = block * kWeightKeys + wave * 64;
    const bool active = key0 < len;
    const int row_tiles = (n_rows + kWeightRows - 1) / kWeightRows, share = row_tiles / n_part, more = row_tiles % n_part;
    const int tile0 = part * share + min(part, more), n_t = share + (part < more ? 1 : 0);

    bf16x8 k[2][D / 16];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
        const uint4* src = (const uint4*)((const uint16_t*)s.k + (set + min(key0 + kb * 32 + l32, len - 1)) * D);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) k[kb][ks] = __builtin_bit_cast(bf16x8, src[ks * 2 + hi]);
    }
    int pk = key0 + lane < len ? (POS ? max(r.row_pos[set + key0 + lane], -1) : 0) : -1, pk_min = pk, pk_max = pk;
    if constexpr (POS) {
        pos_lds[wave][lane] = pk;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            pk_min = min(pk_min, __shfl_xor(pk_min, o));
            pk_max = max(pk_max, __shfl_xor(pk_max, o));
        }
    }
    const bool capped = r.cap2 > 0.f, biased = POS && r.slopes, ragged = key0 + 64 > len;
    const float cu = capped || biased ? 1.f : r.c2, unit_of = capped ? 1.f : r.c2;       // units of log 2 of x below; of what a bias is put to

    // Tile t -> stage t % NS, the tiles in their order; rows behind the last one are it.  Token and head of a lane's first row, and of the
    // row whose numbers it loads, are carried from tile to tile: divisions by the group took as long as the products.
    struct Place {
        int tok, hg;
        __device__ __forceinline__ void add(int toks, int hgs, int group) {
            tok += toks;
            hg += hgs;
            if (hg >= group) { hg -= group; ++tok; }
        }
    };
    const char* const q_unit = (const char*)((const uint16_t*)s.q + ((size_t)b * s.T * s.n_q + (size_t)g * group) * D);
    const int r_in = lane / C::PPR, pp = lane % C::PPR, first = tile0 * kWeightRows + wave * C::RPI + r_in, own = tile0 * kWeightRows + lane;
    constexpr int BETWEEN = C::RPI * kWeightWaves;            // rows between two loads of a wave
    const int tile_toks = kWeightRows / group, tile_hgs = kWeightRows % group, load_toks = BETWEEN / group, load_hgs = BETWEEN % group;
    Place row_at{first / group, first % group}, own_at{own / group, own % group};
    const bool of_pos = POS && wave == 1, of_slope = POS && wave == 2 && r.slopes;
    const char* const info = of_pos ? (const char*)(r.q_pos + (size_t)b * s.T) : of_slope ? (const char*)(r.slopes + g * group)
                                                                                   : (const char*)(lse2 + (size_t)unit * n_rows);
    int issued = 0;
    auto issue = [&]() __attribute__((always_inline)) {
        const int t = min(issued, n_t - 1);
        const uint32_t st = lds_base + (uint32_t)(t % C::NS) * (C::TILE * 2);
        Place at = row_at;
#pragma unroll
        for (int i = 0; i < C::IPW; ++i) {
            const int row = (wave + i * kWeightWaves) * C::RPI + r_in, kp = pp ^ ((row / (16 / C::PPR)) & (C::PPR - 1));
            const bool there = at.tok < s.T;
            const int tok = there ? at.tok : s.T - 1, hg = there ? at.hg : group - 1;
            dma16_addr(q_unit + ((size_t)tok * s.n_q + hg) * (D * 2) + kp * 16, st + (wave + i * kWeightWaves) * 1024);
            at.add(load_toks, load_hgs, group);
        }
        const bool there = own_at.tok < s.T;
        const int tok = there ? own_at.tok : s.T - 1, hg = there ? own_at.hg : group - 1;
        dma4(info, (uint32_t)(of_pos ? tok : of_slope ? hg : tok * group + hg) * 4,
             lds_base + C::INFO_AT + (uint32_t)((t % C::NS) * kWeightWaves + wave) * 256);
        if (++issued < n_t) {
            row_at.add(tile_toks, tile_hgs, group);
            own_at.add(tile_toks, tile_hgs, group);
        }
    };
    auto product = [&](const uint16_t* q, int half, f32x16 (&x)[2]) __attribute__((always_inline)) {
        x[0] = x[1] = zero16();
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
            const bf16x8 a = *(const bf16x8*)(q + k_tile_off<D>(half * 32 + l32, ks * 2 + hi));
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) x[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[kb][ks], a, x[kb], 0, 0, 0);
        }
    };
    auto cap = [&](f32x16 (&x)[2], bool all_seen, const Span& span) __attribute__((always_inline)) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            float c[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) c[i] = x[kb][i];
            cap_logits(c, r, all_seen, [&](const float (&y)[16]) __attribute__((always_inline)) {
                return largest_of(span, r.n_always, pos_lds[POS ? wave : 0] + kb * 32, hi, y);
            });
#pragma unroll
            for (int i = 0; i < 16; ++i) x[kb][i] = c[i];
        }
    };
    f32x16 acc[2] = {zero16(), zero16()};
    auto plain = [&](const f32x16 (&x)[2], float lse) __attribute__((always_inline)) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[kb][i] += __builtin_amdgcn_exp2f(fmaf(x[kb][i], cu, -lse));
    };
    auto by_position = [&](f32x16 (&x)[2], auto&& f) __attribute__((always_inline)) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int rq = 0; rq < 4; ++rq) {
                int p[4];
                if constexpr (POS) {
                    const int4 p4 = *(const int4*)&pos_lds[wave][kb * 32 + rq * 8 + hi * 4];
                    p[0] = p4.x; p[1] = p4.y; p[2] = p4.z; p[3] = p4.w;
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[i] = key0 + kb * 32 + rq * 8 + hi * 4 + i < len ? 0 : -1;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) x[kb][rq * 4 + i] = f(x[kb][rq * 4 + i], p[i]);
            }
    };
    if (n_t > 0) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {             // complete here: no load that the compiler counts is outstanding behind
                typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
                asm volatile("" :: "v"(__builtin_bit_cast(u32x4, k[kb][ks])));
            }
        asm volatile("" :: "v"(pk_min), "v"(pk_max));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < C::NS - 1; ++t) issue();
        for (int t = 0; t < n_t; ++t) {
            wait_vmcnt<(C::NS - 2) * C::LOADS>();             // this wave's part of tile t has landed
            __builtin_amdgcn_s_barrier();                     // ... and everyone's; tile t - 1 is read by nobody any more
            issue();
            if (!active) continue;
            const uint16_t* q = lds + (t % C::NS) * C::TILE;
            const float* infos = (const float*)((const char*)lds + C::INFO_AT) + (t % C::NS) * (kWeightWaves * 64);
            auto lse_of = [&](int half) __attribute__((always_inline)) {
                const float lse = infos[half * 32 + l32];
                return (tile0 + t) * kWeightRows + half * 32 + l32 < n_rows && lse != -INFINITY ? lse : INFINITY;
            };
            auto pos_of = [&](int half) __attribute__((always_inline)) { return POS ? __float_as_int(infos[64 + half * 32 + l32]) : 0; };
            bool all = !ragged;
            if constexpr (POS) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const Span span = span_of(r, pos_of(half));
                    const bool within = ((unsigned)pk_min - (unsigned)span.lo < span.width) & ((unsigned)pk_max - (unsigned)span.lo < span.width);
                    all &= ~__builtin_amdgcn_ballot_w64((pk_min >= 0) & (within | ((unsigned)pk_max < span.na))) == 0;
                }
            }
            if (all && !biased && !capped) {
                const float lse[2] = {lse_of(0), lse_of(1)};
                f32x16 x[2], y[2];                            // (one stretch: a product runs beside the exponentials of the other)
                product(q, 0, x);
                product(q, 1, y);
                plain(x, lse[0]);
                plain(y, lse[1]);
                continue;
            }
            if (all && !biased) {                             // (in one stretch it spills; one branch for both: plain logits 2 % slower)
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    f32x16 x[2];
                    product(q, half, x);
                    cap(x, true, Span{});
                    plain(x, lse_of(half));
                }
                continue;
            }
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
                Row row;
                row.pq = pos_of(half);
                row.span = span_of(r, row.pq);
                if constexpr (POS) {
                    const bool hidden = (row.span.width == 0 || pk_max < row.span.lo || pk_min > row.span.hi()) &&
                                        (pk_max < 0 || (unsigned)max(pk_min, 0) >= row.span.na);
                    if (__builtin_amdgcn_ballot_w64(!hidden) == 0) continue;
                }
                row.lse = lse_of(half);
                row.slope2 = biased ? infos[128 + half * 32 + l32] * kLog2e : 0.f;
                f32x16 x[2];
                product(q, half, x);
                if (capped) cap(x, !POS || all, row.span);
                if (biased) by_position(x, [&](float y, int p) { return fmaf(-row.slope2, (float)abs(row.pq - p), y * unit_of); });
                if (all) {
                    plain(x, row.lse);
                } else {                                      // (what is not seen has weight 0, also where the LSE is no number)
                    if (r.n_always > 0)
                        by_position(x, [&](float y, int p) { return __builtin_amdgcn_exp2f(shown<true>(row.span, p, fmaf(y, cu, -row.lse))); });
                    else
                        by_position(x, [&](float y, int p) { return __builtin_amdgcn_exp2f(shown<false>(row.span, p, fmaf(y, cu, -row.lse))); });
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb) acc[kb] += x[kb];
                }
            }
        }
    }
    wait_vmcnt<0>();                                          // drain the refills before the wave ends
    if (!active) return;
    // Element e = 16 kb + i of the 32 lanes of a half to lane e: half of the elements change lanes at every step.
    float e32[32], e16[16], e8[8], e4[4], e2[2], e1[1];
#pragma unroll
    for (int e = 0; e < 32; ++e) e32[e] = acc[e >> 4][e & 15];
    fold<16>(e32, e16, lane);
    fold<8>(e16, e8, lane);
    fold<4>(e8, e4, lane);
    fold<2>(e4, e2, lane);
    fold<1>(e2, e1, lane);
    const int key = key0 + acc_key(l32 >> 4, l32 & 15, hi);
    if (key >= len) return;
    if (n_part > 1) part_w[((size_t)part * units + unit) * s.cap + key] = e1[0];
    else weight_out[set + key] = (weight ? weight[set + key] : 0.f) + e1[0];
}

// The sum of the parts.
__global__ __launch_bounds__(256) void weights_sum_kernel(const float* __restrict__ part_w, const int32_t* __restrict__ mix_len, const float* weight,
                                                          float* weight_out, int units, int n_kv, int cap, int n_part) {
    const int unit = blockIdx.y, row = blockIdx.x * 256 + threadIdx.x;
    if (row >= min(mix_len[unit / n_kv], cap)) return;
    const size_t at = (size_t)unit * cap + row;
    float w = 0.f;
    for (int p = 0; p < n_part; ++p) w += part_w[(size_t)p * units * cap + at];
    weight_out[at] = (weight ? weight[at] : 0.f) + w;
}

// ------------------------------------------------------------------------------------------
// fp32 sets, on the fp32 matrix instruction: 16 stacked query rows per workgroup, whose four waves take the 32-key tiles of its split in
// turn; operands come from memory in the order that both products use, as in the plain fp32 decode:
//   S^T = K Q^T    lane (i = lane % 16, j = lane / 16): K[key i][16 x + 4 j + e] and Q[row i] of the same; result register r: key 4 j + r, row i
//   O^T = V^T P^T  step r takes the keys 4 j + r, V[key 4 j + r][64 b + 4 i + e]; result register r' of (b, e): O[row i][64 b + 16 j + 4 r' + e]
// Bound by that instruction (a 1/16 of the bf16 one's rate) where there is enough to do; three sets of 705 rows with 5 tokens of 4 heads on
// 2, D = 64, take 6.5 us, of which launch and dependent loads are the most (row by row: 143).
// ------------------------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(4))) float f32x4;
constexpr int kF32Block = 16, kF32Tile = 32, kF32Waves = 4;

// Logits in units of log 2 of the four keys 4 j + r of a block, from the products: -inf where hidden, also behind `left` keys.
template <bool POS>
__device__ __forceinline__ float f32_logit(const Rule& r, const Span& span, float dot, float slope2, int pq, int pk, bool there) {
    float y = r.cap2 > 0.f ? r.cap2 * tanhf(dot * r.cap_in) : dot * r.c2;
    if (POS && r.slopes) y = fmaf(-slope2, (float)abs(pq - pk), y);
    return there && sees(span, pk) ? y : -INFINITY;
}

template <int D, bool POS>
__global__ __launch_bounds__(64 * kF32Waves, 2) void attend_f32_kernel(Sets s, Rule r, Partials part, float* __restrict__ O, float* __restrict__ LSE,
                                                                       float* __restrict__ lse2, float* logits, int stride, int units,
                                                                       int n_split, int n_rtile, const float* weight, float* weight_out) {
    constexpr int NW = kF32Waves, X = D / 16;
    __shared__ float lse_lds[kF32Block];
    __shared__ __attribute__((aligned(16))) float red[NW][kF32Block][D + 4];      // (+ 4: neighbouring rows in other banks)
    __shared__ float2 stats[NW][kF32Block];
    const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, j = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int unit, split, rtile;
    if (!place(units, n_split, n_rtile, &unit, &split, &rtile)) return;
    const int g = unit % s.n_kv, b = unit / s.n_kv, group = s.n_q / s.n_kv, n_rows = group * s.T, row0 = rtile * kF32Block;
    const int len = min(max(s.len[b], 0), s.cap);
    const size_t set = (size_t)unit * s.cap;
    const float *kset = (const float*)s.k + set * D, *vset = (const float*)s.v + set * D;
    const int rho = min(row0 + i, n_rows - 1), tok = rho / group, h = g * group + rho % group;
    const int pq = POS ? r.q_pos[b * s.T + tok] : 0;
    const float slope2 = POS ? slope_of(r, h) : 0.f;
    const Span span = span_of(r, pq);
    float4 q[X];
#pragma unroll
    for (int x = 0; x < X; ++x) q[x] = *(const float4*)((const float*)s.q + (((size_t)b * s.T + tok) * s.n_q + h) * D + 16 * x + 4 * j);
    float* const kept = logits && row0 + i < n_rows ? logits + ((size_t)unit * n_rows + rho) * stride : nullptr;

    f32x4 o[X];
#pragma unroll
    for (int x = 0; x < X; ++x) o[x] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    const int tiles = (len + kF32Tile - 1) / kF32Tile, tile0 = split * NW + wave, every = n_split * NW;
    for (int tile = tile0; tile < tiles; tile += every) {
        const int key0 = tile * kF32Tile;
        int pk[2][4];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 4; ++e) pk[kb][e] = POS ? r.row_pos[set + min(key0 + kb * 16 + 4 * j + e, len - 1)] : 0;
        if constexpr (POS) {                                  // (hidden from all 16 rows: nothing to do)
            bool any = false;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 4; ++e) any |= sees(span, pk[kb][e]);
            if (__builtin_amdgcn_ballot_w64(any) == 0) {
                if (kept)
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb)
                        *(float4*)(kept + key0 + kb * 16 + 4 * j) = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
                continue;
            }
        }
        float4 k[2][X], v[2][4][D / 64];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const float* p = kset + (size_t)min(key0 + kb * 16 + i, len - 1) * D + 4 * j;
#pragma unroll
            for (int x = 0; x < X; ++x) k[kb][x] = *(const float4*)(p + 16 * x);
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float* p = vset + (size_t)min(key0 + kb * 16 + 4 * j + e, len - 1) * D + 4 * i;
#pragma unroll
                for (int y = 0; y < D / 64; ++y) v[kb][e][y] = *(const float4*)(p + 64 * y);
            }
        f32x4 y[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int x = 0; x < X; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
                    y[kb] = __builtin_amdgcn_mfma_f32_16x16x4f32(((const float*)&k[kb][x])[e], ((const float*)&q[x])[e], y[kb], 0, 0, 0);
        float top = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            float keep[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool there = key0 + kb * 16 + 4 * j + e < len;
                y[kb][e] = f32_logit<POS>(r, span, y[kb][e], slope2, pq, pk[kb][e], there);
                keep[e] = there && sees(span, pk[kb][e]) && y[kb][e] == -INFINITY ? kLowest : y[kb][e];
                top = fmaxf(top, y[kb][e]);
            }
            if (kept) *(float4*)(kept + key0 + kb * 16 + 4 * j) = make_float4(keep[0], keep[1], keep[2], keep[3]);
        }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m_new = fmaxf(m, top), ref = m_new == -INFINITY ? 0.f : m_new, alpha = __builtin_amdgcn_exp2f(m - ref);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y[kb][e] = __builtin_amdgcn_exp2f(y[kb][e] - ref);
                l += y[kb][e];
            }
#pragma unroll
        for (int x = 0; x < X; ++x) o[x] *= alpha;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int x = 0; x < X; ++x)
                    o[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(((const float*)&v[kb][e][x / 4])[x % 4], y[kb][e], o[x], 0, 0, 0);
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    // A value that is no number reaches rows that do not see it, 0 * inf: those whose result is none are made again.
    bool odd = false;
#pragma unroll
    for (int x = 0; x < X; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) odd |= !(fabsf(o[x][e]) < INFINITY);
    unsigned long long again = __builtin_amdgcn_ballot_w64(odd && row0 + i < n_rows);
    again = (again | again >> 16 | again >> 32 | again >> 48) & 0xffffull;
    if (!(again >> i & 1)) {
#pragma unroll
        for (int x = 0; x < X; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) red[wave][i][64 * (x / 4) + 16 * j + 4 * e + x % 4] = o[x][e];
        if (j == 0) stats[wave][i] = make_float2(l == 0.f ? -INFINITY : m, l);
    }
    while (again) {                                           // (uniform in the wave; a row's place holds its query until its result is there)
        const int row = __builtin_ctzll(again);
        again &= again - 1;
        const int at = row0 + row, t = at / group, hq = g * group + at % group;
        float* q_row = red[wave][row];
        __builtin_amdgcn_wave_barrier();
        for (int x = lane; x < D; x += 64) q_row[x] = ((const float*)s.q)[(((size_t)b * s.T + t) * s.n_q + hq) * D + x];
        __builtin_amdgcn_wave_barrier();
        float m1, l1, acc[D / 64];
        exact_row<float, D>(r, q_row, kset, vset, r.row_pos ? r.row_pos + set : nullptr, tile0 * kF32Tile, len, kF32Tile, every * kF32Tile,
                            r.q_pos ? r.q_pos[b * s.T + t] : 0, slope_of(r, hq), m1, l1, acc);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int x = 0; x < D / 64; ++x) q_row[lane + 64 * x] = acc[x];
        if (lane == 0) stats[wave][row] = make_float2(m1, l1);
    }
    __syncthreads();
    const size_t part_row0 = ((size_t)unit * n_split + split) * n_rows + row0;
    for (int e = tid; e < min(kF32Block, n_rows - row0) * (D / 4); e += 64 * NW) {
        const int row = e / (D / 4), c = e % (D / 4) * 4;
        float2 st[NW];
        float M = -INFINITY, L = 0.f, a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            st[w] = stats[w][row];
            M = fmaxf(M, st[w].x);
        }
        const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float4 x = *(const float4*)&red[w][row][c];
            const float f = part_weight(st[w], ref);
            L = add_part(f, st[w].y, L);
            a[0] = add_part(f, x.x, a[0]); a[1] = add_part(f, x.y, a[1]); a[2] = add_part(f, x.z, a[2]); a[3] = add_part(f, x.w, a[3]);
        }
        const float y = L == 0.f ? -INFINITY : M + __builtin_amdgcn_logf(L);
        if (c == 0 && (n_split > 1 || logits)) part.ml[part_row0 + row] = make_float2(M, L);
        if (n_split > 1) {
            *(float4*)(part.o + (part_row0 + row) * D + c) = make_float4(a[0], a[1], a[2], a[3]);
        } else {
            const int at = row0 + row;
            const size_t out = ((size_t)b * s.T + at / group) * s.n_q + g * group + at % group;
#pragma unroll
            for (int x = 0; x < 4; ++x) a[x] = L == 0.f ? 0.f : a[x] / L;
            *(float4*)(O + out * D + c) = make_float4(a[0], a[1], a[2], a[3]);
            if (c == 0) {
                if (LSE) LSE[out] = y * kLn2;
                lse2[(size_t)unit * n_rows + at] = y;
                lse_lds[row] = L == 0.f ? INFINITY : y;       // (weighs nothing)
            }
        }
    }
    if (logits && n_split == 1 && n_rtile == 1)
        weigh_set<64 * NW>(logits + (size_t)unit * n_rows * stride, stride, n_rows, len, lse_lds, weight ? weight + set : nullptr, weight_out + set);
}

// The weights of fp32 sets where there are many query rows: a wave has 32 keys and goes over blocks of 16 query rows, four waves of a
// workgroup over parts of them, whose sums are folded through LDS.
template <int D, bool POS>
__global__ __launch_bounds__(64 * kF32Waves, 2) void weights_f32_kernel(Sets s, Rule r, const float* __restrict__ lse2, const float* weight,
                                                                        float* weight_out) {
    constexpr int NW = kF32Waves, X = D / 16;
    __shared__ float sums[NW][kF32Tile];
    const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, j = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int unit = blockIdx.y, g = unit % s.n_kv, b = unit / s.n_kv, group = s.n_q / s.n_kv, n_rows = group * s.T;
    const int len = min(max(s.len[b], 0), s.cap), key0 = (int)blockIdx.x * kF32Tile;
    if (key0 >= len) return;
    const size_t set = (size_t)unit * s.cap;
    float4 k[2][X];
    int pk[2][4];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
        const float* p = (const float*)s.k + (set + min(key0 + kb * 16 + i, len - 1)) * D + 4 * j;
#pragma unroll
        for (int x = 0; x < X; ++x) k[kb][x] = *(const float4*)(p + 16 * x);
#pragma unroll
        for (int e = 0; e < 4; ++e) pk[kb][e] = POS ? r.row_pos[set + min(key0 + kb * 16 + 4 * j + e, len - 1)] : 0;
    }
    f32x4 acc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
    for (int row0 = wave * kF32Block; row0 < n_rows; row0 += NW * kF32Block) {
        const int rho = min(row0 + i, n_rows - 1), tok = rho / group, h = g * group + rho % group;
        const float* src = (const float*)s.q + (((size_t)b * s.T + tok) * s.n_q + h) * D + 4 * j;
        float4 q[X];
#pragma unroll
        for (int x = 0; x < X; ++x) q[x] = *(const float4*)(src + 16 * x);
        const int pq = POS ? r.q_pos[b * s.T + tok] : 0;
        const float slope2 = POS ? slope_of(r, h) : 0.f, at = lse2[(size_t)unit * n_rows + rho];
        const float lse = row0 + i < n_rows && at != -INFINITY ? at : INFINITY;
        const Span span = span_of(r, pq);
        if constexpr (POS) {
            bool any = false;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 4; ++e) any |= sees(span, pk[kb][e]);
            if (__builtin_amdgcn_ballot_w64(any) == 0) continue;
        }
        f32x4 y[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int x = 0; x < X; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
                    y[kb] = __builtin_amdgcn_mfma_f32_16x16x4f32(((const float*)&k[kb][x])[e], ((const float*)&q[x])[e], y[kb], 0, 0, 0);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = f32_logit<POS>(r, span, y[kb][e], slope2, pq, pk[kb][e], true);
                acc[kb][e] += __builtin_amdgcn_exp2f(sees(span, pk[kb][e]) ? x - lse : -INFINITY);
            }
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float w = acc[kb][e];
#pragma unroll
            for (int x = 8; x > 0; x >>= 1) w += __shfl_xor(w, x);
            if (i == 0) sums[wave][kb * 16 + 4 * j + e] = w;
        }
    __syncthreads();
    if (tid >= kF32Tile || key0 + tid >= len) return;
    float w = 0.f;
#pragma unroll
    for (int x = 0; x < NW; ++x) w += sums[x][tid];
    const size_t at = set + key0 + tid;
    weight_out[at] = (weight ? weight[at] : 0.f) + w;
}

}  // namespace

// Test hook (vxl_debug.h).
static std::atomic<int> g_force_waves{0}, g_force_split{0}, g_force_part{0};
extern "C" void vxl_debug_mixed_force(int waves, int n_split, int n_part) {
    g_force_waves = waves == 4 || waves == 8 ? waves : 0;
    g_force_split = std::max(0, n_split);
    g_force_part = std::max(0, n_part);
}

// Many query rows (ring): estimates in us of a launch of workgroups of 256 and of 128 rows and so many splits: rounds over 256 compute
// units, 8 us for one's start and end, 1.75 and 1.13 per tile (0.75 of it for D = 64), 5 and 0.4 per MB for the merge.
static void ring_plan(MixedPlan& p, long long units, long long rows, int D, int l_cap) {
    const long long tiles = (l_cap + kKeyTile - 1) / kKeyTile;
    const int force_waves = g_force_waves, force_split = g_force_split;
    double best = 1e30;
    for (int nw : {8, 4}) {
        if (force_waves && nw != force_waves) continue;
        const long long n_rtile = (rows + 32 * nw - 1) / (32 * nw), base = units * n_rtile;
        const double tile = (nw == 8 ? 1.75 : 1.13) * (D == 64 ? 0.75 : 1.0);
        const long long most = force_split ? std::min<long long>(tiles, force_split)
                                           : std::max<long long>(1, std::min<long long>(tiles, 512 / base));
        for (long long n = force_split ? most : 1; n <= most;) {
            const long long walk = (tiles + n - 1) / n, rounds = (base * n + 255) / 256;
            const double mb = 4e-6 * units * n * rows * D;
            const double us = rounds * (8 + tile * walk) + (n > 1 ? 5 + 0.4 * mb : 0);
            if (us < best) {
                best = us;
                p.waves = nw;
                p.n_split = (int)n;
            }
            n = walk > 1 ? std::max(n + 1, (tiles + walk - 2) / (walk - 1)) : most + 1;           // the next that shortens the walk
        }
    }
}

// Splits: as forced, or from `first` on up to `last` the number that an estimate in us says is faster by a tenth (from eight on the first:
// no more than an eighth of a round is lost, and the search would take longer than it saves).
template <typename F>
static int split_by_rounds(int forced, long long first, long long last, F&& us, long long most) {
    if (forced) return (int)std::min<long long>(most, forced);
    long long best = first;
    for (long long n = first + 1; first < 8 && n <= last; ++n)
        if (us(n) < 0.9 * us(best)) best = n;
    return (int)best;
}

MixedPlan mixed_plan(const vxl_attn_desc* d, int batch, int T, int l_cap) {
    MixedPlan p{};
    const long long rows = (long long)(d->n_q_heads / d->n_kv_heads) * T, units = (long long)batch * d->n_kv_heads;
    const long long key_blocks = (l_cap + kWeightKeys - 1) / kWeightKeys;
    p.fits = units <= 65535 && rows <= 1 << 30 && (__int128)units * ((rows + 15) / 16) <= INT32_MAX / 2 && units * key_blocks <= INT32_MAX / 64;
    if (!p.fits) return p;
    p.n_split = p.n_part = 1;
    p.stride = (l_cap + kStepTile - 1) / kStepTile * kStepTile;
    p.few = rows <= kStepRows;
    if (d->dtype == VXL_F32) {
        // As many splits as fill the chip, each wave of one with a tile at least.  Sets of up to 128 rows are one workgroup's, and with up
        // to 16 query rows one launch's.  28 heads on 4, one token, D = 128: 128 rows 9.7 us, with the second launch 12; 192 rows 13.5 by
        // one workgroup, 12.1 by two and the launch.
        const long long tiles = (l_cap + kF32Tile - 1) / kF32Tile, most = (tiles + kF32Waves - 1) / kF32Waves;
        const long long base = units * ((rows + kF32Block - 1) / kF32Block);
        // More where the last round would leave many compute units idle, by estimates in us.  14 heads on 2 of D = 64, 1 to 5 splits:
        //   300 tokens over 5,000 rows              134, 109, 96, 94, 91
        //   80 tokens of four queries over 3,000    84, 73, 66, 64, 62
        p.n_split = split_by_rounds(g_force_split, std::min(most, std::max(1ll, 512 / base)), std::min(most, 2048 / base), [&](long long n) {
            const double walk = (double)((tiles + kF32Waves * n - 1) / (kF32Waves * n)), rounds = (double)((base * n + 511) / 512);
            return rounds * (5 + (d->head_dim == 64 ? 3 : 5) * walk) + (n > 1 ? 4 + units * rows / 1000. : 0);
        }, most);
    } else if (p.few) {
        // A workgroup on every compute unit, each wave of one with a tile at least.  Short sets by one workgroup each, which needs no
        // second launch.  Us by one workgroup and by splits:          one token      four tokens
        //   28 heads on 4, D = 128    256 rows                  9.0, 10.3      12.1, 13.9
        //                             384 rows                 10.7, 10.3      14.5, 14.1
        //   14 heads on 2, D = 64     384 rows                  8.9, 9.0       11.5, 12.1
        //                             512 rows                  9.7, 9.2       12.4, 12.1
        const long long tiles = (l_cap + kStepTile - 1) / kStepTile, most = (tiles + kStepWaves - 1) / kStepWaves;
        // More where the last round of workgroups would leave many units idle, by estimates in us.  28 heads on 4, from one split on:
        //   132 sets of 6,000 rows, one token       119, 123, 97, 107, 95, 104
        //   300 sets of 2,500 rows, one token       112, 95, 93
        //   144 sets of 2,500 rows, four tokens     69, 91, 79
        const long long full = std::min(most, std::max(1ll, 256 / units));
        const bool one = tiles <= (d->head_dim == 64 ? 12 : 8);
        p.n_split = split_by_rounds(g_force_split, one ? 1 : full, one ? 1 : std::min(most, 1024 / units), [&](long long n) {
            const double walk = (double)((tiles + kStepWaves * n - 1) / (kStepWaves * n)), rounds = (double)((units * n + 255) / 256);
            return rounds * (3 + (d->head_dim == 64 ? 1.75 : 2.4) * walk) + (n > 1 ? 4 + units * rows / 350. : 0);
        }, most);
    } else if (d->dtype == VXL_BF16) {
        ring_plan(p, units, rows, d->head_dim, l_cap);
        // Parts of the query rows, by estimates in us: rounds of two workgroups on a compute unit, but no less than the workgroup whose
        // keys are visible in part takes (tests per element).  What the pass adds in replayed graphs: 448 rows, 23,872 keys, 1 to 4 parts
        // 26, 32, 33, 37; 14,336 rows, 18,688 keys, 1, 3, 5, 7, 12 parts 502, 348, 315, 320, 315.
        const long long row_tiles = (rows + kWeightRows - 1) / kWeightRows, blocks = units * key_blocks;
        double best = 1e30;
        for (long long n = 1; n <= std::min<long long>(row_tiles, 16); ++n) {
            const double walk = (double)((row_tiles + n - 1) / n), rounds = std::max(1.0, blocks * n / 512.0);
            const double us = std::max((rounds + std::ceil(rounds)) / 2 * (8 + 2.1 * walk), 8 + 3.3 * walk) + (n > 1 ? 4 : 0);
            if (us < best) {
                best = us;
                p.n_part = (int)n;
            }
        }
        if (g_force_part) p.n_part = (int)std::min<long long>(row_tiles, g_force_part);
    }
    size_t at = 0;
    auto put = [&](size_t bytes) { const size_t o = at; at += align_up(bytes, 256); return o; };
    p.lse2 = put((size_t)units * rows * sizeof(float));
    p.part_o = put(p.n_split > 1 ? (size_t)units * p.n_split * rows * d->head_dim * sizeof(float) : 0);
    p.part_ml = put(p.n_split > 1 || p.few ? (size_t)units * p.n_split * rows * sizeof(float2) : 0);
    p.logits = put(p.few ? (size_t)units * rows * p.stride * sizeof(float) : 0);
    p.part_w = put(p.n_part > 1 ? (size_t)p.n_part * units * l_cap * sizeof(float) : 0);
    p.total = at;
    return p;
}

extern "C" int vxl_debug_mixed_plan(const vxl_attn_desc* d, int batch, int n_q_tokens, int l_cap, int* plan) {
    if (vxl_workspace_bytes(VXL_OP_MIXED_ATTEND, nullptr, d, batch, n_q_tokens, l_cap) == 0) return 0;
    const MixedPlan p = mixed_plan(d, batch, n_q_tokens, l_cap);
    plan[0] = p.waves;
    plan[1] = p.n_split;
    plan[2] = p.n_part;
    return 1;
}

// Workgroups on the XCDs in turn, as place() takes them.
static dim3 placed_grid(long long all) {
    const long long xcds = std::min<long long>(all, kXcds), each = (all + xcds - 1) / xcds;
    return dim3((unsigned)xcds, (unsigned)std::min<long long>(each, 65535), (unsigned)((each + 65534) / 65535));
}

static vxl_status launch_ring(const MixedPlan& p, const MixedCall& c, const Sets& sets, const Rule& rule, hipStream_t s) {
    const vxl_attn_desc* d = c.d;
    const int units = c.batch * d->n_kv_heads, rows = d->n_q_heads / d->n_kv_heads * c.T;
    const Partials part{(float*)(c.ws + p.part_o), (float2*)(c.ws + p.part_ml)};
    float* lse2 = (float*)(c.ws + p.lse2);
    auto run = [&](auto dim, auto nw, auto pos) {
        using C = RingCfg<dim, nw>;
        static PerDeviceOnce attr;
        const vxl_status st = attr.run([&] {
            VXL_HIP_TRY(hipFuncSetAttribute((const void*)attend_ring_kernel<dim, nw, pos>, hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS_BYTES));
            return VXL_OK;
        });
        if (st != VXL_OK) return st;
        const int n_rtile = (rows + C::ROWS - 1) / C::ROWS;
        hipLaunchKernelGGL((attend_ring_kernel<dim, nw, pos>), placed_grid((long long)units * p.n_split * n_rtile), dim3(64 * nw),
                           C::LDS_BYTES, s, sets, rule, part, (uint16_t*)c.O, c.LSE, lse2, units, p.n_split, n_rtile);
        return mixed_launched();
    };
    auto by_pos = [&](auto dim, auto nw) { return rule.q_pos ? run(dim, nw, std::true_type{}) : run(dim, nw, std::false_type{}); };
    auto by_waves = [&](auto dim) {
        return p.waves == 8 ? by_pos(dim, std::integral_constant<int, 8>{}) : by_pos(dim, std::integral_constant<int, 4>{});
    };
    return d->head_dim == 64 ? by_waves(std::integral_constant<int, 64>{}) : by_waves(std::integral_constant<int, 128>{});
}

// Behind a kernel that keeps its logits: one row per merging workgroup, 1,024 rows of a set per workgroup of the weights.
template <bool F32, int D>
static vxl_status launch_finish(const MixedPlan& p, const MixedCall& c, const Partials& part, const float* logits, hipStream_t s) {
    using T = typename Storage<F32>::T;
    const vxl_attn_desc* d = c.d;
    const int units = c.batch * d->n_kv_heads, rows = d->n_q_heads / d->n_kv_heads * c.T;
    if (p.n_split == 1 && !logits) return VXL_OK;
    const long long n_merge = p.n_split > 1 ? (long long)units * rows : 0, n_blocks = logits ? (c.l_cap + 1023) / 1024 : 0;
    const long long all = n_merge + units * n_blocks;
    auto finish = [&](auto most) {
        hipLaunchKernelGGL((attend_finish_kernel<F32, D, most>), folded_grid(all), dim3(256), 0, s, part, (T*)c.O, c.LSE, logits, c.mix_len, c.weight,
                           c.weight_out, c.T, d->n_q_heads, d->n_kv_heads, c.l_cap, p.stride, p.n_split, (int)n_merge, (int)n_blocks, all);
    };
    if (rows <= 8) finish(std::integral_constant<int, 8>{});
    else if (rows <= 16) finish(std::integral_constant<int, 16>{});
    else finish(std::integral_constant<int, 32>{});
    return mixed_launched();
}

// Keys and values of more bytes than the L2s have between them are read past the caches: 246 MB (302 of capacity, which is what is known
// here) 66 -> 60 us; 8 MB, which the next call finds in them, are not.
constexpr size_t kPastCachesBytes = 32u << 20;
static vxl_status launch_step(const MixedPlan& p, const MixedCall& c, const Sets& sets, const Rule& rule, hipStream_t s) {
    const vxl_attn_desc* d = c.d;
    const int units = c.batch * d->n_kv_heads;
    const Partials part{(float*)(c.ws + p.part_o), (float2*)(c.ws + p.part_ml)};
    float* logits = c.weight_out ? (float*)(c.ws + p.logits) : nullptr;
    auto run = [&](auto dim, auto pos, auto once) {
        using C = StepCfg<dim>;
        static PerDeviceOnce attr;
        vxl_status st = attr.run([&] {
            VXL_HIP_TRY(hipFuncSetAttribute((const void*)attend_step_kernel<dim, pos, once>, hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS_BYTES));
            return VXL_OK;
        });
        if (st != VXL_OK) return st;
        hipLaunchKernelGGL((attend_step_kernel<dim, pos, once>), dim3(p.n_split, units), dim3(64 * kStepWaves), C::LDS_BYTES, s, sets, rule, part,
                           (uint16_t*)c.O, c.LSE, logits, p.stride, p.n_split, c.weight, c.weight_out);
        st = mixed_launched();
        return st != VXL_OK || p.n_split == 1 ? st : launch_finish<false, dim>(p, c, part, logits, s);
    };
    const bool big = (size_t)units * c.l_cap * d->head_dim * 2 * 2 > kPastCachesBytes;
    auto by_size = [&](auto dim, auto pos) { return big ? run(dim, pos, std::true_type{}) : run(dim, pos, std::false_type{}); };
    auto by_pos = [&](auto dim) { return rule.q_pos ? by_size(dim, std::true_type{}) : by_size(dim, std::false_type{}); };
    return d->head_dim == 64 ? by_pos(std::integral_constant<int, 64>{}) : by_pos(std::integral_constant<int, 128>{});
}

static vxl_status launch_merge(const MixedPlan& p, const MixedCall& c, hipStream_t s) {
    const vxl_attn_desc* d = c.d;
    const Partials part{(float*)(c.ws + p.part_o), (float2*)(c.ws + p.part_ml)};
    const long long all = (long long)c.batch * c.T * d->n_q_heads;
    return by_storage(d, [&](auto f32, auto dim) {
        using T = typename Storage<f32>::T;
        hipLaunchKernelGGL((attend_merge_kernel<f32, dim>), folded_grid(all), dim3(256), 0, s, part, (T*)c.O, c.LSE, (float*)(c.ws + p.lse2), c.T,
                           d->n_q_heads, d->n_kv_heads, p.n_split, all);
        return mixed_launched();
    });
}

static vxl_status launch_weights(const MixedPlan& p, const MixedCall& c, const Sets& sets, const Rule& rule, hipStream_t s) {
    const vxl_attn_desc* d = c.d;
    const int units = c.batch * d->n_kv_heads, n_blocks = (c.l_cap + kWeightKeys - 1) / kWeightKeys;
    float *lse2 = (float*)(c.ws + p.lse2), *part_w = (float*)(c.ws + p.part_w);
    auto run = [&](auto dim, auto pos) {
        constexpr int lds = WeightsCfg<dim>::LDS_BYTES;
        static PerDeviceOnce attr;
        const vxl_status st = attr.run([&] {
            VXL_HIP_TRY(hipFuncSetAttribute((const void*)attend_weights_kernel<dim, pos>, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
            return VXL_OK;
        });
        if (st != VXL_OK) return st;
        hipLaunchKernelGGL((attend_weights_kernel<dim, pos>), folded_grid((long long)units * p.n_part * n_blocks), dim3(64 * kWeightWaves),
                           lds, s, sets, rule, lse2, c.weight, c.weight_out, part_w, units, p.n_part);
        return mixed_launched();
    };
    auto by_pos = [&](auto dim) { return rule.q_pos ? run(dim, std::true_type{}) : run(dim, std::false_type{}); };
    const vxl_status st = d->head_dim == 64 ? by_pos(std::integral_constant<int, 64>{}) : by_pos(std::integral_constant<int, 128>{});
    if (st != VXL_OK || p.n_part == 1) return st;
    hipLaunchKernelGGL(weights_sum_kernel, dim3((c.l_cap + 255) / 256, units), dim3(256), 0, s, part_w, c.mix_len, c.weight, c.weight_out, units,
                       d->n_kv_heads, c.l_cap, p.n_part);
    return mixed_launched();
}

static vxl_status launch_f32(const MixedPlan& p, const MixedCall& c, const Sets& sets, const Rule& rule, hipStream_t s) {
    const vxl_attn_desc* d = c.d;
    const int units = c.batch * d->n_kv_heads, rows = d->n_q_heads / d->n_kv_heads * c.T, n_rtile = (rows + kF32Block - 1) / kF32Block;
    const Partials part{(float*)(c.ws + p.part_o), (float2*)(c.ws + p.part_ml)};
    float *logits = p.few && c.weight_out ? (float*)(c.ws + p.logits) : nullptr, *lse2 = (float*)(c.ws + p.lse2);
    auto run = [&](auto dim, auto pos) {
        hipLaunchKernelGGL((attend_f32_kernel<dim, pos>), placed_grid((long long)units * p.n_split * n_rtile), dim3(64 * kF32Waves), 0, s,
                           sets, rule, part, (float*)c.O, c.LSE, lse2, logits, p.stride, units, p.n_split, n_rtile, c.weight, c.weight_out);
        vxl_status st = mixed_launched();
        if (st != VXL_OK) return st;
        if (p.few) return p.n_split == 1 && n_rtile == 1 ? st : launch_finish<true, dim>(p, c, part, logits, s);
        if (p.n_split > 1) st = launch_merge(p, c, s);
        if (st != VXL_OK || !c.weight_out) return st;
        hipLaunchKernelGGL((weights_f32_kernel<dim, pos>), dim3((c.l_cap + kF32Tile - 1) / kF32Tile, units), dim3(64 * kF32Waves), 0, s,
                           sets, rule, lse2, c.weight, c.weight_out);
        return mixed_launched();
    };
    auto by_pos = [&](auto dim) { return rule.q_pos ? run(dim, std::true_type{}) : run(dim, std::false_type{}); };
    return d->head_dim == 64 ? by_pos(std::integral_constant<int, 64>{}) : by_pos(std::integral_constant<int, 128>{});
}

static vxl_status launch_simple(const MixedPlan& p, const MixedCall& c, const Sets& sets, const Rule& rule, hipStream_t s) {
    const vxl_attn_desc* d = c.d;
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

vxl_status launch_mixed_attend(const MixedPlan& p, const MixedCall& c, bool force_simple, hipStream_t s) {
    const vxl_attn_desc* d = c.d;
    const vxl_score_rule none{};
    const vxl_score_rule& u = c.rule ? *c.rule : none;
    const float in = u.softcap > 0.f ? c.scale / u.softcap : 0.f, in2 = in * in;
    // |u| below which the series holds: where higher powers of the scale are lost they are not needed, and all coefficients are numbers.
    const float few = in < 0x1p-20f ? 0x1p-6f : in < 0x1p16f ? 0.125f : 0.f;
    const Rule rule{c.scale * kLog2e, in, u.softcap * kLog2e,
                    in > 0.f ? few / in : 0.f, {in2 * (-1.f / 3), in2 * in2 * (2.f / 15), in2 * in2 * in2 * (-17.f / 315)},
                    2 * kLog2e * in, -2 * kLog2e * u.softcap,
                    u.causal, u.window, u.n_always, u.slopes, c.q_pos, c.row_pos};
    const Sets sets{c.Qd, c.Kmix, c.Vmix, c.mix_len, c.T, d->n_q_heads, d->n_kv_heads, c.l_cap};
    if (force_simple) return launch_simple(p, c, sets, rule, s);
    if (d->dtype == VXL_F32) return launch_f32(p, c, sets, rule, s);
    if (p.few) return launch_step(p, c, sets, rule, s);
    vxl_status st = launch_ring(p, c, sets, rule, s);
    if (st == VXL_OK && p.n_split > 1) st = launch_merge(p, c, s);
    if (st == VXL_OK && c.weight_out) st = launch_weights(p, c, sets, rule, s);
    return st;
}

}  // namespace vxl
