// Rotary positions: of a prompt's queries and keys, and of new tokens on their way into a mixed set.
#include <algorithm>
#include <type_traits>

#include "vxl_mixed.h"

namespace vxl {

namespace {

// A row is D / (2 VEC) items of two chunks of VEC elements each: rotated (chunks i and i + rotary_dim / 2, or two neighbours whose elements
// are pairs among themselves) or copied.  A thread has one item of a token for its heads hg, hg + HG, ..., so the sines and cosines of its
// pairs are made once (in registers, from an angle in 64 bits) and used for all of them.
// HBM bound where there is much to do: 131,328 tokens of 28 + 4 heads, D = 128, bf16, 437 us, 4.9 TB/s read and written, a copy's rate; a
// launch and three dependent loads where there is little: 3.2 us.
// Threads that a launch of few tokens has at least, the heads of a token shared by several of them.  Us in a replayed graph with 2^15,
// 2^16, 2^17: 512 new tokens 7.1, 5.7, 5.7; 1,000 tokens of a prompt 6.6, 6.4, 7.3, 4,000 19.5, 15.7, 15.9.
constexpr long long kThreadsWanted = 1 << 16;
struct Where {                 // element strides between heads and tokens of source and destination
    long long head, tok;
};

template <typename T, int VEC> struct Chunk;
template <> struct Chunk<uint16_t, 8> { using V = uint4; };
template <> struct Chunk<float, 4> { using V = uint4; };
template <> struct Chunk<uint16_t, 1> { using V = uint16_t; };
template <> struct Chunk<float, 1> { using V = float; };

template <typename T, int VEC>
struct Turn {
    float c[VEC], s[VEC];

    // Of item i of a row at position p.  HALF: the pairs of a chunk and its partner; else those inside the two chunks.
    __device__ __forceinline__ void make(const double* freqs, int first, float magnitude, float sign, int p) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const double turns = (double)p * (freqs[first + j] * 0.15915494309189533576888);      // 1 / (2 pi)
            const float part = (float)(turns - rint(turns));
            sincospif(2.f * part, &s[j], &c[j]);
            c[j] *= magnitude;
            s[j] *= magnitude * sign;
        }
    }
    template <bool HALF>
    __device__ __forceinline__ void apply(T (&a)[VEC], T (&b)[VEC]) const {
        auto pair = [&](T& x, T& y, int j) __attribute__((always_inline)) {
            const float u = as_float(x), v = as_float(y);
            store_as(&x, fmaf(u, c[j], -(v * s[j])));
            store_as(&y, fmaf(u, s[j], v * c[j]));
        };
        if constexpr (HALF || VEC == 1) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) pair(a[j], b[j], j);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; j += 2) {
                pair(a[j], a[j + 1], j / 2);
                pair(b[j], b[j + 1], VEC / 2 + j / 2);
            }
        }
    }
};

// Heads 0 .. n_q - 1 are query heads, the next n_kv key heads, and (APPEND) the next n_kv value heads, which are copied.
struct RotateArgs {
    const double* freqs;
    const int32_t* positions;
    float magnitude, sign;
    int rotary_dim, n_tokens, n_q, n_kv, head_groups;
    const void *q, *k, *v;
    void *q_out, *k_out, *v_out;
    Where qs, ks, qo;              // of Q, of K and V, of the queries written
    // (append)
    int n_new, l_cap;
    const int32_t* mix_len;
    int32_t* row_pos;
    float* row_weight;
};

template <typename T, int D, int VEC, bool HALF, bool APPEND>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs a) {
    using V = typename Chunk<T, VEC>::V;
    constexpr int ITEMS = D / (2 * VEC), U = 4;
    const int item = threadIdx.x % ITEMS;
    const long long slot = (long long)folded_id() * (256 / ITEMS) + threadIdx.x / ITEMS;
    const int hg = (int)(slot % a.head_groups);
    const long long tok = slot / a.head_groups;
    if (tok >= a.n_tokens) return;
    const int rot = a.rotary_dim / (2 * VEC);                 // items that are rotated
    const bool turned = item < rot;
    const int c0 = !turned ? 2 * item : HALF ? item : 2 * item, c1 = !turned || !HALF ? c0 + 1 : item + rot;
    const int p = a.positions[tok];
    const int n_heads = a.n_q + (APPEND ? 2 : 1) * a.n_kv;
    int row = 0, b = 0;
    if constexpr (APPEND) {
        b = (int)(tok / a.n_new);
        const long long r = (long long)a.mix_len[b] - a.n_new + tok % a.n_new;
        row = r >= 0 && r < a.l_cap ? (int)r : -1;
    }
    auto is_value = [&](int h) { return APPEND && h >= a.n_q + a.n_kv; };
    auto head_in = [&](int h) { return h < a.n_q ? 0 : (h - a.n_q) % a.n_kv; };
    auto load = [&](int h0, V (&x)[U][2]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * a.head_groups;
            if (h >= n_heads) continue;
            const T* src = h < a.n_q ? (const T*)a.q + h * a.qs.head + tok * a.qs.tok
                                     : (const T*)(is_value(h) ? a.v : a.k) + head_in(h) * a.ks.head + tok * a.ks.tok;
            x[u][0] = *(const V*)(src + c0 * VEC);
            x[u][1] = *(const V*)(src + c1 * VEC);
        }
    };
    V x[U][2] = {};
    load(hg, x);                                              // (on their way while the angles are made)
    Turn<T, VEC> turn;
    if (turned) turn.make(a.freqs, item * VEC, a.magnitude, a.sign, p);
    for (int h0 = hg; h0 < n_heads; h0 += U * a.head_groups) {
        if (h0 != hg) load(h0, x);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * a.head_groups;
            if (h >= n_heads) continue;
            T* dst;
            if (h < a.n_q) dst = (T*)a.q_out + h * a.qo.head + tok * a.qo.tok;
            else if constexpr (APPEND) dst = (T*)(is_value(h) ? a.v_out : a.k_out) + (((long long)b * a.n_kv + head_in(h)) * a.l_cap + row) * D;
            else dst = (T*)a.k_out + head_in(h) * a.ks.head + tok * a.ks.tok;
            if (APPEND && h >= a.n_q && row < 0) continue;
            if (turned && !is_value(h)) {
                T lo[VEC], hi[VEC];
                __builtin_memcpy(lo, &x[u][0], sizeof(V));
                __builtin_memcpy(hi, &x[u][1], sizeof(V));
                turn.template apply<HALF>(lo, hi);
                __builtin_memcpy(&x[u][0], lo, sizeof(V));
                __builtin_memcpy(&x[u][1], hi, sizeof(V));
            }
            *(V*)(dst + c0 * VEC) = x[u][0];
            *(V*)(dst + c1 * VEC) = x[u][1];
            if (APPEND && item == 0 && h >= a.n_q && !is_value(h)) {
                const long long at = ((long long)b * a.n_kv + head_in(h)) * a.l_cap + row;
                if (a.row_pos) a.row_pos[at] = p;
                if (a.row_weight) a.row_weight[at] = 0.f;
            }
        }
    }
}

template <bool APPEND>
vxl_status launch(const vxl_attn_desc* d, const vxl_rotary* r, RotateArgs a, hipStream_t s) {
    const vxl_rotary none{nullptr, 0, 0, 1.f, 0};
    if (!r) r = &none;
    a.freqs = r->freqs;
    a.rotary_dim = r->rotary_dim;
    a.magnitude = r->magnitude;
    a.sign = r->transpose ? -1.f : 1.f;
    return by_storage(d, [&](auto f32, auto dim) {
        using T = typename Storage<f32>::T;
        auto run = [&](auto vec, auto half) {
            constexpr int PER = 256 / (dim / (2 * vec));      // slots of a workgroup
            const int n_heads = a.n_q + (APPEND ? 2 : 1) * a.n_kv;
            // few tokens: the heads of one are shared by several threads
            a.head_groups = 1;
            while (a.head_groups < n_heads && (long long)a.n_tokens * a.head_groups * (dim / (2 * vec)) < kThreadsWanted) a.head_groups *= 2;
            const long long slots = (long long)a.n_tokens * a.head_groups;
            hipLaunchKernelGGL((rotate_kernel<T, dim, vec, half, APPEND>), folded_grid((slots + PER - 1) / PER), dim3(256), 0, s, a);
            return mixed_launched();
        };
        constexpr int VEC = f32 ? 4 : 8;
        using Wide = std::integral_constant<int, VEC>;
        using One = std::integral_constant<int, 1>;
        const bool wide = r->rotary_dim % (2 * VEC) == 0;
        if (r->interleaved) return wide ? run(Wide{}, std::false_type{}) : run(One{}, std::false_type{});
        return wide ? run(Wide{}, std::true_type{}) : run(One{}, std::true_type{});
    });
}

}  // namespace

vxl_status launch_rotate(const vxl_attn_desc* d, const vxl_rotary* r, const int32_t* positions, int n_tokens, const void* Q, const void* K,
                         void* Q_out, void* K_out, hipStream_t s) {
    const TokStrides ts = tok_strides(d, n_tokens);
    RotateArgs a{};
    a.positions = positions;
    a.n_tokens = n_tokens;
    a.n_q = d->n_q_heads;
    a.n_kv = K ? d->n_kv_heads : 0;
    a.q = Q; a.k = K; a.q_out = Q_out; a.k_out = K_out;
    a.qs = a.qo = {ts.qh, ts.qt};
    a.ks = {ts.kh, ts.kt};
    return launch<false>(d, r, a, s);
}

vxl_status launch_mixed_append(const vxl_attn_desc* d, const vxl_rotary* r, const int32_t* positions, int batch, int n_new, const void* Q,
                               const void* K, const void* V, void* Qd, void* Kmix, void* Vmix, int l_cap, const int32_t* mix_len,
                               int32_t* row_pos, float* row_weight, hipStream_t s) {
    const TokStrides ts = tok_strides(d, batch * n_new);
    RotateArgs a{};
    a.positions = positions;
    a.n_tokens = batch * n_new;
    a.n_q = d->n_q_heads;
    a.n_kv = d->n_kv_heads;
    a.q = Q; a.k = K; a.v = V; a.q_out = Qd; a.k_out = Kmix; a.v_out = Vmix;
    a.qs = {ts.qh, ts.qt};
    a.ks = {ts.kh, ts.kt};
    a.qo = {d->head_dim, (long long)d->n_q_heads * d->head_dim};
    a.n_new = n_new; a.l_cap = l_cap; a.mix_len = mix_len; a.row_pos = row_pos; a.row_weight = row_weight;
    return launch<true>(d, r, a, s);
}

}  // namespace vxl
