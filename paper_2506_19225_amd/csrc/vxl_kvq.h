// The quantised cache: its launches, and device and host pieces that its kernels share.
#pragma once

#include <type_traits>

#include "vxl_internal.h"
#include "vxl_mfma.h"

namespace vxl {

// Of the caller's workspace of an in-place decode over either kind of cache, with so many bytes of partial results.
InplaceWorkspace inplace_workspace(int batch, int l_cap, size_t partials);

vxl_status launch_kvq_write(const vxl_attn_desc* d, const void* K, const void* V, int n_rows, const vxl_kvq_cache* c, int first,
                            hipStream_t s);
vxl_status launch_kvq_read(const vxl_attn_desc* d, const vxl_kvq_cache* c, int first, int n_rows, void* K, void* V, hipStream_t s);
// sp: quantised sparse rows read instead of the kept rows of c, or null (here and below)
vxl_status launch_kvq_gather(const vxl_layout* L, const vxl_attn_desc* d, const vxl_kvq_cache* c, const vxl_kvq_cache* sp,
                             const uint8_t* dense_mask, int batch, void* Kmix, void* Vmix, int l_cap, int32_t* mix_len,
                             int32_t* src_idx, hipStream_t s);
struct KvqPlan {
    int blocks;                                // 16-row blocks of a workgroup; 0: the kernel of many rows
    long long n_rtile;                         // workgroups for the rows
    int n_split;                               // key splits per (query, KV head)
    bool fits;                                 // the grid of the call is one that there can be
    size_t part_ml, total;                     // byte offset of the (reference, sum) of the partial results, bytes of both
};
KvqPlan kvq_plan(const vxl_attn_desc* d, int batch, int T, int l_cap);
vxl_status launch_kvq_decode(const KvqPlan& p, const vxl_attn_desc* d, float scale, const void* Qd, int batch, int T,
                             const vxl_kvq_cache* c, const vxl_kvq_cache* sp, const int32_t* src_idx, int l_cap,
                             const int32_t* mix_len, void* O, float* LSE, void* ws, hipStream_t s);

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) short s16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

constexpr int kBlock = 32;                                    // elements per scale

// Bytes of a row: codes (keys, then values) and scales.
template <int D, int BITS>
struct KvqRow {
    static constexpr int CODES = 2 * D * BITS / 8, SCALES = 2 * D / kBlock;
};

// A quantised cache as the kernels see it: row r of head g is row g * capacity + r.
struct KvqView {
    uint8_t* rows;
    uint8_t* scales;
    long long capacity;
};

// N words of global memory (an address that the compiler cannot tell from one in LDS would be read by a flat load).
template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&to)[N]) {
    typedef __attribute__((ext_vector_type(N))) uint32_t Words;
    const Words x = *(const __attribute__((address_space(1))) Words*)(uintptr_t)p;
#pragma unroll
    for (int i = 0; i < N; ++i) to[i] = x[i];
}
__device__ __forceinline__ uint32_t load_half(const uint8_t* p) { return *(const __attribute__((address_space(1))) uint16_t*)(uintptr_t)p; }

// Scale operand of the conversions, which read its exponent as a scale byte: 255 makes NaN of every code, 0 is 2^-127.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Elements 2 * P and 2 * P + 1 of the codes in `w` (two words for 8 bits).
template <int BITS, int P>
__device__ __forceinline__ bf16x2 two_bf16(const uint32_t* w, float scale) {
    if constexpr (BITS == 4) return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[P / 4], scale, P % 4);
    else return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[P / 2], scale, P % 2);
}

// Eight elements, from BITS / 4 words.
template <int BITS>
__device__ __forceinline__ bf16x8 eight_bf16(const uint32_t* w, float scale) {
    const bf16x2 a = two_bf16<BITS, 0>(w, scale), b = two_bf16<BITS, 1>(w, scale), c = two_bf16<BITS, 2>(w, scale),
                 d = two_bf16<BITS, 3>(w, scale);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

inline KvqView view(const vxl_kvq_cache* c) { return c ? KvqView{(uint8_t*)c->rows, (uint8_t*)c->scales, c->capacity} : KvqView{}; }

// f(D, BITS, F32) as constants.
template <typename F>
vxl_status by_kind(const vxl_attn_desc* d, const vxl_kvq_cache* c, F&& f) {
    auto bits = [&](auto dim) {
        auto type = [&](auto bit) {
            return d->dtype == VXL_F32 ? f(dim, bit, std::true_type{}) : f(dim, bit, std::false_type{});
        };
        return c->format == VXL_KVQ_FP4 ? type(std::integral_constant<int, 4>{}) : type(std::integral_constant<int, 8>{});
    };
    return d->head_dim == 64 ? bits(std::integral_constant<int, 64>{}) : bits(std::integral_constant<int, 128>{});
}

inline vxl_status launched() {
    VXL_HIP_TRY(hipGetLastError());
    return VXL_OK;
}

}  // namespace vxl
