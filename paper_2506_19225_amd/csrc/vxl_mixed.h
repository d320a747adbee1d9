// Rotary positions and growing mixed sets: their launches, and what their host and device code share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "vxl_internal.h"
#include "vxl_round.h"

namespace vxl {

// ---- rotary positions ----
vxl_status launch_rotate(const vxl_attn_desc* d, const vxl_rotary* r, const int32_t* positions, int n_tokens, const void* Q, const void* K,
                         void* Q_out, void* K_out, hipStream_t s);
vxl_status launch_mixed_append(const vxl_attn_desc* d, const vxl_rotary* r, const int32_t* positions, int batch, int n_new, const void* Q,
                               const void* K, const void* V, void* Qd, void* Kmix, void* Vmix, int l_cap, const int32_t* mix_len,
                               int32_t* row_pos, float* row_weight, hipStream_t s);

// ---- attention by position ----
struct MixedPlan {
    bool fits;                 // the grids of the call are ones that there can be
    int waves, n_split;        // of the ring's workgroups; key splits
    bool few;                  // at most 32 stacked query rows: the kernel that keeps its logits
    int stride;                // of a query row's logits
    int n_part;                // parts of the query rows in the second pass for the weights
    // byte offsets into the workspace
    size_t lse2;               // base-2 LSE [batch][Hkv][rows]
    size_t part_o, part_ml;    // results of the splits
    size_t logits;             // of a few query rows [batch][Hkv][rows][stride]
    size_t part_w;             // weights of the parts [n_part][batch][Hkv][l_cap]
    size_t total;
};
MixedPlan mixed_plan(const vxl_attn_desc* d, int batch, int T, int l_cap);
struct MixedCall {
    const vxl_attn_desc* d;
    const vxl_score_rule* rule;
    float scale;
    const void* Qd;
    const int32_t* q_pos;      // null: no positions
    int batch, T;
    const void *Kmix, *Vmix;
    int l_cap;
    const int32_t *mix_len, *row_pos;
    void* O;
    float* LSE;
    const float* weight;
    float* weight_out;
    char* ws;
};
vxl_status launch_mixed_attend(const MixedPlan& p, const MixedCall& c, bool force_simple, hipStream_t s);

// ---- eviction ----
struct EvictPlan {
    size_t map;                // byte offset of [batch][Hkv][l_cap] source rows
    size_t n;                  // of [batch] numbers of rows kept
    size_t states;             // of what the launches of long sets leave each other
    size_t total;
};
EvictPlan evict_plan(const vxl_attn_desc* d, int batch, int l_cap);
struct EvictCall {
    const vxl_attn_desc* d;
    const void *Kmix, *Vmix;
    int l_cap;
    const int32_t* mix_len;
    const float* weight;
    const int32_t *row_pos, *newest;
    int batch, keep, n_first, n_recent;
    void *Kout, *Vout;
    int out_cap;
    float* weight_out;
    int32_t *pos_out, *kept;
    char* ws;
};
vxl_status launch_mixed_evict(const EvictPlan& p, const EvictCall& c, hipStream_t s);

inline vxl_status mixed_launched() {
    VXL_HIP_TRY(hipGetLastError());
    return VXL_OK;
}

// Storage types.
template <bool F32> struct Storage { using T = uint16_t; };
template <> struct Storage<true> { using T = float; };
__device__ __forceinline__ float as_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ void store_as(uint16_t* p, float v) { *p = f32_to_bf16(v); }
__device__ __forceinline__ void store_as(float* p, float v) { *p = v; }

// f(F32, D) as constants.
template <typename F>
vxl_status by_storage(const vxl_attn_desc* d, F&& f) {
    auto dim = [&](auto f32) {
        return d->head_dim == 64 ? f(f32, std::integral_constant<int, 64>{}) : f(f32, std::integral_constant<int, 128>{});
    };
    return d->dtype == VXL_F32 ? dim(std::true_type{}) : dim(std::false_type{});
}

}  // namespace vxl
