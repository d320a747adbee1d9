// Quantised KV cache: rows written in 8 or 4 bits, read back, and gathered into mixed sets of plain KVs.
//
// A block is 32 consecutive elements x of a key or value row.  With a = max |x| its scale is 2^e,
//   e = floor(log2 a) - emax + [a / 2^floor(log2 a) >= 1.75],   emax = 8 (e4m3), 2 (e2m1),   e >= -110,
// and its codes are x / 2^e rounded to the nearest code, ties to even.  Powers of two make every step but that one rounding
// exact: x / 2^e, and a code times 2^e, which bf16 and fp32 hold as it is.  The largest element lands in [224, 448) or
// [3.5, 7): the bound at 1.75 and not at 2 keeps e4m3 below its largest number, 448, and lets e2m1 round at most 7 to its 6.
// A block whose a is 1.75 * 2^127 or more, infinite or NaN has scale byte 255 and reads back as NaN.
//
// In memory a row has its key codes and then its value codes side by side (128 bytes for D = 128 in 4 bits, a cache line),
// and likewise its scales: a decode that reads scattered rows touches one line for both.
#include <algorithm>

#include "vxl_kvq.h"
#include "vxl_rows.h"

namespace vxl {

namespace {

// ------------------------------------------------------------------------------------------
// 16 bytes of plain elements (8 bf16, 4 fp32) and their codes: N = elements, CB = bytes of codes.
// ------------------------------------------------------------------------------------------
template <bool F32, int BITS>
struct Piece {
    static constexpr int N = F32 ? 4 : 8, CB = N * BITS / 8;

    // Codes of the piece as 32-bit words (the low CB bytes count).
    static __device__ __forceinline__ void encode(uint4 x, float scale, uint32_t (&c)[2]) {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
        c[0] = c[1] = 0;
        if constexpr (F32) {
            const float f[4] = {__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]), __uint_as_float(w[3])};
            if constexpr (BITS == 4) {
                c[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c[0], f[0], f[1], scale, 0);
                c[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c[0], f[2], f[3], scale, 1);
            } else {
                s16x2 r = {0, 0};
                r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, f[0], f[1], scale, false);
                r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, f[2], f[3], scale, true);
                c[0] = __builtin_bit_cast(uint32_t, r);
            }
        } else if constexpr (BITS == 4) {
            c[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c[0], __builtin_bit_cast(bf16x2, w[0]), scale, 0);
            c[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c[0], __builtin_bit_cast(bf16x2, w[1]), scale, 1);
            c[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c[0], __builtin_bit_cast(bf16x2, w[2]), scale, 2);
            c[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c[0], __builtin_bit_cast(bf16x2, w[3]), scale, 3);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                s16x2 r = {0, 0};
                r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, w[2 * i]), scale, false);
                r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, w[2 * i + 1]), scale, true);
                c[i] = __builtin_bit_cast(uint32_t, r);
            }
        }
    }

    static __device__ __forceinline__ uint4 decode(const uint32_t (&c)[2], float scale) {
        if constexpr (F32) {
            f32x2 a, b;
            if constexpr (BITS == 4) {
                a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[0], scale, 0);
                b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[0], scale, 1);
            } else {
                a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[0], scale, false);
                b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[0], scale, true);
            }
            return make_uint4(__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(b[0]), __float_as_uint(b[1]));
        } else {
            return __builtin_bit_cast(uint4, eight_bf16<BITS>(c, scale));
        }
    }

    static __device__ __forceinline__ void load(const uint8_t* p, uint32_t (&c)[2]) {
        c[0] = c[1] = 0;
        if constexpr (CB == 2) c[0] = *(const uint16_t*)p;
        else if constexpr (CB == 4) c[0] = *(const uint32_t*)p;
        else { const uint2 v = *(const uint2*)p; c[0] = v.x; c[1] = v.y; }
    }
    static __device__ __forceinline__ void store(uint8_t* p, const uint32_t (&c)[2]) {
        if constexpr (CB == 2) *(uint16_t*)p = (uint16_t)c[0];
        else if constexpr (CB == 4) *(uint32_t*)p = c[0];
        else *(uint2*)p = make_uint2(c[0], c[1]);
    }

    // Bits of the largest magnitude, as of a float: NaN above infinity above all others.
    static __device__ __forceinline__ uint32_t peak(uint4 x) {
        if constexpr (F32) {
            const uint32_t m = 0x7fffffffu;
            return max(max(x.x & m, x.y & m), max(x.z & m, x.w & m));
        } else {
            typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
            const uint32_t m = 0x7fff7fffu;
            const u16x2 a = __builtin_elementwise_max(__builtin_bit_cast(u16x2, x.x & m), __builtin_bit_cast(u16x2, x.y & m));
            const u16x2 b = __builtin_elementwise_max(__builtin_bit_cast(u16x2, x.z & m), __builtin_bit_cast(u16x2, x.w & m));
            const u16x2 c = __builtin_elementwise_max(a, b);
            return (uint32_t)max(c[0], c[1]) << 16;
        }
    }
};

// Scale byte of a block by the bits of its largest magnitude.
template <int BITS>
__device__ __forceinline__ uint32_t scale_byte(uint32_t peak) {
    if (peak >= 0x7f600000u) return 255;                      // 1.75 * 2^127
    const int e = (int)((peak + 0x200000u) >> 23) - (BITS == 4 ? 2 : 8);
    return (uint32_t)max(e, 127 - 110);
}

// Place of thread `id`: piece `part` of row r of head g (rows of a head one after the other).
template <int LPR>
struct Place {
    long long r;
    int g, part;
    __device__ __forceinline__ Place(long long id, long long n_rows) {
        part = (int)(id % LPR);
        const long long row = id / LPR;
        g = (int)(row / n_rows);
        r = row - g * n_rows;
    }
};

// x of another lane of the same 16 (CTRL: the DPP control).
template <int CTRL>
__device__ __forceinline__ uint32_t from_lane(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true); }
constexpr int kSwap1 = 0xb1, kSwap2 = 0x4e, kMirror8 = 0x141, kShiftLeft = 0x100;

// ------------------------------------------------------------------------------------------
// Rows [first, first + n_rows) of the cache from K and V: a lane takes 16 bytes of a key row and of its value row, the lanes
// of a block find its largest magnitude by exchange, and the first lane of 16 stores the scales of all of them.
// Bound by HBM: 131,328 rows of four heads, 408 MB in and out, 71 us one after the other (5.7 TB/s), 82 where each is read back
// before the next; 16,640 rows 8.1.
// ------------------------------------------------------------------------------------------
template <int D, int BITS, bool F32>
__global__ __launch_bounds__(256) void kvq_write_kernel(const uint4* __restrict__ K, const uint4* __restrict__ V,
                                                        long long head_u4, long long tok_u4, long long n_rows, int n_heads,
                                                        KvqView c, long long first) {
    using P = Piece<F32, BITS>;
    constexpr int LPR = D / P::N, LPB = kBlock / P::N;        // lanes per row, per block
    constexpr int TOGETHER = std::min(16 / LPB, D / kBlock);  // scales that one lane stores, of the keys and of the values
    const long long id = (long long)folded_id() * 256 + threadIdx.x;
    if (id >= n_rows * n_heads * LPR) return;                 // (all lanes of a row)
    const Place<LPR> at(id, n_rows);
    const long long src = at.g * head_u4 + at.r * tok_u4 + at.part;
    const uint4 x[2] = {K[src], V[src]};
    const long long row = at.g * c.capacity + first + at.r;
    uint32_t bytes[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t peak = P::peak(x[i]);
        peak = max(peak, from_lane<kSwap1>(peak));
        peak = max(peak, from_lane<kSwap2>(peak));
        if constexpr (LPB == 8) peak = max(peak, from_lane<kMirror8>(peak));
        const uint32_t byte = scale_byte<BITS>(peak);
        uint32_t code[2] = {0, 0};
        if (byte != 255) P::encode(x[i], scale_of(byte), code);
        P::store(c.rows + row * KvqRow<D, BITS>::CODES + i * (D * BITS / 8) + at.part * P::CB, code);
        bytes[i] = byte;
        if constexpr (TOGETHER > 1) bytes[i] |= from_lane<kShiftLeft + LPB>(byte) << 8;
        if constexpr (TOGETHER > 2) bytes[i] |= from_lane<kShiftLeft + 2 * LPB>(byte) << 16 | from_lane<kShiftLeft + 3 * LPB>(byte) << 24;
    }
    if (at.part % (LPB * TOGETHER) == 0) {
        uint8_t* p = c.scales + row * KvqRow<D, BITS>::SCALES + at.part / LPB;
        if constexpr (TOGETHER == 4) *(uint2*)p = make_uint2(bytes[0], bytes[1]);
        else if constexpr (TOGETHER == D / kBlock) *(uint32_t*)p = bytes[0] | bytes[1] << 16;
        else {
            *(uint16_t*)p = (uint16_t)bytes[0];
            *(uint16_t*)(p + D / kBlock) = (uint16_t)bytes[1];
        }
    }
}

// The codes and scales of 16 bytes of a key row and of its value row as a lane reads them.
template <int D, int BITS, bool F32>
struct PiecePair {
    using P = Piece<F32, BITS>;
    uint32_t code[2][2];
    uint32_t byte[2];
    __device__ __forceinline__ void load(const KvqView& c, long long row, int part) {
        constexpr int LPB = kBlock / P::N;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            P::load(c.rows + row * KvqRow<D, BITS>::CODES + i * (D * BITS / 8) + part * P::CB, code[i]);
            byte[i] = c.scales[row * KvqRow<D, BITS>::SCALES + i * (D / kBlock) + part / LPB];
        }
    }
    template <bool NT = false>
    __device__ __forceinline__ void store(uint4* k, uint4* v) const {
        store16<NT>(k, P::decode(code[0], scale_of(byte[0])));
        store16<NT>(v, P::decode(code[1], scale_of(byte[1])));
    }
};

// K and V from rows [first, first + n_rows) of the cache.  Bound by HBM: the same 71 us, 63 right behind the write.
template <int D, int BITS, bool F32>
__global__ __launch_bounds__(256) void kvq_read_kernel(uint4* __restrict__ K, uint4* __restrict__ V, long long head_u4,
                                                       long long tok_u4, long long n_rows, int n_heads, KvqView c,
                                                       long long first) {
    constexpr int LPR = D / Piece<F32, BITS>::N;
    const long long id = (long long)folded_id() * 256 + threadIdx.x;
    if (id >= n_rows * n_heads * LPR) return;
    const Place<LPR> at(id, n_rows);
    const long long dst = at.g * head_u4 + at.r * tok_u4 + at.part;
    PiecePair<D, BITS, F32> x;
    x.load(c, at.g * c.capacity + first + at.r, at.part);
    x.store(K + dst, V + dst);
}

// ------------------------------------------------------------------------------------------
// Mixed sets of plain KVs from the quantised rows: the blocks find their rows as those of the plain gather do, and a group of
// LPR lanes per row reads codes and scales of HEADS KV heads and writes 16 bytes of keys and of values of each.  The queries
// of a batch take turns, so that the cache's rows stay on the chip for all of them, and sets that would push them out of there
// are stored past the caches (kPastCaches, by their rows).
// Bound by the writes.  us: eight sets of 25k rows of 8 bits, 497 MB, one head after the other 141, four together 123, past the
// caches 96 (5.2 TB/s); one set of 45,312 rows of 4 bits 40 -> 31 -> 28; queries one after the other instead of in turn 129.
// ------------------------------------------------------------------------------------------
template <int D, int BITS, bool F32, int HEADS>
__global__ __launch_bounds__(256) void kvq_gather_kernel(KvqView dense, KvqView sparse, bool pooled,
                                                         const uint8_t* __restrict__ dense_mask, const int32_t* __restrict__ bounds,
                                                         const int32_t* __restrict__ soff, const int32_t* __restrict__ sidx,
                                                         int n_chunks, int n_prefix, int n_kv_heads, int l_cap, int groups, int batch,
                                                         uint4* __restrict__ Kmix, uint4* __restrict__ Vmix,
                                                         int32_t* __restrict__ mix_len, int32_t* __restrict__ src_idx) {
    constexpr int LPR = D / Piece<F32, BITS>::N, ROWS = 256 / LPR;
    extern __shared__ int off[];
    int* from = off + n_chunks;
    const bool table = n_chunks <= kTableChunks;
    __shared__ int wave_tot[4][4];
    const int tid = threadIdx.x, part = tid % LPR;
    const unsigned id = folded_id();
    const int b = (int)(id % batch), block = (int)(id / batch);
    const int len = scan_mixed_rows(dense_mask + (size_t)b * n_chunks, bounds, soff, n_chunks, n_prefix, off, from, table, wave_tot);
    // a mixed set that does not fit l_cap is reported, not truncated: minus the rows it needs
    if (block == 0 && tid == 0) mix_len[b] = len <= l_cap ? len : -len;
    if (len > l_cap) return;
    const bool past = 2ll * batch * n_kv_heads * len * (LPR * 16) > kPastCaches;
    for (int gi = 0; gi < groups; ++gi) {
        const long long r_ = ((long long)block * groups + gi) * ROWS + tid / LPR;
        if (r_ >= len) break;                                 // (rows ascend with gi; the lanes of a row together)
        const int r = (int)r_;
        const int src = mixed_row_source<LPR>(r, n_prefix, n_chunks, off, from, table, bounds, soff, sidx, pooled);
        if (src_idx && part == 0) src_idx[(size_t)b * l_cap + r] = src;
        const KvqView& c = src >= 0 ? dense : sparse;
        const long long row0 = src >= 0 ? src : ~src;
        const size_t head = (size_t)l_cap * LPR, dst = ((size_t)b * n_kv_heads * l_cap + r) * LPR + part;
        for (int g0 = 0; g0 < n_kv_heads; g0 += HEADS) {
            PiecePair<D, BITS, F32> x[HEADS];
#pragma unroll
            for (int g = 0; g < HEADS; ++g) x[g].load(c, (g0 + g) * c.capacity + row0, part);
            auto store = [&](auto nt) __attribute__((always_inline)) {
#pragma unroll
                for (int g = 0; g < HEADS; ++g) x[g].template store<nt>(Kmix + dst + (g0 + g) * head, Vmix + dst + (g0 + g) * head);
            };
            if (past) store(std::true_type{}); else store(std::false_type{});
        }
    }
}

}  // namespace

vxl_status launch_kvq_write(const vxl_attn_desc* d, const void* K, const void* V, int n_rows, const vxl_kvq_cache* c, int first,
                            hipStream_t s) {
    const TokStrides ts = tok_strides(d, n_rows);
    return by_kind(d, c, [&](auto dim, auto bits, auto f32) {
        using P = Piece<f32, bits>;
        const long long blocks = ((long long)n_rows * d->n_kv_heads * (dim / P::N) + 255) / 256;
        hipLaunchKernelGGL((kvq_write_kernel<dim, bits, f32>), folded_grid(blocks), dim3(256), 0, s, (const uint4*)K, (const uint4*)V,
                           ts.kh / P::N, ts.kt / P::N, (long long)n_rows, d->n_kv_heads, view(c), (long long)first);
        return launched();
    });
}

vxl_status launch_kvq_read(const vxl_attn_desc* d, const vxl_kvq_cache* c, int first, int n_rows, void* K, void* V, hipStream_t s) {
    const TokStrides ts = tok_strides(d, n_rows);
    return by_kind(d, c, [&](auto dim, auto bits, auto f32) {
        using P = Piece<f32, bits>;
        const long long blocks = ((long long)n_rows * d->n_kv_heads * (dim / P::N) + 255) / 256;
        hipLaunchKernelGGL((kvq_read_kernel<dim, bits, f32>), folded_grid(blocks), dim3(256), 0, s, (uint4*)K, (uint4*)V, ts.kh / P::N,
                           ts.kt / P::N, (long long)n_rows, d->n_kv_heads, view(c), (long long)first);
        return launched();
    });
}

vxl_status launch_kvq_gather(const vxl_layout* L, const vxl_attn_desc* d, const vxl_kvq_cache* c, const vxl_kvq_cache* sp,
                             const uint8_t* dense_mask, int batch, void* Kmix, void* Vmix, int l_cap, int32_t* mix_len,
                             int32_t* src_idx, hipStream_t s) {
    return by_kind(d, c, [&](auto dim, auto bits, auto f32) {
        constexpr int rows = 256 / (dim / Piece<f32, bits>::N);
        const long long passes = ((long long)l_cap + rows - 1) / rows;
        // passes of a block: one, more where the scan of many chunks is to be shared and blocks enough are left (us, one, two,
        // four passes: 256 chunks 27.9, 30.1, 30.3, 640 chunks 56.5, 56.0, 57.3, 3,500 chunks 157, 116, 96)
        const int groups = (int)std::max<long long>(1, std::min<long long>(std::min(8, 1 + L->n_chunks / 512), passes * batch / 512));
        const size_t lds = (size_t)L->n_chunks * (L->n_chunks <= kTableChunks ? 2 : 1) * sizeof(int);
        auto run = [&](auto heads) {
            hipLaunchKernelGGL((kvq_gather_kernel<dim, bits, f32, heads>), folded_grid((passes + groups - 1) / groups * batch), dim3(256), lds,
                               s, view(c), view(sp), sp != nullptr, dense_mask, L->d_bounds, L->d_soff, L->d_sidx, L->n_chunks, L->n_prefix,
                               d->n_kv_heads, l_cap, groups, batch, (uint4*)Kmix, (uint4*)Vmix, mix_len, src_idx);
        };
        if (d->n_kv_heads % 4 == 0) run(std::integral_constant<int, 4>{});
        else if (d->n_kv_heads % 2 == 0) run(std::integral_constant<int, 2>{});
        else run(std::integral_constant<int, 1>{});
        return launched();
    });
}

}  // namespace vxl
