// Quantised KV cache: rows written in 8 or 4 bits, read back, gathered into mixed sets of plain KVs, and attended to in place.
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

#include "vxl_internal.h"
#include "vxl_mfma.h"
#include "vxl_rows.h"

namespace vxl {

namespace {

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

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte == 255 ? 0x7fc00000u : byte << 23); }

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

// ------------------------------------------------------------------------------------------
// Rows [first, first + n_rows) of the cache from K and V: a lane takes 16 bytes of a key row and of its value row, the lanes
// of a block find its largest magnitude by exchange.
// ------------------------------------------------------------------------------------------
template <int D, int BITS, bool F32>
__global__ __launch_bounds__(256) void kvq_write_kernel(const uint4* __restrict__ K, const uint4* __restrict__ V,
                                                        long long head_u4, long long tok_u4, long long n_rows, int n_heads,
                                                        KvqView c, long long first) {
    using P = Piece<F32, BITS>;
    constexpr int LPR = D / P::N, LPB = kBlock / P::N;        // lanes per row, per block
    const long long id = (long long)folded_id() * 256 + threadIdx.x;
    if (id >= n_rows * n_heads * LPR) return;                 // (all lanes of a row)
    const Place<LPR> at(id, n_rows);
    const long long src = at.g * head_u4 + at.r * tok_u4 + at.part;
    const uint4 x[2] = {K[src], V[src]};
    const long long row = at.g * c.capacity + first + at.r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t peak = P::peak(x[i]);
#pragma unroll
        for (int o = 1; o < LPB; o <<= 1) peak = max(peak, (uint32_t)__shfl_xor((int)peak, o));
        const uint32_t byte = scale_byte<BITS>(peak);
        uint32_t code[2] = {0, 0};
        if (byte != 255) P::encode(x[i], scale_of(byte), code);
        P::store(c.rows + row * KvqRow<D, BITS>::CODES + i * (D * BITS / 8) + at.part * P::CB, code);
        if (at.part % LPB == 0) c.scales[row * KvqRow<D, BITS>::SCALES + i * (D / kBlock) + at.part / LPB] = (uint8_t)byte;
    }
}

// K and V from rows [first, first + n_rows) of the cache.
template <int D, int BITS, bool F32>
__global__ __launch_bounds__(256) void kvq_read_kernel(uint4* __restrict__ K, uint4* __restrict__ V, long long head_u4,
                                                       long long tok_u4, long long n_rows, int n_heads, KvqView c,
                                                       long long first) {
    using P = Piece<F32, BITS>;
    constexpr int LPR = D / P::N, LPB = kBlock / P::N;
    const long long id = (long long)folded_id() * 256 + threadIdx.x;
    if (id >= n_rows * n_heads * LPR) return;
    const Place<LPR> at(id, n_rows);
    const long long row = at.g * c.capacity + first + at.r, dst = at.g * head_u4 + at.r * tok_u4 + at.part;
    uint32_t code[2][2];
    float scale[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        P::load(c.rows + row * KvqRow<D, BITS>::CODES + i * (D * BITS / 8) + at.part * P::CB, code[i]);
        scale[i] = scale_of(c.scales[row * KvqRow<D, BITS>::SCALES + i * (D / kBlock) + at.part / LPB]);
    }
    K[dst] = P::decode(code[0], scale[0]);
    V[dst] = P::decode(code[1], scale[1]);
}

// ------------------------------------------------------------------------------------------
// Mixed sets of plain KVs from the quantised rows: the blocks find their rows as those of the plain gather do, a group of
// LPR lanes per row reads codes and scales and writes 16 bytes of keys and of values each, head by head.
// ------------------------------------------------------------------------------------------
template <int D, int BITS, bool F32>
__global__ __launch_bounds__(256) void kvq_gather_kernel(KvqView dense, KvqView sparse, bool pooled,
                                                         const uint8_t* __restrict__ dense_mask, const int32_t* __restrict__ bounds,
                                                         const int32_t* __restrict__ soff, const int32_t* __restrict__ sidx,
                                                         int n_chunks, int n_prefix, int n_kv_heads, int l_cap, int groups,
                                                         uint4* __restrict__ Kmix, uint4* __restrict__ Vmix,
                                                         int32_t* __restrict__ mix_len, int32_t* __restrict__ src_idx) {
    using P = Piece<F32, BITS>;
    constexpr int LPR = D / P::N, LPB = kBlock / P::N, ROWS = 256 / LPR;
    extern __shared__ int off[];
    int* from = off + n_chunks;
    const bool table = n_chunks <= kTableChunks;
    __shared__ int wave_tot[4][4];
    const int tid = threadIdx.x, part = tid % LPR, b = blockIdx.y, block = blockIdx.x;
    const int len = scan_mixed_rows(dense_mask + (size_t)b * n_chunks, bounds, soff, n_chunks, n_prefix, off, from, table, wave_tot);
    // a mixed set that does not fit l_cap is reported, not truncated: minus the rows it needs
    if (block == 0 && tid == 0) mix_len[b] = len <= l_cap ? len : -len;
    if (len > l_cap) return;
    for (int gi = 0; gi < groups; ++gi) {
        const int r = (block * groups + gi) * ROWS + tid / LPR;
        if (r >= len) break;                                  // (rows ascend with gi; the lanes of a row together)
        const int src = mixed_row_source<LPR>(r, n_prefix, n_chunks, off, from, table, bounds, soff, sidx, pooled);
        if (src_idx && part == 0) src_idx[(size_t)b * l_cap + r] = src;
        const KvqView& c = src >= 0 ? dense : sparse;
        const long long row0 = src >= 0 ? src : ~src;
        for (int g = 0; g < n_kv_heads; ++g) {
            const long long row = g * c.capacity + row0;
            const size_t dst = (((size_t)b * n_kv_heads + g) * l_cap + r) * LPR + part;
            uint32_t code[2][2];
            float scale[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                P::load(c.rows + row * KvqRow<D, BITS>::CODES + i * (D * BITS / 8) + part * P::CB, code[i]);
                scale[i] = scale_of(c.scales[row * KvqRow<D, BITS>::SCALES + i * (D / kBlock) + part / LPB]);
            }
            Kmix[dst] = P::decode(code[0], scale[0]);
            Vmix[dst] = P::decode(code[1], scale[1]);
        }
    }
}

// ------------------------------------------------------------------------------------------
// Decode in place.  16 stacked query rows per workgroup (row rho = t * G + head of the group), four waves that each walk
// 32-key tiles of the workgroup's split on their own; their (reference, sum, O) are merged through LDS in wave order, the
// splits by the kernel below.
//
// S^T = K Q^T by v_mfma_f32_16x16x32_bf16: lane (l16, q) holds of the A operand row l16, k-slots 8 q .. 8 q + 7, of B the
// same slots of column l16, of the result column l16, rows 4 q .. 4 q + 3.  A lane loads D / 4 consecutive elements of one
// key, those from q * D / 4 on, which lie in one block, and takes them eight at a time as the slots of step i: the order of
// the summation index is free as long as Q has the same.  So key codes go from memory to the matrix cores through one
// conversion with one scale per lane, and never through LDS.
// O^T = V^T P^T: the result registers of the two 16-key halves of a tile are, eight per lane, the slots of P^T for the keys
// 4 q + {0..3} and 16 + 4 q + {0..3}; V^T of the same keys comes transposed out of LDS, where a wave keeps the converted
// rows of its tile.  32-byte pieces of a row are swizzled by its number, halves of 16 bytes by its fourth bit: the writes
// (16 rows at one piece) and the reads (8 rows at one piece per half-wave) both touch every bank evenly.
//
// Quantised values are bf16 numbers.  bf16 queries are the operand as they are; fp32 queries, and probabilities of an fp32
// call, go in as three bf16 parts that add up to all 24 bits (three matrix instructions instead of one).  Probabilities of a
// bf16 call are rounded to bf16 (2^-9 relative at most, of each weight), their sum is taken before that, in fp32.
// ------------------------------------------------------------------------------------------
constexpr int kKvqTile = 32, kKvqWaves = 4, kKvqRows = 16;

template <bool F32> struct Parts { static constexpr int N = F32 ? 3 : 1; };

// x as bf16 parts, each the rounding of what the ones before it leave.
template <int N>
__device__ __forceinline__ void split_bf16(float x, __bf16 (&part)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        part[i] = (__bf16)x;
        if (i + 1 < N) x -= (float)part[i];
    }
}

__device__ __forceinline__ uint16_t to_bf16_bits(float v) {
    const uint32_t b = __float_as_uint(v);
    return (b & 0x7fffffffu) > 0x7f800000u ? 0x7fc0 : (uint16_t)((b + 0x7fffu + ((b >> 16) & 1u)) >> 16);
}
__device__ __forceinline__ void store4(float* p, const float (&v)[4]) { *(float4*)p = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void store4(uint16_t* p, const float (&v)[4]) {
    __attribute__((aligned(8))) const uint16_t o[4] = {to_bf16_bits(v[0]), to_bf16_bits(v[1]), to_bf16_bits(v[2]), to_bf16_bits(v[3])};
    *(uint2*)p = *(const uint2*)o;
}

template <bool F32> struct Elem { using T = uint16_t; };
template <> struct Elem<true> { using T = float; };

// Byte offset in a wave's V tile of 16-byte half `half` of 32-byte piece `piece` of row `key`.
template <int D>
__device__ __forceinline__ int kvq_v_off(int key, int piece, int half) {
    const int turn = D == 128 ? key & 7 : (key >> 1) & 3;
    return key * (D * 2) + ((piece ^ turn) << 5) + ((half ^ ((key >> 3) & 1)) << 4);
}

template <int D, int BITS, bool F32>
__global__ __launch_bounds__(256, 2) void kvq_decode_kernel(
    const typename Elem<F32>::T* __restrict__ Qd, KvqView dense, KvqView sparse, const int32_t* __restrict__ src_idx,
    const int32_t* __restrict__ mix_len, float* __restrict__ part_o, float2* __restrict__ part_ml, int T_q, int n_q_heads,
    int n_kv_heads, int l_cap, int tiles_per_wave, int n_split, int n_rtile, int batch, float c2,
    typename Elem<F32>::T* __restrict__ O, float* __restrict__ LSE) {
    constexpr int NP = Parts<F32>::N, PB = D / 4 * BITS / 8, W = PB / 4, SW = KvqRow<D, BITS>::SCALES / 4, STEPS = D / 32, DB = D / 16;
    __shared__ __attribute__((aligned(16))) uint8_t tiles[kKvqWaves][kKvqTile * D * 2];
    __shared__ float2 stats[kKvqWaves][kKvqRows];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // Workgroups that read the same keys (row tiles, and queries, whose sets overlap) are neighbours on one XCD, whose L2
    // serves all but the first: id = (pair / 8 * members + member) * 8 + pair % 8, pair = (KV head, split).
    const int pairs = n_kv_heads * n_split, members = n_rtile * batch;
    int pair, member;
    {
        const long long id = folded_id();
        if (pairs >= kXcds) {
            const long long seq = id / kXcds;
            pair = (int)(seq / members) * kXcds + (int)(id % kXcds);
            member = (int)(seq % members);
        } else {
            pair = (int)(id / members);
            member = (int)(id % members);
        }
        if (pair >= pairs) return;
    }
    const int g = pair / n_split, split = pair % n_split, b = member / n_rtile, row0 = member % n_rtile * kKvqRows;
    const int group = n_q_heads / n_kv_heads, all_rows = group * T_q, n_rows = min(kKvqRows, all_rows - row0);

    const int32_t* map = src_idx + (size_t)b * l_cap;
    const uint8_t* rows_d = dense.rows + (size_t)g * dense.capacity * KvqRow<D, BITS>::CODES + q * PB;
    const uint8_t* rows_s = sparse.rows + (size_t)g * sparse.capacity * KvqRow<D, BITS>::CODES + q * PB;
    const uint8_t* scales_d = dense.scales + (size_t)g * dense.capacity * KvqRow<D, BITS>::SCALES;
    const uint8_t* scales_s = sparse.scales + (size_t)g * sparse.capacity * KvqRow<D, BITS>::SCALES;
    const int block = D == 128 ? q : q >> 1;                  // the lane's block of a row

    struct Tile {
        uint32_t k[2][W], v[2][W], s[2][SW];                  // by half: 16 keys each
    };
    const int tile0 = split * tiles_per_wave * kKvqWaves + wave;
    const int len = min(max(mix_len[b], 0), l_cap), n_tiles = (len + kKvqTile - 1) / kKvqTile;
    // (entries up to the capacity, so that the first ones do not wait for the length; behind the length they may be
    // anything, and row 0 is read there instead, whose values do not count)
    auto entries = [&](int tile, int (&e)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) e[h] = map[min((long long)tile * kKvqTile + h * 16 + l16, (long long)l_cap - 1)];
    };
    auto request = [&](int tile, const int (&e)[2], Tile& t) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = tile * kKvqTile + h * 16 + l16 < len ? e[h] : 0;
            const size_t row = at >= 0 ? at : ~at;
            const uint8_t* p = (at >= 0 ? rows_d : rows_s) + row * KvqRow<D, BITS>::CODES;
            const uint8_t* s = (at >= 0 ? scales_d : scales_s) + row * KvqRow<D, BITS>::SCALES;
            if constexpr (SW == 2) { const uint2 v = *(const uint2*)s; t.s[h][0] = v.x; t.s[h][1] = v.y; }
            else t.s[h][0] = *(const uint32_t*)s;
            auto piece = [&](const uint8_t* from, uint32_t (&to)[W]) __attribute__((always_inline)) {
                if constexpr (W == 2) { const uint2 v = *(const uint2*)from; to[0] = v.x; to[1] = v.y; }
                else {
#pragma unroll
                    for (int i = 0; i < W; i += 4) {
                        const uint4 v = *(const uint4*)(from + i * 4);
                        to[i] = v.x; to[i + 1] = v.y; to[i + 2] = v.z; to[i + 3] = v.w;
                    }
                }
            };
            piece(p, t.k[h]);
            piece(p + D * BITS / 8, t.v[h]);
        }
    };

    // Q: step i of row l16 has its elements q * D / 4 + 8 i + {0..7}
    bf16x8 qreg[NP][STEPS];
    {
        const int rho = row0 + min(l16, n_rows - 1);
        const auto* src = Qd + (((size_t)b * T_q + rho / group) * n_q_heads + g * group + rho % group) * D + q * (D / 4);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            if constexpr (F32) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    __bf16 part[NP];
                    split_bf16(src[i * 8 + j], part);
#pragma unroll
                    for (int p = 0; p < NP; ++p) qreg[p][i][j] = part[p];
                }
            } else {
                qreg[0][i] = *(const bf16x8*)(src + i * 8);
            }
        }
    }
    f32x4 o[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;
    uint8_t* vt = tiles[wave];

    auto work = [&](int tile, const Tile& t) __attribute__((always_inline)) {
        const int left = len - tile * kKvqTile;               // keys of the tile that count
        f32x4 s[2];
        uint32_t v[2][W];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const bool there = h * 16 + l16 < left;
            // (a row that does not count has scale 1 and codes 0: its own may be NaN)
            const uint32_t ks = t.s[h][0] >> (8 * block) & 255, vs = (SW == 2 ? t.s[h][1] >> (8 * block) : t.s[h][0] >> (16 + 8 * block)) & 255;
            const float kscale = there ? scale_of(ks) : 1.f, vscale = there ? scale_of(vs) : 1.f;
            uint32_t k[W];
#pragma unroll
            for (int i = 0; i < W; ++i) { k[i] = there ? t.k[h][i] : 0; v[h][i] = there ? t.v[h][i] : 0; }
            s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const bf16x8 a = eight_bf16<BITS>(k + i * (BITS / 4), kscale);
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qreg[p][i], s[h], 0, 0, 0);
            }
            const int key = h * 16 + l16;
#pragma unroll
            for (int i = 0; i < STEPS; ++i)
                *(bf16x8*)(vt + kvq_v_off<D>(key, D == 128 ? 2 * q + i / 2 : q, i & 1)) = eight_bf16<BITS>(v[h] + i * (BITS / 4), vscale);
        }
        __builtin_amdgcn_wave_barrier();
        if (left < kKvqTile) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[h][r] = h * 16 + 4 * q + r < left ? s[h][r] : -INFINITY;
        }
        // The reference is raised, and sums and O rescaled, only when a logit is more than 2^8 above it: until then the
        // weights stay in a range that bf16 and fp32 hold with unchanged relative precision.
        float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        if (__builtin_amdgcn_ballot_w64((mx - m_run) * c2 > 8.f) != 0) {
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float m_new = fmaxf(m_run, mx);
            const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m_run - m_new) * c2);
            l_run *= alpha;
            m_run = m_new;
#pragma unroll
            for (int i = 0; i < DB; ++i) o[i] *= alpha;
        }
        const float mc = (m_run == -INFINITY ? 0.f : m_run) * c2;
        bf16x8 pb[NP];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float p = __builtin_amdgcn_exp2f(fmaf(s[h][r], c2, -mc));
                l_run += p;
                __bf16 part[NP];
                split_bf16(p, part);
#pragma unroll
                for (int i = 0; i < NP; ++i) pb[i][h * 4 + r] = part[i];
            }
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const int key = 4 * q + (l16 >> 2);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const uint8_t* p = vt + kvq_v_off<D>(key, db, (l16 >> 1) & 1) + (l16 & 1) * 8;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 16 * D * 2));     // key + 16: same swizzle
            const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int i = NP - 1; i >= 0; --i) o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pb[i], o[db], 0, 0, 0);
        }
        __builtin_amdgcn_wave_barrier();
    };

    int e[2];
    Tile t;
    if (tile0 * (long long)kKvqTile < l_cap) entries(tile0, e);
    for (int i = 0; i < tiles_per_wave; ++i) {
        const int tile = tile0 + i * kKvqWaves;
        if (tile >= n_tiles) break;
        if (i) entries(tile, e);
        request(tile, e, t);
        work(tile, t);
    }

    // ---- merge the waves: 16-byte piece c of row r lies at c ^ r (mod the pieces), which spreads the rows over the banks ----
    constexpr int PPR = D / 4;
    l_run += __shfl_xor(l_run, 16);
    l_run += __shfl_xor(l_run, 32);
    float4* red = (float4*)vt;
    static_assert(kKvqRows * D * 4 <= sizeof(tiles[0]), "the merge area is the wave's tile");
#pragma unroll
    for (int db = 0; db < DB; ++db)
        red[l16 * PPR + ((db * 4 + q) ^ (l16 & (PPR - 1)))] = make_float4(o[db][0], o[db][1], o[db][2], o[db][3]);
    if (q == 0) stats[wave][l16] = make_float2(m_run, l_run);
    __syncthreads();
    const size_t part_base = (((size_t)b * n_kv_heads + g) * n_split + split) * (size_t)all_rows + row0;
    for (int i = tid; i < n_rows * PPR; i += 64 * kKvqWaves) {
        const int row = i / PPR, c = i % PPR;
        float M = -INFINITY, L = 0.f, a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kKvqWaves; ++w) M = fmaxf(M, stats[w][row].x);
#pragma unroll
        for (int w = 0; w < kKvqWaves; ++w) {
            const float2 st = stats[w][row];
            const float4 v = ((const float4*)tiles[w])[row * PPR + (c ^ (row & (PPR - 1)))];
            const float f = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((st.x - M) * c2);
            L = fmaf(f, st.y, L);
            a[0] = fmaf(f, v.x, a[0]); a[1] = fmaf(f, v.y, a[1]); a[2] = fmaf(f, v.z, a[2]); a[3] = fmaf(f, v.w, a[3]);
        }
        if (n_split == 1) {
            const int rho = row0 + row;
            const size_t out = ((size_t)b * T_q + rho / group) * n_q_heads + g * group + rho % group;
#pragma unroll
            for (int j = 0; j < 4; ++j) a[j] = len > 0 ? a[j] / L : 0.f;
            store4(O + out * D + c * 4, a);
            if (LSE && c == 0) LSE[out] = len > 0 ? (M * c2 + __builtin_amdgcn_logf(L)) * kLn2 : -INFINITY;
        } else {
            store4(part_o + (part_base + row) * D + c * 4, a);
            if (c == 0) part_ml[part_base + row] = make_float2(M * c2, L);
        }
    }
}

// The merge of the splits, one workgroup per query row: SG groups of D / 4 lanes take every SG-th split, U of them requested
// together, and are folded through LDS; the order depends on the split index alone.
template <int D, bool F32>
__global__ __launch_bounds__(256) void kvq_merge_kernel(const float* __restrict__ part_o, const float2* __restrict__ part_ml,
                                                        typename Elem<F32>::T* __restrict__ O, float* __restrict__ LSE,
                                                        const int32_t* __restrict__ mix_len, int T_q, int n_q_heads,
                                                        int n_kv_heads, int n_split, int batch) {
    constexpr int NV = D / 4, SG = 256 / NV, U = 4;
    __shared__ __attribute__((aligned(16))) float red[SG][D];
    __shared__ float2 stat[SG];
    const int group = n_q_heads / n_kv_heads, n_rows = T_q * group, sg = threadIdx.x / NV, d = threadIdx.x % NV * 4;
    const long long id = folded_id();
    const int rho = (int)(id % n_rows);
    const long long unit = id / n_rows;                       // (query, KV head)
    if (unit >= (long long)batch * n_kv_heads) return;
    const int g = (int)(unit % n_kv_heads), b = (int)(unit / n_kv_heads);
    const size_t base = (size_t)unit * n_split * n_rows + rho;
    float M = -INFINITY, L = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = sg; s0 < n_split; s0 += U * SG) {
        float2 ml[U];
        float4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {                         // (behind the last split its own values again, not counted)
            const size_t at = base + (size_t)min(s0 + u * SG, n_split - 1) * n_rows;
            ml[u] = part_ml[at];
            v[u] = *(const float4*)(part_o + at * D + d);
        }
        float m_new = M;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (s0 + u * SG < n_split) m_new = fmaxf(m_new, ml[u].x);
        const float ref = m_new == -INFINITY ? 0.f : m_new, f0 = __builtin_amdgcn_exp2f(M - ref);
        M = m_new;
        L *= f0;
        a.x *= f0; a.y *= f0; a.z *= f0; a.w *= f0;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (s0 + u * SG < n_split) {
                const float f = __builtin_amdgcn_exp2f(ml[u].x - ref);
                L = fmaf(f, ml[u].y, L);
                a.x = fmaf(f, v[u].x, a.x); a.y = fmaf(f, v[u].y, a.y);
                a.z = fmaf(f, v[u].z, a.z); a.w = fmaf(f, v[u].w, a.w);
            }
    }
    *(float4*)(&red[sg][d]) = a;
    if (d == 0) stat[sg] = make_float2(M, L);
    __syncthreads();
    if (threadIdx.x >= D / 4) return;
    M = stat[0].x;
#pragma unroll
    for (int i = 1; i < SG; ++i) M = fmaxf(M, stat[i].x);
    const float ref = M == -INFINITY ? 0.f : M;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    L = 0.f;
#pragma unroll
    for (int i = 0; i < SG; ++i) {
        const float f = __builtin_amdgcn_exp2f(stat[i].x - ref);
        const float4 v = *(const float4*)(&red[i][d]);
        L = fmaf(f, stat[i].y, L);
        sum[0] = fmaf(f, v.x, sum[0]); sum[1] = fmaf(f, v.y, sum[1]);
        sum[2] = fmaf(f, v.z, sum[2]); sum[3] = fmaf(f, v.w, sum[3]);
    }
    const bool some = mix_len[b] > 0;
    const size_t row = ((size_t)b * T_q + rho / group) * n_q_heads + g * group + rho % group;
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] = some ? sum[j] / L : 0.f;
    store4(O + row * D + d, sum);
    if (LSE && d == 0) LSE[row] = some ? (M + __builtin_amdgcn_logf(L)) * kLn2 : -INFINITY;
}

KvqView view(const vxl_kvq_cache* c) { return c ? KvqView{(uint8_t*)c->rows, (uint8_t*)c->scales, c->capacity} : KvqView{}; }

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

vxl_status launched() {
    VXL_HIP_TRY(hipGetLastError());
    return VXL_OK;
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
        const int groups = (int)std::max<long long>(1, std::min<long long>(8, passes * batch / 512));
        const size_t lds = (size_t)L->n_chunks * (L->n_chunks <= kTableChunks ? 2 : 1) * sizeof(int);
        hipLaunchKernelGGL((kvq_gather_kernel<dim, bits, f32>), dim3((unsigned)((passes + groups - 1) / groups), batch), dim3(256), lds, s,
                           view(c), view(sp), sp != nullptr, dense_mask, L->d_bounds, L->d_soff, L->d_sidx, L->n_chunks, L->n_prefix,
                           d->n_kv_heads, l_cap, groups, (uint4*)Kmix, (uint4*)Vmix, mix_len, src_idx);
        return launched();
    });
}

KvqPlan kvq_plan(const vxl_attn_desc* d, int batch, int T, int l_cap) {
    KvqPlan p{};
    const long long rows = (long long)(d->n_q_heads / d->n_kv_heads) * T, units = (long long)batch * d->n_kv_heads;
    const long long tiles = ((long long)l_cap + kKvqTile - 1) / kKvqTile;
    p.n_rtile = (int)((rows + kKvqRows - 1) / kKvqRows);
    long long n_split = std::max<long long>(1, std::min<long long>((tiles + kKvqWaves - 1) / kKvqWaves, 1024 / (units * p.n_rtile)));
    p.tiles_per_wave = (int)((tiles + kKvqWaves * n_split - 1) / (kKvqWaves * n_split));
    p.n_split = (int)((tiles + kKvqWaves * p.tiles_per_wave - 1) / (kKvqWaves * p.tiles_per_wave));
    if (p.n_split > 1) {
        p.part_ml = align_up((size_t)units * p.n_split * rows * d->head_dim * sizeof(float), 256);
        p.total = p.part_ml + align_up((size_t)units * p.n_split * rows * sizeof(float2), 256);
    }
    return p;
}

vxl_status launch_kvq_decode(const KvqPlan& p, const vxl_attn_desc* d, float scale, const void* Qd, int batch, int T,
                             const vxl_kvq_cache* c, const vxl_kvq_cache* sp, const int32_t* src_idx, int l_cap,
                             const int32_t* mix_len, void* O, float* LSE, void* ws, hipStream_t s) {
    float* part_o = (float*)ws;
    float2* part_ml = (float2*)((char*)ws + p.part_ml);
    const long long pairs = (long long)d->n_kv_heads * p.n_split, members = (long long)p.n_rtile * batch;
    const long long blocks = (pairs >= kXcds ? (pairs + kXcds - 1) / kXcds * kXcds : pairs) * members;
    return by_kind(d, c, [&](auto dim, auto bits, auto f32) {
        using T_ = typename Elem<f32>::T;
        hipLaunchKernelGGL((kvq_decode_kernel<dim, bits, f32>), folded_grid(blocks), dim3(64 * kKvqWaves), 0, s, (const T_*)Qd, view(c),
                           view(sp), src_idx, mix_len, part_o, part_ml, T, d->n_q_heads, d->n_kv_heads, l_cap, p.tiles_per_wave,
                           p.n_split, p.n_rtile, batch, scale * kLog2e, (T_*)O, LSE);
        const vxl_status st = launched();
        if (st != VXL_OK || p.n_split == 1) return st;
        const long long rows = (long long)(d->n_q_heads / d->n_kv_heads) * T;
        hipLaunchKernelGGL((kvq_merge_kernel<dim, f32>), folded_grid(rows * d->n_kv_heads * batch), dim3(256), 0, s, part_o, part_ml,
                           (T_*)O, LSE, mix_len, T, d->n_q_heads, d->n_kv_heads, p.n_split, batch);
        return launched();
    });
}

}  // namespace vxl
