// Decode attention over a quantised KV cache, its rows read in place through a row map (bf16 and fp32 queries, matrix cores).
#include <algorithm>
#include <limits>

#include "vxl_kvq.h"
#include "vxl_round.h"

namespace vxl {

namespace {

// ------------------------------------------------------------------------------------------
// Decode in place.  16 NB stacked query rows per workgroup (row rho = t * G + head of the group), four waves that each walk
// 32-key tiles of the workgroup's split on their own; their (reference, sum, O) are merged through LDS in wave order, the
// splits by the kernel below.
//
// Both products by v_mfma_f32_16x16x32_bf16: lane (l16, q) holds of the A operand row l16, slots 8 q .. 8 q + 7 of the
// summation, of B the same slots of column l16, of the result column l16, rows 4 q .. 4 q + 3.
//   S^T = K Q^T, summed over d, in any order that Q has too: a lane takes D / 4 consecutive elements of one key, which lie in
// one block, eight at a time.  The loads are of 16-byte chunks of a row by neighbouring lanes (the operand's own order, a lane
// per key, asks the vector cache for a line per lane: 300 look-ups a tile instead of 110, and it was bound by them); the codes
// pass through LDS as they are.
//   O^T = V^T P^T, summed over keys.  A lane's slots of P^T are its result registers of the two halves of a tile, rows 4 q + r;
// as these rows stand for keys 4 r + q of their half, so the lane needs of V the keys 16 h + 4 r + q.  It loads D / 16
// consecutive elements of each, the l16-th piece of the row (a load: four whole rows), and row l16 of matrix instruction m
// is element m of that piece: the transposition of keys and elements happens between the registers of a lane (conversions
// make pairs of elements, a byte permutation makes pairs of keys of them), and V never passes through LDS.  Through it, as
// converted rows read back transposed, a tile cost the LDS 316 cycles instead of 100, and the kernel was bound by that.
//
// Quantised values are bf16 numbers.  bf16 queries are the operand as they are; fp32 queries, and probabilities of an fp32
// call, go in as three bf16 parts that add up to all 24 bits (three matrix instructions instead of one).  Probabilities of a
// bf16 call are rounded to bf16 (2^-8 relative at most, of each weight), their sum is taken before that, in fp32: a result is off
// by up to 2^-8 of sum p |v| before it is rounded itself, and the LSE by fp32's roundings only.  The plain decode divides by the
// sum of the rounded weights, so that a row that one key dominates comes out exact there; elsewhere that has up to twice the
// error, 2^-8 (sum p |v| + |o|), and its sum is not the LSE's.  Both sums, O scaled by their quotient: 1 to 3 % slower; weights in
// two bf16 parts, which leave fp32's error alone: 11 to 26 %; the reference raised by every weight that outweighs the ones before
// it, which is 1 then: 1 to 8 %.
//
// Measured (us, launches with their merge; D = 128, 28 heads on 4): one token, 4,096 keys in 4 bits 7.4 to 8.5 and 18,176 keys in
// 8 bits 11.0 (two dependent launches; a plain decode in place 8.9 and 12.7; 28 layers in turn, none of whose rows is still in an
// L2, 7.6 and 13.0), eight queries' tokens, 64.5k keys each in 4 bits 34 (plain 83.9): vector instructions 74 % and matrix
// instructions 23 % of the cycles; 64 of the 174 vector instructions of a tile are conversions, 32 byte permutations, 8
// exponentials.  A question of 64 tokens, 448 rows by 32 (NB = 2) over 23,800 keys in 4 bits 42.5 (38.7 of them here, 64 % and
// 28 %, 560 TFLOP/s), in 8 bits 45 to 49.
// ------------------------------------------------------------------------------------------
// The workgroup's KV head, split, query and first row.  Workgroups that read the same keys (row tiles, and queries, whose sets
// overlap) are members of a pair (KV head, split), one behind the other on one XCD, whose L2 serves all but the first: workgroups
// go to the XCDs in turn, so the grid is eight (fewer, if there are no more) x as many as each takes, whatever the number of pairs
// (whole pairs on an XCD: 448 rows, 23,800 keys, four heads 45.5 us instead of 42.4; a split's heads together, not a head's splits:
// 1,792 rows, 21.7k keys 95.7 instead of 93.8).
__device__ __forceinline__ bool kvq_place(int n_kv_heads, int n_split, int n_rtile, int members, int rows, int* g, int* split, int* b,
                                          int* row0) {
    const unsigned all = (unsigned)(n_kv_heads * n_split * members), each = (all + gridDim.x - 1) / gridDim.x;
    const unsigned own = blockIdx.z * gridDim.y + blockIdx.y, id = blockIdx.x * each + own;
    if (own >= each || id >= all) return false;
    const int pair = (int)(id / members), member = (int)(id % members);
    *g = pair / n_split;
    *split = pair % n_split;
    *b = member / n_rtile;
    *row0 = member % n_rtile * rows;
    return true;
}

constexpr int kKvqTile = 32, kKvqWaves = 4;

// A row's reference in the units that weights are exponentials of: never -inf, also where the row has met no logit above it (as
// scaled) yet, but its neighbours in the wave have and raise theirs.  The first one that it meets raises it then, and a logit
// of -inf has weight 0.
constexpr float kLowest = -std::numeric_limits<float>::max();
__device__ __forceinline__ float weight_reference(float m, float c2) { return fmaxf(m * c2, kLowest); }

template <bool F32> struct Parts { static constexpr int N = F32 ? 3 : 1; };

// x as one bf16 number, rounded, or as three that add up to it: the upper 8 of the 24 bits, of what is left, and the rest.  They
// have one sign, and the first is no larger than x: a product that overflows does so in the direction of the whole.
template <int N>
__device__ __forceinline__ void split_bf16(float x, __bf16 (&part)[N]) {
    if constexpr (N == 1) {
        part[0] = (__bf16)x;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t upper = __float_as_uint(x) & 0xffff0000u;
            part[i] = __builtin_bit_cast(__bf16, (uint16_t)(upper >> 16));
            x -= __uint_as_float(upper);
        }
    }
}

__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(uint16_t* p, float v) { *p = f32_to_bf16(v); }
__device__ __forceinline__ void store4(float* p, const float (&v)[4]) { *(float4*)p = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void store4(uint16_t* p, const float (&v)[4]) {
    __attribute__((aligned(8))) const uint16_t o[4] = {f32_to_bf16(v[0]), f32_to_bf16(v[1]), f32_to_bf16(v[2]), f32_to_bf16(v[3])};
    *(uint2*)p = *(const uint2*)o;
}

template <bool F32> struct Elem { using T = uint16_t; };
template <> struct Elem<true> { using T = float; };

// Key codes of a 32-key tile as its wave loads them: load j of a lane is 16 bytes, chunk lane % LANES of row
// j * ROWS + lane / LANES.
template <int D, int BITS>
struct KvqLoad {
    static constexpr int LANES = D * BITS / 128, ROWS = 64 / LANES, LOADS = kKvqTile / ROWS;
    // Byte offset in LDS of chunk c of key row r: chunks of a row turned by its 256-byte line, so that writes (rows whole)
    // and reads (one chunk of 16 rows) touch every bank evenly.
    static __device__ __forceinline__ int key_off(int r, int c) { return r * (16 * LANES) + ((c ^ ((r / (16 / LANES)) & (LANES - 1))) << 4); }
};

// (Two workgroups on a compute unit where a third's registers would not do: fp32 with three, 168 registers a lane and up to
// 352 bytes of them in memory: 224 rows over 21.7k keys in 8 bits, pooled, 195 us, with two 58.)
template <int D, int BITS, bool F32, bool POOLED, int NB>
__global__ __launch_bounds__(64 * kKvqWaves, NB == 1 && !F32 ? 3 : 2) void kvq_decode_kernel(
    const typename Elem<F32>::T* __restrict__ Qd, KvqView dense, KvqView sparse, const int32_t* __restrict__ src_idx,
    const int32_t* __restrict__ mix_len, float* __restrict__ part_o, float2* __restrict__ part_ml, int T_q, int n_q_heads,
    int n_kv_heads, int l_cap, int n_split, int share, int more, int n_rtile, int members, float c2,
    typename Elem<F32>::T* __restrict__ O, float* __restrict__ LSE) {
    using R = KvqRow<D, BITS>;
    using G = KvqLoad<D, BITS>;
    using Off = std::conditional_t<POOLED, uint64_t, uint32_t>;                  // of a row: its address, or its distance from the first
    constexpr int NP = Parts<F32>::N, W = D / 4 * BITS / 32, STEPS = D / 32, M = D / 16;
    constexpr int VB = M * BITS / 8, VW = (VB + 3) / 4;       // bytes, words of a piece of a value row
    constexpr int ROWS = 16 * NB;
    struct Area {                                             // of a wave
        uint8_t codes[kKvqTile * D * BITS / 8];               // of the keys
        uint32_t scale[2 * kKvqTile];                         // of the keys, in their order, and of the values, by place (below)
        Off row[2 * kKvqTile];                                // likewise
    };
    __shared__ __attribute__((aligned(16))) uint8_t areas[kKvqWaves][std::max((int)sizeof(Area), ROWS * 4 * D)];
    __shared__ float2 stats[kKvqWaves][ROWS];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int g, split, b, row0;
    if (!kvq_place(n_kv_heads, n_split, n_rtile, members, ROWS, &g, &split, &b, &row0)) return;
    const int group = n_q_heads / n_kv_heads, all_rows = group * T_q, n_rows = min(ROWS, all_rows - row0);

    const int32_t* map = src_idx + (size_t)b * l_cap;
    const uint8_t* rows_d = dense.rows + (size_t)g * dense.capacity * R::CODES;
    const uint8_t* rows_s = sparse.rows + (size_t)g * sparse.capacity * R::CODES;
    const uint8_t* scales_d = dense.scales + (size_t)g * dense.capacity * R::SCALES;
    const uint8_t* scales_s = sparse.scales + (size_t)g * sparse.capacity * R::SCALES;
    Area& area = *(Area*)areas[wave];
    const int row_in = lane / G::LANES, chunk = lane % G::LANES;
    // Lanes 2 k and 2 k + 1 look after key k of a tile: its map entry, and the scales of its key and of its value.  The keys
    // 16 h + 4 r + q that a lane needs of V lie at places 8 q + 4 h + r.
    const int own = lane >> 1, value = lane & 1;
    const int place = (own & 3) * 8 + (own >> 4) * 4 + (own >> 2 & 3);
    const int at_row = value ? kKvqTile + place : own;        // of the row, and of the scales, among those of the keys and values

    struct Tile {
        uint32_t k[G::LOADS][4], v[8][VW], s;
    };
    // The workgroup's tiles are its even share of the set's; of a wave: tile0, tile0 + kKvqWaves, ...
    int tile0 = split * share + min(split, more) + wave;
    // (entries up to the capacity, so that the first ones do not wait for the length; behind the length they may be
    // anything, and row 0 is read there instead, whose values do not count)
    auto entry = [&](int tile) __attribute__((always_inline)) {      // (32-bit byte offsets: a map has fewer than 2^30 entries)
        return *(const int32_t*)((const char*)map + 4u * (uint32_t)min(tile * kKvqTile + own, l_cap - 1));
    };
    int e0 = entry(tile0), e1 = entry(tile0 + kKvqWaves);
    const int len = min(max(mix_len[b], 0), l_cap), tiles = (len + kKvqTile - 1) / kKvqTile;
    if (tiles != n_split * share + more) {                    // (shares of the capacity were a guess: chunks differ in length)
        share = tiles / n_split;
        more = tiles % n_split;
        tile0 = split * share + min(split, more) + wave;
        e0 = entry(tile0);
        e1 = entry(tile0 + kKvqWaves);
    }
    const int end = min(tiles, tile0 - wave + share + (split < more ? 1 : 0));
    const int n = (max(end - tile0, 0) + kKvqWaves - 1) / kKvqWaves;

    auto request = [&](int tile, int e, Tile& t) __attribute__((always_inline)) {
        e = tile * kKvqTile + own < len ? e : 0;
        const uint8_t* s;
        if constexpr (POOLED) {
            const uint64_t row = (uint32_t)(e ^ (e >> 31));
            area.row[at_row] = (uint64_t)(e < 0 ? rows_s : rows_d) + row * R::CODES;
            s = (e < 0 ? scales_s : scales_d) + row * R::SCALES + value * (R::SCALES / 2);
        } else {
            area.row[at_row] = (uint32_t)e * R::CODES;
            s = scales_d + (uint32_t)(e * R::SCALES + value * (R::SCALES / 2));
        }
        if constexpr (R::SCALES == 8) {
            uint32_t w[1];
            load_words(s, w);
            t.s = w[0];
        } else {
            t.s = load_half(s);
        }
        __builtin_amdgcn_wave_barrier();
        auto at = [&](Off row, uint32_t more) __attribute__((always_inline)) {
            if constexpr (POOLED) return (const uint8_t*)row + more;
            else return rows_d + (uint32_t)(row + more);
        };
#pragma unroll
        for (int j = 0; j < G::LOADS; ++j) load_words(at(area.row[j * G::ROWS + row_in], chunk * 16), t.k[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint8_t* p = at(area.row[kKvqTile + q * 8 + i], D * BITS / 8 + l16 * VB);
            if constexpr (VB == 2) t.v[i][0] = load_half(p);
            else load_words(p, t.v[i]);
        }
        __builtin_amdgcn_wave_barrier();
    };

    // Q: step i of row l16 has its elements q * D / 4 + 8 i + {0..7}
    bf16x8 qreg[NB][NP][STEPS];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int rho = row0 + min(nb * 16 + l16, n_rows - 1);
        const auto* src = Qd + (((size_t)b * T_q + rho / group) * n_q_heads + g * group + rho % group) * D + q * (D / 4);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            if constexpr (F32) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    __bf16 part[NP];
                    split_bf16(src[i * 8 + j], part);
#pragma unroll
                    for (int p = 0; p < NP; ++p) qreg[nb][p][i][j] = part[p];
                }
            } else {
                qreg[nb][0][i] = *(const bf16x8*)(src + i * 8);
            }
        }
    }
    f32x4 o[NB][M];                                           // [m][r]: element (4 q + r) * M + m of row l16
    float m_run[NB], mc_run[NB], l_run[NB];                   // reference, the same times c2, sum
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        m_run[nb] = -INFINITY;
        mc_run[nb] = kLowest;
        l_run[nb] = 0.f;
#pragma unroll
        for (int i = 0; i < M; ++i) o[nb][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // Rotations that bring the scale byte of the lane's keys and values to a float's exponent, all that conversions read of it.
    const int kturn = (8 * (q * (D / 4) / kBlock) + 9) & 31, vturn = (8 * (l16 * M / kBlock) + 9) & 31;
    auto turned = [](uint32_t x, int by) __attribute__((always_inline)) { return __uint_as_float(__builtin_amdgcn_alignbit(x, x, by)); };

    // A tile; `left`: its keys that count, 32 unless RAGGED.
    auto work = [&](Tile& t, int left, auto ragged) __attribute__((always_inline)) {
        constexpr bool RAGGED = decltype(ragged)::value;
        if constexpr (RAGGED) {                               // (a row that does not count is 0: its own may be NaN)
            t.s = own < left ? t.s : 0x7f7f7f7f;
#pragma unroll
            for (int j = 0; j < G::LOADS; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) t.k[j][i] = j * G::ROWS + row_in < left ? t.k[j][i] : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int w = 0; w < VW; ++w) t.v[i][w] = (i >> 2) * 16 + (i & 3) * 4 + q < left ? t.v[i][w] : 0;
        }
        area.scale[at_row] = t.s;
#pragma unroll
        for (int j = 0; j < G::LOADS; ++j)
            *(uint4*)(area.codes + G::key_off(j * G::ROWS + row_in, chunk)) = make_uint4(t.k[j][0], t.k[j][1], t.k[j][2], t.k[j][3]);
        __builtin_amdgcn_wave_barrier();
        f32x4 s[NB][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t k[W];
            const int key = h * 16 + (l16 & 3) * 4 + (l16 >> 2);
            if constexpr (W == 2) {                           // half a chunk
                const uint2 x = *(const uint2*)(area.codes + G::key_off(key, q >> 1) + (q & 1) * 8);
                k[0] = x.x; k[1] = x.y;
            } else {
#pragma unroll
                for (int i = 0; i < W / 4; ++i) {
                    const uint4 x = *(const uint4*)(area.codes + G::key_off(key, q * (W / 4) + i));
                    k[4 * i] = x.x; k[4 * i + 1] = x.y; k[4 * i + 2] = x.z; k[4 * i + 3] = x.w;
                }
            }
            const float scale = turned(area.scale[key], kturn);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) s[nb][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const bf16x8 a = eight_bf16<BITS>(k + i * (BITS / 4), scale);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p)
                        s[nb][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qreg[nb][p][i], s[nb][h], 0, 0, 0);
            }
        }
        bf16x8 pb[NB][NP];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            f32x4 (&x)[2] = s[nb];
            if constexpr (RAGGED) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[h][r] = h * 16 + 4 * r + q < left ? x[h][r] : -INFINITY;
            }
            // The reference is raised, and sums and O rescaled, only when a logit is more than 2^8 above it: until then the
            // weights are in a range that bf16 and fp32 hold with unchanged relative precision.
            float y[8], top = -INFINITY;
            auto against = [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = fmaf(x[i >> 2][i & 3], c2, -mc_run[nb]);
            };
            against();
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, y[i]);
            if (__builtin_amdgcn_ballot_w64(top > 8.f) != 0) {
                float m_new = m_run[nb];
#pragma unroll
                for (int i = 0; i < 8; ++i) m_new = fmaxf(m_new, x[i >> 2][i & 3]);
                m_new = fmaxf(m_new, __shfl_xor(m_new, 16));
                m_new = fmaxf(m_new, __shfl_xor(m_new, 32));
                const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m_run[nb] - m_new) * c2);
                l_run[nb] *= alpha;
                m_run[nb] = m_new;
                mc_run[nb] = weight_reference(m_new, c2);
#pragma unroll
                for (int i = 0; i < M; ++i) o[nb][i] *= alpha;
                against();
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float p = __builtin_amdgcn_exp2f(y[i]);
                l_run[nb] += p;
                __bf16 part[NP];
                split_bf16(p, part);
#pragma unroll
                for (int j = 0; j < NP; ++j) pb[nb][j][i] = part[j];
            }
        }
        float vscale[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) vscale[i] = turned(area.scale[kKvqTile + q * 8 + i], vturn);
        __builtin_amdgcn_wave_barrier();
        auto pair = [&](auto m2) __attribute__((always_inline)) {        // matrix instructions 2 m2 and 2 m2 + 1
            bf16x2 x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = two_bf16<BITS, decltype(m2)::value>(t.v[i], vscale[i]);
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const bf16x8 a = {x[0][m], x[1][m], x[2][m], x[3][m], x[4][m], x[5][m], x[6][m], x[7][m]};
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p)
                        o[nb][2 * m2 + m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pb[nb][p], o[nb][2 * m2 + m], 0, 0, 0);
            }
        };
        pair(std::integral_constant<int, 0>{});
        pair(std::integral_constant<int, 1>{});
        if constexpr (M == 8) {
            pair(std::integral_constant<int, 2>{});
            pair(std::integral_constant<int, 3>{});
        }
    };
    // A tile is worked on while the next one is on its way, whose map entries were asked for a tile earlier and before it:
    // loads return in order.  Nothing in the loop is conditional, so that the waits leave the younger loads in flight.
    if (n > 0) {
        Tile a, c;
        request(tile0, e0, a);
        int i = 0;
        for (; i + 2 < n; i += 2) {
            const int tile = tile0 + i * kKvqWaves;
            e0 = entry(tile + 2 * kKvqWaves);
            request(tile + kKvqWaves, e1, c);
            work(a, kKvqTile, std::false_type{});
            e1 = entry(tile + 3 * kKvqWaves);
            request(tile + 2 * kKvqWaves, e0, a);
            work(c, kKvqTile, std::false_type{});
        }
        const int tile = tile0 + i * kKvqWaves;
        if (i + 2 == n) {
            request(tile + kKvqWaves, e1, c);
            work(a, kKvqTile, std::false_type{});
            a = c;
        }
        work(a, len - (tile0 + (n - 1) * kKvqWaves) * kKvqTile, std::true_type{});
    }

    // ---- merge the waves: 16-byte piece c of row r lies at c ^ r (mod the pieces), which spreads the rows over the banks ----
    constexpr int PPR = D / 4;
    float4* red = (float4*)areas[wave];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        l_run[nb] += __shfl_xor(l_run[nb], 16);
        l_run[nb] += __shfl_xor(l_run[nb], 32);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int m = 0; m < M; m += 4)
                red[(nb * 16 + l16) * PPR + ((((4 * q + r) * M + m) / 4) ^ (l16 & (PPR - 1)))] =
                    make_float4(o[nb][m][r], o[nb][m + 1][r], o[nb][m + 2][r], o[nb][m + 3][r]);
        if (q == 0) stats[wave][nb * 16 + l16] = make_float2(m_run[nb], l_run[nb]);
    }
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
            const float4 v = ((const float4*)areas[w])[row * PPR + (c ^ (row & 15 & (PPR - 1)))];
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

// ------------------------------------------------------------------------------------------
// Decode of many stacked rows: 32 rows per wave, eight waves per workgroup.  Here the matrix cores and what feeds them bound the
// call, so each 64-key tile is converted once for all rows of the workgroup: eight threads load the codes of a row between them,
// a tile ahead, and write the bf16 rows to one of two LDS stages while the other is worked on, by the products and layouts of
// the plain decode's ring.  One barrier per tile.
// 896 rows on four heads, 18,176 keys in 4 bits: 49 us, 52 to 55 with the merge (plain decode in place 52.7), 680 TFLOP/s, in 8
// bits 52, 54 to 58; 49 % of the cycles in vector, 40 % in matrix instructions, 31 % of the LDS's in reads of K and V rows by every
// wave.  64 rows per wave would halve those, but spill much: D = 128 takes all 256 registers as it is, and in 4 bits 3 or 4 more,
// 20 bytes a lane.  Four waves per workgroup and converting in turns were no faster.
// ------------------------------------------------------------------------------------------
// Element offset of 16-byte piece `piece` of row `row` of a V tile: its 64-byte parts turned as in the plain tile, for the
// transposing reads, and the pieces of a part by the next bits of the row, for writes of one piece of each part by eight rows.
template <int D>
__device__ __forceinline__ int rows_v_off(int row, int piece) {
    constexpr int CPR = D / 32, RPL = 128 / D;
    return row * D + ((((piece >> 2) ^ ((row / RPL) & (CPR - 1))) << 2 | ((piece & 3) ^ ((row >> 2) & 3))) << 3);
}

constexpr int kRowsWaves = 8, kRowsTile = 32 * kRowsWaves;

template <int D, int BITS, bool POOLED>
__global__ __launch_bounds__(64 * kRowsWaves, 2) void kvq_rows_kernel(
    const uint16_t* __restrict__ Qd, KvqView dense, KvqView sparse, const int32_t* __restrict__ src_idx,
    const int32_t* __restrict__ mix_len, float* __restrict__ part_o, float2* __restrict__ part_ml, int T_q, int n_q_heads,
    int n_kv_heads, int l_cap, int n_split, int n_rtile, int members, float c2, uint16_t* __restrict__ O, float* __restrict__ LSE) {
    using R = KvqRow<D, BITS>;
    constexpr int NW = kRowsWaves, TILE = kKeyTile * D, DB = D / 32;
    constexpr int BYTES = D * BITS / 8 / NW, CW = std::min(4, BYTES / 4), NC = BYTES / (4 * CW);       // of a thread: bytes of a key, words of a chunk, chunks
    constexpr int E = CW * 32 / BITS, SW = R::SCALES / 4;
    extern __shared__ __attribute__((aligned(16))) uint16_t stages[];             // [2][K tile, V tile]
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int g, split, b, row0;
    if (!kvq_place(n_kv_heads, n_split, n_rtile, members, kRowsTile, &g, &split, &b, &row0)) return;
    const int group = n_q_heads / n_kv_heads, all_rows = group * T_q;
    const int len = min(max(mix_len[b], 0), l_cap);
    // the split's tiles: an even share of the query's
    const int tiles = (len + kKeyTile - 1) / kKeyTile, share = tiles / n_split, more = tiles % n_split;
    const int tile0 = split * share + min(split, more), n = share + (split < more ? 1 : 0);

    const int32_t* map = src_idx + (size_t)b * l_cap;
    const int key = tid / NW, part = tid % NW;
    const uint8_t* rows_d = dense.rows + (size_t)g * dense.capacity * R::CODES + part * (CW * 4);
    const uint8_t* rows_s = sparse.rows + (size_t)g * sparse.capacity * R::CODES + part * (CW * 4);
    const uint8_t* scales_d = dense.scales + (size_t)g * dense.capacity * R::SCALES;
    const uint8_t* scales_s = sparse.scales + (size_t)g * sparse.capacity * R::SCALES;
    uint32_t k[NC][CW], v[NC][CW], s[SW];
    auto entry = [&](int tile) __attribute__((always_inline)) {
        const int r = tile * kKeyTile + key;
        return r < len ? map[r] : 0;                          // (row 0 in the place of what is not there)
    };
    auto request = [&](int e) __attribute__((always_inline)) {
        const bool sp = POOLED && e < 0;
        const uint64_t row = (uint32_t)(POOLED ? e ^ (e >> 31) : e);
        const uint8_t* p = (sp ? rows_s : rows_d) + row * R::CODES;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            load_words(p + c * (NW * CW * 4), k[c]);
            load_words(p + D * BITS / 8 + c * (NW * CW * 4), v[c]);
        }
        load_words((sp ? scales_s : scales_d) + row * R::SCALES, s);
    };
    auto convert = [&](uint16_t* kt, int left) __attribute__((always_inline)) {
        uint16_t* vt = kt + TILE;
        if (left < kKeyTile) {                                // (a row that does not count is 0: its own may be NaN)
            const bool there = key < left;
#pragma unroll
            for (int i = 0; i < SW; ++i) s[i] = there ? s[i] : 0x7f7f7f7f;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < CW; ++i) { k[c][i] = there ? k[c][i] : 0; v[c][i] = there ? v[c][i] : 0; }
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int first = (c * NW + part) * E, turn = (8 * (first / kBlock) + 9) & 31;     // (a scale byte to the exponent)
            const uint32_t ks = s[0], vs = SW == 2 ? s[SW - 1] : s[0] >> 16;
            const float kscale = __uint_as_float(__builtin_amdgcn_alignbit(ks, ks, turn));
            const float vscale = __uint_as_float(__builtin_amdgcn_alignbit(vs, vs, turn));
#pragma unroll
            for (int i = 0; i < E / 8; ++i) {
                *(bf16x8*)(kt + k_tile_off<D>(key, first / 8 + i)) = eight_bf16<BITS>(k[c] + i * (BITS / 4), kscale);
                *(bf16x8*)(vt + rows_v_off<D>(key, first / 8 + i)) = eight_bf16<BITS>(v[c] + i * (BITS / 4), vscale);
            }
        }
    };

    const int rho = row0 + wave * 32 + l32;
    bf16x8 qreg[1][D / 16];
    {
        const int r = min(rho, all_rows - 1);
        const uint4* src = (const uint4*)(Qd + (((size_t)b * T_q + r / group) * n_q_heads + g * group + r % group) * D);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) qreg[0][ks] = __builtin_bit_cast(bf16x8, src[ks * 2 + hi]);
    }
    f32x16 o[DB];
    float m_run = -INFINITY, mc_run = kLowest, l_run = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = zero16();
    const int dhalf = (lane >> 4) & 1, t = lane & 15;
    auto work = [&](const uint16_t* kt, int left) __attribute__((always_inline)) {
        const uint16_t* vt = kt + TILE;
        f32x16 x[1][2];
        qk_tile_ahead<D, 3>(kt, qreg, l32, hi, x);
        if (left < kKeyTile) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) x[0][kb][r] = acc_key(kb, r, hi) < left ? x[0][kb][r] : -INFINITY;
        }
        // (the reference as in the kernel above; one decision per tile, so that exponentials and products behind it are one
        // stretch of instructions to be woven)
        float y[2][16], top = -INFINITY;
        auto against = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) y[kb][r] = fmaf(x[0][kb][r], c2, -mc_run);
        };
        against();
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, y[kb][r]);
        if (__builtin_amdgcn_ballot_w64(top > 8.f) != 0) {
            float m_new = m_run;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) m_new = fmaxf(m_new, x[0][kb][r]);
            m_new = fmaxf(m_new, __shfl_xor(m_new, 32));
            const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m_run - m_new) * c2);
            l_run *= alpha;
            m_run = m_new;
            mc_run = weight_reference(m_new, c2);
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
            against();
        }
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                bf16x8 pb;
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const float p = __builtin_amdgcn_exp2f(y[kb][j * 8 + r]);
                    sum[r & 1] += p;
                    pb[r] = (__bf16)p;
                }
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const int row = kb * 32 + j * 16 + 4 * hi + (t >> 2), piece = db * 4 + dhalf * 2 + ((t >> 1) & 1);
                    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vt + rows_v_off<D>(row, piece) + 4 * (t & 1)));
                    const s16x4 up = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vt + rows_v_off<D>(row + 8, piece) + 4 * (t & 1)));
                    const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7));
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb, o[db], 0, 0, 0);
                }
            }
        l_run += sum[0] + sum[1];
    };

    if (n > 0) {
        auto left = [&](int i) __attribute__((always_inline)) { return len - (tile0 + i) * kKeyTile; };
        request(entry(tile0));
        int e = entry(tile0 + 1);
        convert(stages, left(0));
        request(e);                                           // (behind the last tile row 0, not counted)
        e = entry(tile0 + 2);
        __syncthreads();
        for (int i = 0; i < n; ++i) {
            uint16_t *now = stages + (i & 1) * 2 * TILE, *next = stages + (~i & 1) * 2 * TILE;
            convert(next, left(i + 1));
            request(e);
            e = entry(tile0 + i + 3);
            work(now, left(i));
            __syncthreads();
        }
    }
    const size_t part_base = (((size_t)b * n_kv_heads + g) * n_split + split) * (size_t)all_rows;
    const float l = l_run + __shfl_xor(l_run, 32);
    if (rho >= all_rows) return;
    const size_t out = ((size_t)b * T_q + rho / group) * n_q_heads + g * group + rho % group;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int rq = 0; rq < 4; ++rq) {
            float a[4];
            const int d = db * 32 + rq * 8 + hi * 4;
#pragma unroll
            for (int r = 0; r < 4; ++r) a[r] = o[db][rq * 4 + r];
            if (n_split > 1) {
                store4(part_o + (part_base + rho) * D + d, a);
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r) a[r] = len > 0 ? a[r] / l : 0.f;
                store4(O + out * D + d, a);
            }
        }
    if (hi == 0) {
        if (n_split > 1) part_ml[part_base + rho] = make_float2(m_run * c2, l);
        else if (LSE) LSE[out] = len > 0 ? (m_run * c2 + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
    }
}

// The merge of the splits, one workgroup per query row: SG groups of D / 4 lanes take every SG-th split, U of them requested
// together, and are folded through LDS; the order depends on the split index alone.  Bound by the launch and two dependent trips
// to memory: 28 rows of 32 splits 3.3 us, 3,584 rows of 16 splits (29 MB) 7.7.  As the last workgroup's work in the kernels above,
// behind device-wide fences, each of which writes an XCD's L2 back, 7.9 us of a token became 19.
template <int D, bool F32, int THREADS>
__global__ __launch_bounds__(THREADS) void kvq_merge_kernel(const float* __restrict__ part_o, const float2* __restrict__ part_ml,
                                                            typename Elem<F32>::T* __restrict__ O, float* __restrict__ LSE,
                                                            const int32_t* __restrict__ mix_len, int T_q, int n_q_heads,
                                                            int n_kv_heads, int n_split, int batch) {
    constexpr int NV = D / 4, SG = THREADS / NV, U = 4;
    __shared__ __attribute__((aligned(16))) float red[SG][D];
    __shared__ float2 stat[SG];
    const int group = n_q_heads / n_kv_heads, n_rows = T_q * group, sg = threadIdx.x / NV, d = threadIdx.x % NV * 4;
    const unsigned id = folded_id();
    const int rho = (int)(id % n_rows);
    const unsigned unit = id / n_rows;                        // (query, KV head)
    if (unit >= (unsigned)(batch * n_kv_heads)) return;
    const int g = (int)(unit % n_kv_heads), b = (int)(unit / n_kv_heads);
    const size_t base = (size_t)unit * n_split * n_rows + rho;
    const bool some = mix_len[b] > 0;
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
    if (threadIdx.x >= D) return;                             // a column each
    M = stat[0].x;
#pragma unroll 8
    for (int i = 1; i < SG; ++i) M = fmaxf(M, stat[i].x);
    const float ref = M == -INFINITY ? 0.f : M;
    float sum = 0.f;
    L = 0.f;
#pragma unroll 8
    for (int i = 0; i < SG; ++i) {
        const float f = __builtin_amdgcn_exp2f(stat[i].x - ref);
        L = fmaf(f, stat[i].y, L);
        sum = fmaf(f, red[i][threadIdx.x], sum);
    }
    const size_t row = ((size_t)b * T_q + rho / group) * n_q_heads + g * group + rho % group;
    store1(O + row * D + threadIdx.x, some ? sum / L : 0.f);
    if (LSE && threadIdx.x == 0) LSE[row] = some ? (M + __builtin_amdgcn_logf(L)) * kLn2 : -INFINITY;
}

}  // namespace

// How many splits, and for many rows which kernel, by estimates in us, fitted by least squares to timed calls of 1,376 to 98,176
// keys (7 % rms over the 25 calls of profiles/quantised_cache_kernel_times.md): a start, the tiles that a wave or workgroup
// walks, the partial rows, the merge.  More than one workgroup on a compute unit shares its vector and matrix units, so that a
// tile takes longer, but not as much as there are workgroups; the third one pays for a few rows only (one row of seven heads,
// D = 64, 98k keys x 8 queries: one 50.8, two and a bit 44.1, three 34.8).
static KvqPlan kvq_splits(const vxl_attn_desc* d, int batch, long long rows, int l_cap, int blocks, float* us) {
    KvqPlan p{};
    p.blocks = blocks;
    const int wg_rows = blocks ? 16 * blocks : kRowsTile, wg_keys = blocks ? kKvqTile * kKvqWaves : kKeyTile;
    p.n_rtile = (rows + wg_rows - 1) / wg_rows;
    const long long units = (long long)batch * d->n_kv_heads;
    *us = INFINITY;
    p.n_split = 1;
    // The pass that writes the row map has the queries in its grid's second dimension; rows and workgroups are counted in 32
    // bits by the kernels.  (In 128 bits: 64 do not hold what these bounds refuse.)
    p.fits = batch <= 65535 && rows <= 1 << 30 && (__int128)p.n_rtile * units <= INT32_MAX;
    if (!p.fits) return p;
    const long long per = units * p.n_rtile;
    const long long steps = ((long long)l_cap + wg_keys - 1) / wg_keys;           // of a workgroup that has all keys
    const bool d64 = d->head_dim == 64;
    const float tile = blocks == 0 ? (d64 ? 1.27f : 1.76f) : blocks == 2 ? (d64 ? 0.57f : 0.76f)
                       : d->dtype == VXL_F32 ? (d64 ? 0.6f : 0.88f) : d64 ? 0.44f : 0.64f;
    const float start = blocks == 0 ? 8.f : blocks == 2 ? 5.5f : 4.2f, per_mb = blocks ? 0.9f : 0.5f, merged = blocks == 1 ? 2.8f : 2.5f;
    const long long most = std::min<long long>(steps, std::max<long long>(1, 256 * (blocks == 1 ? 3 : blocks == 2 ? 2 : 1) / per));
    for (long long n = 1; n <= most;) {
        const long long walk = (steps + n - 1) / n;
        const long long on_unit = (per * n + 255) / 256;
        const float load = blocks == 1 ? 0.36f + 0.64f * on_unit : blocks == 2 && on_unit > 1 ? 0.78f * on_unit : (float)on_unit;
        const float mb = 4e-6f * units * n * rows * d->head_dim;
        const float merge = n == 1 ? 0.f : merged + per_mb * mb + (n > 32 ? 0.9f : 0.f) + (n > 64 ? 0.4f : 0.f);
        const float t = start + tile * load * walk + merge;
        if (t < *us) {
            *us = t;
            p.n_split = (int)n;
        }
        n = walk > 1 ? (steps + walk - 2) / (walk - 1) : most + 1;                // the next that shortens the walk
    }
    if (p.n_split > 1) {
        p.part_ml = align_up((size_t)units * p.n_split * rows * d->head_dim * sizeof(float), 256);
        p.total = p.part_ml + align_up((size_t)units * p.n_split * rows * sizeof(float2), 256);
    }
    return p;
}

KvqPlan kvq_plan(const vxl_attn_desc* d, int batch, int T, int l_cap) {
    const long long rows = (long long)(d->n_q_heads / d->n_kv_heads) * T;
    float us, us_many;
    if (d->dtype != VXL_BF16 || rows <= 16) return kvq_splits(d, batch, rows, l_cap, 1, &us);
    const KvqPlan p = kvq_splits(d, batch, rows, l_cap, 2, &us);
    if (rows <= 128) return p;
    // (us, blocks of 32 rows and of 256, 21.7k keys: 224 rows 24.3 and 30.4, 448 rows of 4 queries 118 and 102)
    const KvqPlan many = kvq_splits(d, batch, rows, l_cap, 0, &us_many);
    return us_many < us ? many : p;
}

// Test hook (vxl_debug.h).
extern "C" int vxl_debug_kvq_plan(const vxl_attn_desc* d, int batch, int n_q_tokens, int l_cap, int* n_split) {
    const KvqPlan p = kvq_plan(d, batch, n_q_tokens, l_cap);
    *n_split = p.n_split;
    return p.blocks;
}

vxl_status launch_kvq_decode(const KvqPlan& p, const vxl_attn_desc* d, float scale, const void* Qd, int batch, int T,
                             const vxl_kvq_cache* c, const vxl_kvq_cache* sp, const int32_t* src_idx, int l_cap,
                             const int32_t* mix_len, void* O, float* LSE, void* ws, hipStream_t s) {
    float* part_o = (float*)ws;
    float2* part_ml = (float2*)((char*)ws + p.part_ml);
    const int n_rtile = (int)p.n_rtile, members = n_rtile * batch, all = d->n_kv_heads * p.n_split * members;
    const int xcds = std::min(all, kXcds), each = (all + xcds - 1) / xcds;
    const dim3 grid(xcds, std::min(each, 65535), (each + 65534) / 65535);
    const int tiles = (l_cap - 1) / kKvqTile + 1;
    return by_kind(d, c, [&](auto dim, auto bits, auto f32) {
        using T_ = typename Elem<f32>::T;
        auto run = [&](auto pooled, auto nb) {
            hipLaunchKernelGGL((kvq_decode_kernel<dim, bits, f32, pooled, nb>), grid, dim3(64 * kKvqWaves), 0, s,
                               (const T_*)Qd, view(c), view(sp), src_idx, mix_len, part_o, part_ml, T, d->n_q_heads, d->n_kv_heads,
                               l_cap, p.n_split, tiles / p.n_split, tiles % p.n_split, n_rtile, members, scale * kLog2e, (T_*)O, LSE);
        };
        auto rows = [&](auto pooled) {
            if constexpr (!f32) {
                if (p.blocks == 2) return run(pooled, std::integral_constant<int, 2>{});
            }
            run(pooled, std::integral_constant<int, 1>{});
        };
        vxl_status st = VXL_OK;
        if constexpr (!f32) {
            auto many = [&](auto pooled) {
                constexpr int lds = 2 * 2 * kKeyTile * dim * 2;
                static PerDeviceOnce attr;
                st = attr.run([&] {
                    VXL_HIP_TRY(hipFuncSetAttribute((const void*)kvq_rows_kernel<dim, bits, pooled>, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
                    return VXL_OK;
                });
                if (st != VXL_OK) return;
                hipLaunchKernelGGL((kvq_rows_kernel<dim, bits, pooled>), grid, dim3(64 * kRowsWaves), lds, s, (const uint16_t*)Qd, view(c),
                                   view(sp), src_idx, mix_len, part_o, part_ml, T, d->n_q_heads, d->n_kv_heads, l_cap, p.n_split, n_rtile, members,
                                   scale * kLog2e, (uint16_t*)O, LSE);
            };
            if (p.blocks == 0) { if (sp) many(std::true_type{}); else many(std::false_type{}); }
            if (st != VXL_OK) return st;
        }
        if (p.blocks > 0) { if (sp) rows(std::true_type{}); else rows(std::false_type{}); }
        st = launched();
        if (st != VXL_OK || p.n_split == 1) return st;
        const long long n_rows = (long long)(d->n_q_heads / d->n_kv_heads) * T;
        auto merge = [&](auto threads) {
            hipLaunchKernelGGL((kvq_merge_kernel<dim, f32, threads>), folded_grid(n_rows * d->n_kv_heads * batch), dim3(threads), 0, s, part_o,
                               part_ml, (T_*)O, LSE, mix_len, T, d->n_q_heads, d->n_kv_heads, p.n_split, batch);
        };
        if (p.n_split <= 32) merge(std::integral_constant<int, 256>{});
        else if (p.n_split <= 64) merge(std::integral_constant<int, 512>{});
        else merge(std::integral_constant<int, 1024>{});
        return launched();
    });
}

}  // namespace vxl
