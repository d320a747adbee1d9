// The rows of a mixed KV set, as a block of 256 threads finds them: the prefix, then the chunks in order, each with all its
// rows (dense) or its sparse ones.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace vxl {

// Chunks up to which a block keeps where a chunk's rows come from in LDS beside the offsets: more would leave room for
// fewer than the eight blocks per compute unit that the heads one after the other run at (FOUR, at four, always does).
// Beyond, a row asks memory for it.  Eight queries, one head, 3,000 chunks of 40 tokens 55.0 -> 42.3 us, three, two heads
// of D = 64, 4,096 of 40, 2,000 dense 74.9 -> 56.7; one query, one head, 4,096 of 32 22.3 -> 23.0.
constexpr int kTableChunks = 2500;

// In LDS: off[c] = first mixed row of chunk c, top bit: dense; (table) from[c] = its first token, or -1 - its first kept row.
constexpr int kDenseChunk = INT32_MIN;

// Bytes of mixed sets beyond which a gather stores them past the caches.
constexpr long long kPastCaches = 160ll << 20;

// 16 bytes that the caches need not keep (NT)
template <bool NT>
__device__ __forceinline__ void store16(uint4* p, uint4 v) {
    typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
    if constexpr (NT) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), (u32x4*)p);
    else *p = v;
}

// Fills off and from; the number of rows of the set.
__device__ __forceinline__ int scan_mixed_rows(const uint8_t* mask, const int32_t* bounds, const int32_t* soff, int n_chunks,
                                               int n_prefix, int* off, int* from, bool table, int (&wave_tot)[4][4]) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int len = n_prefix;                                       // rows of the chunks so far
    // The rows every chunk contributes, four 256-chunk passes at a time: their loads are all requested before the
    // first scan and do not wait for the mask (one memory round trip and one barrier per 1,024 chunks).
    for (int base4 = 0; base4 < n_chunks; base4 += 1024) {
        int rows[4], inc[4], flag[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int c = base4 + u * 256 + tid;
            rows[u] = flag[u] = 0;
            if (c < n_chunks) {
                const int lo = bounds[c], hi = bounds[c + 1], s_lo = soff[c], s_hi = soff[c + 1];
                const bool dense = mask[c] != 0;
                rows[u] = dense ? hi - lo : s_hi - s_lo;
                flag[u] = dense ? kDenseChunk : 0;
                if (table) from[c] = dense ? lo : -1 - s_lo;
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (base4 + u * 256 >= n_chunks) break;           // (uniform)
            inc[u] = rows[u];                                 // inclusive scan inside the wave
            for (int o = 1; o < 64; o <<= 1) {
                const int t = __shfl_up(inc[u], o);
                if (lane >= o) inc[u] += t;
            }
            if (lane == 63) wave_tot[u][wave] = inc[u];
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (base4 + u * 256 >= n_chunks) break;
            const int c = base4 + u * 256 + tid;
            int before = len;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int t = wave_tot[u][w];
                before += w < wave ? t : 0;
                len += t;
            }
            if (c < n_chunks) off[c] = (before + inc[u] - rows[u]) | flag[u];
        }
        __syncthreads();                                      // off is there; wave_tot may be written again
    }
    return len;
}

// Where mixed row r comes from: a token id, or -1 - (pooled row).  Asked by the LPR lanes of a row together.
template <int LPR>
__device__ __forceinline__ int mixed_row_source(int r, int n_prefix, int n_chunks, const int* off, const int* from, bool table,
                                                const int32_t* bounds, const int32_t* soff, const int32_t* sidx, bool pooled) {
    if (r < n_prefix) return r;
    const int lane = threadIdx.x & 63, part = threadIdx.x % LPR;
    int c = 0;                                                // last chunk with off[c] <= r: it lies in [c, c + span)
    for (int span = n_chunks; span > 1;) {
        const int step = (span + LPR - 1) / LPR;
        const unsigned long long hit = __ballot(part * step < span && (off[min(c + part * step, n_chunks - 1)] & ~kDenseChunk) <= r);
        const int last = __popcll((hit >> (lane & ~(LPR - 1))) & ((1ull << LPR) - 1)) - 1;
        c += last * step;
        span = min(step, span - last * step);
    }
    const int at = off[c], o = r - (at & ~kDenseChunk);
    const int first = table ? from[c] : at < 0 ? bounds[c] : -1 - soff[c];
    if (first >= 0) return first + o;
    return pooled ? first - o : sidx[-1 - first + o];
}

}  // namespace vxl
