// Mixed sets cut back to the rows of the largest weight.
#include <algorithm>
#include <type_traits>

#include "vxl_mixed.h"
#include "vxl_rows.h"

namespace vxl {

namespace {

// Order of preference as a number, larger first: 0 an empty row, 1 NaN, then the weights in their order, all ones a protected row.
__device__ __forceinline__ uint32_t preference(float w, int pos, int n_first, int newest, int n_recent) {
    if (pos < 0) return 0u;
    if (pos < n_first || (long long)newest - pos < n_recent) return ~0u;
    if (w != w) return 1u;
    const uint32_t x = __float_as_uint(w == 0.f ? 0.f : w);
    return (x >> 31) ? ~x : x | 0x80000000u;                  // (-inf: 0x007fffff, +inf: 0xff800000)
}

// Which rows of a set are kept, and from where every place of the result is filled: map[d], d < n.  One workgroup per (query, KV
// head).  The n-th largest preference is found eleven bits at a time by counting; rows above it are kept, and of the rows that equal it
// the lowest.  Dropped rows below n and kept ones above are numbered in order, wave by wave, and matched.
constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64, kBins = 2048;

__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(const float* __restrict__ weight, const int32_t* __restrict__ row_pos,
                                                                   const int32_t* __restrict__ mix_len, const int32_t* __restrict__ newest,
                                                                   int n_kv, int l_cap, int keep, int n_first, int n_recent,
                                                                   int32_t* __restrict__ map, int32_t* __restrict__ n_out) {
    __shared__ int hist[kBins];
    __shared__ int wave_sum[3][kSelWaves];
    __shared__ int found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int unit = blockIdx.x, b = unit / n_kv;
    const int len = min(max(mix_len[b], 0), l_cap), n = min(len, keep);
    const size_t set = (size_t)unit * l_cap;
    if (unit % n_kv == 0 && tid == 0) n_out[b] = n;
    if (n == 0) return;
    const int latest = newest ? newest[b] : 0;
    auto key = [&](int row) { return preference(weight[set + row], row_pos[set + row], n_first, latest, n_recent); };

    // the n-th largest preference: rows with `upper` as their upper bits, of which the `left` first ones are still looked for
    uint32_t upper = 0;
    int left = n;
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
        __syncthreads();
        for (int row = tid; row < len; row += kSelThreads) {
            const uint32_t x = key(row);
            if (pass == 0 || (x >> (shift + bits)) == upper) atomicAdd(&hist[(x >> shift) & ((1 << bits) - 1)], 1);
        }
        __syncthreads();
        // bins from the top: thread t has bins 2 t' and 2 t' + 1 of the reversed order
        const int top = kBins - 1 - 2 * tid;
        const int c0 = hist[top], c1 = hist[top - 1];
        int run = c0 + c1;
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(run, o);
            if (lane >= o) run += x;
        }
        if (lane == 63) wave_sum[0][wave] = run;
        __syncthreads();
        int before = run - c0 - c1;
        for (int w = 0; w < wave; ++w) before += wave_sum[0][w];
        if (before < left && before + c0 >= left) { found[0] = top; found[1] = left - before; }
        else if (before + c0 < left && before + c0 + c1 >= left) { found[0] = top - 1; found[1] = left - before - c0; }
        __syncthreads();
        upper = upper << bits | (uint32_t)found[0];
        left = found[1];
        __syncthreads();
    }
    // Wave w numbers rows [w * per, (w + 1) * per), 64 at a time: rows that equal the threshold, holes below n, movers above.
    const int per = ((len + kSelWaves - 1) / kSelWaves + 63) / 64 * 64, lo = wave * per, hi = min(lo + per, len);
    const unsigned long long below = (1ull << lane) - 1;
    int equal = 0;
    for (int base = lo; base < hi; base += 64) {
        const int row = base + lane;
        equal += __popcll(__ballot(row < hi && key(row) == upper));
    }
    if (lane == 0) wave_sum[0][wave] = equal;
    __syncthreads();
    int first_equal = 0;
    for (int w = 0; w < wave; ++w) first_equal += wave_sum[0][w];
    auto walk = [&](auto&& f) {
        int ties = first_equal;
        for (int base = lo; base < hi; base += 64) {
            const int row = base + lane;
            const uint32_t x = row < hi ? key(row) : 0u;
            const unsigned long long same = __ballot(row < hi && x == upper);
            const bool kept = row < hi && (x > upper || (x == upper && ties + __popcll(same & below) < left));
            ties += __popcll(same);
            f(row, __ballot(row < hi && row < n && !kept), __ballot(kept && row >= n));
        }
    };
    int holes = 0, movers = 0;
    walk([&](int, unsigned long long h, unsigned long long m) { holes += __popcll(h); movers += __popcll(m); });
    if (lane == 0) { wave_sum[1][wave] = holes; wave_sum[2][wave] = movers; }
    __syncthreads();
    holes = movers = 0;
    for (int w = 0; w < wave; ++w) { holes += wave_sum[1][w]; movers += wave_sum[2][w]; }
    // the movers' list lies behind the n places of the map where there is room for it, which is everywhere: there are at most len - n
    int32_t* places = map + set;
    walk([&](int row, unsigned long long h, unsigned long long m) {
        if (m >> lane & 1) places[n + movers + __popcll(m & below)] = row;
        if (row < n) places[row] = h >> lane & 1 ? -1 - (holes + __popcll(h & below)) : row;
        movers += __popcll(m);
        holes += __popcll(h);
    });
}

// Fills the places: a row by D * elem / 16 neighbouring lanes.
template <int ROW16>
__global__ __launch_bounds__(256) void evict_move_kernel(const uint4* K, const uint4* V, const float* weight,
                                                         const int32_t* row_pos, uint4* Kout, uint4* Vout, float* weight_out, int32_t* pos_out,
                                                         const int32_t* __restrict__ map, const int32_t* __restrict__ n_of, int32_t* kept, int n_kv,
                                                         int l_cap, int out_cap, bool in_place) {
    constexpr int ROWS = 256 / ROW16;
    const int unit = blockIdx.y, b = unit / n_kv, part = threadIdx.x % ROW16, n = n_of[b];
    if (unit % n_kv == 0 && blockIdx.x == 0 && threadIdx.x == 0) kept[b] = n;
    const int32_t* places = map + (size_t)unit * l_cap;
    const size_t from = (size_t)unit * l_cap, to = (size_t)unit * out_cap;
    for (int row = blockIdx.x * ROWS + threadIdx.x / ROW16; row < n; row += gridDim.x * ROWS) {
        int src = places[row];
        if (src < 0) src = places[n - 1 - src];
        else if (in_place) continue;
        Kout[(to + row) * ROW16 + part] = K[(from + src) * ROW16 + part];
        Vout[(to + row) * ROW16 + part] = V[(from + src) * ROW16 + part];
        if (part == 0) {
            weight_out[to + row] = weight[from + src];
            pos_out[to + row] = row_pos[from + src];
        }
    }
}

}  // namespace

EvictPlan evict_plan(const vxl_attn_desc* d, int batch, int l_cap) {
    EvictPlan p{};
    p.map = 0;
    p.n = align_up((size_t)batch * d->n_kv_heads * l_cap * sizeof(int32_t), 256);
    p.total = p.n + align_up((size_t)batch * sizeof(int32_t), 256);
    return p;
}

vxl_status launch_mixed_evict(const EvictPlan& p, const EvictCall& c, hipStream_t s) {
    const vxl_attn_desc* d = c.d;
    const int units = c.batch * d->n_kv_heads;
    int32_t *map = (int32_t*)(c.ws + p.map), *n = (int32_t*)(c.ws + p.n);
    hipLaunchKernelGGL(evict_select_kernel, dim3(units), dim3(kSelThreads), 0, s, c.weight, c.row_pos, c.mix_len, c.newest, d->n_kv_heads, c.l_cap,
                       c.keep, c.n_first, c.n_recent, map, n);
    vxl_status st = mixed_launched();
    if (st != VXL_OK) return st;
    return by_storage(d, [&](auto f32, auto dim) {
        constexpr int ROW16 = dim * (f32 ? 4 : 2) / 16, ROWS = 256 / ROW16;
        const int most = std::max(1, std::min(c.keep, c.l_cap));
        const dim3 grid(std::min((most + ROWS - 1) / ROWS, 4096), units);
        hipLaunchKernelGGL((evict_move_kernel<ROW16>), grid, dim3(256), 0, s, (const uint4*)c.Kmix, (const uint4*)c.Vmix, c.weight, c.row_pos,
                           (uint4*)c.Kout, (uint4*)c.Vout, c.weight_out, c.pos_out, map, n, c.kept, d->n_kv_heads, c.l_cap, c.out_cap,
                           c.Kout == c.Kmix);
        return mixed_launched();
    });
}

}  // namespace vxl
