// Mixed sets cut back to the rows of the largest weight.
#include <algorithm>
#include <type_traits>

#include "vxl_mixed.h"

namespace vxl {

namespace {

// Order of preference as a number, larger first: 0 an empty row, 1 NaN, then the weights in their order, all ones a protected row.
__device__ __forceinline__ uint32_t preference(float w, int pos, int n_first, int newest, int n_recent) {
    if (pos < 0) return 0u;
    if (pos < n_first || (n_recent && (long long)newest - pos < n_recent)) return ~0u;
    if (w != w) return 1u;
    const uint32_t x = __float_as_uint(w == 0.f ? 0.f : w);
    return (x >> 31) ? ~x : x | 0x80000000u;                  // (-inf: 0x007fffff, +inf: 0xff800000)
}

// Sets as the kernels see them, and what is kept.
struct Cut {
    const float* weight;
    const int32_t *row_pos, *mix_len, *newest;
    int n_kv, cap, keep, n_first, n_recent;
};
struct Move {
    const uint4 *k, *v;
    uint4 *k_out, *v_out;
    float* weight_out;
    int32_t *pos_out, *kept;
    int out_cap;
    bool in_place;
};

// The n-th largest preference is found by counting, eleven bits at a time from the top: the bin of the bits so far that holds it, and how
// many of that bin's rows are still among the n.  Rows above the last bin are kept, and of those in it the lowest.  Rows below n that are
// not kept are holes, rows from n on that are kept movers; there are as many of one as of the other, and the i-th hole takes the i-th
// mover.
constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 2048;
__device__ __forceinline__ constexpr int shift_of(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
__device__ __forceinline__ constexpr int bins_of(int pass) { return pass == 2 ? 1024 : kBins; }
__device__ __forceinline__ int bin_of(uint32_t x, int pass) { return (int)(x >> shift_of(pass)) & (bins_of(pass) - 1); }
// (whether its bits above this pass's are those found)
__device__ __forceinline__ bool of_bin(uint32_t x, int pass, uint32_t upper) {
    return pass == 0 || x >> (shift_of(pass) + (pass == 2 ? 10 : 11)) == upper;
}

struct Found {
    uint32_t upper;            // the bits found so far
    int left;                  // rows of that bin that are among the n
    int rows;                  // rows of that bin
};
// Sums over the lanes up to this one, in the order of lanes (shifts inside rows of 16 lanes, then the last lane of a row, of two, to those
// behind: a few cycles each, where a shuffle goes through the LDS).
__device__ __forceinline__ int scan_lanes(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}

__device__ __forceinline__ int sum_lanes(int x) { return __builtin_amdgcn_readlane(scan_lanes(x), 63); }

// From counts of this pass's bins, of which thread t has c0 in bin 2047 - 2 t and c1 in the one below.
struct FindArea {
    int wave_sum[kWaves];
    int bin, left, rows;
};
__device__ __forceinline__ void find_bin(FindArea& a, int c0, int c1, int pass, Found& f) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int run = scan_lanes(c0 + c1);
    if (lane == 63) a.wave_sum[wave] = run;
    __syncthreads();
    int before = run - c0 - c1;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) before += w < wave ? a.wave_sum[w] : 0;
    const int top = kBins - 1 - 2 * tid;
    if (before < f.left && before + c0 >= f.left) { a.bin = top; a.left = f.left - before; a.rows = c0; }
    else if (before + c0 < f.left && before + c0 + c1 >= f.left) { a.bin = top - 1; a.left = f.left - before - c0; a.rows = c1; }
    __syncthreads();
    f.upper = (pass == 0 ? 0u : f.upper << (pass == 2 ? 10 : 11)) | (uint32_t)a.bin;
    f.left = a.left;
    f.rows = a.rows;
}

// A row of D elements by ROW16 lanes.
template <int ROW16>
__device__ __forceinline__ void load_row(const Move& m, size_t from, int part, uint4& k, uint4& v) {
    k = m.k[from * ROW16 + part];
    v = m.v[from * ROW16 + part];
}
template <int ROW16>
__device__ __forceinline__ void store_row(const Cut& c, const Move& m, size_t from, size_t to, int part, const uint4& k, const uint4& v) {
    m.k_out[to * ROW16 + part] = k;
    m.v_out[to * ROW16 + part] = v;
    if (part == 0) {
        m.weight_out[to] = c.weight[from];
        m.pos_out[to] = c.row_pos[from];
    }
}
template <int ROW16>
__device__ __forceinline__ void move_row(const Cut& c, const Move& m, size_t from, size_t to, int part) {
    uint4 k, v;
    load_row<ROW16>(m, from, part, k, v);
    store_row<ROW16>(c, m, from, to, part, k, v);
}

// ------------------------------------------------------------------------------------------
// Sets of up to 16,384 rows: a thread has PER rows' preferences in registers (wave w the rows [64 PER w, 64 PER (w + 1)), lanes side by
// side), a workgroup a whole set.  Bound by latency: launch, one trip to memory, and the barriers of two or three passes (the last one is
// left out when all of the bin's rows are kept, which is so where weights differ).  Out of place every workgroup of a set selects for
// itself and moves its share, which saves the second launch; in place the rows' places are written down for the kernel behind.
// 4 KV heads, 2,304 rows to 2,048: 8.8 us (in place 8.2 and 2.3 for the moves, with the second launch 10.9 in a replayed graph, out of
// place 9.2); 16 sets of up to 7,001 fp32 rows to 1,777: 13.4 (9.7 and 5.0; 13.9 either way).  Two groups of workgroups a compute unit
// could hold (512 / units): 23.8.  Counting a wave's most frequent bin by one lane: 28.  PER = 32 (20,000 rows): 33.8 and 48.7 us for a
// quarter and nearly all kept, the launches below 34.2 and 43.1.
// ------------------------------------------------------------------------------------------
template <int PER, int ROW16, bool MOVES>
__global__ __launch_bounds__(kThreads) void evict_set_kernel(Cut c, Move m, int32_t* __restrict__ places, int32_t* __restrict__ n_out) {
    __shared__ int hist[2][kBins];
    __shared__ FindArea area;
    __shared__ int sums[3][kWaves];
    __shared__ uint16_t source[PER * kThreads], movers_of[PER * kThreads / 2];    // (no more movers than half the rows)
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int unit = blockIdx.y, b = unit / c.n_kv;
    const size_t set = (size_t)unit * c.cap;
    const int row0 = wave * (64 * PER) + lane;
    const int len = min(max(c.mix_len[b], 0), c.cap), n = min(len, c.keep), latest = c.newest ? c.newest[b] : 0;
    float w[PER];
    int pos[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {                           // (rows that there are, whatever the length)
        const int row = min(row0 + i * 64, c.cap - 1);
        w[i] = c.weight[set + row];
        pos[i] = c.row_pos[set + row];
    }
    for (int i = tid; i < kBins; i += kThreads) hist[0][i] = 0;
    if (unit % c.n_kv == 0 && blockIdx.x == 0 && tid == 0) {
        if constexpr (MOVES) m.kept[b] = n;
        else n_out[b] = n;
    }
    if (n == 0) return;
    // Most rows stay where they are: the first row of a thread's share is on its way while the set is looked through.
    constexpr int ROWS = kThreads / ROW16;
    const int part = tid % ROW16, own = blockIdx.x * ROWS + tid / ROW16;
    uint4 own_k = make_uint4(0, 0, 0, 0), own_v = own_k;
    if (MOVES && own < n) load_row<ROW16>(m, set + own, part, own_k, own_v);
    uint32_t x[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) x[i] = preference(w[i], pos[i], c.n_first, latest, c.n_recent);
    Found f{0u, n, 0};
    int shift = 0;
    __syncthreads();
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        int* h = hist[pass & 1];
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (row0 + i * 64 < len && of_bin(x[i], pass, f.upper)) atomicAdd(&h[bin_of(x[i], pass)], 1);
        __syncthreads();
        const int top = kBins - 1 - 2 * tid, c0 = h[top], c1 = h[top - 1];
        if (pass < 2) {
            hist[~pass & 1][top] = 0;
            hist[~pass & 1][top - 1] = 0;
        }
        find_bin(area, c0, c1, pass, f);
        shift = shift_of(pass);
        if (f.left == f.rows) break;
    }
    const unsigned long long below = (1ull << lane) - 1;
    int holes = 0, movers = 0;
    unsigned kept = 0;                                        // bit i: row i of the thread
    if (f.left == f.rows) {
#pragma unroll
        for (int i = 0; i < PER; ++i) kept |= row0 + i * 64 < len && x[i] >> shift >= f.upper ? 1u << i : 0u;
    } else {                                                  // (all 32 bits are found) of the rows that equal it the lowest
        int equal = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) equal += __popcll(__ballot(row0 + i * 64 < len && x[i] == f.upper));
        if (lane == 0) sums[0][wave] = equal;
        __syncthreads();
        equal = 0;
#pragma unroll
        for (int y = 0; y < kWaves; ++y) equal += y < wave ? sums[0][y] : 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const bool there = row0 + i * 64 < len;
            const unsigned long long same = __ballot(there && x[i] == f.upper);
            kept |= there && (x[i] > f.upper || (x[i] == f.upper && equal + __popcll(same & below) < f.left)) ? 1u << i : 0u;
            equal += __popcll(same);
        }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const bool keep = kept >> i & 1;
        holes += __popcll(__ballot(row0 + i * 64 < n && !keep));
        movers += __popcll(__ballot(row0 + i * 64 >= n && keep));
    }
    if (lane == 0) { sums[1][wave] = holes; sums[2][wave] = movers; }
    __syncthreads();
    holes = movers = 0;
#pragma unroll
    for (int y = 0; y < kWaves; ++y) {
        holes += y < wave ? sums[1][y] : 0;
        movers += y < wave ? sums[2][y] : 0;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int row = row0 + i * 64;
        const bool keep = kept >> i & 1;
        const unsigned long long up = __ballot(keep && row >= n);
        if (up >> lane & 1) movers_of[movers + __popcll(up & below)] = (uint16_t)row;
        movers += __popcll(up);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int row = row0 + i * 64;
        const bool keep = kept >> i & 1;
        const unsigned long long down = __ballot(row < n && !keep);
        if (row < n) source[row] = keep ? (uint16_t)row : movers_of[holes + __popcll(down & below)];
        holes += __popcll(down);
    }
    __syncthreads();
    if constexpr (MOVES) {
        const size_t to = (size_t)unit * m.out_cap;
        if (own < n) {
            const int from = source[own];
            if (from != own) load_row<ROW16>(m, set + from, part, own_k, own_v);
            store_row<ROW16>(c, m, set + from, to + own, part, own_k, own_v);
        }
        for (int row = own + gridDim.x * ROWS; row < n; row += gridDim.x * ROWS) move_row<ROW16>(c, m, set + source[row], to + row, part);
    } else {
        for (int row = tid; row < n; row += kThreads) places[set + row] = source[row];
    }
}

// ------------------------------------------------------------------------------------------
// Longer sets: each in parts of `part_rows` rows below n and of as many from n on (so that a part has holes or movers, never both), at most
// kParts of them, a workgroup each.  Every pass is a launch: the counts of a part's bins are written down, the next launch adds those of
// all parts, finds the bin and counts on.  The last one knows from the counts how many rows every part before it keeps.
// 131,328 rows of 4 KV heads to 16,384: 4.5, 7.3 and 7.3 us for the passes, 12.8 for the places, 12.6 for the moves, which copy 64 MB (in
// place 11.6: seven of eight kept rows change place); in replayed graphs 48.7 out of place, 46.9 in place.
// ------------------------------------------------------------------------------------------
constexpr int kParts = 20;
struct State {                 // of a set between the launches, in the workspace
    int hist[3][kParts][kBins];
    int above[2][kParts];      // rows above the bin found, by pass and part
    Found found[2];
};
static_assert(sizeof(State) % 8 == 0, "pairs of bins are read together");
struct Part {
    int lo, hi;
};
// (of the rows below n, then of those from n on)
__device__ __forceinline__ int parts_below(int n, int part_rows) { return (int)(((unsigned)n + (unsigned)part_rows - 1) / (unsigned)part_rows); }
__device__ __forceinline__ Part part_of(int i, int first, int n, int len, int part_rows) {         // first: parts_below()
    const long long lo = i < first ? (long long)i * part_rows : n + (long long)(i - first) * part_rows, end = i < first ? n : len;
    return {(int)min(lo, end), (int)min(lo + part_rows, end)};
}

// The bin of a pass, from the counts of all parts; counts[p]: of the part's bins 2046 - 2 t and 2047 - 2 t.
__device__ __forceinline__ void find_from_parts(FindArea& area, const State* st, int pass, int n_parts, int n, Found& f, int2 (&counts)[kParts]) {
    if (pass == 0) f = {0u, n, 0};
    else f = st->found[pass - 1];
    int c0 = 0, c1 = 0;
#pragma unroll
    for (int p = 0; p < kParts; ++p) counts[p] = p < n_parts ? *(const int2*)&st->hist[pass][p][kBins - 2 - 2 * (int)threadIdx.x] : make_int2(0, 0);
#pragma unroll
    for (int p = 0; p < kParts; ++p) {
        c1 += counts[p].x;
        c0 += counts[p].y;
    }
    find_bin(area, c0, c1, pass, f);
}

// Weights and positions of eight rows, `step` apart, of those below hi (which may be none).
struct Batch {
    float w[8];
    int pos[8];
    __device__ __forceinline__ void load(const Cut& c, size_t set, int row, int step, int hi) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int at = max(min(row + u * step, hi - 1), 0);
            w[u] = c.weight[set + at];
            pos[u] = c.row_pos[set + at];
        }
    }
};

template <int PASS>
__global__ __launch_bounds__(kThreads) void evict_count_kernel(Cut c, State* __restrict__ states, int part_rows) {
    __shared__ int hist[kBins];
    __shared__ int above;
    __shared__ FindArea area;
    const int tid = threadIdx.x, unit = blockIdx.y, part = blockIdx.x, b = unit / c.n_kv;
    const size_t set = (size_t)unit * c.cap;
    State* st = states + unit;
    const int len = min(max(c.mix_len[b], 0), c.cap), n = min(len, c.keep), latest = c.newest ? c.newest[b] : 0;
    if (n == 0) return;
    const Part p = part_of(part, parts_below(n, part_rows), n, len, part_rows);
    Batch rows;                                               // (on their way while the bin is found)
    rows.load(c, set, p.lo + tid, kThreads, p.hi);
    for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
    Found f{0u, n, 0};
    if (tid == 0) above = 0;
    if constexpr (PASS > 0) {
        int2 counts[kParts];
        find_from_parts(area, st, PASS - 1, gridDim.x, n, f, counts);
        if (part == 0 && tid == 0) st->found[PASS - 1] = f;
        const int top = kBins - 1 - 2 * tid, bin = (int)(f.upper & (bins_of(PASS - 1) - 1));
        int own = 0;
#pragma unroll
        for (int p = 0; p < kParts; ++p) own = p == part ? (top > bin ? counts[p].y : 0) + (top - 1 > bin ? counts[p].x : 0) : own;
        own = sum_lanes(own);
        if ((tid & 63) == 0) atomicAdd(&above, own);
    }
    __syncthreads();
    if (PASS > 0 && tid == 0) st->above[PASS - 1][part] = above;
    for (int row0 = p.lo; row0 < p.hi; row0 += 8 * kThreads) {
        if (row0 > p.lo) rows.load(c, set, row0 + tid, kThreads, p.hi);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const uint32_t x = preference(rows.w[u], rows.pos[u], c.n_first, latest, c.n_recent);
            if (row0 + tid + u * kThreads < p.hi && of_bin(x, PASS, f.upper)) atomicAdd(&hist[bin_of(x, PASS)], 1);
        }
    }
    __syncthreads();
    for (int i = tid; i < kBins; i += kThreads) st->hist[PASS][part][i] = hist[i];
}

// Places of the result: source rows, -1 - i at the i-th hole; the movers' list lies behind them (there are at most len - n).
__global__ __launch_bounds__(kThreads) void evict_places_kernel(Cut c, const State* __restrict__ states, int32_t* __restrict__ map,
                                                                int32_t* __restrict__ n_out, int part_rows) {
    __shared__ FindArea area;
    __shared__ int above[kParts], equals[kParts], sums[2][kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, unit = blockIdx.y, part = blockIdx.x, b = unit / c.n_kv;
    const size_t set = (size_t)unit * c.cap;
    const State* st = states + unit;
    const int len = min(max(c.mix_len[b], 0), c.cap), n = min(len, c.keep), latest = c.newest ? c.newest[b] : 0;
    if (unit % c.n_kv == 0 && part == 0 && tid == 0) n_out[b] = n;
    if (n == 0) return;
    // Wave w numbers its share of the part's rows in order, 64 at a time; the first eight times 64 are on their way from here on.
    const int first = parts_below(n, part_rows);
    const Part p = part_of(part, first, n, len, part_rows);
    const int per = ((p.hi - p.lo + kWaves - 1) / kWaves + 63) / 64 * 64, lo = (int)min((long long)p.lo + (long long)wave * per, (long long)p.hi);
    const int hi = min(lo + per, p.hi);
    Batch rows;
    rows.load(c, set, lo + lane, 64, hi);
    if (tid < kParts) above[tid] = tid < (int)gridDim.x ? st->above[0][tid] + st->above[1][tid] : 0;
    Found f;
    int2 counts[kParts];
    find_from_parts(area, st, 2, gridDim.x, n, f, counts);
    const int top = kBins - 1 - 2 * tid, bin = (int)(f.upper & 1023);
#pragma unroll
    for (int i = 0; i < kParts; ++i) {                        // (few rows share the 22 bits found before)
        const int over = (top > bin ? counts[i].y : 0) + (top - 1 > bin ? counts[i].x : 0);
        if (over) atomicAdd(&above[i], over);
        if (top == bin || top - 1 == bin) equals[i] = top == bin ? counts[i].y : counts[i].x;
    }
    __syncthreads();
    // In the parts before this one (a lane each): rows that equal the threshold, holes, movers.
    int equal, holes, movers;
    {
        const int i = min(lane, kParts - 1), same = lane < kParts ? equals[i] : 0;
        const int upto = scan_lanes(same);
        const int kept = above[i] + min(max(f.left - (upto - same), 0), same);
        const Part at = part_of(i, first, n, len, part_rows);
        equal = sum_lanes(lane < part ? same : 0);
        holes = sum_lanes(lane < part && i < first ? at.hi - at.lo - kept : 0);
        movers = sum_lanes(lane < part && i >= first ? kept : 0);
    }
    const unsigned long long below = (1ull << lane) - 1;
    uint32_t first_keys[8];
    auto keys_of = [&](const Batch& from, uint32_t (&x)[8]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = preference(from.w[u], from.pos[u], c.n_first, latest, c.n_recent);
    };
    keys_of(rows, first_keys);
    auto walk = [&](auto&& g) __attribute__((always_inline)) {
        for (int base = lo; base < hi; base += 64 * 8) {
            uint32_t x[8];
            if (base > lo) {
                Batch more;
                more.load(c, set, base + lane, 64, hi);
                keys_of(more, x);
            } else {
#pragma unroll
                for (int u = 0; u < 8; ++u) x[u] = first_keys[u];
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) g(base + u * 64 + lane, x[u]);
        }
    };
    int own_above = 0, own_equal = 0;
    walk([&](int row, uint32_t x) {
        own_above += row < hi && x > f.upper ? 1 : 0;
        own_equal += row < hi && x == f.upper ? 1 : 0;
    });
    own_above = sum_lanes(own_above);
    own_equal = sum_lanes(own_equal);
    if (lane == 0) { sums[0][wave] = own_above; sums[1][wave] = own_equal; }
    __syncthreads();
    int kept_before = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        kept_before += w < wave ? sums[0][w] + min(max(f.left - equal, 0), sums[1][w]) : 0;
        equal += w < wave ? sums[1][w] : 0;
    }
    int32_t* places = map + set;
    holes += lo - p.lo - kept_before;
    movers += kept_before;
    const bool ties = f.left < f.rows;                        // (of the rows that equal it, only the lowest are kept)
    walk([&](int row, uint32_t x) {
        bool keep = row < hi && x >= f.upper;
        if (ties) {
            const unsigned long long same = __ballot(row < hi && x == f.upper);
            keep = keep && (x != f.upper || equal + __popcll(same & below) < f.left);
            equal += __popcll(same);
        }
        const unsigned long long list = __ballot(part < first ? row < hi && !keep : keep);        // (holes or movers)
        const int at = (part < first ? holes : movers) + __popcll(list & below);
        if (part < first) {
            if (row < hi) places[row] = list >> lane & 1 ? -1 - at : row;
            holes += __popcll(list);
        } else {
            if (keep) places[n + at] = row;
            movers += __popcll(list);
        }
    });
}

// Fills the places.
template <int ROW16>
__global__ __launch_bounds__(256) void evict_move_kernel(Cut c, Move m, const int32_t* __restrict__ map, const int32_t* __restrict__ n_of) {
    constexpr int ROWS = 256 / ROW16;
    const int unit = blockIdx.y, b = unit / c.n_kv, part = threadIdx.x % ROW16, n = n_of[b];
    if (unit % c.n_kv == 0 && blockIdx.x == 0 && threadIdx.x == 0) m.kept[b] = n;
    const int32_t* places = map + (size_t)unit * c.cap;
    const size_t from = (size_t)unit * c.cap, to = (size_t)unit * m.out_cap;
    for (int row = blockIdx.x * ROWS + threadIdx.x / ROW16; row < n; row += gridDim.x * ROWS) {
        int src = places[row];
        if (src < 0) src = places[n - 1 - src];
        if (m.in_place && src == row) continue;
        move_row<ROW16>(c, m, from + src, to + row, part);
    }
}

// Rows of a set that one workgroup holds in registers, and of a part of a longer one: a set has at most two parts more than part_rows go
// into it, one for its end and one where n cuts one in two.
constexpr int kSetRows = 16 * kThreads;
int part_rows_of(int l_cap) { return std::max(8 * kThreads, (int)(((long long)l_cap + kParts - 3) / (kParts - 2))); }

}  // namespace

EvictPlan evict_plan(const vxl_attn_desc* d, int batch, int l_cap) {
    EvictPlan p{};
    const size_t units = (size_t)batch * d->n_kv_heads;
    p.map = 0;
    p.n = align_up(units * l_cap * sizeof(int32_t), 256);
    p.states = p.n + align_up((size_t)batch * sizeof(int32_t), 256);
    p.total = p.states + (l_cap > kSetRows ? align_up(units * sizeof(State), 256) : 0);
    return p;
}

vxl_status launch_mixed_evict(const EvictPlan& p, const EvictCall& e, hipStream_t s) {
    const vxl_attn_desc* d = e.d;
    const int units = e.batch * d->n_kv_heads;
    int32_t *map = (int32_t*)(e.ws + p.map), *n = (int32_t*)(e.ws + p.n);
    const Cut c{e.weight, e.row_pos, e.mix_len, e.newest, d->n_kv_heads, e.l_cap, e.keep, e.n_first, e.n_recent};
    const Move m{(const uint4*)e.Kmix, (const uint4*)e.Vmix, (uint4*)e.Kout, (uint4*)e.Vout, e.weight_out, e.pos_out,
                 e.kept, e.out_cap, e.Kout == e.Kmix};
    const int most = std::max(1, std::min(e.keep, e.l_cap));
    return by_storage(d, [&](auto f32, auto dim) {
        constexpr int ROW16 = dim * (f32 ? 4 : 2) / 16;
        vxl_status st = VXL_OK;
        if (e.l_cap <= kSetRows) {
            // (in place, and where the lengths are overwritten, no workgroup may write before all have read)
            const bool moves = !m.in_place && (const int32_t*)e.kept != e.mix_len;
            auto run = [&](auto per, auto in_one) {
                const int rows = kThreads / ROW16;
                const int groups = in_one ? std::max(1, std::min((most + rows - 1) / rows, 256 / units)) : 1;
                hipLaunchKernelGGL((evict_set_kernel<per, ROW16, in_one>), dim3(groups, units), dim3(kThreads), 0, s, c, m, map, n);
                return mixed_launched();
            };
            auto by_rows = [&](auto in_one) {
                if (e.l_cap <= 1 * kThreads) return run(std::integral_constant<int, 1>{}, in_one);
                if (e.l_cap <= 2 * kThreads) return run(std::integral_constant<int, 2>{}, in_one);
                if (e.l_cap <= 4 * kThreads) return run(std::integral_constant<int, 4>{}, in_one);
                if (e.l_cap <= 8 * kThreads) return run(std::integral_constant<int, 8>{}, in_one);
                return run(std::integral_constant<int, 16>{}, in_one);
            };
            if (moves) return by_rows(std::true_type{});
            st = by_rows(std::false_type{});
        } else {
            State* states = (State*)(e.ws + p.states);
            const int part_rows = part_rows_of(e.l_cap);
            const dim3 grid((e.l_cap - 1) / part_rows + 2, units);           // (one more where n cuts a part in two)
            hipLaunchKernelGGL(evict_count_kernel<0>, grid, dim3(kThreads), 0, s, c, states, part_rows);
            hipLaunchKernelGGL(evict_count_kernel<1>, grid, dim3(kThreads), 0, s, c, states, part_rows);
            hipLaunchKernelGGL(evict_count_kernel<2>, grid, dim3(kThreads), 0, s, c, states, part_rows);
            hipLaunchKernelGGL(evict_places_kernel, grid, dim3(kThreads), 0, s, c, states, map, n, part_rows);
            st = mixed_launched();
        }
        if (st != VXL_OK) return st;
        constexpr int ROWS = 256 / ROW16;
        hipLaunchKernelGGL((evict_move_kernel<ROW16>), dim3(std::min((most + ROWS - 1) / ROWS, 4096), units), dim3(256), 0, s, c, m, map, n);
        return mixed_launched();
    });
}

}  // namespace vxl
