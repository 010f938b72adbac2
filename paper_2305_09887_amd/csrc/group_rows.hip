// Rows by group: a stable counting sort of row numbers by a small id,
//   offsets[g] = #{ v : 0 <= id_v < g },   order[offsets[g] + i] = the i-th row of group g in ascending row number.
// Rows whose id is outside [0, E) are in no group.  Memory bound: reads the ids, writes the order (8 bytes a row).
//
// A wavefront ranks 64 consecutive rows at once: the lanes with the same id are found with one ballot per bit of the id, a
// row's rank among them is the number of such lanes below its own, and a counter per (wavefront, group) in LDS carries the
// rank on to the next 64 rows.  Integers throughout, every position has one writer: one result.
// Up to kOneBlockRows rows one block does it all (counts, their prefix, positions): 5,000 rows of 8 groups 6.3 us, 16,384 rows of 8, 64 and 512
// groups 13.5, 17.8 and 23.4.  Above that tiles of rows are counted, the counts [group][tile] are prefixed, and the tiles are ranked again from
// their bases: 16,385 to 30,000 rows 17.9, 19.5 and 23.5; 12,500,000 rows of 64 groups count 12, prefix 9, place 36 us (100 MB, 2.8 TB/s: the ballots).
#include "kernels.hpp"

namespace tma {

constexpr int kMaxGroups = 1024;
constexpr int kOneBlockRows = 16384;
constexpr int kOneThreads = 1024;
constexpr int kOneGroups = 512;                                   // 32 KB of counters, and a thread for each
constexpr int kTileThreads = 256;
constexpr int kTileChunks = 16;                                   // 64-row chunks of a wavefront of a tile
constexpr int kTileRows = kTileThreads * kTileChunks;

// the lanes that hold the same id as this one; `bits`: of the largest id.  (Masks of a bit and its two halves: four vector instructions a bit.)
__device__ __forceinline__ uint64_t same_id(int id, bool in, int bits)
{
    const uint64_t all = __ballot(in);
    uint32_t lo = uint32_t(all), hi = uint32_t(all >> 32);
    for (int b = 0; b < bits; ++b) {
        const int mine = __builtin_amdgcn_sbfe(id, b, 1);      // all ones or zero
        const uint64_t set = __ballot(mine);
        lo &= ~(uint32_t(set) ^ uint32_t(mine));
        hi &= ~(uint32_t(set >> 32) ^ uint32_t(mine));
    }
    return uint64_t(hi) << 32 | lo;
}

// lanes of m below this one
__device__ __forceinline__ int below(uint64_t m) { return int(__builtin_amdgcn_mbcnt_hi(uint32_t(m >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(m), 0u))); }

// one chunk of 64 rows: rank in the wavefront's own counters, which are left advanced (a wavefront's LDS operations complete
// in order; the fences keep the compiler from moving them)
__device__ __forceinline__ int take(volatile int32_t *counters, int id, bool in, int bits)
{
    const uint64_t m = same_id(id, in, bits);
    const int rank = below(m);
    int pos = 0;
    if (in) pos = counters[id] + rank;
    __builtin_amdgcn_wave_barrier();
    if (in && rank == 0) counters[id] = pos + __popcll(m);
    __builtin_amdgcn_wave_barrier();
    return pos;
}

__global__ __launch_bounds__(kOneThreads) void group_rows_one_kernel(int n, const int32_t *__restrict__ ids, int E, int bits,
                                                                     int32_t *__restrict__ offsets, int32_t *__restrict__ order)
{
    extern __shared__ int32_t counters[];          // [16 wavefronts][E]
    __shared__ int32_t wave_sums[kOneThreads / kWave];
    constexpr int kWaves = kOneThreads / kWave, kChunks = kOneBlockRows / kOneThreads;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int chunks = (n + kOneThreads - 1) / kOneThreads, r0 = wave * chunks * kWave;   // of a wavefront, one run of rows each
    int id[kChunks], pos[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        const int r = r0 + c * kWave + lane;
        id[c] = c < chunks && r < n ? ids[r] : -1;
    }
    for (int i = threadIdx.x; i < kWaves * E; i += kOneThreads) counters[i] = 0;
    __syncthreads();
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
        if (c < chunks) pos[c] = take(counters + wave * E, id[c], id[c] >= 0 && id[c] < E, bits);
    __syncthreads();
    // counts -> bases: over the wavefronts of a group, then over the groups (a thread each)
    int total = 0;
    if (int(threadIdx.x) < E)
        for (int w = 0; w < kWaves; ++w) total += counters[w * E + threadIdx.x];
    int incl = total;
    for (int d = 1; d < kWave; d <<= 1) {
        const int t = __shfl_up(incl, d, kWave);
        if (lane >= d) incl += t;
    }
    if (lane == kWave - 1) wave_sums[wave] = incl;
    __syncthreads();
    int base = incl - total;
    for (int w = 0; w < wave; ++w) base += wave_sums[w];
    if (int(threadIdx.x) < E) {
        offsets[threadIdx.x] = base;
        if (int(threadIdx.x) == E - 1) offsets[E] = base + total;
        for (int w = 0; w < kWaves; ++w) {
            const int c = counters[w * E + threadIdx.x];
            counters[w * E + threadIdx.x] = base;
            base += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
        if (c < chunks && id[c] >= 0 && id[c] < E) order[counters[wave * E + id[c]] + pos[c]] = r0 + c * kWave + lane;
}

// counts[g][tile]
__global__ __launch_bounds__(kTileThreads) void group_rows_count_kernel(int64_t n, const int32_t *__restrict__ ids, int E, int64_t tiles,
                                                                        int32_t *__restrict__ counts)
{
    __shared__ int32_t total[kMaxGroups];
    const int64_t tile = blockIdx.x, r0 = tile * kTileRows;
    for (int g = threadIdx.x; g < E; g += kTileThreads) total[g] = 0;
    int id[kTileChunks];
#pragma unroll
    for (int c = 0; c < kTileChunks; ++c) {
        const int64_t r = r0 + c * kTileThreads + threadIdx.x;
        id[c] = r < n ? ids[r] : -1;
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < kTileChunks; ++c)
        if (id[c] >= 0 && id[c] < E) atomicAdd(&total[id[c]], 1);      // (whole numbers: any order gives the same)
    __syncthreads();
    for (int g = threadIdx.x; g < E; g += kTileThreads) counts[g * tiles + tile] = total[g];
}

// Positions from bases[g][tile] (and the offsets, by tile 0).  The tile is put in order in LDS first, so that a group's rows go to memory side by
// side: a store of 64 rows as they come goes to as many lines (12,500,000 rows of 64 groups 54 us, with the order through LDS 36).
__global__ __launch_bounds__(kTileThreads) void group_rows_place_kernel(int64_t n, const int32_t *__restrict__ ids, int E, int bits, int64_t tiles,
                                                                        const int32_t *__restrict__ bases, int32_t *__restrict__ offsets,
                                                                        int32_t *__restrict__ order)
{
    extern __shared__ int32_t counters[];          // [4 wavefronts][E], then [E]: what turns a place in the tile into one in the list
    __shared__ int32_t sorted[kTileRows];          // row of the tile and, from bit 12 on, group
    __shared__ int32_t wave_sums[kTileThreads / kWave];
    constexpr int kWaves = kTileThreads / kWave, kPer = kMaxGroups / kTileThreads;
    static_assert(kTileRows <= 4096 && kMaxGroups <= 1024, "a row and a group in a word");
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t tile = blockIdx.x, r0 = tile * kTileRows + wave * (kTileChunks * kWave);
    int32_t *shift = counters + kWaves * E;
    for (int i = threadIdx.x; i < kWaves * E; i += kTileThreads) counters[i] = 0;
    int id[kTileChunks];
#pragma unroll
    for (int c = 0; c < kTileChunks; ++c) {
        const int64_t r = r0 + c * kWave + lane;
        id[c] = r < n ? ids[r] : -1;
    }
    __syncthreads();
    int pos[kTileChunks];
#pragma unroll
    for (int c = 0; c < kTileChunks; ++c) pos[c] = take(counters + wave * E, id[c], id[c] >= 0 && id[c] < E, bits);
    __syncthreads();
    // a thread's four groups: their counts, where they begin in the tile
    int mine[kPer], total = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int g = int(threadIdx.x) * kPer + j;
        mine[j] = 0;
        if (g < E)
            for (int w = 0; w < kWaves; ++w) mine[j] += counters[w * E + g];
        total += mine[j];
    }
    int incl = total;
    for (int d = 1; d < kWave; d <<= 1) {
        const int t = __shfl_up(incl, d, kWave);
        if (lane >= d) incl += t;
    }
    if (lane == kWave - 1) wave_sums[wave] = incl;
    __syncthreads();
    int at = incl - total, all = 0;
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) at += wave_sums[w];
        all += wave_sums[w];
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int g = int(threadIdx.x) * kPer + j;
        if (g < E) {
            const int base = bases[g * tiles + tile];
            if (tile == 0) offsets[g] = base;
            shift[g] = base - at;
            int next = at;
            for (int w = 0; w < kWaves; ++w) {
                const int c = counters[w * E + g];
                counters[w * E + g] = next;
                next += c;
            }
            at = next;
        }
    }
    if (tile == 0 && threadIdx.x == 0) offsets[E] = bases[E * tiles];
    __syncthreads();
#pragma unroll
    for (int c = 0; c < kTileChunks; ++c)
        if (id[c] >= 0 && id[c] < E) sorted[counters[wave * E + id[c]] + pos[c]] = (wave * kTileChunks + c) * kWave + lane | id[c] << 12;
    __syncthreads();
    for (int i = threadIdx.x; i < all; i += kTileThreads) {
        const int v = sorted[i];
        order[shift[v >> 12] + i] = int32_t(tile * kTileRows) + (v & 4095);
    }
}

static bool in_one_block(int64_t n, int E) { return n <= kOneBlockRows && E <= kOneGroups; }

static int bits_of(int E)
{
    int b = 0;
    while ((1 << b) < E) ++b;
    return b;
}

}  // namespace tma

extern "C" size_t tma_group_rows_workspace_bytes(int64_t n, int32_t E)
{
    using namespace tma;
    if (n < 0 || n > INT32_MAX || E < 1 || E > kMaxGroups) return 0;
    if (in_one_block(n, E)) return 256;
    const int64_t cells = (n > 0 ? ceil_div(n, kTileRows) : 1) * E;
    return round_up(size_t(cells) * 4, 256) + round_up(size_t(cells + 1) * 4, 256) + round_up(exclusive_scan_i32_workspace_bytes(cells), 256);
}

extern "C" int tma_group_rows(int64_t n, const int32_t *group, int32_t E, int32_t *offsets_out, int32_t *order_out, void *ws, size_t ws_bytes,
                              tma_stream_t stream)
{
    using namespace tma;
    const char *fn = "tma_group_rows";
    TMA_REQUIRE(n >= 0 && n <= INT32_MAX, TMA_ERR_INVALID_ARG, "%s: n outside [0, 2^31)", fn);
    TMA_REQUIRE(E >= 1 && E <= kMaxGroups, TMA_ERR_BAD_SHAPE, "%s: E=%d outside [1, %d]", fn, E, kMaxGroups);
    TMA_REQUIRE(offsets_out && (n == 0 || (group && order_out)), TMA_ERR_INVALID_ARG, "%s: NULL argument", fn);
    TMA_REQUIRE(ws && aligned(ws, 256), TMA_ERR_INVALID_ARG, "%s: workspace NULL or not 256-byte aligned", fn);
    TMA_REQUIRE(ws_bytes >= tma_group_rows_workspace_bytes(n, E), TMA_ERR_WORKSPACE_TOO_SMALL, "%s: workspace too small", fn);
    hipStream_t s = as_stream(stream);
    const int bits = bits_of(E);
    if (in_one_block(n, E)) {
        TMA_TIMED("group_rows_one", s);
        hipLaunchKernelGGL(group_rows_one_kernel, dim3(1), dim3(kOneThreads), size_t(kOneThreads / kWave) * E * 4, s, int(n), group, E, bits, offsets_out,
                           order_out);
        return check_launch(fn);
    }
    const int64_t tiles = n > 0 ? ceil_div(n, kTileRows) : 1, cells = tiles * E;
    char *at = static_cast<char *>(ws);
    int32_t *counts = reinterpret_cast<int32_t *>(at);
    at += round_up(size_t(cells) * 4, 256);
    int32_t *bases = reinterpret_cast<int32_t *>(at);
    at += round_up(size_t(cells + 1) * 4, 256);
    {
        TMA_TIMED("group_rows_count", s);
        hipLaunchKernelGGL(group_rows_count_kernel, dim3(unsigned(tiles)), dim3(kTileThreads), 0, s, n, group, E, tiles, counts);
        if (int rc = check_launch(fn)) return rc;
    }
    if (int rc = launch_exclusive_scan_i32(cells, counts, bases, at, s)) return rc;
    TMA_TIMED("group_rows_place", s);
    hipLaunchKernelGGL(group_rows_place_kernel, dim3(unsigned(tiles)), dim3(kTileThreads), size_t(kTileThreads / kWave + 1) * E * 4, s, n, group, E, bits,
                       tiles, bases, offsets_out, order_out);
    return check_launch(fn);
}
