// Tile products of the grouped dense layers (grouped_dense.hip), for groups of many rows.
//
// A plan made on the device, with the weights laid out in the same launch, tells every tile its group: tiles of a group's rows
// follow each other, group after group, and a block takes its tiles from one die's run of them (neighbours share weights and,
// where a row's results are several tiles wide, rows in that die's L2).
//
// grouped_rows_kernel (forward and input gradient): C[v] = A[v] B[g] for 64 listed rows v.  A row's k-values are read once, wherever the row lies, in
// pieces of 16 bytes, all of the next tile's on their way in registers while this one is multiplied; through LDS (512 bytes of a row at a
// time) because the matrix instruction wants a row per lane.  The weights go past LDS: laid out as fragments, 1 KB that a
// wavefront loads at once, and the same for all tiles of a group, they come out of L2.  The instruction multiplies weights by
// rows, so that a lane ends with neighbouring results of one row: which column of W is which row of a fragment is the layout's
// choice, and is made so that a lane has 16 or 32 neighbours.  Bound by what a compute unit has on its way: 125,000 rows of 256 -> 128 in fp32
// 64 us (193 MB, 3.0 TB/s), their input gradient behind a mask 86 us (321 MB, 3.7 TB/s; on the fp32 instruction 111).
//
// grouped_resident_kernel: the same product with the weights in LDS, for lists that are long enough (see below).  1,000,003 rows of 256 -> 256 in bf16
// 218 us (1.03 GB, 4.7 TB/s, what a copy reaches), 131 GFLOP at half of a large product's rate.
//
// grouped_weight_kernel (weight gradients): dW[g] += X[v]^T dZ[v] over a run of a group's rows, up to 256 x 256 results a block (all
// of a run's rows are then read once); both operands come as they lie, rows of LDS, and are read along columns by the transposing LDS
// read.  Runs of one group are added up in order by a second kernel; a group of one run is stored at once.  604,000 rows of 256 x 256
// in bf16 196 to 216 us (X, dY and the mask 928 MB, 4.3 to 4.7 TB/s); 125,237 of 128 x 256 in fp32 74 us (321 MB, 4.3 TB/s; on the fp32 instruction 102).
//
// bf16: v_mfma_f32_32x32x16_bf16, weights rounded once to bf16 (as in all products of bf16 storage here), fp32 accumulation, results rounded once.
// fp32: the same instruction, three bf16 parts of each operand and six products of them (gemm_split.hpp says why those suffice): 192 cycles for 16
// k-values where the fp32 instruction takes 512.  A result that is not finite (an operand that is not, or is too large to be taken
// apart) is computed again in fp32, value by value.
#pragma once
#include "kernels.hpp"
#include "row_piece.hpp"
#include "split_pair.hpp"

#include <cfloat>
#include <type_traits>

namespace tma {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kDies = 8;             // workgroups are dealt round-robin to them
constexpr int kTileM = 64;           // rows of a tile
constexpr int kGgThreads = 256;
constexpr int kStepsUp = 4;          // steps of tile products are filled up with zeros to a multiple of this
constexpr int kMaxGroups = 1024;

struct GroupList {
    const int32_t *offsets, *order;
    int E;
    int64_t n;
    // (what an offset says is held inside the list, and a row inside the arrays)
    __device__ __forceinline__ int64_t begin(int g) const
    {
        const int64_t o = offsets[g];
        return o < 0 ? 0 : o < n ? o : n;
    }
    __device__ __forceinline__ int64_t row(int64_t i) const
    {
        if (!order) return i;
        const int64_t r = order[i];
        return r >= 0 && r < n ? r : -1;
    }
};

// ---- plan ----------------------------------------------------------------------
struct TilePlan {        // in the workspace
    int4 *tiles;         // group, first position in the list, rows, 0
    int32_t *first;      // [E + 1]: first tile of each group; [E]: number of tiles
    int height;          // rows of a tile
    int64_t room;        // tiles that fit
};

// Tiles of the groups before each one, in LDS; returns their number.  Blocks of kGgThreads.  Offsets that descend somewhere can ask for any number of
// tiles: no more than there is room for are counted, so that no one looks for others.
__device__ __forceinline__ int tile_prefix(const GroupList &gl, int height, int64_t room, int (&prefix)[kMaxGroups + 1])
{
    __shared__ int64_t wave_sums[kGgThreads / kWave];
    constexpr int kPer = kMaxGroups / kGgThreads;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int count[kPer];
    int64_t total = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int g = int(threadIdx.x) * kPer + j;
        const int64_t rows = g < gl.E ? gl.begin(g + 1) - gl.begin(g) : 0;
        count[j] = rows > 0 ? int((rows + height - 1) / height) : 0;
        total += count[j];
    }
    int64_t incl = total;
    for (int d = 1; d < kWave; d <<= 1) {
        const int64_t t = __shfl_up(incl, d, kWave);
        if (lane >= d) incl += t;
    }
    if (lane == kWave - 1) wave_sums[wave] = incl;
    __syncthreads();
    int64_t at = incl - total, all = 0;
    for (int w = 0; w < kGgThreads / kWave; ++w) {
        if (w < wave) at += wave_sums[w];
        all += wave_sums[w];
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int g = int(threadIdx.x) * kPer + j;
        if (g < gl.E) prefix[g] = int(at < room ? at : room);
        at += count[j];
    }
    if (all > room) all = room;
    if (threadIdx.x == 0) prefix[gl.E] = int(all);
    __syncthreads();
    return int(all);
}

__device__ __forceinline__ void write_plan(const GroupList &gl, const TilePlan &p, int block)
{
    __shared__ int prefix[kMaxGroups + 1];
    const int all = tile_prefix(gl, p.height, p.room, prefix);
    if (block == 0)
        for (int g = threadIdx.x; g <= gl.E; g += kGgThreads) p.first[g] = prefix[g];
    const int i = block * kGgThreads + threadIdx.x;
    if (i >= all) return;
    int lo = 0, hi = gl.E;             // the last group that begins at or before i
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (prefix[mid] <= i) lo = mid;
        else hi = mid;
    }
    const int64_t begin = gl.begin(lo) + int64_t(i - prefix[lo]) * p.height, left = gl.begin(lo + 1) - begin;
    p.tiles[i] = make_int4(lo, int(begin), int(left < p.height ? left : p.height), 0);
}

// ---- weights as fragments --------------------------------------------------------
// A step is 16 k-values, eight a lane.  bf16: piece (g, tile of 32 columns, step, lane) holds of column col(lane % 32) the k-values
// step * 16 + (lane / 32) * 8 + [0, 8).  fp32: three bf16 parts of every value, pieces (g, tile, step, part, lane); a lane's eight are
// those of two pieces of four, step * 16 + (lane / 32) * 4 + [0, 4) and the same + 8.
template <typename T>
struct Step {
    static constexpr int E = 16 / sizeof(T);       // of a row's piece of 16 bytes
};

// result row m of a fragment is column ... of the wavefront's TN * 32 (see above)
__host__ __device__ __forceinline__ int fragment_column(int tile, int m, int TN)
{
    const int hi = (m >> 2) & 1, r = (m >> 3) * 4 + (m & 3);
    return tile / TN * TN * 32 + hi * TN * 16 + tile % TN * 16 + r;
}

// kForward: B = W[g] (k along its rows); else B = W[g]^T
template <typename T, bool kForward>
__device__ __forceinline__ void write_fragments(const GroupList &gl, const float *__restrict__ W, int K, int N, int tiles, int steps, int TN,
                                                uint4 *__restrict__ out, int64_t block, int64_t blocks)
{
    constexpr bool kSplit = sizeof(T) == 4;
    constexpr int E = 8;
    const int64_t per_group = int64_t(tiles) * steps * kWave, total = per_group * gl.E;
    for (int64_t i = block * kGgThreads + threadIdx.x; i < total; i += blocks * kGgThreads) {
        const int g = int(i / per_group);
        if (gl.begin(g + 1) <= gl.begin(g)) continue;
        const int64_t q = i % per_group;
        const int lane = int(q % kWave), step = int(q / kWave % steps), tile = int(q / kWave / steps);
        const int col = fragment_column(tile, lane & 31, TN), hi = lane >> 5;
        const float *w = W + int64_t(g) * K * N;
        float v[E];
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const int k = step * 2 * E + (kSplit ? (j >> 2) * 8 + hi * 4 + (j & 3) : hi * E + j);
            v[j] = 0.0f;
            if (col < N && k < K) v[j] = kForward ? w[int64_t(k) * N + col] : w[int64_t(col) * K + k];
        }
        if constexpr (kSplit) {
            const SplitPair split;
            uint32_t part[3][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) split(v[2 * j], v[2 * j + 1], part[0][j], part[1][j], part[2][j]);
#pragma unroll
            for (int p = 0; p < 3; ++p) out[(i / kWave * 3 + p) * kWave + lane] = make_uint4(part[p][0], part[p][1], part[p][2], part[p][3]);
        } else {
            out[i] = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
        }
    }
}

// ---- pieces of rows ----------------------------------------------------------------
__device__ __forceinline__ float widened(float x) { return x; }
__device__ __forceinline__ float widened(uint16_t x) { return bf16_to_f32(x); }

// open_word, open_piece: g where h > 0 (a NaN in h: not), zeros elsewhere
template <typename T>
__device__ __forceinline__ uint4 from_words(const T *p)
{
    const Words4 w = __builtin_nontemporal_load(reinterpret_cast<const Words4 *>(p));
    return make_uint4(w.x, w.y, w.z, w.w);
}

template <typename T>
__device__ __forceinline__ uint32_t open_word(uint32_t g, uint32_t h)
{
    if constexpr (sizeof(T) == 4) return __uint_as_float(h) > 0.0f ? g : 0u;
    else {
        const uint32_t lo = ((h & 0xFFFFu) - 1u) < 0x7F80u ? 0xFFFFu : 0u, hi = ((h >> 16) - 1u) < 0x7F80u ? 0xFFFF0000u : 0u;
        return g & (lo | hi);
    }
}
template <typename T>
__device__ __forceinline__ uint4 open_piece(const uint4 &g, const uint4 &h)
{
    return make_uint4(open_word<T>(g.x, h.x), open_word<T>(g.y, h.y), open_word<T>(g.z, h.z), open_word<T>(g.w, h.w));
}

__device__ __forceinline__ floatx16 times(const uint4 &a, const uint4 &b, const floatx16 &sum)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), sum, 0, 0, 0);
}

// sum += a b of operands in one part or in three
template <int kParts>
__device__ __forceinline__ void add_product(const uint4 (&a)[kParts], const uint4 (&b)[kParts], floatx16 &sum)
{
    if constexpr (kParts == 3) {
        sum = times(a[2], b[0], sum);
        sum = times(a[0], b[2], sum);
        sum = times(a[1], b[1], sum);
        sum = times(a[1], b[0], sum);
        sum = times(a[0], b[1], sum);
    }
    sum = times(a[0], b[0], sum);
}

// The run of work items that this block's die takes, and this block's first of them; they are a stride apart.
struct Share {
    int64_t item, end, stride;
    __device__ __forceinline__ explicit Share(int64_t total)
    {
        const int64_t per_die = (total + kDies - 1) / kDies, die = blockIdx.x % kDies;
        stride = gridDim.x / kDies;
        end = (die + 1) * per_die < total ? (die + 1) * per_die : total;
        item = die * per_die + blockIdx.x / kDies;
    }
};

// ---- rows times weights ------------------------------------------------------------
struct RowsCall {
    GroupList gl;
    const int4 *tiles;
    const int32_t *tile_count;
    const uint4 *B;            // fragments: [E][column tiles][steps][64]
    const float *bias;         // [E][n_tiles BN], zeros past N, or NULL
    const void *A, *H;         // rows; H: their mask (kMask)
    void *C;
    const float *W;            // as they are, [E][K N], value (k, column) at k w_k + column w_col
    int64_t lda, ldc, w_k, w_col;
    int K, N, steps, n_tiles;  // n_tiles: of BN columns
    bool relu;
};

// column col of row v from what the operands are, in fp32 (for results that parts of them cannot give)
template <bool kMask>
__device__ __forceinline__ float in_fp32(const float *a, const float *h, const float *w, int64_t w_k, int K)
{
    float sum = 0.0f;
    for (int k = 0; k < K; ++k) sum = fmaf(kMask && !(h[k] > 0.0f) ? 0.0f : a[k], w[k * w_k], sum);
    return sum;
}

// Place of a row's piece in LDS, rows of PP pieces: exchanged by the row's number, so that what 16 lanes take at once, a piece each of 16
// neighbouring rows, lies in all banks.
template <int PP>
__device__ __forceinline__ int spread(int row, int piece)
{
    constexpr int kSpan = PP < 16 ? PP : 16;
    return row * PP + (piece ^ ((row / (16 / kSpan)) & (kSpan - 1)));
}

constexpr int kRowPP = 32;                 // 16-byte pieces of a row in LDS at a time
// blocks of a compute unit that the registers leave room for (four wavefronts each)
template <int TN>
constexpr int kRowBlocksPerCu = TN > 1 ? 2 : 3;

// The numbers of a tile's rows are fetched two tiles ahead, its rows one.  fp32: in LDS three bf16 parts, [part][row][16 bytes: eight k-values].
template <typename T, int WN, int TN, bool kMask, bool kWords, bool kStore16>
__global__ __launch_bounds__(kGgThreads, kRowBlocksPerCu<TN>) void grouped_rows_kernel(RowsCall q)
{
    constexpr bool kSplit = sizeof(T) == 4;
    constexpr int WM = 4 / WN, TM = kTileM / WM / 32, E = Step<T>::E, PP = kRowPP, kParts = kSplit ? 3 : 1, kUnits = kSplit ? PP / 2 : PP;
    constexpr int kRowsAtOnce = kGgThreads / PP, kPieces = kTileM / kRowsAtOnce;    // of a thread
    constexpr int kSteps = kUnits / 2, kAhead = kSplit ? 2 : 4;                     // of 16 k-values; steps that weights are fetched ahead
    typedef RowPiece<T, kWords> P;
    constexpr int kRowPieces = TN * 32 / E;    // of a wavefront's columns of a row
    constexpr int kOut = 4 * 32 * kRowPieces, kIn = kParts * kTileM * kUnits;
    __shared__ uint4 As[kIn > kOut ? kIn : kOut];
    __shared__ int32_t rows[2][kTileM];        // of this tile and the next, -1: none
    const SplitPair split;
    const T *A = static_cast<const T *>(q.A), *H = static_cast<const T *>(q.H);
    const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, hi = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int piece = tid % PP, row0 = tid / PP;
    const int64_t last = P::last_place(q.gl.n, q.lda, q.K);
    Share share(int64_t(*q.tile_count) * q.n_tiles);
    if (share.item >= share.end) return;
    const int chunks = (q.steps + kSteps - 1) / kSteps;
    const bool ragged = kWords && q.K % E != 0;

    auto tile_of = [&](int64_t item) { return q.n_tiles == 1 ? item : item / q.n_tiles; };
    auto row_of = [&](int64_t item) {          // of thread tid < 64
        const int4 t = q.tiles[tile_of(item)];
        return tid < t.z ? int32_t(q.gl.row(t.y + tid)) : -1;
    };
    auto element = [&](int at, int i, int chunk) {
        const int v = rows[at][row0 + i * kRowsAtOnce], k = (chunk * PP + piece) * E;
        return int64_t(v < 0 ? 0 : v) * q.lda + (k < q.K ? k : 0);
    };
    uint4 held[kPieces], mask[kMask ? kPieces : 1];
    auto fetch = [&](int at, int chunk) {
        const int valid = q.K - (chunk * PP + piece) * E;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int64_t e = element(at, i, chunk);
            held[i] = P::load(A, e, valid, last);
            if constexpr (kMask) mask[i] = P::load(H, e, valid, last);
        }
    };

    if (tid < kTileM) rows[0][tid] = row_of(share.item);
    int32_t pending = -1;                      // of the tile after this one
    if (tid < kTileM && share.item + share.stride < share.end) pending = row_of(share.item + share.stride);
    __syncthreads();
    fetch(0, 0);
    for (int at = 0;; at ^= 1) {
        const int64_t item = share.item, next = item + share.stride;
        const bool more = next < share.end;
        const int64_t tile = tile_of(item);
        const int group = __builtin_amdgcn_readfirstlane(q.tiles[tile].x);
        const int nt = int(item - tile * q.n_tiles) * WN * TN + wn * TN;      // first of the wavefront's column tiles
        const int n0 = nt * 32 + hi * TN * 16;                         // first of the lane's columns
        const uint4 *B = q.B + (int64_t(group) * q.n_tiles * WN * TN + nt) * q.steps * (kParts * kWave);
        auto weights = [&](int j, int step, uint4 (&w)[kParts]) {
#pragma unroll
            for (int o = 0; o < kParts; ++o) w[o] = (B + ((j * q.steps + step) * kParts + o) * kWave)[lane];
        };
        const float *bias = q.bias ? q.bias + int64_t(group) * q.n_tiles * (WN * TN * 32) + n0 : nullptr;      // of the lane's columns
        floatx16 acc[TM][TN];
        if (!kSplit && bias) {
            const float4 *b4 = reinterpret_cast<const float4 *>(bias);
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float4 b = b4[j * 4 + r];
#pragma unroll
                    for (int i = 0; i < TM; ++i) {
                        acc[i][j][4 * r] = b.x;
                        acc[i][j][4 * r + 1] = b.y;
                        acc[i][j][4 * r + 2] = b.z;
                        acc[i][j][4 * r + 3] = b.w;
                    }
                }
        } else {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
        }
        for (int c = 0; c < chunks; ++c) {
            const int s0 = c * kSteps, s1 = q.steps - s0 < kSteps ? q.steps - s0 : kSteps;      // multiples of kStepsUp
            uint4 b[kSteps][TN][kParts];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int j = 0; j < TN; ++j) weights(j, s0 + u, b[u][j]);
            __syncthreads();           // everyone has read what was there
            const int valid = q.K - (c * PP + piece) * E;
            if constexpr (kMask) {
#pragma unroll
                for (int i = 0; i < kPieces; ++i) held[i] = open_piece<T>(held[i], mask[i]);
            }
            if (ragged) {
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    const int64_t over = element(at, i, c) - last;
                    if (over > 0) held[i] = P::moved(held[i], int(over), P::left_out(A, kMask ? H : nullptr, q.gl.n, q.lda, q.K));
                    held[i] = P::cut(held[i], valid);
                }
            }
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const uint4 p = valid > 0 ? held[i] : make_uint4(0u, 0u, 0u, 0u);
                if constexpr (kSplit) {        // pieces 4 s + hi and 4 s + 2 + hi of a row are the eight values of a lane at step s
                    uint32_t part[3][2];
                    split(__uint_as_float(p.x), __uint_as_float(p.y), part[0][0], part[1][0], part[2][0]);
                    split(__uint_as_float(p.z), __uint_as_float(p.w), part[0][1], part[1][1], part[2][1]);
                    const int at16 = spread<kUnits>(row0 + i * kRowsAtOnce, piece / 4 * 2 + piece % 2);
#pragma unroll
                    for (int o = 0; o < 3; ++o)
                        reinterpret_cast<uint2 *>(&As[o * kTileM * kUnits + at16])[piece / 2 % 2] = make_uint2(part[o][0], part[o][1]);
                } else {
                    As[spread<kUnits>(row0 + i * kRowsAtOnce, piece)] = p;
                }
            }
            if (c == 0 && tid < kTileM) rows[at ^ 1][tid] = pending;
            __syncthreads();
            if (c + 1 < chunks) fetch(at, c + 1);
            else if (more) {
                fetch(at ^ 1, 0);
                pending = -1;
                if (tid < kTileM && next + share.stride < share.end) pending = row_of(next + share.stride);
            }
            // unrolled, and each step's loads kept in their place: of a loop the compiler makes copies of what is in flight, and waits for it
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                if (s % kAhead == 0 && s >= s1) break;
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    uint4 a[kParts];
#pragma unroll
                    for (int o = 0; o < kParts; ++o) a[o] = As[o * kTileM * kUnits + spread<kUnits>((wm * TM + i) * 32 + l31, 2 * s + hi)];
#pragma unroll
                    for (int j = 0; j < TN; ++j) add_product<kParts>(b[s][j], a, acc[i][j]);
                }
                if (s + kAhead < kSteps) {
                    const int ahead = s0 + s + kAhead < q.steps ? s0 + s + kAhead : q.steps - 1;     // (past the last one: again)
#pragma unroll
                    for (int j = 0; j < TN; ++j) weights(j, ahead, b[s + kAhead < kSteps ? s + kAhead : 0][j]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        // A lane has, of row l31 of the tile's 32, the columns [0, 16 TN) or the next as many of its wavefront's.  Through LDS, 32 rows at a
        // time: a store then goes to whole rows of the wavefront's columns, 64 to 256 bytes each.
        T *C = static_cast<T *>(q.C);
        __syncthreads();               // everyone has read the last steps
        uint4 *mine = As + wave * (32 * kRowPieces);
        const int col0 = nt * 32;      // the wavefront's first column
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            uint32_t odd = 0;              // the lane's columns whose sum is not finite
#pragma unroll
            for (int x = 0; x < TN * 16 / E; ++x) {
                float z[E];
#pragma unroll
                for (int y = 0; y < E; ++y) {
                    z[y] = acc[i][x * E / 16][x * E % 16 + y];
                    if constexpr (kSplit) {
                        z[y] *= kSplitUnscale;
                        if (!(fabsf(z[y]) <= FLT_MAX)) odd |= 1u << (x * E + y);
                        if (bias) z[y] += bias[x * E + y];
                    }
                    if (q.relu) z[y] = z[y] > 0.0f ? z[y] : 0.0f;
                }
                Chunk<T>::store(reinterpret_cast<T *>(&mine[spread<kRowPieces>(l31, hi * (kRowPieces / 2) + x)]), z);
            }
            if constexpr (kSplit) {
                const int64_t v = rows[at][(wm * TM + i) * 32 + l31];
                if (__any(odd && v >= 0))
                    for (int y = 0; y < TN * 16; ++y)
                        if (v >= 0 && (odd >> y & 1) && n0 + y < q.N) {
                            float z = in_fp32<kMask>(A + v * q.lda, H + v * q.lda, q.W + int64_t(group) * q.K * q.N + (n0 + y) * q.w_col, q.w_k, q.K);
                            if (bias) z += bias[y];
                            if (q.relu) z = z > 0.0f ? z : 0.0f;
                            reinterpret_cast<float *>(&mine[spread<kRowPieces>(l31, hi * (kRowPieces / 2) + y / E)])[y % E] = z;
                        }
            }
            __builtin_amdgcn_wave_barrier();
            constexpr int kStores = kRowPieces / 2;
            uint4 z[kStores];
            int32_t v[kStores];
            bool full = true;
            const int p = lane % kRowPieces, col = col0 + p * E;
#pragma unroll
            for (int x = 0; x < kStores; ++x) {
                const int r = x * (64 / kRowPieces) + lane / kRowPieces;
                z[x] = mine[spread<kRowPieces>(r, p)];
                v[x] = rows[at][(wm * TM + i) * 32 + r];
                full = full && v[x] >= 0;
            }
            __builtin_amdgcn_wave_barrier();
            if (kStore16 && __all(full) && col0 + TN * 32 <= q.N) {      // (without a branch between the stores)
#pragma unroll
                for (int x = 0; x < kStores; ++x)
                    __builtin_nontemporal_store(Words4{z[x].x, z[x].y, z[x].z, z[x].w}, reinterpret_cast<Words4 *>(C + int64_t(v[x]) * q.ldc + col));
                continue;
            }
#pragma unroll
            for (int x = 0; x < kStores; ++x) {
                if (v[x] < 0 || col >= q.N) continue;
                T *out = C + int64_t(v[x]) * q.ldc + col;
                if (kStore16 && col + E <= q.N) {
                    *reinterpret_cast<Words4 *>(out) = Words4{z[x].x, z[x].y, z[x].z, z[x].w};
                } else {
                    float w[E];
                    Chunk<T>::widen(z[x], w);
#pragma unroll
                    for (int y = 0; y < E; ++y)
                        if (col + y < q.N) {
                            if constexpr (sizeof(T) == 4) out[y] = w[y];
                            else out[y] = uint16_t(__float_as_uint(w[y]) >> 16);
                        }
                }
            }
        }
        if (!more) return;
        share.item = next;
    }
}

// ---- rows times weights that stay in LDS -----------------------------------------------
// Where a group's weights, or those of 64 to 256 of its columns, fit 128 KB of LDS (256 x 256 of bf16, 128 x 128 of fp32), a block per compute unit
// holds them for a run of the group's rows.  Its eight wavefronts then have nothing in common: each takes 32 rows at a time,
// its lanes' k-values of a row straight into registers (512 bytes of a row: sixteen steps), all columns from them, and the
// results through 4 KB of LDS of its own into whole lines.  No barrier but where the weights change, and of the L2 only rows and
// results are asked (64-row tiles that fetched the weights from it: 128 KB a tile beside 64 KB of rows and results; 1,000,003 rows of
// 256 -> 256 in bf16 268 us; without rows and stores still 175).
constexpr int kResWaves = 8;
constexpr int kResRows = 32;              // rows of a wavefront's tile
constexpr int kResPieces = 8192;          // 16-byte pieces of weights in LDS
constexpr int kResChunkCols = 4;          // column tiles where a row has several chunks: all their sums are in registers
// A step is 16 k-values.
template <typename T>
struct ResStep {
    static constexpr bool kSplit = sizeof(T) == 4;
    static constexpr int kParts = kSplit ? 3 : 1, kChunk = kSplit ? 8 : 16;      // parts of an operand; steps of 512 bytes of a row
};

struct ResidentCall {
    GroupList gl;
    const int4 *tiles;
    const int32_t *first;      // tiles of the groups before each one, [E + 1]
    const uint4 *B;            // fragments: [E][n_tiles][CT][steps][64]
    const float *bias;         // [E][n_tiles CT 32], zeros past N, or NULL
    const void *A, *H;
    void *C;
    const float *W;            // as they are, [E][K N], value (k, column) at k w_k + column w_col
    int64_t lda, ldc, w_k, w_col;
    int K, N, steps, n_tiles, CT;      // CT: column tiles of 32 in LDS
    bool relu;
};

// NT: column tiles whose sums are in registers at once; kMulti: a row has several chunks (then NT = CT; bf16 without a mask)
template <typename T, int NT, bool kMulti, bool kMask, bool kWords, bool kStore16>
__global__ __launch_bounds__(kResWaves * 64, 2) void grouped_resident_kernel(ResidentCall q)
{
    constexpr int E = 16 / sizeof(T), TN = sizeof(T) == 2 ? 2 : 1;     // TN column tiles make 128 bytes of a row of results
    constexpr int kUnit = 8;                                           // pieces of those
    constexpr bool kSplit = ResStep<T>::kSplit;
    constexpr int kParts = ResStep<T>::kParts, kResSteps = ResStep<T>::kChunk, kQuarterSteps = kResSteps / 4;
    const SplitPair split;
    typedef RowPiece<T, kWords> P;
    __shared__ uint4 Ws[kResPieces];
    __shared__ uint4 staging[kResWaves][kResRows * kUnit];
    const T *A = static_cast<const T *>(q.A), *H = static_cast<const T *>(q.H);
    T *C = static_cast<T *>(q.C);
    const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, hi = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t last = P::last_place(q.gl.n, q.lda, q.K);
    const int chunks = kMulti ? (q.steps + kResSteps - 1) / kResSteps : 1;
    uint4 *mine = staging[wave];

    // this block's range of the items (group, column part, tile), a die's blocks side by side
    const int64_t total = int64_t(q.first[q.gl.E]) * q.n_tiles;
    const int64_t blocks = gridDim.x, b = (blockIdx.x % kDies) * (blocks / kDies) + blockIdx.x / kDies;
    int64_t item = total * b / blocks;
    const int64_t end = total * (b + 1) / blocks;
    if (item >= end) return;
    int group = 0;
    for (int lo = 0, hi_ = q.gl.E; hi_ - lo > 1;) {      // the last group that begins at or before the item
        const int mid = (lo + hi_) / 2;
        if (int64_t(q.first[mid]) * q.n_tiles <= item) lo = mid;
        else hi_ = mid;
        group = lo;
    }
    while (item < end) {
        group = __builtin_amdgcn_readfirstlane(group);
        const int64_t g0 = q.first[group], g1 = q.first[group + 1], size = g1 - g0;
        if (item >= g1 * q.n_tiles) {      // (also steps over empty groups)
            ++group;
            continue;
        }
        const int64_t in_group = item - g0 * q.n_tiles;
        const int part = int(in_group / size);
        int64_t t = g0 + in_group % size;                           // tiles [t, t_end) of the plan
        const int64_t left = end - item, t_end = t + left < g1 ? t + left : g1;
        item += t_end - t;

        __syncthreads();                                            // everyone is done with the weights before
        const int pieces = q.CT * q.steps * kParts * kWave;
        const uint4 *B = q.B + (int64_t(group) * q.n_tiles + part) * pieces;
        {
            constexpr int kT = kResWaves * 64;
            int i = tid;
            for (; i + 7 * kT < pieces; i += 8 * kT) {
                uint4 v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u] = B[i + u * kT];
#pragma unroll
                for (int u = 0; u < 8; ++u) Ws[i + u * kT] = v[u];
            }
            for (; i < pieces; i += kT) Ws[i] = B[i];
        }
        __syncthreads();

        const int n0 = part * q.CT * 32;
        const float *bias = q.bias ? q.bias + (int64_t(group) * q.n_tiles + part) * q.CT * 32 : nullptr;
        auto row_of = [&](int64_t tile) {
            int32_t v = -1;
            if (tile < t_end) {
                const int4 d = q.tiles[tile];
                if (l31 < d.z) v = int32_t(q.gl.row(d.y + l31));
            }
            return v;
        };
        t += wave;
        int32_t row = row_of(t), coming = row_of(t + kResWaves);
        for (; t < t_end; t += kResWaves) {
            const int32_t after = row_of(t + 2 * kResWaves);
            // rows x * 8 + lane / 8 of the tile, whose pieces lane % 8, + 8, ... this lane loads and stores
            int32_t v[4];
            int limit[4];                  // the last place in the row where 16 bytes of whole words are left
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                v[x] = __shfl(row, x * 8 + lane / 8, kWave);
                const int64_t from = int64_t(v[x] < 0 ? 0 : v[x]) * q.lda;       // (a row that is none reads the first, and is not stored)
                limit[x] = last - from < q.K ? int(last - from) : q.K;
            }
            auto row_at = [&](const T *p, int r) { return p + int64_t(v[r] < 0 ? 0 : v[r]) * q.lda; };
            const bool full = __all((v[0] | v[1] | v[2] | v[3]) >= 0);
            // A chunk: 128 bytes of 32 rows at a time through the wavefront's LDS, from whole lines to a row per lane.  (Loads that could go one
            // way or the other were waited for one by one: the common case has a path without a branch.)
            uint4 x[16];       // fp32: two a step, taken apart as the step is multiplied (parts of all steps would take half as many registers again)
            auto turn = [&](int quarter, const uint4 (&p)[4]) {
#pragma unroll
                for (int r = 0; r < 4; ++r) mine[spread<kUnit>(r * 8 + lane / 8, lane % 8)] = p[r];
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int s = 0; s < 4; ++s) x[quarter * 4 + s] = mine[spread<kUnit>(l31, 2 * s + hi)];
                __builtin_amdgcn_wave_barrier();
            };
            auto fetch = [&](int c) {
                const int k0 = c * kResSteps * 16 + lane % 8 * E;
                constexpr int kQuarter = 8 * E;
                if (kWords && (c + 1) * kResSteps * 16 <= q.K) {
                    uint4 p[4][4], m[kMask ? 4 : 1][4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            p[i][r] = from_words(row_at(A, r) + k0 + i * kQuarter);
                            if constexpr (kMask) m[i][r] = from_words(row_at(H, r) + k0 + i * kQuarter);
                        }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (kMask) {
#pragma unroll
                            for (int r = 0; r < 4; ++r) p[i][r] = open_piece<T>(p[i][r], m[i][r]);
                        }
                        turn(i, p[i]);
                    }
                    return;
                }
                uint4 p[4][4], m[kMask ? 4 : 1][4];
                auto in_row = [&](int quarter) { return k0 + quarter * kQuarter < q.K ? k0 + quarter * kQuarter : 0; };
#pragma unroll
                for (int quarter = 0; quarter < 4; ++quarter)
                    if (c * kResSteps + quarter * kQuarterSteps < q.steps) {
                        const int valid = q.K - k0 - quarter * kQuarter;
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            p[quarter][r] = P::load(row_at(A, r), in_row(quarter), valid, limit[r]);
                            if constexpr (kMask) m[quarter][r] = P::load(row_at(H, r), in_row(quarter), valid, limit[r]);
                        }
                    }
#pragma unroll
                for (int quarter = 0; quarter < 4; ++quarter)
                    if (c * kResSteps + quarter * kQuarterSteps < q.steps) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            uint4 &o = p[quarter][r];
                            if constexpr (kMask) o = open_piece<T>(o, m[quarter][r]);
                            if (kWords && in_row(quarter) > limit[r])
                                o = P::moved(o, in_row(quarter) - limit[r], P::left_out(A, kMask ? H : nullptr, q.gl.n, q.lda, q.K));
                            if (kWords) o = P::cut(o, q.K - k0 - quarter * kQuarter);
                        }
                        turn(quarter, p[quarter]);
                    }
            };
            floatx16 acc[NT], rest[kSplit ? NT : 1];       // fp32: the five smaller products have sums of their own
            // a lane's columns of a column tile, and their bias: see fragment_column
            auto bias_of = [&](int tile, float (&v)[16]) {
                const float4 *b4 = reinterpret_cast<const float4 *>(bias + tile / TN * TN * 32 + hi * TN * 16 + tile % TN * 16);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float4 b = bias ? b4[r] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    v[4 * r] = b.x;
                    v[4 * r + 1] = b.y;
                    v[4 * r + 2] = b.z;
                    v[4 * r + 3] = b.w;
                }
            };
            auto start = [&](int ct) {
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    float v[16];
                    if constexpr (!kSplit) bias_of(ct + j, v);
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        acc[j][r] = kSplit ? 0.0f : v[r];
                        if constexpr (kSplit) rest[j][r] = 0.0f;
                    }
                }
            };
            auto again = [&](int col) {
                float sum = 0.0f;
                if constexpr (kSplit)
                    if (row >= 0 && col < q.N)
                        sum = in_fp32<kMask>(A + int64_t(row) * q.lda, H + int64_t(row) * q.lda, q.W + int64_t(group) * q.K * q.N + col * q.w_col, q.w_k, q.K);
                return sum;
            };
            auto store = [&](int ct) {
#pragma unroll
                for (int unit = 0; unit < NT / TN; ++unit) {
                    const int col0 = (ct + unit * TN) * 32;        // of the part
                    if (n0 + col0 >= q.N) break;
                    if constexpr (kSplit) {
                        float b[16];
                        bias_of(ct + unit, b);
                        bool odd = false;
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const float v = (acc[unit][r] + rest[unit][r]) * kSplitUnscale;
                            odd = odd || !(fabsf(v) <= FLT_MAX);
                            acc[unit][r] = v;
                        }
                        if (__any(odd && row >= 0))
#pragma unroll
                            for (int r = 0; r < 16; ++r)
                                if (!(fabsf(acc[unit][r]) <= FLT_MAX)) acc[unit][r] = again(n0 + col0 + hi * 16 + r);
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[unit][r] += b[r];
                    }
#pragma unroll
                    for (int x = 0; x < TN * 16 / E; ++x) {
                        float z[E];
#pragma unroll
                        for (int y = 0; y < E; ++y) {
                            z[y] = acc[unit * TN + x * E / 16][x * E % 16 + y];
                            if (q.relu) z[y] = z[y] > 0.0f ? z[y] : 0.0f;
                        }
                        Chunk<T>::store(reinterpret_cast<T *>(&mine[spread<kUnit>(l31, hi * (kUnit / 2) + x)]), z);
                    }
                    __builtin_amdgcn_wave_barrier();
                    const int col = n0 + col0 + lane % 8 * E;
                    uint4 z[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) z[x] = mine[spread<kUnit>(x * 8 + lane / 8, lane % 8)];
                    __builtin_amdgcn_wave_barrier();
                    if (kStore16 && full && n0 + col0 + TN * 32 <= q.N) {
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            __builtin_nontemporal_store(Words4{z[x].x, z[x].y, z[x].z, z[x].w}, reinterpret_cast<Words4 *>(C + int64_t(v[x]) * q.ldc + col));
                        continue;
                    }
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        if (v[x] < 0 || col >= q.N) continue;
                        T *o = C + int64_t(v[x]) * q.ldc + col;
                        if (kStore16 && col + E <= q.N) {
                            __builtin_nontemporal_store(Words4{z[x].x, z[x].y, z[x].z, z[x].w}, reinterpret_cast<Words4 *>(o));
                            continue;
                        }
                        float w[E];
                        Chunk<T>::widen(z[x], w);
#pragma unroll
                        for (int y = 0; y < E; ++y)
                            if (col + y < q.N) {
                                if constexpr (sizeof(T) == 4) o[y] = w[y];
                                else o[y] = uint16_t(__float_as_uint(w[y]) >> 16);
                            }
                    }
                }
            };
            if (kMulti) start(0);
            for (int c = 0; c < chunks; ++c) {
                fetch(c);
                for (int ct = 0; ct < q.CT; ct += NT) {
                    if (!kMulti) start(ct);
#pragma unroll
                    for (int s = 0; s < kResSteps; ++s) {
                        if (s % kQuarterSteps == 0 && c * kResSteps + s >= q.steps) break;
                        uint4 xp[kParts];
                        if constexpr (kSplit) {
                            // (held in the loop: taken out of it, the parts of all steps would not fit the registers)
                            asm volatile("" : "+v"(x[2 * s].x), "+v"(x[2 * s].y), "+v"(x[2 * s].z), "+v"(x[2 * s].w), "+v"(x[2 * s + 1].x), "+v"(x[2 * s + 1].y),
                                         "+v"(x[2 * s + 1].z), "+v"(x[2 * s + 1].w));
                            const uint32_t v[8] = {x[2 * s].x, x[2 * s].y, x[2 * s].z, x[2 * s].w, x[2 * s + 1].x, x[2 * s + 1].y, x[2 * s + 1].z, x[2 * s + 1].w};
                            uint32_t part[3][4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) split(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]), part[0][j], part[1][j], part[2][j]);
#pragma unroll
                            for (int o = 0; o < kParts; ++o) xp[o] = make_uint4(part[o][0], part[o][1], part[o][2], part[o][3]);
                        } else {
                            xp[0] = x[s];
                        }
#pragma unroll
                        for (int j = 0; j < NT; ++j) {
                            const uint4 *w = Ws + (((ct + j) * q.steps + c * kResSteps + s) * kParts) * kWave + lane;
                            if constexpr (kSplit) {
                                const uint4 h = w[0], m = w[kWave], l = w[2 * kWave];
                                acc[j] = times(h, xp[0], acc[j]);
                                rest[j] = times(l, xp[0], rest[j]);
                                rest[j] = times(h, xp[2], rest[j]);
                                rest[j] = times(m, xp[1], rest[j]);
                                rest[j] = times(m, xp[0], rest[j]);
                                rest[j] = times(h, xp[1], rest[j]);
                            } else {
                                acc[j] = times(w[0], xp[0], acc[j]);
                            }
                        }
                        if constexpr (kSplit) __builtin_amdgcn_sched_barrier(0);
                    }
                    if (!kMulti) store(ct);
                }
            }
            if (kMulti) store(0);
            row = coming;
            coming = after;
        }
    }
}

// ---- weight gradients ----------------------------------------------------------------
struct WeightCall {
    GroupList gl;
    const int4 *runs;
    const int32_t *first;          // runs of each group before it, [E + 1]
    const void *X, *G, *H;         // H: the mask of G (kMask)
    int64_t ldx, ldg;
    int M, N, m_tiles, n_tiles;
    float *dW, *db;                // [E][M][N], [E][N] or NULL
    float *partial, *colsum;       // of each run: [M][N], [N]
};

typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;
// eight k-values (rows of LDS) of a lane's column: of rows 0..3 and 4..7 from `at` on, `row` elements apart
__device__ __forceinline__ uint4 along_rows(const uint16_t *at, int row)
{
    const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)(at)));
    const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)(at + 4 * row)));
    return make_uint4(lo.x, lo.y, hi.x, hi.y);
}

// One operand's slabs of ROWS rows x COLS columns on their way through registers into LDS: kDepth slabs in flight.
template <typename T, int ROWS, int COLS, int THREADS, bool kWords>
struct SlabPieces {
    static constexpr int E = 16 / sizeof(T), PP = COLS / E, kAtOnce = THREADS / PP, kPieces = ROWS / kAtOnce;
    static_assert(kPieces >= 1 && kPieces * kAtOnce == ROWS, "pieces of a slab");
    typedef RowPiece<T, kWords> P;
    // in LDS, in bf16: blocks of 32 columns exchanged by the row's number, for the transposing read takes 4 rows x 16 columns at once
    static __device__ __forceinline__ int place(int row, int c) { return row * COLS + ((c >> 5) ^ (row & 3)) * 32 + (c & 31); }
    // fp32: three parts, a slab each
    static __device__ __forceinline__ void put(uint16_t *slab, int row, int c, const uint4 &p)
    {
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint4 *>(&slab[place(row, c)]) = p;
        else {
            const SplitPair split;
            uint32_t part[3][2];
            split(__uint_as_float(p.x), __uint_as_float(p.y), part[0][0], part[1][0], part[2][0]);
            split(__uint_as_float(p.z), __uint_as_float(p.w), part[0][1], part[1][1], part[2][1]);
#pragma unroll
            for (int o = 0; o < 3; ++o) *reinterpret_cast<uint2 *>(&slab[o * ROWS * COLS + place(row, c)]) = make_uint2(part[o][0], part[o][1]);
        }
    }
    static __device__ __forceinline__ int row(int i) { return int(threadIdx.x) / PP + i * kAtOnce; }
    static __device__ __forceinline__ int column() { return int(threadIdx.x) % PP * E; }
};

// A block's tile is (WM TM 32) x (WN TN 32); kDepth slabs of rows are in flight in registers, two in LDS (one barrier a slab).
template <typename T, int WM, int WN, int TM, int TN, bool kMask, bool kWords>
__global__ __launch_bounds__(WM *WN * 64, 2) void grouped_weight_kernel(WeightCall q)
{
    constexpr int kThreads = WM * WN * 64, BM = WM * TM * 32, BN = WN * TN * 32, kDepth = 2;
    constexpr bool kSplit = sizeof(T) == 4;
    constexpr int E = Step<T>::E, kParts = kSplit ? 3 : 1, kSlab = kSplit ? 16 : 32;
    constexpr int kListed = 64 * kSlab;                    // rows whose numbers lie in LDS, twice: these and the ones to come
    typedef SlabPieces<T, kSlab, BM, kThreads, kWords> XS;
    typedef SlabPieces<T, kSlab, BN, kThreads, kWords> ZS;
    typedef RowPiece<T, kWords> P;
    __shared__ __attribute__((aligned(16))) uint16_t Xs[2][kParts * kSlab * BM];
    __shared__ __attribute__((aligned(16))) uint16_t Zs[2][kParts * kSlab * BN];
    __shared__ int32_t listed[2][kListed];
    const T *X = static_cast<const T *>(q.X), *G = static_cast<const T *>(q.G), *H = static_cast<const T *>(q.H);
    const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, hi = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int64_t x_last = P::last_place(q.gl.n, q.ldx, q.M), g_last = P::last_place(q.gl.n, q.ldg, q.N);
    const int tiles = q.m_tiles * q.n_tiles;
    const int quarter = lane >> 4, i16 = lane & 15;
    const int tr_row = 8 * (quarter >> 1) + (i16 >> 2), tr_col = 16 * (quarter & 1) + 4 * (i16 & 3);

    Share share(int64_t(q.first[q.gl.E]) * tiles);
    for (; share.item < share.end; share.item += share.stride) {
        const int64_t run = share.item / tiles;
        const int tile = int(share.item % tiles), m0 = tile / q.n_tiles * BM, n0 = tile % q.n_tiles * BN;
        const int4 t = q.runs[run];
        const int slabs = (t.z + kSlab - 1) / kSlab;
        const bool sum = m0 == 0 && q.db;
        const int xc = m0 + XS::column(), zc = n0 + ZS::column(), xv = q.M - xc, zv = q.N - zc;
        const bool x_ragged = kWords && q.M % E != 0, z_ragged = kWords && q.N % E != 0;
        auto list = [&](int block) {           // numbers of the rows [block kListed, + kListed) of the run
            for (int r = tid; r < kListed; r += kThreads) {
                const int at = block * kListed + r;
                listed[block & 1][r] = at < t.z ? int32_t(q.gl.row(t.y + at)) : -1;
            }
        };
        auto row = [&](int slab, int r) { return listed[slab / 64 & 1][slab % 64 * kSlab + r]; };
        uint4 xh[kDepth][XS::kPieces], zh[kDepth][ZS::kPieces], hh[kDepth][kMask ? ZS::kPieces : 1];
        auto fetch = [&](int slab, int d) {
#pragma unroll
            for (int i = 0; i < XS::kPieces; ++i) {
                const int v = row(slab, XS::row(i));
                xh[d][i] = P::load(X, int64_t(v < 0 ? 0 : v) * q.ldx + (xv > 0 ? xc : 0), v < 0 ? 0 : xv, x_last);
            }
#pragma unroll
            for (int i = 0; i < ZS::kPieces; ++i) {
                const int v = row(slab, ZS::row(i));
                const int64_t e = int64_t(v < 0 ? 0 : v) * q.ldg + (zv > 0 ? zc : 0);
                zh[d][i] = P::load(G, e, v < 0 ? 0 : zv, g_last);
                if constexpr (kMask) hh[d][i] = P::load(H, e, v < 0 ? 0 : zv, g_last);
            }
        };
        floatx16 acc[TM][TN];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
        float col[E];
#pragma unroll
        for (int j = 0; j < E; ++j) col[j] = 0.0f;
        __syncthreads();                       // (the run before is done with LDS)
        list(0);
        __syncthreads();
#pragma unroll
        for (int d = 0; d < kDepth; ++d)
            if (d < slabs) fetch(d, d);
        for (int s0 = 0; s0 < slabs; s0 += kDepth) {
#pragma unroll
            for (int d = 0; d < kDepth; ++d) {
                const int s = s0 + d;
                if (s >= slabs) break;
                uint16_t *x = Xs[s & 1], *z = Zs[s & 1];
#pragma unroll
                for (int i = 0; i < XS::kPieces; ++i) {
                    const int v = row(s, XS::row(i));
                    uint4 p = xh[d][i];
                    if (x_ragged && v >= 0) {        // (fp32: a column is taken apart together with its neighbour, which may be none)
                        const int64_t over = int64_t(v) * q.ldx + (xv > 0 ? xc : 0) - x_last;
                        if (over > 0) p = P::moved(p, int(over), P::left_out(X, nullptr, q.gl.n, q.ldx, q.M));
                        if constexpr (kSplit) p = P::cut(p, xv);
                    }
                    if (v < 0) p = make_uint4(0u, 0u, 0u, 0u);
                    XS::put(x, XS::row(i), XS::column(), p);
                }
#pragma unroll
                for (int i = 0; i < ZS::kPieces; ++i) {
                    const int v = row(s, ZS::row(i));
                    uint4 p = zh[d][i];
                    if constexpr (kMask) p = open_piece<T>(p, hh[d][i]);
                    if (z_ragged && v >= 0) {
                        const int64_t over = int64_t(v) * q.ldg + (zv > 0 ? zc : 0) - g_last;
                        if (over > 0) p = P::moved(p, int(over), P::left_out(G, kMask ? H : nullptr, q.gl.n, q.ldg, q.N));
                        if constexpr (kSplit) p = P::cut(p, zv);
                    }
                    if (v < 0) p = make_uint4(0u, 0u, 0u, 0u);
                    ZS::put(z, ZS::row(i), ZS::column(), p);
                    if (sum) {
                        float w[E];
                        Chunk<T>::widen(p, w);
#pragma unroll
                        for (int j = 0; j < E; ++j) col[j] += w[j];
                    }
                }
                if (s % 64 == 0 && (s + 64) < slabs) list(s / 64 + 1);       // (in use from slab s + 64 - kDepth on, some barriers away)
                __syncthreads();
                if (s + kDepth < slabs) fetch(s + kDepth, d);
#pragma unroll
                for (int k = 0; k < kSlab; k += 16) {
                    uint4 b[TN][kParts];
#pragma unroll
                    for (int j = 0; j < TN; ++j)
#pragma unroll
                        for (int o = 0; o < kParts; ++o) b[j][o] = along_rows(&z[o * kSlab * BN + ZS::place(k + tr_row, (wn * TN + j) * 32 + tr_col)], BN);
#pragma unroll
                    for (int i = 0; i < TM; ++i) {
                        uint4 a[kParts];
#pragma unroll
                        for (int o = 0; o < kParts; ++o) a[o] = along_rows(&x[o * kSlab * BM + XS::place(k + tr_row, (wm * TM + i) * 32 + tr_col)], BM);
#pragma unroll
                        for (int j = 0; j < TN; ++j) add_product<kParts>(a, b[j], acc[i][j]);
                    }
                }
            }
        }
        const bool only = q.first[t.x + 1] - q.first[t.x] == 1;
        float *out = only ? q.dW + int64_t(t.x) * q.M * q.N : q.partial + run * int64_t(q.M) * q.N;
        // register r of a lane: row 8 (r / 4) + 4 (lane / 32) + r % 4, column lane % 32
        bool odd = false;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int m = m0 + (wm * TM + i) * 32 + 8 * (r / 4) + 4 * hi + r % 4;
                if (m < q.M) {
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        const int n = n0 + (wn * TN + j) * 32 + l31;
                        const float v = kSplit ? acc[i][j][r] * kSplitUnscale : acc[i][j][r];
                        if (n < q.N) {
                            out[int64_t(m) * q.N + n] = v;
                            odd = odd || !(fabsf(v) <= FLT_MAX);
                        }
                    }
                }
            }
        if (kSplit && odd)          // in fp32, from what the operands are
            for (int c = 0; c < TM * TN * 16; ++c) {
                const int r = c % 16, m = m0 + (wm * TM + c / 16 / TN) * 32 + 8 * (r / 4) + 4 * hi + r % 4, n = n0 + (wn * TN + c / 16 % TN) * 32 + l31;
                if (m >= q.M || n >= q.N || fabsf(out[int64_t(m) * q.N + n]) <= FLT_MAX) continue;
                float total = 0.0f;
                for (int at = 0; at < t.z; ++at) {
                    const int64_t v = q.gl.row(t.y + at);
                    if (v < 0 || (kMask && !(widened(H[v * q.ldg + n]) > 0.0f))) continue;
                    total = fmaf(widened(X[v * q.ldx + m]), widened(G[v * q.ldg + n]), total);
                }
                out[int64_t(m) * q.N + n] = total;
            }
        if (sum) {      // (uniform over the block); the threads that share a column, in order
            __syncthreads();
            float *sums = reinterpret_cast<float *>(&Zs[0][0]);       // [kAtOnce][BN]
            static_assert(sizeof(float) * ZS::kAtOnce * BN <= sizeof(Zs), "room for the column sums");
#pragma unroll
            for (int j = 0; j < E; ++j) sums[int(threadIdx.x) / ZS::PP * BN + ZS::column() + j] = col[j];
            __syncthreads();
            float *o = only ? q.db + int64_t(t.x) * q.N : q.colsum + run * q.N;
            for (int c = tid; c < BN; c += kThreads)
                if (n0 + c < q.N) {
                    float total = 0.0f;
                    for (int r = 0; r < ZS::kAtOnce; ++r) total += sums[r * BN + c];
                    o[n0 + c] = total;
                }
        }
    }
}

// dW[g], db[g]: the runs of a group added up in order; zeros for a group without rows (one run is there already)
__global__ __launch_bounds__(kGgThreads) void grouped_join_kernel(const int32_t *__restrict__ first, int64_t cells, int N, const float *__restrict__ partial,
                                                                  const float *__restrict__ colsum, float *__restrict__ dW, float *__restrict__ db)
{
    const int g = blockIdx.y;
    const int64_t a = first[g], b = first[g + 1];
    if (b - a == 1) return;
    auto add_up = [&](const float *from, int64_t width, int64_t i) {
        float s0 = 0.0f;
        int64_t r = a;
        for (; r + 7 < b; r += 8) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = from[(r + u) * width + i];
#pragma unroll
            for (int u = 0; u < 8; ++u) s0 += v[u];
        }
        for (; r < b; ++r) s0 += from[r * width + i];
        return s0;
    };
    for (int64_t i = int64_t(blockIdx.x) * kGgThreads + threadIdx.x; i < cells; i += int64_t(gridDim.x) * kGgThreads) dW[g * cells + i] = add_up(partial, cells, i);
    if (db && blockIdx.x == 0)
        for (int i = threadIdx.x; i < N; i += kGgThreads) db[int64_t(g) * N + i] = add_up(colsum, N, i);
}

// ---- the launch before: plans and weights ------------------------------------------------
struct PrepareCall {
    GroupList gl;
    TilePlan rows, runs;                  // room 0: not wanted
    int row_blocks, run_blocks;           // blocks that write them; the others lay out weights
    const float *W, *bias;                // bias (may be NULL): copied to bias_out [E][col_tiles * 32] with zeros past N
    uint4 *B;
    float *bias_out;
    int K, N, col_tiles, steps, TN;
};

template <typename T, bool kForward>
__global__ __launch_bounds__(kGgThreads) void grouped_prepare_kernel(PrepareCall q)
{
    const int b = blockIdx.x;
    if (q.bias && b < q.gl.E)
        for (int c = threadIdx.x; c < q.col_tiles * 32; c += kGgThreads)
            q.bias_out[int64_t(b) * q.col_tiles * 32 + c] = c < q.N ? q.bias[int64_t(b) * q.N + c] : 0.0f;
    if (b < q.row_blocks) write_plan(q.gl, q.rows, b);
    else if (b < q.row_blocks + q.run_blocks) write_plan(q.gl, q.runs, b - q.row_blocks);
    else write_fragments<T, kForward>(q.gl, q.W, q.K, q.N, q.col_tiles, q.steps, q.TN, q.B, b - q.row_blocks - q.run_blocks,
                                      gridDim.x - q.row_blocks - q.run_blocks);
}

}  // namespace tma
