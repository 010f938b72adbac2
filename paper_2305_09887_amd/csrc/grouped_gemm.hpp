// Tile products of the grouped dense layers (grouped_dense.hip), for groups of many rows.
//
// A plan made on the device, with the weights laid out in the same launch, tells every tile its group: tiles of a group's rows
// follow each other, group after group, and a block takes its tiles from one die's run of them (neighbours share weights and,
// where a row's results are several tiles wide, rows in that die's L2).
//
// grouped_rows_kernel (forward and input gradient): C[v] = A[v] B[g] for 64 listed rows v.  Bound by streaming the rows in and the
// results out (bf16 256 -> 256: 1 KB and 131 kFLOP a row), so: a row's k-values are read once, wherever the row lies, in
// pieces of 16 bytes, all of the next tile's on their way in registers while this one is multiplied; through LDS (512 bytes of a row at a
// time) because the matrix instruction wants a row per lane.  The weights go past LDS: laid out as fragments, 1 KB that a
// wavefront loads at once, and the same for all tiles of a group, they come out of L2.  The instruction multiplies weights by
// rows, so that a lane ends with neighbouring results of one row: which column of W is which row of a fragment is the layout's
// choice, and is made so that a lane stores 16 or 32 neighbours in pieces of 16 bytes.
//
// grouped_weight_kernel (weight gradients): dW[g] += X[v]^T dZ[v] over a run of a group's rows, 128 x 128 results a block; both
// operands come as they lie, rows of LDS, and are read along columns (bf16: the transposing LDS read).  Runs of one group are
// added up in order by a second kernel; a group of one run is stored at once.
//
// fp32: v_mfma_f32_32x32x2_f32, fp32 throughout.  bf16: v_mfma_f32_32x32x16_bf16, weights rounded once to bf16 (as in all products of
// bf16 storage here), fp32 accumulation, results rounded once.
#pragma once
#include "kernels.hpp"

#include <type_traits>

namespace tma {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kDies = 8;             // workgroups are dealt round-robin to them
constexpr int kTileM = 64;           // rows of a tile
constexpr int kGgThreads = 256;
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

// tiles of the groups before each one, in LDS; returns their number.  Blocks of kGgThreads.
__device__ __forceinline__ int tile_prefix(const GroupList &gl, int height, int (&prefix)[kMaxGroups + 1])
{
    __shared__ int wave_sums[kGgThreads / kWave];
    constexpr int kPer = kMaxGroups / kGgThreads;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int count[kPer], total = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int g = int(threadIdx.x) * kPer + j;
        const int64_t rows = g < gl.E ? gl.begin(g + 1) - gl.begin(g) : 0;
        count[j] = rows > 0 ? int((rows + height - 1) / height) : 0;
        total += count[j];
    }
    int incl = total;
    for (int d = 1; d < kWave; d <<= 1) {
        const int t = __shfl_up(incl, d, kWave);
        if (lane >= d) incl += t;
    }
    if (lane == kWave - 1) wave_sums[wave] = incl;
    __syncthreads();
    int at = incl - total, all = 0;
    for (int w = 0; w < kGgThreads / kWave; ++w) {
        if (w < wave) at += wave_sums[w];
        all += wave_sums[w];
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int g = int(threadIdx.x) * kPer + j;
        if (g < gl.E) prefix[g] = at;
        at += count[j];
    }
    if (threadIdx.x == 0) prefix[gl.E] = all;
    __syncthreads();
    return all;
}

__device__ __forceinline__ void write_plan(const GroupList &gl, const TilePlan &p, int block)
{
    __shared__ int prefix[kMaxGroups + 1];
    const int all = tile_prefix(gl, p.height, prefix);
    if (block == 0)
        for (int g = threadIdx.x; g <= gl.E; g += kGgThreads) p.first[g] = prefix[g];
    const int i = block * kGgThreads + threadIdx.x;
    if (i >= all || i >= p.room) return;
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
// A step is 16 bytes of k-values a lane: 16 of bf16, 8 of fp32.  Piece (g, tile of 32 columns, step, lane) holds of column
// col(lane % 32) the k-values step * 2 E + (lane / 32) * E + [0, E).
template <typename T>
struct Step {
    static constexpr int E = 16 / sizeof(T), K = 2 * E;
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
    constexpr int E = Step<T>::E;
    const int64_t per_group = int64_t(tiles) * steps * kWave, total = per_group * gl.E;
    for (int64_t i = block * kGgThreads + threadIdx.x; i < total; i += blocks * kGgThreads) {
        const int g = int(i / per_group);
        if (gl.begin(g + 1) <= gl.begin(g)) continue;
        const int64_t q = i % per_group;
        const int lane = int(q % kWave), step = int(q / kWave % steps), tile = int(q / kWave / steps);
        const int col = fragment_column(tile, lane & 31, TN), k0 = step * Step<T>::K + (lane >> 5) * E;
        const float *w = W + int64_t(g) * K * N;
        float v[E];
#pragma unroll
        for (int j = 0; j < E; ++j) {
            v[j] = 0.0f;
            if (col < N && k0 + j < K) v[j] = kForward ? w[int64_t(k0 + j) * N + col] : w[int64_t(col) * K + k0 + j];
        }
        uint4 piece;
        if constexpr (sizeof(T) == 4) piece = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        else piece = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
        out[i] = piece;
    }
}

// ---- pieces of rows ----------------------------------------------------------------
struct __attribute__((packed, aligned(4))) Words4 {
    uint32_t w[4];
};

__device__ __forceinline__ uint32_t bits1(const float *p) { return __float_as_uint(*p); }
__device__ __forceinline__ uint32_t bits1(const uint16_t *p) { return *p; }

// A piece of 16 bytes from element `at` on of an array, of which the first `valid` elements are wanted and the others read as zero.
// kWords (4-byte aligned, the load needs no more): one load without a branch; a piece that would run past `last`, the last place where
// 16 bytes are left, comes from there and is moved back in registers.  Else element by element.
template <typename T, bool kWords>
struct RowPiece {
    static constexpr int E = 16 / sizeof(T);
    static __device__ __forceinline__ uint4 load(const T *__restrict__ x, int64_t at, int valid, int64_t last)
    {
        if constexpr (kWords) {
            const Words4 w = *reinterpret_cast<const Words4 *>(x + (at < last ? at : last));
            return make_uint4(w.w[0], w.w[1], w.w[2], w.w[3]);
        } else {
            uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (j < valid) w[j * int(sizeof(T)) / 4] |= bits1(x + at + j) << (sizeof(T) == 2 ? 16 * (j & 1) : 0);
            return make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    // back: elements by which the piece was fetched too early
    static __device__ __forceinline__ uint4 moved(const uint4 &p, int back)
    {
        uint64_t lo = uint64_t(p.y) << 32 | p.x, hi = uint64_t(p.w) << 32 | p.z;
        int bits = back * int(sizeof(T)) * 8;
        if (bits >= 64) {
            lo = hi;
            hi = 0;
            bits -= 64;
        }
        if (bits > 0) {
            lo = lo >> bits | hi << (64 - bits);
            hi >>= bits;
        }
        return make_uint4(uint32_t(lo), uint32_t(lo >> 32), uint32_t(hi), uint32_t(hi >> 32));
    }
    static __device__ __forceinline__ uint4 cut(const uint4 &p, int valid)
    {
        uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) w[i] = valid > i ? w[i] : 0u;
            else w[i] &= valid > 2 * i + 1 ? ~0u : valid > 2 * i ? 0xFFFFu : 0u;
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// g where h > 0 (a NaN in h: not), zeros elsewhere
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

// acc[i][j] += a step's products; the fp32 instruction's four in a row go to different accumulators
template <typename T, int TM, int TN>
__device__ __forceinline__ void multiply(const uint4 (&w)[TN], const uint4 (&x)[TM], floatx16 (&acc)[TM][TN])
{
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i)
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w[j]), __builtin_bit_cast(bf16x8, x[i]), acc[i][j], 0, 0, 0);
    } else {
        auto word = [](const uint4 &v, int k) { return __uint_as_float(k == 0 ? v.x : k == 1 ? v.y : k == 2 ? v.z : v.w); };
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int i = 0; i < TM; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(word(w[j], k), word(x[i], k), acc[i][j], 0, 0, 0);
    }
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
    int64_t lda, ldc;
    int K, N, steps, n_tiles;  // n_tiles: of BN columns
    bool relu;
};

// blocks of a compute unit that the registers leave room for (four wavefronts each)
template <int TN, int PP, bool kMask>
constexpr int kRowBlocksPerCu = kMask && TN * PP > 32 ? 2 : 3;

// PP: 16-byte pieces of a row in LDS at a time.  The numbers of a tile's rows are fetched two tiles ahead, its rows one.
template <typename T, int WN, int TN, int PP, bool kMask, bool kWords, bool kStore16>
__global__ __launch_bounds__(kGgThreads, (kRowBlocksPerCu<TN, PP, kMask>)) void grouped_rows_kernel(RowsCall q)
{
    constexpr int WM = 4 / WN, TM = kTileM / WM / 32, E = Step<T>::E;
    constexpr int kRowsAtOnce = kGgThreads / PP, kPieces = kTileM / kRowsAtOnce;    // of a thread
    constexpr int kSteps = PP / 2, kAhead = 4;
    typedef RowPiece<T, kWords> P;
    __shared__ uint4 As[kTileM * PP];
    __shared__ int32_t rows[2][kTileM];        // of this tile and the next, -1: none
    const T *A = static_cast<const T *>(q.A), *H = static_cast<const T *>(q.H);
    const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, hi = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int piece = tid % PP, row0 = tid / PP;
    const int64_t last = (q.gl.n - 1) * q.lda + q.K - E;
    // pieces of a row exchanged by its number, so that the 16 rows that are read at once lie in all banks
    constexpr int kSpread = PP < 16 ? PP : 16;
    auto place = [](int row, int p) { return row * PP + (p ^ ((row / (16 / kSpread)) & (kSpread - 1))); };

    Share share(int64_t(*q.tile_count) * q.n_tiles);
    if (share.item >= share.end) return;
    const int chunks = (q.steps + kSteps - 1) / kSteps;
    const bool ragged = kWords && q.K % E != 0;

    auto row_of = [&](int64_t item) {          // of thread tid < 64
        const int4 t = q.tiles[item / q.n_tiles];
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
        const int group = q.tiles[item / q.n_tiles].x;
        const int nt = int(item % q.n_tiles) * WN * TN + wn * TN;      // first of the wavefront's column tiles
        const int n0 = nt * 32 + hi * TN * 16;                         // first of the lane's columns
        const uint4 *B = q.B + (int64_t(group) * q.n_tiles * WN * TN + nt) * q.steps * kWave;
        auto weights = [&](int j, int step) { return B[uint32_t((j * q.steps + step) * kWave + lane)]; };
        floatx16 acc[TM][TN];
        if (q.bias) {
            const float4 *b4 = reinterpret_cast<const float4 *>(q.bias + int64_t(group) * q.n_tiles * (WN * TN * 32) + n0);
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
            const int s0 = c * kSteps, s1 = q.steps - s0 < kSteps ? q.steps - s0 : kSteps;
            uint4 b[kAhead][TN];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int j = 0; j < TN; ++j) b[u][j] = weights(j, s0 + (u < s1 ? u : s1 - 1));
            __syncthreads();           // everyone has read what was there
            const int valid = q.K - (c * PP + piece) * E;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                uint4 p = held[i];
                if constexpr (kMask) p = open_piece<T>(p, mask[i]);
                if (ragged) {
                    const int64_t over = element(at, i, c) - last;
                    if (over > 0) p = P::moved(p, int(over));
                    p = P::cut(p, valid);
                } else if (valid <= 0) p = make_uint4(0u, 0u, 0u, 0u);
                As[place(row0 + i * kRowsAtOnce, piece)] = p;
            }
            if (c == 0 && tid < kTileM) rows[at ^ 1][tid] = pending;
            __syncthreads();
            if (c + 1 < chunks) fetch(at, c + 1);
            else if (more) {
                fetch(at ^ 1, 0);
                pending = -1;
                if (tid < kTileM && next + share.stride < share.end) pending = row_of(next + share.stride);
            }
            for (int s = 0; s < s1; s += kAhead) {
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    if (s + u >= s1) break;
                    uint4 a[TM];
#pragma unroll
                    for (int i = 0; i < TM; ++i) a[i] = As[place((wm * TM + i) * 32 + l31, 2 * (s + u) + hi)];
                    multiply<T, TM, TN>(b[u], a, acc);
                    const int ahead = s + u + kAhead < s1 ? s + u + kAhead : s1 - 1;
#pragma unroll
                    for (int j = 0; j < TN; ++j) b[u][j] = weights(j, s0 + ahead);
                }
            }
        }
        // lane: row l31 of the tile's 32, columns n0 + [0, 16 TN)
        T *C = static_cast<T *>(q.C);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t v = rows[at][(wm * TM + i) * 32 + l31];
            if (v < 0) continue;
            T *out = C + v * q.ldc + n0;
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                float z[16];
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    z[r] = acc[i][j][r];
                    if (q.relu) z[r] = z[r] > 0.0f ? z[r] : 0.0f;
                }
                if (kStore16 && n0 + j * 16 + 16 <= q.N) {
#pragma unroll
                    for (int r = 0; r < 16; r += E) {
                        float w[E];
#pragma unroll
                        for (int x = 0; x < E; ++x) w[x] = z[r + x];
                        Chunk<T>::store(out + j * 16 + r, w);
                    }
                } else {
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (n0 + j * 16 + r < q.N) {
                            if constexpr (sizeof(T) == 4) out[j * 16 + r] = z[r];
                            else out[j * 16 + r] = f32_to_bf16(z[r]);
                        }
                }
            }
        }
        if (!more) return;
        share.item = next;
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
    // bf16: blocks of 32 columns exchanged by the row's number, for the transposing read takes 4 rows x 16 columns at once
    static __device__ __forceinline__ int place(int row, int c) { return row * COLS + (sizeof(T) == 2 ? ((c >> 5) ^ (row & 3)) * 32 + (c & 31) : c); }
    static __device__ __forceinline__ int row(int i) { return int(threadIdx.x) / PP + i * kAtOnce; }
    static __device__ __forceinline__ int column() { return int(threadIdx.x) % PP * E; }
};

// A block's tile is (WM TM 32) x (WN TN 32); kDepth slabs of rows are in flight in registers, two in LDS (one barrier a slab).
template <typename T, int WM, int WN, int TM, int TN, bool kMask, bool kWords>
__global__ __launch_bounds__(WM *WN * 64, 2) void grouped_weight_kernel(WeightCall q)
{
    constexpr int kThreads = WM * WN * 64, BM = WM * TM * 32, BN = WN * TN * 32, kDepth = 2;
    constexpr int E = Step<T>::E, kSlab = sizeof(T) == 2 ? 32 : 16;
    constexpr int kListed = 64 * kSlab;                    // rows whose numbers lie in LDS, twice: these and the ones to come
    typedef SlabPieces<T, kSlab, BM, kThreads, kWords> XS;
    typedef SlabPieces<T, kSlab, BN, kThreads, kWords> ZS;
    typedef RowPiece<T, kWords> P;
    __shared__ __attribute__((aligned(16))) T Xs[2][kSlab * BM];
    __shared__ __attribute__((aligned(16))) T Zs[2][kSlab * BN];
    __shared__ int32_t listed[2][kListed];
    const T *X = static_cast<const T *>(q.X), *G = static_cast<const T *>(q.G), *H = static_cast<const T *>(q.H);
    const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, hi = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int64_t x_last = (q.gl.n - 1) * q.ldx + q.M - E, g_last = (q.gl.n - 1) * q.ldg + q.N - E;
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
                T *x = Xs[s & 1], *z = Zs[s & 1];
#pragma unroll
                for (int i = 0; i < XS::kPieces; ++i) {
                    const int v = row(s, XS::row(i));
                    uint4 p = xh[d][i];
                    if (x_ragged && v >= 0) {
                        const int64_t over = int64_t(v) * q.ldx + (xv > 0 ? xc : 0) - x_last;
                        if (over > 0) p = P::moved(p, int(over));
                    }
                    if (v < 0) p = make_uint4(0u, 0u, 0u, 0u);
                    *reinterpret_cast<uint4 *>(&x[XS::place(XS::row(i), XS::column())]) = p;
                }
#pragma unroll
                for (int i = 0; i < ZS::kPieces; ++i) {
                    const int v = row(s, ZS::row(i));
                    uint4 p = zh[d][i];
                    if constexpr (kMask) p = open_piece<T>(p, hh[d][i]);
                    if (z_ragged && v >= 0) {
                        const int64_t over = int64_t(v) * q.ldg + (zv > 0 ? zc : 0) - g_last;
                        if (over > 0) p = P::moved(p, int(over));
                    }
                    if (v < 0) p = make_uint4(0u, 0u, 0u, 0u);
                    *reinterpret_cast<uint4 *>(&z[ZS::place(ZS::row(i), ZS::column())]) = p;
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
                if constexpr (sizeof(T) == 2) {
#pragma unroll
                    for (int k = 0; k < kSlab; k += 16) {
                        uint4 a[TM], b[TN];
#pragma unroll
                        for (int i = 0; i < TM; ++i) a[i] = along_rows(&x[XS::place(k + tr_row, (wm * TM + i) * 32 + tr_col)], BM);
#pragma unroll
                        for (int j = 0; j < TN; ++j) b[j] = along_rows(&z[ZS::place(k + tr_row, (wn * TN + j) * 32 + tr_col)], BN);
#pragma unroll
                        for (int i = 0; i < TM; ++i)
#pragma unroll
                            for (int j = 0; j < TN; ++j)
                                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[i]), __builtin_bit_cast(bf16x8, b[j]), acc[i][j], 0, 0, 0);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < kSlab; k += 2) {
                        float a[TM], b[TN];
#pragma unroll
                        for (int i = 0; i < TM; ++i) a[i] = x[(k + hi) * BM + (wm * TM + i) * 32 + l31];
#pragma unroll
                        for (int j = 0; j < TN; ++j) b[j] = z[(k + hi) * BN + (wn * TN + j) * 32 + l31];
#pragma unroll
                        for (int i = 0; i < TM; ++i)
#pragma unroll
                            for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[j], acc[i][j], 0, 0, 0);
                    }
                }
            }
        }
        const bool only = q.first[t.x + 1] - q.first[t.x] == 1;
        float *out = only ? q.dW + int64_t(t.x) * q.M * q.N : q.partial + run * int64_t(q.M) * q.N;
        // register r of a lane: row 8 (r / 4) + 4 (lane / 32) + r % 4, column lane % 32
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int m = m0 + (wm * TM + i) * 32 + 8 * (r / 4) + 4 * hi + r % 4;
                if (m < q.M) {
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        const int n = n0 + (wn * TN + j) * 32 + l31;
                        if (n < q.N) out[int64_t(m) * q.N + n] = acc[i][j][r];
                    }
                }
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
