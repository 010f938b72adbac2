// Dense layers of rows that are of several kinds: group g of the listed rows has weights of its own,
//   forward   Y[v] = act(X[v] W[g] + b[g])
//   backward  dZ = dY (.) act'(Y);  dX[v] = dZ[v] W[g]^T;  dW[g] = sum over g's rows of X[v]^T dZ[v];  db[g] = sum of dZ[v]
// Group g has the positions [offsets[g], offsets[g+1]) of the list; position i is row order[i] of X, Y and their gradients
// (order NULL: row i).  Sizes of groups are known to the device alone.
//
// Here: the entry points, and the kernels for groups of few rows, which the weights bound: they are read once as they are, in
// fp32, every multiplication and sum is fp32.  Grids go over (group, slice of 32 columns), so that small layers still have
// some hundred blocks; rows of a group go through LDS eight at a time, beside a thread's weights of a chunk in registers.  24 rows of 16 groups, 256 ->
// 256, 7.9 us: one memory latency for positions, one for rows, one for weights (4.2 MB) and the launch.
#include "grouped_gemm.hpp"

namespace tma {

constexpr int kFewThreads = 256;
constexpr int kFewCols = 32;      // columns of a block's slice: eight lanes with four each
constexpr int kSideRows = 8;       // rows of a group side by side in registers
constexpr int kFewK = 512;        // of the summed dimension in LDS at a time

__device__ __forceinline__ float read1(const float *p) { return *p; }
__device__ __forceinline__ float read1(const uint16_t *p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void write1(float *p, float v) { *p = v; }
__device__ __forceinline__ void write1(uint16_t *p, float v) { *p = f32_to_bf16(v); }

// four elements from p on, `left` of them inside (any alignment unless vec)
__device__ __forceinline__ float4 weights4(const float *p, int left, bool vec)
{
    if (vec) return left > 0 ? *reinterpret_cast<const float4 *>(p) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    return make_float4(left > 0 ? p[0] : 0.0f, left > 1 ? p[1] : 0.0f, left > 2 ? p[2] : 0.0f, left > 3 ? p[3] : 0.0f);
}

// rows[r][k - k0] of the chunk's rows at columns [k0, k0 + kFewK), zeros outside; g where h > 0 with h given
template <typename T>
__device__ __forceinline__ void stage_rows(const GroupList &gl, int64_t i0, int m, const T *g, const T *h, int64_t ld, int k0, int K,
                                           float (&rows)[kSideRows][kFewK + 4])
{
    int64_t v[kSideRows];
#pragma unroll
    for (int r = 0; r < kSideRows; ++r) v[r] = r < m ? gl.row(i0 + r) : -1;
    constexpr int kEach = kFewK / kFewThreads;
    float x[kSideRows][kEach];
#pragma unroll
    for (int r = 0; r < kSideRows; ++r)
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int k = k0 + j * kFewThreads + int(threadIdx.x);
            const bool in = v[r] >= 0 && k < K;
            const int64_t at = in ? v[r] * ld + k : 0;
            x[r][j] = in ? read1(g + at) : 0.0f;
            if (h && !(in && read1(h + at) > 0.0f)) x[r][j] = 0.0f;
        }
#pragma unroll
    for (int r = 0; r < kSideRows; ++r)
#pragma unroll
        for (int j = 0; j < kEach; ++j) rows[r][j * kFewThreads + int(threadIdx.x)] = x[r][j];
}

constexpr int kFewW = kFewK / 32;      // pieces of weights of a thread in registers: all of its k-values of a chunk, on their way while rows are staged

// Y[v][c] for the block's group and 32 columns.  Eight lanes share the columns, 32 of them the k-values.
template <typename T>
__global__ __launch_bounds__(kFewThreads) void grouped_few_fwd_kernel(GroupList gl, const T *__restrict__ X, int64_t ldx, int K, const float *__restrict__ W,
                                                                      const float *__restrict__ bias, int N, bool relu, bool vec, T *__restrict__ Y,
                                                                      int64_t ldy, int slices)
{
    __shared__ float rows[kSideRows][kFewK + 4];
    __shared__ __attribute__((aligned(16))) float sums[kFewThreads / kWave][kSideRows][kFewCols];
    const int g = int(blockIdx.x) / slices, n0 = int(blockIdx.x) % slices * kFewCols;
    const int64_t begin = gl.begin(g), end = gl.begin(g + 1);
    const int q = int(threadIdx.x) % 8, ks = int(threadIdx.x) / 8, wave = int(threadIdx.x) / kWave, lane = int(threadIdx.x) % kWave;
    const int left = N - n0 - 4 * q;
    const float *Wg = W + int64_t(g) * K * N + n0 + 4 * q;
    float4 w[kFewW];
    for (int64_t i0 = begin; i0 < end; i0 += kSideRows) {
        const int m = end - i0 < kSideRows ? int(end - i0) : kSideRows;
        float4 acc[kSideRows];
#pragma unroll
        for (int r = 0; r < kSideRows; ++r) acc[r] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int k0 = 0; k0 < K; k0 += kFewK) {
            if (K > kFewK || i0 == begin) {        // (of a single chunk they stay)
#pragma unroll
                for (int j = 0; j < kFewW; ++j) {
                    const int k = k0 + j * 32 + ks;
                    w[j] = weights4(Wg + int64_t(k < K ? k : 0) * N, k < K ? left : 0, vec);
                }
            }
            __syncthreads();
            stage_rows<T>(gl, i0, m, X, nullptr, ldx, k0, K, rows);
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kFewW; ++j) {
                if (k0 + j * 32 >= K) break;
#pragma unroll
                for (int r = 0; r < kSideRows; ++r) {
                    const float x = rows[r][j * 32 + ks];
                    acc[r].x = fmaf(x, w[j].x, acc[r].x);
                    acc[r].y = fmaf(x, w[j].y, acc[r].y);
                    acc[r].z = fmaf(x, w[j].z, acc[r].z);
                    acc[r].w = fmaf(x, w[j].w, acc[r].w);
                }
            }
        }
#pragma unroll
        for (int r = 0; r < kSideRows; ++r) {
#pragma unroll
            for (int d = 8; d < kWave; d *= 2) {
                acc[r].x += __shfl_xor(acc[r].x, d, kWave);
                acc[r].y += __shfl_xor(acc[r].y, d, kWave);
                acc[r].z += __shfl_xor(acc[r].z, d, kWave);
                acc[r].w += __shfl_xor(acc[r].w, d, kWave);
            }
            if (lane < 8) *reinterpret_cast<float4 *>(&sums[wave][r][4 * q]) = acc[r];
        }
        __syncthreads();
        const int r = int(threadIdx.x) / kFewCols, c = int(threadIdx.x) % kFewCols;
        if (r < m && n0 + c < N) {
            float z = (sums[0][r][c] + sums[1][r][c]) + (sums[2][r][c] + sums[3][r][c]);
            if (bias) z += bias[int64_t(g) * N + n0 + c];
            if (relu) z = z > 0.0f ? z : 0.0f;
            const int64_t v = gl.row(i0 + r);
            if (v >= 0) write1(Y + v * ldy + n0 + c, z);
        }
    }
}

// dX[v][i] for the block's group and 32 columns i: eight lanes share a row of W.
template <typename T>
__global__ __launch_bounds__(kFewThreads) void grouped_few_bwd_data_kernel(GroupList gl, const T *__restrict__ dY, const T *__restrict__ Yh, int64_t ldy, int K,
                                                                           const float *__restrict__ W, int N, bool vec, T *__restrict__ dX, int64_t ldx,
                                                                           int slices)
{
    __shared__ __attribute__((aligned(16))) float rows[kSideRows][kFewK + 4];
    const int g = int(blockIdx.x) / slices, i = int(blockIdx.x) % slices * kFewCols + int(threadIdx.x) / 8, q = int(threadIdx.x) % 8;
    const int64_t begin = gl.begin(g), end = gl.begin(g + 1);
    const float *Wi = W + (int64_t(g) * N + (i < N ? i : 0)) * K;
    float4 w[kFewW];
    for (int64_t i0 = begin; i0 < end; i0 += kSideRows) {
        const int m = end - i0 < kSideRows ? int(end - i0) : kSideRows;
        float acc[kSideRows];
#pragma unroll
        for (int r = 0; r < kSideRows; ++r) acc[r] = 0.0f;
        for (int k0 = 0; k0 < K; k0 += kFewK) {
            if (K > kFewK || i0 == begin) {
#pragma unroll
                for (int j = 0; j < kFewW; ++j) {
                    const int k = k0 + j * 32 + 4 * q;
                    w[j] = weights4(Wi + (k < K ? k : 0), K - k, vec);
                }
            }
            __syncthreads();
            stage_rows<T>(gl, i0, m, dY, Yh, ldy, k0, K, rows);
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kFewW; ++j) {
                if (k0 + j * 32 >= K) break;
#pragma unroll
                for (int r = 0; r < kSideRows; ++r) {
                    const float4 x = *reinterpret_cast<const float4 *>(&rows[r][j * 32 + 4 * q]);
                    acc[r] = fmaf(x.x, w[j].x, fmaf(x.y, w[j].y, fmaf(x.z, w[j].z, fmaf(x.w, w[j].w, acc[r]))));
                }
            }
        }
#pragma unroll
        for (int r = 0; r < kSideRows; ++r) {
#pragma unroll
            for (int d = 1; d < 8; d *= 2) acc[r] += __shfl_xor(acc[r], d, kWave);
            const int64_t v = r < m ? gl.row(i0 + r) : -1;
            if (q == 0 && i < N && v >= 0) write1(dX + v * ldx + i, acc[r]);
        }
    }
}

// dW[g][i][o] for the block's group, 32 rows i and all o (128 at a time); db with the first slice.
constexpr int kFewO = 128;

template <typename T>
__global__ __launch_bounds__(kFewThreads) void grouped_few_bwd_weight_kernel(GroupList gl, const T *__restrict__ X, int64_t ldx, const T *__restrict__ dY,
                                                                             const T *__restrict__ Yh, int64_t ldy, int M, int N, float *__restrict__ dW,
                                                                             float *__restrict__ db, int slices)
{
    __shared__ float xs[kSideRows][kFewCols];
    __shared__ __attribute__((aligned(16))) float zs[kSideRows][kFewO];
    const int g = int(blockIdx.x) / slices, m0 = int(blockIdx.x) % slices * kFewCols, il = int(threadIdx.x) / 8, q = int(threadIdx.x) % 8;
    const int64_t begin = gl.begin(g), end = gl.begin(g + 1);
    for (int o0 = 0; o0 < N; o0 += kFewO) {
        float acc[kFewO / 32][4], sum = 0.0f;
        for (int j = 0; j < kFewO / 32; ++j)
            for (int c = 0; c < 4; ++c) acc[j][c] = 0.0f;
        for (int64_t i0 = begin; i0 < end; i0 += kSideRows) {
            const int m = end - i0 < kSideRows ? int(end - i0) : kSideRows;
            __syncthreads();
            {
                const int r = int(threadIdx.x) / kFewCols, c = int(threadIdx.x) % kFewCols;
                const int64_t v = r < m ? gl.row(i0 + r) : -1;
                xs[r][c] = v >= 0 && m0 + c < M ? read1(X + v * ldx + m0 + c) : 0.0f;
            }
            for (int at = threadIdx.x; at < kSideRows * kFewO; at += kFewThreads) {
                const int r = at / kFewO, o = o0 + at % kFewO;
                const int64_t v = r < m ? gl.row(i0 + r) : -1;
                float z = 0.0f;
                if (v >= 0 && o < N) {
                    z = read1(dY + v * ldy + o);
                    if (Yh && !(read1(Yh + v * ldy + o) > 0.0f)) z = 0.0f;
                }
                zs[r][at % kFewO] = z;
            }
            __syncthreads();
#pragma unroll
            for (int r = 0; r < kSideRows; ++r) {
                const float x = xs[r][il];
#pragma unroll
                for (int j = 0; j < kFewO / 32; ++j) {
                    const float4 z = *reinterpret_cast<const float4 *>(&zs[r][j * 32 + 4 * q]);
                    acc[j][0] = fmaf(x, z.x, acc[j][0]);
                    acc[j][1] = fmaf(x, z.y, acc[j][1]);
                    acc[j][2] = fmaf(x, z.z, acc[j][2]);
                    acc[j][3] = fmaf(x, z.w, acc[j][3]);
                }
                if (threadIdx.x < kFewO) sum += zs[r][threadIdx.x];
            }
        }
        if (m0 + il < M) {
            float *out = dW + (int64_t(g) * M + m0 + il) * N + o0;
#pragma unroll
            for (int j = 0; j < kFewO / 32; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (o0 + j * 32 + 4 * q + c < N) out[j * 32 + 4 * q + c] = acc[j][c];
        }
        if (db && m0 == 0 && int(threadIdx.x) < kFewO && o0 + int(threadIdx.x) < N) db[int64_t(g) * N + o0 + threadIdx.x] = sum;
    }
}

template <typename T>
static int few_fwd(const char *fn, const GroupList &gl, const void *X, int64_t ldx, int K, const float *W, const float *bias, int N, bool relu, void *Y,
                   int64_t ldy, hipStream_t s)
{
    const int slices = int(ceil_div(N, kFewCols));
    TMA_TIMED(sizeof(T) == 2 ? "grouped_few_fwd_bf16" : "grouped_few_fwd", s);
    hipLaunchKernelGGL((grouped_few_fwd_kernel<T>), dim3(unsigned(gl.E) * unsigned(slices)), dim3(kFewThreads), 0, s, gl, static_cast<const T *>(X), ldx, K, W,
                       bias, N, relu, N % 4 == 0 && aligned(W, 16), static_cast<T *>(Y), ldy, slices);
    return check_launch(fn);
}

template <typename T>
static int few_bwd(const char *fn, const GroupList &gl, const void *X, int64_t ldx, const void *Y, const void *dY, int64_t ldy, const float *W, int F_in,
                   int F_out, bool relu, float *dW, float *db, void *dX, int64_t ld_dx, hipStream_t s)
{
    const T *g = static_cast<const T *>(dY), *h = relu ? static_cast<const T *>(Y) : nullptr;
    const int slices = int(ceil_div(F_in, kFewCols));
    const dim3 grid(unsigned(gl.E) * unsigned(slices));
    if (dX) {
        TMA_TIMED(sizeof(T) == 2 ? "grouped_few_bwd_data_bf16" : "grouped_few_bwd_data", s);
        hipLaunchKernelGGL((grouped_few_bwd_data_kernel<T>), grid, dim3(kFewThreads), 0, s, gl, g, h, ldy, F_out, W, F_in, F_out % 4 == 0 && aligned(W, 16),
                           static_cast<T *>(dX), ld_dx, slices);
        if (int rc = check_launch(fn)) return rc;
    }
    TMA_TIMED(sizeof(T) == 2 ? "grouped_few_bwd_weight_bf16" : "grouped_few_bwd_weight", s);
    hipLaunchKernelGGL((grouped_few_bwd_weight_kernel<T>), grid, dim3(kFewThreads), 0, s, gl, static_cast<const T *>(X), ldx, g, h, ldy, F_in, F_out, dW, db,
                       slices);
    return check_launch(fn);
}

// ---- tiles ---------------------------------------------------------------------
// Few rows: the vector kernels, which read the weights once as they are; else tiles, which first lay them out.  Forward + backward in a graph, us,
// few rows and tiles.  fp32, 6 rows a group: 16 groups of 256 -> 256 12 + 27 and 23 + 42, 256 of 128 -> 64 15.5 + 31 and 15.4 + 31.5, 16 of 64 -> 64
// 10 + 18.5 and 10 + 19, 16 of 128 -> 512 11 + 41 and 18 + 37.5; 8 rows: 16 + 34 and 23 + 42, 19 + 40 and 15 + 31.5, 13 + 23.5 and 10 + 20, 14 + 52 and
// 18 + 39.  bf16, 2 rows: 8 + 18 and 11 + 24, 11 + 23 and 9 + 24, 7 + 12 and 8 + 17; 3 rows: 12 + 25 and 11 + 24, 12 + 24 and 9 + 23.5, 10 + 17 and 8 + 17.
// That is for groups alike.  The host knows the mean alone, and rows that are nearly all of one group are a few blocks' work: 384 rows of 64 groups in fp32, 256 ->
// 256, 9 + 21 where groups are alike and 174 + 399 where all are of one, which tiles do in 21 + 53; 6,000 of 1,024 groups 107 + 241 and 2,756 + 8,507.
static bool few_rows_a_group(int64_t n, int E, int32_t dtype) { return n <= (dtype == TMA_BF16 ? 2 : 6) * int64_t(E); }

struct TileShape {
    bool resident;         // weights in LDS, tiles of 32 rows; else tiles of 64 rows that fetch them
    int TN, BN;            // column tiles of 32 whose columns are shuffled together, columns of a part of the result
    int steps, n_tiles, height;      // steps of 16 k-values, parts of the result, rows of a tile
    size_t fragment_bytes, bias_bytes;
};

// Product of rows of K with N columns.  Weights stay in LDS where every compute unit has some rounds of eight wavefronts' rows to take them through (its
// load and the last round's empty places are shared by those); fewer go in tiles, us resident and in tiles: fp32 128 -> 128 125,000 rows 56 and
// 49, 400,000 rows 130 and 152; 64 -> 64 250,000 rows 40 and 45; bf16 256 -> 256 60,000 rows 32 and 25, 250,000 rows 71 and 70, 500,000 rows 136 and 163.
// In tiles at any size: masked rows of several chunks, for beside all sums the registers do not hold the pieces of rows and masks that the loads need
// to overlap (300,000 rows of 384 -> 384 in bf16 with its weight gradient 684 resident, 597 in tiles), and fp32 rows of several chunks, whose
// parts fit LDS for 64 columns only (125,000 rows of 256 -> 128 89 resident, 69 in tiles; bf16, 300,000 rows of 384 -> 384 without a mask, 174 and 215).
constexpr int64_t kResRounds = 3;
static TileShape tile_shape(int64_t n, int E, int K, int N, size_t elem, bool masked)
{
    TileShape t;
    // steps of 16 k-values, filled up to a quarter of a chunk; column tiles that fit LDS beside each other, pairs of them
    const int parts = elem == 4 ? 3 : 1, chunk = elem == 4 ? 8 : 16;
    t.steps = int(round_up(size_t(ceil_div(K, 16)), chunk / 4));
    int cols = kResPieces / (t.steps * parts * kWave) / 2 * 2;
    const bool multi = t.steps > chunk;
    const int most = multi ? kResChunkCols : 8;
    if (cols > most) cols = most;
    const int want = int(ceil_div(N, 64)) * 2, parts_of_N = cols >= 2 ? int(ceil_div(want, cols)) : 0;
    t.resident = cols >= 2 && !(multi && (masked || elem == 4)) && n * parts_of_N >= kResRounds * 256 * kResWaves * kResRows;
    if (t.resident) {
        t.n_tiles = parts_of_N;
        const int each = int(ceil_div(want, 2 * t.n_tiles)) * 2;       // parts alike
        t.BN = each * 32;
        t.TN = elem == 2 ? 2 : 1;
        t.height = kResRows;
        t.fragment_bytes = round_up(size_t(E) * size_t(t.n_tiles) * size_t(t.BN / 32) * size_t(t.steps) * size_t(parts) * 1024, 256);
    } else {
        t.steps = int(round_up(size_t(ceil_div(K, 16)), kStepsUp));
        t.TN = N > 128 ? 2 : 1;
        t.BN = N > 128 ? 256 : N > 64 ? 128 : 64;
        t.n_tiles = int(ceil_div(N, t.BN));
        t.height = kTileM;
        t.fragment_bytes = round_up(size_t(E) * size_t(t.n_tiles) * size_t(t.BN / 32) * size_t(t.steps) * size_t(parts) * 1024, 256);
    }
    t.bias_bytes = round_up(size_t(E) * size_t(t.n_tiles) * size_t(t.BN) * 4, 256);
    return t;
}

static int64_t tile_room(int64_t n, int E, int height) { return ceil_div(n, height) + E; }
static size_t plan_bytes(int64_t n, int E, int height) { return round_up(size_t(tile_room(n, E, height)) * 16, 256) + round_up(size_t(E + 1) * 4, 256); }

static TilePlan plan_at(char *&at, int64_t n, int E, int height)
{
    TilePlan p;
    p.height = height;
    p.room = tile_room(n, E, height);
    p.tiles = reinterpret_cast<int4 *>(at);
    p.first = reinterpret_cast<int32_t *>(at + round_up(size_t(p.room) * 16, 256));
    at += plan_bytes(n, E, height);
    return p;
}

// Tiles of the weight gradient: as wide as the result up to 256 x 256, so that rows are read once.  Runs: as many as the chip holds at
// once with all their tiles, or a few rounds of it; E fewer, since each group's last run may be short (a run more than a round's costs a round).
struct WeightShape {
    int BM, BN, m_tiles, n_tiles, per_cu, height;
};
static WeightShape weight_shape(int64_t n, int E, int M, int N)
{
    WeightShape w;
    w.BM = M > 128 ? 256 : 128;
    w.BN = N > 128 ? 256 : 128;
    w.m_tiles = int(ceil_div(M, w.BM));
    w.n_tiles = int(ceil_div(N, w.BN));
    w.per_cu = w.BM * w.BN > 128 * 128 ? 1 : 2;
    const int64_t slots = 256 * w.per_cu, tiles = int64_t(w.m_tiles) * w.n_tiles;
    int64_t round = ceil_div(slots, tiles), runs = round - E;
    while (runs < (round + 1) / 2) runs += round;
    const int64_t rows = int64_t(round_up(size_t(ceil_div(n > 0 ? n : 1, runs)), 32));
    w.height = int(rows < 64 ? 64 : rows < (1 << 30) ? rows : 1 << 30);
    return w;
}

template <typename T>
static void launch_prepare(const PrepareCall &q, bool forward, hipStream_t s)
{
    const int64_t pieces = q.B ? int64_t(q.gl.E) * q.col_tiles * q.steps * kWave : 0;
    int64_t blocks = ceil_div(pieces, kGgThreads);
    if (blocks > 4096) blocks = 4096;
    int64_t all = q.row_blocks + q.run_blocks + blocks;
    if (q.bias && all < q.gl.E) all = q.gl.E;
    const dim3 grid{unsigned(all)};
    TMA_TIMED(sizeof(T) == 2 ? "grouped_prepare_bf16" : "grouped_prepare", s);
    if (forward) hipLaunchKernelGGL((grouped_prepare_kernel<T, true>), grid, dim3(kGgThreads), 0, s, q);
    else hipLaunchKernelGGL((grouped_prepare_kernel<T, false>), grid, dim3(kGgThreads), 0, s, q);
}

template <typename T, int WN, int TN, bool kMask>
static void launch_rows_as(const RowsCall &q, bool words, bool store16, int64_t most_items, hipStream_t s)
{
    constexpr int kPerCu = kRowBlocksPerCu<TN>;
    int64_t per_die = ceil_div(most_items, kDies);
    if (per_die > 32 * kPerCu) per_die = 32 * kPerCu;
    const dim3 grid(unsigned(per_die * kDies));
    if (words && store16) hipLaunchKernelGGL((grouped_rows_kernel<T, WN, TN, kMask, true, true>), grid, dim3(kGgThreads), 0, s, q);
    else hipLaunchKernelGGL((grouped_rows_kernel<T, WN, TN, kMask, false, false>), grid, dim3(kGgThreads), 0, s, q);
}

// rows whose pieces of 16 bytes one load fetches: words throughout, and such a piece in the array
template <typename T>
static bool rows_in_words(const void *p, int64_t ld, int64_t n, int F)
{
    return (sizeof(T) == 4 || (aligned(p, 4) && ld % 2 == 0)) && RowPiece<T, true>::last_place(n, ld, F) >= 0;
}

template <typename T, bool kMask>
static int launch_rows(const char *fn, const char *name, const RowsCall &q, const TileShape &t, hipStream_t s)
{
    const T *A = static_cast<const T *>(q.A), *H = static_cast<const T *>(q.H);
    const bool words = rows_in_words<T>(A, q.lda, q.gl.n, q.K) && (!kMask || aligned(H, 4));
    const bool store16 = sizeof(T) == 4 || (aligned(q.C, 4) && q.ldc % 2 == 0);      // (the store needs words, no more)
    TMA_TIMED(name, s);
    if (t.resident) {
        const ResidentCall r{q.gl, q.tiles, q.tile_count - q.gl.E, q.B, q.bias, q.A, q.H, q.C, q.W, q.lda, q.ldc, q.w_k, q.w_col, q.K, q.N, q.steps,
                             q.n_tiles, t.BN / 32, q.relu};
        const dim3 grid(256), block(kResWaves * 64);      // one block a compute unit: its weights take the LDS
        auto go = [&](auto nt, auto multi) {
            constexpr int NT = decltype(nt)::value;
            constexpr bool kMulti = decltype(multi)::value;
            if (words && store16) hipLaunchKernelGGL((grouped_resident_kernel<T, NT, kMulti, kMask, true, true>), grid, block, 0, s, r);
            else hipLaunchKernelGGL((grouped_resident_kernel<T, NT, kMulti, kMask, false, false>), grid, block, 0, s, r);
        };
        const std::integral_constant<int, 2> two;
        const std::integral_constant<int, 4> four;
        if (t.steps <= ResStep<T>::kChunk) go(two, std::false_type{});
        else if constexpr (!kMask && sizeof(T) == 2) {
            if (t.BN == 128) go(four, std::true_type{});
            else go(two, std::true_type{});
        }
        return check_launch(fn);
    }
    const int64_t items = tile_room(q.gl.n, q.gl.E, kTileM) * q.n_tiles;
    if (t.BN == 256) launch_rows_as<T, 4, 2, kMask>(q, words, store16, items, s);
    else if (t.BN == 128) launch_rows_as<T, 4, 1, kMask>(q, words, store16, items, s);
    else launch_rows_as<T, 2, 1, kMask>(q, words, store16, items, s);
    return check_launch(fn);
}

template <typename T>
static void launch_weight(const WeightCall &q, const WeightShape &w, bool relu, bool words, int64_t runs, hipStream_t s)
{
    int64_t per_die = ceil_div(runs * w.m_tiles * w.n_tiles, kDies);
    if (per_die > 32 * w.per_cu) per_die = 32 * w.per_cu;
    const dim3 grid(unsigned(per_die * kDies));
    auto go = [&](auto wm, auto wn, auto tm, auto tn) {
        constexpr int WM = decltype(wm)::value, WN = decltype(wn)::value, TM = decltype(tm)::value, TN = decltype(tn)::value;
        const dim3 block(WM * WN * 64);
        if (relu && words) hipLaunchKernelGGL((grouped_weight_kernel<T, WM, WN, TM, TN, true, true>), grid, block, 0, s, q);
        else if (relu) hipLaunchKernelGGL((grouped_weight_kernel<T, WM, WN, TM, TN, true, false>), grid, block, 0, s, q);
        else if (words) hipLaunchKernelGGL((grouped_weight_kernel<T, WM, WN, TM, TN, false, true>), grid, block, 0, s, q);
        else hipLaunchKernelGGL((grouped_weight_kernel<T, WM, WN, TM, TN, false, false>), grid, block, 0, s, q);
    };
    const std::integral_constant<int, 2> two;
    const std::integral_constant<int, 4> four;
    if (w.BM == 256 && w.BN == 256) go(two, four, four, two);
    else if (w.BM == 256) go(four, two, two, two);
    else if (w.BN == 256) go(two, four, two, two);
    else go(two, two, two, two);
}

template <typename T>
static int tiles_fwd(const char *fn, const GroupList &gl, const void *X, int64_t ldx, int K, const float *W, const float *bias, int N, bool relu, void *Y,
                     int64_t ldy, void *ws, hipStream_t s)
{
    const TileShape t = tile_shape(gl.n, gl.E, K, N, sizeof(T), false);
    char *at = static_cast<char *>(ws);
    PrepareCall p{};
    p.gl = gl;
    p.rows = plan_at(at, gl.n, gl.E, t.height);
    p.row_blocks = int(ceil_div(p.rows.room, kGgThreads));
    p.W = W;
    p.bias = bias;
    p.bias_out = reinterpret_cast<float *>(at);
    at += t.bias_bytes;
    p.B = reinterpret_cast<uint4 *>(at);
    p.K = K;
    p.N = N;
    p.col_tiles = t.n_tiles * t.BN / 32;
    p.steps = t.steps;
    p.TN = t.TN;
    launch_prepare<T>(p, true, s);
    if (int rc = check_launch(fn)) return rc;
    const RowsCall q{gl, p.rows.tiles, p.rows.first + gl.E, p.B, bias ? p.bias_out : nullptr, X, nullptr, Y, W, ldx, ldy, N, 1, K, N,
                     t.steps, t.n_tiles, relu};
    return launch_rows<T, false>(fn, sizeof(T) == 2 ? "grouped_fwd_bf16" : "grouped_fwd", q, t, s);
}

template <typename T>
static int tiles_bwd(const char *fn, const GroupList &gl, const void *X, int64_t ldx, const void *Y, const void *dY, int64_t ldy, const float *W, int F_in,
                     int F_out, bool relu, float *dW, float *db, void *dX, int64_t ld_dx, void *ws, hipStream_t s)
{
    const TileShape t = tile_shape(gl.n, gl.E, F_out, F_in, sizeof(T), relu);
    const int height = weight_shape(gl.n, gl.E, F_in, F_out).height;
    char *at = static_cast<char *>(ws);
    PrepareCall p{};
    p.gl = gl;
    p.runs = plan_at(at, gl.n, gl.E, height);
    p.run_blocks = int(ceil_div(p.runs.room, kGgThreads));
    float *partial = reinterpret_cast<float *>(at);
    at += round_up(size_t(p.runs.room) * size_t(F_in) * size_t(F_out) * 4, 256);
    float *colsum = reinterpret_cast<float *>(at);
    at += round_up(size_t(p.runs.room) * size_t(F_out) * 4, 256);
    if (dX) {
        p.rows = plan_at(at, gl.n, gl.E, t.height);
        p.row_blocks = int(ceil_div(p.rows.room, kGgThreads));
        p.W = W;
        p.B = reinterpret_cast<uint4 *>(at);
        p.K = F_out;
        p.N = F_in;
        p.col_tiles = t.n_tiles * t.BN / 32;
        p.steps = t.steps;
        p.TN = t.TN;
    }
    launch_prepare<T>(p, false, s);
    if (int rc = check_launch(fn)) return rc;
    if (dX) {
        const RowsCall q{gl, p.rows.tiles, p.rows.first + gl.E, p.B, nullptr, dY, relu ? Y : nullptr, dX, W, ldy, ld_dx, 1, F_out, F_out, F_in,
                         t.steps, t.n_tiles, false};
        const char *name = sizeof(T) == 2 ? "grouped_bwd_data_bf16" : "grouped_bwd_data";
        if (int rc = relu ? launch_rows<T, true>(fn, name, q, t, s) : launch_rows<T, false>(fn, name, q, t, s)) return rc;
    }
    {
        const WeightShape w = weight_shape(gl.n, gl.E, F_in, F_out);
        const WeightCall q{gl, p.runs.tiles, p.runs.first, X, dY, relu ? Y : nullptr, ldx, ldy, F_in, F_out, w.m_tiles, w.n_tiles, dW, db, partial, colsum};
        const bool words = rows_in_words<T>(X, ldx, gl.n, F_in) && rows_in_words<T>(dY, ldy, gl.n, F_out) && (!relu || aligned(Y, 4));
        TMA_TIMED(sizeof(T) == 2 ? "grouped_bwd_weight_bf16" : "grouped_bwd_weight", s);
        launch_weight<T>(q, w, relu, words, p.runs.room, s);
        if (int rc = check_launch(fn)) return rc;
    }
    const int64_t cells = int64_t(F_in) * F_out;
    int64_t blocks = ceil_div(cells, kGgThreads);
    if (blocks > 1024) blocks = 1024;
    TMA_TIMED("grouped_join", s);
    hipLaunchKernelGGL(grouped_join_kernel, dim3(unsigned(blocks), unsigned(gl.E)), dim3(kGgThreads), 0, s, p.runs.first, cells, F_out, partial, colsum, dW, db);
    return check_launch(fn);
}

// sizes that the calls take; their workspaces are computed for no others (a width near the end of 32 bits would leave a count of zero to divide by)
static bool sizes_ok(int64_t n, int32_t E, int32_t F_in, int32_t F_out)
{
    return n >= 0 && n <= INT32_MAX && E >= 1 && E <= kMaxGroups && F_in >= 1 && F_out >= 1 && F_in <= (1 << 16) && F_out <= (1 << 16);
}

static int check_grouped(const char *fn, int64_t n, int32_t E, const int32_t *offsets, int32_t F_in, int32_t F_out, int32_t act, int32_t dtype,
                         const void *ws, size_t ws_bytes, size_t need)
{
    TMA_REQUIRE(n >= 0 && n <= INT32_MAX, TMA_ERR_INVALID_ARG, "%s: n outside [0, 2^31)", fn);
    TMA_REQUIRE(E >= 1 && E <= kMaxGroups, TMA_ERR_BAD_SHAPE, "%s: E=%d outside [1, %d]", fn, E, kMaxGroups);
    TMA_REQUIRE(F_in >= 1 && F_out >= 1 && F_in <= (1 << 16) && F_out <= (1 << 16), TMA_ERR_BAD_SHAPE, "%s: F_in=%d F_out=%d", fn, F_in, F_out);
    TMA_REQUIRE(act == TMA_ACT_NONE || act == TMA_ACT_RELU, TMA_ERR_INVALID_ARG, "%s: act %d", fn, act);
    TMA_REQUIRE(dtype == TMA_F32 || dtype == TMA_BF16, TMA_ERR_UNSUPPORTED_DTYPE, "%s: dtype %d", fn, dtype);
    TMA_REQUIRE(offsets, TMA_ERR_INVALID_ARG, "%s: offsets is NULL", fn);
    TMA_REQUIRE(ws && aligned(ws, 256), TMA_ERR_INVALID_ARG, "%s: workspace NULL or not 256-byte aligned", fn);
    TMA_REQUIRE(ws_bytes >= need, TMA_ERR_WORKSPACE_TOO_SMALL, "%s: workspace %zu < %zu", fn, ws_bytes, need);
    return TMA_OK;
}

}  // namespace tma

extern "C" size_t tma_grouped_dense_fwd_workspace_bytes(int64_t n, int32_t E, int32_t F_in, int32_t F_out, int32_t dtype)
{
    using namespace tma;
    if (!sizes_ok(n, E, F_in, F_out)) return 0;
    if (few_rows_a_group(n, E, dtype)) return 256;
    const TileShape t = tile_shape(n, E, F_in, F_out, dtype == TMA_BF16 ? 2 : 4, false);
    return plan_bytes(n, E, t.height) + t.bias_bytes + t.fragment_bytes;
}

extern "C" int tma_grouped_dense_fwd(int64_t n, int32_t E, const int32_t *offsets, const int32_t *order, const void *X, int64_t ldx, int32_t F_in,
                                     const float *W, const float *bias, int32_t F_out, int32_t act, int32_t dtype, void *Y_out, int64_t ldy, void *ws,
                                     size_t ws_bytes, tma_stream_t stream)
{
    using namespace tma;
    const char *fn = "tma_grouped_dense_fwd";
    if (int rc = check_grouped(fn, n, E, offsets, F_in, F_out, act, dtype, ws, ws_bytes, tma_grouped_dense_fwd_workspace_bytes(n, E, F_in, F_out, dtype)))
        return rc;
    if (n == 0) return TMA_OK;
    TMA_REQUIRE(X && W && Y_out && X != Y_out, TMA_ERR_INVALID_ARG, "%s: NULL argument, or X and Y_out are one", fn);
    TMA_REQUIRE(ldx >= F_in && ldy >= F_out, TMA_ERR_BAD_SHAPE, "%s: ldx < F_in or ldy < F_out", fn);
    const GroupList gl{offsets, order, E, n};
    hipStream_t s = as_stream(stream);
    const bool relu = act == TMA_ACT_RELU;
    if (!few_rows_a_group(n, E, dtype))
        return dtype == TMA_F32 ? tiles_fwd<float>(fn, gl, X, ldx, F_in, W, bias, F_out, relu, Y_out, ldy, ws, s)
                                : tiles_fwd<uint16_t>(fn, gl, X, ldx, F_in, W, bias, F_out, relu, Y_out, ldy, ws, s);
    return dtype == TMA_F32 ? few_fwd<float>(fn, gl, X, ldx, F_in, W, bias, F_out, relu, Y_out, ldy, s)
                            : few_fwd<uint16_t>(fn, gl, X, ldx, F_in, W, bias, F_out, relu, Y_out, ldy, s);
}

extern "C" size_t tma_grouped_dense_bwd_workspace_bytes(int64_t n, int32_t E, int32_t F_in, int32_t F_out, int32_t dtype, int32_t need_dX)
{
    using namespace tma;
    if (!sizes_ok(n, E, F_in, F_out)) return 0;
    if (few_rows_a_group(n, E, dtype)) return 256;
    const int height = weight_shape(n, E, F_in, F_out).height;
    const size_t runs = size_t(tile_room(n, E, height));
    size_t bytes = plan_bytes(n, E, height) + round_up(runs * size_t(F_in) * size_t(F_out) * 4, 256) + round_up(runs * size_t(F_out) * 4, 256);
    if (need_dX) {
        size_t most = 0;           // with a mask or without
        for (bool masked : {false, true}) {
            const TileShape t = tile_shape(n, E, F_out, F_in, dtype == TMA_BF16 ? 2 : 4, masked);
            const size_t need = plan_bytes(n, E, t.height) + t.fragment_bytes;
            if (need > most) most = need;
        }
        bytes += most;
    }
    return bytes;
}

extern "C" int tma_grouped_dense_bwd(int64_t n, int32_t E, const int32_t *offsets, const int32_t *order, const void *X, int64_t ldx, const void *Y,
                                     const void *dY, int64_t ldy, const float *W, int32_t F_in, int32_t F_out, int32_t act, int32_t dtype, float *dW,
                                     float *dbias, void *dX_out, int64_t ld_dx, void *ws, size_t ws_bytes, tma_stream_t stream)
{
    using namespace tma;
    const char *fn = "tma_grouped_dense_bwd";
    if (int rc = check_grouped(fn, n, E, offsets, F_in, F_out, act, dtype, ws, ws_bytes,
                               tma_grouped_dense_bwd_workspace_bytes(n, E, F_in, F_out, dtype, dX_out != nullptr)))
        return rc;
    TMA_REQUIRE(dW, TMA_ERR_INVALID_ARG, "%s: dW is NULL", fn);
    if (n > 0) {
        TMA_REQUIRE(X && dY && W, TMA_ERR_INVALID_ARG, "%s: NULL argument", fn);
        TMA_REQUIRE(act == TMA_ACT_NONE || Y, TMA_ERR_INVALID_ARG, "%s: Y is required with ReLU", fn);
        TMA_REQUIRE(ldx >= F_in && ldy >= F_out && (!dX_out || ld_dx >= F_in), TMA_ERR_BAD_SHAPE, "%s: a leading dimension is below its width", fn);
        TMA_REQUIRE(dX_out != X && (!dX_out || (dX_out != dY && dX_out != Y)), TMA_ERR_INVALID_ARG, "%s: dX_out is one of the inputs", fn);
    }
    const GroupList gl{offsets, order, E, n};
    hipStream_t s = as_stream(stream);
    const bool relu = act == TMA_ACT_RELU;
    if (!few_rows_a_group(n, E, dtype))
        return dtype == TMA_F32 ? tiles_bwd<float>(fn, gl, X, ldx, Y, dY, ldy, W, F_in, F_out, relu, dW, dbias, dX_out, ld_dx, ws, s)
                                : tiles_bwd<uint16_t>(fn, gl, X, ldx, Y, dY, ldy, W, F_in, F_out, relu, dW, dbias, dX_out, ld_dx, ws, s);
    return dtype == TMA_F32 ? few_bwd<float>(fn, gl, X, ldx, Y, dY, ldy, W, F_in, F_out, relu, dW, dbias, n > 0 ? dX_out : nullptr, ld_dx, s)
                            : few_bwd<uint16_t>(fn, gl, X, ldx, Y, dY, ldy, W, F_in, F_out, relu, dW, dbias, n > 0 ? dX_out : nullptr, ld_dx, s);
}
