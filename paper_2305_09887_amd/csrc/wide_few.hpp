// Forward products of few rows (serving: one token, a few requests together): bound by reading the fp32 weights once, so nothing is laid out before.
//
// A block takes 16 columns of both weights, or 32 of one, and all of k or a range of it; its wavefronts share that out, and each loads the weights as they lie, eight
// neighbours along k of a column a lane, straight into the registers that v_mfma_f32_16x16x32_bf16 wants them in.  The matrix unit has time to spare, so the
// weights are taken as they are, in three bf16 parts (24 bits).  Their shares of k are joined in LDS, in their order.
//
// A compute unit reads some 20 bytes a nanosecond, whatever the others do: 128 blocks, alone on theirs, take as long as 256, and 352 twice as long.  So k is split over
// blocks where that spreads the bytes, and a second kernel joins the ranges, in their order.
#pragma once
#include "wide_gemm.hpp"

namespace tma {

constexpr int kFewMost = 64;       // rows

typedef float floatx4 __attribute__((ext_vector_type(4)));

struct FewCall {
    const void *X;
    int64_t ldx;
    const float *W[2];
    int n, K, N, blocks, splits;   // blocks: of 32 / kSides columns
    bool whole;                    // rows of X begin at 16 bytes
    float *partial;                // [splits][kSides][n][N], where k is split over blocks
};

// kFrags: of 16 rows.  A wavefront has two fragments of weights: one of either matrix, or one matrix's even and odd columns.
template <typename T, int kSides, int kFrags, int kWaves, class Out>
__global__ __launch_bounds__(kWaves * 64, kWaves == 8 ? 4 : 2) void few_rows_kernel(FewCall q, Out out)
{
    constexpr int kX = sizeof(T) == 2 ? 1 : 3, kWide = 2 / kSides, kCols = 16 * kWide;
    __shared__ __attribute__((aligned(16))) float shares[kWaves][kFrags * kSides * kWide][256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l15 = lane & 15, group = lane >> 4;
    // neighbours on one die
    const int units = q.blocks * q.splits, per_die = (units + kWideDies - 1) / kWideDies, in_die = int(blockIdx.x) / kWideDies, unit = int(blockIdx.x) % kWideDies * per_die + in_die;
    if (in_die >= per_die || unit >= units) return;
    const int split = unit / q.blocks, c0 = unit % q.blocks * kCols;
    const bool inside = c0 + kCols <= q.N;
    const int steps = (q.K + 31) / 32, from_step = int(int64_t(steps) * split / q.splits), mine = int(int64_t(steps) * (split + 1) / q.splits) - from_step;
    const int first = from_step + mine * wave / kWaves, last = from_step + mine * (wave + 1) / kWaves;

    floatx4 acc[kFrags][kSides][kWide];
#pragma unroll
    for (int f = 0; f < kFrags; ++f)
#pragma unroll
        for (int s = 0; s < kSides; ++s)
#pragma unroll
            for (int c = 0; c < kWide; ++c) acc[f][s][c] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    struct Loaded {
        float w[kSides][kWide][8];
        float x32[kX == 3 ? kFrags : 1][8];
        uint4 x16[kX == 1 ? kFrags : 1];
    };
    // of a whole step the addresses are a scalar base and a lane's offsets that stay
    uint32_t at[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) at[j] = uint32_t((group * 8 + j) * int64_t(q.N) + c0 + l15 * kWide) * 4u;
    const int whole_steps = inside ? q.K / 32 : 0;
    auto load = [&](int t, Loaded &v) {
        if (t >= last) return;
        if (t < whole_steps) {
#pragma unroll
            for (int s = 0; s < kSides; ++s) {
                const char *base = reinterpret_cast<const char *>(q.W[s] + int64_t(t) * 32 * q.N);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float w[kWide];
                    __builtin_memcpy(w, base + at[j], sizeof(w));
#pragma unroll
                    for (int c = 0; c < kWide; ++c) v.w[s][c][j] = w[c];
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int k = t * 32 + group * 8 + j;
#pragma unroll
                for (int s = 0; s < kSides; ++s)
#pragma unroll
                    for (int c = 0; c < kWide; ++c) {
                        const int col = c0 + l15 * kWide + c;
                        const float w = q.W[s][int64_t(k < q.K ? k : q.K - 1) * q.N + (col < q.N ? col : q.N - 1)];
                        v.w[s][c][j] = k < q.K ? w : 0.0f;
                    }
            }
        }
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
            const int row = f * 16 + l15, k0 = t * 32 + group * 8;
            const T *from = static_cast<const T *>(q.X) + row * q.ldx;
            if constexpr (kX == 1) {
                v.x16[f] = make_uint4(0, 0, 0, 0);
                if (row < q.n) {
                    if (q.whole && k0 + 8 <= q.K) {
                        v.x16[f] = *reinterpret_cast<const uint4 *>(from + k0);
                    } else {
                        float one[8];
                        uint4 packed[1];
                        load_eight(from, k0, q.K, false, one);
                        pack_eight<1>(one, packed);
                        v.x16[f] = packed[0];
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) v.x32[f][j] = 0.0f;
                if (row < q.n) load_eight(from, k0, q.K, q.whole, v.x32[f]);
            }
        }
    };
    auto multiply = [&](int t, const Loaded &v) {
        if (t >= last) return;
        uint4 x[kFrags][kX];
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
            if constexpr (kX == 1) x[f][0] = v.x16[f];
            else pack_eight<3>(v.x32[f], x[f]);
        }
#pragma unroll
        for (int s = 0; s < kSides; ++s)
#pragma unroll
            for (int c = 0; c < kWide; ++c) {
                uint4 parts[3];
                pack_eight<3>(v.w[s][c], parts);
#pragma unroll
                for (int f = 0; f < kFrags; ++f) {
                    auto add = [&](int p, int r) {
                        acc[f][s][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, parts[p]), __builtin_bit_cast(bf16x8, x[f][r]), acc[f][s][c], 0, 0, 0);
                    };
                    if constexpr (kX == 3) {
                        add(2, 0);
                        add(0, 2);
                        add(1, 1);
                        add(1, 0);
                        add(0, 1);
                        add(0, 0);
                    } else {
                        add(2, 0);
                        add(1, 0);
                        add(0, 0);
                    }
                }
            }
    };
    Loaded v[2];
    load(first, v[0]);
    for (int t = first; t < last; t += 2) {
        load(t + 1, v[1]);
        multiply(t, v[0]);
        load(t + 2, v[0]);
        multiply(t + 1, v[1]);
    }
    // register r of lane l: column kWide (4 (l / 16) + r) + c of row l % 16
#pragma unroll
    for (int f = 0; f < kFrags; ++f)
#pragma unroll
        for (int s = 0; s < kSides; ++s)
#pragma unroll
            for (int c = 0; c < kWide; ++c) {
                const floatx4 &a = acc[f][s][c];
                *reinterpret_cast<float4 *>(&shares[wave][(f * kSides + s) * kWide + c][lane * 4]) = make_float4(a[0], a[1], a[2], a[3]);
            }
    __syncthreads();
    for (int t = threadIdx.x; t < kFrags * 16 * kCols; t += kWaves * 64) {
        const int c = t % kCols, in = t / kCols % 16, f = t / (16 * kCols), row = f * 16 + in, i = c / kWide;
        if (row >= q.n || c0 + c >= q.N) continue;
        float sum[kSides] = {};
        for (int w = 0; w < kWaves; ++w)
#pragma unroll
            for (int s = 0; s < kSides; ++s) sum[s] += shares[w][(f * kSides + s) * kWide + c % kWide][(i / 4 * 16 + in) * 4 + i % 4];
        if (q.splits == 1) {
            out.one(row, c0 + c, sum[0], sum[kSides - 1]);
        } else {
#pragma unroll
            for (int s = 0; s < kSides; ++s) q.partial[(int64_t(split * kSides + s) * q.n + row) * q.N + c0 + c] = sum[s];
        }
    }
}

// the shares of k added up in their order, and what becomes of them
template <int kSides, class Out>
__global__ __launch_bounds__(256) void few_join_kernel(const float *__restrict__ partial, int splits, int n, int N, Out out)
{
    const int i = int(blockIdx.x) * 256 + int(threadIdx.x), cells = n * N;
    if (i >= cells) return;
    float sum[kSides] = {};
#pragma unroll 4
    for (int p = 0; p < splits; ++p)
#pragma unroll
        for (int s = 0; s < kSides; ++s) sum[s] += partial[int64_t(p * kSides + s) * cells + i];
    out.one(i / N, i % N, sum[0], sum[kSides - 1]);
}

// Ranges of k: as many as make the bytes least that the busiest compute unit moves, eight wavefronts at a time, for all have the same rate, some 20 bytes a
// nanosecond; such a turn costs as much as 8 KB more, the second kernel as much as 50.  (One range, then the one chosen: 24 rows 2048 -> 2 x 5632 in bf16, 352 blocks,
// 39.6 and 30 us; one row 4096 -> 1024 in fp32, 32 blocks, 37 and 11.5; one row 1024 -> 2 x 4096 in bf16, 256 blocks, 11.5, of two 14.5.)
struct FewPlan {
    int blocks, splits;
    size_t bytes;
};
inline int few_waves(int64_t n) { return n <= 16 ? 8 : 4; }
inline FewPlan plan_few(int64_t n, int32_t F_in, int32_t F_out, int sides, int size)
{
    const int64_t blocks = ceil_div(F_out, 32 / sides), steps = ceil_div(F_in, 32), waves = few_waves(n);
    FewPlan best{int(blocks), 1, 0};
    int64_t least = INT64_MAX;
    for (int splits = 1; splits <= 16; splits *= 2) {
        const int64_t turns = ceil_div(blocks * splits * waves, 8 * 256);
        const size_t partial = splits > 1 ? size_t(splits) * size_t(sides) * size_t(n) * size_t(F_out) * 4 : 0;
        const int64_t moved = turns * (8 * ceil_div(steps, splits * waves) * (4096 + n * 32 * size) + 8000) + (splits > 1 ? 50000 + int64_t(partial) * 2 / 256 : 0);
        if (moved < least) {
            least = moved;
            best.splits = splits;
            best.bytes = partial;
        }
    }
    return best;
}

template <typename T, int kSides, class Out>
static int launch_few(const char *fn, const char *name, int64_t n, const void *X, int64_t ldx, const float *W, const float *second, int32_t F_in, int32_t F_out, const Out &out,
                      void *ws, hipStream_t s)
{
    const FewPlan p = plan_few(n, F_in, F_out, kSides, sizeof(T));
    const FewCall q{X, ldx, {W, second}, int(n), F_in, F_out, p.blocks, p.splits, whole_rows(static_cast<const T *>(X), ldx), static_cast<float *>(ws)};
    const dim3 grid(unsigned(round_up(size_t(q.blocks) * size_t(q.splits), kWideDies)));
    {
        TMA_TIMED(name, s);
        if (n <= 16) hipLaunchKernelGGL((few_rows_kernel<T, kSides, 1, 8, Out>), grid, dim3(512), 0, s, q, out);
        else if (n <= 32) hipLaunchKernelGGL((few_rows_kernel<T, kSides, 2, 4, Out>), grid, dim3(256), 0, s, q, out);
        else hipLaunchKernelGGL((few_rows_kernel<T, kSides, 4, 4, Out>), grid, dim3(256), 0, s, q, out);
        if (int rc = check_launch(fn)) return rc;
    }
    if (q.splits == 1) return TMA_OK;
    TMA_TIMED("few_join", s);
    hipLaunchKernelGGL((few_join_kernel<kSides, Out>), dim3(unsigned(ceil_div(n * F_out, 256))), dim3(256), 0, s, q.partial, q.splits, q.n, q.N, out);
    return check_launch(fn);
}

}  // namespace tma
