// Forward products of few rows (serving: one token, a few requests together): bound by reading the fp32 weights once, so nothing is laid out before.
//
// A block takes 16 columns (of both weights where there are two) and all of k; its sixteen wavefronts share k out, and each loads the weights as they lie, eight
// neighbours along k of a column a lane, straight into the registers that v_mfma_f32_16x16x32_bf16 wants them in: 64 bytes of a weight's row by 16 lanes, the rest of
// the line by the block beside it, which runs on the same die.  One row 2048 -> 5632 gated in bf16 (92 MB) 24 us, 3.8 TB/s.  The matrix unit has time to spare, so the weights are taken as they are, in three bf16 parts (24 bits).
// The shares of k are joined in LDS, in their order.
#pragma once
#include "wide_gemm.hpp"

namespace tma {

constexpr int kFewMost = 64;       // rows

typedef float floatx4 __attribute__((ext_vector_type(4)));

struct FewCall {
    const void *X;
    int64_t ldx;
    const float *W[2];
    int n, K, N, blocks;
    bool whole;                    // rows of X begin at 16 bytes
};

// kFrags: of 16 rows.  kWaves: 16 where a compute unit has one block at most and 128 registers suffice, else 8 (64 rows 4096 -> 1024 in fp32 99 -> 48 us: with 16
// their registers went to scratch memory).
template <typename T, int kSides, int kFrags, int kWaves, class Out>
__global__ __launch_bounds__(kWaves * 64) void few_rows_kernel(FewCall q, Out out)
{
    constexpr int kX = sizeof(T) == 2 ? 1 : 3, kDeep = kSides * kFrags > 1 ? 1 : 2;      // (what 128 registers hold, twice)
    __shared__ __attribute__((aligned(16))) float shares[kWaves][kFrags * kSides][256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l15 = lane & 15, group = lane >> 4;
    // neighbours on one die
    const int per_die = (q.blocks + kWideDies - 1) / kWideDies, unit = int(blockIdx.x) % kWideDies * per_die + int(blockIdx.x) / kWideDies;
    if (unit >= q.blocks) return;
    const int c0 = unit * 16, col = c0 + l15 < q.N ? c0 + l15 : q.N - 1;
    const int steps = (q.K + 31) / 32, first = int(int64_t(steps) * wave / kWaves), last = int(int64_t(steps) * (wave + 1) / kWaves);

    floatx4 acc[kFrags][kSides];
#pragma unroll
    for (int f = 0; f < kFrags; ++f)
#pragma unroll
        for (int s = 0; s < kSides; ++s) acc[f][s] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    struct Loaded {
        float w[kDeep][kSides][8];
        uint4 x[kDeep][kFrags][kX];
    };
    // steps [step, step + kDeep) before `last`.  A whole step's addresses are a scalar base and a lane's offsets that stay.
    uint32_t at[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) at[j] = uint32_t((group * 8 + j) * int64_t(q.N) + col) * 4u;
    const int whole_steps = q.K / 32;
    auto load = [&](int step, Loaded &v) {
#pragma unroll
        for (int d = 0; d < kDeep; ++d) {
            const int t = step + d;
            if (t >= last) break;
            if (t < whole_steps) {
#pragma unroll
                for (int s = 0; s < kSides; ++s) {
                    const char *base = reinterpret_cast<const char *>(q.W[s] + int64_t(t) * 32 * q.N);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v.w[d][s][j] = *reinterpret_cast<const float *>(base + at[j]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int k = t * 32 + group * 8 + j;
#pragma unroll
                    for (int s = 0; s < kSides; ++s) v.w[d][s][j] = q.W[s][int64_t(k < q.K ? k : q.K - 1) * q.N + col];      // (past the end: times a zero)
                }
            }
#pragma unroll
            for (int f = 0; f < kFrags; ++f) {
                const int row = f * 16 + l15, k0 = t * 32 + group * 8;
                const T *from = static_cast<const T *>(q.X) + row * q.ldx;
                if constexpr (kX == 1) {
                    v.x[d][f][0] = make_uint4(0, 0, 0, 0);
                    if (row < q.n) {
                        if (q.whole && k0 + 8 <= q.K) {
                            v.x[d][f][0] = *reinterpret_cast<const uint4 *>(from + k0);
                        } else {
                            float one[8];
                            load_eight(from, k0, q.K, false, one);
                            pack_eight<1>(one, v.x[d][f]);
                        }
                    }
                } else {
                    float one[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                    if (row < q.n) load_eight(from, k0, q.K, q.whole, one);
                    pack_eight<kX>(one, v.x[d][f]);
                }
            }
        }
    };
    auto multiply = [&](int step, const Loaded &v) {
#pragma unroll
        for (int d = 0; d < kDeep; ++d) {
            if (step + d >= last) break;
#pragma unroll
            for (int s = 0; s < kSides; ++s) {
                uint4 parts[3];
                pack_eight<3>(v.w[d][s], parts);
#pragma unroll
                for (int f = 0; f < kFrags; ++f) {
                    auto add = [&](int p, int r) {
                        acc[f][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, parts[p]), __builtin_bit_cast(bf16x8, v.x[d][f][r]), acc[f][s], 0, 0, 0);
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
        }
    };
    Loaded v[2];
    load(first, v[0]);
    for (int step = first; step < last; step += 2 * kDeep) {
        load(step + kDeep, v[1]);
        multiply(step, v[0]);
        load(step + 2 * kDeep, v[0]);
        multiply(step + kDeep, v[1]);
    }
    // register r of lane l: column 4 (l / 16) + r of row l % 16
#pragma unroll
    for (int f = 0; f < kFrags; ++f)
#pragma unroll
        for (int s = 0; s < kSides; ++s) *reinterpret_cast<float4 *>(&shares[wave][f * kSides + s][lane * 4]) = make_float4(acc[f][s][0], acc[f][s][1], acc[f][s][2], acc[f][s][3]);
    __syncthreads();
    for (int t = threadIdx.x; t < kFrags * 256; t += kWaves * 64) {
        const int c = t % 16, in = t / 16 % 16, f = t / 256, row = f * 16 + in;
        if (row >= q.n || c0 + c >= q.N) continue;
        float sum[kSides] = {};
        for (int w = 0; w < kWaves; ++w)
#pragma unroll
            for (int s = 0; s < kSides; ++s) sum[s] += shares[w][f * kSides + s][(c / 4 * 16 + in) * 4 + c % 4];
        out.one(row, c0 + c, sum[0], sum[kSides - 1]);
    }
}

template <typename T, int kSides, class Out>
static int launch_few(const char *fn, const char *name, int64_t n, const void *X, int64_t ldx, const float *W, const float *second, int32_t F_in, int32_t F_out, const Out &out,
                      hipStream_t s)
{
    const FewCall q{X, ldx, {W, second}, int(n), F_in, F_out, int(ceil_div(F_out, 16)), whole_rows(static_cast<const T *>(X), ldx)};
    const dim3 grid(unsigned(round_up(size_t(q.blocks), kWideDies)));
    TMA_TIMED(name, s);
    auto go = [&](auto frags, auto waves) {
        constexpr int F = decltype(frags)::value, V = decltype(waves)::value;
        hipLaunchKernelGGL((few_rows_kernel<T, kSides, F, V, Out>), grid, dim3(V * 64), 0, s, q, out);
    };
    const std::integral_constant<int, 16> sixteen;
    const std::integral_constant<int, 8> eight;
    const bool alone = q.blocks <= 256;
    if (n <= 16) alone ? go(std::integral_constant<int, 1>{}, sixteen) : go(std::integral_constant<int, 1>{}, eight);
    else if (n <= 32) go(std::integral_constant<int, 2>{}, eight);
    else go(std::integral_constant<int, 4>{}, eight);
    return check_launch(fn);
}

}  // namespace tma
