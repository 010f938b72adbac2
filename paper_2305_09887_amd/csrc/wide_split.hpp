// Products of fp32 operands, laid out in three bf16 parts each (wide_gemm.hpp; why three parts and six products suffice: gemm_split.hpp).
//
// A slab is 16 k-values of all parts of 128 rows and 128 columns, 24 KB, fetched once and multiplied six times: 192 cycles of a matrix unit for 16 k-values of a
// fragment, where the fp32 instruction takes 512.  The product of the first parts has accumulators of its own, the other five, 2^-8 and less of
// it, share the rest.  Three blocks a compute unit, one tile each (two where something is added to the results, which takes registers): one multiplies while the others
// wait, fill their ring or write (gated 128 -> 256, 125,237 rows: two 163 us, three 148).
// (Plane after plane through the bf16 kernel, six sweeps over operands that no cache holds: weight gradients of 128 x 512 from 125,237 rows 199 us, so 127; 30,011 rows
// 301 -> 777 146 and 111, their input gradient 147 and 117.)
#pragma once
#include "wide_gemm.hpp"

namespace tma {

template <bool kTurnedRows, class Epi>
__global__ __launch_bounds__(256, Epi::kPast ? 2 : 3) void wide_split_kernel(WideCall q, Epi epi)
{
    constexpr int F = 4, T = 2, kStages = Epi::kPast ? 3 : 2, kUnits = 6 * F, kLoads = 6, kStageBytes = kUnits * kUnitBytes;
    __shared__ __attribute__((aligned(1024))) uint4 ring[kStages * kUnits * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / 2, wn = wave % 2;
    const int64_t total = int64_t(q.m_tiles) * q.n_tiles * q.splits, per_die = (total + kWideDies - 1) / kWideDies;
    const int64_t work = blockIdx.x % kWideDies * per_die + blockIdx.x / kWideDies;
    if (blockIdx.x / kWideDies >= per_die || work >= total) return;
    const WideTile tile = wide_tile(q, work);
    const int steps = q.slabs_of(tile.split) * 2;
    const AlongRows turned_at(lane, 512);
    const int weights_at[2] = {weights_place(lane & 31, lane >> 5, 0), weights_place(lane & 31, lane >> 5, 1)};

    // A slab in LDS: [operand][part][unit].  This wavefront fetches half of one operand's: parts 0 0 0 0 1 1 or 1 1 2 2 2 2, units 0 1 2 3 0 1 or 2 3 0 1 2 3, in
    // three pairs of neighbours.
    const bool rows_side = wave < 2, turned = kTurnedRows && rows_side;
    const int half = wave & 1;
    const Packed &o = rows_side ? q.a : q.b;
    // turned: 16 of a unit's rows are a slab's k-values, 512 bytes, and a load takes those of two units, 32 rows of the result; units past the last are the last again
    const int kg = tile.m * (2 * F), rb = (rows_side ? tile.m : tile.n) * F, units_left = turned ? (o.kgs - kg) / 2 : o.rbs - rb;
    const char *first = turned ? o.at : o.at + o.unit(rb, int64_t(tile.split) * q.split_slabs * 2);
    const char *from[3] = {first + half * o.plane(), first + half * 2 * o.plane(), first + (1 + half) * o.plane()};
    const int unit[3] = {half * 2, half ? 0 : 2, half * 2};
    const uint32_t ring0 = lds_address(&ring[0]) + uint32_t(wave * kLoads * kUnitBytes);
    const uint32_t lane_at = uint32_t((turned ? lane & 31 : lane) * 16);
    // the slab that is fetched next: bytes from `from`, from slab to slab (turned: in a group), and from unit to unit along the result's rows (turned: as many as the group has)
    int step = turned ? tile.split * q.split_slabs * 2 : 0;
    uint64_t along = 0;
    uint32_t apart = 512, group = kUnitBytes, lane_from = lane_at;
    auto enter_group = [&]() {
        along = uint64_t(o.unit(step >> 1, kg));
        group = uint32_t(o.group(step >> 1)) * uint32_t(2 * kUnitBytes);
        lane_from = lane_at + (lane >> 5) * (group / 2);      // (a pair of units)
    };
    if (turned) enter_group();
    else apart = uint32_t(o.group(rb)) * uint32_t(kUnitBytes);
    auto fetch = [&](int at_step) {
        const uint32_t to = ring0 + uint32_t(at_step % kStages * kStageBytes);
        auto scalar = [](uint64_t at) {
            return reinterpret_cast<const char *>(uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(int(at >> 32)))) << 32 | uint32_t(__builtin_amdgcn_readfirstlane(int(at))));
        };
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            const uint64_t at = reinterpret_cast<uint64_t>(from[p]) + along;
            const char *base = scalar(at);
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                const int u = unit[p] + v < units_left ? unit[p] + v : units_left - 1;
                const uint32_t place = to + uint32_t((2 * p + v) * kUnitBytes);
                // (turned: registers are short)
                if constexpr (kTurnedRows) fetch_unit(place, scalar(at + uint32_t(u) * group), lane_from);
                else fetch_unit(place, base, lane_at + uint32_t(u) * uint32_t(kUnitBytes));
            }
        }
        along += apart;
        if constexpr (kTurnedRows)
            if (turned && (++step & 15) == 0 && (step >> 1) < o.rbs) enter_group();
    };
    // a wavefront whose units are all past the last fetches for the others only
    const bool idle = tile.n * F + wn * T >= q.b.rbs || (!kTurnedRows && tile.m * F + wm * T >= q.a.rbs);
    floatx16 sum[T][T], rest[T][T];
#pragma unroll
    for (int j = 0; j < T; ++j)
#pragma unroll
        for (int i = 0; i < T; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[j][i][r] = rest[j][i][r] = 0.0f;
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s)
        if (s < steps) fetch(s);
    for (int s = 0; s < steps; ++s) {
        if (s + kStages - 2 < steps) wait_and_meet<(kStages - 2) * kLoads>();
        else wait_and_meet<0>();
        if (s + kStages - 1 < steps) fetch(s + kStages - 1);      // into the place that every wavefront has read before this meeting
        if (idle) continue;
        const uint4 *slab = &ring[s % kStages * (kUnits * 64)], *units = slab + lane, *weights = slab + (s & 1 ? weights_at[1] : weights_at[0]);
        uint4 a[3][T], b[3][T];
#pragma unroll
        for (int p = 0; p < 3; ++p)
#pragma unroll
            for (int i = 0; i < T; ++i) {
                if constexpr (kTurnedRows) a[p][i] = along_rows(slab + (p * F + wm * T + i) * 64, turned_at);
                else a[p][i] = units[(p * F + wm * T + i) * 64];
                b[p][i] = weights[(3 * F + p * F + wn * T + i) * 64];
            }
        auto add = [&](int pa, int pb, floatx16 (&to)[T][T]) {
#pragma unroll
            for (int j = 0; j < T; ++j)
#pragma unroll
                for (int i = 0; i < T; ++i)
                    to[j][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, b[pb][j]), __builtin_bit_cast(bf16x8, a[pa][i]), to[j][i], 0, 0, 0);
        };
        add(0, 0, sum);
        add(1, 0, rest);
        add(0, 1, rest);
        add(1, 1, rest);
        add(2, 0, rest);
        add(0, 2, rest);
    }
#pragma unroll
    for (int j = 0; j < T; ++j)
#pragma unroll
        for (int i = 0; i < T; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[j][i][r] += rest[j][i][r];
    wait_and_meet<0>();      // the ring is read: its place takes the results
    constexpr int S = Epi::kSides;
    write_out<T, T>(epi, sum, int64_t(tile.m) * (F * 32) + wm * T * 32, (tile.n * F + wn * T) / S * 32, tile.split, reinterpret_cast<float *>(&ring[wave * 512]), lane);
}

}  // namespace tma
