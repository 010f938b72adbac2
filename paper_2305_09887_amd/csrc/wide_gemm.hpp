// Products of wide layers (gated_dense.hip, dense_residual.hip) on v_mfma_f32_32x32x16_bf16: both operands are laid out as fragments first, so that a product
// has one form for every type, width, pitch, alignment and direction.
//
// Packed operands.  A unit is 1 KB: 32 rows of an operand by 16 k-values, 16 bytes a lane, in the order in which the matrix instruction wants them; what lies
// outside the operand is zero.  Eight units of 256 rows follow each other, then those of the next k-values, of the next rows (a slab of a tile is one run of
// memory; the last rows' groups have the units that there are, so that a narrow layer's gradients, whose rows are its columns, take no more than they are; a
// tile past them has the last one again, for results that are not stored), then planes: fp32 values are taken apart into bf16 parts whose sum
// they are (three of them hold all 24 bits, two hold 17), one plane a part, and a product of such operands is the sum of products of planes, the small ones
// first: a weight gradient in fp32 from bf16 rows is a product of twice the length; fp32 operands have a kernel of their own (wide_split.hpp).
//
// A unit is what one wavefront fetches straight into LDS with one instruction and what it reads from there without conflicts: no swizzle, no edges, no
// masks between memory and the matrix units.  The layout costs a pass over the operands, bytes against the product's rows times columns.
//
// The instruction multiplies weights (its rows) by rows (its columns): a lane ends with results of one row.  Which column a fragment's row is, is the layout's choice: fragment row
// m holds column 16 (m / 4 mod 2) + 4 (m / 8) + m mod 4 of its 32, which makes a lane's sixteen results neighbours.
#pragma once
#include "kernels.hpp"
#include "lds_fetch.hpp"

#include <type_traits>
#include <utility>

namespace tma {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kUnitRows = 32, kUnitK = 16, kUnitBytes = 1024;
constexpr int kWideDies = 8;

struct Packed {
    char *at;
    int rbs, kgs;              // units along the rows and along k (an even number: a slab is two)
    // (planes begin 64 KB apart: what a tile reads of a group, eight units by eight, then lies in one such block; backward of 30,011 rows 301 -> 777 in fp32 362 -> 355 us)
    __host__ __device__ __forceinline__ int64_t plane() const { return (int64_t(rbs) * kgs + 63) / 64 * (64 * kUnitBytes); }
    // units of the group of eight, or of the last ones, that rb is in
    __host__ __device__ __forceinline__ int group(int rb) const { return rbs - (rb & ~7) < 8 ? rbs - (rb & ~7) : 8; }
    __host__ __device__ __forceinline__ int64_t unit(int rb, int64_t kg) const { return (int64_t(rb & ~7) * kgs + kg * group(rb) + (rb & 7)) * kUnitBytes; }
    __host__ size_t bytes(int parts) const { return size_t(plane()) * size_t(parts); }
};
inline Packed packed_shape(int64_t rows, int64_t k)
{
    return Packed{nullptr, int(ceil_div(rows > 0 ? rows : 1, kUnitRows)), int(round_up(size_t(ceil_div(k > 0 ? k : 1, kUnitK)), 2))};
}

// the row of a unit in which column c (of 32) of the weights' side lies
__host__ __device__ __forceinline__ int fragment_row(int c) { return ((c >> 4) & 1) * 4 + ((c >> 2) & 3) * 8 + (c & 3); }
// Where in a unit row r's eight k-values `half` lie, in pieces of 16 bytes.  A unit of rows is in the order of the lanes.  On the weights' side a row's two pieces are
// neighbours, exchanged in every second eight rows: so 16 lanes that read as many rows meet in no bank, and a unit can be read along its rows as
// well (the transposing read takes 16 k-values of four rows): the gradients of pre-activations, laid out for dW with their columns as rows, are dX's rows of k.  In every
// second unit along k rows are four apart exchanged: such a read takes two of them at once.
__host__ __device__ __forceinline__ int rows_place(int r, int half) { return half * 32 + r; }
__host__ __device__ __forceinline__ int weights_place(int r, int half, int kg) { return (r ^ (kg & 1) * 4) * 2 + (half ^ ((r >> 3) & 1)); }

// ---- parts ---------------------------------------------------------------------
// x as a sum of bf16 parts, each the rounding of what the ones before left over.  A finite value beyond the largest bf16 is cut instead of rounded; of an
// infinity or a NaN the first part is that and the others are zero.  Parts below 2^-126 are lost: an error of 2^-126, whatever the value.
template <int kParts>
__device__ __forceinline__ void take_apart(float x, float (&part)[kParts])
{
#pragma unroll
    for (int p = 0; p < kParts; ++p) {
        float h = bf16_to_f32(f32_to_bf16(x));
        if constexpr (kParts > 1) {
            const bool beyond = (__float_as_uint(h) & 0x7F800000u) == 0x7F800000u;
            if (beyond && (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u) h = __uint_as_float(__float_as_uint(x) & 0xFFFF0000u);
            part[p] = h;
            x = (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u ? 0.0f : x - h;
        } else {
            part[p] = h;
        }
    }
}

// Eight values of a row along k -> the lane's 16 bytes of each part.  What a rounding left over comes from one instruction, as in split_pair.hpp: v - h as the dot
// product of the pair (h0, h1) with (-1, 0) or (0, -1), plus v.  (Value by value, with its selects, the parts took the few-row products 600 cycles a wavefront
// and 32 k-values: one row 4096 -> 1024 23 us.)  Values beyond the largest bf16, and what is no number, take the careful way.
struct Remainder {
    typedef __bf16 Pair __attribute__((ext_vector_type(2)));
    uint32_t first, second;
    __device__ __forceinline__ Remainder() : first(0x0000BF80u), second(0xBF800000u)
    {
        // held in registers: as an inline constant of this instruction -1.0 would stand in the other half
        asm("" : "+s"(first));
        asm("" : "+s"(second));
    }
    __device__ __forceinline__ void operator()(float &x, float &y, uint32_t parts) const
    {
        x = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(Pair, parts), __builtin_bit_cast(Pair, first), x, false);
        y = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(Pair, parts), __builtin_bit_cast(Pair, second), y, false);
    }
};
template <int kParts>
__device__ __forceinline__ void pack_eight(const float (&v)[8], uint4 (&out)[kParts])
{
    if constexpr (kParts == 1) {
        out[0] = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
        return;
    }
    uint32_t w[kParts][4];
    // (a NaN makes the comparison false: fmaxf would drop it)
    bool plain = true;
#pragma unroll
    for (int j = 0; j < 8; ++j) plain = plain && fabsf(v[j]) < 0x1p127f;
    if (__all(plain)) {
        const Remainder rest;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float x = v[2 * j], y = v[2 * j + 1];
#pragma unroll
            for (int p = 0; p < kParts; ++p) {
                w[p][j] = pack_bf16(x, y);
                if (p + 1 < kParts) rest(x, y, w[p][j]);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float a[kParts], b[kParts];
            take_apart<kParts>(v[2 * j], a);
            take_apart<kParts>(v[2 * j + 1], b);
#pragma unroll
            for (int p = 0; p < kParts; ++p) w[p][j] = (__float_as_uint(a[p]) >> 16) | (__float_as_uint(b[p]) & 0xFFFF0000u);
        }
    }
#pragma unroll
    for (int p = 0; p < kParts; ++p) out[p] = make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]);
}

__device__ __forceinline__ float widen1(float x) { return x; }
__device__ __forceinline__ float widen1(uint16_t x) { return bf16_to_f32(x); }

// eight neighbours of a row from column c on, zeros past `cols`; kWhole: rows begin at 16 bytes
template <typename T>
__device__ __forceinline__ void load_eight(const T *row, int64_t c, int64_t cols, bool whole, float (&v)[8])
{
    if (whole && c + 8 <= cols) {
        if constexpr (sizeof(T) == 2) {
            Chunk<uint16_t>::load(row + c, v);
        } else {
            const float4 a = *reinterpret_cast<const float4 *>(row + c), b = *reinterpret_cast<const float4 *>(row + c + 4);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
            v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < cols ? widen1(row[c + j]) : 0.0f;
    }
}
template <typename T>
inline bool whole_rows(const T *p, int64_t ld) { return aligned(p, 16) && ld * int64_t(sizeof(T)) % 16 == 0; }

// ---- layouts -------------------------------------------------------------------
constexpr int kPackThreads = 256;

// Operand rows are the rows of src [rows, cols], k along them.  A block takes 32 rows by 64 columns at a time, through LDS: 128 bytes of a row (bf16) are read
// at once and four whole units written.
// The operand may come from `sides` matrices side by side along k, side_kgs units each.  weights: its rows are a fragment's columns, and its k-values, 32 of them,
// stand in the order of such a unit's rows (the other operand is read along those).
struct RowsPack {
    const void *src[2];
    int64_t ld, rows, cols;
    bool whole, weights;
    int side_kgs;
    Packed out;
};
template <int kParts>
using RowsTile = uint4[kParts][kPackThreads];
template <typename T, int kParts>
__device__ __forceinline__ void pack_rows(const RowsPack &q, int block, int blocks, RowsTile<kParts> &tile)
{
    const int t = threadIdx.x, r = t / 8, piece = t % 8;
    const int quads = (q.out.kgs + 3) / 4;
    const int64_t all = int64_t(q.out.rbs) * quads;
    const int slot = (piece / 2) * 64 + (q.weights ? weights_place(fragment_row(r), piece % 2, piece / 2) : rows_place(r, piece % 2));
    for (int64_t i = block; i < all; i += blocks) {
        const int rb = int(i / quads);
        const int64_t row = int64_t(rb) * kUnitRows + r;
        const int kg0 = int(i % quads) * 4, kg = kg0 + piece / 2;
        const int side = kg < q.side_kgs ? 0 : 1;
        const int64_t c = int64_t(kg - side * q.side_kgs) * kUnitK + piece % 2 * 8;
        float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (row < q.rows && kg < q.out.kgs) {
            const T *from = static_cast<const T *>(q.src[side]) + row * q.ld;
            if (q.weights) {      // rows 8 e + [0, 8) of a unit: its columns 4 e + [0, 4) and 16 + 4 e + [0, 4)
                const int64_t c4 = c / 32 * 32 + c % 32 / 8 * 4;
                bool fours = false;
                if constexpr (sizeof(T) == 4) {
                    fours = q.whole && c4 + 20 <= q.cols;
                    if (fours) {
                        const float4 x = *reinterpret_cast<const float4 *>(from + c4), y = *reinterpret_cast<const float4 *>(from + c4 + 16);
                        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
                        v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
                    }
                }
                if (!fours) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int64_t at = c4 + j / 4 * 16 + j % 4;
                        v[j] = at < q.cols ? widen1(from[at]) : 0.0f;
                    }
                }
            } else {
                load_eight(from, c, q.cols, q.whole, v);
            }
        }
        uint4 parts[kParts];
        pack_eight<kParts>(v, parts);
        __syncthreads();
#pragma unroll
        for (int p = 0; p < kParts; ++p) tile[p][slot] = parts[p];
        __syncthreads();
        if (kg0 + t / 64 < q.out.kgs) {
#pragma unroll
            for (int p = 0; p < kParts; ++p)
                *reinterpret_cast<uint4 *>(q.out.at + p * q.out.plane() + q.out.unit(rb, kg0 + t / 64) + t % 64 * 16) = tile[p][t];
        }
    }
}

// Operand rows are the columns of src [rows, cols], k along its rows: a thread takes eight rows of kTogether columns (two of bf16, where words allow it), 32 threads
// of a half wavefront write 512 bytes.
// `sides` matrices give every other unit of 32 operand rows each (a gated layer's two weights).
struct ColsPack {
    const void *src[2];
    int64_t ld, rows, cols;
    int sides;
    bool weights, pairs;
    Packed out;
};
template <typename T, int kParts, int kTogether>
__device__ __forceinline__ void pack_cols_as(const ColsPack &q, int block, int blocks)
{
    constexpr int kWidth = 128 * kTogether;
    const int t = threadIdx.x, c_in = t % 128 * kTogether, half = t / 128;
    const int side_rbs = q.out.rbs / q.sides, strips = (side_rbs * kUnitRows + kWidth - 1) / kWidth;
    const int64_t all = int64_t(strips) * q.out.kgs * q.sides;
    for (int64_t i = block; i < all; i += blocks) {
        const int strip = int(i % strips), side = int(i / strips % q.sides);
        const int64_t kg = i / strips / q.sides;
        const int64_t col = int64_t(strip) * kWidth + c_in, k0 = kg * kUnitK + half * 8;
        const int rb = int(col / kUnitRows);
        if (rb >= side_rbs) continue;
        const T *src = static_cast<const T *>(q.src[side]) + col;
        float v[kTogether][8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool in = k0 + j < q.rows;
            if constexpr (kTogether == 2) {
                const uint32_t w = in && col < q.cols ? *reinterpret_cast<const uint32_t *>(src + (k0 + j) * q.ld) : 0u;      // (cols is even)
                v[0][j] = __uint_as_float(w << 16);
                v[1][j] = __uint_as_float(w & 0xFFFF0000u);
            } else {
                v[0][j] = in && col < q.cols ? widen1(src[(k0 + j) * q.ld]) : 0.0f;
            }
        }
#pragma unroll
        for (int w = 0; w < kTogether; ++w) {
            uint4 parts[kParts];
            pack_eight<kParts>(v[w], parts);
            const int c = (c_in + w) % kUnitRows, slot = q.weights ? weights_place(fragment_row(c), half, int(kg & 1)) : rows_place(c, half);
#pragma unroll
            for (int p = 0; p < kParts; ++p) *reinterpret_cast<uint4 *>(q.out.at + p * q.out.plane() + q.out.unit(rb * q.sides + side, kg) + slot * 16) = parts[p];
        }
    }
}

template <typename T, int kParts>
__device__ __forceinline__ void pack_cols(const ColsPack &q, int block, int blocks)
{
    if constexpr (sizeof(T) == 2)
        if (q.pairs) return pack_cols_as<T, kParts, 2>(q, block, blocks);
    pack_cols_as<T, kParts, 1>(q, block, blocks);
}

inline int pack_blocks(int64_t items) { return int(items < 1 ? 1 : items > 8192 ? 8192 : items); }
template <typename T>
inline RowsPack rows_pack(const void *first, const void *second, int64_t ld, int64_t rows, int64_t cols, bool weights, const Packed &out)
{
    const bool whole = whole_rows(static_cast<const T *>(first), ld) && (!second || whole_rows(static_cast<const T *>(second), ld));
    return {{first, second}, ld, rows, cols, whole, weights, second ? out.kgs / 2 : out.kgs, out};
}
inline int blocks_of(const RowsPack &q) { return pack_blocks(int64_t(q.out.rbs) * ((q.out.kgs + 3) / 4)); }
template <typename T>
inline ColsPack cols_pack(const void *first, const void *second, int64_t ld, int64_t rows, int64_t cols, bool weights, const Packed &out)
{
    const bool pairs = sizeof(T) == 2 && cols % 2 == 0 && ld % 2 == 0 && aligned(first, 4) && aligned(second, 4);
    return {{first, second}, ld, rows, cols, second ? 2 : 1, weights, pairs, out};
}
inline int blocks_of(const ColsPack &q) { return pack_blocks(ceil_div(q.out.rbs / q.sides, q.pairs ? 8 : 4) * q.out.kgs * q.sides); }

// Forward: weights by columns, in the first `cols` blocks, and rows, in what blocks there are beyond
template <typename T, int kParts>
__global__ __launch_bounds__(kPackThreads) void forward_layouts_kernel(ColsPack w, RowsPack x, int cols)
{
    __shared__ __attribute__((aligned(16))) RowsTile<kParts> tile;
    if (int(blockIdx.x) < cols) pack_cols<float, kParts>(w, int(blockIdx.x), cols);
    else pack_rows<T, kParts>(x, int(blockIdx.x) - cols, int(gridDim.x) - cols, tile);
}

// ---- the product ---------------------------------------------------------------
struct Planes {            // pairs of planes, four bits each, the first multiplied in the lowest
    int count;
    uint32_t a, b;
};
inline Planes planes_of(int b_parts)
{
    if (b_parts == 2) return {2, 0x00u, 0x01u};             // (0,1) (0,0)
    return {1, 0u, 0u};
}

// C[m][n] = sum over k of A[m][k] B[n][k]: A's rows are rows of the result, B's are the weights' side.
// kLying: A are rows of bf16 where they lie, at multiples of 16 bytes, of a multiple of 32 elements: nothing of them is laid out.  A wavefront's load then takes
// 64 bytes of 16 rows, and LDS has those rows, their 16-byte pieces exchanged by a quarter of the row's number (16 lanes read as many rows: all banks).
// kTurned: A is laid out as the weights' side of another product, its k-values as rows; a slab is 32 of those, of 16 of A's rows a unit, and is read along them.
enum RowsAs { kUnits_, kLying, kTurned };
struct WideCall {
    Packed a, b;
    Planes planes;
    int m_tiles, n_tiles, panel;      // panel: column tiles that a die's blocks share rows of
    int splits, split_slabs;          // ranges of k, of that many slabs
    int64_t lda, rows;                // kLying: A's pitch in elements, its rows
    int row_units;                    // of 32 rows of the result
    __host__ __device__ __forceinline__ int slabs_of(int split) const
    {
        const int left = b.kgs / 2 - split * split_slabs;
        return left < split_slabs ? left : split_slabs;
    }
};
struct WideTile {
    int m, n, split;
};
__device__ __forceinline__ WideTile wide_tile(const WideCall &q, int64_t work)
{
    const int tiles = q.m_tiles * q.n_tiles, t = int(work % tiles);
    const int per_panel = q.panel * q.m_tiles, p = t / per_panel, in = t % per_panel;
    const int width = (p + 1) * q.panel <= q.n_tiles ? q.panel : q.n_tiles - p * q.panel;
    return {in / width, p * q.panel + in % width, int(work / tiles)};
}

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// A unit into LDS.  The base may come from a vector register by way of a scalar one just before: five wait states, which only the compiler's own
// instructions get from it, are kept here.
__device__ __forceinline__ void fetch_unit(uint32_t lds, const char *base, uint32_t offset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop

// Write-out.  A lane has sixteen columns of a row, and a store of those would go to 32 rows.  So a wavefront's results go through its part of LDS, kRows rows by
// kCols columns of sums at a time, and come back as the E neighbours that 16 bytes of storage hold, of a few rows: bias, activation and addition happen there,
// in loops that are short enough to be unrolled, on whole lines of memory.  (What the compiler does not unroll indexes the results and so keeps them in scratch
// memory: 8,192 rows 2048 -> 4096 in bf16 took 177 us so.)  32 rows by 64 columns, but where two results make one (gated) and two bytes are stored: 16 rows by
// 128, for half lines stored one after the other are dear (2048 -> 8192 with three results 640 us).  The 16-byte pieces of a row are exchanged by its number, so that 16
// lanes never meet in a bank, whether they write 16 rows or read one, two or four.
template <int kRows_, int kCols_>
struct Stage {
    static constexpr int kRows = kRows_, kCols = kCols_;
    float *at;
    int lane;
    static __device__ __forceinline__ int place(int row, int piece)
    {
        return row * kCols + (piece ^ ((piece >> 4 & 1) * 8) ^ (((row & 1) * 9) ^ ((row >> 1) & 7))) * 4;
    }
    // of columns `block` * 32 + [0, 32) this lane's sixteen, where its row is one of `part`'s
    __device__ __forceinline__ void put(int part, int block, const floatx16 &v) const
    {
        const int row = lane & 31, first = block * 8 + (lane >> 5) * 4;
        if (kRows == 32 || row / kRows == part) {
#pragma unroll
            for (int p = 0; p < 4; ++p) *reinterpret_cast<float4 *>(at + place(row % kRows, first + p)) = make_float4(v[4 * p], v[4 * p + 1], v[4 * p + 2], v[4 * p + 3]);
        }
    }
    template <int E>
    __device__ __forceinline__ void get(int row, int col, float (&v)[E]) const
    {
#pragma unroll
        for (int p = 0; p < E / 4; ++p) {
            const float4 x = *reinterpret_cast<const float4 *>(at + place(row, col / 4 + p));
            v[4 * p] = x.x;
            v[4 * p + 1] = x.y;
            v[4 * p + 2] = x.z;
            v[4 * p + 3] = x.w;
        }
    }
};

// The value is there: a load that a path leaves without a use would be waited for, with all fetches, in the main loop, each time its register is written.
__device__ __forceinline__ void arrived(float &v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ void arrived(uint4 &v) { asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w)); }

// A fragment of 32 rows that are the k-values of two units, 16 of each, `stride` bytes apart, and of 16 k-values that are rows of theirs: this lane's eight.  Of four
// rows' 16 k-values, which the lanes of a quarter wavefront address in pieces of four, the transposing read gives each lane one k-value's four.
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;
struct AlongRows {
    uint32_t low, high;      // of the lower four of its eight rows, of the other four
    __device__ __forceinline__ AlongRows(int lane, int stride)
    {
        const int quarter = lane >> 4, i = lane & 15, row = 8 * (quarter >> 1) + (i >> 2), unit = quarter & 1;
        low = uint32_t(unit * stride + weights_place(row, (i & 3) >> 1, unit) * 16 + (i & 1) * 8);
        high = uint32_t(unit * stride + weights_place(row + 4, (i & 3) >> 1, unit) * 16 + (i & 1) * 8);
    }
};
__device__ __forceinline__ uint4 along_rows(const uint4 *units, const AlongRows &at)
{
    const char *p = reinterpret_cast<const char *>(units);
    const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)(p + at.low)));
    const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)(p + at.high)));
    return make_uint4(lo.x, lo.y, hi.x, hi.y);
}

// A wavefront's TN by TM fragments, of rows from row0 and columns from col0 on, by way of its part of LDS
template <int TM, int TN, class Epi>
__device__ __forceinline__ void write_out(const Epi &epi, const floatx16 (&acc)[TN][TM], int64_t row0, int col0, int split, float *at, int lane)
{
    constexpr int S = Epi::kSides;
    typedef typename Epi::template StageOf<TN> Staged;
    constexpr int kJ = Staged::kCols / 32, kGroups = TN / kJ, kParts = 32 / Staged::kRows, kSteps = TM * kGroups * kParts;
    const Staged staged{at, lane};
    typename Epi::template Cols<Staged> cols[kGroups];
#pragma unroll
    for (int j = 0; j < kGroups; ++j) epi.columns(col0 + j * (Staged::kCols / S), lane, cols[j]);
    typename Epi::Past past[2];
    epi.past(row0, col0, lane, past[0]);
#pragma unroll
    for (int j = 0; j < kGroups; ++j) cols[j].wait();
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < kGroups; ++j)
#pragma unroll
            for (int h = 0; h < kParts; ++h) {
                const int step = (i * kGroups + j) * kParts + h;
                if (step + 1 < kSteps && Epi::kPast)
                    epi.past(row0 + (step + 1) / kGroups * 32, col0 + (step + 1) % kGroups * (Staged::kCols / S), lane, past[(step + 1) % 2]);
#pragma unroll
                for (int b = 0; b < kJ; ++b) staged.put(h, b, acc[j * kJ + b][i]);
                __builtin_amdgcn_wave_barrier();      // lanes read what others wrote, and these write again: in the order of the program, which LDS keeps
                epi.emit(staged, row0 + i * 32 + h * Staged::kRows, col0 + j * (Staged::kCols / S), split, cols[j], past[step % 2]);
                __builtin_amdgcn_wave_barrier();
            }
}

// MF x NF units a tile, WM x WN wavefronts.  A ring of slabs of 32 k-values, fetched kStages - 1 ahead through tile boundaries.  One wavefront a SIMD has to keep its
// matrix unit busy by itself: the fragments of the next 16 k-values are read, and the units of a later slab fetched, one between every two matrix
// instructions (each takes the unit 32 cycles).
template <int MF, int NF, int WM, int WN, int kStages, RowsAs kRows, class Epi>
__global__ __launch_bounds__(WM *WN * 64, kStages * (MF + NF) >= 64 ? 1 : 2) void wide_gemm_kernel(WideCall q, Epi epi)
{
    constexpr int kWaves = WM * WN, TM = MF / WM, TN = NF / WN, kUnits = (MF + NF) * 2, kLoads = kUnits / kWaves, kAhead = kStages - 1;
    constexpr int kYoung = (kAhead - 1) * kLoads;
    constexpr int kYoungStores = kYoung + TM * TN * Epi::kStores < 63 ? kYoung + TM * TN * Epi::kStores : 63;
    static_assert(MF % WM == 0 && NF % WN == 0 && kUnits % kWaves == 0 && MF % kLoads == 0 && NF % kLoads == 0 && 8 % MF == 0 && 8 % NF == 0 && kYoung <= 63 && TN % 2 == 0, "tile shape");
    __shared__ __attribute__((aligned(1024))) uint4 ring[kStages * kUnits * 64];
    __shared__ __attribute__((aligned(1024))) uint4 stages[kWaves][512];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;

    const int64_t total = int64_t(q.m_tiles) * q.n_tiles * q.splits;
    const int64_t per_die = (total + kWideDies - 1) / kWideDies, die = blockIdx.x % kWideDies, stride = gridDim.x / kWideDies;
    const int64_t end = (die + 1) * per_die < total ? (die + 1) * per_die : total;
    int64_t work = die * per_die + blockIdx.x / kWideDies;
    if (work >= end) return;

    // ---- the cursor: the slab that is fetched next.  Past the last it stays there: fetched again, into places that nobody reads.
    const uint32_t ring0 = lds_address(&ring[0]);
    // this wavefront's units of a slab: kLoads neighbours of one operand and one of its two k-units
    const int u0 = wave * kLoads;
    const bool rows_side = u0 < 2 * MF;
    const int in_side = rows_side ? u0 : u0 - 2 * MF, k_unit = in_side / (rows_side ? MF : NF), rb_in = in_side % (rows_side ? MF : NF);
    int64_t c_work = work;
    int c_at = 0, c_slabs = 1, c_last = INT32_MAX, c_pair = -1, c_stage = kStages - 1;
    int c_first = 0, c_kg = 0;      // kTurned: the range's first slab, this wavefront's first unit along k
    uint32_t c_apart = 0;           // else: bytes from slab to slab
    // Load v of a lane, from the slab's base on.  kLying: row min(row_in + 16 v, most), this lane's piece of it (of the other operand: 64 bytes of a unit's 1 KB);
    // else unit min(v, most), of 1 KB, or, kTurned, as far apart as its group has units.
    const bool lying = kRows == kLying && rows_side, turned = kRows == kTurned && rows_side;
    uint32_t pitch = lying ? uint32_t(q.lda * 2) : kRows == kLying ? 64u : uint32_t(kUnitBytes);
    const uint32_t piece_at = kRows != kLying ? uint32_t(lane) * 16u : uint32_t(lying ? (lane & 3) ^ (lane >> 4) : lane & 3) * 16u;
    const int row_in = lane / 4 + (lying ? u0 * 16 : 0);
    int most = INT32_MAX;
    const char *from = nullptr;
    uint32_t to = 0;
    auto step = [&]() {
        c_stage = c_stage == kStages - 1 ? 0 : c_stage + 1;
        to = ring0 + uint32_t(c_stage) * uint32_t(kUnits * kUnitBytes) + uint32_t(u0) * uint32_t(kUnitBytes);
        if (++c_at < c_slabs) return;
        if (++c_pair == q.planes.count) {
            c_pair = 0;
            c_work += stride;
            if (c_work >= end) {
                c_last = c_slabs - 1;
                c_slabs = INT32_MAX;
                return;
            }
        }
        c_at = 0;
        const WideTile tile = wide_tile(q, c_work);
        const int rb = (rows_side ? tile.m * MF : tile.n * NF) + rb_in, pair = 4 * c_pair;
        c_slabs = q.slabs_of(tile.split);
        if (lying) {
            const int64_t row0 = int64_t(tile.m) * (MF * 32), left = q.rows - 1 - row0;
            most = left < MF * 32 ? int(left) : MF * 32;
            from = q.a.at + row0 * q.lda * 2 + int64_t(tile.split) * q.split_slabs * 64;
            c_apart = 64;
        } else if (turned) {
            const int kg = tile.m * (MF * 2) + u0, left = q.a.kgs - 1 - kg;
            most = left > 0 ? left : 0;
            from = q.a.at;
            c_kg = left < 0 ? q.a.kgs - 1 : kg;
            c_first = tile.split * q.split_slabs;
        } else {
            const Packed &o = rows_side ? q.a : q.b;
            const int left = o.rbs - 1 - rb, there = left < 0 ? o.rbs - 1 : rb;
            most = left > 0 ? left : 0;
            if (kRows == kLying) most = most * 16 + 15;
            from = o.at + (((rows_side ? q.planes.a : q.planes.b) >> pair) & 15u) * o.plane() + o.unit(there, int64_t(tile.split) * q.split_slabs * 2 + k_unit);
            c_apart = uint32_t(o.group(there)) * uint32_t(2 * kUnitBytes);
        }
    };
    const char *base = nullptr;      // `from` in scalar registers
    auto fetch = [&](int v) {
        const int row = row_in + v * 16;
        const uint32_t place = to + uint32_t(v) * uint32_t(kUnitBytes), unit_at = uint32_t(v < most ? v : most) * pitch;
        if constexpr (kRows == kLying) fetch_unit(place, base, uint32_t(row < most ? row : most) * pitch + piece_at);
        else fetch_unit(place, base + unit_at, piece_at);
    };
    auto next_slab = [&]() {
        step();
        const uint32_t slab = uint32_t((c_at < c_last ? c_at : c_last) + (kRows == kTurned ? c_first : 0));
        uint64_t step_bytes = uint64_t(slab) * c_apart;
        if (turned) {      // the slab is a unit along the gradients' columns
            pitch = uint32_t(q.a.group(int(slab))) * uint32_t(kUnitBytes);
            step_bytes = uint64_t(q.a.unit(int(slab), c_kg));
        }
        const uint64_t at = reinterpret_cast<uint64_t>(from) + step_bytes;
        base = reinterpret_cast<const char *>(uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(int(at >> 32)))) << 32 | uint32_t(__builtin_amdgcn_readfirstlane(int(at))));
    };
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
        next_slab();
#pragma unroll
        for (int v = 0; v < kLoads; ++v) fetch(v);
    }

    // fragments, in the order in which they are wanted: the first of the weights, all rows, the other weights
    uint4 xa[2][TM], xb[2][TN];
    constexpr int kReads = TM + TN, kProducts = TM * TN;
    static_assert(kReads <= kProducts && kLoads <= kProducts, "a read and a fetch for every product");
    const int weights_at0 = weights_place(lane & 31, lane >> 5, 0), weights_at1 = weights_place(lane & 31, lane >> 5, 1);
    const AlongRows turned_at(lane, kUnitBytes);
    // kLying: of 32 rows of 64 bytes this lane's piece of the first and of the second 16 k-values
    const int row_at0 = (lane & 31) * 4 + ((lane >> 5) ^ ((lane >> 2) & 3)), row_at1 = row_at0 ^ 2;
    auto read = [&](int at, int g, int v, uint4 (&a)[TM], uint4 (&b)[TN]) {
        const uint4 *slab = &ring[at * (kUnits * 64)], *units = slab + lane, *weights = slab + (g ? weights_at1 : weights_at0);
        if (v == 0) b[0] = weights[(2 * MF + g * NF + wn * TN) * 64];
        else if (v <= TM && kRows == kLying) a[v - 1] = slab[(wm * TM + v - 1) * 128 + (g ? row_at1 : row_at0)];
        else if (v <= TM && kRows == kTurned) a[v - 1] = along_rows(slab + (wm * TM + v - 1) * 128 + g * 32, turned_at);
        else if (v <= TM) a[v - 1] = units[(g * MF + wm * TM + v - 1) * 64];
        else b[v - TM] = weights[(2 * MF + g * NF + wn * TN + v - TM) * 64];
    };
    int stage = 0, storing = 0;
    wait_and_meet<kYoung>();
    next_slab();
#pragma unroll
    for (int v = 0; v < kLoads; ++v) fetch(v);
#pragma unroll
    for (int v = 0; v < kReads; ++v) read(0, 0, v, xa[0], xb[0]);
    for (;;) {
        const WideTile tile = wide_tile(q, work);
        const int slabs = q.slabs_of(tile.split) * q.planes.count;
        floatx16 acc[TN][TM];
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[j][i][r] = 0.0f;
        auto multiply = [&](int p, const uint4 (&a)[TM], const uint4 (&b)[TN]) {
            const int j = p / TM, i = p % TM;
            acc[j][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, b[j]), __builtin_bit_cast(bf16x8, a[i]), acc[j][i], 0, 0, 0);
        };
        for (int s = 0; s < slabs; ++s) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int p = 0; p < kProducts; ++p) {
                if (p < kReads) read(stage, 1, p, xa[1], xb[1]);
                multiply(p, xa[0], xb[0]);
                __builtin_amdgcn_sched_barrier(0);
            }
            stage = stage == kStages - 1 ? 0 : stage + 1;
            next_slab();
            // the next slab is there, and all have read this one, whose place the fetches take
            if (storing > 0) wait_and_meet<kYoungStores>();
            else wait_and_meet<kYoung>();
            --storing;
#pragma unroll
            for (int p = 0; p < kProducts; ++p) {
                if (p < kReads) read(stage, 0, p, xa[0], xb[0]);
                if (p < kLoads) fetch(p);
                multiply(p, xa[1], xb[1]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        constexpr int S = Epi::kSides;
        write_out<TM, TN>(epi, acc, int64_t(tile.m) * (MF * 32) + wm * TM * 32, (tile.n * NF + wn * TN) / S * 32, tile.split, reinterpret_cast<float *>(&stages[wave][0]), lane);
        const bool whole = epi.whole(int64_t(tile.m) * (MF * 32) + MF * 32, (tile.n + 1) * NF / S * 32);
        storing = whole ? kAhead : 0;     // (fewer stores may not be counted on)
        work += stride;
        if (work >= end) break;
    }
    wait_and_meet<0>();      // (what is still on its way writes into this block's LDS)
}

}  // namespace tma
