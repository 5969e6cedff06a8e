// Tiles of the attention kernels: 32 x 32 products on the matrix cores of
// gfx950, for bf16 (v_mfma_f32_32x32x16_bf16) and fp32 (v_mfma_f32_32x32x2_f32)
// operands alike, and the ragged layout of a batch of graphs.
//
// Layouts used. A product C = A B over 32 x 32 results: lane l (m = l % 32, h =
// l / 32) supplies row m of A and column m of B. One operand piece is 16 bytes:
// 8 bf16 values (one instruction contracts 16) or 4 fp32 values (four
// instructions contract 2 each). Lane l ends with column m of C, rows
// 8 (r / 4) + 4 h + r % 4 in register r = 0 .. 15.
//
// A contraction may run over its index in any order, as long as A and B agree.
// That is used twice. Rows of a matrix (contraction over the features) are
// read as 16 consecutive bytes from feature 2 E s + E h on in step s. And a
// result C is the next product's B operand without any exchange between
// lanes: its registers, in order, are the contraction over C's rows, if A's
// columns are read in the order 8 (r / 4) + 4 h + r % 4 too.
#pragma once

#include "common.hpp"

namespace pyg {
namespace attn {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLowest = -3.402823466e38f;

template <typename T>
struct Elem;
template <>
struct Elem<__bf16> {
    static constexpr int E = 8;      // values of a 16-byte piece
    static constexpr int kSteps = 2; // pieces of a contraction over 32 rows
};
template <>
struct Elem<float> {
    static constexpr int E = 4;
    static constexpr int kSteps = 4;
};

template <typename T>
union Piece {
    uint4 u;
    T v[16 / sizeof(T)];
    bf16x8 b;
    f32x4 f;
};

// C += A B over one piece of each operand.
template <typename T>
__device__ __forceinline__ f32x16 mma(uint4 a, uint4 b, f32x16 c) {
    Piece<T> x, y;
    x.u = a;
    y.u = b;
    if constexpr (sizeof(T) == 2) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.b, y.b, c, 0, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x.f[i], y.f[i], c, 0, 0, 0);
        return c;
    }
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const bf16x2 p = __builtin_convertvector(f32x2{a, b}, bf16x2);  // one rounding to nearest even, NaN kept
    return __builtin_bit_cast(uint32_t, p);
}

// Piece u of a result's registers, as the B operand of a product over its rows.
template <typename T>
__device__ __forceinline__ uint4 piece_of(const f32x16 &c, int u) {
    if constexpr (sizeof(T) == 2) {
        return make_uint4(pack_bf16(c[8 * u], c[8 * u + 1]), pack_bf16(c[8 * u + 2], c[8 * u + 3]),
                          pack_bf16(c[8 * u + 4], c[8 * u + 5]), pack_bf16(c[8 * u + 6], c[8 * u + 7]));
    } else {
        return make_uint4(__float_as_uint(c[4 * u]), __float_as_uint(c[4 * u + 1]), __float_as_uint(c[4 * u + 2]),
                          __float_as_uint(c[4 * u + 3]));
    }
}

// Elements of one tile row in LDS: 16 bytes more than its DP features, so that
// the 16-byte pieces of consecutive rows start four banks apart.
template <typename T, int DP>
constexpr int tile_stride() {
    return DP + Elem<T>::E;
}

// Piece s of row `row` (contraction over the features).
template <typename T, int DP>
__device__ __forceinline__ uint4 row_piece(const T *tile, int row, int s, int h) {
    constexpr int E = Elem<T>::E;
    return *reinterpret_cast<const uint4 *>(tile + row * tile_stride<T, DP>() + 2 * E * s + E * h);
}

// Piece u of features d0 .. d0 + 31 of rows r0 .. r0 + 31 (contraction over the
// rows): lane m holds feature d0 + m of the rows that piece_of's registers are.
// bf16 goes through the transposing LDS read: lane i of 16 lanes names 8 bytes
// (row i / 4 of 4, features 4 (i % 4) ..) and receives feature i of all four.
template <typename T, int DP>
__device__ __forceinline__ uint4 col_piece(const T *tile, int r0, int d0, int u, int lane) {
    constexpr int S = tile_stride<T, DP>();
    const int h = lane >> 5;
    if constexpr (sizeof(T) == 2) {
        const T *p = tile + (r0 + 16 * u + 4 * h + ((lane & 15) >> 2)) * S + d0 + (lane & 16) + 4 * (lane & 3);
        typedef __attribute__((address_space(3))) short4v *lds4;
        const uint2 a = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p)));
        const uint2 b = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + 8 * S)));
        return make_uint4(a.x, a.y, b.x, b.y);
    } else {
        const T *p = tile + (r0 + 8 * u + 4 * h) * S + d0 + (lane & 31);
        return make_uint4(__float_as_uint(p[0]), __float_as_uint(p[S]), __float_as_uint(p[2 * S]),
                          __float_as_uint(p[3 * S]));
    }
}

// One 16-byte piece of a row in memory, from feature d on: zeros past D or
// where `there` is false.
template <typename T>
__device__ __forceinline__ uint4 load_piece(const T *__restrict__ row, int d, int D, bool vec, bool there) {
    constexpr int E = Elem<T>::E;
    Piece<T> p;
    p.u = make_uint4(0, 0, 0, 0);
    if (!there || d >= D) return p.u;
    if (vec) return *reinterpret_cast<const uint4 *>(row + d);
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (d + i < D) p.v[i] = row[d + i];
    return p.u;
}

// ROWS rows of a matrix, one head, held by a workgroup of NT threads between
// memory and LDS.
template <typename T, int DP, int ROWS, int NT>
struct Stage {
    static constexpr int E = Elem<T>::E, kRow = DP / E, kEach = (ROWS * kRow + NT - 1) / NT;
    static_assert(ROWS * kRow % NT == 0, "whole pieces for every thread");
    uint4 r[kEach];
    // rows first .. first + ROWS of `base`, those from `end` on are zeros
    __device__ __forceinline__ void load(const T *__restrict__ base, int64_t stride, int64_t first, int64_t end, int D,
                                         bool vec) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int p = i * NT + threadIdx.x, row = p / kRow, d = p % kRow * E;
            r[i] = load_piece<T>(base + (first + row) * stride, d, D, vec, first + row < end);
        }
    }
    __device__ __forceinline__ void store(T *tile) const {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int p = i * NT + threadIdx.x, row = p / kRow, d = p % kRow * E;
            *reinterpret_cast<uint4 *>(tile + row * tile_stride<T, DP>() + d) = r[i];
        }
    }
};

// The slots of a ragged batch cut into tiles of `tile` rows, without a pass over
// the lengths: graph g's tiles start at slot ptr[g] / tile + g. A graph of n rows
// has ceil(n / tile) <= (ptr[g] + n) / tile - ptr[g] / tile + 1 of them, so slots
// never meet; at most one a graph stays idle. The rows behind the last graph
// are graph B. slots(): how many there are.
__host__ __device__ inline int64_t slots(int64_t rows, int64_t graphs, int64_t tile) { return rows / tile + graphs + 1; }

struct Place {
    int64_t graph, first, last;  // the graph's rows
    int64_t tile;                // which of its tiles
};

// mul: rows of the batch count `mul` times (query rows of several heads in one tile).
__device__ __forceinline__ int64_t ptr_at(const int64_t *__restrict__ ptr, int64_t g, int64_t N) {
    const int64_t v = ptr[g];
    return v < 0 ? 0 : v > N ? N : v;
}
__device__ __forceinline__ Place place_of(const int64_t *__restrict__ ptr, int64_t B, int64_t N, int64_t slot, int tile,
                                          int mul, int lane) {
    int64_t lo = 0, hi = B + 1;  // graph lo's slots start at or before `slot`, graph hi's after it
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + kWave - 1) / kWave;
        const int64_t g = lo + (lane + 1) * step;
        const bool before = g < hi && ptr_at(ptr, g, N) * mul / tile + g <= slot;
        const int n = __popcll(__ballot(before));
        const int64_t nlo = lo + n * step;
        hi = nlo + step < hi ? nlo + step : hi;
        lo = nlo;
    }
    Place p;
    p.graph = uniform64(lo);
    p.first = uniform64(ptr_at(ptr, p.graph, N));
    p.last = p.graph < B ? uniform64(ptr_at(ptr, p.graph + 1, N)) : N;
    p.tile = slot - (p.first * mul / tile + p.graph);
    return p;
}

}  // namespace attn
}  // namespace pyg
