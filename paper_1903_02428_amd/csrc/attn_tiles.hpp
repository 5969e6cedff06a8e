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
    typedef uint16_t Bits;
    static constexpr int E = 8;      // values of a 16-byte piece
    static constexpr int kSteps = 2; // pieces of a contraction over 32 rows
};
template <>
struct Elem<float> {
    typedef uint32_t Bits;
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

// Whether piece s of a row holds nothing but padding: skipped where a product takes
// long (fp32: 256 cycles a piece); elsewhere the test costs more than it saves.
template <typename T>
__device__ __forceinline__ bool past(int s, int D) {
    return sizeof(T) == 4 && 2 * Elem<T>::E * s >= D;
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

// A tile of rows in LDS: rows of C chunks of 16 bytes, without padding (the
// loads to LDS write 1 KB in a row), chunk c of a row at place c ^ swizzle(row). 16
// consecutive rows then have any one chunk in 16 different groups of banks (row
// pieces), and 4 rows times 4 chunks fill the 16 groups too (the transposing reads of
// column pieces).
template <int C>
__device__ __forceinline__ int swizzle(int row) {
    if constexpr (C == 4) return (row >> 2) & 3;
    else if constexpr (C == 8) return ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
    else return (row & 3) << 2 | ((row >> 2) & 3);
}

// Hides a value from the compiler: what is derived from it is made again where it is
// used (an instruction a read) and not kept in a register across the loop.
__device__ __forceinline__ int opaque(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

template <typename T, int DP>
struct Tile {
    static constexpr int E = Elem<T>::E, C = DP / E;
    static constexpr int kRowBytes = DP * sizeof(T);
    template <int ROWS>
    static constexpr int bytes() { return ROWS * kRowBytes; }

    // A lane's place for row pieces: row m of each 32, byte offset of piece s is at(s) + 32 n rows.
    struct RowLane {
        int base, x;
        __device__ __forceinline__ explicit RowLane(int lane) {
            const int m = lane & 31, h = lane >> 5;
            base = m * kRowBytes, x = (h ^ swizzle<C>(m)) << 4;
        }
    };
    static __device__ __forceinline__ uint4 row_piece(const char *tile, const RowLane &l, int n, int s) {
        return *reinterpret_cast<const uint4 *>(tile + l.base + (l.x ^ (2 * s << 4)) + 32 * n * kRowBytes);
    }

    // A lane's place for column pieces. bf16 goes through the transposing LDS read:
    // lane i of 16 lanes names 8 bytes (row i / 4 of 4, features 4 (i % 4) ..) and
    // receives feature i of all four.
    struct ColLane {
        int base, x, lane;
        __device__ __forceinline__ explicit ColLane(int lane_) : lane(lane_) {
            const int h = lane >> 5;
            if constexpr (sizeof(T) == 2) {
                const int row = 4 * h + ((lane & 15) >> 2);
                base = row * kRowBytes + (lane & 1) * 8;
                x = (((lane & 16) >> 3 | (lane & 3) >> 1) ^ swizzle<C>(row)) << 4;
            } else {
                base = 4 * h * kRowBytes + (lane & 3) * 4;
                x = ((lane & 31) >> 2 ^ h) << 4;  // swizzle of row 4 h + i + 8 u: h, and what i and u add
            }
        }
    };
    // Piece u of features 32 t .. of rows 32 n .. (contraction over the rows).
    static __device__ __forceinline__ uint4 col_piece(const char *tile, const ColLane &l, int n, int t, int u) {
        if constexpr (sizeof(T) == 2) {
            const char *p = tile + l.base + (32 * n + 16 * u) * kRowBytes;
            const int x = l.x ^ (t * 4 << 4);
            typedef __attribute__((address_space(3))) short4v *lds4;
            const uint2 a = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + x)));
            const uint2 b = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + 8 * kRowBytes + (x ^ 32))));
            return make_uint4(a.x, a.y, b.x, b.y);
        } else {
            const char *p = tile + l.base + (32 * n + 8 * u) * kRowBytes;
            uint32_t v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int add = swizzle<C>(i) ^ (u & 1) << 1 ^ t * 8;  // (row >> 2) & 3 = h + 2 (u & 1)
                v[i] = *reinterpret_cast<const uint32_t *>(p + i * kRowBytes + (l.x ^ add << 4));
            }
            return make_uint4(v[0], v[1], v[2], v[3]);
        }
    }
};

// One 16-byte piece of a row in memory, from feature d on: zeros past D or
// where `there` is false. Rows may start at any element (vector loads from memory
// need no alignment here); the last piece of an odd width goes value by value.
template <typename T>
__device__ __forceinline__ uint4 load_piece(const T *__restrict__ row, int d, int D, bool there) {
    constexpr int E = Elem<T>::E;
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    typedef u32x4 __attribute__((aligned(2))) any;
    if (there && d + E <= D) {
        const u32x4 v = *reinterpret_cast<const any *>(row + d);
        return make_uint4(v[0], v[1], v[2], v[3]);
    }
    uint64_t lo = 0, hi = 0;
    if (there) {
        typedef typename Elem<T>::Bits Bits;
#pragma unroll 1
        for (int i = 0; d + i < D; ++i) {
            const uint64_t b = static_cast<uint64_t>(reinterpret_cast<const Bits *>(row)[d + i]) << (8 * sizeof(T) * (i % (E / 2)));
            (i < E / 2 ? lo : hi) |= b;
        }
    }
    return make_uint4(static_cast<uint32_t>(lo), static_cast<uint32_t>(lo >> 32), static_cast<uint32_t>(hi),
                      static_cast<uint32_t>(hi >> 32));
}

// A lane's row as operand pieces (features 2 E s + E h .. in piece s); `row` can be
// read in any case, `there` says whether it counts. Widths of whole pieces are read without a branch, so
// that all loads are under way together.
template <typename T, int N>
__device__ __forceinline__ void load_row(const T *__restrict__ row, int D, bool there, int h, uint4 (&p)[N]) {
    constexpr int E = Elem<T>::E;
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    typedef u32x4 __attribute__((aligned(2))) any;
    if (D % E == 0) {
        u32x4 v[N];
#pragma unroll
        for (int s = 0; s < N; ++s) {
            const int d = 2 * E * s + E * h;
            v[s] = *reinterpret_cast<const any *>(row + (d < D ? d : 0));
        }
#pragma unroll
        for (int s = 0; s < N; ++s)
            p[s] = there && 2 * E * s + E * h < D ? make_uint4(v[s][0], v[s][1], v[s][2], v[s][3]) : make_uint4(0, 0, 0, 0);
        return;
    }
#pragma unroll
    for (int s = 0; s < N; ++s) p[s] = load_piece<T>(row, 2 * E * s + E * h, D, there);
}

// ROWS rows of one head, from memory to an LDS tile by a workgroup of NT
// threads. 16-byte rows (vec) go without passing registers
// (buffer_load_dwordx4 .. lds: 64 lanes write 1 KB in a row): the swizzle is in which
// chunk a lane asks for, and rows past the end and features past D lie outside
// the buffer, which reads as zeros. Other rows pass registers.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint32_t to_scalar(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ uint32_t lds_offset(const char *p) {
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char *)(p)));
}
// 16 bytes a lane from the buffer's byte `off` to LDS bytes lds + 16 lane. In
// assembly because the compiler, which cannot tell the halves of the LDS apart, makes
// every LDS read wait for all such loads; loads_done() waits for them where it is
// due, ahead of the barrier that hands the tile over.
__device__ __forceinline__ void load_to_lds(const u32x4 &rsrc, uint32_t off, uint32_t lds) {
    // m0 is the compiler's (it takes no clobber of it) and gets its value back; the load has read it when it was issued
    uint32_t m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0\n\ts_nop 0"
                 : "=&s"(m0)
                 : "s"(lds), "v"(off), "s"(rsrc)
                 : "memory");
}
__device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
// Ahead of a loop with such loads: the wavefront's own loads into registers arrive now, and the
// compiler knows (vmcnt 0), or the loop's first use of one would wait in every round.
__device__ __forceinline__ void registers_loaded() {
    __builtin_amdgcn_s_waitcnt(0x0F70);
    asm volatile("" ::: "memory");
}

constexpr uint32_t kOutside = 0x80000000u;
constexpr int64_t kMaxRowStride = 1 << 22;  // in elements: 64 rows stay below kOutside

template <typename T, int DP, int ROWS, int NT>
struct Stage {
    using L = Tile<T, DP>;
    static constexpr int E = L::E, C = L::C, kEach = ROWS * C / NT;
    static_assert(ROWS * C % NT == 0, "whole pieces for every thread");
    uint32_t row_bytes;
    int D;
    bool vec;
    __device__ __forceinline__ Stage(int64_t stride, int D_, bool vec_) : row_bytes(stride * sizeof(T)), D(D_), vec(vec_) {}
    // rows first .. of `head` (a [rows] array of this head's features); there are `left` of them
    __device__ __forceinline__ void load(const T *head, int64_t first, int64_t left, char *tile) const {
        const T *base = head + first * (row_bytes / sizeof(T));
        const int rows = left < ROWS ? static_cast<int>(left) : ROWS;
        if (vec) {
            const uint64_t at = reinterpret_cast<uint64_t>(base);
            const u32x4 rsrc{to_scalar(static_cast<uint32_t>(at)), to_scalar(static_cast<uint32_t>(at >> 32) & 0xFFFFu),
                             to_scalar(rows * row_bytes), 0x00020000u};
            const uint32_t wave = to_scalar(lds_offset(tile) + (threadIdx.x >> 6) * 1024u);
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int p = i * NT + threadIdx.x, row = p / C, d = ((p % C) ^ swizzle<C>(row)) * E;
                load_to_lds(rsrc, d < D ? row * row_bytes + d * sizeof(T) : kOutside, wave + i * NT * 16u);
            }
        } else {
#pragma unroll 1
            for (int p = threadIdx.x; p < ROWS * C; p += NT) {
                const int row = p / C, d = ((p % C) ^ swizzle<C>(row)) * E;
                *reinterpret_cast<uint4 *>(tile + p * 16) =
                    load_piece<T>(base + (int64_t)row * (row_bytes / sizeof(T)), d, D, row < rows);
            }
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

__device__ __forceinline__ int64_t ptr_at(const int64_t *__restrict__ ptr, int64_t g, int64_t N) {
    const int64_t v = ptr[g];
    return v < 0 ? 0 : v > N ? N : v;
}
// Where a slot lies. mul: rows of the batch count `mul` times (query rows of several heads in one tile).
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
