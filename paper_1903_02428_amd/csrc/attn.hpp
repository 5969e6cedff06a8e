// What the attention kernels share: the call's arguments, the bias by relative
// position, masks and the scores of a 32 x 32 tile.
//
// The scores are a_ij = c q_i . k_j + T[bucket(j - i'), h], with i' = i + nk - nq.
// They are held as s = a / c: the bias over c is what a bf16 tile's accumulators
// start from, so that the matrix cores add it (fp32 tiles add it last), and far from the diagonal, where
// one bucket holds all offsets, it costs nothing. p = exp(a - max) is then
// exp2(c2 (s - m)), c2 = c log2(e).
#pragma once

#include "attn_tiles.hpp"

namespace pyg {
namespace attn {

struct Args {
    const int64_t *q_ptr, *k_ptr;  // [B + 1]
    int64_t B, Nq, Nk;
    int H, Hkv, G, D;  // G = H / Hkv query heads share a key head
    int64_t q_row, q_head, k_row, k_head, v_row, v_head;  // strides in elements
    float scale, inv_scale, c2;
    bool causal, vec_q, vec_k, vec_v, vec_o, zero_rest;
    const void *table;    // [buckets, H] in the operands' type, or NULL
    const int32_t *lut;   // [2 * reach + 1]
    int buckets, reach;
    const void *q, *k, *v;
    void *out;
    void *rest;   // [Nq, H, D], bf16 only: what rounding took from out, itself rounded; or NULL
    float *stat;  // [Nq, H, 2]: the row's largest s, log2 of its sum of exp2(c2 (s - m)); or NULL
};

constexpr int kMaxReach = 1024;  // the sums by offset of four wavefronts fit the LDS beside the widest tiles

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__bf16 v) { return static_cast<float>(v); }

// The bias over c of every offset, for head h, in LDS. Finite values stay
// finite: a table entry of the type's lowest value masks without leaving the
// row empty, as it does in the formula.
// Returns, in every thread and after a barrier, whether any of it is so large that
// c2 s - c2 m in one fused multiply-add leaves more than the exponent's own
// rounding (tables of lowest values): s - m has to come first then.
constexpr float kWild = 65536.f;
template <typename T>
__device__ __forceinline__ bool stage_bias(const Args &a, int h, float *bias, int *buckets = nullptr) {
    int wild = 0;
    const T *t = static_cast<const T *>(a.table);
    for (int o = threadIdx.x; o <= 2 * a.reach; o += blockDim.x) {
        float v = 0.f;
        if (t) {
            int b = a.lut[o];
            b = b < 0 ? 0 : b >= a.buckets ? a.buckets - 1 : b;
            if (buckets) buckets[o] = b;
            const float raw = to_f32(t[(int64_t)b * a.H + h]);
            v = raw * a.inv_scale;
            if (fabsf(raw) <= -kLowest) v = fminf(fmaxf(v, kLowest), -kLowest);
        }
        bias[o] = v;
        wild |= fabsf(v) > kWild && fabsf(v) <= -kLowest;
    }
    return __syncthreads_or(wild) != 0;
}

// Whether the offsets first .. last all lie in an end bucket, and none is masked.
__device__ __forceinline__ bool flat(int first, int last, int reach, bool causal) {
    return last <= -reach || (first >= reach && !causal);
}

// The bias over c of offset d (key minus query) for head h, from memory, as stage_bias() makes it.
template <typename T>
__device__ __forceinline__ float bias_of(const Args &a, int h, int64_t d) {
    if (!a.table) return 0.f;
    int b = a.lut[d < -a.reach ? 0 : d > a.reach ? 2 * a.reach : static_cast<int>(d) + a.reach];
    b = b < 0 ? 0 : b >= a.buckets ? a.buckets - 1 : b;
    const float raw = to_f32(static_cast<const T *>(a.table)[(int64_t)b * a.H + h]);
    return fabsf(raw) <= -kLowest ? fminf(fmaxf(raw * a.inv_scale, kLowest), -kLowest) : raw * a.inv_scale;
}
// The other half's value of the same column (lanes l and l ^ 32).
__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

// A count or an offset in 32 bits: beyond 2^30 only its side matters.
__device__ __forceinline__ int near(int64_t v) {
    constexpr int64_t most = int64_t(1) << 30;
    return static_cast<int>(v < -most ? -most : v > most ? most : v);
}

// Start of a 32 x 32 tile of scores whose lane holds column offset `col` and
// rows 8 (r / 4) + 4 h + r % 4, offsets (key minus query) d0 + SIGN-ed index:
// KEYS_IN_ROWS: rows are keys, the lane's column a query: d = d0 + row - m;
// else rows are queries and the column a key: d = d0 + m - row.
template <bool KEYS_IN_ROWS>
__device__ __forceinline__ f32x16 bias_tile(const float *bias, int reach, int d0, int lane) {
    f32x16 c;
    // offsets of the tile: d0 - 31 .. d0 + 31
    if (d0 - 31 >= reach || d0 + 31 <= -reach) {
        const float v = bias[d0 > 0 ? 2 * reach : 0];
#pragma unroll
        for (int r = 0; r < 16; ++r) c[r] = v;
        return c;
    }
    lane = opaque(lane);  // near the diagonal only: nothing of this is kept in registers for it
    const int m = lane & 31, h = lane >> 5, base = d0 + reach + (KEYS_IN_ROWS ? 4 * h - m : m - 4 * h);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int row = 8 * (r >> 2) + (r & 3);
        int o = KEYS_IN_ROWS ? base + row : base - row;
        o = o < 0 ? 0 : o > 2 * reach ? 2 * reach : o;
        c[r] = bias[o];
    }
    return c;
}

// The same added to scores that are there already (fp32: products begun from a bias would round every partial sum at
// its magnitude; bf16 ones take an eighth of the additions and have 16 bits less to lose).
template <typename T>
constexpr bool kBiasLate = sizeof(T) == 4;
template <bool KEYS_IN_ROWS>
__device__ __forceinline__ void add_bias(f32x16 &c, const float *bias, int reach, int d0, int lane) {
    lane = opaque(lane);
    const int m = lane & 31, h = lane >> 5, base = d0 + reach + (KEYS_IN_ROWS ? 4 * h - m : m - 4 * h);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int row = 8 * (r >> 2) + (r & 3);
        int o = KEYS_IN_ROWS ? base + row : base - row;
        o = o < 0 ? 0 : o > 2 * reach ? 2 * reach : o;
        c[r] += bias[o];
    }
}

// -infinity where there is no such key (rows from `keys` on) or it comes later
// than the query (causal, offset > 0); in the backward `none` for dP there, whatever it is.
template <bool KEYS_IN_ROWS, bool BACKWARD = false>
__device__ __forceinline__ void mask_tile(f32x16 &c, int keys, int queries, bool causal, int d0, int lane, f32x16 *dp = nullptr,
                                          float none = 0.f) {
    if (keys >= 32 && queries >= 32 && (!causal || d0 + 31 <= 0)) return;
    lane = opaque(lane);
    const int m = lane & 31, h = lane >> 5;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int row = 8 * (r >> 2) + 4 * h + (r & 3);
        const int key = KEYS_IN_ROWS ? row : m, query = KEYS_IN_ROWS ? m : row;
        if (key >= keys || query >= queries || (causal && d0 + key - query > 0)) {
            c[r] = kNegInf;
            if constexpr (BACKWARD) (*dp)[r] = none;
        }
    }
}

// Rows [first, last) of a [N, H, D] output, head h, get zeros (rows of no graph).
template <typename T>
__device__ __forceinline__ void zero_rows(T *out, int64_t first, int64_t last, int H, int h, int D) {
    const int64_t n = (last - first) * D;
    for (int64_t i = threadIdx.x; i < n; i += blockDim.x) {
        const int64_t row = first + i / D;
        out[(row * H + h) * D + i % D] = T(0.f);
    }
}

// out[row, head h] from a wavefront's D x 32 result (lane: column = row, registers = features), times `mul`.
// REST: what the results lose to the type's rounding instead.
template <typename T, int DP, bool REST = false>
__device__ __forceinline__ void store_rows(T *out, int64_t row, bool there, int H, int h, int D, bool vec,
                                           const f32x16 (&acc)[DP / 32], float mul, int lane) {
    if (!there) return;
    T *o = out + (row * H + h) * D;
    const auto value = [&](float v) { return REST ? v * mul - to_f32(T(v * mul)) : v * mul; };
    const int hh = lane >> 5;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int d = 32 * t + 8 * r + 4 * hh;
            if (d >= D) continue;
            const float v0 = value(acc[t][4 * r]), v1 = value(acc[t][4 * r + 1]), v2 = value(acc[t][4 * r + 2]),
                        v3 = value(acc[t][4 * r + 3]);
            if (vec) {
                if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2 *>(o + d) = make_uint2(pack_bf16(v0, v1), pack_bf16(v2, v3));
                else *reinterpret_cast<float4 *>(o + d) = make_float4(v0, v1, v2, v3);
            } else {
                const float v[4] = {v0, v1, v2, v3};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (d + i < D) o[d + i] = T(v[i]);
            }
        }
}

// ---- Causal calls whose later keys (or, for the keys' gradients, earlier queries) are not finite. Their weights are 0,
// but 0 times them is NaN in the matrix cores, for every row of the tile that crosses the diagonal. The tile loops
// let that happen: a wavefront that ends with results that are not finite looks whether they ought to be, and makes those
// anew, value by value, that see nothing but finite ones. (Looking through the tiles in the loops made the
// forward 4 to 14 % slower, without any such value; this takes nothing.)

// The kernel's first argument from memory: what is read through it is not kept in scalar registers through the loops.
template <typename A = Args>
__device__ __forceinline__ const A &args_again() {
    auto p = __builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *reinterpret_cast<const A *>((const void *)(p));
}

__device__ __forceinline__ bool finite(float v) { return fabsf(v) <= -kLowest; }
// Whether a word of two bf16 values or one fp32 value holds one that is not finite.
template <typename T>
__device__ __forceinline__ bool not_finite(uint32_t w) {
    return (w & 0x7F800000u) == 0x7F800000u || (sizeof(T) == 2 && (w & 0x7F80u) == 0x7F80u);
}
template <typename T>
__device__ __forceinline__ bool row_finite(const T *__restrict__ row, int D) {
    bool fine = true;
#pragma unroll 2
    for (int d = 0; d < D; d += Elem<T>::E) {
        const uint4 p = load_piece<T>(row, d, D, true);
        fine = fine && !(not_finite<T>(p.x) || not_finite<T>(p.y) || not_finite<T>(p.z) || not_finite<T>(p.w));
    }
    return fine;
}

// Whether any of the results of a lane's column is not finite.
template <int N>
__device__ __forceinline__ bool column_odd(const f32x16 (&acc)[N]) {
    float t = 0.f;  // 0 times each
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) t = fmaf(acc[i][r], 0.f, t);
    t += other_half(t);
    return t != t;
}

// Of the lanes with `flag`, those for which no row of first .. last that they see (seen(row)) fails fine(row), a lane a row.
template <typename FINE, typename SEEN>
__device__ __forceinline__ bool sees_only_fine(bool flag, int64_t first, int64_t last, int lane, FINE fine, SEEN seen) {
#pragma unroll 1
    for (int64_t j = first; j < last && __any(flag); j += kWave) {
        uint64_t odd = __ballot(j + lane < last && !fine(j + lane));
        for (; odd && __any(flag); odd &= odd - 1) flag = flag && !seen(j + __ffsll(static_cast<unsigned long long>(odd)) - 1);
    }
    return flag;
}

template <typename T>
__device__ __forceinline__ float row_dot(const T *__restrict__ x, const T *__restrict__ y, int D) {
    float t = 0.f;
#pragma unroll 4
    for (int d = 0; d < D; d += Elem<T>::E) {
        Piece<T> p, q;
        p.u = load_piece<T>(x, d, D, true), q.u = load_piece<T>(y, d, D, true);
#pragma unroll
        for (int e = 0; e < Elem<T>::E; ++e) t = fmaf(to_f32(p.v[e]), to_f32(q.v[e]), t);
    }
    return t;
}

// Features d .. d + 3 of a row, zeros past D.
template <typename T>
__device__ __forceinline__ void load_four(const T *__restrict__ row, int d, int D, float (&v)[4]) {
    typedef T four __attribute__((ext_vector_type(4)));
    typedef four __attribute__((aligned(2))) any;
    if (d + 4 <= D) {
        const four x = *reinterpret_cast<const any *>(row + d);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = to_f32(x[i]);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = d + i < D ? to_f32(row[d + i]) : 0.f;
}

// o += w row, a lane's features: 32 t + 8 (r / 4) + 4 h + r % 4 in o[t][r]. Nothing where w is 0, whatever the row holds.
template <typename T, int DP>
__device__ __forceinline__ void add_row(f32x16 (&o)[DP / 32], const T *__restrict__ row, float w, int D, int lane) {
    w = to_f32(T(w));  // as the matrix cores take it
    const int first = opaque(4 * (lane >> 5));
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int d = first + 32 * t + 8 * q;
            float v[4];
            load_four(row, d, D, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[t][4 * q + i] = w != 0.f ? fmaf(w, v[i], o[t][4 * q + i]) : o[t][4 * q + i];
        }
}

int forward(const Args &a, bool bf16, hipStream_t s);
// The same where a graph has few queries: its keys cut into few_splits() ranges.
int few_splits(const Args &a);
int forward_few(const Args &a, bool bf16, void *ws, hipStream_t s);

struct BackwardArgs {
    Args f;  // out: the forward's result
    const void *grad_out;
    void *grad_q, *grad_k, *grad_v, *grad_table;  // NULL: not wanted (grad_k and grad_v together)
};
// Which gradients are wanted.
struct Wanted {
    bool q, kv, table;
};
size_t backward_workspace(const Args &a, const Wanted &w);
int backward(const BackwardArgs &a, bool bf16, void *ws, hipStream_t s);

}  // namespace attn
}  // namespace pyg
