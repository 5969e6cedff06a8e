// Attention of few queries a graph over many keys (a readout, one new node
// over a long history): forward.
//
// Bound by reading K and V once. The query rows that share a key head (nq * G
// of them) make 16-row tiles of v_mfma_f32_16x16x32_bf16 / 16x16x4_f32; the keys
// are cut into S ranges a graph so that a handful of rows fills the card, and
// the ranges' maxima, sums and outputs are joined by k_join. K and V go from
// memory to registers as the matrix cores take them, without LDS: S^T = K Q^T reads a
// key's features as 16-byte pieces, and O^T = V^T P^T lets lane m hold features m W
// .. m W + W - 1 (W = DP / 16) of its keys, so that each of the W result tiles
// takes every lane's t-th feature (bf16: two keys' values joined by one byte
// permute).
//
// 16 x 16 layouts: lane l (m = l % 16, g = l / 16) supplies row m of A, column m
// of B: 8 contraction values 8 g .. (bf16), one value g (fp32); the result's
// register r is row 4 g + r, column m.
#include "attn.hpp"

namespace pyg {
namespace attn {
namespace {

template <typename T, int DP>
struct Few {
    static constexpr bool kBf16 = sizeof(T) == 2;
    static constexpr int SUB = kBf16 ? 2 : 1;        // 16-key tiles a step
    static constexpr int KEYS = 16 * SUB;
    static constexpr int E = 16 / sizeof(T);
    static constexpr int STEPS = DP / (4 * E);       // 16-byte pieces of a row
    static constexpr int W = DP / 16;
    static constexpr int VW = (W * sizeof(T) + 3) / 4;  // registers of a lane's W features
};

// N words at any element's address.
template <int N>
struct Words {
    typedef uint32_t U __attribute__((ext_vector_type(N)));
    typedef U __attribute__((aligned(2))) type;
};
template <>
struct Words<1> {
    typedef uint32_t U __attribute__((ext_vector_type(1)));
    typedef U __attribute__((aligned(2))) type;
};
template <int N>
using Any = typename Words<N>::type;

template <typename T, int DP>
struct FewTile {
    using F = Few<T, DP>;
    uint4 k[F::SUB][F::STEPS];
    uint32_t v[4 * F::SUB][F::VW];

    // keys j .. j + KEYS of the graph, those from `end` on are zeros
    __device__ __forceinline__ void load(const Args &a, const T *__restrict__ kb, const T *__restrict__ vb, int64_t j,
                                         int64_t end, int lane) {
        const int m = lane & 15, g = lane >> 4;
        if (a.D % F::E == 0 && a.D % F::W == 0) {
            // without a branch, so that all loads are under way together: keys past the end are the last one again,
            // features past D the first ones; clear() takes them out where they would count
            const int64_t last = end - 1;
            const int d = m * F::W < a.D ? m * F::W : 0;
#pragma unroll
            for (int u = 0; u < F::SUB; ++u) {
                const int64_t key = j + 16 * u + m, safe = key < end ? key : last;
#pragma unroll
                for (int s = 0; s < F::STEPS; ++s) {
                    const int f = 4 * F::E * s + F::E * g;
                    const auto x = *reinterpret_cast<const Any<4> *>(kb + safe * a.k_row + (f < a.D ? f : 0));
                    k[u][s] = make_uint4(x[0], x[1], x[2], x[3]);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int64_t vkey = j + 16 * u + 4 * g + r;
                    const T *p = vb + (vkey < end ? vkey : last) * a.v_row + d;
                    constexpr int N = F::VW >= 4 ? 4 : F::VW;
#pragma unroll
                    for (int i = 0; i < F::VW; i += N) {
                        const auto x = *reinterpret_cast<const Any<N> *>(p + i * 4 / sizeof(T));
#pragma unroll
                        for (int n = 0; n < N; ++n) v[4 * u + r][i + n] = x[n];
                    }
                }
            }
            return;
        }
#pragma unroll
        for (int u = 0; u < F::SUB; ++u) {
            const int64_t key = j + 16 * u + m;
#pragma unroll
            for (int s = 0; s < F::STEPS; ++s)
                k[u][s] = load_piece<T>(kb + key * a.k_row, 4 * F::E * s + F::E * g, a.D, key < end);
#pragma unroll
            for (int r = 0; r < 4; ++r) row(a, vb, j + 16 * u + 4 * g + r, end, m, v[4 * u + r]);
        }
    }
    // What load() put in the place of nothing, to zeros before it is used: 0 times an infinity would be NaN. (K past the
    // end is masked, features of V past D are not kept.)
    __device__ __forceinline__ void clear(const Args &a, int64_t j, int64_t end, int lane) {
        const int g = lane >> 4;
        if (a.D < DP) {
#pragma unroll
            for (int s = 0; s < F::STEPS; ++s)
                if (4 * F::E * s + F::E * g >= a.D)
#pragma unroll
                    for (int u = 0; u < F::SUB; ++u) k[u][s] = make_uint4(0, 0, 0, 0);
        }
        if (j + F::KEYS > end) {
#pragma unroll
            for (int u = 0; u < F::SUB; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (j + 16 * u + 4 * g + r >= end)
#pragma unroll
                        for (int i = 0; i < F::VW; ++i) v[4 * u + r][i] = 0;
        }
    }
    __device__ __forceinline__ void row(const Args &a, const T *__restrict__ vb, int64_t key, int64_t end, int m,
                                        uint32_t (&o)[F::VW]) {
#pragma unroll
        for (int i = 0; i < F::VW; ++i) o[i] = 0;
        const int d = m * F::W;
        if (key >= end || d >= a.D) return;
        const T *p = vb + key * a.v_row + d;
#pragma unroll
        for (int i = 0; i < F::W; ++i) {
            if (d + i >= a.D) break;
            if constexpr (F::kBf16) {
                const uint32_t x = reinterpret_cast<const uint16_t *>(p)[i];
                o[i / 2] |= i & 1 ? x << 16 : x;
            } else {
                o[i] = reinterpret_cast<const uint32_t *>(p)[i];
            }
        }
    }
};

constexpr int kFewWaves = 4;

template <typename T>
__device__ __forceinline__ void put(const Args &a, int64_t at, float v) {
    const T r = T(v);
    static_cast<T *>(a.out)[at] = r;
    if constexpr (sizeof(T) == 2)
        if (a.rest) static_cast<T *>(a.rest)[at] = T(v - to_f32(r));
}

// Of a wavefront's results, before they are divided by the sums, the rows that are not finite (flag) though they see
// nothing but finite values among the workgroup's keys (attn.hpp).
template <typename T, int DP>
__device__ __forceinline__ void repair(int64_t nslots, int splits, float top, bool flag, f32x4 (&acc)[DP / 16]) {
    using F = Few<T, DP>;
    const Args &a = args_again();
    const int lane = opaque(threadIdx.x & 63), wave = to_scalar(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
    const uint32_t id = opaque(blockIdx.x);
    const int hk = to_scalar(id % a.Hkv), sp = to_scalar(id / a.Hkv % splits);
    const Place p = place_of(a.q_ptr, a.B, a.Nq, to_scalar(id / a.Hkv / splits), 16, a.G, lane);
    const int64_t k_first = uniform64(ptr_at(a.k_ptr, p.graph, a.Nk)), k_last = uniform64(ptr_at(a.k_ptr, p.graph + 1, a.Nk));
    const int64_t nk = k_last > k_first ? k_last - k_first : 0, nq = p.last - p.first, rr = p.tile * 16 + m;
    const bool there = rr < nq * a.G;
    const int64_t i = there ? rr / a.G : 0, shift = i + nk - nq;
    const int head = hk * a.G + static_cast<int>(rr % a.G);
    const T *k = static_cast<const T *>(a.k) + k_first * a.k_row + hk * a.k_head;
    const T *v = static_cast<const T *>(a.v) + k_first * a.v_row + hk * a.v_head;
    const T *q = static_cast<const T *>(a.q) + (p.first + i) * a.q_row + head * a.q_head;
    const int64_t len = (nk + splits - 1) / splits, begin = len * sp, end = begin + len < nk ? begin + len : nk;
    flag = sees_only_fine(flag && there, begin, end, lane, [&](int64_t j) {
        return row_finite(k + j * a.k_row, a.D) && row_finite(v + j * a.v_row, a.D);
    }, [&](int64_t j) { return j <= shift; });
    if (!__any(flag)) return;
    f32x4 o[F::W];
#pragma unroll
    for (int t = 0; t < F::W; ++t) o[t] = f32x4(0.f);
#pragma unroll 1
    for (int64_t j = begin + wave * F::KEYS; j < end; j += (j - begin + 1) % F::KEYS ? 1 : (kFewWaves - 1) * F::KEYS + 1) {  // the wavefront's own
        const bool seen = flag && j <= shift;
        if (!__any(seen)) continue;
        const float s = row_dot(q, k + j * a.k_row, a.D) + bias_of<T>(a, head, j - shift);
        const float w = to_f32(T(seen ? __builtin_amdgcn_exp2f(a.c2 * (s - top)) : 0.f));  // as the matrix cores take it
        const int first = opaque(4 * g * F::W);
#pragma unroll
        for (int t = 0; t < F::W; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = first + r * F::W + t;
                const float x = to_f32(v[j * a.v_row + (d < a.D ? d : 0)]);  // past D: not kept
                o[t][r] = w != 0.f ? fmaf(w, x, o[t][r]) : o[t][r];
            }
    }
#pragma unroll
    for (int t = 0; t < F::W; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[t][r] = flag ? o[t][r] : acc[t][r];
}

template <typename T, int DP>
__global__ __launch_bounds__(64 * kFewWaves, 2) void k_few(const Args a, int64_t nslots, int splits, float *__restrict__ part) {
    using F = Few<T, DP>;
    constexpr int W = F::W;
    __shared__ float lo[kFewWaves][16][DP + 1];
    __shared__ float lt[kFewWaves][16], ls[kFewWaves][16];
    const int lane = threadIdx.x & 63, wave = to_scalar(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
    const int64_t id = blockIdx.x;
    const int hk = id % a.Hkv;
    const int sp = static_cast<int>(id / a.Hkv % splits);
    const int64_t slot = id / a.Hkv / splits;
    const Place p = place_of(a.q_ptr, a.B, a.Nq, slot, 16, a.G, lane);
    if (p.tile < 0) return;
    const int64_t rows = (p.last - p.first) * a.G, r0 = p.tile * 16;
    if (r0 >= rows) return;
    T *out = static_cast<T *>(a.out);
    const int64_t rr = r0 + m;  // the lane's row: query rr / G, head rr % G of the key head's
    const bool there = rr < rows;
    const int64_t row = p.first + rr / a.G;
    const int head = hk * a.G + static_cast<int>(rr % a.G);
    if (p.graph == a.B) {
        if (a.zero_rest && sp == 0 && threadIdx.x < 16 && there)
            for (int d = 0; d < a.D; ++d) out[(row * a.H + head) * a.D + d] = T(0.f);
        return;
    }
    const int64_t k_first = uniform64(ptr_at(a.k_ptr, p.graph, a.Nk)),
                  k_last = uniform64(ptr_at(a.k_ptr, p.graph + 1, a.Nk));
    const int64_t nk = k_last > k_first ? k_last - k_first : 0, nq = p.last - p.first;
    const T *kb = static_cast<const T *>(a.k) + k_first * a.k_row + hk * a.k_head;
    const T *vb = static_cast<const T *>(a.v) + k_first * a.v_row + hk * a.v_head;
    const T *qr = static_cast<const T *>(a.q) + row * a.q_row + head * a.q_head;
    uint4 qf[F::STEPS];
#pragma unroll
    for (int s = 0; s < F::STEPS; ++s) qf[s] = load_piece<T>(qr, 4 * F::E * s + F::E * g, a.D, there);

    // the range of this workgroup's keys
    const int64_t len = (nk + splits - 1) / splits, begin = len * sp;
    const int64_t end = begin + len < nk ? begin + len : nk;
    const int64_t shift = rr / a.G + nk - nq;  // offset of key j and the lane's query: j - shift
    const bool biased = a.table && there;
    const float far = biased ? bias_of<T>(a, head, -a.reach) : 0.f;

    f32x4 acc[W];
#pragma unroll
    for (int t = 0; t < W; ++t) acc[t] = f32x4(0.f);
    float top = kNegInf, sum = 0.f;
    FewTile<T, DP> cur, next;
    int64_t j = begin + wave * F::KEYS;
    if (j < end) cur.load(a, kb, vb, j, end, lane);
    for (; j < end; j += kFewWaves * F::KEYS) {
        if (j + kFewWaves * F::KEYS < end) next.load(a, kb, vb, j + kFewWaves * F::KEYS, end, lane);
        cur.clear(a, j, end, lane);
        f32x4 s[F::SUB];
        // all offsets of the tile at or below -reach, for all of the wavefront's rows
        const bool is_far = j + F::KEYS - 1 - (r0 / a.G + nk - nq) <= -a.reach;
#pragma unroll
        for (int u = 0; u < F::SUB; ++u) {
            s[u] = f32x4(0.f);
#pragma unroll
            for (int i = 0; i < F::STEPS; ++i) {
                Piece<T> x, y;
                x.u = cur.k[u][i];
                y.u = qf[i];
                if constexpr (F::kBf16) {
                    s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.b, y.b, s[u], 0, 0, 0);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.f[e], y.f[e], s[u], 0, 0, 0);
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t key = j + 16 * u + 4 * g + r;
                s[u][r] += !biased ? 0.f : is_far ? far : bias_of<T>(a, head, key - shift);
                if (key >= end || (a.causal && key > shift)) s[u][r] = kNegInf;
            }
        }
        float t = kNegInf;
#pragma unroll
        for (int u = 0; u < F::SUB; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r) t = fmaxf(t, s[u][r]);
        t = fmaxf(t, __shfl_xor(t, 16));
        t = fmaxf(t, __shfl_xor(t, 32));
        const float top_new = fmaxf(top, t), ref = top_new == kNegInf ? 0.f : top_new;
        const float shrink = __builtin_amdgcn_exp2f(a.c2 * (top - ref));
        top = top_new;
        sum *= shrink;
#pragma unroll
        for (int i = 0; i < W; ++i) acc[i] *= shrink;
#pragma unroll
        for (int u = 0; u < F::SUB; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[u][r] = __builtin_amdgcn_exp2f(a.c2 * (s[u][r] - ref));
                sum += s[u][r];
            }
        if constexpr (F::kBf16) {
            Piece<T> pp;  // P rounded to bf16, as in the tiled forward
            pp.u = make_uint4(pack_bf16(s[0][0], s[0][1]), pack_bf16(s[0][2], s[0][3]), pack_bf16(s[1][0], s[1][1]),
                              pack_bf16(s[1][2], s[1][3]));
#pragma unroll
            for (int i = 0; i < W; ++i) {
                Piece<T> x;
                const uint32_t sel = i & 1 ? 0x07060302u : 0x05040100u;  // the high or low halves of two keys
                x.u = make_uint4(__builtin_amdgcn_perm(cur.v[1][i / 2], cur.v[0][i / 2], sel),
                                 __builtin_amdgcn_perm(cur.v[3][i / 2], cur.v[2][i / 2], sel),
                                 __builtin_amdgcn_perm(cur.v[5][i / 2], cur.v[4][i / 2], sel),
                                 __builtin_amdgcn_perm(cur.v[7][i / 2], cur.v[6][i / 2], sel));
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.b, pp.b, acc[i], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(cur.v[r][i]), s[0][r], acc[i], 0, 0, 0);
        }
        cur = next;
    }
    if (a.causal) {
        float odd = 0.f;  // 0 times each of the column's results
#pragma unroll
        for (int i = 0; i < W; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) odd = fmaf(acc[i][r], 0.f, odd);
        odd += __shfl_xor(odd, 16);
        odd += __shfl_xor(odd, 32);
        if (__any(odd != odd)) repair<T, DP>(nslots, splits, top, odd != odd, acc);
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (g == 0) lt[wave][m] = top, ls[wave][m] = sum;
#pragma unroll
    for (int i = 0; i < W; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) lo[wave][m][(4 * g + r) * W + i] = acc[i][r];
    __syncthreads();
    // 16 threads a row join the wavefronts
    const int q = threadIdx.x >> 4, c = threadIdx.x & 15;
    const int64_t rq = r0 + q;
    if (rq >= rows) return;
    const int64_t orow = p.first + rq / a.G;
    const int ohead = hk * a.G + static_cast<int>(rq % a.G);
    float best = kNegInf, all = 0.f, wgt[kFewWaves];
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) best = fmaxf(best, lt[w][q]);
    const float ref = best == kNegInf ? 0.f : best;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
        wgt[w] = __builtin_amdgcn_exp2f(a.c2 * (lt[w][q] - ref));
        all = fmaf(wgt[w], ls[w][q], all);
    }
    float *pr = splits > 1 ? part + ((orow * a.H + ohead) * splits + sp) * (a.D + 2) : nullptr;
    const float mul = pr ? 1.f : best == kNegInf ? 0.f : 1.f / all;
    for (int d = c; d < a.D; d += 16) {
        float o = 0.f;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) o = fmaf(wgt[w], lo[w][q][d], o);
        if (pr) pr[2 + d] = o;
        else put<T>(a, (orow * a.H + ohead) * a.D + d, o * mul);
    }
    if (c == 0) {
        if (pr) pr[0] = best, pr[1] = all;
        else if (a.stat) {
            float *st = a.stat + (orow * a.H + ohead) * 2;
            st[0] = best, st[1] = best == kNegInf ? 0.f : __log2f(all);
        }
    }
}

// Joins the S ranges of a (row, head): one wavefront each. Rows of no graph were written by k_few.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_join(const Args a, int splits, const float *__restrict__ part) {
    const int lane = threadIdx.x & 63;
    const int64_t at = (int64_t)blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6);
    if (at >= a.Nq * a.H || at / a.H >= uniform64(ptr_at(a.q_ptr, a.B, a.Nq))) return;
    const float *p = part + at * splits * (a.D + 2);
    float best = kNegInf;
    for (int s = lane; s < splits; s += 64) best = fmaxf(best, p[(int64_t)s * (a.D + 2)]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) best = fmaxf(best, __shfl_xor(best, o));
    const float ref = best == kNegInf ? 0.f : best;
    float all = 0.f, o0 = 0.f, o1 = 0.f;
    const int d0 = lane < a.D ? lane : 0, d1 = lane + 64 < a.D ? lane + 64 : 0;  // read in any case, kept where it is one
    const bool in0 = lane < a.D, in1 = lane + 64 < a.D;
    for (int s0 = 0; s0 < splits; s0 += 64) {
        // a lane a range for the weights, then the ranges' outputs, whose loads do not wait for one another
        const int n = splits - s0 < 64 ? splits - s0 : 64;
        const float *x = p + (int64_t)s0 * (a.D + 2);
        float w = 0.f;
        if (lane < n) {
            w = __builtin_amdgcn_exp2f(a.c2 * (x[lane * (a.D + 2)] - ref));
            all = fmaf(w, x[lane * (a.D + 2) + 1], all);
        }
        for (int s = 0; s < n; s += 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {  // past the last range the weight is 0, and what stands there may be infinite
                const float ws = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), s + i));
                const float *o = x + (s + i < n ? s + i : n - 1) * (a.D + 2) + 2;
                const float x0 = o[d0], x1 = o[d1];
                o0 = fmaf(ws, s + i < n ? x0 : 0.f, o0);
                o1 = fmaf(ws, s + i < n ? x1 : 0.f, o1);
            }
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) all += __shfl_xor(all, o);
    const float mul = best == kNegInf ? 0.f : 1.f / all;
    if (in0) put<T>(a, at * a.D + lane, o0 * mul);
    if (in1) put<T>(a, at * a.D + lane + 64, o1 * mul);
    if (a.stat && lane == 0) a.stat[2 * at] = best, a.stat[2 * at + 1] = best == kNegInf ? 0.f : __log2f(all);
}

template <typename T, int DP>
int launch(const Args &a, int splits, float *part, hipStream_t s) {
    const int64_t n = slots(a.Nq * a.G, a.B, 16), grid = n * a.Hkv * splits;
    if (grid * 64 * kFewWaves >= (int64_t(1) << 32)) return PYG_ERR_UNSUPPORTED;
    k_few<T, DP><<<static_cast<unsigned>(grid), 64 * kFewWaves, 0, s>>>(a, n, splits, part);
    PYG_LAUNCH_CHECK();
    if (splits > 1) {
        k_join<T><<<static_cast<unsigned>((a.Nq * a.H + kBlock / 64 - 1) / (kBlock / 64)), kBlock, 0, s>>>(a, splits, part);
        PYG_LAUNCH_CHECK();
    }
    return PYG_OK;
}

template <typename T>
int by_width(const Args &a, int splits, float *part, hipStream_t s) {
    if (a.D <= 32) return launch<T, 32>(a, splits, part, s);
    if (a.D <= 64) return launch<T, 64>(a, splits, part, s);
    return launch<T, 128>(a, splits, part, s);
}

}  // namespace

int few_splits(const Args &a) {
    // eight workgroups a CU, ranges of 256 keys or more on average
    const int64_t tiles = (a.Nq * a.G / 16 > a.B ? a.Nq * a.G / 16 : a.B) * a.Hkv;
    int64_t s = 2048 / tiles, most = a.Nk / a.B / 256;
    s = s < most ? s : most;
    return static_cast<int>(s < 1 ? 1 : s);
}

int forward_few(const Args &a, bool bf16, void *ws, hipStream_t s) {
    const int n = few_splits(a);
    float *part = static_cast<float *>(ws);
    return bf16 ? by_width<__bf16>(a, n, part, s) : by_width<float>(a, n, part, s);
}

}  // namespace attn
}  // namespace pyg
