// Attention among the nodes of each graph of a batch with a learned bias by
// relative position: gradients. With P the softmax's rows and g the gradient of
// the output,
//   delta_i = sum_d g_id o_id,  dP = g V^T,  dS = P (dP - delta),
//   dQ = c dS K,  dK = c dS^T Q,  dV = P^T g,  dT[b, h] = sum of dS over bucket b.
// P and dS are made again from the row statistics that the forward kept, once
// by the kernel that owns queries (dQ, delta, dT) and once by the one that owns
// keys (dK, dV): no gradient is added to by two workgroups, so the results do
// not depend on their order. bf16 operands: P and dS are each rounded to bf16 for the products
// that take them (half a step, 2^-8, of every summand), the results once more; delta, which dS
// subtracts, is taken of out + rest and keeps 8 bits more. Gradients are 0.0024 off 64 bits where fp32 weights
// leave 0.0017.
#include "attn.hpp"

namespace pyg {
namespace attn {
namespace {

// Keys or queries a tile of four wavefronts.
template <typename T, int DP>
constexpr int kTileOfFour = DP * sizeof(T) <= 128 ? 64 : 32;

// A row's statistics in units of s: p = exp2(c2 (s + start)), start = -(top + log2 sum / c2), -infinity for a row that
// sees no key. bf16 tiles' accumulators begin with it, as dP's do with -delta; in fp32 that would round every
// partial sum at start's magnitude (a table's gradient 1.3e-6 off instead of 4e-7), so it is added after the
// products. Where the bias holds lowest values (wild) s - top comes first and rest = -log2 sum / c2 after it.
template <typename T>
constexpr bool kStartLate = kBiasLate<T>;
struct RowStat {
    float top, start, rest;
};
__device__ __forceinline__ RowStat row_stat(float2 s, float c2) {
    const float rest = -s.y / c2;
    return {s.x, s.x == kNegInf ? kNegInf : rest - s.x, rest};
}

// Statistics that are not finite (the row sees something that is not): its weights become infinite where it sees
// something and stay 0 where it sees nothing, which NaN would not leave alone.
constexpr float kHuge = -kLowest;
__device__ __forceinline__ RowStat settled(const RowStat &s) {
    return finite(s.start) || s.top == kNegInf ? s : RowStat{0.f, kHuge, kHuge};
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// Between LDS accesses of different lanes of one wavefront to the same place. The LDS serves a wavefront in order;
// this keeps the compiler from another one (no instruction comes of it).
__device__ __forceinline__ void lanes_meet() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Adds a 32 x 32 tile of dS^T (rows keys, the lane's column a query) to the wavefront's sums
// by offset (key - query). The tile is laid down in LDS and read along its 63 diagonals, a lane
// each, so that no two lanes add to one place: LDS float atomics, a lane at a time, made the
// tiles near the diagonal a fifth of the kernel (three graphs, 9,001 nodes, 16 heads of 64).
constexpr int kSkewRow = 40, kSkew = 32 * kSkewRow;  // 40: the two halves' rows are 32 banks apart
__device__ __forceinline__ void add_diagonals(const f32x16 &ds, float *own, float *skew, int d0, int reach, bool causal, int lane) {
    lane = opaque(lane);
    const int m = lane & 31, h = lane >> 5;
    lanes_meet();  // the last tile's reads
#pragma unroll
    for (int r = 0; r < 16; ++r) skew[(8 * (r >> 2) + 4 * h + (r & 3)) * kSkewRow + m] = ds[r];
    lanes_meet();
    const int o = lane - 31;  // the lane's diagonal: key - query of the tile; lane 63 has none
    float t = 0.f;
#pragma unroll 8
    for (int row = 0; row < 32; ++row) {
        const int c = row - o;
        const float v = skew[row * kSkewRow + (c & 31)];
        t += static_cast<unsigned>(c) < 32u ? v : 0.f;
    }
    const int at = d0 + o;
    const bool mine = lane < 63 && !(causal && at > 0);  // later keys: nothing, whatever their dP
    const bool low = mine && at < -reach, high = mine && at > reach;
    if (mine && !low && !high) own[at + reach] += t;
    lanes_meet();  // the ends' sums, of whichever lane
    // the ends stand for all offsets beyond them
    const float below = wave_sum(low ? t : 0.f), above = wave_sum(high ? t : 0.f);
    if (lane == 0) own[0] += below, own[2 * reach] += above;
}

// Wavefronts a SIMD that the registers have to leave room for.
template <typename T, int DP>
constexpr int kGradWaves = DP <= 64 || sizeof(T) == 2 ? 2 : 1;
// The owned rows of V in LDS instead of registers: bf16 heads of 128 would need more than the 256 of two wavefronts a SIMD.
template <typename T, int DP>
constexpr bool kValuesInLds = DP == 128 && sizeof(T) == 2;

// A row's statistics, and delta where its kernel has not stored it: g (out + rest).
template <typename T>
__device__ __forceinline__ RowStat stat_of(const Args &a, int64_t row, int head) {
    return row_stat(*reinterpret_cast<const float2 *>(a.stat + (row * a.H + head) * 2), a.c2);
}
template <typename T>
__device__ __forceinline__ float delta_of(const BackwardArgs &b, int64_t row, int head) {
    const int64_t at = (row * b.f.H + head) * b.f.D;
    const T *g = static_cast<const T *>(b.grad_out) + at, *o = static_cast<const T *>(b.f.out) + at;
    const float d = row_dot(g, o, b.f.D);
    return b.f.rest ? d + row_dot(g, static_cast<const T *>(b.f.rest) + at, b.f.D) : d;
}

// Of a wavefront's dQ, already stored, the rows that are not finite (flag) though they see nothing but finite values
// (attn.hpp).
template <typename T, int DP, int WAVES>
__device__ __forceinline__ void repair_q(int64_t nslots, int splits, float *dq_part, bool flag) {
    constexpr int BK = WAVES == 1 ? 32 : kTileOfFour<T, DP>;
    const BackwardArgs &b = args_again<BackwardArgs>();
    const Args &a = b.f;
    const int lane = opaque(threadIdx.x & 63), wave = to_scalar(threadIdx.x >> 6);
    const uint32_t id = opaque(blockIdx.x);
    const int hk = to_scalar(id % a.Hkv), head = to_scalar(hk * a.G + id / a.Hkv % a.G), sp = to_scalar(id / a.H % splits);
    const Place pq = place_of(a.q_ptr, a.B, a.Nq, nslots - 1 - to_scalar(id / a.H / splits), 32 * WAVES, 1, lane);
    const int64_t k_first = uniform64(ptr_at(a.k_ptr, pq.graph, a.Nk)), k_last = uniform64(ptr_at(a.k_ptr, pq.graph + 1, a.Nk));
    const int64_t nk = k_last > k_first ? k_last - k_first : 0, i = (pq.tile * WAVES + wave) * 32 + (lane & 31);
    const bool there = pq.first + i < pq.last;
    const int64_t row = there ? pq.first + i : pq.first, shift = i + nk - (pq.last - pq.first);
    const T *k = static_cast<const T *>(a.k) + hk * a.k_head + k_first * a.k_row;
    const T *v = static_cast<const T *>(a.v) + hk * a.v_head + k_first * a.v_row;
    const T *q = static_cast<const T *>(a.q) + row * a.q_row + head * a.q_head;
    const T *g = static_cast<const T *>(b.grad_out) + (row * a.H + head) * a.D;
    const RowStat st = stat_of<T>(a, row, head);
    const float delta = delta_of<T>(b, row, head);
    flag = flag && there && row_finite(q, a.D) && row_finite(g, a.D);
    flag = sees_only_fine(flag, 0, nk, lane, [&](int64_t j) {
        return row_finite(k + j * a.k_row, a.D) && row_finite(v + j * a.v_row, a.D);
    }, [&](int64_t j) { return j <= shift; });
    if (!__any(flag)) return;
    const int64_t share = splits > 1 ? ((nk + BK - 1) / BK + splits - 1) / splits * BK : nk;  // the workgroup's keys
    const int64_t last = (sp + 1) * share < nk ? (sp + 1) * share : nk;
    f32x16 o[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) o[t] = f32x16(0.f);
#pragma unroll 1
    for (int64_t j = sp * share; j < last; ++j) {
        const bool seen = flag && j <= shift && st.top != kNegInf;
        if (!__any(seen)) continue;
        const float s = row_dot(q, k + j * a.k_row, a.D) + bias_of<T>(a, head, j - shift), dp = row_dot(g, v + j * a.v_row, a.D);
        add_row<T, DP>(o, k + j * a.k_row, seen ? __builtin_amdgcn_exp2f(a.c2 * ((s - st.top) + st.rest)) * (dp - delta) : 0.f, a.D, lane);
    }
    if (splits > 1) store_rows<float, DP>(dq_part, row, flag, a.H, head, a.D, a.D % 4 == 0, o, a.scale, lane);
    else store_rows<T, DP>(static_cast<T *>(b.grad_q), row, flag, a.H, head, a.D, a.vec_o, o, a.scale, lane);
}

// A workgroup owns 32 * WAVES queries, as in the forward.
template <typename T, int DP, int WAVES, int BK>
__global__ __launch_bounds__(64 * WAVES, (kGradWaves<T, DP>)) void k_grad_q(const BackwardArgs b, int64_t nslots, float *__restrict__ delta,
                                                       float *__restrict__ part, int splits, float *__restrict__ dq_part) {
    const Args &a = b.f;
    constexpr int NT = 64 * WAVES, BM = 32 * WAVES, E = Elem<T>::E, SQ = DP / (2 * E), NK = BK / 32;
    using L = Tile<T, DP>;
    constexpr int kTile = L::template bytes<BK>();
    constexpr int HALVES = WAVES == 1 ? 1 : 2;
    extern __shared__ __align__(16) char lds[];  // K and V of one or two tiles, the bias, the sums by offset
    float *bias = reinterpret_cast<float *>(lds + 2 * HALVES * kTile);
    float *hist = bias + (2 * a.reach + 1);  // a wavefront's own sums by offset
    const int lane = threadIdx.x & 63, wave = to_scalar(threadIdx.x >> 6), m = lane & 31, h = lane >> 5;
    const uint32_t id = blockIdx.x;
    const int hk = id % a.Hkv, head = hk * a.G + id / a.Hkv % a.G;
    const int sp = id / a.H % splits;  // the workgroup's share of the keys
    const int64_t slot = nslots - 1 - id / a.H / splits;
    float *mine = part ? part + ((slot * splits + sp) * a.H + head) * a.buckets : nullptr;  // its share of dT
    dq_part += sp * a.Nq * a.H * a.D;
    const Place pq = place_of(a.q_ptr, a.B, a.Nq, slot, BM, 1, lane);
    const int64_t q0 = pq.first + pq.tile * BM;
    if (pq.tile < 0 || q0 >= pq.last || pq.graph == a.B) {
        if (mine)
            for (int i = threadIdx.x; i < a.buckets; i += NT) mine[i] = 0.f;
        if (b.grad_q && pq.graph == a.B && pq.tile >= 0 && q0 < pq.last) {
            const int64_t e = q0 + BM < pq.last ? q0 + BM : pq.last;
            if (splits > 1) zero_rows(dq_part, q0, e, a.H, head, a.D);
            else zero_rows(static_cast<T *>(b.grad_q), q0, e, a.H, head, a.D);
        }
        return;
    }
    const int offsets = 2 * a.reach + 1;
    if (mine)
        for (int i = threadIdx.x; i < offsets * WAVES; i += NT) hist[i] = 0.f;
    float *own = hist + wave * offsets, *skew = hist + WAVES * offsets + wave * kSkew;
    int *bucket = reinterpret_cast<int *>(hist + WAVES * (offsets + kSkew));  // of every offset
    const int64_t k_first = uniform64(ptr_at(a.k_ptr, pq.graph, a.Nk)),
                  k_last = uniform64(ptr_at(a.k_ptr, pq.graph + 1, a.Nk));
    const int64_t nk = k_last > k_first ? k_last - k_first : 0, nq = pq.last - pq.first;
    const T *kb = static_cast<const T *>(a.k) + hk * a.k_head + k_first * a.k_row;
    const T *vb = static_cast<const T *>(a.v) + hk * a.v_head + k_first * a.v_row;

    const int64_t i0 = pq.tile * BM + wave * 32, row = pq.first + i0 + m;
    const bool there = row < pq.last;
    uint4 qf[SQ], gf[SQ];
    int64_t end = nk;
    if (a.causal) {
        const int64_t seen = pq.tile * BM + BM + nk - nq;
        end = seen < nk ? (seen < 0 ? 0 : seen) : nk;
    }
    int64_t from = 0;
    if (splits > 1) {
        const int64_t share = ((nk + BK - 1) / BK + splits - 1) / splits * BK;
        from = sp * share;
        end = end < from + share ? end : from + share;
    }
    if (!b.grad_q && !mine) end = from;  // delta alone is wanted
    const Stage<T, DP, BK, NT> sk(a.k_row, a.D, a.vec_k), sv(a.v_row, a.D, a.vec_v);
    auto fetch = [&](int64_t j0, int half) {
        if (j0 >= end) return;
        sk.load(kb, j0, nk - j0, lds + 2 * half * kTile);
        sv.load(vb, j0, nk - j0, lds + (2 * half + 1) * kTile);
    };
    // the first tile, the bias and the queries' rows wait for memory together
    fetch(from, 0);
    const bool wild = stage_bias<T>(a, head, bias, mine ? bucket : nullptr);
    const int64_t safe = there ? row : pq.first, at = (safe * a.H + head) * a.D;
    float dl = 0.f;
    {
        uint4 of[SQ], rf[SQ];
        load_row(static_cast<const T *>(a.q) + safe * a.q_row + head * a.q_head, a.D, there, h, qf);
        load_row(static_cast<const T *>(b.grad_out) + at, a.D, there, h, gf);
        load_row(static_cast<const T *>(a.out) + at, a.D, there, h, of);
        // what rounding took from the output; where it was not kept (a.rest NULL) nothing is added
        const bool more = sizeof(T) == 2 && a.rest;
        if (more) load_row(static_cast<const T *>(a.rest) + at, a.D, there, h, rf);
#pragma unroll
        for (int s = 0; s < SQ; ++s) {
            Piece<T> g, o, r;
            g.u = gf[s], o.u = of[s], r.u = more ? rf[s] : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < E; ++i) dl = fmaf(to_f32(g.v[i]), to_f32(o.v[i]) + to_f32(r.v[i]), dl);
        }
    }
    dl += other_half(dl);
    float2 raw = make_float2(kNegInf, 0.f);
    if (there) {
        raw = *reinterpret_cast<const float2 *>(a.stat + (row * a.H + head) * 2);
        if (h == 0 && sp == 0) delta[row * a.H + head] = dl;
    }
    RowStat st = row_stat(raw, a.c2);
    if (!finite(dl)) st.start = dl, dl = 0.f;  // an infinite P leaves dS as little finite, where anything is seen
    st = settled(st);
    constexpr bool kDeltaFirst = DP < 128 && !kStartLate<T>;  // dP starts from it, but where registers are short
    const f32x16 no_delta(-dl);

    registers_loaded();
    f32x16 acc[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) acc[t] = f32x16(0.f);
    float below = 0.f, above = 0.f;  // the lane's dS of whole tiles beyond the reach

    const typename L::RowLane rl(lane);
    const typename L::ColLane cl(lane);
    const int64_t shift = i0 + nk - nq;
    auto step = [&](const char *kt, const char *vt, int64_t j0) {
        const int d0 = near(j0 - shift), left = near(nk - j0);
        if (a.causal && d0 > 31) return;
        // inner tiles: no mask, no end, one bias; they jump over what the others need
        const bool inner = left >= BK && !wild && flat(d0 - 31, d0 + BK - 1, a.reach, a.causal);
        f32x16 s[NK], dp[NK];
        float late = 0.f;  // what fp32 scores get after the products
        if (inner) {
            const float begin = bias[d0 > 0 ? 2 * a.reach : 0] + st.start;
            if (kStartLate<T>) late = fminf(a.c2 * begin, kHuge);
#pragma unroll
            for (int n = 0; n < NK; ++n) s[n] = f32x16(kStartLate<T> ? 0.f : begin);
        } else if constexpr (kStartLate<T>) {
            late = wild ? 0.f : fminf(a.c2 * st.start, kHuge);
#pragma unroll
            for (int n = 0; n < NK; ++n) s[n] = f32x16(0.f);
        } else {
#pragma unroll
            for (int n = 0; n < NK; ++n) {
                s[n] = bias_tile<true>(bias, a.reach, d0 + 32 * n, lane);
                if (!wild) s[n] += st.start;
            }
        }
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
            for (int u = 0; u < SQ; ++u) {
                if (past<T>(u, a.D)) break;
                s[n] = mma<T>(L::row_piece(kt, rl, n, u), qf[u], s[n]);
                dp[n] = mma<T>(L::row_piece(vt, rl, n, u), gf[u], u == 0 ? (kDeltaFirst ? no_delta : f32x16(0.f)) : dp[n]);
            }
        if (!inner) {
#pragma unroll
            for (int n = 0; n < NK; ++n) {
                if constexpr (kStartLate<T>) add_bias<true>(s[n], bias, a.reach, d0 + 32 * n, lane);
                if (wild) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[n][r] = st.top == kNegInf ? kNegInf : (s[n][r] - st.top) + st.rest;
                }
                mask_tile<true, true>(s[n], left - 32 * n, 32, a.causal, d0 + 32 * n, lane, &dp[n], kDeltaFirst ? 0.f : dl);
            }
        }
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r)  // dS^T
                s[n][r] = __builtin_amdgcn_exp2f(kStartLate<T> ? fmaf(a.c2, s[n][r], late) : a.c2 * s[n][r]) *
                          (kDeltaFirst ? dp[n][r] : dp[n][r] - dl);
        if (mine) {
            if (inner) {
                float t = 0.f;
#pragma unroll
                for (int n = 0; n < NK; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r) t += s[n][r];
                (d0 > 0 ? above : below) += t;
            } else {
#pragma unroll
                for (int n = 0; n < NK; ++n) add_diagonals(s[n], own, skew, d0 + 32 * n, a.reach, a.causal, lane);
            }
        }
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
            for (int u = 0; u < Elem<T>::kSteps; ++u) {
                const uint4 p = piece_of<T>(s[n], u);  // dS rounded once to the operands' type
#pragma unroll
                for (int t = 0; t < DP / 32; ++t) acc[t] = mma<T>(L::col_piece(kt, cl, n, t, u), p, acc[t]);
            }
    };
    if constexpr (HALVES == 1) {
        for (int64_t j0 = from; j0 < end; j0 += BK) {
            if (j0 > from) {
                __syncthreads();
                fetch(j0, 0);
            }
            loads_done();
            __syncthreads();
            step(lds, lds + kTile, j0);
        }
    } else {
        for (int64_t j0 = from; j0 < end; j0 += 2 * BK) {
            loads_done();
            __syncthreads();
            fetch(j0 + BK, 1);
            step(lds, lds + kTile, j0);
            if (j0 + BK >= end) break;
            loads_done();
            __syncthreads();
            fetch(j0 + 2 * BK, 0);
            step(lds + 2 * kTile, lds + 3 * kTile, j0 + BK);
        }
    }
    if (b.grad_q) {
        if (splits > 1) store_rows<float, DP>(dq_part, row, there, a.H, head, a.D, a.D % 4 == 0, acc, a.scale, lane);
        else store_rows<T, DP>(static_cast<T *>(b.grad_q), row, there, a.H, head, a.D, a.vec_o, acc, a.scale, lane);
        const bool odd = a.causal && column_odd(acc);
        if (__any(odd)) repair_q<T, DP, WAVES>(nslots, splits, dq_part, odd);
    }
    if (mine) {
        below = wave_sum(below), above = wave_sum(above);
        lanes_meet();
        if (lane == 0) own[0] += below, own[offsets - 1] += above;
        __syncthreads();
        for (int i = threadIdx.x; i < a.buckets; i += NT) {
            float t = 0.f;
            for (int o = 0; o < offsets; ++o) {
                const bool here = bucket[o] == i;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) t += here ? hist[w * offsets + o] : 0.f;
            }
            mine[i] = t;
        }
    }
}

// The same of dK and dV: keys whose gradients are not finite (flag) though every query that sees them, over the heads that
// the workgroup has, is finite with its gradient and its statistics.
template <typename T, int DP, int WAVES>
__device__ __forceinline__ void repair_kv(const float *__restrict__ delta, int splits, float *__restrict__ part, bool flag) {
    const BackwardArgs &b = args_again<BackwardArgs>();
    const Args &a = b.f;
    const int lane = opaque(threadIdx.x & 63), wave = to_scalar(threadIdx.x >> 6);
    const uint32_t id = opaque(blockIdx.x);
    const int hk = to_scalar(id % a.Hkv), heads = a.G / splits, first = hk * a.G + to_scalar(id / a.Hkv % splits) * heads;
    const Place pk = place_of(a.k_ptr, a.B, a.Nk, to_scalar(id / a.Hkv / splits), 32 * WAVES, 1, lane);
    const int64_t q_first = uniform64(ptr_at(a.q_ptr, pk.graph, a.Nq)), q_last = uniform64(ptr_at(a.q_ptr, pk.graph + 1, a.Nq));
    const int64_t nq = q_last > q_first ? q_last - q_first : 0, j = (pk.tile * WAVES + wave) * 32 + (lane & 31);
    const bool there = pk.first + j < pk.last;
    const int64_t row = there ? pk.first + j : pk.first, shift = j - (pk.last - pk.first - nq);  // query i is at offset shift - i
    const T *k = static_cast<const T *>(a.k) + row * a.k_row + hk * a.k_head;
    const T *v = static_cast<const T *>(a.v) + row * a.v_row + hk * a.v_head;
    const auto q_of = [&](int64_t i, int head) { return static_cast<const T *>(a.q) + (q_first + i) * a.q_row + head * a.q_head; };
    const auto g_of = [&](int64_t i, int head) { return static_cast<const T *>(b.grad_out) + ((q_first + i) * a.H + head) * a.D; };
    flag = flag && there && row_finite(k, a.D) && row_finite(v, a.D);
#pragma unroll 1
    for (int head = first; head < first + heads && __any(flag); ++head)
        flag = sees_only_fine(flag, 0, nq, lane, [&](int64_t i) {
            const RowStat st = stat_of<T>(a, q_first + i, head);
            return row_finite(q_of(i, head), a.D) && row_finite(g_of(i, head), a.D) &&
                   (st.top == kNegInf || finite(st.start)) && finite(delta[(q_first + i) * a.H + head]);
        }, [&](int64_t i) { return i >= shift; });
    if (!__any(flag)) return;
    const auto walk = [&](auto visit) {
#pragma unroll 1
        for (int head = first; head < first + heads; ++head)
#pragma unroll 1
            for (int64_t i = 0; i < nq; ++i) {
                const RowStat st = stat_of<T>(a, q_first + i, head);
                const bool seen = flag && i >= shift && st.top != kNegInf;
                if (__any(seen)) {
                    const float s = row_dot(q_of(i, head), k, a.D) + bias_of<T>(a, head, shift - i);
                    visit(i, head, seen ? __builtin_amdgcn_exp2f(a.c2 * ((s - st.top) + st.rest)) : 0.f);
                }
            }
    };
    // dV, then dK
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        f32x16 o[DP / 32];
#pragma unroll
        for (int t = 0; t < DP / 32; ++t) o[t] = f32x16(0.f);
        walk([&](int64_t i, int head, float p) {
            const T *row = g_of(i, head);
            if (which) {
                p = p != 0.f ? p * (row_dot(row, v, a.D) - delta[(q_first + i) * a.H + head]) : 0.f;
                row = q_of(i, head);
            }
            add_row<T, DP>(o, row, p, a.D, lane);
        });
        const float mul = which ? a.scale : 1.f;
        if (splits > 1) store_rows<float, DP>(which ? part : part + a.Nk * a.Hkv * a.D, row, flag, a.Hkv, hk, a.D, a.D % 4 == 0, o, mul, lane);
        else store_rows<T, DP>(static_cast<T *>(which ? b.grad_k : b.grad_v), row, flag, a.Hkv, hk, a.D, a.vec_o, o, mul, lane);
    }
}

// A workgroup owns 32 * WAVES keys of one graph and key head and walks over
// the queries of all G heads that share it, in tiles of BQ. S = Q K^T puts a
// key in a lane's column: P and dS are the operands of dV^T = g^T P and
// dK^T = Q^T dS as they stand.
template <typename T, int DP, int WAVES, int BQ>
__global__ __launch_bounds__(64 * WAVES, (kGradWaves<T, DP>)) void k_grad_kv(const BackwardArgs b, int64_t nslots,
                                                        const float *__restrict__ delta, int splits, float *__restrict__ part) {
    const Args &a = b.f;
    constexpr int NT = 64 * WAVES, BN = 32 * WAVES, E = Elem<T>::E, SQ = DP / (2 * E), NQ = BQ / 32;
    using L = Tile<T, DP>;
    constexpr int kTile = L::template bytes<BQ>();
    static_assert(BQ <= NT, "a thread a query's statistics");
    extern __shared__ __align__(16) char lds[];  // Q and dO of two tiles, their statistics, the bias
    constexpr bool VL = kValuesInLds<T, DP>;
    char *vown = lds + 4 * kTile;
    float *stats = reinterpret_cast<float *>(vown + (VL ? L::template bytes<BN>() : 0));  // [2][4][BQ]: start, -delta, top, rest
    float *bias = stats + 8 * BQ;
    const int lane = threadIdx.x & 63, wave = to_scalar(threadIdx.x >> 6), m = lane & 31, h = lane >> 5;
    const uint32_t id = blockIdx.x;
    const int hk = id % a.Hkv, sp = id / a.Hkv % splits, heads = a.G / splits;  // the workgroup's share of the G heads
    const int64_t slot = id / a.Hkv / splits;  // causal: the first keys are seen by the most queries
    const int64_t whole = a.Nk * a.Hkv * a.D;
    float *dk_part = part + 2 * sp * whole, *dv_part = dk_part + whole;  // where there are several
    const Place pk = place_of(a.k_ptr, a.B, a.Nk, slot, BN, 1, lane);
    const int64_t k0 = pk.first + pk.tile * BN;
    if (pk.tile < 0 || k0 >= pk.last) return;
    if (pk.graph == a.B) {
        const int64_t e = k0 + BN < pk.last ? k0 + BN : pk.last;
        if (splits > 1) {
            zero_rows(dk_part, k0, e, a.Hkv, hk, a.D);
            zero_rows(dv_part, k0, e, a.Hkv, hk, a.D);
        } else {
            zero_rows(static_cast<T *>(b.grad_k), k0, e, a.Hkv, hk, a.D);
            zero_rows(static_cast<T *>(b.grad_v), k0, e, a.Hkv, hk, a.D);
        }
        return;
    }
    const int64_t q_first = uniform64(ptr_at(a.q_ptr, pk.graph, a.Nq)),
                  q_last = uniform64(ptr_at(a.q_ptr, pk.graph + 1, a.Nq));
    const int64_t nq = q_last > q_first ? q_last - q_first : 0, nk = pk.last - pk.first;
    const int64_t j0 = pk.tile * BN + wave * 32, row = pk.first + j0 + m;
    const bool there = row < pk.last;
    uint4 kf[SQ], vf[VL ? 1 : SQ];
    const int64_t safe = there ? row : pk.first;
    load_row(static_cast<const T *>(a.k) + safe * a.k_row + hk * a.k_head, a.D, there, h, kf);
    if constexpr (!VL) load_row(static_cast<const T *>(a.v) + safe * a.v_row + hk * a.v_head, a.D, there, h, vf);
    if constexpr (VL)
        Stage<T, DP, BN, NT>(a.v_row, a.D, a.vec_v)
            .load(static_cast<const T *>(a.v) + hk * a.v_head + pk.first * a.v_row, pk.tile * BN, nk - pk.tile * BN, vown);
    const int keys = near(nk - j0);
    f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) dk[t] = dv[t] = f32x16(0.f);

    int64_t begin = 0;
    if (a.causal) {  // the first query that sees the workgroup's first key
        begin = pk.tile * BN - (nk - nq);
        begin = begin < 0 ? 0 : begin / 32 * 32;
    }
    const Stage<T, DP, BQ, NT> sq(a.q_row, a.D, a.vec_q), sg((int64_t)a.H * a.D, a.D, a.vec_o);
    const typename L::RowLane rows(lane);
    const typename L::ColLane columns(lane);
    const char *vmine = vown + wave * 32 * L::kRowBytes;
    for (int g = sp * heads; g < (sp + 1) * heads && begin < nq; ++g) {
        const int head = hk * a.G + g;
        const T *qb = static_cast<const T *>(a.q) + head * a.q_head + q_first * a.q_row;
        const T *gb = static_cast<const T *>(b.grad_out) + (q_first * a.H + head) * a.D;
        bool wild = false;
        float2 next{};
        float next_delta = 0.f;
        const int query = threadIdx.x % BQ;
        // Q and dO of the next tile go to the other half of the LDS, its statistics by way of registers
        auto fetch = [&](int64_t i0, int half) {
            if (i0 >= nq) return;
            // every thread loads (the last query's where there is none): a branch here would have the compiler wait for
            // the old values' registers, and with them for the tiles
            const int64_t last = nq - 1 - i0, r = i0 + (last < query ? last : query);
            next = *reinterpret_cast<const float2 *>(a.stat + ((q_first + r) * a.H + head) * 2);
            next_delta = delta[(q_first + r) * a.H + head];
            sq.load(qb, i0, nq - i0, lds + 2 * half * kTile);
            sg.load(gb, i0, nq - i0, lds + (2 * half + 1) * kTile);
        };
        auto put = [&](int64_t i0, int half) {
            const RowStat t = settled(row_stat(make_float2(i0 + query < nq ? next.x : kNegInf, next.y), a.c2));
            float *s = stats + half * 4 * BQ + query;
            s[0] = t.start, s[BQ] = i0 + query < nq ? -next_delta : 0.f, s[2 * BQ] = t.top, s[3 * BQ] = t.rest;  // the same from several threads
        };
        // one form for all tiles, its accumulators being most of the registers: inner tiles jump over what they do not need
        auto step = [&](const char *qt, const char *gt, const float *stat, int64_t i0) {
            const int d0 = near(j0 - (i0 + nk - nq)), left = near(nq - i0);
            if (a.causal && d0 - (BQ - 1) > 31) return;  // all of the wavefront's keys come later than all queries
            const bool inner = left >= BQ && keys >= 32 && !wild && flat(d0 - (BQ - 1), d0 + 31, a.reach, a.causal);
            f32x16 s[NQ], dp[NQ];
            typename L::RowLane rl = rows;
            typename L::ColLane cl = columns;
            rl.x = opaque(rl.x), cl.x = opaque(cl.x);
            const float *mine = stat + opaque(4 * h);
            const float constant = inner ? a.c2 * bias[d0 > 0 ? 2 * a.reach : 0] : 0.f;  // the bias of an inner tile
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    f32x4 x(0.f), y(0.f);
                    if constexpr (!kStartLate<T>) {
                        x = *reinterpret_cast<const f32x4 *>(mine + 32 * n + 8 * q);
                        y = *reinterpret_cast<const f32x4 *>(mine + BQ + 32 * n + 8 * q);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[n][4 * q + i] = x[i], dp[n][4 * q + i] = y[i];
                }
            if (!inner && !kStartLate<T>) {
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    const f32x16 b = bias_tile<false>(bias, a.reach, d0 - 32 * n, lane);
                    s[n] = wild ? b : s[n] + b;
                }
            }
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int u = 0; u < SQ; ++u) {
                    if (past<T>(u, a.D)) break;
                    s[n] = mma<T>(L::row_piece(qt, rl, n, u), kf[u], s[n]);
                    dp[n] = mma<T>(L::row_piece(gt, rl, n, u), VL ? L::row_piece(vmine, rl, 0, u) : vf[VL ? 0 : u], dp[n]);
                }
            if (!inner) {
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    if constexpr (kStartLate<T>) add_bias<false>(s[n], bias, a.reach, d0 - 32 * n, lane);
                    if (wild) {
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const float *at = mine + 2 * BQ + 32 * n + 8 * (r >> 2) + (r & 3);
                            s[n][r] = at[0] == kNegInf ? kNegInf : (s[n][r] - at[0]) + at[BQ];
                        }
                    }
                    mask_tile<false, !kStartLate<T>>(s[n], keys, left - 32 * n, a.causal, d0 - 32 * n, lane, &dp[n]);
                }
            }
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float *at = mine + 32 * n + 8 * (r >> 2) + (r & 3);
                    const float e = kStartLate<T> && !wild ? s[n][r] + at[0] : s[n][r];
                    s[n][r] = __builtin_amdgcn_exp2f(fmaf(a.c2, e, constant));
                    dp[n][r] = s[n][r] * (kStartLate<T> ? dp[n][r] + at[BQ] : dp[n][r]);  // dS
                }
            if (kStartLate<T> && !inner && a.causal) {  // as mask_tile() does where delta is there already
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r) dp[n][r] = s[n][r] == 0.f ? 0.f : dp[n][r];
            }
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int u = 0; u < Elem<T>::kSteps; ++u) {
                    const uint4 p = piece_of<T>(s[n], u), d = piece_of<T>(dp[n], u);
#pragma unroll
                    for (int t = 0; t < DP / 32; ++t) {
                        dv[t] = mma<T>(L::col_piece(gt, cl, n, t, u), p, dv[t]);
                        dk[t] = mma<T>(L::col_piece(qt, cl, n, t, u), d, dk[t]);
                    }
                }
        };
        __syncthreads();  // the last head's tiles and bias are done with
        fetch(begin, 0);
        wild = stage_bias<T>(a, head, bias);
        registers_loaded();
        for (int64_t i0 = begin; i0 < nq; i0 += 2 * BQ) {
            put(i0, 0);
            loads_done();
            __syncthreads();
            fetch(i0 + BQ, 1);
            step(lds, lds + kTile, stats, i0);
            if (i0 + BQ >= nq) break;
            put(i0 + BQ, 1);
            loads_done();
            __syncthreads();
            fetch(i0 + 2 * BQ, 0);
            step(lds + 2 * kTile, lds + 3 * kTile, stats + 4 * BQ, i0 + BQ);
        }
    }
    const bool odd = a.causal && (column_odd(dk) || column_odd(dv));
    if (splits > 1) {
        store_rows<float, DP>(dk_part, row, there, a.Hkv, hk, a.D, a.D % 4 == 0, dk, a.scale, lane);
        store_rows<float, DP>(dv_part, row, there, a.Hkv, hk, a.D, a.D % 4 == 0, dv, 1.f, lane);
    } else {
        store_rows<T, DP>(static_cast<T *>(b.grad_k), row, there, a.Hkv, hk, a.D, a.vec_o, dk, a.scale, lane);
        store_rows<T, DP>(static_cast<T *>(b.grad_v), row, there, a.Hkv, hk, a.D, a.vec_o, dv, 1.f, lane);
    }
    if (__any(odd)) repair_kv<T, DP, WAVES>(delta, splits, dk_part, odd);
}

// dK and dV from the shares of the head groups [splits][2][Nk, Hkv, D], in order.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_join_kv(const float *__restrict__ part, int64_t n, int splits,
                                                    T *__restrict__ dk, T *__restrict__ dv) {
    for (int64_t i = blockIdx.x * (int64_t)kBlock + threadIdx.x; i < n; i += (int64_t)gridDim.x * kBlock) {
        float x = 0.f, y = 0.f;
        for (int s = 0; s < splits; ++s) x += part[2 * s * n + i], y += part[(2 * s + 1) * n + i];
        dk[i] = T(x), dv[i] = T(y);
    }
}

// Where few key tiles leave the card idle, the G heads that share a key head are
// dealt out over several workgroups: up to 1,024 (two rounds of two a CU). 8,192 ordered nodes, 16 heads of
// 128 on 4: one workgroup a tile 513 us, four and their sum 281 us.
int kv_splits(const Args &a, int64_t tiles) {
    int s = 1;
    while (s < a.G && tiles * a.Hkv * s < 1024) {
        do ++s;
        while (a.G % s);
    }
    return s;
}
// dQ from the shares of the key ranges [splits][Nq, H, D], in order.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_join_q(const float *__restrict__ part, int64_t n, int splits, T *__restrict__ dq) {
    for (int64_t i = blockIdx.x * (int64_t)kBlock + threadIdx.x; i < n; i += (int64_t)gridDim.x * kBlock) {
        float x = 0.f;
        for (int s = 0; s < splits; ++s) x += part[s * n + i];
        dq[i] = T(x);
    }
}
// Key ranges of dQ, where few queries over long histories leave the card idle: 1,024
// lone wavefronts, ranges of 256 keys or more (one query of 8 heads of 64 over 100,000 keys, bf16: all
// gradients 4,120 us without, 280 with).
int q_splits(const Args &a) {
    const int64_t tiles = (a.Nq / 32 + a.B) * a.H;
    if (a.B < 1 || tiles >= 512 || a.Nk < 1024 * a.B || a.Nq * 4 > a.Nk) return 1;
    const int64_t s = 1024 / tiles, most = a.Nk / a.B / 256;
    return static_cast<int>(s < most ? s : most);
}
int64_t key_tiles(const Args &a) { return a.Nk / 128 + 1; }

// dT[b, h] from the workgroups' shares [slots, H, buckets], in a fixed order: every
// 64th slot by each of the workgroup's 64 rows of threads, then the rows.
template <typename T>
__global__ __launch_bounds__(1024) void k_grad_table(const float *__restrict__ part, int64_t nslots, int H, int buckets,
                                                       T *__restrict__ out) {
    __shared__ double sums[1024];
    const int head = blockIdx.x, i = threadIdx.x & 15, r = threadIdx.x >> 4;
    const int bk = blockIdx.y * 16 + i;
    double t = 0;
    if (bk < buckets)
#pragma unroll 8
        for (int64_t s = r; s < nslots; s += 64) t += part[(s * H + head) * buckets + bk];
    sums[threadIdx.x] = t;
    __syncthreads();
    if (r == 0 && bk < buckets) {
        for (int k = 1; k < 64; ++k) t += sums[16 * k + i];
        out[(int64_t)bk * H + head] = T(static_cast<float>(t));
    }
}

constexpr int64_t kMost = (int64_t(1) << 32) - 1;  // threads of a launch

// How a call is cut up. The launches and the workspace go by the same plan.
struct Plan {
    bool lone_q, lone_kv;  // workgroups of one wavefront (32 rows) instead of four
    int q_splits, kv_splits;
    int64_t q_slots, kv_slots;
};
Plan plan_of(const Args &a, const Wanted &want) {
    // lone wavefronts for small graphs, as in the forward, and where tiles of 128 are few: one graph of 1,024 nodes
    // (4 heads of 64, bf16) 111 us against 126, 16 of 512 83 against 100; one of 4,096 (8 heads) 315 against 281.
    // Ranges of keys are for lone wavefronts too: 2,000 queries of 2 heads of 64 over 100,000 keys (bf16), all
    // gradients 800 us, 2,570 by workgroups of four that walk all keys.
    const bool lone = a.Nq <= 128 * a.B || (a.Nq <= 1024 * a.B && a.Nq / 128 * a.H <= 256);
    Plan p;
    p.q_splits = want.q || want.table ? q_splits(a) : 1;
    p.lone_q = lone || p.q_splits > 1, p.lone_kv = lone;
    p.kv_splits = lone ? 1 : kv_splits(a, key_tiles(a));
    p.q_slots = slots(a.Nq, a.B, p.lone_q ? 32 : 128);
    p.kv_slots = slots(a.Nk, a.B, p.lone_kv ? 32 : 128);
    return p;
}

struct Buffers {
    float *delta, *table, *kv, *dq;  // table, kv, dq: the shares, or NULL
    size_t bytes;
};
Buffers carve(const Args &a, const Plan &p, const Wanted &want, void *ws) {
    Carver c(ws);
    Buffers b{};
    b.delta = c.take<float>(a.Nq * a.H);
    if (want.table) b.table = c.take<float>(p.q_slots * p.q_splits * a.H * a.buckets);
    if (want.kv && p.kv_splits > 1) b.kv = c.take<float>(2 * p.kv_splits * a.Nk * a.Hkv * a.D);
    if (want.q && p.q_splits > 1) b.dq = c.take<float>(p.q_splits * a.Nq * a.H * a.D);
    b.bytes = align_up(c.used, 256);
    return b;
}

template <typename T, int DP, int WAVES, int BK>
int launch_q(const BackwardArgs &b, const Plan &p, const Buffers &w, hipStream_t s) {
    const Args &a = b.f;
    const size_t pair = 2 * Tile<T, DP>::template bytes<BK>(), bias = (2 * a.reach + 1) * sizeof(float);
    k_grad_q<T, DP, WAVES, BK><<<static_cast<unsigned>(p.q_slots * a.H * p.q_splits), 64 * WAVES,
                                 pair * (WAVES == 1 ? 1 : 2) + bias * (w.table ? 2 + WAVES : 1) +
                                     (w.table ? WAVES * kSkew * sizeof(float) : 0), s>>>(
        b, p.q_slots, w.delta, w.table, p.q_splits, w.dq);
    PYG_LAUNCH_CHECK();
    return PYG_OK;
}

template <typename T, int DP, int WAVES, int BK>
int launch_kv(const BackwardArgs &b, const Plan &p, const Buffers &w, hipStream_t s) {
    const Args &a = b.f;
    const size_t pair = 2 * Tile<T, DP>::template bytes<BK>(), bias = (2 * a.reach + 1) * sizeof(float);
    const size_t own = kValuesInLds<T, DP> ? Tile<T, DP>::template bytes<32 * WAVES>() : 0;
    k_grad_kv<T, DP, WAVES, BK><<<static_cast<unsigned>(p.kv_slots * a.Hkv * p.kv_splits), 64 * WAVES,
                                  2 * pair + own + 8 * BK * sizeof(float) + bias, s>>>(b, p.kv_slots, w.delta, p.kv_splits, w.kv);
    PYG_LAUNCH_CHECK();
    return PYG_OK;
}

template <typename T, int DP>
int launch(const BackwardArgs &b, void *ws, hipStream_t s) {
    const Args &a = b.f;
    constexpr int BK = kTileOfFour<T, DP>;
    const Wanted want{b.grad_q != nullptr, b.grad_k != nullptr, b.grad_table != nullptr};
    const Plan p = plan_of(a, want);
    if (p.q_slots * a.H * p.q_splits * (p.lone_q ? 64 : 256) > kMost || p.kv_slots * a.Hkv * p.kv_splits * (p.lone_kv ? 64 : 256) > kMost)
        return PYG_ERR_UNSUPPORTED;
    const Buffers w = carve(a, p, want, ws);
    PYG_TRY((p.lone_q ? launch_q<T, DP, 1, 32>(b, p, w, s) : launch_q<T, DP, 4, BK>(b, p, w, s)));
    if (w.dq) {
        const int64_t n = a.Nq * a.H * a.D;
        k_join_q<T><<<grid_for(n, kBlock, 8192), kBlock, 0, s>>>(w.dq, n, p.q_splits, static_cast<T *>(b.grad_q));
        PYG_LAUNCH_CHECK();
    }
    if (want.kv) PYG_TRY((p.lone_kv ? launch_kv<T, DP, 1, 32>(b, p, w, s) : launch_kv<T, DP, 4, BK>(b, p, w, s)));
    if (w.kv) {
        const int64_t n = a.Nk * a.Hkv * a.D;
        k_join_kv<T><<<grid_for(n, kBlock, 8192), kBlock, 0, s>>>(w.kv, n, p.kv_splits, static_cast<T *>(b.grad_k),
                                                                  static_cast<T *>(b.grad_v));
        PYG_LAUNCH_CHECK();
    }
    if (w.table) {
        k_grad_table<T><<<dim3(a.H, (a.buckets + 15) / 16), 1024, 0, s>>>(w.table, p.q_slots * p.q_splits, a.H, a.buckets,
                                                                            static_cast<T *>(b.grad_table));
        PYG_LAUNCH_CHECK();
    }
    return PYG_OK;
}

template <typename T>
int by_width(const BackwardArgs &b, void *ws, hipStream_t s) {
    if (b.f.D <= 32) return launch<T, 32>(b, ws, s);
    if (b.f.D <= 64) return launch<T, 64>(b, ws, s);
    return launch<T, 128>(b, ws, s);
}

}  // namespace

size_t backward_workspace(const Args &a, const Wanted &want) { return carve(a, plan_of(a, want), want, nullptr).bytes; }

int backward(const BackwardArgs &b, bool bf16, void *ws, hipStream_t s) {
    return bf16 ? by_width<__bf16>(b, ws, s) : by_width<float>(b, ws, s);
}

}  // namespace attn
}  // namespace pyg
