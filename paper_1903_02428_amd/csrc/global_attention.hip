// Attention among the nodes of each graph of a batch with a learned bias by
// relative position: forward.
#include "attn.hpp"

namespace pyg {
namespace attn {
namespace {

// Wavefronts a SIMD that the registers have to leave room for.
template <typename T, int DP, int WAVES>
constexpr int kForwardWaves = DP <= 64 ? 2 : sizeof(T) == 2 ? 2 : 1;

// Of a wavefront's rows, already stored, those that are not finite (flag) though they see nothing but finite values (see
// attn.hpp). Everything but their maxima and sums is found out again: the tile loop keeps nothing for this.
template <typename T, int DP, int WAVES>
__device__ __forceinline__ void repair(int64_t nslots, float top, float mul, bool flag) {
    const Args &a = args_again();
    const int lane = opaque(threadIdx.x & 63), wave = to_scalar(threadIdx.x >> 6);
    const uint32_t id = opaque(blockIdx.x);
    const int hk = to_scalar(id % a.Hkv), head = to_scalar(hk * a.G + id / a.Hkv % a.G);
    const Place pq = place_of(a.q_ptr, a.B, a.Nq, nslots - 1 - to_scalar(id / a.H), 32 * WAVES, 1, lane);
    const int64_t k_first = uniform64(ptr_at(a.k_ptr, pq.graph, a.Nk)), k_last = uniform64(ptr_at(a.k_ptr, pq.graph + 1, a.Nk));
    const int64_t nk = k_last > k_first ? k_last - k_first : 0, i = (pq.tile * WAVES + wave) * 32 + (lane & 31);
    const bool there = pq.first + i < pq.last;
    const int64_t row = there ? pq.first + i : pq.first, shift = i + nk - (pq.last - pq.first);  // key j is at offset j - shift
    const T *k = static_cast<const T *>(a.k) + hk * a.k_head + k_first * a.k_row;
    const T *v = static_cast<const T *>(a.v) + hk * a.v_head + k_first * a.v_row;
    const T *q = static_cast<const T *>(a.q) + row * a.q_row + head * a.q_head;
    flag = sees_only_fine(flag && there, 0, nk, lane, [&](int64_t j) {
        return row_finite(k + j * a.k_row, a.D) && row_finite(v + j * a.v_row, a.D);
    }, [&](int64_t j) { return j <= shift; });
    if (!__any(flag)) return;
    f32x16 o[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) o[t] = f32x16(0.f);
#pragma unroll 1
    for (int64_t j = 0; j < nk; ++j) {
        const bool seen = flag && j <= shift;
        if (!__any(seen)) continue;
        const float s = row_dot(q, k + j * a.k_row, a.D) + bias_of<T>(a, head, j - shift);
        add_row<T, DP>(o, v + j * a.v_row, seen ? __builtin_amdgcn_exp2f(a.c2 * (s - top)) : 0.f, a.D, lane);
    }
    store_rows<T, DP>(static_cast<T *>(a.out), row, flag, a.H, head, a.D, a.vec_o, o, mul, lane);
    if constexpr (sizeof(T) == 2)
        if (a.rest) store_rows<T, DP, true>(static_cast<T *>(a.rest), row, flag, a.H, head, a.D, a.vec_o, o, mul, lane);
}

// A workgroup owns 32 * WAVES queries of one graph and head and walks over the
// graph's keys in tiles of BK, staged in LDS for its wavefronts; a wavefront
// keeps 32 queries. S^T = K Q^T puts a query in a lane's column, so the running
// maximum and sum are one value a lane and P^T is the second product's operand
// as it stands: O^T = V^T P^T.
template <typename T, int DP, int WAVES, int BK>
__global__ __launch_bounds__(64 * WAVES, (kForwardWaves<T, DP, WAVES>)) void k_forward(const Args a, int64_t nslots) {
    constexpr int NT = 64 * WAVES, BM = 32 * WAVES, E = Elem<T>::E, SQ = DP / (2 * E), NK = BK / 32;
    using L = Tile<T, DP>;
    constexpr int kTile = L::template bytes<BK>();
    constexpr int HALVES = WAVES == 1 ? 1 : 2;   // a lone wavefront's graphs are mostly one tile: others hide its waits
    extern __shared__ __align__(16) char lds[];  // K and V of one or two tiles, the bias
    float *bias = reinterpret_cast<float *>(lds + 2 * HALVES * kTile);
    const int lane = threadIdx.x & 63, wave = to_scalar(threadIdx.x >> 6), m = lane & 31, h = lane >> 5;
    // key heads vary fastest: with up to 8 of them (or a multiple) every XCD's L2 sees its own heads' keys only
    const uint32_t id = blockIdx.x;
    const int hk = id % a.Hkv, head = hk * a.G + id / a.Hkv % a.G;
    const int64_t slot = nslots - 1 - id / a.H;  // causal: the longest walks first
    const Place pq = place_of(a.q_ptr, a.B, a.Nq, slot, BM, 1, lane);
    const int64_t q0 = pq.first + pq.tile * BM;  // the workgroup's first query row
    if (pq.tile < 0 || q0 >= pq.last) return;
    T *out = static_cast<T *>(a.out);
    if (pq.graph == a.B) {
        if (a.zero_rest) zero_rows(out, q0, q0 + BM < pq.last ? q0 + BM : pq.last, a.H, head, a.D);
        return;
    }
    const int64_t k_first = uniform64(ptr_at(a.k_ptr, pq.graph, a.Nk)),
                  k_last = uniform64(ptr_at(a.k_ptr, pq.graph + 1, a.Nk));
    const int64_t nk = k_last > k_first ? k_last - k_first : 0, nq = pq.last - pq.first;
    const T *kb = static_cast<const T *>(a.k) + hk * a.k_head + k_first * a.k_row;
    const T *vb = static_cast<const T *>(a.v) + hk * a.v_head + k_first * a.v_row;

    const int64_t i0 = pq.tile * BM + wave * 32;  // first query of the wavefront, in the graph
    const int64_t row = pq.first + i0 + m;        // the lane's query row
    const bool there = row < pq.last;
    f32x16 acc[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) acc[t] = f32x16(0.f);
    float top = kNegInf, sum = 0.f;  // of the lane's query: sum over this half's keys

    int64_t end = nk;
    if (a.causal) {
        const int64_t seen = pq.tile * BM + BM + nk - nq;  // keys that the last query of the workgroup may see
        end = seen < nk ? (seen < 0 ? 0 : seen) : nk;
    }
    const Stage<T, DP, BK, NT> sk(a.k_row, a.D, a.vec_k), sv(a.v_row, a.D, a.vec_v);
    auto fetch = [&](int64_t j0, int half) {
        if (j0 >= end) return;
        sk.load(kb, j0, nk - j0, lds + 2 * half * kTile);
        sv.load(vb, j0, nk - j0, lds + (2 * half + 1) * kTile);
    };
    // the bias, the first tile and the queries wait for memory together
    uint4 qf[SQ];
    fetch(0, 0);
    const bool wild = stage_bias<T>(a, head, bias);
    load_row(static_cast<const T *>(a.q) + (there ? row : pq.first) * a.q_row + head * a.q_head, a.D, there, h, qf);
    registers_loaded();
    const typename L::RowLane rl(lane);
    const typename L::ColLane cl(lane);
    const int64_t shift = i0 + nk - nq;  // offset of key j and the wavefront's first query: j - shift
    auto step = [&](const char *kt, const char *vt, int64_t j0) {
        const int d0 = near(j0 - shift), left = near(nk - j0);
        if (a.causal && d0 > 31) return;  // later than all of the wavefront's queries
        // inner tiles: no mask, no end, one bias; they jump over what the others need
        const bool inner = left >= BK && !wild && flat(d0 - 31, d0 + BK - 1, a.reach, a.causal);
        const float constant = inner ? bias[d0 > 0 ? 2 * a.reach : 0] : 0.f;  // the bias of an inner tile
        f32x16 st[NK];
#pragma unroll
        for (int n = 0; n < NK; ++n) st[n] = f32x16(0.f);
        if (!kBiasLate<T> && !inner) {
#pragma unroll
            for (int n = 0; n < NK; ++n) st[n] = bias_tile<true>(bias, a.reach, d0 + 32 * n, lane);
        }
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
            for (int s = 0; s < SQ; ++s) {
                if (past<T>(s, a.D)) break;
                st[n] = mma<T>(L::row_piece(kt, rl, n, s), qf[s], st[n]);
            }
        if (!inner) {
#pragma unroll
            for (int n = 0; n < NK; ++n) {
                if constexpr (kBiasLate<T>) add_bias<true>(st[n], bias, a.reach, d0 + 32 * n, lane);
                mask_tile<true>(st[n], left - 32 * n, 32, a.causal, d0 + 32 * n, lane);
            }
        }
        float t = kNegInf;
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) t = fmaxf(t, st[n][r]);
        t = fmaxf(t, other_half(t)) + constant;
        const float top_new = fmaxf(top, t), ref = top_new == kNegInf ? 0.f : top_new;
        const float shrink = __builtin_amdgcn_exp2f(a.c2 * (top - ref));
        top = top_new;
        sum *= shrink;
        if (__any(shrink != 1.f)) {
#pragma unroll
            for (int u = 0; u < DP / 32; ++u) acc[u] *= shrink;
        }
        float z = a.c2 * (constant - ref);
        if (wild) {  // s - m first, and nothing left to subtract
#pragma unroll
            for (int n = 0; n < NK; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) st[n][r] -= ref;
            z = 0.f;
        }
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                st[n][r] = __builtin_amdgcn_exp2f(fmaf(a.c2, st[n][r], z));
                sum += st[n][r];
            }
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
            for (int u = 0; u < Elem<T>::kSteps; ++u) {
                // P is rounded to the operands' type for the matrix cores (bf16: half a step, 2^-8 of each weight, before the
                // result's own half step; against 64 bits the output is 0.0019 off where fp32 weights leave 0.0016).
                // In two bf16 parts it would take half as many products again. The sum of P keeps 32 bits.
                const uint4 p = piece_of<T>(st[n], u);
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) acc[d] = mma<T>(L::col_piece(vt, cl, n, d, u), p, acc[d]);
            }
    };
    if constexpr (HALVES == 1) {
        for (int64_t j0 = 0; j0 < end; j0 += BK) {
            if (j0 > 0) {
                __syncthreads();
                fetch(j0, 0);
            }
            loads_done();
            __syncthreads();
            step(lds, lds + kTile, j0);
        }
    } else {
        // the next tile is on its way to one half of the LDS while the other is worked on
        for (int64_t j0 = 0; j0 < end; j0 += 2 * BK) {
            loads_done();
            __syncthreads();  // the tile is there, and nobody reads the other half any more
            fetch(j0 + BK, 1);
            step(lds, lds + kTile, j0);
            if (j0 + BK >= end) break;
            loads_done();
            __syncthreads();
            fetch(j0 + 2 * BK, 0);
            step(lds + 2 * kTile, lds + 3 * kTile, j0 + BK);
        }
    }
    sum += other_half(sum);
    const float mul = top == kNegInf ? 0.f : 1.f / sum;
    store_rows<T, DP>(out, row, there, a.H, head, a.D, a.vec_o, acc, mul, lane);
    if constexpr (sizeof(T) == 2)
        if (a.rest) store_rows<T, DP, true>(static_cast<T *>(a.rest), row, there, a.H, head, a.D, a.vec_o, acc, mul, lane);
    if (a.stat && there && h == 0)
        *reinterpret_cast<float2 *>(a.stat + (row * a.H + head) * 2) = make_float2(top, top == kNegInf ? 0.f : __log2f(sum));
    const bool odd = a.causal && column_odd(acc);
    if (__any(odd)) repair<T, DP, WAVES>(nslots, top, mul, odd);
}

template <typename T, int DP, int WAVES, int BK>
int launch(const Args &a, hipStream_t s) {
    const int64_t n = slots(a.Nq, a.B, 32 * WAVES);
    const size_t bytes = (WAVES == 1 ? 2 : 4) * Tile<T, DP>::template bytes<BK>() + (2 * a.reach + 1) * sizeof(float);
    if (n * a.H >= (int64_t(1) << 32) / (64 * WAVES)) return PYG_ERR_UNSUPPORTED;
    k_forward<T, DP, WAVES, BK><<<static_cast<unsigned>(n * a.H), 64 * WAVES, bytes, s>>>(a, n);
    PYG_LAUNCH_CHECK();
    return PYG_OK;
}

template <typename T, int DP>
int by_waves(const Args &a, hipStream_t s) {
    // graphs of up to 128 queries on average: 32 queries and a wavefront a tile. 64 graphs of 96 nodes (4 heads of 64,
    // fp32) 20 us against 29 with 128-query tiles, 8 of 256 alike, one of 4,096 (8 heads, bf16) 127 against 92.
    if (a.Nq <= 128 * a.B) return launch<T, DP, 1, 32>(a, s);
    return launch<T, DP, 4, DP * sizeof(T) <= 256 ? 64 : 32>(a, s);
}

template <typename T>
int by_width(const Args &a, hipStream_t s) {
    if (a.D <= 32) return by_waves<T, 32>(a, s);
    if (a.D <= 64) return by_waves<T, 64>(a, s);
    return by_waves<T, 128>(a, s);
}

}  // namespace

int forward(const Args &a, bool bf16, hipStream_t s) { return bf16 ? by_width<__bf16>(a, s) : by_width<float>(a, s); }

}  // namespace attn

namespace {

using namespace attn;

constexpr int64_t kMax32 = int64_t(1) << 31;

// Whether the 16-row form takes the queries: up to 16 rows that share a key head, on average over the graphs; or more,
// where whole walks over long histories would be too few for the card (bf16: one query of 32 heads on
// one over 100,000 keys 62 us instead of 3,726, 64 queries of 8 heads over as many 145 instead of 3,236).
bool few(const Args &a) {
    if (a.Nq * a.G <= 16 * a.B) return true;
    return (a.Nq / 32 + a.B) * a.H < 512 && a.Nk >= 1024 * a.B && a.Nq * 16 <= a.Nk;
}

bool vectors(const void *p, int64_t row, int64_t head, int64_t D, size_t e) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && row * e % 16 == 0 && head * e % 16 == 0 && D * e % 16 == 0;
}

// Host checks of a call; fills the kernels' arguments.
int take(const pyg_attention *c, Args *a) {
    if (!c) return PYG_ERR_INVALID_ARG;
    if (c->dtype != PYG_F32 && c->dtype != PYG_BF16) return PYG_ERR_INVALID_ARG;
    if (c->B < 0 || c->Nq < 0 || c->Nk < 0 || c->H < 1 || c->Hkv < 1 || c->D < 1 || c->H % c->Hkv) return PYG_ERR_INVALID_ARG;
    if (!(c->scale >= 1e-30f) || c->scale > 1e30f) return PYG_ERR_INVALID_ARG;
    if (c->Nq >= kMax32 || c->Nk >= kMax32 || c->B >= kMax32 || c->D > 128 || c->H > 65535) return PYG_ERR_UNSUPPORTED;
    if (c->table) {
        if (!c->bucket || c->buckets < 1 || c->reach < 0) return PYG_ERR_INVALID_ARG;
        if (c->reach > kMaxReach || c->buckets > kMaxReach) return PYG_ERR_UNSUPPORTED;
    }
    *a = Args{};
    a->q_ptr = c->q_ptr, a->k_ptr = c->k_ptr;
    a->B = c->B, a->Nq = c->Nq, a->Nk = c->Nk;
    a->H = static_cast<int>(c->H), a->Hkv = static_cast<int>(c->Hkv), a->G = a->H / a->Hkv, a->D = static_cast<int>(c->D);
    a->q_row = c->q_row, a->q_head = c->q_head, a->k_row = c->k_row, a->k_head = c->k_head, a->v_row = c->v_row,
    a->v_head = c->v_head;
    a->scale = c->scale, a->inv_scale = 1.f / c->scale, a->c2 = c->scale * 1.4426950408889634f;
    a->causal = c->causal != 0, a->zero_rest = c->zero_rest != 0;
    a->table = c->table, a->lut = c->table ? c->bucket : nullptr;
    a->buckets = c->table ? static_cast<int>(c->buckets) : 0, a->reach = c->table ? static_cast<int>(c->reach) : 0;
    return PYG_OK;
}

size_t bytes_of(const pyg_attention *c) { return c->dtype == PYG_BF16 ? 2 : 4; }

// Whether N rows of H heads of D features do not overlap: heads inside rows, or rows inside heads.
bool strided(int64_t row, int64_t head, int64_t N, int64_t H, int64_t D) {
    if ((N > 1 && row < D) || (H > 1 && head < D)) return false;
    return N <= 1 || H <= 1 || row >= head * (H - 1) + D || head >= row * (N - 1) + D;
}

int take_inputs(const pyg_attention *c, const void *q, const void *k, const void *v, Args *a) {
    if (!c->q_ptr || !c->k_ptr) return PYG_ERR_INVALID_ARG;
    if ((c->Nq > 0 && !q) || (c->Nk > 0 && (!k || !v))) return PYG_ERR_INVALID_ARG;
    if (!strided(c->q_row, c->q_head, c->Nq, c->H, c->D) || !strided(c->k_row, c->k_head, c->Nk, c->Hkv, c->D) ||
        !strided(c->v_row, c->v_head, c->Nk, c->Hkv, c->D))
        return PYG_ERR_INVALID_ARG;
    if (c->q_row >= kMaxRowStride || c->k_row >= kMaxRowStride || c->v_row >= kMaxRowStride) return PYG_ERR_UNSUPPORTED;
    if (c->Nq <= 1) a->q_row = c->D;  // a single row's stride says nothing
    if (c->Nk <= 1) a->k_row = a->v_row = c->D;
    const size_t e = bytes_of(c);
    a->q = q, a->k = k, a->v = v;
    a->vec_q = vectors(q, a->q_row, c->q_head, c->D, e);
    a->vec_k = vectors(k, a->k_row, c->k_head, c->D, e);
    a->vec_v = vectors(v, a->v_row, c->v_head, c->D, e);
    return PYG_OK;
}

attn::Wanted wanted(const pyg_attention *c) {
    return {!(c->skip & PYG_SKIP_GRAD_Q), !(c->skip & PYG_SKIP_GRAD_KV), c->table && !(c->skip & PYG_SKIP_GRAD_TABLE)};
}

// Bytes from the first to the last of N rows of H heads of D features.
int64_t span(int64_t N, int64_t H, int64_t D, int64_t row, int64_t head, size_t e) {
    return N < 1 ? 0 : static_cast<int64_t>((row * (N - 1) + head * (H - 1) + D) * e);
}
// What both directions read.
struct Inputs {
    Span s[7];
};
Inputs inputs_of(const Args &a, size_t e) {
    return {{{a.q, span(a.Nq, a.H, a.D, a.q_row, a.q_head, e)},
             {a.k, span(a.Nk, a.Hkv, a.D, a.k_row, a.k_head, e)},
             {a.v, span(a.Nk, a.Hkv, a.D, a.v_row, a.v_head, e)},
             {a.q_ptr, static_cast<int64_t>((a.B + 1) * sizeof(int64_t))},
             {a.k_ptr, static_cast<int64_t>((a.B + 1) * sizeof(int64_t))},
             {a.table, static_cast<int64_t>(a.buckets * a.H * e)},
             {a.lut, static_cast<int64_t>((2 * a.reach + 1) * sizeof(int32_t))}}};
}

}  // namespace
}  // namespace pyg

using namespace pyg;

extern "C" int pyg_global_attention_workspace(const pyg_attention *c, size_t *bytes) {
    Args a;
    if (!bytes) return PYG_ERR_INVALID_ARG;
    PYG_TRY(take(c, &a));
    *bytes = 0;
    if (a.B > 0 && few(a)) {
        const int s = few_splits(a);
        if (s > 1) *bytes = static_cast<size_t>(a.Nq) * a.H * s * (a.D + 2) * sizeof(float);
    }
    return PYG_OK;
}

extern "C" int pyg_global_attention(const pyg_attention *c, const void *q, const void *k, const void *v, void *out,
                                    float *stat, void *rest, void *ws, size_t ws_bytes, void *stream) {
    Args a;
    size_t need = 0;
    PYG_TRY(take(c, &a));
    PYG_TRY(take_inputs(c, q, k, v, &a));
    if (a.Nq > 0 && !out) return PYG_ERR_INVALID_ARG;
    PYG_TRY(pyg_global_attention_workspace(c, &need));
    if (ws_bytes < need || (need && !ws)) return PYG_ERR_WORKSPACE;
    if (a.Nq == 0) return PYG_OK;
    if (rest && c->dtype != PYG_BF16) return PYG_ERR_INVALID_ARG;
    const int64_t n = a.Nq * a.H * a.D, e = bytes_of(c);
    const Span results[] = {{out, n * e}, {rest, n * e}, {stat, a.Nq * a.H * 8}, {ws, static_cast<int64_t>(need)}};
    if (!apart(results, inputs_of(a, e).s)) return PYG_ERR_INVALID_ARG;
    a.out = out, a.stat = stat, a.rest = rest;
    a.vec_o = vectors(out, a.D, a.D, a.D, bytes_of(c)) && vectors(rest, a.D, a.D, a.D, bytes_of(c));
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool bf16 = c->dtype == PYG_BF16;
    return a.B > 0 && few(a) ? attn::forward_few(a, bf16, ws, s) : attn::forward(a, bf16, s);
}

extern "C" int pyg_global_attention_backward_workspace(const pyg_attention *c, size_t *bytes) {
    Args a;
    if (!bytes) return PYG_ERR_INVALID_ARG;
    PYG_TRY(take(c, &a));
    *bytes = attn::backward_workspace(a, wanted(c));
    return PYG_OK;
}

extern "C" int pyg_global_attention_backward(const pyg_attention *c, const void *grad_out, const void *q, const void *k,
                                             const void *v, const void *out, const float *stat, const void *rest, void *grad_q, void *grad_k,
                                             void *grad_v, void *grad_table, void *ws, size_t ws_bytes, void *stream) {
    attn::BackwardArgs b{};
    PYG_TRY(take(c, &b.f));
    PYG_TRY(take_inputs(c, q, k, v, &b.f));
    Args &a = b.f;
    const attn::Wanted want = wanted(c);
    if (a.Nq > 0 && (!grad_out || !out || !stat || (want.q && !grad_q))) return PYG_ERR_INVALID_ARG;
    if (a.Nk > 0 && want.kv && (!grad_k || !grad_v)) return PYG_ERR_INVALID_ARG;
    if (grad_table && !c->table) return PYG_ERR_INVALID_ARG;
    if (!want.q) grad_q = nullptr;
    if (!want.kv) grad_k = grad_v = nullptr;
    if (!want.table) grad_table = nullptr;
    const size_t need = attn::backward_workspace(a, want);
    if (ws_bytes < need || (need && !ws)) return PYG_ERR_WORKSPACE;
    if (rest && c->dtype != PYG_BF16) return PYG_ERR_INVALID_ARG;
    const int64_t e = bytes_of(c), nq = a.Nq * a.H * a.D * e, nk = a.Nk * a.Hkv * a.D * e;
    const Span results[] = {{grad_q, nq}, {grad_k, nk}, {grad_v, nk}, {grad_table, a.buckets * a.H * e}, {ws, static_cast<int64_t>(need)}};
    const Span kept[] = {{grad_out, nq}, {out, nq}, {rest, nq}, {stat, a.Nq * a.H * 8}};
    if (!apart(results, inputs_of(a, e).s) || !apart(results, kept)) return PYG_ERR_INVALID_ARG;
    a.out = const_cast<void *>(out), a.stat = const_cast<float *>(stat), a.rest = const_cast<void *>(rest);
    b.grad_out = grad_out, b.grad_q = grad_q, b.grad_k = grad_k, b.grad_v = grad_v, b.grad_table = grad_table;
    a.vec_o = true;
    for (const void *p : {grad_out, out, static_cast<const void *>(grad_q), static_cast<const void *>(grad_k),
                          static_cast<const void *>(grad_v)})
        a.vec_o = a.vec_o && vectors(p, a.D, a.D, a.D, bytes_of(c));
    if (!want.q && !want.kv && !want.table) return PYG_OK;
    return attn::backward(b, c->dtype == PYG_BF16, ws, static_cast<hipStream_t>(stream));
}
