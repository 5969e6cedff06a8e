// The norms around a block of a transformer, with its gate and residual scale:
//   u = norm(h; post),  r = residual + scale * sigmoid(gate) * u,  y = norm(r; pre),
// norm(x) = (x - mean) / sqrt(var + eps) w + b (layer) or x / sqrt(mean x^2 + eps) w
// (rms); each part may be left out.
//
// Bound by memory: every input is read once and r and y written once, a row
// staying in registers between. L lanes share a row (8 to 64 of them, a
// wavefront or a workgroup, by its width), a lane holding NV pieces of 16 bytes;
// means and variances are fp32 and two-pass (the deviations from the mean are
// squared). The backward reads the same inputs and the two gradients, makes the
// statistics again from the registers, and keeps the columns' sums (gradients of
// scale, weights and biases) in registers over all rows of its lanes; the
// workgroups' sums are joined in a fixed order by a second kernel.
#include <initializer_list>

#include "eight_bit.hpp"

namespace pyg {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
// rows of any width start at any element: the loads say so
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 __attribute__((aligned(2))) u32x4_any;

template <typename T>
__device__ __forceinline__ void unpack16(const u32x4 &u, float *v) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(u[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(u[i] << 16);
            v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
        }
    }
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// One piece of a row from feature f on, as it lies in memory: zeros past F.
template <typename T>
__device__ __forceinline__ u32x4 load_piece(const T *__restrict__ row, int f, int F) {
    constexpr int E = 16 / sizeof(T);
    if (f + E <= F) return *reinterpret_cast<const u32x4_any *>(row + f);
    u32x4 u{0, 0, 0, 0};
    if (f < F) {  // the last piece of a row whose width is no multiple
        uint64_t lo = 0, hi = 0;
#pragma unroll 1
        for (int i = 0; f + i < F; ++i) {
            const uint64_t b = sizeof(T) == 4 ? reinterpret_cast<const uint32_t *>(row)[f + i]
                                              : reinterpret_cast<const uint16_t *>(row)[f + i];
            (i < E / 2 ? lo : hi) |= b << (8 * sizeof(T) * (i % (E / 2)));
        }
        u = u32x4{static_cast<uint32_t>(lo), static_cast<uint32_t>(lo >> 32), static_cast<uint32_t>(hi), static_cast<uint32_t>(hi >> 32)};
    }
    return u;
}

template <typename T>
__device__ __forceinline__ void store_piece(T *__restrict__ row, int f, int F, const float *v) {
    constexpr int E = 16 / sizeof(T);
    if (f + E <= F) {
        u32x4 u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) u[i] = __float_as_uint(v[i]);
            else u[i] = pack2(v[2 * i], v[2 * i + 1]);
        }
        *reinterpret_cast<u32x4_any *>(row + f) = u;
        return;
    }
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (f + i < F) row[f + i] = T(v[i]);
}

struct Norm {
    int64_t N;
    int F;
    bool layer;
    float eps, inv_F;
    const void *h, *residual, *gate;
    bool gate_rows;
    const float *scale, *post_w, *post_b, *w, *b;
    bool post, pre;
    void *r, *y;
    int8_t *codes;
    uint8_t *steps;
    int blocks;  // of 32 features a row
    // backward
    const void *grad_r, *grad_y;
    void *grad_h, *grad_residual, *grad_gate;
    float *part;  // [workgroups, sums, F]
    int need_scale, need_post_w, need_post_b, need_w, need_b;  // place of the columns' sums, or -1
    int sums;
};

constexpr int kRowLds = 2 * 16;  // sums of a workgroup's wavefronts
struct Sums {
    float *lds;  // [2][kRowLds]
    int turn = 0;
};

// Rows within a wavefront share a workgroup of four; a wider row has its own.
constexpr int threads_of(int L) { return L <= 64 ? 256 : L; }

template <int CTRL>
__device__ __forceinline__ float moved(float v) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xF, 0xF, true));
}

// Sums over the L lanes of a row, K at once: 16 lanes by moves within the vector unit
// (neighbours, pairs, then mirrored halves and rows), further ones through LDS.
template <int L, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], Sums &at) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
        v[k] += moved<0xB1>(v[k]);   // quad_perm [1, 0, 3, 2]
        v[k] += moved<0x4E>(v[k]);   // quad_perm [2, 3, 0, 1]
        v[k] += moved<0x141>(v[k]);  // row_half_mirror
        if constexpr (L >= 16) v[k] += moved<0x140>(v[k]);  // row_mirror
        if constexpr (L >= 32) v[k] += __shfl_xor(v[k], 16);
        if constexpr (L >= 64) v[k] += __shfl_xor(v[k], 32);
    }
    if constexpr (L > 64) {
        constexpr int waves = L / 64;
        const int wave = threadIdx.x >> 6;
        // two halves in turn: who writes one has passed the barrier after which all had read it
        float *lds = at.lds + at.turn * kRowLds;
        at.turn ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) lds[k * waves + wave] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float t = 0.f;
            for (int w = 0; w < waves; ++w) t += lds[k * waves + w];
            v[k] = t;
        }
    }
}

template <typename T, int L, int NV>
struct Body {
    static constexpr int E = 16 / sizeof(T), M = NV * E;
    static __device__ __forceinline__ int feature(int lane, int i) { return (lane + L * i) * E; }
    struct Raw {
        u32x4 u[NV];
    };
    static __device__ __forceinline__ void fetch(const void *p, int64_t row, int F, int lane, Raw &r) {
        const T *x = static_cast<const T *>(p) + row * F;
#pragma unroll
        for (int i = 0; i < NV; ++i) r.u[i] = load_piece<T>(x, feature(lane, i), F);
    }
    static __device__ __forceinline__ void open(const Raw &r, float (&v)[M]) {
#pragma unroll
        for (int i = 0; i < NV; ++i) unpack16<T>(r.u[i], v + i * E);
    }
    static __device__ __forceinline__ void store(void *p, int64_t row, int F, int lane, const float (&v)[M]) {
        T *x = static_cast<T *>(p) + row * F;
#pragma unroll
        for (int i = 0; i < NV; ++i) store_piece<T>(x, feature(lane, i), F, v + i * E);
    }
    // a [F] parameter in fp32, `other` where it is missing
    static __device__ __forceinline__ void load_param(const float *p, int F, int lane, float other, float (&v)[M]) {
#pragma unroll
        for (int k = 0; k < M; ++k) v[k] = other;
        if (!p) return;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < E; e += 4) unpack16<float>(load_piece<float>(p, feature(lane, i) + e, F), v + i * E + e);
    }
    static __device__ __forceinline__ bool inside(int lane, int k, int F) { return feature(lane, k / E) + k % E < F; }

    // x -> its normalised values; returns 1 / deviation
    static __device__ __forceinline__ float normalise(float (&x)[M], const Norm &a, int lane, Sums &lds) {
        if (a.layer) {
            float s[1] = {0.f};
#pragma unroll
            for (int k = 0; k < M; ++k) s[0] += x[k];
            row_sums<L, 1>(s, lds);
            const float mean = s[0] * a.inv_F;
#pragma unroll
            for (int k = 0; k < M; ++k) x[k] = inside(lane, k, a.F) ? x[k] - mean : 0.f;
        }
        float q[1] = {0.f};
#pragma unroll
        for (int k = 0; k < M; ++k) q[0] = fmaf(x[k], x[k], q[0]);
        row_sums<L, 1>(q, lds);
        const float rstd = __builtin_amdgcn_rsqf(fmaf(q[0], a.inv_F, a.eps));  // within one step of fp32
#pragma unroll
        for (int k = 0; k < M; ++k) x[k] *= rstd;
        return rstd;
    }
    // gradient t of the normalised values n -> gradient of x
    static __device__ __forceinline__ void through(float (&t)[M], const float (&n)[M], float rstd, const Norm &a, int lane,
                                                   Sums &lds) {
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < M; ++k) s[0] = fmaf(t[k], n[k], s[0]), s[1] += t[k];
        row_sums<L, 2>(s, lds);
        const float tn = s[0] * a.inv_F, tm = a.layer ? s[1] * a.inv_F : 0.f;
#pragma unroll
        for (int k = 0; k < M; ++k) t[k] = inside(lane, k, a.F) ? (t[k] - n[k] * tn - tm) * rstd : 0.f;
    }
};

// exp and reciprocal by the hardware's instructions, each within one step of fp32 (and the exponent's rounding)
__device__ __forceinline__ float sigmoid_of(float e) { return __builtin_amdgcn_rcpf(1.f + e); }  // e = exp(-x)
__device__ __forceinline__ float exp_minus(float x) { return __builtin_amdgcn_exp2f(-1.4426950408889634f * x); }
__device__ __forceinline__ float sigmoid(float x) { return sigmoid_of(exp_minus(x)); }

template <typename T, int L, int NV>
__global__ __launch_bounds__(threads_of(L)) void k_block_norm(const Norm a) {
    using B = Body<T, L, NV>;
    constexpr int M = B::M, E = B::E, R = threads_of(L) / L;
    __shared__ float sums_lds[2 * kRowLds];
    Sums lds{sums_lds};
    const int lane = threadIdx.x % L;
    float sc[M], pw[M], pb[M], w[M], b[M];
    B::load_param(a.scale, a.F, lane, 1.f, sc);
    B::load_param(a.post_w, a.F, lane, 1.f, pw);
    B::load_param(a.post_b, a.F, lane, 0.f, pb);
    B::load_param(a.w, a.F, lane, 1.f, w);
    B::load_param(a.b, a.F, lane, 0.f, b);
    const int64_t step = (int64_t)gridDim.x * R;
    int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / L;
    typename B::Raw rh, rr, rg;
    auto fetch = [&](int64_t at) {
        B::fetch(a.h, at, a.F, lane, rh);
        if (a.residual) B::fetch(a.residual, at, a.F, lane, rr);
        if (a.gate && !a.gate_rows) B::fetch(a.gate, at, a.F, lane, rg);
    };
    if (row < a.N) fetch(row);
    for (; row < a.N; row += step) {
        float x[M], res[M], g[M];
        B::open(rh, x);
        B::open(rr, res);
        B::open(rg, g);
        float gr = 0.f;
        if (a.gate && a.gate_rows) gr = sigmoid(static_cast<float>(static_cast<const T *>(a.gate)[row]));
        if (row + step < a.N) fetch(row + step);  // on its way while this row is worked on
        if (a.post) {
            B::normalise(x, a, lane, lds);
#pragma unroll
            for (int k = 0; k < M; ++k) x[k] = fmaf(x[k], pw[k], pb[k]);
        }
#pragma unroll
        for (int k = 0; k < M; ++k) {
            if (a.gate) x[k] *= a.gate_rows ? gr : sigmoid(g[k]);
            x[k] = a.residual ? fmaf(sc[k], x[k], res[k]) : sc[k] * x[k];
        }
        if (a.r) B::store(a.r, row, a.F, lane, x);
        if (!a.pre) continue;
#pragma unroll
        for (int k = 0; k < M; ++k)
            if (!B::inside(lane, k, a.F)) x[k] = 0.f;
        B::normalise(x, a, lane, lds);
#pragma unroll
        for (int k = 0; k < M; ++k) x[k] = fmaf(x[k], w[k], b[k]);
        B::store(a.y, row, a.F, lane, x);
        if (a.codes) {
            // the checkpoint holds y as it was stored
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int f = B::feature(lane, i);
                uint32_t top = 0;
                float *v = x + i * E;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    v[e] = f + e < a.F ? static_cast<float>(T(v[e])) : 0.f;
                    const uint32_t m = eight::magnitude(v[e]);
                    top = m > top ? m : top;
                }
#pragma unroll
                for (int o = 1; o < 32 / E; o <<= 1) {
                    const uint32_t m = __shfl_xor(top, o);
                    top = m > top ? m : top;
                }
                if (f >= a.blocks * 32) continue;
                const uint32_t e = eight::step_of(top);
                const float inv = eight::step_inverse(e);
                uint32_t q[E / 4];
#pragma unroll
                for (int j = 0; j < E / 4; ++j)
                    q[j] = eight::code(v[4 * j], inv, e) | eight::code(v[4 * j + 1], inv, e) << 8 |
                           eight::code(v[4 * j + 2], inv, e) << 16 | eight::code(v[4 * j + 3], inv, e) << 24;
                int8_t *c = a.codes + row * a.blocks * 32 + f;
                if constexpr (E == 4) *reinterpret_cast<uint32_t *>(c) = q[0];
                else *reinterpret_cast<uint2 *>(c) = make_uint2(q[0], q[E / 4 - 1]);
                if (f % 32 == 0) a.steps[row * a.blocks + f / 32] = static_cast<uint8_t>(e);
            }
        }
    }
}

template <typename T, int L, int NV>
__global__ __launch_bounds__(threads_of(L)) void k_block_norm_grad(const Norm a) {
    using B = Body<T, L, NV>;
    constexpr int M = B::M, E = B::E, NT = threads_of(L), R = NT / L;
    __shared__ float sums_lds[2 * kRowLds];
    Sums lds{sums_lds};
    __shared__ float cols[R > 1 ? R * L * M : 1];
    const int lane = threadIdx.x % L;
    float s_sc[M], s_pw[M], s_pb[M], s_w[M], s_b[M];
#pragma unroll
    for (int k = 0; k < M; ++k) s_sc[k] = s_pw[k] = s_pb[k] = s_w[k] = s_b[k] = 0.f;
    // parameters and the next row stay in registers where there is room for them (128 a lane in workgroups of 1,024)
    constexpr bool kRoom = L < 1024, kHold = M <= 8 && kRoom;
    float h_sc[kHold ? M : 1], h_p[kHold ? M : 1], h_pb[kHold ? M : 1], h_w[kHold ? M : 1];
    if constexpr (kHold) {
        B::load_param(a.scale, a.F, lane, 1.f, h_sc);
        B::load_param(a.post_w, a.F, lane, 1.f, h_p);
        B::load_param(a.post_b, a.F, lane, 0.f, h_pb);
        B::load_param(a.w, a.F, lane, 1.f, h_w);
    }
    auto param = [&](const float *p, const auto &held, float other, float (&v)[M]) {
        if constexpr (kHold) {
#pragma unroll
            for (int k = 0; k < M; ++k) v[k] = held[k];
        } else {
            B::load_param(p, a.F, lane, other, v);
        }
    };
    const int64_t step = (int64_t)gridDim.x * R;
    int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / L;
    typename B::Raw rh, rr, rg, ry, rt;
    auto fetch = [&](int64_t at) {
        B::fetch(a.h, at, a.F, lane, rh);
        if (a.residual) B::fetch(a.residual, at, a.F, lane, rr);
        if (a.gate && !a.gate_rows) B::fetch(a.gate, at, a.F, lane, rg);
        if (a.grad_y) B::fetch(a.grad_y, at, a.F, lane, ry);
        if (a.grad_r) B::fetch(a.grad_r, at, a.F, lane, rt);
    };
    if (kRoom && row < a.N) fetch(row);
    for (; row < a.N; row += step) {
        if (!kRoom) fetch(row);
        float nh[M], ge[M], nr[M], t[M], p[M], gy[M];
        B::open(rh, nh);
        B::open(rr, nr);
        B::open(rg, ge);
        B::open(ry, gy);
        B::open(rt, t);
        // the gate as e = exp(-x): sigmoid(x) = 1 / (1 + e), sigmoid(-x) = e sigmoid(x), each with all its bits (1 - sigmoid(x)
        // would lose them from logits of about 12 on)
        float gr = 0.f;
        if (a.gate && a.gate_rows) gr = exp_minus(static_cast<float>(static_cast<const T *>(a.gate)[row]));
        if (kRoom && row + step < a.N) fetch(row + step);  // on its way while this row is worked on
        float rstd_h = 0.f;
        if (a.post) rstd_h = B::normalise(nh, a, lane, lds);
        float sc[M], u[M];
        param(a.scale, h_sc, 1.f, sc);
        param(a.post_w, h_p, 1.f, p);
#pragma unroll
        for (int k = 0; k < M; ++k) u[k] = nh[k];
        if (a.post) {
            float pb[M];
            param(a.post_b, h_pb, 0.f, pb);
#pragma unroll
            for (int k = 0; k < M; ++k) u[k] = fmaf(nh[k], p[k], pb[k]);
        }
#pragma unroll
        for (int k = 0; k < M; ++k) {
            ge[k] = !a.gate || a.gate_rows ? gr : exp_minus(ge[k]);
            const float c = sc[k] * sigmoid_of(ge[k]) * u[k];
            nr[k] = !B::inside(lane, k, a.F) ? 0.f : a.residual ? nr[k] + c : c;
            if (!a.grad_r) t[k] = 0.f;
        }
        if (a.pre && a.grad_y) {
            const float rstd_r = B::normalise(nr, a, lane, lds);
            float w[M];
            param(a.w, h_w, 1.f, w);
#pragma unroll
            for (int k = 0; k < M; ++k) {
                s_w[k] = fmaf(gy[k], nr[k], s_w[k]);
                s_b[k] += gy[k];
                gy[k] *= w[k];
            }
            B::through(gy, nr, rstd_r, a, lane, lds);
#pragma unroll
            for (int k = 0; k < M; ++k) t[k] += gy[k];
        }
        if (a.grad_residual) B::store(a.grad_residual, row, a.F, lane, t);
        float dg[M], row_gate[1] = {0.f};
#pragma unroll
        for (int k = 0; k < M; ++k) {
            // made again where registers are short, not kept beside e
            if constexpr (!kRoom) asm volatile("" : "+v"(ge[k]));
            const float g = sigmoid_of(ge[k]);
            s_sc[k] = fmaf(t[k] * g, u[k], s_sc[k]);
            t[k] *= sc[k];
            dg[k] = t[k] * u[k] * g * (fminf(ge[k], 0x1p126f) * g);  // e beyond 2^126: g is 0
            row_gate[0] += dg[k];
            t[k] *= g;  // the gradient of u
        }
        if (a.grad_gate) {
            if (a.gate_rows) {
                row_sums<L, 1>(row_gate, lds);
                if (lane == 0) static_cast<T *>(a.grad_gate)[row] = T(row_gate[0]);
            } else {
                B::store(a.grad_gate, row, a.F, lane, dg);
            }
        }
        if (a.post) {
#pragma unroll
            for (int k = 0; k < M; ++k) {
                s_pw[k] = fmaf(t[k], nh[k], s_pw[k]);
                s_pb[k] += t[k];
                t[k] *= p[k];
            }
            B::through(t, nh, rstd_h, a, lane, lds);
        }
        if (a.grad_h) B::store(a.grad_h, row, a.F, lane, t);
    }
    // the workgroup's columns: its R rows' lanes in order
    float *part = a.part + (int64_t)blockIdx.x * a.sums * a.F;
    auto put = [&](const float (&s)[M], int at) {
        if (at < 0) return;  // the same for every thread
        if constexpr (R == 1) {
#pragma unroll
            for (int k = 0; k < M; ++k) {
                const int f = B::feature(lane, k / E) + k % E;
                if (f < a.F) part[(int64_t)at * a.F + f] = s[k];
            }
        } else {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < M; ++k) cols[(threadIdx.x / L) * L * M + B::feature(lane, k / E) + k % E] = s[k];
            __syncthreads();
            for (int f = threadIdx.x; f < a.F; f += NT) {
                float v = 0.f;
                for (int r = 0; r < R; ++r) v += cols[r * L * M + f];
                part[(int64_t)at * a.F + f] = v;
            }
        }
    };
    put(s_sc, a.need_scale);
    put(s_pw, a.need_post_w);
    put(s_pb, a.need_post_b);
    put(s_w, a.need_w);
    put(s_b, a.need_b);
}

struct Columns {
    float *out[5];
};

// out[s][f] = sum over the workgroups of part[g][s][f]: 64 columns a workgroup,
// 16 threads a column, each every 16th workgroup, then the 16 in order.
__global__ __launch_bounds__(1024) void k_join_columns(const float *__restrict__ part, int groups, int sums, int F,
                                                       Columns c) {
    __shared__ float lds[16][64];
    const int i = threadIdx.x & 63, r = threadIdx.x >> 6;
    const int64_t col = (int64_t)blockIdx.x * 64 + i, all = (int64_t)sums * F;
    float v = 0.f;
    if (col < all)
#pragma unroll 8
        for (int g = r; g < groups; g += 16) v += part[g * all + col];
    lds[r][i] = v;
    __syncthreads();
    if (r == 0 && col < all) {
        for (int k = 1; k < 16; ++k) v += lds[k][i];
        c.out[col / F][col % F] = v;
    }
}

// Workgroups of the backward: 4,096 wavefronts (2,048 of rows of two), so that the sums they leave are few.
int64_t most_groups(int L) { return L == 128 ? 1024 : 4096 * 64 / threads_of(L); }

struct Shape {
    int L, NV;
};
// Lanes of a row and pieces a lane. The backward holds five arrays of a row and as many sums, so a lane has at most 8
// values there where a wider workgroup can take the rest: 16,000 rows of 1,433 (fp32) 185 us with 512
// lanes of one piece, 210 with 256 of two; the forward 111 and 82.
Shape shape_of(int64_t F, int E, bool backward) {
    const int64_t v = (F + E - 1) / E;
    const bool two = !backward || E == 4;  // two pieces of 4 values in the backward
    for (int L = 8; L <= 64; L *= 2)
        if (v <= L) return {L, 1};
    if (v <= 128) return two ? Shape{64, 2} : Shape{128, 1};
    if (v <= 256) return {256, 1};
    if (v <= 512) return backward ? Shape{512, 1} : Shape{256, 2};
    if (v <= 1024) return two ? Shape{512, 2} : Shape{1024, 1};
    return {1024, 2};
}

template <typename T, int L, int NV, bool BACKWARD>
int launch(const Norm &a, int64_t groups, hipStream_t s) {
    constexpr int NT = threads_of(L), R = NT / L;
    if constexpr (BACKWARD) k_block_norm_grad<T, L, NV><<<static_cast<unsigned>(groups), NT, 0, s>>>(a);
    else k_block_norm<T, L, NV><<<grid_for(a.N, R, 2048 * 256 / NT), NT, 0, s>>>(a);
    PYG_LAUNCH_CHECK();
    return PYG_OK;
}

template <typename T, bool BACKWARD>
int by_shape(const Norm &a, int64_t groups, hipStream_t s) {
    constexpr int E = 16 / sizeof(T);
    constexpr bool two = !BACKWARD || E == 4;
    const Shape h = shape_of(a.F, E, BACKWARD);
    if (h.L == 8) return launch<T, 8, 1, BACKWARD>(a, groups, s);
    if (h.L == 16) return launch<T, 16, 1, BACKWARD>(a, groups, s);
    if (h.L == 32) return launch<T, 32, 1, BACKWARD>(a, groups, s);
    if (h.L == 64 && h.NV == 1) return launch<T, 64, 1, BACKWARD>(a, groups, s);
    if (h.L == 256 && h.NV == 1) return launch<T, 256, 1, BACKWARD>(a, groups, s);
    if constexpr (two) {
        if (h.L == 64) return launch<T, 64, 2, BACKWARD>(a, groups, s);
        if (h.L == 512 && h.NV == 2) return launch<T, 512, 2, BACKWARD>(a, groups, s);
    } else {
        if (h.L == 128) return launch<T, 128, 1, BACKWARD>(a, groups, s);
        if (h.L == 1024) return launch<T, 1024, 1, BACKWARD>(a, groups, s);
    }
    if constexpr (BACKWARD) {
        if (h.L == 512) return launch<T, 512, 1, BACKWARD>(a, groups, s);
    } else {
        if (h.L == 256) return launch<T, 256, 2, BACKWARD>(a, groups, s);
    }
    if constexpr (E == 4)
        if (h.L == 1024) return launch<T, 1024, 2, BACKWARD>(a, groups, s);
    return PYG_ERR_UNSUPPORTED;  // not reached: F <= 8192
}

int64_t grad_groups(const pyg_block_norm_args *c) {
    const int E = c->dtype == PYG_BF16 ? 8 : 4;
    const Shape h = shape_of(c->F, E, true);
    const int64_t R = threads_of(h.L) / h.L, rows = (c->N + R - 1) / R, most = most_groups(h.L);
    return rows < 1 ? 1 : rows < most ? rows : most;
}

int check(const pyg_block_norm_args *c) {
    if (!c || (c->dtype != PYG_F32 && c->dtype != PYG_BF16) || (c->norm != PYG_NORM_LAYER && c->norm != PYG_NORM_RMS))
        return PYG_ERR_INVALID_ARG;
    if (c->N < 0 || c->F < 1 || !(c->eps >= 0.f)) return PYG_ERR_INVALID_ARG;
    if (c->N >= (int64_t(1) << 31) || c->F > 8192) return PYG_ERR_UNSUPPORTED;
    if (c->post_bias && !c->post_weight) return PYG_ERR_INVALID_ARG;
    if (c->bias && !c->weight) return PYG_ERR_INVALID_ARG;
    return PYG_OK;
}

Norm fill(const pyg_block_norm_args *c) {
    Norm a{};
    a.N = c->N, a.F = static_cast<int>(c->F), a.layer = c->norm == PYG_NORM_LAYER, a.eps = c->eps, a.inv_F = 1.f / c->F;
    a.h = c->h, a.residual = c->residual, a.gate = c->gate, a.gate_rows = c->gate_rows != 0;
    a.scale = c->scale, a.post_w = c->post_weight, a.post_b = c->post_bias, a.w = c->weight, a.b = c->bias;
    a.post = c->post_weight, a.pre = c->weight;
    a.blocks = (a.F + 31) / 32;
    return a;
}

// What both directions read.
struct Inputs {
    Span s[8];
};
Inputs inputs_of(const pyg_block_norm_args *c) {
    const int64_t rows = c->N * (c->dtype == PYG_BF16 ? 2 : 4), all = rows * c->F, p = c->F * 4;
    return {{{c->h, all}, {c->residual, all}, {c->gate, c->gate_rows ? rows : all}, {c->scale, p}, {c->post_weight, p},
             {c->post_bias, p}, {c->weight, p}, {c->bias, p}}};
}

}  // namespace
}  // namespace pyg

using namespace pyg;

extern "C" int pyg_block_norm(const pyg_block_norm_args *c, void *r, void *y, int8_t *codes, uint8_t *steps, void *stream) {
    PYG_TRY(check(c));
    if ((codes == nullptr) != (steps == nullptr) || (!c->weight && (y || codes))) return PYG_ERR_INVALID_ARG;
    if (c->weight && !y && c->N > 0) return PYG_ERR_INVALID_ARG;
    if (c->N == 0) return PYG_OK;
    if (!c->h || (!r && !y) || reinterpret_cast<uintptr_t>(codes) % 16) return PYG_ERR_INVALID_ARG;
    const int64_t all = c->N * c->F * (c->dtype == PYG_BF16 ? 2 : 4), blocks = c->N * ((c->F + 31) / 32);
    const Span results[] = {{r, all}, {y, all}, {codes, blocks * 32}, {steps, blocks}};
    if (!apart(results, inputs_of(c).s)) return PYG_ERR_INVALID_ARG;
    Norm a = fill(c);
    a.r = r, a.y = y, a.codes = codes, a.steps = steps;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return c->dtype == PYG_BF16 ? by_shape<__bf16, false>(a, 0, s) : by_shape<float, false>(a, 0, s);
}

extern "C" int pyg_block_norm_backward_workspace(const pyg_block_norm_args *c, size_t *bytes) {
    if (!bytes) return PYG_ERR_INVALID_ARG;
    PYG_TRY(check(c));
    *bytes = static_cast<size_t>(grad_groups(c)) * 5 * c->F * sizeof(float);
    return PYG_OK;
}

extern "C" int pyg_block_norm_backward(const pyg_block_norm_args *c, const void *grad_r, const void *grad_y, void *grad_h,
                                       void *grad_residual, void *grad_gate, float *grad_scale, float *grad_post_weight,
                                       float *grad_post_bias, float *grad_weight, float *grad_bias, void *ws,
                                       size_t ws_bytes, void *stream) {
    PYG_TRY(check(c));
    if (c->N > 0 && (!c->h || (!grad_r && !grad_y))) return PYG_ERR_INVALID_ARG;
    if (grad_y && !c->weight) return PYG_ERR_INVALID_ARG;
    if ((grad_residual && !c->residual) || (grad_gate && !c->gate) || (grad_scale && !c->scale) ||
        (grad_post_weight && !c->post_weight) || (grad_post_bias && !c->post_bias) || (grad_weight && !c->weight) ||
        (grad_bias && !c->bias))
        return PYG_ERR_INVALID_ARG;
    const int64_t groups = grad_groups(c);
    if (ws_bytes < static_cast<size_t>(groups) * 5 * c->F * sizeof(float) || !ws) return PYG_ERR_WORKSPACE;
    const int64_t rows = c->N * (c->dtype == PYG_BF16 ? 2 : 4), all = rows * c->F, p = c->F * 4;
    const Span results[] = {{grad_h, all}, {grad_residual, all}, {grad_gate, c->gate_rows ? rows : all}, {grad_scale, p},
                            {grad_post_weight, p}, {grad_post_bias, p}, {grad_weight, p}, {grad_bias, p}, {ws, groups * 5 * p}};
    const Span grads[] = {{grad_r, all}, {grad_y, all}};
    if (!apart(results, inputs_of(c).s) || !apart(results, grads)) return PYG_ERR_INVALID_ARG;
    Norm a = fill(c);
    a.grad_r = grad_r, a.grad_y = grad_y, a.grad_h = grad_h, a.grad_residual = grad_residual, a.grad_gate = grad_gate;
    a.part = static_cast<float *>(ws);
    Columns cols{};
    int n = 0;
    auto place = [&](float *out) {
        if (!out) return -1;
        cols.out[n] = out;
        return n++;
    };
    a.need_scale = place(grad_scale), a.need_post_w = place(grad_post_weight), a.need_post_b = place(grad_post_bias),
    a.need_w = place(grad_weight), a.need_b = place(grad_bias);
    a.sums = n;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int rc = c->dtype == PYG_BF16 ? by_shape<__bf16, true>(a, groups, s) : by_shape<float, true>(a, groups, s);
    if (rc != PYG_OK) return rc;
    if (n > 0) {
        const int64_t all = (int64_t)n * a.F;
        k_join_columns<<<static_cast<unsigned>((all + 63) / 64), 1024, 0, s>>>(a.part, static_cast<int>(groups), n, a.F, cols);
        PYG_LAUNCH_CHECK();
    }
    return PYG_OK;
}
