// The norms around a block of a transformer, with its gate and residual scale:
//   u = norm(h; post),  r = residual + scale * sigmoid(gate) * u,  y = norm(r; pre),
// norm(x) = (x - mean) / sqrt(var + eps) w + b (layer) or x / sqrt(mean x^2 + eps) w
// (rms); each part may be left out.
//
// Bound by memory: every input is read once and r and y written once, a row
// staying in registers between. L lanes share a row (a 16-lane group, a
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

template <typename T, int NV>
struct Row {
    static constexpr int E = 16 / sizeof(T);
    float v[NV * E];
};

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

// One piece of a row from feature f on: zeros past F.
template <typename T>
__device__ __forceinline__ void load_piece(const T *__restrict__ row, int f, int F, float *v) {
    constexpr int E = 16 / sizeof(T);
    if (f + E <= F) {
        const u32x4 u = *reinterpret_cast<const u32x4_any *>(row + f);
        unpack16<T>(u, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = f + i < F ? static_cast<float>(row[f + i]) : 0.f;
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

// Sums over the L lanes of a row, K at once.
template <int L, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float *lds) {
    constexpr int W = L < 64 ? L : 64;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int o = W / 2; o > 0; o >>= 1) v[k] += __shfl_xor(v[k], o);
    if constexpr (L > 64) {
        constexpr int waves = L / 64;
        const int wave = threadIdx.x >> 6;
        __syncthreads();
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
    static __device__ __forceinline__ void load(const void *p, int64_t row, int F, int lane, float (&v)[M]) {
        const T *x = static_cast<const T *>(p) + row * F;
#pragma unroll
        for (int i = 0; i < NV; ++i) load_piece<T>(x, feature(lane, i), F, v + i * E);
    }
    static __device__ __forceinline__ void store(void *p, int64_t row, int F, int lane, const float (&v)[M]) {
        T *x = static_cast<T *>(p) + row * F;
#pragma unroll
        for (int i = 0; i < NV; ++i) store_piece<T>(x, feature(lane, i), F, v + i * E);
    }
    // a [F] parameter in fp32, `other` where it is missing
    static __device__ __forceinline__ void load_param(const float *p, int F, int lane, float other, float (&v)[M]) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int f = feature(lane, i) + e;
                v[i * E + e] = !p ? other : f < F ? p[f] : 0.f;
            }
    }
    static __device__ __forceinline__ bool inside(int lane, int k, int F) { return feature(lane, k / E) + k % E < F; }

    // x -> its normalised values; returns 1 / deviation
    static __device__ __forceinline__ float normalise(float (&x)[M], const Norm &a, int lane, float *lds) {
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
        const float rstd = 1.f / sqrtf(fmaf(q[0], a.inv_F, a.eps));
#pragma unroll
        for (int k = 0; k < M; ++k) x[k] *= rstd;
        return rstd;
    }
    // gradient t of the normalised values n -> gradient of x
    static __device__ __forceinline__ void through(float (&t)[M], const float (&n)[M], float rstd, const Norm &a, int lane,
                                                   float *lds) {
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < M; ++k) s[0] = fmaf(t[k], n[k], s[0]), s[1] += t[k];
        row_sums<L, 2>(s, lds);
        const float tn = s[0] * a.inv_F, tm = a.layer ? s[1] * a.inv_F : 0.f;
#pragma unroll
        for (int k = 0; k < M; ++k) t[k] = inside(lane, k, a.F) ? (t[k] - n[k] * tn - tm) * rstd : 0.f;
    }
};

__device__ __forceinline__ float sigmoid(float x) { return 1.f / (1.f + expf(-x)); }

constexpr int kRowLds = 2 * 16;  // sums of a workgroup's wavefronts

template <typename T, int L, int NV>
__global__ __launch_bounds__(L < 256 ? 256 : L) void k_block_norm(const Norm a) {
    using B = Body<T, L, NV>;
    constexpr int M = B::M, E = B::E, R = (L < 256 ? 256 : L) / L;
    __shared__ float lds[kRowLds];
    const int lane = threadIdx.x % L;
    float sc[M], pw[M], pb[M], w[M], b[M];
    B::load_param(a.scale, a.F, lane, 1.f, sc);
    B::load_param(a.post_w, a.F, lane, 1.f, pw);
    B::load_param(a.post_b, a.F, lane, 0.f, pb);
    B::load_param(a.w, a.F, lane, 1.f, w);
    B::load_param(a.b, a.F, lane, 0.f, b);
    for (int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / L; row < a.N; row += (int64_t)gridDim.x * R) {
        float x[M], res[M], g[M];
        B::load(a.h, row, a.F, lane, x);
        if (a.residual) B::load(a.residual, row, a.F, lane, res);
        float gr = 0.f;
        if (a.gate && !a.gate_rows) B::load(a.gate, row, a.F, lane, g);
        if (a.gate && a.gate_rows) gr = sigmoid(static_cast<float>(static_cast<const T *>(a.gate)[row]));
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
__global__ __launch_bounds__(L < 256 ? 256 : L) void k_block_norm_grad(const Norm a) {
    using B = Body<T, L, NV>;
    constexpr int M = B::M, E = B::E, NT = L < 256 ? 256 : L, R = NT / L;
    __shared__ float lds[kRowLds];
    __shared__ float cols[R > 1 ? R * L * M : 1];
    const int lane = threadIdx.x % L;
    float s_sc[M], s_pw[M], s_pb[M], s_w[M], s_b[M];
#pragma unroll
    for (int k = 0; k < M; ++k) s_sc[k] = s_pw[k] = s_pb[k] = s_w[k] = s_b[k] = 0.f;
    for (int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / L; row < a.N; row += (int64_t)gridDim.x * R) {
        float nh[M], sg[M], nr[M], t[M], p[M], gy[M];
        B::load(a.h, row, a.F, lane, nh);
        if (a.residual) B::load(a.residual, row, a.F, lane, nr);
        if (a.gate && !a.gate_rows) B::load(a.gate, row, a.F, lane, sg);
        if (a.grad_y) B::load(a.grad_y, row, a.F, lane, gy);
        if (a.grad_r) B::load(a.grad_r, row, a.F, lane, t);
        float gr = 1.f;
        if (a.gate && a.gate_rows) gr = sigmoid(static_cast<float>(static_cast<const T *>(a.gate)[row]));
        float rstd_h = 0.f;
        if (a.post) rstd_h = B::normalise(nh, a, lane, lds);
        float sc[M], u[M];
        B::load_param(a.scale, a.F, lane, 1.f, sc);
        B::load_param(a.post_w, a.F, lane, 1.f, p);
#pragma unroll
        for (int k = 0; k < M; ++k) u[k] = nh[k];
        if (a.post) {
            float pb[M];
            B::load_param(a.post_b, a.F, lane, 0.f, pb);
#pragma unroll
            for (int k = 0; k < M; ++k) u[k] = fmaf(nh[k], p[k], pb[k]);
        }
#pragma unroll
        for (int k = 0; k < M; ++k) {
            sg[k] = !a.gate ? 1.f : a.gate_rows ? gr : sigmoid(sg[k]);
            const float c = sc[k] * sg[k] * u[k];
            nr[k] = !B::inside(lane, k, a.F) ? 0.f : a.residual ? nr[k] + c : c;
            if (!a.grad_r) t[k] = 0.f;
        }
        if (a.pre && a.grad_y) {
            const float rstd_r = B::normalise(nr, a, lane, lds);
            float w[M];
            B::load_param(a.w, a.F, lane, 1.f, w);
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
            s_sc[k] = fmaf(t[k] * sg[k], u[k], s_sc[k]);
            t[k] *= sc[k];
            dg[k] = t[k] * u[k] * sg[k] * (1.f - sg[k]);
            row_gate[0] += dg[k];
            t[k] *= sg[k];  // the gradient of u
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

int64_t most_groups(int64_t N, int F) { return F <= 512 ? 1024 : 512; }

struct Shape {
    int L, NV;
};
// Lanes of a row: groups of 16 up to one piece each, a wavefront up to two, then workgroups.
Shape shape_of(int64_t F, int E) {
    const int64_t v = (F + E - 1) / E;
    if (v <= 16) return {16, 1};
    if (v <= 64) return {64, 1};
    if (v <= 128) return {64, 2};
    if (v <= 256) return {256, 1};
    if (v <= 512) return {256, 2};
    if (v <= 1024) return {512, 2};
    return {1024, 2};
}

template <typename T, int L, int NV>
int launch(const Norm &a, bool backward, int64_t groups, hipStream_t s) {
    constexpr int NT = L < 256 ? 256 : L, R = NT / L;
    if (backward) k_block_norm_grad<T, L, NV><<<static_cast<unsigned>(groups), NT, 0, s>>>(a);
    else k_block_norm<T, L, NV><<<grid_for(a.N, R, 2048 * 256 / NT), NT, 0, s>>>(a);
    PYG_LAUNCH_CHECK();
    return PYG_OK;
}

template <typename T>
int by_shape(const Norm &a, bool backward, int64_t groups, hipStream_t s) {
    const Shape h = shape_of(a.F, 16 / sizeof(T));
    if (h.L == 16) return launch<T, 16, 1>(a, backward, groups, s);
    if (h.L == 64) return h.NV == 1 ? launch<T, 64, 1>(a, backward, groups, s) : launch<T, 64, 2>(a, backward, groups, s);
    if (h.L == 256) return h.NV == 1 ? launch<T, 256, 1>(a, backward, groups, s) : launch<T, 256, 2>(a, backward, groups, s);
    if constexpr (sizeof(T) == 4)
        if (h.L == 1024) return launch<T, 1024, 2>(a, backward, groups, s);  // bf16 rows end at 1,024 pieces
    return launch<T, 512, 2>(a, backward, groups, s);
}

int64_t grad_groups(const pyg_block_norm_args *c) {
    const int E = c->dtype == PYG_BF16 ? 8 : 4;
    const Shape h = shape_of(c->F, E);
    const int64_t R = (h.L < 256 ? 256 : h.L) / h.L, rows = (c->N + R - 1) / R, most = most_groups(c->N, (int)c->F);
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

}  // namespace
}  // namespace pyg

using namespace pyg;

extern "C" int pyg_block_norm(const pyg_block_norm_args *c, void *r, void *y, int8_t *codes, uint8_t *steps, void *stream) {
    PYG_TRY(check(c));
    if ((codes == nullptr) != (steps == nullptr) || (!c->weight && (y || codes))) return PYG_ERR_INVALID_ARG;
    if (c->weight && !y && c->N > 0) return PYG_ERR_INVALID_ARG;
    if (c->N == 0) return PYG_OK;
    if (!c->h || (!r && !y)) return PYG_ERR_INVALID_ARG;
    Norm a = fill(c);
    a.r = r, a.y = y, a.codes = codes, a.steps = steps;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return c->dtype == PYG_BF16 ? by_shape<__bf16>(a, false, 0, s) : by_shape<float>(a, false, 0, s);
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
    PYG_TRY(c->dtype == PYG_BF16 ? by_shape<__bf16>(a, true, groups, s) : by_shape<float>(a, true, groups, s));
    if (n > 0) {
        const int64_t all = (int64_t)n * a.F;
        k_join_columns<<<static_cast<unsigned>((all + 63) / 64), 1024, 0, s>>>(a.part, static_cast<int>(groups), n, a.F, cols);
        PYG_LAUNCH_CHECK();
    }
    return PYG_OK;
}
