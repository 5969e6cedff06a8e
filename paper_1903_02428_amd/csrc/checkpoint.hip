// Activations in 8 bits and back, and the gradients of the dense transform from
// them: dTheta = X^T G on the matrix cores with X straight from its codes.
//
// A code times its step is a bf16 value, so X enters v_mfma_f32_32x32x16_bf16
// unrounded; bf16 gradients too. fp32 gradients are cut into three bf16 parts that add
// up to them, three exact products instead of fp32 instructions at an eighth of the rate.
// The products contract over the rows n, which both operands hold as rows: tiles of
// 32 rows go to LDS as they lie, and the transposing LDS read makes the operands.
#include "attn_tiles.hpp"
#include "eight_bit.hpp"

namespace pyg {
namespace {

using attn::f32x16;

// One thread a piece of 16 bytes of x: E lanes' neighbours share a block of 32.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_checkpoint(const T *__restrict__ x, int64_t N, int F, int pieces,
                                                       uint8_t *__restrict__ codes, uint8_t *__restrict__ steps) {
    constexpr int E = 16 / sizeof(T);
    const int64_t all = N * pieces, step = (int64_t)gridDim.x * kBlock;
    for (int64_t i = blockIdx.x * (int64_t)kBlock + threadIdx.x; i < all; i += step) {  // pieces * E is a multiple of 32:
        const int64_t row = i / pieces;                                                 // blocks stay in 8 or 4 lanes
        const int f = static_cast<int>(i - row * pieces) * E;
        attn::Piece<T> p;
        p.u = attn::load_piece<T>(x + row * F, f, F, true);
        float v[E];
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            v[e] = static_cast<float>(p.v[e]);
            const uint32_t m = eight::magnitude(v[e]);
            top = m > top ? m : top;
        }
#pragma unroll
        for (int o = 1; o < 32 / E; o <<= 1) {
            const uint32_t m = __shfl_xor(top, o);
            top = m > top ? m : top;
        }
        const uint32_t ex = eight::step_of(top);
        const float inv = eight::step_inverse(ex);
        uint32_t q[E / 4];
#pragma unroll
        for (int j = 0; j < E / 4; ++j)
            q[j] = eight::code(v[4 * j], inv, ex) | eight::code(v[4 * j + 1], inv, ex) << 8 |
                   eight::code(v[4 * j + 2], inv, ex) << 16 | eight::code(v[4 * j + 3], inv, ex) << 24;
        uint8_t *c = codes + i * E;
        if constexpr (E == 4) *reinterpret_cast<uint32_t *>(c) = q[0];
        else *reinterpret_cast<uint2 *>(c) = make_uint2(q[0], q[E / 4 - 1]);
        if (f % 32 == 0) steps[i * E / 32] = static_cast<uint8_t>(ex);
    }
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_restore(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ steps,
                                                    int64_t N, int F, int pieces, bool vec, T *__restrict__ x) {
    constexpr int E = 16 / sizeof(T);
    const int64_t all = N * pieces, step = (int64_t)gridDim.x * kBlock;
    for (int64_t i = blockIdx.x * (int64_t)kBlock + threadIdx.x; i < all; i += step) {
        const int64_t row = i / pieces;
        const int f = static_cast<int>(i - row * pieces) * E;
        if (f >= F) continue;
        const float s = eight::step_value(steps[i * E / 32]);
        attn::Piece<T> p;
#pragma unroll
        for (int j = 0; j < E / 4; ++j) {
            float v[4];
            eight::unpack(*reinterpret_cast<const uint32_t *>(codes + i * E + 4 * j), v);
#pragma unroll
            for (int e = 0; e < 4; ++e) p.v[4 * j + e] = T(v[e] * s);
        }
        T *o = x + row * F + f;
        if (vec) {
            *reinterpret_cast<uint4 *>(o) = p.u;
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (f + e < F) o[e] = p.v[e];
        }
    }
}

// ------------------------------------------------------------ dTheta = X^T G

constexpr int kTileI = 128, kTileO = 128, kTileN = 32;
typedef __bf16 bf16;
using Rows = attn::Tile<bf16, 128>;

// One 16-byte piece of an operand as PARTS bf16 pieces, part k at place(k): bf16 values as they are, fp32 ones as the
// nearest bf16 value, the nearest to what is left, and the rest: exactly, since what is left of a value of exponent
// e is a multiple of 2^(e - 23) and at most 2^(e - 8), then at most 2^(e - 17). Parts have either sign.
template <typename T, int PARTS, typename PLACE>
__device__ __forceinline__ void put_parts(uint4 piece, PLACE place) {
    if constexpr (PARTS == 1) {
        *reinterpret_cast<uint4 *>(place(0)) = piece;
    } else {
        attn::Piece<T> v;
        v.u = piece;
        float f[4] = {v.v[0], v.v[1], v.v[2], v.v[3]};
        bool huge = false;  // the nearest bf16 value is an infinity, or the value is one or a NaN
#pragma unroll
        for (int e = 0; e < 4; ++e) huge |= (__float_as_uint(f[e]) & 0x7FFFFFFFu) >= 0x7F7F8000u;
#pragma unroll
        for (int k = 0; k < PARTS; ++k) {
            uint32_t b[2] = {attn::pack_bf16(f[0], f[1]), attn::pack_bf16(f[2], f[3])};
            if (k == 0 && __any(huge)) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t u = __float_as_uint(f[e]), m = u & 0x7FFFFFFFu;
                    if (m >= 0x7F7F8000u && m < 0x7F800000u)  // finite: its first 8 bits, and so in what is left
                        b[e / 2] = e & 1 ? (b[e / 2] & 0xFFFFu) | (u & 0xFFFF0000u) : (b[e / 2] & 0xFFFF0000u) | u >> 16;
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] -= __uint_as_float(e & 1 ? b[e / 2] & 0xFFFF0000u : b[e / 2] << 16);
            if (k == 0 && __any(huge)) {
#pragma unroll
                for (int e = 0; e < 4; ++e) f[e] = f[e] == f[e] ? f[e] : 0.f;  // an infinity or NaN is all in the first part
            }
            *reinterpret_cast<uint2 *>(place(k)) = make_uint2(b[0], b[1]);
        }
    }
}

// A workgroup owns 128 x 128 of dTheta and every splits-th tile of 32 rows. PARTS
// bf16 parts of G (1: bf16 G, 3: fp32 G).
template <typename T, int PARTS>
__global__ __launch_bounds__(kBlock) void k_theta_grad(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ steps,
                                                       const T *__restrict__ g, int64_t N, int Fi, int Fo, int blocks,
                                                       int splits, float *__restrict__ part) {
    constexpr int E = 16 / sizeof(T), GP = kTileN * kTileO / E / kBlock;
    __shared__ __align__(16) char xt[Rows::bytes<kTileN>()];
    __shared__ __align__(16) char gt[PARTS][Rows::bytes<kTileN>()];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int tiles_o = (Fo + kTileO - 1) / kTileO;
    const int sp = blockIdx.x % splits, tile = blockIdx.x / splits;
    const int i0 = tile / tiles_o * kTileI, o0 = tile % tiles_o * kTileO;
    const int wi = wave / 2 * 64, wo = wave % 2 * 64;  // the wavefront's 64 x 64
    const int64_t width = (int64_t)blocks * 32;
    const Rows::ColLane cl(lane);
    f32x16 acc[2][2];
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b) acc[a][b] = f32x16(0.f);

    // 16 codes and their step, and GP pieces of G a thread
    const int xr = threadIdx.x / 8, xc = threadIdx.x % 8 * 16;
    uint4 cx;
    uint32_t ex;
    uint4 cg[GP];
    auto load = [&](int64_t n0) {
        cx = make_uint4(0, 0, 0, 0);
        ex = 1;
        if (n0 + xr < N && i0 + xc < width) {
            cx = *reinterpret_cast<const uint4 *>(codes + (n0 + xr) * width + i0 + xc);
            ex = steps[(n0 + xr) * blocks + (i0 + xc) / 32];
        }
#pragma unroll
        for (int j = 0; j < GP; ++j) {
            const int p = j * kBlock + threadIdx.x, r = p / (kTileO / E), c = p % (kTileO / E) * E;
            cg[j] = attn::load_piece<T>(g + (n0 + r) * Fo, o0 + c, Fo, n0 + r < N);
        }
    };
    auto store = [&]() {
        const float s = eight::step_value(ex);
        const uint32_t w[4] = {cx.x, cx.y, cx.z, cx.w};
        uint32_t o[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float v[4];
            eight::unpack(w[j], v);
            o[2 * j] = attn::pack_bf16(v[0] * s, v[1] * s), o[2 * j + 1] = attn::pack_bf16(v[2] * s, v[3] * s);  // exact
        }
        char *x = xt + xr * Rows::kRowBytes;
        const int sw = attn::swizzle<Rows::C>(xr);
        *reinterpret_cast<uint4 *>(x + ((xc / 8 ^ sw) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
        *reinterpret_cast<uint4 *>(x + ((xc / 8 + 1 ^ sw) << 4)) = make_uint4(o[4], o[5], o[6], o[7]);
#pragma unroll
        for (int j = 0; j < GP; ++j) {
            const int p = j * kBlock + threadIdx.x, r = p / (kTileO / E), c = p % (kTileO / E) * E;
            put_parts<T, PARTS>(cg[j], [&](int k) {
                return gt[k] + r * Rows::kRowBytes + ((c / 8 ^ attn::swizzle<Rows::C>(r)) << 4) + c % 8 * 2;
            });
        }
    };
    int64_t n0 = (int64_t)sp * kTileN;
    if (n0 < N) load(n0);
    for (; n0 < N; n0 += (int64_t)splits * kTileN) {
        __syncthreads();
        store();
        __syncthreads();
        if (n0 + (int64_t)splits * kTileN < N) load(n0 + (int64_t)splits * kTileN);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            uint4 a[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) a[t] = Rows::col_piece(xt, cl, 0, wi / 32 + t, u);
#pragma unroll
            for (int k = PARTS - 1; k >= 0; --k)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const uint4 y = Rows::col_piece(gt[k], cl, 0, wo / 32 + b, u);
#pragma unroll
                    for (int t = 0; t < 2; ++t) acc[t][b] = attn::mma<bf16>(a[t], y, acc[t][b]);
                }
        }
    }
    float *p = part + (int64_t)sp * Fi * Fo;
    const int h = lane >> 5;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int o = o0 + wo + 32 * b + (lane & 31);
            if (o >= Fo) continue;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int i = i0 + wi + 32 * t + 8 * (r >> 2) + 4 * h + (r & 3);
                if (i < Fi) p[(int64_t)i * Fo + o] = acc[t][b][r];
            }
        }
}

// ------------------------------------------------------------- dX = G Theta^T

// Both operands contract over the features o they hold adjacent, so rows go to LDS as they lie
// and come back as row pieces. fp32 operands are three bf16 parts each; of the nine products the six with a + b <= 2
// (parts a, b) are taken, smallest first. The others come to less than 2^-24 of the whole product, half a
// step of fp32, with either sign. Six at the bf16 rate (1,220 TFLOP/s) are 1.3 times the fp32 instructions' rate (154).
// A workgroup owns 128 rows and 128 of the Fi columns, a wavefront
// 64 x 64; Theta is the A operand, so that a lane ends with four adjacent features of one row.
template <typename T, int PARTS>
__global__ __launch_bounds__(kBlock) void k_input_grad(const T *__restrict__ g, const T *__restrict__ theta, int64_t N, int Fi,
                                                       int Fo, int tiles_i, bool vec, T *__restrict__ out) {
    using Rows = attn::Tile<bf16, 32>;
    constexpr int E = 16 / sizeof(T), GP = 128 * 32 / E / kBlock;
    __shared__ __align__(16) char gt[PARTS][Rows::bytes<128>()], tt[PARTS][Rows::bytes<128>()];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
    const int64_t n0 = (int64_t)(blockIdx.x / tiles_i) * 128;
    const int i0 = blockIdx.x % tiles_i * 128;
    const int wi = wave / 2 * 2, wn = wave % 2 * 2;  // the wavefront's blocks of 32
    const Rows::RowLane rl(lane);
    f32x16 acc[2][2];
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b) acc[a][b] = f32x16(0.f);
    uint4 cg[GP], ct[GP];
    auto load = [&](int o0) {
#pragma unroll
        for (int j = 0; j < GP; ++j) {
            const int p = j * kBlock + threadIdx.x, r = p / (32 / E), c = o0 + p % (32 / E) * E;
            cg[j] = attn::load_piece<T>(g + (n0 + r) * Fo, c, Fo, n0 + r < N);
            ct[j] = attn::load_piece<T>(theta + (int64_t)(i0 + r) * Fo, c, Fo, i0 + r < Fi);
        }
    };
    auto store = [&](const uint4 (&v)[GP], char (&tile)[PARTS][Rows::bytes<128>()]) {
#pragma unroll
        for (int j = 0; j < GP; ++j) {
            const int p = j * kBlock + threadIdx.x, r = p / (32 / E), c = p % (32 / E) * E;
            put_parts<T, PARTS>(v[j], [&](int k) {
                return tile[k] + r * Rows::kRowBytes + ((c / 8 ^ attn::swizzle<Rows::C>(r)) << 4) + c % 8 * 2;
            });
        }
    };
    load(0);
    for (int o0 = 0; o0 < Fo; o0 += 32) {
        __syncthreads();
        store(cg, gt);
        store(ct, tt);
        __syncthreads();
        if (o0 + 32 < Fo) load(o0 + 32);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            uint4 a[PARTS][2], b[PARTS][2];
#pragma unroll
            for (int k = 0; k < PARTS; ++k)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    a[k][t] = Rows::row_piece(tt[k], rl, wi + t, u);
                    b[k][t] = Rows::row_piece(gt[k], rl, wn + t, u);
                }
#pragma unroll
            for (int sum = PARTS - 1; sum >= 0; --sum)
#pragma unroll
                for (int k = 0; k <= sum; ++k)
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int y = 0; y < 2; ++y) acc[x][y] = attn::mma<bf16>(a[k][x], b[sum - k][y], acc[x][y]);
        }
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
        const int64_t n = n0 + 32 * (wn + y) + (lane & 31);
        if (n >= N) continue;
        T *o = out + n * Fi;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int i = i0 + 32 * (wi + x) + 8 * q + 4 * h;
                if (i >= Fi) continue;
                const float v[4] = {acc[x][y][4 * q], acc[x][y][4 * q + 1], acc[x][y][4 * q + 2], acc[x][y][4 * q + 3]};
                if (vec) {
                    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(o + i) = make_float4(v[0], v[1], v[2], v[3]);
                    else *reinterpret_cast<uint2 *>(o + i) = make_uint2(attn::pack_bf16(v[0], v[1]), attn::pack_bf16(v[2], v[3]));
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (i + e < Fi) o[i + e] = T(v[e]);
                }
            }
    }
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_join_theta(const float *__restrict__ part, int64_t n, int splits,
                                                       T *__restrict__ out) {
    // 32 values at a time, 8 threads a value
    __shared__ float lds[8][32];
    const int i = threadIdx.x & 31, r = threadIdx.x >> 5;
    for (int64_t first = (int64_t)blockIdx.x * 32; first < n; first += (int64_t)gridDim.x * 32) {
        const int64_t at = first + i;
        float v = 0.f;
        if (at < n)
#pragma unroll 8
            for (int s = r; s < splits; s += 8) v += part[(int64_t)s * n + at];
        lds[r][i] = v;
        __syncthreads();
        if (r == 0 && at < n) {
            for (int k = 1; k < 8; ++k) v += lds[k][i];
            out[at] = T(v);
        }
        __syncthreads();
    }
}

constexpr int64_t kMax32 = int64_t(1) << 31, kMaxF = int64_t(1) << 24;

// Row ranges of dTheta: two workgroups a CU, 128 rows or more each (19,717 rows, 500 to 64 features, bf16:
// 256 rows 20 us, 128 18).
int64_t theta_tiles(int64_t Fi, int64_t Fo) { return ((Fi + kTileI - 1) / kTileI) * ((Fo + kTileO - 1) / kTileO); }
int splits_of(int64_t N, int64_t Fi, int64_t Fo) {
    const int64_t tiles = theta_tiles(Fi, Fo);
    int64_t s = 512 / tiles, most = N / 128;
    s = s < most ? s : most;
    return static_cast<int>(s < 1 ? 1 : s);
}

bool aligned(const void *p, int64_t row_bytes) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && row_bytes % 16 == 0; }

template <typename T>
int theta_grad(const T *g, int64_t N, int Fo, int Fi, const int8_t *codes, const uint8_t *steps, T *out, float *part,
               hipStream_t s) {
    const int splits = splits_of(N, Fi, Fo), blocks = (Fi + 31) / 32;
    const int64_t tiles = theta_tiles(Fi, Fo), n = (int64_t)Fi * Fo;
    k_theta_grad<T, sizeof(T) == 2 ? 1 : 3><<<static_cast<unsigned>(tiles * splits), kBlock, 0, s>>>(
        reinterpret_cast<const uint8_t *>(codes), steps, g, N, Fi, Fo, blocks, splits, part);
    PYG_LAUNCH_CHECK();
    k_join_theta<T><<<grid_for(n, 32), kBlock, 0, s>>>(part, n, splits, out);
    PYG_LAUNCH_CHECK();
    return PYG_OK;
}

}  // namespace
}  // namespace pyg

using namespace pyg;

extern "C" int pyg_activation_checkpoint(const void *x, int dtype, int64_t N, int64_t F, int8_t *codes, uint8_t *steps,
                                         void *stream) {
    if ((dtype != PYG_F32 && dtype != PYG_BF16) || N < 0 || F < 1) return PYG_ERR_INVALID_ARG;
    if (N >= kMax32 || F >= kMaxF) return PYG_ERR_UNSUPPORTED;
    if (N == 0) return PYG_OK;
    if (!x || !codes || !steps || reinterpret_cast<uintptr_t>(codes) % 16) return PYG_ERR_INVALID_ARG;
    const Span results[] = {{codes, N * ((F + 31) / 32) * 32}, {steps, N * ((F + 31) / 32)}};
    const Span inputs[] = {{x, N * F * (dtype == PYG_BF16 ? 2 : 4)}};
    if (!apart(results, inputs)) return PYG_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int width = static_cast<int>((F + 31) / 32 * 32), f = static_cast<int>(F);
    uint8_t *c = reinterpret_cast<uint8_t *>(codes);
    const unsigned grid = grid_for(N * (width / (dtype == PYG_BF16 ? 8 : 4)), kBlock, 1 << 16);
    if (dtype == PYG_BF16)
        k_checkpoint<__bf16><<<grid, kBlock, 0, s>>>(static_cast<const __bf16 *>(x), N, f, width / 8, c, steps);
    else
        k_checkpoint<float><<<grid, kBlock, 0, s>>>(static_cast<const float *>(x), N, f, width / 4, c, steps);
    PYG_LAUNCH_CHECK();
    return PYG_OK;
}

extern "C" int pyg_checkpoint_restore(const int8_t *codes, const uint8_t *steps, int64_t N, int64_t F, void *x, int dtype,
                                      void *stream) {
    if ((dtype != PYG_F32 && dtype != PYG_BF16) || N < 0 || F < 1) return PYG_ERR_INVALID_ARG;
    if (N >= kMax32 || F >= kMaxF) return PYG_ERR_UNSUPPORTED;
    if (N == 0) return PYG_OK;
    if (!x || !codes || !steps || reinterpret_cast<uintptr_t>(codes) % 16) return PYG_ERR_INVALID_ARG;
    const Span inputs[] = {{codes, N * ((F + 31) / 32) * 32}, {steps, N * ((F + 31) / 32)}};
    const Span results[] = {{x, N * F * (dtype == PYG_BF16 ? 2 : 4)}};
    if (!apart(results, inputs)) return PYG_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int width = static_cast<int>((F + 31) / 32 * 32), f = static_cast<int>(F);
    const uint8_t *c = reinterpret_cast<const uint8_t *>(codes);
    const unsigned grid = grid_for(N * (width / (dtype == PYG_BF16 ? 8 : 4)), kBlock, 1 << 16);
    if (dtype == PYG_BF16)
        k_restore<__bf16><<<grid, kBlock, 0, s>>>(c, steps, N, f, width / 8, aligned(x, F * 2), static_cast<__bf16 *>(x));
    else
        k_restore<float><<<grid, kBlock, 0, s>>>(c, steps, N, f, width / 4, aligned(x, F * 4), static_cast<float *>(x));
    PYG_LAUNCH_CHECK();
    return PYG_OK;
}

namespace {

int check_dense(int dtype, int64_t N, int64_t Fi, int64_t Fo, size_t *bytes) {
    if ((dtype != PYG_F32 && dtype != PYG_BF16) || N < 0 || Fi < 1 || Fo < 1) return PYG_ERR_INVALID_ARG;
    if (N >= kMax32 || Fi >= kMaxF || Fo >= kMaxF) return PYG_ERR_UNSUPPORTED;
    *bytes = static_cast<size_t>(splits_of(N, Fi, Fo)) * Fi * Fo * sizeof(float);
    return PYG_OK;
}

template <typename T>
int input_grad(const T *g, const T *theta, int64_t N, int Fi, int Fo, T *out, hipStream_t s) {
    const int tiles_i = (Fi + 127) / 128;
    k_input_grad<T, sizeof(T) == 2 ? 1 : 3><<<static_cast<unsigned>((N + 127) / 128 * tiles_i), kBlock, 0, s>>>(
        g, theta, N, Fi, Fo, tiles_i, Fi % 4 == 0 && reinterpret_cast<uintptr_t>(out) % 16 == 0, out);
    PYG_LAUNCH_CHECK();
    return PYG_OK;
}

}  // namespace

extern "C" int pyg_dense_transform_backward_workspace(int dtype, int64_t N, int64_t Fi, int64_t Fo, size_t *bytes) {
    return bytes ? check_dense(dtype, N, Fi, Fo, bytes) : PYG_ERR_INVALID_ARG;
}

extern "C" int pyg_dense_transform_backward(const void *grad_out, int dtype, int64_t N, int64_t Fo, const void *theta,
                                            int64_t Fi, const int8_t *codes, const uint8_t *steps, void *grad_x,
                                            void *grad_theta, void *ws, size_t ws_bytes, void *stream) {
    size_t need = 0;
    PYG_TRY(check_dense(dtype, N, Fi, Fo, &need));
    // before anything is launched: either result's grid
    constexpr int64_t most = (int64_t(1) << 32) / kBlock;
    if ((grad_x && (N + 127) / 128 * ((Fi + 127) / 128) >= most) || (grad_theta && theta_tiles(Fi, Fo) * splits_of(N, Fi, Fo) >= most))
        return PYG_ERR_UNSUPPORTED;
    if (N > 0 && !grad_out) return PYG_ERR_INVALID_ARG;
    if (grad_x && N > 0 && !theta) return PYG_ERR_INVALID_ARG;
    if (grad_theta && N > 0 && (!codes || !steps || reinterpret_cast<uintptr_t>(codes) % 16)) return PYG_ERR_INVALID_ARG;
    if (!grad_theta) need = 0;  // grad_x works without
    if (ws_bytes < need || (need && !ws)) return PYG_ERR_WORKSPACE;
    const int64_t e = dtype == PYG_BF16 ? 2 : 4, blocks = (Fi + 31) / 32;
    const Span results[] = {{grad_x, N * Fi * e}, {grad_theta, Fi * Fo * e}, {ws, static_cast<int64_t>(need)}};
    const Span inputs[] = {{grad_out, N * Fo * e}, {theta, Fi * Fo * e}, {codes, N * blocks * 32}, {steps, N * blocks}};
    if (!apart(results, inputs)) return PYG_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int fi = static_cast<int>(Fi), fo = static_cast<int>(Fo);
    float *part = static_cast<float *>(ws);
    int rc = PYG_OK;
    if (grad_x && N > 0) {
        rc = dtype == PYG_BF16 ? input_grad(static_cast<const __bf16 *>(grad_out), static_cast<const __bf16 *>(theta), N, fi, fo,
                                            static_cast<__bf16 *>(grad_x), s)
                               : input_grad(static_cast<const float *>(grad_out), static_cast<const float *>(theta), N, fi, fo,
                                            static_cast<float *>(grad_x), s);
    }
    if (rc != PYG_OK || !grad_theta) return rc;
    return dtype == PYG_BF16 ? theta_grad(static_cast<const __bf16 *>(grad_out), N, fo, fi, codes, steps,
                                          static_cast<__bf16 *>(grad_theta), part, s)
                             : theta_grad(static_cast<const float *>(grad_out), N, fo, fi, codes, steps,
                                          static_cast<float *>(grad_theta), part, s);
}
