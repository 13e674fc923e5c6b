// mp8_orthogonal_momentum_fp16_sr: a momentum step whose direction is orthogonalised before it is applied to the half-precision
// master weights (the weight-update path of Figure 1b of arXiv 1905.12334 with another rule between the gradient and the weights).
//
// Per matrix, with g the un-scaled gradient:
//   v' = mu v + g,   u = v' or, as Nesterov, g + mu v'
//   X0 = u / |u|_F;  X <- a X + (b A + c A^2) X,  A = X X^T  (steps times);   w' = w - lr (X + wd w)
// A step maps every singular value s to a s + b s^3 + c s^5 and leaves the singular vectors alone: with (a, b, c) = (3.4445,
// -4.7750, 2.0315), whose slope at zero is steep, five steps bring all but the smallest to 0.7 .. 1.2.
//
// X lies with its shorter side (m) as rows, whatever the weights' layout, so that A is m x m.  Operands of the products are
// halves, sums FP32.  A power of two keeps each of them in the format's range: singular values stay below 1.21, so that entries of A
// are below 1.46 and those of bA + cA^2 below 2.81 in magnitude; A and the polynomial are stored times 2^14, X times S = 2^round(log2
// sqrt n), which makes the entries of an orthogonal X about 1.  What half operands cost: entries of X are off by 1.3e-3 of
// their root mean square after five steps from a Gaussian u, 1.4e-2 where eight directions hold nearly all of it (bfloat16
// operands: 1e-2 and 0.11; FP32: 1.3e-6 and 5e-6).
#include <cmath>

#include "half_gemm.hpp"

namespace mp8 {

constexpr float kOrthoA = 3.4445f, kOrthoB = -4.7750f, kOrthoC = 2.0315f;
constexpr float kUp = 16384.0f, kDown = 1.0f / 16384.0f;  // the scale of A and of the polynomial

// A symmetric output of halves, made from its upper tiles: v = linear * in[r, c] + scale * acc at (r, c) and, off the diagonal's
// tiles, at (c, r).
struct OrthoSymmetric {
    const uint16_t *in;  // nullable
    uint16_t *out;
    int64_t ld, batch;   // in halves
    int m;               // rows and columns that are stored (a multiple of 8)
    float linear, scale;
    template <class T>
    __device__ __forceinline__ void operator()(const HalfPlace<T> &at, f32x16 (&acc)[T::MT][T::NT]) const {
        const uint16_t *x = in != nullptr ? in + at.batch * batch : nullptr;
        uint16_t *o = out + at.batch * batch;
        const bool mirror = at.tm != at.tn;
#pragma unroll
        for (int i = 0; i < T::MT; ++i) {
            const int r = at.row(i);
#pragma unroll
            for (int j = 0; j < T::NT; ++j) {
                if (at.col0 + 32 * j >= m) break;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int c = at.col(j) + 8 * g;
                    if (r >= m || c >= m) continue;
                    float v[4];
                    uint32_t h[4];
                    u32x2 xw = {0, 0};
                    if (x != nullptr) xw = *reinterpret_cast<const u32x2 *>(x + r * ld + c);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        v[e] = scale * acc[i][j][4 * g + e];
                        if (x != nullptr) v[e] = __builtin_fmaf(linear, half_bits_to_f32((e < 2 ? xw.x : xw.y) >> (16 * (e & 1))), v[e]);
                        h[e] = f16_from_f32<false>(v[e], 0u);
                    }
                    const u32x2 w = {h[0] | (h[1] << 16), h[2] | (h[3] << 16)};
                    *reinterpret_cast<u32x2 *>(o + r * ld + c) = w;
                    if (mirror) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[(c + e) * ld + r] = (uint16_t)h[e];
                    }
                }
            }
        }
    }
};

// The next iterate, a X + scale * acc, as halves; or, after the last step, as FP32 without X's scale.
struct OrthoNext {
    const uint16_t *x;
    uint16_t *out;     // null after the last step
    float *last;
    int64_t ld, batch; // in elements
    int m, n;          // stored rows and columns (n a multiple of 8)
    float inv_s;
    template <class T>
    __device__ __forceinline__ void operator()(const HalfPlace<T> &at, f32x16 (&acc)[T::MT][T::NT]) const {
#pragma unroll
        for (int i = 0; i < T::MT; ++i) {
            const int r = at.row(i);
#pragma unroll
            for (int j = 0; j < T::NT; ++j) {
                if (at.col0 + 32 * j >= n) break;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int c = at.col(j) + 8 * g;
                    if (r >= m || c >= n) continue;
                    const int64_t i0 = at.batch * batch + r * ld + c;
                    const u32x2 xw = *reinterpret_cast<const u32x2 *>(x + i0);
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[e] = __builtin_fmaf(kOrthoA, half_bits_to_f32((e < 2 ? xw.x : xw.y) >> (16 * (e & 1))), kDown * acc[i][j][4 * g + e]);
                    if (out != nullptr) {
                        uint32_t h[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) h[e] = f16_from_f32<false>(v[e], 0u);
                        const u32x2 w = {h[0] | (h[1] << 16), h[2] | (h[3] << 16)};
                        *reinterpret_cast<u32x2 *>(out + i0) = w;
                    } else {
                        const f32x4 o = {v[0] * inv_s, v[1] * inv_s, v[2] * inv_s, v[3] * inv_s};
                        *reinterpret_cast<f32x4 *>(last + i0) = o;
                    }
                }
            }
        }
    }
};

// ---------------------------------------------------------------------------------------
// Momentum, and the squared norm of the direction (in double: neither squares of gradients around 1e-25 nor those around 1e25 leave its
// range).  `blocks` workgroups per matrix.
// ---------------------------------------------------------------------------------------
struct OrthoMomentum {
    float *v;
    const uint8_t *g8;
    int64_t n;        // elements of a matrix
    float inv_scale, mu;
    int nesterov, blocks;
    const uint32_t *skip;
    double *squares;  // [batch, blocks]
    mp8_stats *stats;
};
__device__ __forceinline__ float ortho_direction(float v, float g, float mu, int nesterov) { return nesterov ? __builtin_fmaf(mu, v, g) : v; }

__global__ __launch_bounds__(256) void ortho_momentum_kernel(const OrthoMomentum p) {
    __shared__ double sh[4];
    const bool skipping = p.skip != nullptr && *p.skip != 0u;
    if (skipping && p.stats == nullptr) return;
    const int64_t base = (int64_t)blockIdx.y * p.n;
    const int64_t per = (((p.n + p.blocks - 1) / p.blocks) + 3) & ~(int64_t)3;
    const int64_t first = blockIdx.x * per, end = first + per < p.n ? first + per : p.n;
    // (a matrix may start anywhere: groups of four by address)
    double sum = 0.0;
    uint32_t nonfinite = 0;
    auto one = [&](int64_t i) {
        const uint32_t code = p.g8[base + i];
        nonfinite += (code & 0x7Cu) == 0x7Cu ? 1u : 0u;
        if (skipping) return;
        const float g = e5m2_to_f32(code) * p.inv_scale;
        const float v = __builtin_fmaf(p.mu, p.v[base + i], g);
        p.v[base + i] = v;
        const double u = (double)ortho_direction(v, g, p.mu, p.nesterov);
        sum += u * u;
    };
    if (((base | p.n) & 3) == 0) {
        for (int64_t i = first + 4 * threadIdx.x; i < end; i += 1024) {
            const uint32_t codes = *reinterpret_cast<const uint32_t *>(p.g8 + base + i);
            nonfinite += __builtin_popcount(((codes & 0x7C7C7C7Cu) + 0x04040404u) & 0x80808080u);
            if (skipping) continue;
            f32x4 v = *reinterpret_cast<const f32x4 *>(p.v + base + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float g = e5m2_to_f32((codes >> (8 * e)) & 0xFFu) * p.inv_scale;
                v[e] = __builtin_fmaf(p.mu, v[e], g);
                const double u = (double)ortho_direction(v[e], g, p.mu, p.nesterov);
                sum += u * u;
            }
            *reinterpret_cast<f32x4 *>(p.v + base + i) = v;
        }
    } else {
        for (int64_t i = first + threadIdx.x; i < end; i += 256) one(i);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) p.squares[(int64_t)blockIdx.y * p.blocks + blockIdx.x] = (sh[0] + sh[1]) + (sh[2] + sh[3]);
    if (p.stats != nullptr) {
        StatsAcc st;
        st.nonfinite = nonfinite;
        st.flush(p.stats);
    }
}

// X0 times S as halves, [m8, ld] per matrix, from the new momentum and the gradient: a workgroup per 64x64 tile, transposed through
// LDS where the weights are taller than wide.  Zeros beyond m and n.
struct OrthoStart {
    const float *v;
    const uint8_t *g8;
    int rows, cols;   // of the weights
    int transposed;
    float inv_scale, mu;
    int nesterov, blocks;
    const double *squares;
    const uint32_t *skip;
    double s;
    uint16_t *x;
    int64_t ld, batch;
    int m8;
};
__global__ __launch_bounds__(256) void ortho_start_kernel(const OrthoStart p) {
    __shared__ uint16_t sh[64][66];
    if (p.skip != nullptr && *p.skip != 0u) return;
    double sum = 0.0;
    for (int b = threadIdx.x & 63; b < p.blocks; b += 64) sum += p.squares[(int64_t)blockIdx.z * p.blocks + b];
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    const double inv = sum == 0.0 ? 0.0 : p.s / sqrt(sum);
    // tile of the weights' matrix
    const int r0 = 64 * (p.transposed ? blockIdx.x : blockIdx.y), c0 = 64 * (p.transposed ? blockIdx.y : blockIdx.x);
    const int64_t base = (int64_t)blockIdx.z * p.rows * p.cols;
    const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
#pragma unroll 4
    for (int k = 0; k < 16; ++k) {
        const int r = r0 + y + 4 * k, c = c0 + x;
        uint32_t h = 0;
        if (r < p.rows && c < p.cols) {
            const int64_t i = base + (int64_t)r * p.cols + c;
            const float g = e5m2_to_f32(p.g8[i]) * p.inv_scale;
            h = f16_from_f32<false>((float)((double)ortho_direction(p.v[i], g, p.mu, p.nesterov) * inv), 0u);
        }
        sh[y + 4 * k][x] = (uint16_t)h;
    }
    __syncthreads();
    uint16_t *out = p.x + blockIdx.z * p.batch;
#pragma unroll 4
    for (int k = 0; k < 16; ++k) {
        const int r = 64 * blockIdx.y + y + 4 * k, c = 64 * blockIdx.x + x;  // of X
        if (r < p.m8) out[r * p.ld + c] = p.transposed ? sh[x][y + 4 * k] : sh[y + 4 * k][x];
    }
}

// w' = w - lr (X + wd w), rounded to half, and its 8-bit copy.  A workgroup per 64x64 tile of the weights.
struct OrthoApply {
    const float *o;
    int64_t ld, batch;
    int rows, cols, transposed;
    uint16_t *w16;
    uint8_t *w8;
    float neg_lr, wd;
    int sr;
    uint64_t seed, offset;
    const uint32_t *skip;
};
__global__ __launch_bounds__(256) void ortho_apply_kernel(const OrthoApply p) {
    __shared__ float sh[64][65];
    if (p.skip != nullptr && *p.skip != 0u) return;
    const int r0 = 64 * blockIdx.y, c0 = 64 * blockIdx.x;
    const float *o = p.o + blockIdx.z * p.batch;
    const int64_t base = (int64_t)blockIdx.z * p.rows * p.cols;
    const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
    if (p.transposed) {
#pragma unroll 4
        for (int k = 0; k < 16; ++k) {
            const int c = c0 + y + 4 * k, r = r0 + x;  // row c of X, column r
            sh[x][y + 4 * k] = c < p.cols && r < p.rows ? o[c * p.ld + r] : 0.0f;
        }
        __syncthreads();
    }
    const Philox rng(p.seed, p.offset);
    // four neighbouring columns per thread
    const int cx = 4 * (threadIdx.x & 15), ry = threadIdx.x >> 4;
    const bool whole = (p.cols & 3) == 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int lr = ry + 16 * k, r = r0 + lr, c = c0 + cx;
        if (r >= p.rows || c >= p.cols) continue;
        const int64_t i = base + (int64_t)r * p.cols + c;
        const int n = p.cols - c < 4 ? p.cols - c : 4;
        float d[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) d[e] = p.transposed ? sh[lr][cx + e] : e < n ? o[r * p.ld + c + e] : 0.0f;
        uint32_t w[4], h[4];
        if (whole) {
            const u32x2 in = *reinterpret_cast<const u32x2 *>(p.w16 + i);
            w[0] = in.x & 0xFFFFu; w[1] = in.x >> 16; w[2] = in.y & 0xFFFFu; w[3] = in.y >> 16;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = e < n ? p.w16[i + e] : 0u;
        }
        Words4 words = {0, 0};
        if (p.sr) words = rng.words_at((uint64_t)i);
        const uint32_t rw[4] = {words.r01 << 16, words.r01 & 0xFFFF0000u, words.r23 << 16, words.r23 & 0xFFFF0000u};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float f = half_bits_to_f32(w[e]);
            float wn = __builtin_fmaf(p.neg_lr, __builtin_fmaf(p.wd, f, d[e]), f);
            asm volatile("" : "+v"(wn));  // (two roundings: see update_four)
            h[e] = p.sr ? f16_from_f32<true>(wn, rw[e]) : f16_from_f32<false>(wn, 0u);
        }
        if (whole) {
            const u32x2 out = {h[0] | (h[1] << 16), h[2] | (h[3] << 16)};
            *reinterpret_cast<u32x2 *>(p.w16 + i) = out;
            if (p.w8 != nullptr) {
                const uint32_t two[2] = {out.x, out.y};
                *reinterpret_cast<uint32_t *>(p.w8 + i) = e5m2_of_halves(two);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < n) {
                    p.w16[i + e] = (uint16_t)h[e];
                    if (p.w8 != nullptr) p.w8[i + e] = (uint8_t)e5m2_of_half(h[e]);
                }
        }
    }
}

// ---------------------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------------------
namespace {

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

struct OrthoLayout {
    int64_t m, n, m8, n8, ld, lda;  // X [m8, ld], A [m8, lda]
    int blocks;                     // workgroups of the momentum pass per matrix
    size_t squares, x0, x1, a, b, last, total;
};
OrthoLayout ortho_layout(int64_t batch, int64_t rows, int64_t cols) {
    OrthoLayout l{};
    l.m = rows < cols ? rows : cols;
    l.n = rows < cols ? cols : rows;
    l.m8 = up(l.m, 8);
    l.n8 = up(l.n, 8);
    l.ld = half_pitch(l.n);
    l.lda = half_pitch(l.m);
    const int64_t want = (rows * cols + 4095) / 4096, most = batch >= 256 ? 4 : 1024 / batch;
    l.blocks = (int)(want < 1 ? 1 : want > most ? most : want);
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t here = at;
        at += (size_t)up(bytes, 256);
        return here;
    };
    l.squares = take(8 * batch * l.blocks);
    l.x0 = take(2 * batch * l.m8 * l.ld);
    l.x1 = take(2 * batch * l.m8 * l.ld);
    l.a = take(2 * batch * l.m8 * l.lda);
    l.b = take(2 * batch * l.m8 * l.lda);
    l.last = take(4 * batch * l.m8 * l.ld);
    l.total = at;
    return l;
}

mp8_status ortho_sizes(int64_t batch, int64_t rows, int64_t cols) {
    if (batch < 0 || rows < 0 || cols < 0) return MP8_ERR_INVALID_ARG;
    // 32-bit offsets within a tile, workgroups of a launch
    const int64_t side = (int64_t)1 << 20;
    if (rows > side || cols > side || batch > 65535) return MP8_ERR_UNSUPPORTED;
    if (batch * ((rows + 63) / 64) * ((cols + 63) / 64) > ((int64_t)1 << 23)) return MP8_ERR_UNSUPPORTED;
    if ((rows + 63) / 64 > 65535 || (cols + 63) / 64 > 65535) return MP8_ERR_UNSUPPORTED;
    return MP8_OK;
}

template <bool BTN, class Epi>
bool ortho_product(int64_t batch, const uint16_t *a, int64_t lda, int64_t a_batch, const uint16_t *b, int64_t ldb, int64_t b_batch, int64_t rows,
                   int64_t cols, int64_t kc, bool symmetric, const uint32_t *skip, const Epi &epi, hipStream_t stream) {
    const int tile = half_plan(batch, rows, cols, kc, symmetric, 1).tile;
    HalfGemm p = half_gemm_args(a, lda, a_batch, b, ldb, b_batch, rows, cols, kc, tile, tile, 1, symmetric);
    p.skip = skip;
    if (tile == 256) return half_gemm_launch<Half256, false, BTN>(p, batch, epi, stream);
    if (tile == 128) return half_gemm_launch<Half128, false, BTN>(p, batch, epi, stream);
    return half_gemm_launch<Half64, false, BTN>(p, batch, epi, stream);
}

}  // namespace
}  // namespace mp8

extern "C" size_t mp8_orthogonal_momentum_workspace_bytes(int64_t batch, int64_t rows, int64_t cols) {
    using namespace mp8;
    if (ortho_sizes(batch, rows, cols) != MP8_OK || batch == 0 || rows == 0 || cols == 0) return 0;
    return ortho_layout(batch, rows, cols).total;
}

extern "C" mp8_status mp8_orthogonal_momentum_fp16_sr(int64_t batch, int64_t rows, int64_t cols, uint16_t *w16, float *velocity,
                                                      const uint8_t *g8, float lr, float inv_loss_scale, float momentum, int nesterov,
                                                      float weight_decay, int steps, mp8_round round, uint64_t seed, uint64_t offset,
                                                      const uint32_t *skip_if_nonzero, uint8_t *w8_out, mp8_stats *stats,
                                                      void *workspace, size_t workspace_bytes, void *stream) {
    using namespace mp8;
    const mp8_status sizes = ortho_sizes(batch, rows, cols);
    if (sizes != MP8_OK) return sizes;
    if (steps < 1 || steps > 64 || (round != MP8_RNE && round != MP8_SR)) return MP8_ERR_INVALID_ARG;
    if (batch == 0 || rows == 0 || cols == 0) return MP8_OK;
    if (!w16 || !velocity || !g8) return MP8_ERR_INVALID_ARG;
    if (((uintptr_t)w16 | (uintptr_t)velocity | (uintptr_t)g8 | (uintptr_t)w8_out | (uintptr_t)workspace) & 15u) return MP8_ERR_ALIGNMENT;
    // a flag that this very call may raise between its first launch and its last
    const uintptr_t flag = (uintptr_t)skip_if_nonzero, counted = (uintptr_t)stats;
    if (flag && counted && flag + sizeof(uint32_t) > counted && flag < counted + sizeof(mp8_stats)) return MP8_ERR_INVALID_ARG;
    const OrthoLayout l = ortho_layout(batch, rows, cols);
    if (!workspace || workspace_bytes < l.total) return MP8_ERR_WORKSPACE;
    uint8_t *ws = (uint8_t *)workspace;
    hipStream_t st = (hipStream_t)stream;
    double *squares = (double *)(ws + l.squares);
    uint16_t *x[2] = {(uint16_t *)(ws + l.x0), (uint16_t *)(ws + l.x1)}, *a = (uint16_t *)(ws + l.a), *b = (uint16_t *)(ws + l.b);
    float *last = (float *)(ws + l.last);
    const int transposed = rows > cols;
    const double s = std::exp2(std::nearbyint(0.5 * std::log2((double)l.n)));
    const auto ok = [] { return hipGetLastError() == hipSuccess; };

    const OrthoMomentum mom{velocity, g8, rows * cols, inv_loss_scale, momentum, nesterov, l.blocks, skip_if_nonzero, squares, stats};
    hipLaunchKernelGGL(ortho_momentum_kernel, dim3((unsigned)l.blocks, (unsigned)batch), dim3(256), 0, st, mom);
    if (!ok()) return MP8_ERR_HIP;
    const OrthoStart start{velocity, g8, (int)rows, (int)cols, transposed, inv_loss_scale, momentum, nesterov, l.blocks, squares, skip_if_nonzero,
                           s, x[0], l.ld, l.m8 * l.ld, (int)l.m8};
    hipLaunchKernelGGL(ortho_start_kernel, dim3((unsigned)(l.ld / 64), (unsigned)(l.lda / 64), (unsigned)batch), dim3(256), 0, st, start);
    if (!ok()) return MP8_ERR_HIP;
    const int64_t xb = l.m8 * l.ld, ab = l.m8 * l.lda;
    for (int k = 0; k < steps; ++k) {
        const uint16_t *now = x[k & 1];
        const OrthoSymmetric gram{nullptr, a, l.lda, ab, (int)l.m8, 0.0f, (float)(kUp / (s * s))};
        if (!ortho_product<false>(batch, now, l.ld, xb, now, l.ld, xb, l.m8, l.m8, l.n8, true, skip_if_nonzero, gram, st)) return MP8_ERR_HIP;
        const OrthoSymmetric poly{a, b, l.lda, ab, (int)l.m8, kOrthoB, kOrthoC * kDown};
        if (!ortho_product<false>(batch, a, l.lda, ab, a, l.lda, ab, l.m8, l.m8, l.m8, true, skip_if_nonzero, poly, st)) return MP8_ERR_HIP;
        const OrthoNext next{now, k + 1 < steps ? x[(k + 1) & 1] : nullptr, last, l.ld, xb, (int)l.m8, (int)l.n8, (float)(1.0 / s)};
        if (!ortho_product<true>(batch, b, l.lda, ab, now, l.ld, xb, l.m8, l.n8, l.m8, false, skip_if_nonzero, next, st)) return MP8_ERR_HIP;
    }
    const OrthoApply apply{last, l.ld, xb, (int)rows, (int)cols, transposed, w16, w8_out, -lr, weight_decay, round == MP8_SR, seed, offset, skip_if_nonzero};
    hipLaunchKernelGGL(ortho_apply_kernel, dim3((unsigned)((cols + 63) / 64), (unsigned)((rows + 63) / 64), (unsigned)batch), dim3(256), 0, st, apply);
    return ok() ? MP8_OK : MP8_ERR_HIP;
}
