// mp8_orthogonal_momentum_fp16_sr: a momentum step whose direction is orthogonalised before it is applied to the half-precision
// master weights (the weight-update path of Figure 1b of arXiv 1905.12334 with another rule between the gradient and the weights).
//
// Per matrix, with g the un-scaled gradient:
//   v' = mu v + g,   u = v' or, as Nesterov, g + mu v'
//   X0 = u / |u|_F;  X <- a X + (b A + c A^2) X,  A = X X^T  (steps times);   w' = w - lr (X + wd w)
// A step maps every singular value s to a s + b s^3 + c s^5 and leaves the singular vectors alone: with (a, b, c) = (3.4445,
// -4.7750, 2.0315), whose slope at zero is steep, five steps bring all but the smallest to 0.7 .. 1.2.
//
// X has the weights' rows and columns, in panels of 64 columns, and so have A and the polynomial.  A is formed over the shorter side:
// X X^T and (bA + cA^2) X where rows <= cols, X^T X and X (bA + cA^2) otherwise; the second product of the last step updates the weights
// itself.  Operands of the products are halves, sums FP32.  A power of two keeps each of them in the format's range: singular values stay
// below 1.21, so that entries of A are below 1.46 and those of bA + cA^2 below 2.81 in magnitude; A and the polynomial are stored times
// 2^14, X times S = 2^round(log2 sqrt n), which makes the entries of an orthogonal X about 1.  What half operands cost: entries of X are off
// by 0.7e-3 to 1.2e-3 of their root mean square after five steps from a Gaussian u (ortho_combine); where few directions hold most of u, by
// more, since what the rounding of u leaves beside them grows by a per step: eight directions with noise of 0.05, 0.01 and 0 of their size
// 5.6e-3, 2.3e-2 and 4.3e-2, a single one without noise 0.15 (FP32 operands: 3e-6, 1e-5, 4e-5 and 1e-4).  The coefficients are those that
// Jordan et al. (2024) published for this iteration.
#include <cmath>

#include "half_gemm.hpp"

namespace mp8 {

// Wide accesses at addresses of any alignment, which cost as much as others where they are aligned.
template <class V>
__device__ __forceinline__ V any_aligned(const void *p) {
    V v;
    __builtin_memcpy(&v, p, sizeof(V));
    return v;
}

constexpr float kOrthoA = 3.4445f, kOrthoB = -4.7750f, kOrthoC = 2.0315f;
constexpr float kUp = 16384.0f, kDown = 1.0f / 16384.0f;  // the scale of A and of the polynomial

// Polynomials are operands in halves (times 2^14).  What the rounding takes from their diagonal, d, is kept in FP32 and comes back
// with the term in a: (a + d) x + sum.  Near the end the diagonal is the largest part of every row (b A + c A^2 is near (b + c) I), and its
// rounding was the largest of all errors: of the update of a noisy 700 x 1500 gradient 1.3e-3 of its norm, with d 0.86e-3.
__device__ __forceinline__ float ortho_combine(float d, float x, float sum) { return __builtin_fmaf(__builtin_fmaf(kDown, d, kOrthoA), x, kDown * sum); }
__device__ __forceinline__ float ortho_lost(float v) { return v - (float)(_Float16)v; }

// d where the next iterate's epilogues want it: of the rows (one per lane and band), or (TALL) of a lane's eight columns.
template <class T, bool TALL>
struct OrthoDiagonal {
    float d[TALL ? 8 : T::MT];
};
template <bool TALL, class T>
__device__ __forceinline__ OrthoDiagonal<T, TALL> ortho_diagonal(const HalfPlace<T> &at, const float *diagonal, int m) {
    OrthoDiagonal<T, TALL> in;
    if constexpr (TALL) {
        const int c = at.col0 + 8 * (at.lane % (T::WTN / 8));
#pragma unroll
        for (int e = 0; e < 8; ++e) in.d[e] = c + e < m ? diagonal[c + e] : 0.0f;
    } else {
#pragma unroll
        for (int i = 0; i < T::MT; ++i) {
            const int r = at.row0 + 32 * i + (at.lane & 31);
            in.d[i] = r < m ? diagonal[r] : 0.0f;
        }
    }
    return in;
}
// f(r, c, v, x) as in half_bands, v with the elements of d instead of a: for rows they lie behind the band's columns.
template <int MOST_U, bool TALL, class T, class Load, class F>
__device__ __forceinline__ void ortho_bands(const HalfPlace<T> &at, f32x16 (&acc)[T::MT][T::NT], const OrthoDiagonal<T, TALL> &in, const Load &load, const F &f) {
    const float *rows = nullptr;
    half_bands<MOST_U>(at, acc, load, [&](int r, int c, const float (&sum)[8], const decltype(load(0, 0)) &x) {
        float d[8];
        const float row = TALL ? 0.0f : rows[((r - at.row0) & 31) * kHalfBandPitch<T>];
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = TALL ? in.d[TALL ? e : 0] : row;
        f(r, c, sum, d, x);
    }, [&](int i, float *band) {
        if constexpr (!TALL) {
            if (at.lane < 32) band[at.lane * kHalfBandPitch<T> + T::WTN] = in.d[i];
            half_wave_lds();
            rows = band + T::WTN;
        }
    });
}

// Eight columns from c on, zeros where they do not exist.
__device__ __forceinline__ void ortho_clear_behind(u32x4 &w, int c, int cols) {
    if (cols - c >= 8) return;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e >= cols - c) w[e >> 1] &= e & 1 ? 0xFFFFu : 0xFFFF0000u;
}

// A symmetric output of halves, made from its upper tiles: v = scale * acc (POLY: + linear * in[r, c]) at (r, c) and, off the diagonal's
// tiles, at (c, r), turned round by the lanes that read the band.  Columns m .. m8 - 1 are zero.
// With the conversions of the results' epilogues (canonical NaN, a test per element) two bands of a 128x128 tile took 5 us.
template <bool POLY>
struct OrthoSymmetric {
    static constexpr bool kJoin = !POLY, k192 = true;
    const uint16_t *in;
    uint16_t *out;
    int64_t panel, batch;  // in halves
    int m;
    float linear, scale;
    float *diagonal;  // POLY: what the halves' diagonal lacks
    int64_t diagonal_batch;
    template <class T>
    struct Ahead {
        float d[T::MT];  // in[r, r] of this lane's rows, in a wave's part on the diagonal
    };
    template <class T>
    __device__ __forceinline__ Ahead<T> ahead(const HalfPlace<T> &at) const {
        Ahead<T> a{};
        if (POLY && at.row0 == at.col0) {
#pragma unroll
            for (int i = 0; i < T::MT; ++i) {
                const int r = at.row0 + 32 * i + (at.lane & 31);
                if (r < m) a.d[i] = half_bits_to_f32(in[at.batch * batch + HalfMatrix::at(r, r, panel)]);
            }
        }
        return a;
    }
    template <class T>
    __device__ __forceinline__ void operator()(const HalfPlace<T> &at, f32x16 (&acc)[T::MT][T::NT], const Ahead<T> &ahead) const {
        const uint16_t *x = in + at.batch * batch;
        uint16_t *o = out + at.batch * batch;
        const bool mirror = at.tm != at.tn;
        auto load = [&](int r, int c) {
            u32x4 xw = {0, 0, 0, 0};
            if (POLY && r < m && c < m) xw = *reinterpret_cast<const u32x4 *>(x + HalfMatrix::at(r, c, panel));
            return xw;
        };
        auto value = [&](const u32x4 &xw, float (&v)[8]) {
            const half8 h = __builtin_bit_cast(half8, xw);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = POLY ? __builtin_fmaf(linear, (float)h[e], scale * v[e]) : scale * v[e];
        };
        half_bands(at, acc, load, [&](int r, int c, const float (&sum)[8], const u32x4 &xw) {
            if (r >= m || c >= m) return;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = sum[e];
            value(xw, v);
            u32x4 w = half_operand8(v);
            ortho_clear_behind(w, c, m);
            *reinterpret_cast<u32x4 *>(o + HalfMatrix::at(r, c, panel)) = w;
        }, [&](int i, const float *band) {
            if (POLY && at.row0 == at.col0) {
                const int k = at.lane & 31, r = at.row0 + 32 * i + k;
                if (at.lane < 32 && r < m)
                    diagonal[at.batch * diagonal_batch + r] = ortho_lost(__builtin_fmaf(linear, ahead.d[i], scale * band[k * kHalfBandPitch<T> + 32 * i + k]));
            }
            if (!mirror) return;
            // four lanes per row of the turned band: its rows are the band's columns, its columns rows of the tile, all of which exist
            // (a tile below the diagonal's ends at a tile border)
            const int k = 8 * (at.lane & 3), r = at.row0 + 32 * i + k;
            constexpr int U = T::WTN / 16 < 4 ? T::WTN / 16 : T::WTN % 64 == 0 ? 4 : 3;
#pragma unroll 1
            for (int n0 = at.lane >> 2; n0 < T::WTN; n0 += 16 * U) {
                u32x4 xw[U];
#pragma unroll
                for (int u = 0; u < U; ++u) xw[u] = load(at.col0 + n0 + 16 * u, r);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int n = n0 + 16 * u, c = at.col0 + n;
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = band[(k + e) * kHalfBandPitch<T> + n];
                    value(xw[u], v);
                    if (c < m) *reinterpret_cast<u32x4 *>(o + HalfMatrix::at(c, r, panel)) = half_operand8(v);
                }
            }
        });
    }
};

// The next iterate, a X + scale * acc, as halves.  Columns up to the next multiple of eight are stored, as zeros: TALL, the product has the
// polynomial's last row there (rows behind it are read as that one), and left as they are these columns grow by a factor of a per step,
// to infinity in ten.
template <bool TALL>
struct OrthoNext {
    static constexpr bool kJoin = false, k192 = true;
    const uint16_t *x;
    uint16_t *out;
    int64_t panel, batch;  // in halves
    int rows, cols;
    const float *diagonal;
    int64_t diagonal_batch;
    template <class T>
    __device__ __forceinline__ OrthoDiagonal<T, TALL> ahead(const HalfPlace<T> &at) const {
        return ortho_diagonal<TALL>(at, diagonal + at.batch * diagonal_batch, TALL ? cols : rows);
    }
    template <class T>
    __device__ __forceinline__ void operator()(const HalfPlace<T> &at, f32x16 (&acc)[T::MT][T::NT], const OrthoDiagonal<T, TALL> &ahead) const {
        const int64_t base = at.batch * batch;
        ortho_bands<4, TALL>(at, acc, ahead, [&](int r, int c) {
            u32x4 xw = {0, 0, 0, 0};
            if (r < rows && c < cols) xw = *reinterpret_cast<const u32x4 *>(x + base + HalfMatrix::at(r, c, panel));
            return xw;
        }, [&](int r, int c, const float (&sum)[8], const float (&d)[8], const u32x4 &xw) {
            if (r >= rows || c >= cols) return;
            const half8 h = __builtin_bit_cast(half8, xw);
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = ortho_combine(d[e], (float)h[e], sum[e]);
            u32x4 w = half_operand8(v);
            if constexpr (TALL) ortho_clear_behind(w, c, cols);
            *reinterpret_cast<u32x4 *>(out + base + HalfMatrix::at(r, c, panel)) = w;
        });
    }
};

// The last iterate goes straight into the weights: w' = w - lr (X + wd w), rounded to half, and its 8-bit copy.
template <bool TALL>
struct OrthoUpdate {
    static constexpr bool kJoin = false, k192 = true;
    const uint16_t *x;
    int64_t panel, batch;
    int rows, cols;
    const float *diagonal;
    int64_t diagonal_batch;
    float inv_s, neg_lr, wd;
    uint16_t *w16;
    uint8_t *w8;
    int sr;
    uint64_t seed, offset;
    template <class T>
    __device__ __forceinline__ OrthoDiagonal<T, TALL> ahead(const HalfPlace<T> &at) const {
        return ortho_diagonal<TALL>(at, diagonal + at.batch * diagonal_batch, TALL ? cols : rows);
    }
    template <class T>
    __device__ __forceinline__ void operator()(const HalfPlace<T> &at, f32x16 (&acc)[T::MT][T::NT], const OrthoDiagonal<T, TALL> &ahead) const {
        const Philox rng(seed, offset);
        const bool whole = (cols & 7) == 0;
        const int64_t first = (int64_t)at.batch * rows * cols;
        struct Eight {
            u32x4 x, w;
        };
        // (four copies of this code per band are too much for the compiler where there are three or four bands)
        ortho_bands<(T::BM > 128 ? 1 : 4), TALL>(at, acc, ahead, [&](int r, int c) {
            Eight in{};
            if (r >= rows || c >= cols) return in;
            in.x = *reinterpret_cast<const u32x4 *>(x + at.batch * batch + HalfMatrix::at(r, c, panel));
            const int64_t i0 = first + (int64_t)r * cols + c;
            if (whole || c + 8 <= cols) {
                in.w = any_aligned<u32x4>(w16 + i0);
            } else {
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (c + e < cols) in.w[e >> 1] |= (uint32_t)w16[i0 + e] << (16 * (e & 1));
            }
            return in;
        }, [&](int r, int c, const float (&sum)[8], const float (&diag)[8], const Eight &in) {
            if (r >= rows || c >= cols) return;
            const int64_t i0 = first + (int64_t)r * cols + c;
            const int n = cols - c < 8 ? cols - c : 8;
            const u32x4 xw = in.x, ww = in.w;
            uint32_t rw[4] = {0, 0, 0, 0};
            if (sr) {
                const uint4 b = whole ? rng.block((uint64_t)i0 >> 3) : rng.eight_at((uint64_t)i0);
                rw[0] = b.x; rw[1] = b.y; rw[2] = b.z; rw[3] = b.w;
            }
            u32x4 o;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t hw[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float d = ortho_combine(diag[2 * q + e], half_bits_to_f32(xw[q] >> (16 * e)), sum[2 * q + e]) * inv_s;
                    const float f = half_bits_to_f32(ww[q] >> (16 * e));
                    float wn = __builtin_fmaf(neg_lr, __builtin_fmaf(wd, f, d), f);
                    asm volatile("" : "+v"(wn));  // (two roundings: see update_four)
                    hw[e] = sr ? f16_from_f32<true>(wn, e ? rw[q] & 0xFFFF0000u : rw[q] << 16) : f16_from_f32<false>(wn, 0u);
                }
                o[q] = hw[0] | (hw[1] << 16);
            }
            const uint32_t lo[2] = {o.x, o.y}, hi[2] = {o.z, o.w};
            const u32x2 codes = {w8 != nullptr ? e5m2_of_halves(lo) : 0u, w8 != nullptr ? e5m2_of_halves(hi) : 0u};
            if (n == 8) {
                __builtin_memcpy(w16 + i0, &o, 16);
                if (w8 != nullptr) __builtin_memcpy(w8 + i0, &codes, 8);
            } else {
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (e < n) {
                        w16[i0 + e] = (uint16_t)(o[e >> 1] >> (16 * (e & 1)));
                        if (w8 != nullptr) w8[i0 + e] = (uint8_t)((e < 4 ? codes.x : codes.y) >> (8 * (e & 3)));
                    }
            }
        });
    }
};

// ---------------------------------------------------------------------------------------
// Short sides: polynomial and product in one launch.  Every workgroup (a 64x64 tile of the product) makes the 64 rows of
// P = b A + c A A that its tile needs, from all of A in LDS, rounds them to half as the pass of its own would, and multiplies them with
// its part of X, which was requested together with A.  That is up to m / 64 times as many products as necessary, but a launch of its own
// costs 3 to 5 us whatever it multiplies.
// ---------------------------------------------------------------------------------------
struct OrthoJoint {
    const uint16_t *a, *x;
    int64_t a_batch, x_batch;  // in halves
    int m, m8, rows;           // of A, up to a multiple of eight, of X
    const uint32_t *skip;
};
// TALL: X P, the tile's rows of X as they are; otherwise P X, a panel of X, read transposed.  LDS images as half_gemm_kernel's.  S: slabs of
// 64 of the shorter side, so that all reads of LDS can be requested at once (with a loop of unknown length 10 us instead of 5.1 at 128x128).
template <int S, bool TALL, class Epi>
__global__ __launch_bounds__(256, S > 2 ? 1 : 2) void ortho_joint_kernel(const OrthoJoint p, const Epi epi) {
    constexpr int A_SLAB = S * 64 * 128, S_SLAB = 64 * 128;  // per 64 columns: all of A; 64 rows of P or X
    constexpr bool LATER = S * (A_SLAB + 2 * S_SLAB) > 160 * 1024;  // X takes A's place, and waits in registers until it is free
    constexpr int OPERANDS = S * (A_SLAB + (LATER ? 1 : 2) * S_SLAB);
    __shared__ __attribute__((aligned(1024))) uint8_t lds[OPERANDS + (LATER ? 0 : 256)];
    float *const diagonal = reinterpret_cast<float *>(lds + (LATER ? A_SLAB * S / 2 : OPERANDS));  // of the band (LATER: in A's place too)
    uint8_t *const la = lds, *const lp = lds + S * A_SLAB, *const lx = LATER ? la : lp + S * S_SLAB;
    if (p.skip != nullptr && *p.skip != 0u) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
    const int batch = blockIdx.y, along = blockIdx.x / S, band = blockIdx.x % S;  // (S tiles along the shorter side)
    const int tm = TALL ? along : band, tn = TALL ? band : along;
    const uint16_t *a = p.a + batch * p.a_batch, *x = p.x + batch * p.x_batch;

    auto row_slot = [](int r, int c) { return r * 128 + ((c ^ ((r >> 1) & 7)) << 4); };  // chunk c of row r, contraction along the row
    const int r0 = threadIdx.x >> 3, c0 = threadIdx.x & 7;
    u32x4 va[S][2 * S], vx[2 * S];  // [panel][32 rows]; see below
#pragma unroll
    for (int h = 0; h < S; ++h)
#pragma unroll
        for (int q = 0; q < 2 * S; ++q) {
            const int r = 32 * q + r0, c = 64 * h + 8 * c0;
            va[h][q] = u32x4{0, 0, 0, 0};
            if (r < p.m && c < p.m8) va[h][q] = *reinterpret_cast<const u32x4 *>(a + HalfMatrix::at(r, c, 64 * (int64_t)p.m));
        }
#pragma unroll
    for (int q = 0; q < 2 * S; ++q) {
        vx[q] = u32x4{0, 0, 0, 0};
        if constexpr (TALL) {  // panel q / 2, rows 32 (q % 2) + r0 of the tile
            const int r = 64 * along + 32 * (q & 1) + r0, c = 64 * (q >> 1) + 8 * c0;
            if (r < p.rows && c < p.m8) vx[q] = *reinterpret_cast<const u32x4 *>(x + HalfMatrix::at(r, c, 64 * (int64_t)p.rows));
        } else {  // rows 32 q + r0 of the panel
            const int r = 32 * q + r0;
            if (r < p.rows) vx[q] = *reinterpret_cast<const u32x4 *>(x + HalfMatrix::at(r, 64 * along + 8 * c0, 64 * (int64_t)p.rows));
        }
    }
#pragma unroll
    for (int h = 0; h < S; ++h)
#pragma unroll
        for (int q = 0; q < 2 * S; ++q) *reinterpret_cast<u32x4 *>(la + h * A_SLAB + row_slot(32 * q + r0, c0)) = va[h][q];
    auto put_x = [&]() {
#pragma unroll
        for (int q = 0; q < 2 * S; ++q) {
            if constexpr (TALL) *reinterpret_cast<u32x4 *>(lx + (q >> 1) * S_SLAB + row_slot(32 * (q & 1) + r0, c0)) = vx[q];
            else *reinterpret_cast<u32x4 *>(lx + (32 * q + r0) * 128 + ((c0 ^ (((r0 >> 1) & 1) << 2)) << 4)) = vx[q];
        }
    };
    if constexpr (!LATER) put_x();
    __syncthreads();

    const int frow = lane & 31, fk = lane >> 5, t16 = lane & 15;
    auto row_fragment = [&](const uint8_t *image, int slab, int sub, int m) {
        return *reinterpret_cast<const half8 *>(image + (sub >> 2) * slab + row_slot(m + frow, 2 * (sub & 3) + fk));
    };
    const int own = 32 * wm + frow;  // row of the band
    float own_diagonal = 0.0f;
    bool has_diagonal = false;
    {  // this wave's 32 rows of P, columns 32 (S wn + i) ..
        f32x16 acc[S];
#pragma unroll
        for (int i = 0; i < S; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][e] = 0.0f;
#pragma unroll
        for (int sub = 0; sub < 4 * S; ++sub) {
            const half8 fa = row_fragment(la, A_SLAB, sub, 64 * band + 32 * wm);
#pragma unroll
            for (int i = 0; i < S; ++i)
                acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(row_fragment(la, A_SLAB, sub, 32 * (S * wn + i)), fa, acc[i], 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < S; ++i) {
            using half4 = _Float16 __attribute__((ext_vector_type(4)));
            const int block = S * wn + i;
            float v[4][4];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const half4 h = *reinterpret_cast<const half4 *>(la + (block >> 1) * A_SLAB + row_slot(64 * band + own, 4 * (block & 1) + g) + 8 * fk);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[g][e] = __builtin_fmaf(kOrthoB, (float)h[e], kOrthoC * kDown * acc[i][4 * g + e]);
            }
            if (block == 2 * band + wm) {  // (of the columns 8 g + 4 fk + e, frow)
                has_diagonal = ((frow >> 2) & 1) == fk;
#pragma unroll
                for (int g = 0; g < 4; ++g)
#pragma unroll
                    for (int e = 0; e < 4; ++e) own_diagonal = 8 * g + 4 * fk + e == frow ? v[g][e] : own_diagonal;
            }
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                half4 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = (_Float16)v[g][e];
                *reinterpret_cast<half4 *>(lp + (block >> 1) * S_SLAB + row_slot(own, 4 * (block & 1) + g) + 8 * fk) = o;
            }
        }
    }
    if constexpr (LATER) {
        __syncthreads();  // (A has been read)
        if (has_diagonal) diagonal[own] = ortho_lost(own_diagonal);
        put_x();
    } else {
        if (has_diagonal) diagonal[own] = ortho_lost(own_diagonal);
    }
    __syncthreads();  // (X, P and its diagonal are complete)

    const int kt = 8 * fk + (t16 >> 2), ct = ((lane >> 4) & 1) * 2 + ((t16 & 3) >> 1);
    const int ft = kt * 128 + ((ct ^ (((t16 >> 3) & 1) << 2)) << 4) + 8 * (t16 & 1);
    auto panel_fragment = [&](int sub, int m) {  // columns m .. m + 31 of the panel
        using h4 = short __attribute__((ext_vector_type(4)));
        using lds_h4 = __attribute__((address_space(3))) h4;
        const uint8_t *at = lx + (ft ^ ((m & 32) << 1)) + 16 * sub * 128;
        const h4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_h4 *)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_h4 *)(at + 512));
        return __builtin_bit_cast(half8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    f32x16 acc[1][1];
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[0][0][e] = 0.0f;
#pragma unroll
    for (int sub = 0; sub < 4 * S; ++sub) {
        const half8 fa = row_fragment(TALL ? lx : lp, S_SLAB, sub, 32 * wm);
        const half8 fb = TALL ? row_fragment(lp, S_SLAB, sub, 32 * wn) : panel_fragment(sub, 32 * wn);
        acc[0][0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fb, fa, acc[0][0], 0, 0, 0);
    }
    const HalfPlace<Half64> at{batch, 0, tm, tn, 64 * tm + 32 * wm, 64 * tn + 32 * wn, wave, lane, lds};
    HalfPlace<Half64> in_band = at;  // (the diagonal counts from the band's first row or column)
    (TALL ? in_band.col0 : in_band.row0) -= 64 * band;
    epi(at, acc, ortho_diagonal<TALL>(in_band, diagonal, 64));
}

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
    uint32_t *arrived;  // `words` of them become zero (HalfGemm::arrived)
    int words;
};
__device__ __forceinline__ float ortho_direction(float v, float g, float mu, int nesterov) { return nesterov ? __builtin_fmaf(mu, v, g) : v; }

__global__ __launch_bounds__(256) void ortho_momentum_kernel(const OrthoMomentum p) {
    __shared__ double sh[4];
    if (blockIdx.y == 0)
        for (int i = blockIdx.x * 256 + threadIdx.x; i < p.words; i += gridDim.x * 256) p.arrived[i] = 0u;
    const bool skipping = p.skip != nullptr && *p.skip != 0u;
    if (skipping && p.stats == nullptr) return;
    const int64_t base = (int64_t)blockIdx.y * p.n;
    const int64_t per = (((p.n + p.blocks - 1) / p.blocks) + 3) & ~(int64_t)3;
    const int64_t first = blockIdx.x * per, end = first + per < p.n ? first + per : p.n;
    double sum = 0.0;
    uint32_t nonfinite = 0;
    auto one = [&](uint32_t code, float v) {
        const float g = e5m2_to_f32(code) * p.inv_scale;
        v = __builtin_fmaf(p.mu, v, g);
        const double u = (double)ortho_direction(v, g, p.mu, p.nesterov);
        sum += u * u;
        return v;
    };
    // (a matrix may start anywhere: 2001 x 1013 took 11.4 us element by element, 1024 x 4096 8.1)
    for (int64_t i = first + 4 * threadIdx.x; i < end; i += 1024) {
        if (i + 4 <= end) {
            const uint32_t codes = any_aligned<uint32_t>(p.g8 + base + i);
            nonfinite += __builtin_popcount(((codes & 0x7C7C7C7Cu) + 0x04040404u) & 0x80808080u);
            if (skipping) continue;
            f32x4 v = any_aligned<f32x4>(p.v + base + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = one((codes >> (8 * e)) & 0xFFu, v[e]);
            __builtin_memcpy(p.v + base + i, &v, 16);
        } else {
            for (int64_t k = base + i; k < base + end; ++k) {
                const uint32_t code = p.g8[k];
                nonfinite += (code & 0x7Cu) == 0x7Cu ? 1u : 0u;
                if (!skipping) p.v[k] = one(code, p.v[k]);
            }
        }
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

// X0 times S as halves, in panels, from the new momentum and the gradient: eight columns per thread, zeros behind the last.
struct OrthoStart {
    const float *v;
    const uint8_t *g8;
    int rows, cols;
    float inv_scale, mu;
    int nesterov, blocks;
    const double *squares;
    const uint32_t *skip;
    double s;
    uint16_t *x;
    int64_t batch;
    FastDiv div_groups;  // by the groups of eight in a row, cols / 8 rounded up
};
__global__ __launch_bounds__(256) void ortho_start_kernel(const OrthoStart p) {
    const uint32_t groups = (uint32_t)p.rows * p.div_groups.d, stride = gridDim.x * 256;
    const int64_t base = (int64_t)blockIdx.y * p.rows * p.cols;
    if (p.skip != nullptr && *p.skip != 0u) return;
    double sum = 0.0;  // (by all lanes of the wave, also those without a group)
    for (int b = threadIdx.x & 63; b < p.blocks; b += 64) sum += p.squares[(int64_t)blockIdx.y * p.blocks + b];
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    const double inv = sum == 0.0 ? 0.0 : p.s / sqrt(sum);
    for (uint32_t t = blockIdx.x * 256 + threadIdx.x; t < groups; t += stride) {
        uint32_t k;
        const uint32_t r = fastdiv(t, p.div_groups, k);
        const int c = 8 * (int)k;
        const int64_t i = base + (int64_t)r * p.cols + c;
        uint32_t code[2] = {0, 0};
        float v[8];
        if (c + 8 <= p.cols) {
            const u32x2 g = any_aligned<u32x2>(p.g8 + i);
            const f32x4 a = any_aligned<f32x4>(p.v + i), b = any_aligned<f32x4>(p.v + i + 4);
            code[0] = g.x;
            code[1] = g.y;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = a[e], v[4 + e] = b[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool in = c + e < p.cols;
                code[e >> 2] |= (in ? (uint32_t)p.g8[i + e] : 0u) << (8 * (e & 3));
                v[e] = in ? p.v[i + e] : 0.0f;
            }
        }
        u32x4 o;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint32_t h[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int n = 2 * q + e;
                const float g = e5m2_to_f32((code[n >> 2] >> (8 * (n & 3))) & 0xFFu) * p.inv_scale;
                h[e] = f16_from_f32<false>((float)((double)ortho_direction(v[n], g, p.mu, p.nesterov) * inv), 0u);
            }
            o[q] = h[0] | (h[1] << 16);
        }
        *reinterpret_cast<u32x4 *>(p.x + blockIdx.y * p.batch + HalfMatrix::at(r, c, 64 * (int64_t)p.rows)) = o;
    }
}

// ---------------------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------------------
namespace {

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

struct OrthoLayout {
    int64_t m, n, x_batch, a_batch;  // shorter and longer side; halves of an X and of an A
    int blocks;             // workgroups of the momentum pass per matrix
    HalfPlan gram;
    int64_t words;          // tiles of the Gram matrices
    size_t squares, x0, x1, a, b, diagonal, parts, arrived, total;
};
OrthoLayout ortho_layout(int64_t batch, int64_t rows, int64_t cols) {
    OrthoLayout l{};
    l.m = rows < cols ? rows : cols;
    l.n = rows < cols ? cols : rows;
    l.x_batch = rows * up(cols, 64);
    l.a_batch = l.m * up(l.m, 64);
    const int64_t want = (rows * cols + 4095) / 4096, most = batch >= 256 ? 4 : 1024 / batch;
    l.blocks = (int)(want < 1 ? 1 : want > most ? most : want);
    l.gram = half_plan(batch, l.m, l.m, l.n, true, 32, true);
    const int64_t t = (l.m + l.gram.tile - 1) / l.gram.tile;
    l.words = l.gram.splits > 1 ? batch * (t * (t + 1) / 2) : 0;
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t here = at;
        at += (size_t)up(bytes, 256);
        return here;
    };
    l.squares = take(8 * batch * l.blocks);
    l.x0 = take(2 * batch * l.x_batch);
    l.x1 = take(2 * batch * l.x_batch);
    l.a = take(2 * batch * l.a_batch);
    l.b = take(2 * batch * l.a_batch);
    l.diagonal = take(4 * batch * up(l.m, 64));
    l.parts = take(4 * l.words * l.gram.splits * l.gram.tile * l.gram.tile);
    l.arrived = take(4 * l.words);
    l.total = at;
    return l;
}

// Whether polynomial and product go together: shorter sides up to 64 always, up to 256 while all workgroups run at once (two per CU, from three
// slabs on one).  A whole call, us, apart / together: 64x64 50 / 34, 64 of 64x4096 267 / 188, 128x128 68 / 52, 128x20000 156 / 147, 256x256
// 84 / 74, 256x4096 117 / 116; with more workgroups 64 of 128x1024 149 / 191, 8 of 192x768 96 / 108, 256x8192 143 / 170.
bool ortho_joint(const OrthoLayout &l, int64_t batch) {
    const int64_t across = (l.m + 63) / 64, tiles = batch * across * ((l.n + 63) / 64);
    return across == 1 || (across <= 4 && tiles <= (across == 2 ? 512 : 256));
}

mp8_status ortho_sizes(int64_t batch, int64_t rows, int64_t cols) {
    if (batch < 0 || rows < 0 || cols < 0) return MP8_ERR_INVALID_ARG;
    // 32-bit offsets within a tile, workgroups of a launch
    const int64_t side = (int64_t)1 << 20;
    if (rows > side || cols > side || batch > 65535) return MP8_ERR_UNSUPPORTED;
    if (batch * ((rows + 63) / 64) * ((cols + 63) / 64) > ((int64_t)1 << 23)) return MP8_ERR_UNSUPPORTED;
    return MP8_OK;
}

template <bool ATN, bool BTN, class Epi>
bool ortho_product(const HalfPlan &plan, int64_t batch, const HalfMatrix &a, const HalfMatrix &b, int64_t rows, int64_t cols, int64_t kc, bool symmetric,
                   const uint32_t *skip, float *parts, uint32_t *arrived, const Epi &epi, hipStream_t stream) {
    HalfGemm p = half_gemm_args(a, b, rows, cols, kc, plan.tile, plan.splits, symmetric, batch);
    p.skip = skip;
    p.parts = parts;
    p.arrived = arrived;
    return half_gemm_launch_plan<ATN, BTN>(plan.tile, p, epi, stream);
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
    float *parts = (float *)(ws + l.parts), *diagonal = (float *)(ws + l.diagonal);
    uint32_t *arrived = (uint32_t *)(ws + l.arrived);
    const double s = std::exp2(std::nearbyint(0.5 * std::log2((double)l.n)));
    const auto ok = [] { return hipGetLastError() == hipSuccess; };

    const OrthoMomentum mom{velocity, g8, rows * cols, inv_loss_scale, momentum, nesterov, l.blocks, skip_if_nonzero, squares, stats, arrived, (int)l.words};
    hipLaunchKernelGGL(ortho_momentum_kernel, dim3((unsigned)l.blocks, (unsigned)batch), dim3(256), 0, st, mom);
    if (!ok()) return MP8_ERR_HIP;
    const int64_t c8 = up(cols, 8), m8 = up(l.m, 8), xb = l.x_batch, ab = l.a_batch, x_panel = 64 * rows, a_panel = 64 * l.m, db = up(l.m, 64);
    const OrthoStart start{velocity, g8, (int)rows, (int)cols, inv_loss_scale, momentum, nesterov, l.blocks, squares, skip_if_nonzero, s, x[0], xb,
                           make_fastdiv((uint32_t)(c8 / 8))};
    const int64_t blocks = up(rows * (c8 / 8), 256) / 256;
    hipLaunchKernelGGL(ortho_start_kernel, dim3((unsigned)(blocks < 2048 ? blocks : 2048), (unsigned)batch), dim3(256), 0, st, start);
    if (!ok()) return MP8_ERR_HIP;
    const HalfMatrix A = HalfMatrix::panels(a, l.m, ab), P = HalfMatrix::panels(b, l.m, ab);
    const bool joint = ortho_joint(l, batch);
    for (int k = 0; k < steps; ++k) {
        const HalfMatrix X = HalfMatrix::panels(x[k & 1], rows, xb);
        const OrthoSymmetric<false> gram{nullptr, a, a_panel, ab, (int)l.m, 0.0f, (float)(kUp / (s * s)), nullptr, 0};
        if (rows <= cols ? !ortho_product<false, false>(l.gram, batch, X, X, l.m, l.m, l.n, true, skip_if_nonzero, parts, arrived, gram, st)
                         : !ortho_product<true, true>(l.gram, batch, X, X, m8, m8, l.n, true, skip_if_nonzero, parts, arrived, gram, st))
            return MP8_ERR_HIP;
        if (!joint) {
            const OrthoSymmetric<true> poly{a, b, a_panel, ab, (int)l.m, kOrthoB, kOrthoC * kDown, diagonal, db};
            if (!ortho_product<false, false>(half_plan(batch, l.m, l.m, l.m, true, 1), batch, A, A, l.m, l.m, l.m, true, skip_if_nonzero, nullptr, nullptr, poly, st))
                return MP8_ERR_HIP;
        }
        // X' or the weights, made by `epi` (the polynomial is symmetric: its rows are its columns)
        auto second = [&](auto tall, auto epi) {
            constexpr bool TALL = decltype(tall)::value;
            if (joint) {
                const OrthoJoint p{a, X.p, ab, xb, (int)l.m, (int)m8, (int)rows, skip_if_nonzero};
                const int64_t across = (l.m + 63) / 64;
                const dim3 grid((unsigned)(across * ((l.n + 63) / 64)), (unsigned)batch);
                if (across == 1) hipLaunchKernelGGL((ortho_joint_kernel<1, TALL, decltype(epi)>), grid, dim3(256), 0, st, p, epi);
                else if (across == 2) hipLaunchKernelGGL((ortho_joint_kernel<2, TALL, decltype(epi)>), grid, dim3(256), 0, st, p, epi);
                else if (across == 3) hipLaunchKernelGGL((ortho_joint_kernel<3, TALL, decltype(epi)>), grid, dim3(256), 0, st, p, epi);
                else hipLaunchKernelGGL((ortho_joint_kernel<4, TALL, decltype(epi)>), grid, dim3(256), 0, st, p, epi);
                return ok();
            }
            const HalfPlan plan = half_plan(batch, rows, cols, l.m, false, 1);
            if constexpr (TALL) return ortho_product<false, false>(plan, batch, X, P, rows, cols, l.m, false, skip_if_nonzero, nullptr, nullptr, epi, st);
            else return ortho_product<false, true>(plan, batch, P, X, rows, c8, l.m, false, skip_if_nonzero, nullptr, nullptr, epi, st);
        };
        auto advance = [&](auto tall) {
            constexpr bool TALL = decltype(tall)::value;
            if (k + 1 < steps) return second(tall, OrthoNext<TALL>{X.p, x[(k + 1) & 1], x_panel, xb, (int)rows, (int)cols, diagonal, db});
            return second(tall, OrthoUpdate<TALL>{X.p, x_panel, xb, (int)rows, (int)cols, diagonal, db, (float)(1.0 / s), -lr, weight_decay, w16, w8_out,
                                                  round == MP8_SR, seed, offset});
        };
        if (!(rows > cols ? advance(std::true_type{}) : advance(std::false_type{}))) return MP8_ERR_HIP;
    }
    return MP8_OK;
}
