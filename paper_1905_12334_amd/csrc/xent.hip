// Softmax cross entropy of a last layer's logits z = x . w^T (M tokens, N classes, K features) and its gradient, on the
// half-precision matrix instruction.  Section 4 of arXiv 1905.12334 keeps the last layer in 16 bits; the error that its
// backward pass hands down is where the loss scale of Section 3.1 enters.
//
//   forward   m = max_j z_ij,  lse_i = m + log sum_j exp(z_ij - m),  loss_i = lse_i - z_it
//   backward  e_ij = scale dloss_i (exp(z_ij - lse_i) - [j = t]),  dx = e . w,  dw = e^T . x
//
// The logits are never stored.  The forward pass reduces every tile of them to a maximum and a sum per row, and a second kernel joins these.
// The backward pass makes the logits once more, a piece of the vocabulary at a time, stores e of that piece as halves and
// multiplies it by w (added up over the pieces in FP32) and x (complete per piece).
#include <cmath>

#include "half_gemm.hpp"

namespace mp8 {

constexpr float kLog2e = 1.4426950408889634f;
// e is stored times 2^14: values of up to 1 in magnitude fill the half format from its top, and a probability keeps eleven bits
// down to 2^-28 and an absolute precision of 2^-39 below.
constexpr int kErrorExponent = 14;

// ---------------------------------------------------------------------------------------
// What becomes of a tile of logits.
// ---------------------------------------------------------------------------------------
// Sums are of powers of two: with base B = fl(m log2 e), sum 2^(z log2 e - B), one rounding per exponent (a fused multiply-add);
// what B itself was rounded by cancels when the sums are joined.  The target's logit is kept apart: the loss is
// log(1 + what the others have beside it), which lse - z would not give where the target has nearly everything.
// An empty part has the base 0 and the sum 0.
__device__ __forceinline__ void xent_join(f32x2 &t, f32x2 p) {
    const float b = p.y == 0.0f ? t.x : t.y == 0.0f ? p.x : __builtin_fmaxf(t.x, p.x);
    const float s0 = t.y == 0.0f ? 0.0f : t.y * __builtin_amdgcn_exp2f(t.x - b), s1 = p.y == 0.0f ? 0.0f : p.y * __builtin_amdgcn_exp2f(p.x - b);
    t = f32x2{b, s0 + s1};
}

// Column of a target among a wave's, the first of which is class `first`; -1 if it is none of them (`left`: that exist).
template <class T>
__device__ __forceinline__ int xent_column(int64_t target, int64_t first, int left) {
    const int64_t rel = target - first;
    return rel >= 0 && rel < T::WTN && rel < left ? (int)rel : -1;
}

struct XentStats {
    static constexpr bool kJoin = false, k192 = false;  // (logits_plan)
    const int64_t *targets;
    f32x2 *part;     // [parts, M]: (B, sum) of the columns of one tile, without the target
    float *z_target; // [M]
    int M, N, first; // `first`: class of this piece's column 0
    int part0;       // of this piece
    template <int MT>
    struct Ahead {
        int target[MT];  // of the wave's columns, or -1
    };
    template <class T>
    __device__ __forceinline__ Ahead<T::MT> ahead(const HalfPlace<T> &at) const {
        Ahead<T::MT> a;
#pragma unroll
        for (int i = 0; i < T::MT; ++i) a.target[i] = at.row(i) < M ? xent_column<T>(targets[at.row(i)], first + at.col0, N - at.col0) : -1;
        return a;
    }
    template <class T>
    __device__ __forceinline__ void operator()(const HalfPlace<T> &at, f32x16 (&acc)[T::MT][T::NT], const Ahead<T::MT> &a) const {
        const int h4 = 4 * (at.lane >> 5), left = N - at.col0;  // columns of this wave's tile that exist
        f32x2 mine[T::MT];
        // The (base, sum) of a row's accumulators.  Most waves have neither a target among their columns nor columns that do not exist;
        // with both tests in one path for all, 4096 x 32000 x 512 took 268 us in 256x256 tiles.
        auto row_sum = [&](int i, auto plain) {
            constexpr bool PLAIN = decltype(plain)::value;
            f32x16 z[T::NT];
#pragma unroll
            for (int j = 0; j < T::NT; ++j) z[j] = acc[i][j];
            if constexpr (!PLAIN) {
                int end = left - h4, c = a.target[i] - h4;  // (-1 - 4 h meets no column)
                asm volatile("" : "+v"(end), "+v"(c));  // (the comparisons anew in every row: sixty-four masks do not fit the registers)
                float zt = 0.0f;
#pragma unroll
                for (int j = 0; j < T::NT; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int column = 32 * j + 8 * (e >> 2) + (e & 3);
                        zt = c == column ? z[j][e] : zt;
                        z[j][e] = c == column || column >= end ? -__builtin_inff() : z[j][e];
                    }
                // (of the two lanes of the row the one that holds the column)
                if (a.target[i] >= 0 && ((a.target[i] >> 2) & 1) == (at.lane >> 5)) z_target[at.row(i)] = zt;
            }
            float m = -__builtin_inff();
#pragma unroll
            for (int j = 0; j < T::NT; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) m = __builtin_fmaxf(m, z[j][e]);
            const auto both = __builtin_amdgcn_permlane32_swap(f2u(m), f2u(m), false, false);
            m = __builtin_fmaxf(u2f(both[0]), u2f(both[1]));
            const float base = m == -__builtin_inff() ? 0.0f : m * kLog2e;
            float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};  // (four chains of additions)
#pragma unroll
            for (int j = 0; j < T::NT; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e & 3] += __builtin_amdgcn_exp2f(__builtin_fmaf(z[j][e], kLog2e, -base));
            const float four = (s[0] + s[1]) + (s[2] + s[3]);
            const auto sums = __builtin_amdgcn_permlane32_swap(f2u(four), f2u(four), false, false);
            mine[i] = f32x2{base, u2f(sums[0]) + u2f(sums[1])};
        };
#pragma unroll
        for (int i = 0; i < T::MT; ++i) {
            __builtin_amdgcn_sched_barrier(0);  // (one row of accumulators at a time: together they overflow the registers)
            if (left >= T::WTN && __builtin_amdgcn_ballot_w64(a.target[i] >= 0) == 0) row_sum(i, std::true_type{});
            else row_sum(i, std::false_type{});
        }
        // the right-hand waves hand over to the left-hand ones
        f32x2 *right = reinterpret_cast<f32x2 *>(at.lds);  // [BM]
        __syncthreads();
        const int wm = at.wave / T::WGN, wn = at.wave % T::WGN;
        if (wn == 1 && at.lane < 32) {
#pragma unroll
            for (int i = 0; i < T::MT; ++i) right[wm * T::WTM + 32 * i + at.lane] = mine[i];
        }
        __syncthreads();
        if (wn == 0 && at.lane < 32) {
#pragma unroll
            for (int i = 0; i < T::MT; ++i) {
                xent_join(mine[i], right[wm * T::WTM + 32 * i + at.lane]);
                if (at.row(i) < M) part[(int64_t)(part0 + at.tn) * M + at.row(i)] = mine[i];
            }
        }
    }
};

// e of a tile, as halves times 2^14 and the token's weight.
using half4 = _Float16 __attribute__((ext_vector_type(4)));
struct XentError {
    static constexpr bool kJoin = false, k192 = false;  // (logits_plan)
    const int64_t *targets;
    const float *loss, *lse, *factor;  // factor [M]: 2^14 and the token's weight; 0 without a target
    uint16_t *out;                     // panels of 64 columns, `wide` columns in all
    int64_t panel;
    int wide;
    int M, N, first;                   // N: columns that exist; those behind them, to the tile's end, become zero
    template <int MT>
    struct Ahead {
        float factor[MT], base[MT], at_target[MT];  // of the rows; what e is at the target, without the factor
        int target[MT];
    };
    template <class T>
    __device__ __forceinline__ Ahead<T::MT> ahead(const HalfPlace<T> &at) const {
        Ahead<T::MT> a;
#pragma unroll
        for (int i = 0; i < T::MT; ++i) {
            const int r = at.row(i);
            const bool row = r < M;
            a.factor[i] = row ? factor[r] : 0.0f;
            a.base[i] = row ? lse[r] : 0.0f;
            a.at_target[i] = row ? loss[r] : 0.0f;
            a.target[i] = row ? xent_column<T>(targets[r], first + at.col0, N - at.col0) : -1;
        }
        return a;
    }
    template <class T>
    __device__ __forceinline__ void operator()(const HalfPlace<T> &at, f32x16 (&acc)[T::MT][T::NT], const Ahead<T::MT> &a) const {
        const int h4 = 4 * (at.lane >> 5), left = N - at.col0;
        HalfLines<T> lines(at);
        __syncthreads();  // (LDS: the last stage's fragments have been read everywhere)
        auto row_errors = [&](int i, auto plain) {
            constexpr bool PLAIN = decltype(plain)::value;
            const float f = a.factor[i];
            // |f| 2^(z log2 e - lse log2 e) with one exponent; a masked token's (its logits are 0, its lse may be anything) is minus infinity
            const float shift = f == 0.0f ? -__builtin_inff() : __builtin_amdgcn_logf(__builtin_fabsf(f)) - a.base[i] * kLog2e;
            const uint32_t sign = f < 0.0f ? 0x80008000u : 0u;
            // exp(-loss) - 1: the target's probability is one less what the others have, to the loss's precision
            float at_target = 0.0f;
            int end = 0, c = -1;
            if constexpr (!PLAIN) {
                at_target = __builtin_fabsf(f) * expm1f(-a.at_target[i]);
                end = left - h4;
                c = a.target[i] - h4;  // (-1 - 4 h meets no column)
                asm volatile("" : "+v"(end), "+v"(c));  // (the comparisons anew in every row: they would all be kept)
            }
#pragma unroll
            for (int j = 0; j < T::NT; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    half4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int column = 32 * j + 8 * g + e;
                        float y = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][4 * g + e], kLog2e, shift));
                        if constexpr (!PLAIN) y = c == column ? at_target : column >= end ? 0.0f : y;
                        v[e] = (_Float16)y;
                    }
                    u32x2 w = __builtin_bit_cast(u32x2, v);
                    w.x ^= sign;
                    w.y ^= sign;
                    lines.put(j, g, w);
                }
        };
#pragma unroll
        for (int i = 0; i < T::MT; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            if (left >= T::WTN && __builtin_amdgcn_ballot_w64(a.target[i] >= 0) == 0) row_errors(i, std::true_type{});
            else row_errors(i, std::false_type{});
            lines.each([&](int r, int c, const u32x4 &v) {
                const int row = at.row0 + 32 * i + r;
                // (read again when it has left the caches: 8192 x 32768 x 2048 984 -> 958 us, in 128x128 tiles 1240 -> 1109)
                if (row < M && at.col0 + c < wide) __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(out + HalfMatrix::at(row, at.col0 + c, panel)));
            });
        }
    }
};

// Statistics of a value that is stored as a half.
__device__ __forceinline__ void xent_count_half(StatsAcc &st, float y) {
    const uint32_t h = f16_from_f32<false>(y, 0u);
    if (y != y) st.nan_seen = 1u;
    st.amax = __builtin_fmaxf(st.amax, __builtin_fabsf(y));
    st.zero_inputs += y == 0.0f ? 1u : 0u;
    st.nonfinite += (h & 0x7C00u) == 0x7C00u ? 1u : 0u;
    st.zero_codes += (h & 0x7FFFu) == 0u ? 1u : 0u;
}

// A gradient, complete in its tile: unscaled, rounded and stored.  WHOLE: rows of whole groups of eight; others get a kernel of their own, whose
// code is there once per band (four times, and the compiler keeps the accumulators in memory).
template <bool WHOLE>
struct XentOut : HalfNoneAhead {
    const int *exponent;
    float scale;
    int rows, cols;
    int64_t row0;  // of the whole output (pieces of dw), for addresses and random bits
    uint16_t *out16;
    uint8_t *out8;
    int sr, sat;
    uint64_t seed, offset;
    mp8_stats *stats;
    template <class T>
    __device__ __forceinline__ void operator()(const HalfPlace<T> &at, f32x16 (&acc)[T::MT][T::NT], HalfNothing) const {
        const float unscale = ldexpf(scale, *exponent - kErrorExponent);
        const Philox rng(seed, offset);
        StatsAcc st;
        const uint32_t seen = stats != nullptr ? StatsAcc::peek(stats) : 0u;
        half_bands<WHOLE ? 4 : 1>(at, acc, [](int, int) { return HalfNothing{}; }, [&](int r, int c, const float (&sum)[8], HalfNothing) {
            if (r >= rows || c >= cols) return;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = sum[e] * unscale;
            const int64_t i = (row0 + r) * (int64_t)cols + c;
            const int n = cols - c;  // of the eight, those that exist
            if (out16 != nullptr) {
                const u32x4 h = half_round8(v);
                if constexpr (WHOLE) {
                    *reinterpret_cast<u32x4 *>(out16 + i) = h;
                } else if (n >= 8) {
                    __builtin_memcpy(out16 + i, &h, 16);
                } else {
#pragma unroll
                    for (int e = 0; e < 7; ++e)
                        if (e < n) out16[i + e] = (uint16_t)(h[e >> 1] >> (16 * (e & 1)));
                }
            }
            if (out8 != nullptr) {
                uint4 w = make_uint4(0u, 0u, 0u, 0u);
                if (sr) w = WHOLE ? rng.block((uint64_t)i >> 3) : rng.eight_at((uint64_t)i);
                const float lo[4] = {v[0], v[1], v[2], v[3]}, hi[4] = {v[4], v[5], v[6], v[7]};
                const u32x2 o = {e5m2_pack4_rt(lo, w.x, w.y, sr != 0, sat != 0), e5m2_pack4_rt(hi, w.z, w.w, sr != 0, sat != 0)};
                if constexpr (WHOLE) {
                    *reinterpret_cast<u32x2 *>(out8 + i) = o;
                } else if (n >= 8) {
                    __builtin_memcpy(out8 + i, &o, 8);
                } else {
#pragma unroll
                    for (int e = 0; e < 7; ++e)
                        if (e < n) out8[i + e] = (uint8_t)(o[e >> 2] >> (8 * (e & 3)));
                }
                if (stats != nullptr) {
                    if (WHOLE || n >= 8) {
                        st.add4(lo, o.x);
                        st.add4(hi, o.y);
                    } else {
#pragma unroll
                        for (int e = 0; e < 7; ++e)
                            if (e < n) st.add1(v[e], (o[e >> 2] >> (8 * (e & 3))) & 0xFFu);
                    }
                }
            } else if (stats != nullptr) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (WHOLE || e < n) xent_count_half(st, v[e]);
            }
        }, [](int, float *) {});
        if (stats != nullptr) {
            __syncthreads();  // (the bands' LDS)
            st.flush(stats, seen, reinterpret_cast<uint32_t (*)[16]>(at.lds));
        }
    }
};

// ---------------------------------------------------------------------------------------
// The small kernels.
// ---------------------------------------------------------------------------------------
// Joins the sums of a row: R rows per block, 256 / R threads each.
template <int R>
__global__ __launch_bounds__(256) void xent_join_kernel(const f32x2 *__restrict__ part, const float *__restrict__ z_target,
                                                        const int64_t *__restrict__ targets, float *__restrict__ loss,
                                                        float *__restrict__ lse, int M, int N, int parts) {
    constexpr int Y = 256 / R;
    __shared__ f32x2 sh[Y][R];
    const int x = threadIdx.x % R, y = threadIdx.x / R, r = blockIdx.x * R + x;
    f32x2 t = {0.0f, 0.0f};
    if (r < M) {
#pragma unroll 4
        for (int k = y; k < parts; k += Y) xent_join(t, part[(int64_t)k * M + r]);
    }
    sh[y][x] = t;
#pragma unroll
    for (int h = Y / 2; h; h /= 2) {
        __syncthreads();
        if (y < h) {
            xent_join(t, sh[y + h][x]);
            sh[y][x] = t;
        }
    }
    if (y != 0 || r >= M) return;
    const int64_t target = targets[r];
    // The base as a logit.  (Divided by log2 e as the tiles' sums have it, in FP32: by one with more digits, what all logits have in common would
    // not cancel, 2e-4 of the loss at logits around 2^14.)
    const double base = (double)t.x / (double)kLog2e;
    if (target < 0 || target >= N) {
        lse[r] = (float)(base + log((double)t.y));
        loss[r] = 0.0f;
    } else {
        const double z = (double)z_target[r], d = base - z;
        double l, all;
        if (t.y == 0.0f || z == (double)__builtin_inff()) {  // nothing beside the target: 0, but for a logit that is not finite
            l = z - z;
            all = z;
        } else if (d >= 600.0) {  // nothing but the others
            all = base + log((double)t.y);
            l = all - z;
        } else {  // log(1 + sum exp(z_j - z))
            l = log1p((double)t.y * exp(d));
            all = z + l;
        }
        loss[r] = (float)l;
        lse[r] = (float)all;
    }
}

// Wide accesses at addresses of any alignment.
template <class V, bool ALIGNED>
__device__ __forceinline__ V xent_load(const void *p) {
    if constexpr (ALIGNED) return *reinterpret_cast<const V *>(p);
    V v;
    __builtin_memcpy(&v, p, sizeof(V));
    return v;
}
// dst <- src [rows, cols] halves or 8-bit codes, as halves in panels, zeros up to the `wide` columns of the last one, tr threads per row; rows
// whose target is none are zero too where targets are given (what a padded token holds must not reach the weights' gradient, not even as
// 0 x NaN).  VEC: rows of whole, aligned groups of eight.  factor, where given, becomes that of a call without token weights.
template <bool CODES, bool VEC>
__global__ __launch_bounds__(256) void xent_copy_kernel(const void *__restrict__ src, int64_t ld_src, uint16_t *__restrict__ dst, int wide,
                                                        int rows, int cols, const int64_t *__restrict__ targets, int N, int tr,
                                                        float *__restrict__ factor, int *__restrict__ exponent) {
    const int64_t r = (int64_t)blockIdx.x * (256 / tr) + threadIdx.x / tr;
    const int c0 = 8 * (threadIdx.x % tr);
    if (r >= rows) return;
    const bool live = targets == nullptr || (targets[r] >= 0 && targets[r] < N);
    if (factor != nullptr && c0 == 0) {
        factor[r] = live ? (float)(1 << kErrorExponent) : 0.0f;
        if (r == 0) *exponent = 0;
    }
    for (int c = c0; c < wide; c += 8 * tr) {
        u32x4 o = {0, 0, 0, 0};
        if (live && c < cols) {
            const auto *from = (const uint8_t *)src + (r * ld_src + c) * (CODES ? 1 : 2);
            if (c + 8 <= cols) {
                if (CODES) {
                    const u32x2 w = xent_load<u32x2, VEC>(from);
                    o = __builtin_bit_cast(u32x4, halves_of((int)w.x, (int)w.y));
                } else {
                    o = xent_load<u32x4, VEC>(from);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (c + e < cols) o[e >> 1] |= (CODES ? (uint32_t)from[e] << 8 : ((const uint16_t *)from)[e]) << (16 * (e & 1));
            }
        }
        *reinterpret_cast<u32x4 *>(dst + HalfMatrix::at(r, c, 64 * (int64_t)rows)) = o;
    }
}

// One block: the exponent of the largest token weight (0 without weights), and every token's factor.
__global__ __launch_bounds__(1024) void xent_factor_kernel(const int64_t *__restrict__ targets, const float *__restrict__ dloss,
                                                           float *__restrict__ factor, int *__restrict__ exponent, int M, int N) {
    __shared__ float sh[16];
    auto live = [&](int r) { return targets[r] >= 0 && targets[r] < N; };
    int e = 0;
    if (dloss != nullptr) {
        float m = 0.0f;
#pragma unroll 4
        for (int r = threadIdx.x; r < M; r += 1024) {
            const float a = live(r) ? __builtin_fabsf(dloss[r]) : 0.0f;
            if (a < __builtin_inff()) m = __builtin_fmaxf(m, a);
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) m = __builtin_fmaxf(m, __shfl_xor(m, d));
        if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = m;
        __syncthreads();
        m = sh[0];
#pragma unroll
        for (int k = 1; k < 16; ++k) m = __builtin_fmaxf(m, sh[k]);
        e = m > 0.0f ? ilogbf(m) + 1 : 0;  // m < 2^e
    }
#pragma unroll 4
    for (int r = threadIdx.x; r < M; r += 1024)
        factor[r] = live(r) ? ldexpf(dloss != nullptr ? dloss[r] : 1.0f, kErrorExponent - e) : 0.0f;
    if (threadIdx.x == 0) *exponent = e;
}

// out = unscaled sum of `slabs` FP32 matrices [rows, ld]: as halves to nearest, and / or as 8-bit codes.  TR threads per row, four columns
// each.
struct XentFinish {
    const float *sum;
    int64_t ld, slab;
    int slabs;
    const int *exponent;
    float scale;
    int64_t rows, cols, row0;  // row0: of the whole output (pieces of dw), for addresses and random bits
    uint16_t *out16;
    uint8_t *out8;
    int sr, sat;
    uint64_t seed, offset;
    mp8_stats *stats;
};
__global__ __launch_bounds__(256) void xent_finish_kernel(const XentFinish p, int tr) {
    const float unscale = ldexpf(p.scale, *p.exponent - kErrorExponent);
    const Philox rng(p.seed, p.offset);
    StatsAcc st;
    const uint32_t seen = p.stats != nullptr ? StatsAcc::peek(p.stats) : 0u;
    const int per = 256 / tr;  // rows of a block
    const bool whole = (p.cols & 3) == 0;
    for (int64_t r = (int64_t)blockIdx.x * per + threadIdx.x / tr; r < p.rows; r += (int64_t)gridDim.x * per) {
        for (int64_t c = 4 * (threadIdx.x % tr); c < p.cols; c += 4 * tr) {
            f32x4 v = *reinterpret_cast<const f32x4 *>(p.sum + r * p.ld + c);
            // (eight loads under way: one by one the 64 slabs of 12 x 460 took 26 us)
            const float *from = p.sum + r * p.ld + c;
            for (int s = 1; s < p.slabs; s += 8) {
                f32x4 more[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) more[u] = s + u < p.slabs ? *reinterpret_cast<const f32x4 *>(from + (s + u) * p.slab) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int u = 0; u < 8; ++u) v += more[u];
            }
            const float y[4] = {v.x * unscale, v.y * unscale, v.z * unscale, v.w * unscale};
            const int64_t at = (p.row0 + r) * p.cols + c;
            const int n = p.cols - c < 4 ? (int)(p.cols - c) : 4;
            uint32_t h[4];
            if (p.out16 != nullptr) {
#pragma unroll
                for (int e = 0; e < 4; ++e) h[e] = f16_from_f32<false>(y[e], 0u);
                if (whole) {
                    const u32x2 o = {h[0] | (h[1] << 16), h[2] | (h[3] << 16)};
                    *reinterpret_cast<u32x2 *>(p.out16 + at) = o;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (e < n) p.out16[at + e] = (uint16_t)h[e];
                }
            }
            if (p.out8 != nullptr) {
                Words4 w = {0, 0};
                if (p.sr) w = rng.words_at((uint64_t)at);
                const uint32_t pk = e5m2_pack4_rt(y, w.r01, w.r23, p.sr != 0, p.sat != 0);
                if (whole) {
                    *reinterpret_cast<uint32_t *>(p.out8 + at) = pk;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (e < n) p.out8[at + e] = (uint8_t)(pk >> (8 * e));
                }
                if (p.stats != nullptr)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (e < n) st.add1(y[e], (pk >> (8 * e)) & 0xFFu);
            } else if (p.stats != nullptr) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < n) xent_count_half(st, y[e]);
            }
        }
    }
    if (p.stats != nullptr) st.flush(p.stats, seen);
}

// ---------------------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------------------
namespace {

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

struct Shape {
    int64_t M, N, K, Kp;
    bool copy_x, copy_w;
    int64_t piece;  // classes per piece
};

constexpr int64_t kPieceBytes = (int64_t)512 << 20;

bool aligned_ld(int64_t K, int64_t ld) { return K % 8 == 0 && ld % 8 == 0; }

Shape make_shape(int64_t M, int64_t N, int64_t K, bool copy_x, bool copy_w, bool backward) {
    Shape s{M, N, K, up(K, 64), copy_x, copy_w, N};
    // bytes per class: of e and of the FP32 sums of dw, of a copy of w
    const int64_t row_e = backward ? (2 * M > 4 * s.Kp ? 2 * M : 4 * s.Kp) : 0, row_w = copy_w ? 2 * s.Kp : 0, row = row_e > row_w ? row_e : row_w;
    if (row) {
        int64_t n = kPieceBytes / row / 256 * 256;
        n = n < 2048 ? 2048 : n;
        const int64_t pieces = (N + n - 1) / n;
        s.piece = pieces == 1 ? N : up((N + pieces - 1) / pieces, 256);
    }
    return s;
}

// The workspace, in order; every part starts at a multiple of 256 bytes.
struct Layout {
    size_t x, w, part, z_target;             // forward: copies of x and of a piece of w, the sums, the targets' logits
    size_t factor, exponent, e, dx, dw, total;  // backward: (copies as above,) the tokens' factors, e, FP32 sums
};
// The logits' tiles: their epilogues take longer than others, and two workgroups per CU hide them behind each other's products.  Measured,
// us, statistics in 256x256 / 128x128 tiles: 9243 x 24384 x 64 166 / 124, 8192 x 32000 x 256 267 / 238, 4096 x 32000 x 512 216 / 211,
// 1021 x 32003 x 1000 85 / 102, 8192 x 32768 x 2048 905 / 1032; the errors 206 / 149, 304 / 279, 235 / 222, 87 / 96, 958 / 1109.
HalfPlan logits_plan(int64_t M, int64_t cols, int64_t K) {
    HalfPlan best = half_plan(1, M, cols, K, false, 1);
    if (best.tile == 64) return best;
    double least = 1e300;
    for (const int tile : {256, 128}) {
        const int64_t tiles = ((M + tile - 1) / tile) * ((cols + tile - 1) / tile);
        if (tiles > (int64_t)1 << 23) continue;  // (of 128x128 only: check_sizes; a launch holds less than 2^32 threads)
        const double slots = tile == 256 ? 256.0 : 512.0, epilogue = tile == 256 ? 8.0 : 2.2;
        const double rounds = std::ceil((double)tiles / slots);
        const double t = rounds * (double)((K + 63) / 64) * (tile == 256 ? 1.6 : 1.05) + (rounds + 1.0) * epilogue;
        if (t < least) {
            least = t;
            best.tile = tile;
        }
    }
    return best;
}
int parts_of(const Shape &s) {  // sums per token
    int n = 0;
    for (int64_t c = 0; c < s.N; c += s.piece) {
        const int64_t cols = s.N - c < s.piece ? s.N - c : s.piece;
        const int w = logits_plan(s.M, cols, s.K).tile;
        n += (int)((cols + w - 1) / w);
    }
    return n;
}
// dx and dw.  A tile that holds the complete sum stores the gradient itself; otherwise FP32 sums (of every slice; of all pieces, for dx) pass
// through the workspace.
struct BwdPlans {
    HalfPlan dx, dw;
    bool dx_direct, dw_direct;
};
BwdPlans bwd_plans(const Shape &s) {
    BwdPlans p;
    p.dx = half_plan(1, s.M, s.K, s.piece, false, 64);
    p.dw = half_plan(1, s.piece, s.K, s.M, false, 64);
    p.dx_direct = p.dx.splits == 1 && s.piece >= s.N;
    p.dw_direct = p.dw.splits == 1;
    return p;
}
Layout make_layout(const Shape &s, bool backward, bool dx, bool dw) {
    Layout l{};
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t here = at;
        at += (size_t)up(bytes, 256);
        return here;
    };
    if (s.copy_x) l.x = take(2 * s.M * s.Kp);
    if (s.copy_w) l.w = take(2 * up(s.piece, 8) * s.Kp);
    if (!backward) {
        l.part = take(8 * (int64_t)parts_of(s) * s.M);
        l.z_target = take(4 * s.M);
    } else {
        l.factor = take(4 * s.M);
        l.exponent = take(4);
        l.e = take(2 * s.M * up(s.piece, 64));
        const BwdPlans p = bwd_plans(s);
        if (dx && !p.dx_direct) l.dx = take(4 * p.dx.splits * s.M * s.Kp);
        if (dw && !p.dw_direct) l.dw = take(4 * p.dw.splits * s.piece * s.Kp);
    }
    l.total = at;
    return l;
}

// Sizes every product of which fits 63 bits and every 32-bit offset of a kernel: a tile's rows span 256 * ld * 2 bytes.
mp8_status check_sizes(int64_t M, int64_t N, int64_t K, int64_t ldx, int64_t ldw) {
    if (M < 0 || N < 0 || K < 0) return MP8_ERR_INVALID_ARG;
    const int64_t most = (int64_t)1 << 22;
    if (M > most || N > most || K > ((int64_t)1 << 20)) return MP8_ERR_UNSUPPORTED;
    if (((M + 255) / 256) * ((N + 255) / 256) > ((int64_t)1 << 23)) return MP8_ERR_UNSUPPORTED;  // workgroups of a launch
    if (ldx < K || ldw < K) return MP8_ERR_INVALID_ARG;
    if (ldx > ((int64_t)1 << 21) || ldw > ((int64_t)1 << 21)) return MP8_ERR_UNSUPPORTED;
    return MP8_OK;
}

template <bool BTN, bool ATN, class Epi>
bool product(int tile, const HalfMatrix &a, const HalfMatrix &b, int64_t rows, int64_t cols, int64_t kc, int splits, const Epi &epi, hipStream_t stream) {
    return half_gemm_launch_plan<ATN, BTN>(tile, half_gemm_args(a, b, rows, cols, kc, tile, splits, false, 1), epi, stream);
}

bool copy_half(const void *src, bool codes, int64_t ld_src, uint16_t *dst, int64_t rows, int64_t cols,
               const int64_t *targets, int64_t N, float *factor, int *exponent, hipStream_t stream) {
    const int64_t wide = up(cols, 64);
    int tr = 1;
    while (tr < 256 && 8 * tr < wide) tr *= 2;
    const bool vec = cols % 8 == 0 && ld_src % 8 == 0;
    const auto kernel = codes ? (vec ? xent_copy_kernel<true, true> : xent_copy_kernel<true, false>)
                              : (vec ? xent_copy_kernel<false, true> : xent_copy_kernel<false, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + 256 / tr - 1) / (256 / tr))), dim3(256), 0, stream, src, ld_src, dst, (int)wide, (int)rows, (int)cols,
                       targets, (int)N, tr, factor, exponent);
    return hipGetLastError() == hipSuccess;
}

}  // namespace
}  // namespace mp8

extern "C" size_t mp8_softmax_xent_fwd_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t ldw) {
    using namespace mp8;
    if (check_sizes(M, N, K, K, ldw) != MP8_OK || M == 0 || N == 0 || K == 0) return 0;
    return make_layout(make_shape(M, N, K, true, !aligned_ld(K, ldw), false), false, false, false).total;
}

extern "C" size_t mp8_softmax_xent_bwd_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t ldw) {
    using namespace mp8;
    if (check_sizes(M, N, K, K, ldw) != MP8_OK || M == 0 || N == 0 || K == 0) return 0;
    return make_layout(make_shape(M, N, K, true, !aligned_ld(K, ldw), true), true, true, true).total;
}

extern "C" mp8_status mp8_softmax_xent_fwd_fp16(int64_t M, int64_t N, int64_t K, const void *x, int x_is_e5m2, int64_t ldx,
                                                const uint16_t *w, int64_t ldw, const int64_t *targets, float *loss, float *lse,
                                                void *workspace, size_t workspace_bytes, void *stream) {
    using namespace mp8;
    const mp8_status sizes = check_sizes(M, N, K, ldx, ldw);
    if (sizes != MP8_OK) return sizes;
    if (M == 0 || N == 0 || K == 0) return MP8_OK;
    if (!x || !w || !targets || !loss || !lse) return MP8_ERR_INVALID_ARG;
    if (((uintptr_t)x | (uintptr_t)w | (uintptr_t)workspace) & 15u) return MP8_ERR_ALIGNMENT;
    const Shape s = make_shape(M, N, K, x_is_e5m2 || !aligned_ld(K, ldx), !aligned_ld(K, ldw), false);
    const Layout l = make_layout(s, false, false, false);
    if (!workspace || workspace_bytes < l.total) return MP8_ERR_WORKSPACE;
    uint8_t *ws = (uint8_t *)workspace;
    hipStream_t st = (hipStream_t)stream;
    HalfMatrix X = HalfMatrix::rows((const uint16_t *)x, ldx);
    if (s.copy_x) {
        X = HalfMatrix::panels((uint16_t *)(ws + l.x), M);
        if (!copy_half(x, x_is_e5m2 != 0, ldx, (uint16_t *)(ws + l.x), M, K, nullptr, N, nullptr, nullptr, st)) return MP8_ERR_HIP;
    }
    int parts = 0;
    for (int64_t c = 0; c < N; c += s.piece) {
        const int64_t cols = N - c < s.piece ? N - c : s.piece;
        HalfMatrix W = HalfMatrix::rows(w + c * ldw, ldw);
        if (s.copy_w) {
            if (!copy_half(W.p, false, ldw, (uint16_t *)(ws + l.w), cols, K, nullptr, N, nullptr, nullptr, st)) return MP8_ERR_HIP;
            W = HalfMatrix::panels((uint16_t *)(ws + l.w), cols);
        }
        const int tile = logits_plan(M, cols, K).tile;
        const XentStats epi{targets, (f32x2 *)(ws + l.part), (float *)(ws + l.z_target), (int)M, (int)cols, (int)c, parts};
        if (!product<false, false>(tile, X, W, M, cols, K, 1, epi, st)) return MP8_ERR_HIP;
        parts += (int)((cols + tile - 1) / tile);
    }
    const int per = M >= 512 ? 8 : 1;
    hipLaunchKernelGGL((per == 8 ? xent_join_kernel<8> : xent_join_kernel<1>), dim3((unsigned)((M + per - 1) / per)), dim3(256), 0, st, (const f32x2 *)(ws + l.part), (const float *)(ws + l.z_target),
                       targets, loss, lse, (int)M, (int)N, parts);
    return hipGetLastError() == hipSuccess ? MP8_OK : MP8_ERR_HIP;
}

extern "C" mp8_status mp8_softmax_xent_bwd_fp16(int64_t M, int64_t N, int64_t K, const void *x, int x_is_e5m2, int64_t ldx,
                                                const uint16_t *w, int64_t ldw, const int64_t *targets, const float *loss,
                                                const float *lse, const float *dloss, float scale, uint16_t *dx16, uint8_t *dx8,
                                                uint16_t *dw16, uint8_t *dw8, mp8_round round, int flags, uint64_t seed,
                                                uint64_t dx_offset, uint64_t dw_offset, mp8_stats *dx_stats, mp8_stats *dw_stats,
                                                void *workspace, size_t workspace_bytes, void *stream) {
    using namespace mp8;
    const mp8_status sizes = check_sizes(M, N, K, ldx, ldw);
    if (sizes != MP8_OK) return sizes;
    if (round != MP8_RNE && round != MP8_SR) return MP8_ERR_INVALID_ARG;
    if (flags & ~MP8_FLAG_SATURATE) return MP8_ERR_INVALID_ARG;
    if (M == 0 || N == 0 || K == 0) return MP8_OK;
    const bool dx = dx16 || dx8, dw = dw16 || dw8;
    if (!dx && !dw) return MP8_ERR_INVALID_ARG;
    if (!x || !w || !targets || !loss || !lse) return MP8_ERR_INVALID_ARG;
    if (((uintptr_t)x | (uintptr_t)w | (uintptr_t)dx16 | (uintptr_t)dx8 | (uintptr_t)dw16 | (uintptr_t)dw8 | (uintptr_t)workspace) & 15u)
        return MP8_ERR_ALIGNMENT;
    const Shape s = make_shape(M, N, K, true, !aligned_ld(K, ldw), true);
    const Layout l = make_layout(s, true, dx, dw);
    if (!workspace || workspace_bytes < l.total) return MP8_ERR_WORKSPACE;
    uint8_t *ws = (uint8_t *)workspace;
    hipStream_t st = (hipStream_t)stream;
    uint16_t *xs = (uint16_t *)(ws + l.x), *e = (uint16_t *)(ws + l.e);
    float *factor = (float *)(ws + l.factor), *dxs = (float *)(ws + l.dx), *dws = (float *)(ws + l.dw);
    int *exponent = (int *)(ws + l.exponent);
    if (!copy_half(x, x_is_e5m2 != 0, ldx, xs, M, K, targets, N, dloss ? nullptr : factor, exponent, st)) return MP8_ERR_HIP;
    if (dloss) {
        hipLaunchKernelGGL(xent_factor_kernel, dim3(1), dim3(1024), 0, st, targets, dloss, factor, exponent, (int)M, (int)N);
        if (hipGetLastError() != hipSuccess) return MP8_ERR_HIP;
    }
    const int64_t K8 = up(K, 8);
    const HalfMatrix E = HalfMatrix::panels(e, M), X = HalfMatrix::panels(xs, M);
    const BwdPlans plans = bwd_plans(s);
    auto finish = [&](const float *sum, int64_t slab, int slabs, int64_t rows, int64_t row0, uint16_t *out16, uint8_t *out8, uint64_t offset,
                      mp8_stats *stats) {
        const XentFinish f{sum, s.Kp, slab, slabs, exponent, scale, rows, K, row0, out16, out8, round == MP8_SR, (flags & MP8_FLAG_SATURATE) != 0,
                           seed, offset, stats};
        int tr = 1;
        while (tr < 256 && 4 * tr < K) tr *= 2;
        int64_t blocks = (rows + 256 / tr - 1) / (256 / tr);
        if (stats != nullptr && blocks > 2048) blocks = 2048;
        hipLaunchKernelGGL(xent_finish_kernel, dim3((unsigned)blocks), dim3(256), 0, st, f, tr);
        return hipGetLastError() == hipSuccess;
    };
    // (a, b) -> rows [row0, row0 + rows) of a gradient, complete
    auto direct = [&](auto atn, int tile, const HalfMatrix &a, const HalfMatrix &b, int64_t rows, int64_t kc, int64_t row0, uint16_t *out16,
                      uint8_t *out8, uint64_t offset, mp8_stats *stats) {
        constexpr bool ATN = decltype(atn)::value;
        auto run = [&](auto whole) {
            const XentOut<decltype(whole)::value> epi{{}, exponent, scale, (int)rows, (int)K, row0, out16, out8, round == MP8_SR, (flags & MP8_FLAG_SATURATE) != 0,
                                                      seed, offset, stats};
            return product<true, ATN>(tile, a, b, ATN ? up(rows, 8) : rows, K8, kc, 1, epi, st);
        };
        return K % 8 == 0 ? run(std::true_type{}) : run(std::false_type{});
    };
    for (int64_t c = 0; c < N; c += s.piece) {
        const int64_t cols = N - c < s.piece ? N - c : s.piece;
        HalfMatrix W = HalfMatrix::rows(w + c * ldw, ldw);
        if (s.copy_w) {
            if (!copy_half(W.p, false, ldw, (uint16_t *)(ws + l.w), cols, K, nullptr, N, nullptr, nullptr, st)) return MP8_ERR_HIP;
            W = HalfMatrix::panels((uint16_t *)(ws + l.w), cols);
        }
        const XentError epi{targets, loss, lse, factor, e, E.panel, (int)up(cols, 64), (int)M, (int)cols, (int)c};
        if (!product<false, false>(logits_plan(M, cols, K).tile, X, W, M, cols, K, 1, epi, st)) return MP8_ERR_HIP;
        if (dx) {
            if (plans.dx_direct) {
                if (!direct(std::false_type{}, plans.dx.tile, E, W, M, cols, 0, dx16, dx8, dx_offset, dx_stats)) return MP8_ERR_HIP;
            } else {
                const HalfEpiSum sum{{}, dxs, s.Kp, M * s.Kp, (int)M, (int)K, c != 0};
                if (!product<true, false>(plans.dx.tile, E, W, M, K8, cols, plans.dx.splits, sum, st)) return MP8_ERR_HIP;
            }
        }
        if (dw) {
            if (plans.dw_direct) {
                if (!direct(std::true_type{}, plans.dw.tile, E, X, cols, M, c, dw16, dw8, dw_offset, dw_stats)) return MP8_ERR_HIP;
            } else {
                const HalfEpiSum sum{{}, dws, s.Kp, s.piece * s.Kp, (int)cols, (int)K, 0};
                if (!product<true, true>(plans.dw.tile, E, X, up(cols, 8), K8, M, plans.dw.splits, sum, st)) return MP8_ERR_HIP;
                if (!finish(dws, s.piece * s.Kp, plans.dw.splits, cols, c, dw16, dw8, dw_offset, dw_stats)) return MP8_ERR_HIP;
            }
        }
    }
    if (dx && !plans.dx_direct && !finish(dxs, M * s.Kp, plans.dx.splits, M, 0, dx16, dx8, dx_offset, dx_stats)) return MP8_ERR_HIP;
    return MP8_OK;
}
