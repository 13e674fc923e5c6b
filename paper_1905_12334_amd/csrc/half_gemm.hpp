// Products of half-precision matrices, out[r, c] = sum_j a[r, j] b[c, j], FP32 accumulation, on the half-precision matrix
// instruction, with what becomes of a finished FP32 tile left to the caller (Epi): the softmax's statistics or its gradient
// (xent.hip), a Gram matrix, a polynomial of it or the next iterate (ortho.hip).
#pragma once

#include "gemm_common.hpp"

namespace mp8 {

// A matrix of halves: element (r, c) at r ld + (c / 64) panel + c % 64.  panel = 64: rows as usual; otherwise columns in panels of 64, which
// matrices made here are laid out in (ld = 64, panel = 64 times the rows): what a stage needs of an operand, and what a tile stores, is
// contiguous then but for the panels.
struct HalfMatrix {
    const uint16_t *p;
    int64_t ld, panel, batch;  // in halves; batch: between matrices
    static __host__ __device__ int64_t at(int64_t r, int64_t c, int64_t panel) { return (c >> 6) * panel + 64 * r + (c & 63); }  // in panels
    static HalfMatrix rows(const uint16_t *p, int64_t ld) { return {p, ld, 64, 0}; }
    static HalfMatrix panels(const uint16_t *p, int64_t rows, int64_t batch = 0) { return {p, 64, 64 * rows, batch}; }
};

// An operand is stored with its contraction index contiguous ([rows, kc]), or contraction-major ([kc, rows]).  Leading dimensions, panel and
// batch strides in bytes; addresses and all of them are multiples of 16.  A row-major operand is read to the next multiple of 8 of its
// contraction, where it has to hold zeros (or finite values, if the other operand holds zeros there); a contraction-major one has a
// multiple of 8 rows.
struct HalfGemm {
    const uint8_t *a, *b;
    int64_t lda, ldb, a_panel, b_panel, a_batch, b_batch;
    int rows, cols;      // of the output; loads beyond them are clamped to the last row (or eight rows), and never stored
    int ksteps, tail;    // stages of 64, and the contraction indices of a last, incomplete one (0: none; see GemmArgs::tail)
    int splits, ks_per, ks_extra;
    int tiles_m, tiles_n;
    int symmetric;       // square output of which only the tiles on and above the diagonal are made
    const uint32_t *skip;  // nullable: a call that is skipped if this is not zero
    uint32_t total;        // tiles of all slices and batches
    // A sliced contraction whose epilogue wants the whole sum (Epi::kJoin): every slice's tile goes to `parts`, and the workgroup that finds
    // in `arrived` (one word per tile, zero before and after the call) that it is the last one adds them up, in the order of the slices.
    float *parts;
    uint32_t *arrived;
    FastDiv div_tiles;   // by the tiles of one slice
    FastDiv div_splits;
    FastDiv div_band, div_last;  // by 8 * tiles_n, by the height of the last band of 8 tile rows
};

// Which part of the output a workgroup makes.
struct HalfTile {
    int batch, split, tm, tn;
    uint32_t tile;  // among those of its batch
};

// Consecutive workgroups go to different XCDs, each with an L2 of its own: number i is the i/8-th tile of the i%8-th eighth of
// them, so that what runs on one XCD is a run of neighbours, in bands of eight tile rows.
__device__ __forceinline__ HalfTile half_tile(const HalfGemm &p) {
    const uint32_t n = gridDim.x, i = blockIdx.x, q = n >> 3, r = n & 7, x = i & 7;
    uint32_t id = x * q + (x < r ? x : r) + (i >> 3);
    HalfTile t;
    uint32_t tile, split;
    id = fastdiv(id, p.div_tiles, tile);
    t.batch = (int)fastdiv(id, p.div_splits, split);
    t.split = (int)split;
    t.tile = tile;
    if (p.symmetric) {
        // row i of the upper triangle starts at i (2 T - i + 1) / 2; counted from the end, row T - 1 - k has k + 1 tiles
        const uint32_t T = (uint32_t)p.tiles_m, back = T * (T + 1) / 2 - 1 - tile;
        uint32_t k = (uint32_t)((__builtin_sqrtf(8.0f * (float)back + 1.0f) - 1.0f) * 0.5f);
        if (k * (k + 1) / 2 > back) --k;
        if ((k + 1) * (k + 2) / 2 <= back) ++k;
        t.tm = (int)(T - 1 - k);
        t.tn = (int)(T - 1 - (back - k * (k + 1) / 2));
    } else {
        uint32_t in_band, y;
        const uint32_t band = fastdiv(tile, p.div_band, in_band);
        const uint32_t left = (uint32_t)p.tiles_m - 8 * band;
        if (left >= 8) {
            t.tn = (int)(in_band >> 3);
            y = in_band & 7;
        } else {
            t.tn = (int)fastdiv(in_band, p.div_last, y);
        }
        t.tm = (int)(8 * band + y);
    }
    t.batch = __builtin_amdgcn_readfirstlane(t.batch);
    t.split = __builtin_amdgcn_readfirstlane(t.split);
    t.tm = __builtin_amdgcn_readfirstlane(t.tm);
    t.tn = __builtin_amdgcn_readfirstlane(t.tn);
    return t;
}

// Tiles of four waves; their schedules are described at the kernel.  WGM x WGN waves have a part of the tile each, a grid of 32x32
// accumulators (kByIndex: when the sums are complete).
enum HalfSchedule { kAhead, kWhole, kByIndex };
template <int BM_, int BN_, int NSTAGE_, int MINBLOCKS_, HalfSchedule SCHEDULE_>
struct HalfTiling {
    static constexpr int BM = BM_, BN = BN_, WGM = 2, WGN = 2, NSTAGE = NSTAGE_, MINBLOCKS = MINBLOCKS_;
    static constexpr int WTM = BM / WGM, WTN = BN / WGN, MT = WTM / 32, NT = WTN / 32;
    static constexpr HalfSchedule SCHEDULE = SCHEDULE_;
};
using Half256 = HalfTiling<256, 256, 2, 1, kAhead>;
using Half192 = HalfTiling<192, 192, 2, 1, kAhead>;
using Half128 = HalfTiling<128, 128, 2, 2, kWhole>;
using Half64 = HalfTiling<64, 64, 4, 2, kWhole>;
using Half64Few = HalfTiling<64, 64, 8, 1, kByIndex>;  // up to one per CU
using f32x2 = float __attribute__((ext_vector_type(2)));

// Where a lane's accumulators lie.  Element e of accumulator (i, j) is row row(i), column col(j) + 8 (e / 4) + e % 4.
template <class T>
struct HalfPlace {
    int batch, split, tm, tn;
    int row0, col0;  // of the wave's part
    int wave, lane;
    uint8_t *lds;    // the operand ring, which other waves may still be reading
    __device__ __forceinline__ int row(int i) const { return row0 + 32 * i + (lane & 31); }
    __device__ __forceinline__ int col(int j) const { return col0 + 32 * j + 4 * (lane >> 5); }
};

// Operands pass through a ring of 128-byte-wide slabs in LDS, filled by direct-to-LDS loads, a stage (64 contraction indices)
// being four sub-steps of sixteen.  Three schedules:
//   kAhead (one wave per SIMD): as in gemm_mfma_kernel, fragments are fetched one sub-step ahead, everything stands between two
//     matrix instructions, and the barrier stands behind the third sub-step, by which all fragments of the stage have been read;
//     a's ring is one slab longer, all 160 KB of LDS at 256x256, so that its loads are spread over the stage
//   kWhole (two workgroups per CU): behind the barrier all fragments of the next stage are requested, then the loads of the stage that
//     takes the place of the current one, then the current stage is multiplied; the other workgroup fills what is left
//   kByIndex (few tiles, long contractions): the same, but each wave multiplies the whole tile over one of the four sub-steps, so that no
//     fragment is read from LDS twice, and the waves' sums are added up at the end; a ring of eight stages
// Gaussian operands: 8192 x 2048 over 32768 in 256x256 tiles 838 us = 1310 TFLOP/s (a library product of these sizes 1072 us; bounded by the
// power that such data draws and the clock it leaves, below 2 GHz), 6007 x 1000 over 37003 in 256x256 tiles 418 us = 1060, in 128x128 tiles
// 536 us = 830 (the other schedule is 10 % slower there).  Small tiles are bounded by what a CU gets from L2 (14 TB/s in all: 0.6 us per
// stage of 256 tiles of 128x128).
// Slab images:
//   row-major: row r is 128 bytes, its 16-byte chunk c sits in slot c ^ ((r >> 1) & 7)
//   contraction-major: panels of 64 tile rows; 64 contraction rows of 128 bytes, chunk c of contraction row k in slot
//     c ^ (4 ((k >> 1) & 1)).  The transposing read names 4 x 4 halves per 16 lanes: lanes 0 .. 31 read four contraction
//     rows of four chunks, which this swizzle spreads over all 64 banks.
template <class T, bool ATN, bool BTN, class Epi>
__global__ __launch_bounds__(256, T::MINBLOCKS) void half_gemm_kernel(const HalfGemm p, const Epi epi) {
    constexpr int BM = T::BM, BN = T::BN, WTM = T::WTM, WTN = T::WTN, MT = T::MT, NT = T::NT, NSTAGE = T::NSTAGE;
    constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, STAGE = A_BYTES + B_BYTES;
    constexpr int A_DMA = BM / 32, B_DMA = BN / 32, G = A_DMA + B_DMA;  // direct loads per wave and stage
    constexpr int F = MT + NT, NM = MT * NT;                             // fragments and matrix instructions per sub-step
    static_assert(G * (NSTAGE - 1) < 64, "vmcnt range");
    // kAhead: the ring of a has one slab more than that of b
    constexpr bool AHEAD = T::SCHEDULE == kAhead;
    constexpr int RING_A = (NSTAGE + 1) * A_BYTES;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[NSTAGE * STAGE + (AHEAD ? A_BYTES : 0)];

    if (p.skip != nullptr && *p.skip != 0u) return;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / T::WGN, wn = wave % T::WGN;

    const bool has_tail = p.tail != 0;
    const int64_t a_kstep = ATN ? 64 * p.lda : p.a_panel, b_kstep = BTN ? 64 * p.ldb : p.b_panel;

    // load q of this wave: the slab's KB u = wave + 4 q
    auto krow = [&](int q) { return 8 * ((wave + 4 * q) & 7) + (lane >> 3); };  // contraction-major: of the stage's 64
    const int lchunk = (lane & 7) ^ ((4 * wave + (lane >> 4)) & 7), lchunk_t = (lane & 7) ^ (((lane >> 4) & 1) << 2);
    auto offset = [&](bool km, int q, int origin, int extent, int64_t ld, int64_t panel) -> uint32_t {
        if (km) {
            int m = 64 * ((wave + 4 * q) >> 3) + 8 * lchunk_t;
            m = origin + m + 8 <= extent ? m : extent - 8 - origin;
            return (uint32_t)(krow(q) * ld + (m >> 6) * panel + 2 * (m & 63));
        }
        int r = 8 * (wave + 4 * q) + (lane >> 3);
        r = origin + r < extent ? r : extent - 1 - origin;
        return (uint32_t)(r * ld) + 16 * lchunk;
    };
    const HalfTile tile = half_tile(p);
    const int row0 = tile.tm * BM, col0 = tile.tn * BN;
    const int ks_begin = tile.split * p.ks_per + (tile.split < p.ks_extra ? tile.split : p.ks_extra);
    const int ks_count = __builtin_amdgcn_readfirstlane(p.ks_per + (tile.split < p.ks_extra ? 1 : 0));
    const int first = ks_begin - (has_tail ? 1 : 0);  // stage s of this slice covers indices 64 (first + s) ..
    const bool tail_first = has_tail && ks_begin == 0;
    const uint8_t *a_tile = uniform_ptr(p.a + tile.batch * p.a_batch + (ATN ? (row0 >> 6) * p.a_panel : row0 * p.lda) + first * a_kstep);
    const uint8_t *b_tile = uniform_ptr(p.b + tile.batch * p.b_batch + (BTN ? (col0 >> 6) * p.b_panel : col0 * p.ldb) + first * b_kstep);
    uint32_t oa[A_DMA], ob[B_DMA];
#pragma unroll
    for (int q = 0; q < A_DMA; ++q) oa[q] = offset(ATN, q, row0, p.rows, p.lda, p.a_panel);
#pragma unroll
    for (int q = 0; q < B_DMA; ++q) ob[q] = offset(BTN, q, col0, p.cols, p.ldb, p.b_panel);
    const HalfPlace<T> at{tile.batch, tile.split, tile.tm, tile.tn, row0 + wm * WTM, col0 + wn * WTN, wave, lane, lds};
    auto ahead = epi.ahead(at);  // what the epilogue wants to have read by then
    const uint32_t lds0 = lds_address(lds);
    auto issue_one = [&](int s, int q) {  // load q (0 .. G-1) of stage s
        const uint32_t at = lds0 + (s % NSTAGE) * STAGE + wave * 1024;
        if (q < A_DMA) dma16(a_tile + s * a_kstep, oa[q < A_DMA ? q : 0], at + q * 4096);
        else dma16(b_tile + s * b_kstep, ob[q >= A_DMA ? q - A_DMA : 0], at + A_BYTES + (q - A_DMA) * 4096);
    };
    // the incomplete stage (stage 0 of the first slice): the contraction's last indices, and zeros
    auto issue_tail = [&]() {
        const uint32_t at = lds0 + wave * 1024;
        const uint8_t *ak = a_tile + (int64_t)p.ksteps * a_kstep, *bk = b_tile + (int64_t)p.ksteps * b_kstep;
        auto inside = [&](bool km, int q) { return (km ? krow(q) : 8 * lchunk) < p.tail; };
#pragma unroll
        for (int q = 0; q < A_DMA; ++q) dma16_or_zero(ak, oa[q], inside(ATN, q), at + q * 4096);
#pragma unroll
        for (int q = 0; q < B_DMA; ++q) dma16_or_zero(bk, ob[q], inside(BTN, q), at + (AHEAD ? RING_A : A_BYTES) + q * 4096);
    };

    // The fragment of A (or B) tile rows m .. m + 31 for sub-step `sub`: lane l holds contraction indices 16 sub + 8 (l / 32) .. +7 of row
    // m + l % 32.
    const int frow = lane & 31, fk = lane >> 5, fsw = (frow >> 1) & 7, t16 = lane & 15;
    const int kt = 8 * fk + (t16 >> 2);                                  // transposing reads: this lane's contraction row
    const int ct = ((lane >> 4) & 1) * 2 + ((t16 & 3) >> 1);             // and chunk
    const int ft = kt * 128 + ((ct ^ (((t16 >> 3) & 1) << 2)) << 4) + 8 * (t16 & 1);
    auto fragment_at = [&](const uint8_t *slab, int sub, bool of_a, int m) -> half8 {
        if (of_a ? ATN : BTN) {
            using h4 = short __attribute__((ext_vector_type(4)));
            using lds_h4 = __attribute__((address_space(3))) h4;
            // (the panel's upper 32 tile rows are chunks 4 .. 7: the other value of the swizzled bit)
            const uint8_t *at = slab + (m >> 6) * 8192 + (ft ^ ((m & 32) << 1)) + 16 * sub * 128;
            const h4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_h4 *)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_h4 *)(at + 512));
            return __builtin_bit_cast(half8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
        return *reinterpret_cast<const half8 *>(slab + (m + frow) * 128 + (((2 * sub + fk) ^ fsw) << 4));
    };
    auto fragment_of = [&](int s, int sub, bool of_a, int m) { return fragment_at(lds + (s % NSTAGE) * STAGE + (of_a ? 0 : A_BYTES), sub, of_a, m); };
    // fragment f of this wave's part: A tile f for f < MT, B tile f - MT otherwise
    auto fragment = [&](int s, int sub, int f) { return f < MT ? fragment_of(s, sub, true, wm * WTM + 32 * f) : fragment_of(s, sub, false, wn * WTN + 32 * (f - MT)); };
    auto order = [&](int n) { return n == 0 ? MT : n == 1 ? 0 : n < NT + 1 ? MT + n - 1 : n - NT; };  // as first needed

    f32x16 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

    // at most `later` (0 .. NSTAGE - 1) whole stages of this wave's loads under way
    auto wait_later = [&](int later) {
        if (later >= NSTAGE - 1) wait_vm_lds<G * (NSTAGE - 1)>();
        else if (later == NSTAGE - 2) wait_vm_lds<G * (NSTAGE - 2)>();
        else if (NSTAGE == 4 && later == 1) wait_vm_lds<NSTAGE == 4 ? G : 0>();
        else wait_vm_lds<0>();
    };
    auto wait_stage = [&](int s) {  // stage s has landed; the buffer of stage s - 1 has not been given away yet
        const int later = ks_count - 1 - s;
        wait_later(later < NSTAGE - 2 ? later : NSTAGE - 2);
    };
    // load q of a slab of a or b into LDS at `slot`
    auto issue_a = [&](int s, int q, uint32_t slot) { dma16(a_tile + s * a_kstep, oa[q], lds0 + slot + wave * 1024 + q * 4096); };
    auto issue_b = [&](int s, int q, uint32_t slot) { dma16(b_tile + s * b_kstep, ob[q], lds0 + RING_A + slot + wave * 1024 + q * 4096); };
    if constexpr (AHEAD) {
#pragma unroll
        for (int s = 0; s < NSTAGE; ++s)
            if (s < ks_count) {
                if (s == 0 && tail_first) issue_tail();
                else {
#pragma unroll
                    for (int q = 0; q < A_DMA; ++q) issue_a(s, q, s * A_BYTES);
#pragma unroll
                    for (int q = 0; q < B_DMA; ++q) issue_b(s, q, s * B_BYTES);
                }
            }
    } else {
#pragma unroll
        for (int s = 0; s < NSTAGE; ++s)
            if (s < ks_count) {
                if (s == 0 && tail_first) issue_tail();
                else
#pragma unroll
                    for (int q = 0; q < G; ++q) issue_one(s, q);
            }
    }
    wait_later((ks_count < NSTAGE ? ks_count : NSTAGE) - 1);
    __syncthreads();
    if constexpr (T::SCHEDULE == kByIndex) {
        constexpr int MK = BM / 32, NK = BN / 32;
        static_assert(4 * MK * NK * 4096 <= NSTAGE * STAGE, "the waves' sums fit the ring");
        f32x16 part[MK][NK] = {};
        half8 fr[2][MK + NK];
        auto read = [&](int s, half8 (&to)[MK + NK]) {
#pragma unroll
            for (int f = 0; f < MK + NK; ++f) to[f] = fragment_of(s, wave, f < MK, 32 * (f < MK ? f : f - MK));
        };
        auto stage = [&](int t, half8 (&now)[MK + NK], half8 (&then)[MK + NK]) {
            if (t + 1 < ks_count) {
                wait_stage(t + 1);
                __syncthreads();  // the fragments of stage t have been read everywhere
                read(t + 1, then);
                if (t + NSTAGE < ks_count) {
#pragma unroll
                    for (int q = 0; q < G; ++q) issue_one(t + NSTAGE, q);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < MK; ++i)
#pragma unroll
                for (int j = 0; j < NK; ++j) part[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(now[MK + j], now[i], part[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        };
        read(0, fr[0]);
        int t = 0;
        for (; t + 1 < ks_count; t += 2) {
            stage(t, fr[0], fr[1]);
            stage(t + 1, fr[1], fr[0]);
        }
        if (t < ks_count) stage(t, fr[0], fr[1]);
        __syncthreads();
        f32x4 *sums = reinterpret_cast<f32x4 *>(lds);  // [wave][i][j][e / 4][lane]
#pragma unroll
        for (int i = 0; i < MK; ++i)
#pragma unroll
            for (int j = 0; j < NK; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    sums[(((wave * MK + i) * NK + j) * 4 + g) * 64 + lane] = f32x4{part[i][j][4 * g], part[i][j][4 * g + 1], part[i][j][4 * g + 2], part[i][j][4 * g + 3]};
        __syncthreads();
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    f32x4 v = sums[((wm * MT + i) * NK + wn * NT + j) * 256 + g * 64 + lane];
#pragma unroll
                    for (int w = 1; w < 4; ++w) v += sums[(((w * MK + wm * MT + i) * NK + wn * NT + j) * 4 + g) * 64 + lane];
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][4 * g + e] = v[e];
                }
    } else if constexpr (T::SCHEDULE == kWhole) {
        half8 fr[2][4][F];
        auto read = [&](int s, half8 (&to)[4][F]) {
#pragma unroll
            for (int sub = 0; sub < 4; ++sub)
#pragma unroll
                for (int n = 0; n < F; ++n) to[sub][order(n)] = fragment(s, sub, order(n));
        };
        auto stage = [&](int t, half8 (&now)[4][F], half8 (&then)[4][F]) {
            if (t + 1 < ks_count) {
                wait_stage(t + 1);
                __syncthreads();  // the fragments of stage t have been read everywhere
                read(t + 1, then);
                if (t + NSTAGE < ks_count) {
#pragma unroll
                    for (int q = 0; q < G; ++q) issue_one(t + NSTAGE, q);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int sub = 0; sub < 4; ++sub)
#pragma unroll
                for (int k = 0; k < NM; ++k)
                    acc[k / NT][k % NT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(now[sub][MT + k % NT], now[sub][k / NT], acc[k / NT][k % NT], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        };
        read(0, fr[0]);
        int t = 0;
        for (; t + 1 < ks_count; t += 2) {
            stage(t, fr[0], fr[1]);
            stage(t + 1, fr[1], fr[0]);
        }
        if (t < ks_count) stage(t, fr[0], fr[1]);
    } else {
        // Stage t: behind the barrier of stage t - 1 its slabs are free.  The loads of a's stage t + NSTAGE go out over the first three
        // sub-steps, those of b's, whose ring is one slab shorter, behind this stage's own barrier: sixteen loads in a row stood in each
        // other's way.
        half8 fr[2][F];
        auto fetch = [&](uint32_t slot_a, uint32_t slot_b, int sub, int f) {
            return f < MT ? fragment_at(lds + slot_a, sub, true, wm * WTM + 32 * f) : fragment_at(lds + RING_A + slot_b, sub, false, wn * WTN + 32 * (f - MT));
        };
#pragma unroll
        for (int n = 0; n < F; ++n) fr[0][order(n)] = fetch(0, 0, 0, order(n));
        constexpr int R = (F + NM - 1) / NM;                                        // fragment reads per matrix instruction
        constexpr int DA = (A_DMA + 3 * NM - 1) / (3 * NM), SA = 3 * NM * DA / A_DMA;  // a's loads: DA every SA-th of them
        constexpr int DB = (B_DMA + NM - 1) / NM, SB = NM * DB / B_DMA;
        uint32_t now_a = 0, now_b = 0;  // slots of stage t
        auto after = [](uint32_t slot, uint32_t bytes, uint32_t ring) { return slot + bytes == ring ? 0u : slot + bytes; };
        // (the steady state has no branch: with a test around every read and load of the last sub-step, 8192^3 took 3 % longer)
        auto stage = [&](int t, auto more_, auto next_) {
            constexpr bool more = decltype(more_)::value, next = decltype(next_)::value;
            const uint32_t next_a = after(now_a, A_BYTES, RING_A), next_b = after(now_b, B_BYTES, NSTAGE * B_BYTES), last_a = after(next_a, A_BYTES, RING_A);
#pragma unroll
            for (int sub = 0; sub < 4; ++sub) {
#pragma unroll
                for (int k = 0; k < NM; ++k) {
                    const int i = k / NT, j = k % NT;
                    // b goes in as the "row" matrix so that a lane ends up with consecutive output columns
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fr[sub & 1][MT + j], fr[sub & 1][i], acc[i][j], 0, 0, 0);
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const int n = k * R + r;
                        if (n < F && (sub < 3 || next))
                            fr[(sub + 1) & 1][order(n)] = fetch(sub < 3 ? now_a : next_a, sub < 3 ? now_b : next_b, (sub + 1) & 3, order(n));
                    }
                    const int slot = sub * NM + k;
                    if (more && sub < 3 && slot % SA == 0) {
#pragma unroll
                        for (int d = 0; d < DA; ++d)
                            if (slot / SA * DA + d < A_DMA) issue_a(t + NSTAGE, slot / SA * DA + d, last_a);
                    }
                    if (more && sub == 3 && k % SB == 0) {
#pragma unroll
                        for (int d = 0; d < DB; ++d)
                            if (k / SB * DB + d < B_DMA) issue_b(t + NSTAGE, k / SB * DB + d, now_b);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (sub == 2 && next) {
                    wait_vm_lds<more ? A_DMA : 0>();
                    __syncthreads();
                }
            }
            now_a = next_a;
            now_b = next_b;
        };
        static_assert(NSTAGE == 2, "what the waits count");
        int t = 0;
        for (; t + NSTAGE < ks_count; ++t) stage(t, std::true_type{}, std::true_type{});
        for (; t + 1 < ks_count; ++t) stage(t, std::false_type{}, std::true_type{});
        if (t < ks_count) stage(t, std::false_type{}, std::false_type{});
    }
    if constexpr (Epi::kJoin) {
        if (p.splits > 1) {
            constexpr int PART = BM * BN / 4;  // groups of four floats of a tile, as the lanes hold them
            const uint32_t place = (uint32_t)tile.batch * p.div_tiles.d + (uint32_t)__builtin_amdgcn_readfirstlane((int)tile.tile);
            f32x4 *parts = reinterpret_cast<f32x4 *>(p.parts) + (int64_t)place * p.splits * PART + wave * (PART / 4) + lane;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        store_through(parts + (int64_t)tile.split * PART + ((i * NT + j) * 4 + g) * 64,
                                      f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]});
            // The parts go past the XCDs' L2 caches, so that the counter's release has little to write back (with an acquire in every
            // workgroup, not only the last, 128 x 128 x 1152 took 4 us longer).
            wait_vm_lds<0>();
            __syncthreads();
            uint32_t *last = reinterpret_cast<uint32_t *>(lds);
            if (threadIdx.x == 0) {
                const uint32_t before = __hip_atomic_fetch_add(p.arrived + place, 1u, __ATOMIC_RELEASE, __HIP_MEMORY_SCOPE_AGENT);
                *last = before + 1u == (uint32_t)p.splits ? 1u : 0u;
                if (*last) __hip_atomic_store(p.arrived + place, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (*last == 0u) return;
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
            constexpr int N = MT * NT * 4, U = N == 4 ? 8 : 1;  // loads of a slice, slices under way together
            for (int s0 = 0; s0 < p.splits; s0 += U) {
                u32x4 v[U][N];
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int n = 0; n < N; ++n)
                        v[u][n] = s0 + u < p.splits
                                      ? __builtin_amdgcn_global_load_b128((__attribute__((address_space(1))) u32x4 *)(parts + (int64_t)(s0 + u) * PART + n * 64), "agent")
                                      : u32x4{0, 0, 0, 0};
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int n = 0; n < N; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[n / 4 / NT][n / 4 % NT][4 * (n % 4) + e] += u2f(v[u][n][e]);
            }
        }
    }
    epi(at, acc, ahead);
}

// Eight halves from eight FP32 values, to nearest: operands of further products, in which a NaN may have any payload.
__device__ __forceinline__ u32x4 half_operand8(const float v[8]) {
    half8 h;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = (_Float16)v[e];
    return __builtin_bit_cast(u32x4, h);
}

// The bands are private to a wave, whose LDS accesses are carried out in order: what one lane writes and another reads has to stay in it.
__device__ __forceinline__ void half_wave_lds() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// Rows of halves through LDS, so that a store covers whole 128-byte lines (pieces of 32 bytes, as the accumulators lie, kept the L2 busy
// for as long as four times their size: 8192 x 32768 halves in 256x256 tiles 9 us per round of tiles).  A band of 32 rows of a wave's
// part takes WTN * 64 bytes; 16-byte chunk c of row r sits in slot c ^ (r & MASK), and its halves change places in rows 16 .. 31, which
// keeps the lanes of a write apart.  LDS operations of a wave are done in order.
template <class T>
struct HalfLines {
    static constexpr int PER = T::WTN / 8, MASK = PER - 1, ROWS = 64 / PER, PASSES = 32 / ROWS;
    static_assert((PER & MASK) == 0, "the lanes of a row");
    uint8_t *band;
    int lane;
    __device__ __forceinline__ HalfLines(const HalfPlace<T> &at) : band(at.lds + at.wave * T::WTN * 64), lane(at.lane) {}
    // four columns from 32 j + 8 g + 4 (lane / 32) on of row lane % 32
    __device__ __forceinline__ void put(int j, int g, u32x2 v) {
        const int r = lane & 31, h = lane >> 5;
        *reinterpret_cast<u32x2 *>(band + r * T::WTN * 2 + (((4 * j + g) ^ (r & MASK)) << 4) + 8 * (h ^ (r >> 4))) = v;
    }
    // f(row, first of eight columns, halves) for the band's rows
    template <class F>
    __device__ __forceinline__ void each(const F &f) {
        const int lr = lane / PER, c = lane % PER;
        half_wave_lds();
#pragma unroll
        for (int k = 0; k < PASSES; ++k) {
            const int r = ROWS * k + lr;
            const u32x4 v = *reinterpret_cast<const u32x4 *>(band + r * T::WTN * 2 + ((c ^ (r & MASK)) << 4));
            f(r, 8 * c, r < 16 ? v : u32x4{v.z, v.w, v.x, v.y});
        }
        half_wave_lds();
    }
};

// f(r, c, v, x) for every eight neighbouring columns c .. c+7 of rows r of the wave's part, x = load(r, c): bands of 32 rows pass through
// LDS (a region of the ring per wave), so that the lanes that share a row lie side by side and store and load whole 128-byte lines, and
// that f's code is there MOST_U times per band and not once per eight accumulators; as many loads are under way together.  before(i, band):
// called when the i-th band lies in LDS, 32 rows of kHalfBandPitch floats.
template <class T>
constexpr int kHalfBandPitch = T::WTN + 4;
template <int MOST_U = 4, class T, class Load, class F, class Before>
__device__ __forceinline__ void half_bands(const HalfPlace<T> &at, f32x16 (&acc)[T::MT][T::NT], const Load &load, const F &f, const Before &before) {
    constexpr int PITCH = kHalfBandPitch<T>, PER = T::WTN / 8, ROWS = 64 / PER;  // lanes of a row, rows of a pass (192: 5 rows, 60 lanes)
    constexpr int PASSES = (32 + ROWS - 1) / ROWS, U = PASSES < MOST_U ? PASSES : MOST_U;
    static_assert(4 * 32 * PITCH * 4 <= T::NSTAGE * (T::BM + T::BN) * 128, "the bands fit the ring");
    float *band = reinterpret_cast<float *>(at.lds) + at.wave * 32 * PITCH;
    const int lr = at.lane / PER, lc = 8 * (at.lane % PER);
    const bool lane_used = 64 % PER == 0 || lr < ROWS;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < T::MT; ++i) {
#pragma unroll
        for (int j = 0; j < T::NT; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 v = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                *reinterpret_cast<f32x4 *>(band + (at.lane & 31) * PITCH + 32 * j + 8 * g + 4 * (at.lane >> 5)) = v;
            }
        half_wave_lds();
        const int r0 = at.row0 + 32 * i, c = at.col0 + lc;
#pragma unroll 1
        for (int q = 0; q < PASSES; q += U) {
            decltype(load(0, 0)) x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int k = lr + (q + u) * ROWS;
                if (lane_used && k < 32) x[u] = load(r0 + k, c);
            }
            if (q == 0) before(i, band);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int k = lr + (q + u) * ROWS;
                if (!lane_used || k >= 32) continue;
                const f32x4 lo = *reinterpret_cast<const f32x4 *>(band + k * PITCH + lc), hi = *reinterpret_cast<const f32x4 *>(band + k * PITCH + lc + 4);
                const float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                f(r0 + k, c, v, x[u]);
            }
        }
        half_wave_lds();
    }
}
struct HalfNothing {};

// Results: with the canonical NaN.
__device__ __forceinline__ u32x4 half_round8(const float v[8]) {
    u32x4 w;
#pragma unroll
    for (int q = 0; q < 4; ++q) w[q] = f16_from_f32<false>(v[2 * q], 0u) | f16_from_f32<false>(v[2 * q + 1], 0u) << 16;
    return w;
}

struct HalfNoneAhead {
    static constexpr bool kJoin = false, k192 = true;  // k192: plans may hold 192x192 tiles
    template <class P>
    __device__ __forceinline__ HalfNothing ahead(const P &) const { return {}; }
};

// The FP32 tile itself, scaled by nothing, stored or added to what is there: slab `split` of [rows, ld] floats (ld a multiple of
// eight and at least the columns, so that whole groups of eight may be stored).
struct HalfEpiSum : HalfNoneAhead {
    float *out;
    int64_t ld, slab;  // in floats
    int rows, cols, add;
    template <class T>
    __device__ __forceinline__ void operator()(const HalfPlace<T> &at, f32x16 (&acc)[T::MT][T::NT], HalfNothing) const {
        float *base = out + at.split * slab;
        struct Eight {
            f32x4 lo, hi;
        };
        half_bands(at, acc, [&](int r, int c) {
            Eight x{};
            if (add && r < rows && c < cols) {
                x.lo = *reinterpret_cast<const f32x4 *>(base + r * ld + c);
                x.hi = *reinterpret_cast<const f32x4 *>(base + r * ld + c + 4);
            }
            return x;
        }, [&](int r, int c, const float (&v)[8], const Eight &x) {
            if (r >= rows || c >= cols) return;
            f32x4 *to = reinterpret_cast<f32x4 *>(base + r * ld + c);
            to[0] = x.lo + f32x4{v[0], v[1], v[2], v[3]};
            to[1] = x.hi + f32x4{v[4], v[5], v[6], v[7]};
        }, [](int, float *) {});
    }
};

// ---------------------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------------------
// Which tiles a product takes and into how many slices its contraction is cut.
struct HalfPlan {
    int tile, splits;
};

// Estimated time, us, of `tiles` tiles over `stages` stages.  Measured (4096 x 4096 x 4096 and parts of it), us per stage: 64x64 tiles, up to
// 256 of them 0.26 (kByIndex 0.19), 512 (two per CU) 0.41; 128x128, 256 0.69, 512 0.93 (1.08 over long contractions, as the clock sinks:
// 6007 x 1000 over 37003 536 us; in 256x256 tiles, estimated slower with 0.93, 418); 192x192, 64 0.81, 256 1.06; 256x256, 128 1.36,
// 256 1.73; more tiles take rounds.  On top come start and end of a workgroup.
static inline double half_cost(int tile, int64_t tiles, double stages) {
    const int64_t slots = tile > 128 ? 256 : 512, full = tiles / slots, rest = tiles % slots;
    const double whole = tile == 256 ? 1.73 : tile == 192 ? 1.06 : tile == 128 ? 1.08 : 0.41, half = tile == 256 ? 1.36 : tile == 192 ? 0.85 : tile == 128 ? 0.69 : 0.25;
    const double base = tile == 256 ? 10.0 : tile == 192 ? 8.0 : tile == 128 ? 5.0 : 3.5;
    const double rounds = (double)(full + (rest != 0)), over = (double)(rest - slots / 2) / (double)(slots / 2);
    const double part = rest == 0 ? 0.0 : over <= 0.0 ? half : half + over * (whole - half);
    const double t = base * (rounds < 1 ? 1 : 0.5 + 0.5 * rounds) + stages * ((double)full * whole + part), few = 4.4 + 0.19 * stages;
    return tile == 64 && tiles <= 256 && few < t ? few : t;
}
// Few 64x64 tiles over a long contraction: kByIndex (the waves' sums cost 1 us, a stage 0.08 us less).
static inline bool half_by_index(int64_t tiles, double stages) { return tiles <= 256 && stages >= 14; }

// most_splits > 1: the slices' FP32 sums are written and added up, by a pass of its own or (joined) by the last workgroup of every tile.
static inline HalfPlan half_plan(int64_t batch, int64_t rows, int64_t cols, int64_t kc, bool symmetric, int most_splits, bool joined = false) {
    HalfPlan best{64, 1};
    double least = 1e300;
    for (const int tile : {256, 192, 128, 64}) {
        const int64_t tm = (rows + tile - 1) / tile, tn = (cols + tile - 1) / tile;
        const int64_t tiles = batch * (symmetric ? tm * (tm + 1) / 2 : tm * tn), steps = (kc + 63) / 64;
        if (tiles > (int64_t)1 << 23) continue;
        for (int s = 1; s <= most_splits && s <= steps; s = s < 8 ? s + 1 : s + s / 4) {
            // slices of one more pass: 4 bytes out and in again per element and slice, at 4 TB/s; joined: a tile's out and in of one CU, and
            // every workgroup's release of its L2 (measured on Gram products: 128 x 128 x 1152 in 6 slices 7.4 us, unsplit 9.3;
            // 1024 x 1024 x 4096 in 3 slices of 136 tiles 20.4, unsplit 16.4)
            const double more = s == 1 ? 0.0 : joined ? 2.0 + 1.6e-5 * (double)(tile * tile) * s + 1.0e-6 * (double)(tiles * tile * tile) * s + 0.014 * (double)(tiles * s)
                                                      : 2.0e-6 * (double)(batch * rows * cols) * s;
            const double t = half_cost(tile, tiles * s, (double)((steps + s - 1) / s)) + more;
            if (t < least) {
                least = t;
                best = {tile, s};
            }
        }
    }
    return best;
}

// The geometry of a call.  Sizes have been checked: rows, cols, kc >= 1 and what HalfGemm says.
static inline HalfGemm half_gemm_args(const HalfMatrix &a, const HalfMatrix &b, int64_t rows, int64_t cols, int64_t kc, int tile, int splits,
                                      bool symmetric, int64_t batch) {
    HalfGemm p{};
    p.a = (const uint8_t *)a.p;
    p.b = (const uint8_t *)b.p;
    p.lda = 2 * a.ld;
    p.ldb = 2 * b.ld;
    p.a_panel = 2 * a.panel;
    p.b_panel = 2 * b.panel;
    p.a_batch = 2 * a.batch;
    p.b_batch = 2 * b.batch;
    p.rows = (int)rows;
    p.cols = (int)cols;
    p.ksteps = (int)((kc + 63) / 64);
    p.tail = (int)(kc % 64);
    p.splits = splits;
    p.ks_per = p.ksteps / splits;
    p.ks_extra = p.ksteps % splits;
    p.tiles_m = (int)((rows + tile - 1) / tile);
    p.tiles_n = (int)((cols + tile - 1) / tile);
    p.symmetric = symmetric;
    const int tiles = symmetric ? p.tiles_m * (p.tiles_m + 1) / 2 : p.tiles_m * p.tiles_n;
    p.total = (uint32_t)((int64_t)tiles * splits * batch);
    p.div_tiles = make_fastdiv((uint32_t)tiles);
    p.div_splits = make_fastdiv((uint32_t)splits);
    p.div_band = make_fastdiv((uint32_t)(8 * p.tiles_n));
    p.div_last = make_fastdiv((uint32_t)(p.tiles_m % 8 ? p.tiles_m % 8 : 8));
    return p;
}

template <class T, bool ATN, bool BTN, class Epi>
static inline bool half_gemm_launch(const HalfGemm &p, const Epi &epi, hipStream_t stream) {
    hipLaunchKernelGGL((half_gemm_kernel<T, ATN, BTN, Epi>), dim3(p.total), dim3(256), 0, stream, p, epi);
    return hipGetLastError() == hipSuccess;
}

// The tiles of a plan.
template <bool ATN, bool BTN, class Epi>
static inline bool half_gemm_launch_plan(int tile, const HalfGemm &p, const Epi &epi, hipStream_t stream) {
    if (tile == 256) return half_gemm_launch<Half256, ATN, BTN>(p, epi, stream);
    if constexpr (Epi::k192) {
        if (tile == 192) return half_gemm_launch<Half192, ATN, BTN>(p, epi, stream);
    }
    if (tile == 128) return half_gemm_launch<Half128, ATN, BTN>(p, epi, stream);
    if (half_by_index(p.total, (double)p.ks_per)) return half_gemm_launch<Half64Few, ATN, BTN>(p, epi, stream);
    return half_gemm_launch<Half64, ATN, BTN>(p, epi, stream);
}

}  // namespace mp8
