// tppo_orthogonalize: Newton-Schulz products that drive the singular values of an update to one another.
//     X = G / (|G|_F + eps), wide;   steps times:  A = X X^T,  B = b A + c A A,  X = a X + B X
// Three matrix products a step on the matrix cores, 2 m (m n + m m + m n) flop, of which the first two have symmetric results: only the
// tiles on and below the diagonal are computed, and written twice.
// Bound by the matrix cores: 5120 x 5120, 5 steps: 2580 to 2630 us, 1.03 PFLOP/s of the flops that are needed; 1.45 within a round of tiles, as a
// large library product reaches, of which X X^T and A A fill 82 % of the CUs and B X two rounds by 78 %.
//
// Precision.  A rounding of X is a matrix with singular values in every direction, and the iteration multiplies small ones by up to a
// each time, a^steps = 485 in all: bf16 operands turn a gradient of rank one into noise (error 1.2 of 1), fp16 ones still 0.15.  So
//   X     is a pair of fp16, hi + lo / 2048, 22 bits, and a X is taken from both; the product B X takes hi alone: what that loses lies in
//         the range of B, where the large singular values are, and is not amplified;
//   A, B  have their diagonals, which tend to 1 and a - 1 .. in fp32 vectors, and only what is off the diagonal in fp16.
// What is off the diagonal is small against it in large matrices only, and errors grow as small singular values do; where m < kSplitBelow, or
// |a|^steps > m, or where a + b l + c l l cancels (ns_one_pass), A and B are pairs as well, and a product is hi hi + (hi lo + lo hi) / 2048,
// three passes over its contraction.  Against 64 bits, before the rounding to bf16 (1.7e-3), emulated, 5 / 6 / 7 / 8 / 10 steps:
//   one pass      m = 512, rank one  1.3e-3 / 2.6e-3 / 1.4e-2 / 3.2e-2 / 0.37,  singular values down to 10^-6  7e-4 / 1.4e-3 / 3.3e-3 / 8e-3 / 5e-2;
//                 m = 2048           3e-4 / 5e-4 / 2.5e-3 / 6e-3 / 7e-2,                                       5e-4 / 9e-4 / 1.9e-3 / 5e-3 / 3e-2;
//   three passes  any m              1e-4 / 3e-4 / 1.6e-3 / 4e-3 / 4e-2,                                       4e-6 / 1e-5 / 3e-5 / 7e-5 / 4e-4:
// what products in fp32 give, 2e-7 |a|^steps.  (One pass, 5 steps:  m = 256 2.3e-3;  64 9e-3.)
// All scales are powers of two: X is held times S = 2^round(log2(n) / 2), so that entries are around one from the first step to the last,
// A and B off the diagonal times 64.  Where |G|_F is so far below eps that X stays under 1/4 to the end, S is larger by as much.
#include <cmath>

#include "ortho.h"

namespace tppo {

constexpr int kSplitBelow = 512;

enum NsMode { kGram, kPoly, kUpdate, kLast };        // A = X X^T;  B = b A + c A A;  X = a X + B X;  the same into the caller's array

struct NsArgs {
    // out tile [T rows][V columns]:  sum_k t_op[t, k] * v_op[v, k], or v_op[k, v] where that operand lies with K as its row
    const half_t *t_op, *v_op;
    int64_t ld_t, ld_v, each_t, each_v;              // in elements; from one matrix of the stack to the next
    int64_t lo_t, lo_v;                              // bytes from an operand to its low halves
    int n_t, n_v, k;                                 // rows of either side; contraction, a multiple of 64
    int tiles_t, tiles_v, tiles;                     // tiles: of one matrix
    // kGram: off, diag out;  kPoly: off, diag in, off_out, diag_out out;  kUpdate, kLast: diag (of B), hi, lo in, hi_out, lo_out / out out
    half_t *off, *off_out, *off_lo, *off_out_lo, *hi, *lo, *hi_out, *lo_out;
    float *diag, *diag_out;
    int64_t each_off, each_diag, each_x;
    int ld_off, ld_x;
    const float2* scales;                            // by matrix: 1 / S^2, scale / S
    float a, b, c;
    uint16_t* out;                                   // kLast: bf16, times out_scale
    int64_t ld_out, each_out;
    int m, n, transposed;
};

template <int TV, int TT, int WV, int WT, bool KMAJOR, bool SPLIT>
struct NsCfg {
    static constexpr int kTileV = TV, kTileT = TT, kWavesV = WV, kWavesT = WT, kWaves = WV * WT, kThreads = kWaves * 64;
    static constexpr int kBK = 64, kRowBytes = 128, kRows = TV + TT, kStageBytes = kRows * kRowBytes, kLdsBytes = 2 * kStageBytes;
    static constexpr int kWaveV = TV / WV, kWaveT = TT / WT, kVB = kWaveV / 16, kTB = kWaveT / 16;
    // transfers of a stage: the first kDmaMore wavefronts have kDmaPerWave of them, the others one less
    static constexpr int kDma = kStageBytes / 1024, kDmaPerWave = (kDma + kWaves - 1) / kWaves, kDmaMore = kDma - (kDmaPerWave - 1) * kWaves;
    static constexpr int kDmaV = TV * kRowBytes / 1024;
    static constexpr int kSteps = 2 * kVB;           // of kTB MFMAs each
    static constexpr int kSpreadSteps = kSteps / 2;  // a stage's transfers go out over so many
    static constexpr bool kKMajor = KMAJOR, kSplit = SPLIT;
    static constexpr int kKRowBytes = TV * 2;        // K-major: a stage is 64 rows of TV columns
    static_assert(kDma * 1024 == kStageBytes && kWaveV % 16 == 0 && kWaveT % 16 == 0, "whole transfers and blocks");
};

// Tile `id` of a matrix: blocks of 8 T tiles, column by column, so that an XCD's workgroups share operands in its L2.  Symmetric: of those
// that hold an entry on or above the diagonal, v >= t.
template <class C, bool SYMMETRIC>
__host__ __device__ __forceinline__ int ns_first_v(int t) { return SYMMETRIC ? t * C::kTileT / C::kTileV : 0; }
template <class C, bool SYMMETRIC>
__device__ __forceinline__ void ns_tile_at(int id, int tiles_t, int tiles_v, int& t, int& v) {
    constexpr int kBlock = 8;
    if constexpr (!SYMMETRIC) {
        const int block = id / (kBlock * tiles_v), in = id - block * kBlock * tiles_v, height = min(kBlock, tiles_t - block * kBlock);
        v = in / height;
        t = block * kBlock + in - v * height;
    } else {
        for (int first = 0;; first += kBlock) {
            const int height = min(kBlock, tiles_t - first);
            int all = 0;
            for (int i = 0; i < height; ++i) all += tiles_v - ns_first_v<C, true>(first + i);
            if (id >= all) {
                id -= all;
                continue;
            }
            int there = 0;                           // T tiles of the block that have column v
            for (v = ns_first_v<C, true>(first);; ++v) {
                while (there < height && ns_first_v<C, true>(first + there) <= v) ++there;
                if (there == height || id < there) break;
                id -= there;
            }
            v += id / there;
            t = first + id % there;
            return;
        }
    }
}

template <class C, NsMode MODE>
__global__ __launch_bounds__(C::kThreads, C::kLdsBytes <= 80 * 1024 ? C::kWaves / 2 : C::kWaves / 4) void ns_product_kernel(NsArgs p) {
    constexpr bool kSymmetric = MODE == kGram || MODE == kPoly;
    constexpr int kVB = C::kVB, kTB = C::kTB, kDmaPerWave = C::kDmaPerWave;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int id = ns_by_xcd(blockIdx.x, gridDim.x);
    const int mat = id / p.tiles;
    int tile_t, tile_v;
    ns_tile_at<C, kSymmetric>(id - mat * p.tiles, p.tiles_t, p.tiles_v, tile_t, tile_v);
    const int t0 = tile_t * C::kTileT, v0 = tile_v * C::kTileV;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wv = wave / C::kWavesT, wt = wave % C::kWavesT, col = lane & 15, grp = lane >> 4;
    const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem;

    // transfers: this wavefront's of the stage's, the V side's first
    const bool more = wave < C::kDmaMore;
    const int first_dma = wave * (kDmaPerWave - 1) + min(wave, C::kDmaMore);
    const char* src[kDmaPerWave];
    const char *t_base = reinterpret_cast<const char*>(p.t_op + mat * p.each_t), *v_base = reinterpret_cast<const char*>(p.v_op + mat * p.each_v);
#pragma unroll
    for (int q = 0; q < kDmaPerWave; ++q) {
        const int d = first_dma + q;             // (one too many where there are fewer: an address that is not used)
        if (d < C::kDmaV && C::kKMajor) {
            constexpr int kPerRow = C::kKRowBytes / 16;
            const int at = d * 64 + lane, k = at / kPerRow, c = (at % kPerRow) ^ ns_swz_k<C::kTileV>(k);
            src[q] = v_base + ((int64_t)k * p.ld_v + min(v0 + c * 8, p.n_v - 8)) * 2;
        } else {
            const int r = (d < C::kDmaV ? d : d - C::kDmaV) * 8 + (lane >> 3), staged = d * 8 + (lane >> 3);
            const int chunk = ((lane & 7) ^ ns_swz(staged)) * 16;
            if (d < C::kDmaV) src[q] = v_base + (int64_t)min(v0 + r, p.n_v - 1) * p.ld_v * 2 + chunk;
            else src[q] = t_base + (int64_t)min(t0 + r, p.n_t - 1) * p.ld_t * 2 + chunk;
        }
    }
    // (three passes: T's low halves, V's, neither's)
    int64_t pos = C::kSplit ? p.lo_t : 0, pos_v = 0;
    const int stages_once = p.k / C::kBK, stages = C::kSplit ? 3 * stages_once : stages_once;
    int issued = 0;
    const int64_t step_v = C::kKMajor ? (int64_t)C::kBK * p.ld_v * 2 : C::kRowBytes;
    const unsigned dst0 = lds_base + first_dma * 1024;
    unsigned dst = dst0;
    auto issue_one = [&](int q) {
        if (C::kDmaMore != C::kWaves && q + 1 == kDmaPerWave && !more) return;
        const bool on_v = first_dma + q < C::kDmaV;
        const char* from = src[q] + (on_v ? pos_v : pos);
        asm volatile("s_add_u32 m0, %0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                     :
                     : "s"(dst), "v"(from), "i"(q * 1024)
                     : "memory", "m0", "scc");
    };
    auto issue_advance = [&]() {
        pos += C::kRowBytes;
        pos_v += step_v;
        dst = 2 * dst0 + C::kStageBytes - dst;
        if constexpr (C::kSplit) {
            if (++issued == stages_once) {
                pos = 0;
                pos_v = p.lo_v;
            } else if (issued == 2 * stages_once) {
                pos = pos_v = 0;
            }
        }
    };
    f32x4 acc[kVB][kTB] = {};
    half8 fa[2], fb[2][kTB];
    auto load_frags = [&](int stage, int step) {
        const int k32 = step / kVB, vb = step % kVB, c = k32 * 4 + grp;
        const unsigned char* st = smem + stage * C::kStageBytes;
        if constexpr (C::kKMajor) {
            fa[step & 1] = ns_k_major_frag<C::kTileV>(lds_base + stage * C::kStageBytes, wv * kVB + vb, k32, lane);
        } else {
            const int r = wv * C::kWaveV + vb * 16 + col;
            fa[step & 1] = *reinterpret_cast<const half8*>(st + r * C::kRowBytes + ((c ^ ns_swz(r)) << 4));
        }
        if (vb == 0)
#pragma unroll
            for (int tb = 0; tb < kTB; ++tb) {
                const int r = C::kTileV + wt * C::kWaveT + tb * 16 + col;
                fb[k32][tb] = *reinterpret_cast<const half8*>(st + r * C::kRowBytes + ((c ^ ns_swz(r)) << 4));
            }
    };
    // an MFMA step; this wavefront's transfers of the stage that was freed go out between those of the first kSpreadSteps
    auto mfma_step = [&](int step, int part, bool on) {
        const int k32 = step / kVB, vb = step % kVB;
        constexpr int kSpread = C::kSpreadSteps * kTB;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int tb = 0; tb < kTB; ++tb) {
            acc[vb][tb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fa[step & 1], fb[k32][tb], acc[vb][tb], 0, 0, 0);
            if (part < C::kSpreadSteps) {
                if (on) {
#pragma unroll
                    for (int j = 0; j < kDmaPerWave; ++j)
                        if (j * kSpread / kDmaPerWave == part * kTB + tb) issue_one(j);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
#pragma unroll
    for (int q = 0; q < kDmaPerWave; ++q) issue_one(q);
    issue_advance();
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    __syncthreads();
    if (stages > 1) {
#pragma unroll
        for (int q = 0; q < kDmaPerWave; ++q) issue_one(q);
        issue_advance();
    }
    load_frags(0, 0);
    int stage = 0;
    bool refill = false;
    for (int it = 0; it < stages; ++it) {
#pragma unroll
        for (int ks = 0; ks + 1 < C::kSteps; ++ks) {
            load_frags(stage, ks + 1);
            mfma_step(ks, ks + 1, refill);
            if (ks + 2 == C::kSpreadSteps && refill) issue_advance();
        }
        refill = false;
        __builtin_amdgcn_s_waitcnt(kLgkm0);
        if (it + 1 < stages) {
            __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
            __syncthreads();
            refill = it + 2 < stages;
            load_frags(stage ^ 1, 0);
        }
        mfma_step(C::kSteps - 1, 0, refill);
        stage ^= 1;
        if constexpr (C::kSplit) {
            if (it + 1 == 2 * stages_once) {
#pragma unroll
                for (int vb = 0; vb < kVB; ++vb)
#pragma unroll
                    for (int tb = 0; tb < kTB; ++tb) acc[vb][tb] *= 1.f / kLoScale;
            }
        }
    }

    // Epilogue, half of the tile's rows at a time: the sums go through LDS, so that all reads and writes of memory are whole pieces of 16
    // bytes of rows, eight entries each, and what a half reads is asked for before its sums are there.  Mirrored entries are taken
    // from LDS by columns.  (From the registers, four entries of 16 rows an instruction and two bytes at a time across the diagonal, a
    // round of 256 tiles of 256 x 256 took 37 us for B X and 10 for b A + c A A.)
    // 16-byte piece c of a half's row r lies at c ^ key(r): consecutive rows, and rows 8 apart, at different places of the bank window
    auto key = [](int r) { return (r ^ (r >> 3)) & 15; };
    constexpr int kHalf = C::kTileT / 2, kPieces = C::kTileV / 8, kRowsAtOnce = C::kThreads / kPieces, kTurns = kHalf / kRowsAtOnce;
    static_assert(kHalf * C::kTileV * 4 <= C::kLdsBytes && kTurns * kRowsAtOnce == kHalf && C::kWavesT % 2 == 0, "half a tile");
    const float2 scales = p.scales[mat];
    const int piece = tid % kPieces, row = tid / kPieces, v = v0 + piece * 8;
    const bool v_there = v < p.n_v;
    float dv[8];
    if constexpr (MODE == kPoly)
#pragma unroll
        for (int e = 0; e < 8; ++e) dv[e] = v_there ? p.diag[mat * p.each_diag + v + e] : 0.f;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int th = t0 + half * kHalf;
        half8 in_hi[kTurns], in_lo[kTurns];
        float in_d[kTurns];
        if constexpr (MODE != kGram) {
#pragma unroll
            for (int k = 0; k < kTurns; ++k) {
                const int t = min(th + k * kRowsAtOnce + row, p.n_t - 1);
                const half_t *from = MODE == kPoly ? p.off : p.hi, *from_lo = MODE == kPoly ? p.off_lo : p.lo;
                const int64_t at = MODE == kPoly ? mat * p.each_off + (int64_t)t * p.ld_off + v : mat * p.each_x + (int64_t)t * p.ld_x + v;
                in_d[k] = p.diag[mat * p.each_diag + t];
                if (v_there) {
                    in_hi[k] = *reinterpret_cast<const half8*>(from + at);
                    if constexpr (MODE != kPoly || C::kSplit) in_lo[k] = *reinterpret_cast<const half8*>(from_lo + at);
                }
            }
        }
        __syncthreads();                             // the stages, or the first half, are read
        if (wt / (C::kWavesT / 2) == half)
#pragma unroll
            for (int tb = 0; tb < kTB; ++tb) {
                const int r = (wt % (C::kWavesT / 2)) * C::kWaveT + tb * 16 + col;
#pragma unroll
                for (int vb = 0; vb < kVB; ++vb)
                    *reinterpret_cast<f32x4*>(smem + r * (C::kTileV * 4) + (((wv * (C::kWaveV / 4) + vb * 4 + grp) ^ key(r)) << 4)) = acc[vb][tb];
            }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            const int r = k * kRowsAtOnce + row, t = th + r;
            f32x4 *low = reinterpret_cast<f32x4*>(smem + r * (C::kTileV * 4) + (((piece * 2) ^ key(r)) << 4));
            f32x4 *high = reinterpret_cast<f32x4*>(smem + r * (C::kTileV * 4) + (((piece * 2 + 1) ^ key(r)) << 4));
            const f32x4 sum[2] = {*low, *high};
            if (t >= p.n_t || !v_there) continue;
            float x[8];
            if constexpr (MODE == kGram) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = sum[e >> 2][e & 3] * scales.x;
                    if (v + e == t) p.diag[mat * p.each_diag + t] = x[e];
                    x[e] = v + e == t ? 0.f : x[e] * kOffScale;
                }
            } else if constexpr (MODE == kPoly) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float w = C::kSplit ? fmaf((float)in_lo[k][e], 1.f / kLoScale, (float)in_hi[k][e]) : (float)in_hi[k][e], s = sum[e >> 2][e & 3];
                    if (v + e == t) p.diag_out[mat * p.each_diag + t] = fmaf(p.c, fmaf(s, 1.f / (kOffScale * kOffScale), in_d[k] * in_d[k]), p.b * in_d[k]);
                    x[e] = v + e == t ? 0.f : fmaf(p.c, fmaf(in_d[k] + dv[e], w, s * (1.f / kOffScale)), p.b * w);
                }
            } else {
                const float lead = p.a + in_d[k];
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[e] = fmaf(lead, fmaf((float)in_lo[k][e], 1.f / kLoScale, (float)in_hi[k][e]), sum[e >> 2][e & 3] * (1.f / kOffScale));
            }
            if constexpr (kSymmetric) {
                half_t *to = (MODE == kGram ? p.off : p.off_out) + mat * p.each_off + (int64_t)t * p.ld_off + v, *to_lo = nullptr;
                if constexpr (C::kSplit) to_lo = (MODE == kGram ? p.off_lo : p.off_out_lo) + mat * p.each_off + (int64_t)t * p.ld_off + v;
                half8 h, l;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    h[e] = (half_t)x[e];
                    l[e] = (half_t)((x[e] - (float)h[e]) * kLoScale);
                }
                if (v >= t) {
                    *reinterpret_cast<half8*>(to) = h;
                    if constexpr (C::kSplit) *reinterpret_cast<half8*>(to_lo) = l;
                } else if (v + 7 >= t) {
#pragma unroll
                    for (int e = 1; e < 8; ++e)
                        if (v + e >= t) {
                            to[e] = h[e];
                            if constexpr (C::kSplit) to_lo[e] = l[e];
                        }
                }
                *low = f32x4{x[0], x[1], x[2], x[3]};
                *high = f32x4{x[4], x[5], x[6], x[7]};
            } else if constexpr (MODE == kUpdate) {
                half8 h, l;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    h[e] = (half_t)x[e];
                    l[e] = (half_t)((x[e] - (float)h[e]) * kLoScale);
                }
                const int64_t at = mat * p.each_x + (int64_t)t * p.ld_x + v;
                *reinterpret_cast<half8*>(p.hi_out + at) = h;
                *reinterpret_cast<half8*>(p.lo_out + at) = l;
            } else if (!p.transposed) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= scales.y;
                if (t < p.m && v < p.n) put_whole_or_part(p.out + mat * p.each_out + (int64_t)t * p.ld_out + v, p.n - v, x);
            } else {
                *low = f32x4{x[0], x[1], x[2], x[3]} * scales.y;
                *high = f32x4{x[4], x[5], x[6], x[7]} * scales.y;
            }
        }
        if (kSymmetric || (MODE == kLast && p.transposed)) {
            __syncthreads();
            constexpr int kAcross = kHalf / 8, kItems = kAcross * C::kTileV / C::kThreads;     // pieces of eight rows of a column
#pragma unroll 2
            for (int k = 0; k < kItems; ++k) {
                const int item = k * C::kThreads + tid, c = item / kAcross, r0 = (item - c * kAcross) * 8, vc = v0 + c, t = th + r0;
                if (vc >= p.n_v || t >= p.n_t || (kSymmetric && t > vc)) continue;
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = *reinterpret_cast<const float*>(smem + (r0 + e) * (C::kTileV * 4) + (((c >> 2) ^ key(r0 + e)) << 4) + (c & 3) * 4);
                if constexpr (kSymmetric) {
                    half_t *to = (MODE == kGram ? p.off : p.off_out) + mat * p.each_off + (int64_t)vc * p.ld_off + t, *to_lo = nullptr;
                    if constexpr (C::kSplit) to_lo = (MODE == kGram ? p.off_lo : p.off_out_lo) + mat * p.each_off + (int64_t)vc * p.ld_off + t;
                    half8 h, l;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        h[e] = (half_t)x[e];
                        l[e] = (half_t)((x[e] - (float)h[e]) * kLoScale);
                    }
                    if (t + 7 <= vc) {
                        *reinterpret_cast<half8*>(to) = h;
                        if constexpr (C::kSplit) *reinterpret_cast<half8*>(to_lo) = l;
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (t + e <= vc) {
                                to[e] = h[e];
                                if constexpr (C::kSplit) to_lo[e] = l[e];
                            }
                    }
                } else if (vc < p.n && t < p.m) {
                    put_whole_or_part(p.out + mat * p.each_out + (int64_t)vc * p.ld_out + t, p.m - t, x);
                }
            }
        }
    }
}

// ---- |G|_F and the first X
constexpr int kNsThreads = 256, kNsParts = 1024;     // partial sums of squares a matrix
__device__ __forceinline__ double ns_workgroup_sum(double x, double* place) {
    x = wave_prefix(x);
    if ((threadIdx.x & 63) == 63) place[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0;
#pragma unroll
    for (int w = 0; w < kNsThreads / kWave; ++w) x += place[w];
    return x;
}
// Bound by memory: 16 bytes a thread, wherever rows begin: 5120 x 5120, fp32: 26 us, 4.0 TB/s (two workgroups to a CU instead of four: 34).  (In
// 64 bits: squares of large fp32 values overflow.)
template <class T, bool RAGGED>
__global__ __launch_bounds__(kNsThreads) void ns_norm_kernel(const T* __restrict__ g, int rows, int cols, int64_t ld, int64_t each,
                                                             double* __restrict__ parts) {
    constexpr int kN = Piece<T>::kN;
    __shared__ double place[kNsThreads / kWave];
    const T* from = g + blockIdx.y * each;
    const unsigned per_row = (cols + kN - 1) / kN, all = per_row * rows;                       // (2^30 at most)
    double sum = 0.0;
#pragma unroll 4
    for (unsigned i = blockIdx.x * kNsThreads + threadIdx.x; i < all; i += gridDim.x * kNsThreads) {
        const unsigned r = i / per_row, c = i - r * per_row;
        const int start = piece_start<kN, RAGGED>(c, cols);
        const Piece<T> p = piece_at<T, RAGGED>(from + (int64_t)r * ld, start, cols);
#pragma unroll
        for (int e = 0; e < kN; ++e) {
            const double x = own<kN, RAGGED>(c, start, e, cols) ? (double)p.get(e) : 0.0;
            sum = fma(x, x, sum);
        }
    }
    sum = ns_workgroup_sum(sum, place);
    if (threadIdx.x == 0) parts[(int64_t)blockIdx.y * kNsParts + blockIdx.x] = sum;
}

// X [mp, np], zeros beyond m x n, from G or its transpose (through LDS), a 64 x 64 tile a workgroup's turn.  hi == NULL: no products follow, X
// times `scale` goes to the caller's array.
template <class T>
__global__ __launch_bounds__(kNsThreads) void ns_begin_kernel(const T* __restrict__ g, int64_t ld, int64_t each, const double* __restrict__ parts,
                                                              int count_parts, float eps, float scale, float s_scale, double growth,
                                                              half_t* __restrict__ hi, half_t* __restrict__ lo, float2* scales, int mp, int np,
                                                              int m, int n, int transposed, uint16_t* __restrict__ out, int64_t ld_out,
                                                              int64_t each_out) {
    __shared__ double place[kNsThreads / kWave];
    __shared__ float tile[64][65];
    const int mat = blockIdx.y;
    const T* from = g + mat * each;
    const int tiles_n = np / 64, tiles = tiles_n * (mp / 64);
    double by = 0.0;
    for (int id = blockIdx.x; id < tiles; id += gridDim.x) {
        const int i0 = id / tiles_n * 64, j0 = (id - id / tiles_n * tiles_n) * 64;
        // all of a thread's entries are asked for at once, those of the first tile before the norm is added up: rows of G, or (G is [n, m])
        // a column of 16 of its rows, which passes through LDS
        float x[2][8];
        if (transposed) {
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int r = (threadIdx.x >> 6) + k * 4, c = threadIdx.x & 63;
                x[k >> 3][k & 7] = j0 + r < n && i0 + c < m ? to_f32(from[(int64_t)(j0 + r) * ld + i0 + c]) : 0.f;
            }
        } else {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int i = i0 + half * 32 + (threadIdx.x >> 3), j = j0 + (threadIdx.x & 7) * 8;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[half][e] = 0.f;
                if (i < m && j < n) get_piece<T, 8, true>(from + (int64_t)i * ld, j, n, x[half]);
            }
        }
        if (id == (int)blockIdx.x) {
            double sum = 0.0;
            for (int i = threadIdx.x; i < count_parts; i += kNsThreads) sum += parts[(int64_t)mat * kNsParts + i];
            sum = ns_workgroup_sum(sum, place);
            const double norm = sqrt(sum) + (double)eps;
            // growth: what the steps make of small singular values
            const double most = sqrt(sum) / norm * growth;
            const double lift = hi && most > 0.0 && most < 0.25 ? ldexp(1.0, -ilogb(most) - 3) : 1.0;
            const double s_all = hi ? (double)s_scale * lift : (double)scale;
            // (one of zeros with eps = 0 gives NaN, as 0 / 0 does; an infinity in G makes all of it NaN)
            by = norm < 1.0e300 ? s_all / norm : __builtin_nan("");
            if (hi && threadIdx.x == 0 && id == 0) scales[mat] = make_float2((float)(1.0 / (s_all * s_all)), (float)((double)scale / s_all));
        }
        if (transposed) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 16; ++k) tile[threadIdx.x & 63][(threadIdx.x >> 6) + k * 4] = x[k >> 3][k & 7];
            __syncthreads();
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {       // eight columns of a row
            const int r = half * 32 + (threadIdx.x >> 3), c = (threadIdx.x & 7) * 8, i = i0 + r, j = j0 + c;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[half][e] = (float)((double)(transposed ? tile[r][c + e] : x[half][e]) * by);
            if (hi) {
                half8 h, l;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float y = i < m && j + e < n ? x[half][e] : 0.f;                     // (zeros, also where `by` is no number)
                    h[e] = (half_t)y;
                    l[e] = (half_t)((y - (float)h[e]) * kLoScale);
                }
                const int64_t at = ((int64_t)mat * mp + i) * np + j;
                *reinterpret_cast<half8*>(hi + at) = h;
                *reinterpret_cast<half8*>(lo + at) = l;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (i < m && j + e < n) out[mat * each_out + (transposed ? (int64_t)(j + e) * ld_out + i : (int64_t)i * ld_out + j + e)] = ns_bf16(x[half][e]);
            }
        }
    }
}

// (a vocabulary's rows among them; pieces and tiles of one matrix are numbered in 32 bits)
constexpr int64_t kNsMaxSide = 262144, kNsMaxEntries = (int64_t)1 << 32;
static bool ns_sides(int64_t rows, int64_t cols) {
    return rows >= 1 && cols >= 1 && rows <= kNsMaxSide && cols <= kNsMaxSide && rows * cols <= kNsMaxEntries;
}

struct NsLayout {
    int m, n, mp, np;
    size_t parts, scales, shared, diag_a, diag_b, off_a, off_b, off_a_lo, off_b_lo, hi[2], lo[2], total;
};
static NsLayout ns_layout(int64_t count, int64_t rows, int64_t cols) {
    NsLayout L;
    L.m = (int)std::min(rows, cols);
    L.n = (int)std::max(rows, cols);
    L.mp = (L.m + 63) / 64 * 64;
    L.np = (L.n + 63) / 64 * 64;
    size_t o = 0;
    auto take = [&](size_t each) {
        const size_t at = o;
        o += round_up((size_t)count * each, 256);
        return at;
    };
    L.parts = take(kNsParts * sizeof(double));
    L.scales = take(sizeof(float2));
    L.hi[0] = take((size_t)L.mp * L.np * 2);
    L.lo[0] = take((size_t)L.mp * L.np * 2);
    L.shared = o;                                    // what the two ways need from here on
    L.diag_a = take((size_t)L.mp * 4);
    L.diag_b = take((size_t)L.mp * 4);
    L.off_a = take((size_t)L.mp * L.mp * 2);
    L.off_b = take((size_t)L.mp * L.mp * 2);
    L.off_a_lo = take((size_t)L.mp * L.mp * 2);      // (three passes)
    L.off_b_lo = take((size_t)L.mp * L.mp * 2);
    L.hi[1] = take((size_t)L.mp * L.np * 2);
    L.lo[1] = take((size_t)L.mp * L.np * 2);
    if (L.m < kGramBelow) o = std::max(o, L.shared + ns_gram_bytes(count, L.m, L.n));
    L.total = o;
    return L;
}

template <class C, bool SYMMETRIC>
static int ns_tiles(int n_t, int n_v) {
    const int tiles_t = (n_t + C::kTileT - 1) / C::kTileT, tiles_v = (n_v + C::kTileV - 1) / C::kTileV;
    int tiles = 0;
    for (int t = 0; t < tiles_t; ++t) tiles += tiles_v - ns_first_v<C, SYMMETRIC>(t);
    return tiles;
}
template <class C, NsMode MODE>
static int launch_ns(NsArgs& p, int64_t count, hipStream_t s) {
    if (C::kLdsBytes > 64 * 1024 && !allow_lds(reinterpret_cast<const void*>(ns_product_kernel<C, MODE>), C::kLdsBytes)) return TPPO_ERR_LAUNCH;
    p.tiles_t = (p.n_t + C::kTileT - 1) / C::kTileT;
    p.tiles_v = (p.n_v + C::kTileV - 1) / C::kTileV;
    p.tiles = ns_tiles<C, MODE == kGram || MODE == kPoly>(p.n_t, p.n_v);
    hipLaunchKernelGGL((ns_product_kernel<C, MODE>), dim3((unsigned)(p.tiles * count)), dim3(C::kThreads), C::kLdsBytes, s, p);
    return launch_result();
}

// The tiles of a product.  256 V columns by 256 T rows read the least; fewer rows make finer parts of it, whose number comes nearer to whole
// rounds of 256 workgroups; 128 x 128, two workgroups to a CU, are for what is too small for either.
// A stage (64 of the contraction) takes so many us a round: what LDS passes, fragments and transfers together, and the MFMAs, which cover
// each other but in part (5120 x 5120, X X^T, 256 x 256: 123 us; without the transfers 96, without the MFMAs 96).  (Stages of 32, four under
// way: 143; four wavefronts of 128 x 128: 149.)  Measured, us, the products of a step (X X^T, b A + c A A, B X) by rows of a tile, 256 / 192 /
// 160 / 128 x 128; * what the rule takes:
//   5120 x 5120:  *125 / 197 / 179 / 157   *134 / 212 / 190 / 167   *265 / 317 / 287 / 302
//   3584 x 3584:   83 / 71 / 64 / *58         91 / 78 / 70 / *62       *95 / 147 / 131 / 112
//   2048 x 2048:   52 / 45 / 40 / *30         60 / 52 / 46 / *31        72 / 57 / 50 / *34
// (224 rows take no less than 256, 128 rows with 256 columns what two of 128 x 128 take.)
template <bool ACROSS, int T>
using NsLarge = NsCfg<256, T, (T % 64 ? 4 : 2), (T % 64 ? 2 : 4), ACROSS, false>;
constexpr int kNsShapes = 4;
constexpr double kNsStage[kNsShapes - 1] = {1.49, 1.25, 1.12};                                 // 256, 192, 160 rows
constexpr double kNsSmallPair = 0.95, kNsSmallAlone = 0.66;                                    // two that share a CU; one
struct NsShapeCost {
    int shape;
    double stage;                                    // us for 64 of the contraction
};
template <bool SYMMETRIC>
static NsShapeCost ns_shape(int n_t, int n_v, int64_t count) {
    const int64_t tiles[kNsShapes - 1] = {ns_tiles<NsLarge<!SYMMETRIC, 256>, SYMMETRIC>(n_t, n_v) * count,
                                          ns_tiles<NsLarge<!SYMMETRIC, 192>, SYMMETRIC>(n_t, n_v) * count,
                                          ns_tiles<NsLarge<!SYMMETRIC, 160>, SYMMETRIC>(n_t, n_v) * count};
    const int64_t small = ns_tiles<NsCfg<128, 128, 2, 2, !SYMMETRIC, false>, SYMMETRIC>(n_t, n_v) * count;
    const int64_t each = (small + kSweepGroups - 1) / kSweepGroups;                            // on the busiest CU
    double least = (double)(each / 2) * kNsSmallPair + (double)(each % 2) * kNsSmallAlone;
    int best = kNsShapes - 1;
    for (int i = 0; i + 1 < kNsShapes; ++i) {
        const double cost = rounds_of(tiles[i]) * kNsStage[i];
        if (cost < least) {
            least = cost;
            best = i;
        }
    }
    return {best, least};
}

// Which way is the shorter.  Both by their launches: what they cost without their stages, in us, and the stages.  This way has three
// products a step, of X's length and of its width; the other (ortho_gram.hip) three passes over pairs, 64 x 64 tiles, of X's width but for
// the first and the last.  Measured, us, this way / the other, * what the rule takes:  512 x 512: 228 / *132;  1024 x 1024: 318 / *206;  1536:
// *401 / 426;  2047: *500 / 906;  1024 x 4096: 478 / *254;  1536 x 6144: 730 / *563;  2047 x 8192: *995 / 1217;  four of 1024 x 1024: *330 / 498;  four
// of 1024 x 4096: *626 / 666;  1024 x 16384: 1231 / *424.
static double ns_direct_us(int mp, int np, int64_t count, int steps) {
    const double gram = ns_shape<true>(mp, mp, count).stage, update = ns_shape<false>(mp, np, count).stage;
    return steps * (3 * 9.0 + gram * (np + mp) / 64 + update * mp / 64);
}
static double ns_gram_us(int mp, int np, int64_t count, int steps) {
    const int side = mp / 64;
    const double tiles = (double)side * (side + 1) / 2 * (double)count;
    auto launch = [](double groups, double stages) {
        return 5.0 + stages * (groups <= kSweepGroups ? 0.5 : 0.8 * std::ceil(groups / (2 * kSweepGroups)));
    };
    const double poly = launch(tiles, side), both = launch(2 * tiles, side);
    return steps * (2 * poly + both) - poly + 10.0 + 0.8 * tiles * (np / 64) / (2 * kSweepGroups) + launch((double)side * (np / 64) * (double)count, side);
}
// Whether one pass with operands of 11 bits will do: large matrices, whose small singular values are not amplified by more than m (the errors are
// 1.1e-3 |a|^steps / m at most where that is how they grow, and else 0.7e-3), and a polynomial whose terms do not cancel, 1.5e-3 of the result at most at
// 24 (m = 512, 180 sets of coefficients; up to 9e-3 beyond).
static bool ns_one_pass(const NsReach& r, int m, int steps, float a, float b, float c) {
    return m >= kSplitBelow && pow(fabs((double)a), steps) <= m && fabs((double)a) + fabs((double)b) + fabs((double)c) <= 24.0 * r.least;
}
enum NsWay { kNsPairs, kNsOnePass, kNsThreePasses };  // X X^T alone; products of X
static NsWay ns_way(const NsLayout& L, int64_t count, int steps, float a, float b, float c) {
    const NsReach reach = ns_reach(steps, a, b, c);
    const bool one = ns_one_pass(reach, L.m, steps, a, b, c);
    if (L.m < kGramBelow && (!one || ns_gram_us(L.mp, L.np, count, steps) < ns_direct_us(L.mp, L.np, count, steps)) &&
        ns_gram_fits(reach, steps, a, b, c))
        return kNsPairs;
    return one ? kNsOnePass : kNsThreePasses;
}
template <bool SPLIT, NsMode MODE>
static int launch_ns_tiles(NsArgs& p, int64_t count, hipStream_t s) {
    constexpr bool kAcross = MODE == kUpdate || MODE == kLast;
    const int shape = SPLIT ? kNsShapes - 1 : ns_shape<!kAcross>(p.n_t, p.n_v, count).shape;
    if constexpr (!SPLIT) {
        switch (shape) {
            case 0: return launch_ns<NsLarge<kAcross, 256>, MODE>(p, count, s);
            case 1: return launch_ns<NsLarge<kAcross, 192>, MODE>(p, count, s);
            case 2: return launch_ns<NsLarge<kAcross, 160>, MODE>(p, count, s);
        }
    }
    return launch_ns<NsCfg<128, 128, 2, 2, kAcross, SPLIT>, MODE>(p, count, s);
}

template <class T>
static int run_ns(const T* g, int64_t count, int64_t rows, int64_t cols, int64_t ld_g, int64_t stride_g, int steps, float a, float b,
                  float c, float eps, float scale, uint16_t* out, int64_t ld_out, int64_t stride_out, char* ws, hipStream_t s) {
    const NsLayout L = ns_layout(count, rows, cols);
    const bool transposed = rows > cols;
    double* parts = reinterpret_cast<double*>(ws + L.parts);
    float2* scales = reinterpret_cast<float2*>(ws + L.scales);
    // (a workgroup for every 1024 pieces of 16 bytes, four to a CU over the whole stack, eight a matrix whatever its size)
    constexpr int kN = Piece<T>::kN;
    const int64_t pieces = rows * ((cols + kN - 1) / kN);
    const int n_parts = (int)std::max<int64_t>(1, std::min<int64_t>({(pieces + 1023) / 1024, kNsParts, std::max<int64_t>(1024 / count, 8)}));
    hipLaunchKernelGGL((cols % kN ? ns_norm_kernel<T, true> : ns_norm_kernel<T, false>), dim3(n_parts, (unsigned)count), dim3(kNsThreads), 0, s, g,
                       (int)rows, (int)cols, ld_g, stride_g, parts);
    int log2n = 0;
    while ((2LL << log2n) <= L.n) ++log2n;
    const float s_scale = (float)(1 << (log2n + 1) / 2);
    half_t *hi[2], *lo[2];
    for (int i = 0; i < 2; ++i) {
        hi[i] = reinterpret_cast<half_t*>(ws + L.hi[i]);
        lo[i] = reinterpret_cast<half_t*>(ws + L.lo[i]);
    }
    const int64_t begin_tiles = (int64_t)(L.np / 64) * (L.mp / 64);
    hipLaunchKernelGGL(ns_begin_kernel<T>, dim3((unsigned)std::min<int64_t>(begin_tiles, 2048), (unsigned)count), dim3(kNsThreads), 0, s, g, ld_g, stride_g, parts, n_parts,
                       eps, scale, s_scale, pow(std::max(1.0, fabs((double)a)), steps), steps ? hi[0] : nullptr, lo[0], scales, L.mp, L.np, L.m,
                       L.n, transposed, out, ld_out, stride_out);
    if (hipGetLastError() != hipSuccess) return TPPO_ERR_LAUNCH;
    NsArgs x = {};
    x.each_off = (int64_t)L.mp * L.mp;
    x.each_diag = L.mp;
    x.each_x = (int64_t)L.mp * L.np;
    x.ld_off = L.mp;
    x.ld_x = L.np;
    x.a = a; x.b = b; x.c = c;
    x.m = L.m; x.n = L.n; x.transposed = transposed;
    x.out = out; x.ld_out = ld_out; x.each_out = stride_out; x.scales = scales;
    const NsWay way = ns_way(L, count, steps, a, b, c);
    if (way == kNsPairs) {
        const NsShape shape = {L.m, L.n, L.mp, L.np, transposed, count, steps, a, b, c, out, ld_out, stride_out};
        return ns_gram(shape, hi[0], lo[0], scales, ws + L.shared, s);
    }
    half_t *off_a = reinterpret_cast<half_t*>(ws + L.off_a), *off_b = reinterpret_cast<half_t*>(ws + L.off_b);
    float *diag_a = reinterpret_cast<float*>(ws + L.diag_a), *diag_b = reinterpret_cast<float*>(ws + L.diag_b);
    half_t *off_a_lo = reinterpret_cast<half_t*>(ws + L.off_a_lo), *off_b_lo = reinterpret_cast<half_t*>(ws + L.off_b_lo);
    auto bytes = [](const half_t* from, const half_t* to) { return reinterpret_cast<const char*>(to) - reinterpret_cast<const char*>(from); };
    auto products = [&](auto split) {
        constexpr bool kSplit = decltype(split)::value;
        for (int i = 0; i < steps; ++i) {
            half_t *x_hi = hi[i & 1], *x_lo = lo[i & 1];
            NsArgs p = x;                            // A = X X^T
            p.t_op = p.v_op = x_hi;
            p.lo_t = p.lo_v = bytes(x_hi, x_lo);
            p.ld_t = p.ld_v = L.np;
            p.each_t = p.each_v = x.each_x;
            p.n_t = p.n_v = L.mp;
            p.k = L.np;
            p.off = off_a; p.off_lo = off_a_lo; p.diag = diag_a;
            if (const int rc = launch_ns_tiles<kSplit, kGram>(p, count, s)) return rc;
            p = x;                                   // B = b A + c A A
            p.t_op = p.v_op = off_a;
            p.lo_t = p.lo_v = bytes(off_a, off_a_lo);
            p.ld_t = p.ld_v = L.mp;
            p.each_t = p.each_v = x.each_off;
            p.n_t = p.n_v = p.k = L.mp;
            p.off = off_a; p.off_lo = off_a_lo; p.diag = diag_a;
            p.off_out = off_b; p.off_out_lo = off_b_lo; p.diag_out = diag_b;
            if (const int rc = launch_ns_tiles<kSplit, kPoly>(p, count, s)) return rc;
            p = x;                                   // X = a X + B X
            p.t_op = off_b; p.lo_t = bytes(off_b, off_b_lo); p.ld_t = L.mp; p.each_t = x.each_off; p.n_t = L.mp;
            p.v_op = x_hi; p.lo_v = bytes(x_hi, x_lo); p.ld_v = L.np; p.each_v = x.each_x; p.n_v = L.np;
            p.k = L.mp;
            p.diag = diag_b; p.hi = x_hi; p.lo = x_lo; p.hi_out = hi[~i & 1]; p.lo_out = lo[~i & 1];
            if (const int rc = i + 1 < steps ? launch_ns_tiles<kSplit, kUpdate>(p, count, s) : launch_ns_tiles<kSplit, kLast>(p, count, s)) return rc;
        }
        return (int)TPPO_OK;
    };
    return way == kNsThreePasses ? products(std::true_type()) : products(std::false_type());
}

}  // namespace tppo

extern "C" size_t tppo_orthogonalize_workspace_bytes(int64_t count, int64_t rows, int64_t cols) {
    using namespace tppo;
    if (count < 1 || !ns_sides(rows, cols) || count > INT32_MAX / 2) return 256;
    return ns_layout(count, rows, cols).total;
}

extern "C" int tppo_orthogonalize(const void* g, int64_t count, int64_t rows, int64_t cols, int64_t ld_g, int64_t stride_g, tppo_dtype dt,
                                  int32_t steps, float a, float b, float c, float eps, float scale, void* out, int64_t ld_out,
                                  int64_t stride_out, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace tppo;
    if (dt != TPPO_F32 && dt != TPPO_BF16) return TPPO_ERR_DTYPE;
    if (count < 0 || count > 65535 || !ns_sides(rows, cols) || ld_g < cols || ld_out < cols) return TPPO_ERR_SIZE;
    if (count > 1 && (stride_g < 0 || stride_out < (rows - 1) * ld_out + cols)) return TPPO_ERR_SIZE;
    if (steps < 0 || steps > 64 || !(eps >= 0.f)) return TPPO_ERR_PARAM;
    for (float v : {a, b, c, eps, scale})
        if (!(v - v == 0.f)) return TPPO_ERR_PARAM;
    // an X that shrinks below what its pairs of fp16 hold; the last step's stays in fp32
    if (steps > 1 && pow(fabs((double)a), steps - 1) < 1.0 / 4096) return TPPO_ERR_PARAM;
    if (count == 0) return TPPO_OK;
    if (!g || !out) return TPPO_ERR_NULL;
    if (!is_aligned(g, dt == TPPO_F32 ? 4 : 2) || !is_aligned(out, 2)) return TPPO_ERR_PARAM;
    const NsLayout L = ns_layout(count, rows, cols);
    // (tiles of the whole stack are numbered in 32 bits)
    if (count * ((L.mp / 64) * (int64_t)(L.np / 64)) > INT32_MAX) return TPPO_ERR_SIZE;
    if (!workspace || !is_aligned(workspace, 256) || workspace_bytes < L.total) return TPPO_ERR_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dt == TPPO_F32)
        return run_ns(static_cast<const float*>(g), count, rows, cols, ld_g, stride_g, steps, a, b, c, eps, scale, static_cast<uint16_t*>(out),
                      ld_out, stride_out, static_cast<char*>(workspace), s);
    return run_ns(static_cast<const uint16_t*>(g), count, rows, cols, ld_g, stride_g, steps, a, b, c, eps, scale, static_cast<uint16_t*>(out),
                  ld_out, stride_out, static_cast<char*>(workspace), s);
}
