// tppo_orthogonalize for matrices with a short side: the iteration on X X^T alone (ortho.hip chooses).
//     X_k = P_k X_0 with P_k a polynomial of A_0 = X_0 X_0^T, and all of these m x m matrices are symmetric and commute:
//     M = a I + b A + c A A,   A <- M A M,   P <- M P;   at the end X = P X_0.
// X is read twice instead of twice a step, and what is left between is m x m: 6 m^2 n + 17 m^3 flop (5 steps, halves of symmetric
// results not counted) against 15 m^2 n + 5 m^3.
// Bound by the chain of products that wait for each other: 64 x 1024: 27.4 us (norm 3, first X 4, X X^T 5, all steps 12, P X 4); eight of
// 1000 x 333: 155, of which 14 products of 6.5 to 9.
// Precision.  A holds squares of singular values, and its errors where they are small grow by a^2 a step.  So everything here is a pair of
// fp16, hi + lo, rounded to nearest, 22 bits of what is not far below 1, products are hi hi + hi lo + lo hi with sums in fp32, and A is made
// symmetric to the bit, step by step.  Emulated against 64 bits: 1.6e-3 of the result's norm at worst (2 x 3, singular values 1 and 0.01), 1e-3
// from 64 on; with halves cut instead of rounded three times that.  (X itself, whose entries are smaller, has its low halves times 2048.)
#include <algorithm>
#include <cmath>

#include "ortho.h"

namespace tppo {

constexpr float kPolyScale = 16.f;                   // of P, whose eigenvalues go up to a^steps
constexpr int kPairThreads = 512, kPairTile = 64, kPairStage = 4 * kPairTile * 128;

enum PairMode { kPairGram, kPairWhole, kPairPoly, kPairMul, kPairLast };        // X X^T: partial sums of it; all of it, as pairs

// One product of pairs, out[t, v] = sum_k t_op[t, k] v_op[v, k] (kPairLast: v_op[k, v]).
struct PairProblem {
    const half_t* op[4];                             // T's high halves, its low ones, V's
    half_t *out_hi, *out_lo;
    float in_scale, out_scale;                       // the sum times in_scale is the value; stored times out_scale
};
struct PairArgs {
    PairProblem problem[2];
    int64_t each_t, each_v, each_out;
    int ld_t, ld_v, ld_out;
    int tiles, stages, chunks, count;                // tiles: of one matrix, kPairLast: of V; chunks: of the contraction (kPairGram)
    int deep;                                        // chunks; kPairLast: T tiles; or 1
    double by_deep, by_tiles, by_count;              // their reciprocals
    float* part;                                     // kPairGram: [chunk][matrix][mp][mp], tiles on one side of the diagonal
    const float2* scales;
    NsShape x;
};

// quotient and remainder by a number whose reciprocal is there (a division in integers is forty instructions of the few that a small product is)
__device__ __forceinline__ int pair_divide(int x, int by, double inverse, int& over) {
    int q = (int)((double)x * inverse);
    over = x - q * by;
    if (over < 0) {
        --q;
        over += by;
    } else if (over >= by) {
        ++q;
        over -= by;
    }
    return q;
}

// tile `id` of those with v >= t
__device__ __forceinline__ void pair_tile_at(int id, int& t, int& v) {
    v = 0;
    while ((v + 1) * (v + 2) / 2 <= id) ++v;
    t = id - v * (v + 1) / 2;
}

// A tile of a symmetric matrix as pairs to both sides of the diagonal, from LDS (fp32, tile[t][v]), eight entries of a row at a time.  A
// tile on the diagonal is taken from where v >= t.
constexpr int kTileLd = kPairTile + 1;
template <int THREADS>
__device__ __forceinline__ void pair_store(const float (*tile)[kTileLd], int t0, int v0, half_t* hi, half_t* lo, int ld) {
#pragma unroll
    for (int turn = 0; turn < 1024 / THREADS; ++turn) {
        const bool back = turn >= 512 / THREADS;                     // the mirrored tile: row v0 + r, columns t0 + c ..
        if (back && t0 == v0) break;
        const int r = turn % (512 / THREADS) * (THREADS / 8) + ((int)threadIdx.x >> 3), c = (threadIdx.x & 7) * 8;
        half8 h, l;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool flip = back || (t0 == v0 && c + e < r);
            const float y = flip ? tile[c + e][r] : tile[r][c + e];
            h[e] = (half_t)y;
            l[e] = (half_t)(y - (float)h[e]);
        }
        const int64_t to = (int64_t)((back ? v0 : t0) + r) * ld + (back ? t0 : v0) + c;
        *reinterpret_cast<half8*>(hi + to) = h;
        *reinterpret_cast<half8*>(lo + to) = l;
    }
}

// 64 x 64 tiles, eight wavefronts of 16 x 32 (four of 32 x 32, us:  1024 x 1024: 212, so: 206;  333 x 512: 117.5, 112;  1536 x 6144: 557, 563).  A
// stage holds 64 of K of both operands' halves, an eighth of it loaded by each wavefront.  Few
// workgroups keep two stages under way, one to a CU; many one, two to a CU.  One / two / three / four stages under way, by four wavefronts, us:  1024 x 1024: 231 /
// 214 / 225 / 231;  512 x 512: 146 / 142 / 150 / 155;  333 x 512: 127 / 119 / 125 / 129.
template <PairMode MODE, int STAGES>                 // STAGES: places for them, 2 or 3
__global__ __launch_bounds__(kPairThreads, STAGES == 2 ? 4 : 2) void ns_pair_kernel(PairArgs p) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    constexpr bool kKMajor = MODE == kPairLast, kBothX = MODE == kPairGram || MODE == kPairWhole;
    // chunk by chunk, or V tile by V tile, of a tile, tile by tile, matrix by matrix, problem by problem; consecutive ones on an XCD, whose L2
    // holds a small matrix (eight of 333 rows spread over all: 174 -> 183 us a call)
    int rest = ns_by_xcd(blockIdx.x, gridDim.x), inner, tile, mat;
    rest = pair_divide(rest, p.deep, p.by_deep, inner);
    rest = pair_divide(rest, p.tiles, p.by_tiles, tile);
    rest = pair_divide(rest, p.count, p.by_count, mat);
    const int chunk = MODE == kPairGram ? inner : 0;
    const PairProblem& q = p.problem[MODE == kPairMul ? rest : 0];
    int tile_t, tile_v;
    if constexpr (MODE == kPairLast) {
        tile_t = inner;
        tile_v = tile;
    } else {
        pair_tile_at(tile, tile_t, tile_v);
    }
    const int t0 = tile_t * kPairTile, v0 = tile_v * kPairTile;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wv = wave >> 1, wt = wave & 1, kind = wave >> 1, col = lane & 15, grp = lane >> 4;
    const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const int first = (int)((int64_t)p.stages * chunk / p.chunks), stages = (int)((int64_t)p.stages * (chunk + 1) / p.chunks) - first;

    // loader: a half of an operand's high or low halves to a wavefront; lane l of transfer d has row d * 8 + l / 8 of it, slot l % 8
    const bool on_v = kind >= 2;
    const half_t* base = q.op[kind];
    const int ld = on_v ? p.ld_v : p.ld_t;
    const char* src = reinterpret_cast<const char*>(base + mat * (on_v ? p.each_v : p.each_t));
    int64_t row_step, k_step;
    const int row = (wave & 1) * 32 + (lane >> 3);
    int chunk_at[2];                                 // of even and odd transfers: their rows are 8 apart
    if (on_v && kKMajor) {
        src += ((int64_t)row * ld + v0) * 2;
        row_step = (int64_t)8 * ld * 2;
        k_step = (int64_t)64 * ld * 2;
        chunk_at[0] = ((lane & 7) ^ ns_swz_k<64>(row)) * 16;
        chunk_at[1] = ((lane & 7) ^ ns_swz_k<64>(row + 8)) * 16;
    } else {
        src += (int64_t)((on_v ? v0 : t0) + row) * ld * 2;
        row_step = (int64_t)8 * ld * 2;
        k_step = 128;
        chunk_at[0] = ((lane & 7) ^ ns_swz(row)) * 16;
        chunk_at[1] = ((lane & 7) ^ ns_swz(row + 8)) * 16;
    }
    auto issue = [&](int stage, int slot) {
        const char* from = src + stage * k_step;
        const unsigned dst = lds_base + slot * kPairStage + wave * 4096;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            dma_16b_per_lane(from + chunk_at[d & 1], dst, d * 1024);
            from += row_step;
        }
    };
    f32x4 acc[2] = {}, cross[2] = {};
    for (int it = 0; it < STAGES - 1 && it < stages; ++it) issue(first + it, it);
    for (int it = 0; it < stages; ++it) {
        const int behind = min(STAGES - 2, stages - 1 - it);         // stages asked for after this one, four transfers each
        if (behind == 0) __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
        else __builtin_amdgcn_s_waitcnt(vmcnt_imm(4));
        __syncthreads();                             // this stage is there for everyone, and everyone has left the one before
        if (it + STAGES - 1 < stages) issue(first + it + STAGES - 1, (it + STAGES - 1) % STAGES);
        const unsigned at = it % STAGES * kPairStage;
#pragma unroll
        for (int k32 = 0; k32 < 2; ++k32) {
            half8 t[2][2], v[2];                     // [hi, lo], T's [block]
            const int c = k32 * 4 + grp, rv = wv * 16 + col;
#pragma unroll
            for (int part = 0; part < 2; ++part) {
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int rt = wt * 32 + b * 16 + col;
                    t[part][b] = *reinterpret_cast<const half8*>(smem + at + part * 8192 + rt * 128 + ((c ^ ns_swz(rt)) << 4));
                }
                if constexpr (kKMajor) v[part] = ns_k_major_frag<64>(lds_base + at + (2 + part) * 8192, wv, k32, lane);
                else v[part] = *reinterpret_cast<const half8*>(smem + at + (2 + part) * 8192 + rv * 128 + ((c ^ ns_swz(rv)) << 4));
            }
#pragma unroll
            for (int tb = 0; tb < 2; ++tb) {
                acc[tb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[0], t[0][tb], acc[tb], 0, 0, 0);
                f32x4& with_t = kBothX ? cross[tb] : acc[tb];                      // (X's low halves are scaled)
                f32x4& with_v = kBothX || MODE == kPairLast ? cross[tb] : acc[tb];
                with_t = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[0], t[1][tb], with_t, 0, 0, 0);
                with_v = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[1], t[0][tb], with_v, 0, 0, 0);
            }
        }
    }
    float(*tile_out)[kTileLd] = reinterpret_cast<float(*)[kTileLd]>(smem);
    if constexpr (MODE != kPairGram) __syncthreads();                // (the stages are read)
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
        const int t = t0 + wt * 32 + tb * 16 + col;
        const int v = v0 + wv * 16 + grp * 4;
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            x[e] = kBothX || MODE == kPairLast ? fmaf(cross[tb][e], 1.f / kLoScale, acc[tb][e]) : acc[tb][e];
        if constexpr (MODE == kPairGram) {
            *reinterpret_cast<float4*>(p.part + ((int64_t)chunk * p.count + mat) * p.each_out + (int64_t)t * p.ld_out + v) =
                make_float4(x[0], x[1], x[2], x[3]);
        } else if constexpr (MODE == kPairLast) {
            const float by = q.in_scale * p.scales[mat].y;
#pragma unroll
            for (int e = 0; e < 4; ++e) tile_out[t - t0][v - v0 + e] = x[e] * by;
        } else {
            half4 a_hi, a_lo;
            if constexpr (MODE == kPairPoly) {   // (t_op is A)
                const int64_t at = mat * p.each_t + (int64_t)t * p.ld_t + v;
                a_hi = *reinterpret_cast<const half4*>(q.op[0] + at);
                a_lo = *reinterpret_cast<const half4*>(q.op[1] + at);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float y = x[e] * (MODE == kPairWhole ? p.scales[mat].x : q.in_scale);
                if constexpr (MODE == kPairPoly)
                    y = fmaf(p.x.c, y, fmaf(p.x.b * (1.f / kOffScale), (float)a_hi[e] + (float)a_lo[e], t == v + e ? p.x.a : 0.f));
                tile_out[t - t0][v - v0 + e] = y * q.out_scale;
            }
        }
    }
    if constexpr (MODE == kPairLast) {               // eight entries of a row of the caller's matrix at a time
        __syncthreads();
        {
            const int r = (int)threadIdx.x >> 3, c = (threadIdx.x & 7) * 8;
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = p.x.transposed ? tile_out[c + e][r] : tile_out[r][c + e];
            const int row_at = p.x.transposed ? v0 + r : t0 + r, rows = p.x.transposed ? p.x.n : p.x.m;
            const int col_at = p.x.transposed ? t0 + c : v0 + c, cols = p.x.transposed ? p.x.m : p.x.n;
            if (row_at < rows && col_at < cols)
                put_whole_or_part(p.x.out + mat * p.x.each_out + (int64_t)row_at * p.x.ld_out + col_at, cols - col_at, x);
        }
    }
    if constexpr (MODE == kPairWhole || MODE == kPairPoly || MODE == kPairMul) {
        __syncthreads();
        pair_store<kPairThreads>(tile_out, t0, v0, q.out_hi + mat * p.each_out, q.out_lo + mat * p.each_out, p.ld_out);
    }
}

// A from the partial sums of its tiles, scaled, as pairs on both sides of the diagonal.
__global__ __launch_bounds__(256) void ns_gather_kernel(const float* part, int chunks, int count, int mp, const float2* scales, half_t* hi, half_t* lo) {
    __shared__ float tile[kPairTile][kTileLd];
    const int mat = blockIdx.y;
    int tile_t, tile_v;
    pair_tile_at(blockIdx.x, tile_t, tile_v);
    const int t0 = tile_t * kPairTile, v0 = tile_v * kPairTile;
    const float by = scales[mat].x * kOffScale;
#pragma unroll
    for (int turn = 0; turn < 4; ++turn) {
        const int r = turn * 16 + ((int)threadIdx.x >> 4), c = (threadIdx.x & 15) * 4;
        const float* at = part + ((int64_t)mat * mp + t0 + r) * mp + v0 + c;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int k = 0; k < chunks; ++k) {
            const float4 x = *reinterpret_cast<const float4*>(at + (int64_t)k * count * mp * mp);
            sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
        }
        tile[r][c] = sum.x * by;
        tile[r][c + 1] = sum.y * by;
        tile[r][c + 2] = sum.z * by;
        tile[r][c + 3] = sum.w * by;
    }
    __syncthreads();
    pair_store<256>(tile, t0, v0, hi + (int64_t)mat * mp * mp, lo + (int64_t)mat * mp * mp, mp);
}

// All steps of one matrix of up to MP = 64 or 128 rows in one workgroup, a strip of 16 columns of every matrix to a wavefront.
// A block of 16 x 16 comes out of an MFMA as it goes into one: lane l has column l % 16 and rows 4 (l / 16) .. + 3, and two blocks are the
// 32 of K of the next one's operand, in an order of their own, the same on both sides.  So a strip stays in registers from product to
// product (M A, then M (M A)); as the matrices are symmetric the other operand, all rows of A or M, is every wavefront's strip as well, and
// passes through LDS once a step each, in the order of the lanes.  Only the new A is exchanged across the diagonal, where it is
// made the mean of both sides.
// Bound by the chain of products: 17 for 5 steps, 24 MFMAs a wavefront each (96 at 128 rows), and by LDS, which every wavefront reads whole.
// 64 rows, us: so, 12.2; blocks of lower triangles dealt out to 16 wavefronts, mirrored in LDS by pieces of two bytes, 16.5; all blocks where
// they lie, operands from LDS, 16 wavefronts 20.7, four 26.5.  A call with 128 x 1024: 61; two strips to each of four wavefronts 68; sums read
// where each lane wants them, across the diagonal, 117.
template <int MP>
__global__ __launch_bounds__(MP * 4, MP / 64) void ns_iterate_kernel(const float* part, int chunks, int count, const float2* scales, int steps,
                                                                     float a, float b, float c, half_t* p_hi, half_t* p_lo) {
    constexpr int kThreads = MP * 4, kB = MP / 16, kPairs = kB / 2;                   // blocks of a column; operands of 32 of K
    constexpr int kOperand = kB * kPairs * 2 * 1024, kTurnLd = MP + 1;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    unsigned char *const all_m = smem, *const all_a = smem + kOperand;
    float* const turned = reinterpret_cast<float*>(all_a);           // (MP x kTurnLd, when A has been read)
    const int mat = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4, t = wave * 16 + col;
    typedef f32x4 Strip[kB];
    struct Pairs {
        half8 hi[kPairs], lo[kPairs];
    };
    Strip A, M, S;
    Pairs pa, pm, pp;
    const float by = scales[mat].x * kOffScale;
    {   // the parts' sum, in whole pieces and through LDS (there are sums on and above the diagonal)
        constexpr int kPieces = MP * MP / 4 / kThreads;
        float4 sum[kPieces];
#pragma unroll
        for (int q = 0; q < kPieces; ++q) sum[q] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
        for (int k = 0; k < chunks; ++k) {
            const float4* at = reinterpret_cast<const float4*>(part + ((int64_t)k * count + mat) * MP * MP) + threadIdx.x;
#pragma unroll
            for (int q = 0; q < kPieces; ++q) {
                const float4 x = at[q * kThreads];
                sum[q].x += x.x; sum[q].y += x.y; sum[q].z += x.z; sum[q].w += x.w;
            }
        }
#pragma unroll
        for (int q = 0; q < kPieces; ++q) {
            const int at = (q * kThreads + (int)threadIdx.x) * 4;
            float* to = turned + at / MP * kTurnLd + at % MP;
            to[0] = sum[q].x; to[1] = sum[q].y; to[2] = sum[q].z; to[3] = sum[q].w;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kB; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int v = j * 16 + grp * 4 + e;
                A[j][e] = turned[min(t, v) * kTurnLd + max(t, v)] * by;
            }
        __syncthreads();
    }
    auto split = [&](const Strip& x, Pairs& p) {
        typedef float f2 __attribute__((ext_vector_type(2)));
        typedef half_t h2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int j = 0; j < kB; ++j)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const f2 y = {x[j][e], x[j][e + 1]};
                const h2 h = __builtin_convertvector(y, h2);
                const f2 rest = {y[0] - (float)h[0], y[1] - (float)h[1]};
                const h2 l = __builtin_convertvector(rest, h2);
                const int at = (j & 1) * 4 + e;
                p.hi[j >> 1][at] = h[0];
                p.hi[j >> 1][at + 1] = h[1];
                p.lo[j >> 1][at] = l[0];
                p.lo[j >> 1][at + 1] = l[1];
            }
    };
    // this strip as rows of the other operand
    auto publish = [&](unsigned char* all, const Pairs& p) {
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            half8* at = reinterpret_cast<half8*>(all + ((wave * kPairs + j) * 2) * 1024) + lane;
            at[0] = p.hi[j];
            at[64] = p.lo[j];
        }
    };
    // (chains of MFMAs on one sum side by side: four rows of blocks at a time; at 128 rows no operand is asked for further ahead, or they all
    // are, which takes 221 registers more than there are)
    auto product = [&](const unsigned char* all, const Pairs& p, Strip& out) {
#pragma unroll
        for (int r0 = 0; r0 < kB; r0 += 4) {
#pragma unroll
            for (int r = r0; r < r0 + 4; ++r) out[r] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                if constexpr (MP > 64) __builtin_amdgcn_sched_barrier(0);
                half8 hi[4], lo[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const half8* at = reinterpret_cast<const half8*>(all + (((r0 + r) * kPairs + j) * 2) * 1024) + lane;
                    hi[r] = at[0];
                    lo[r] = at[64];
                }
#pragma unroll
                for (int part = 0; part < 3; ++part)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        out[r0 + r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(part < 2 ? hi[r] : lo[r], part == 1 ? p.lo[j] : p.hi[j], out[r0 + r], 0, 0, 0);
            }
        }
    };
    // A is held times kOff, P times kPolyScale, M as it is: what M multiplies keeps its scale
    constexpr float kOff = kOffScale;
    split(A, pa);
    publish(all_a, pa);
    __syncthreads();
    for (int step = 0; step < steps; ++step) {
        const bool last = step + 1 == steps;
        product(all_a, pa, S);
#pragma unroll
        for (int j = 0; j < kB; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                M[j][e] = fmaf(c * (1.f / (kOff * kOff)), S[j][e], fmaf(b * (1.f / kOff), A[j][e], t == j * 16 + grp * 4 + e ? a : 0.f));
        split(M, pm);
        publish(all_m, pm);
        if (step == 0) {
#pragma unroll
            for (int j = 0; j < kB; ++j) M[j] *= kPolyScale;
            split(M, pp);
        }
        __syncthreads();                                             // all of M is there; A has been read
        if (step > 0) {
            product(all_m, pp, S);                                   // M P
            split(S, pp);
        }
        if (last) break;
        product(all_m, pa, S);                                       // M A
        split(S, pa);
        product(all_m, pa, S);                                       // M M A
#pragma unroll
        for (int j = 0; j < kB; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) turned[(j * 16 + grp * 4 + e) * kTurnLd + t] = S[j][e];
        __syncthreads();                                             // and M has been read
#pragma unroll
        for (int j = 0; j < kB; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) A[j][e] = (S[j][e] + turned[t * kTurnLd + j * 16 + grp * 4 + e]) * 0.5f;
        split(A, pa);
        __syncthreads();
        publish(all_a, pa);
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < kB; ++j) {
        const int64_t at = ((int64_t)mat * MP + t) * MP + j * 16 + grp * 4;
        const half8 h = pp.hi[j >> 1], l = pp.lo[j >> 1];
        *reinterpret_cast<half4*>(p_hi + at) = j & 1 ? half4{h[4], h[5], h[6], h[7]} : half4{h[0], h[1], h[2], h[3]};
        *reinterpret_cast<half4*>(p_lo + at) = j & 1 ? half4{l[4], l[5], l[6], l[7]} : half4{l[0], l[1], l[2], l[3]};
    }
}

// Partial sums of many chunks into the first one's place: 64 float4 a workgroup, its four wavefronts a quarter of the chunks each.
constexpr int kFewChunks = 8;
__global__ __launch_bounds__(256) void ns_reduce_kernel(float4* part, int chunks, int64_t each) {
    __shared__ float4 place[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t at = (int64_t)blockIdx.x * 64 + lane;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int k = wave; k < chunks; k += 4) {
        const float4 x = part[k * each + at];
        sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
    }
    place[wave][lane] = sum;
    __syncthreads();
    if (wave == 0) {
        for (int w = 1; w < 4; ++w) {
            const float4 x = place[w][lane];
            sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
        }
        part[at] = sum;
    }
}

// g maps [0, u] onto [0, its largest value there], which lies at u or where g' = m (m + 2 l m') = 0, m + 2 l m' = a + 3 b l + 5 c l l.  So the
// ranges follow from one another, and m has its extremes at their ends or at its vertex.  (A thousandth more is for roundings.)
NsReach ns_reach(int steps, float a_, float b_, float c_) {
    const double a = a_, b = b_, c = c_, none = HUGE_VAL;
    NsReach r = {1.0, 0.0, none, 1.0};
    double u = 1.0, product = 1.0;
    auto m = [&](double l) { return a + l * (b + l * c); };
    for (int k = 0; k < steps; ++k) {
        if (!(u < 1e60)) return {none, none, 0.0, none};
        const double top = u * 1.001, vertex = c != 0.0 ? -b / (2.0 * c) : -1.0;
        double low = std::min(m(0.0), m(top)), high = std::max(m(0.0), m(top));
        if (vertex > 0.0 && vertex < top) {
            low = std::min(low, m(vertex));
            high = std::max(high, m(vertex));
        }
        u = top * m(top) * m(top);
        auto also = [&](double l) {
            if (l > 0.0 && l < top) u = std::max(u, l * m(l) * m(l));
        };
        const double inside = 9.0 * b * b - 20.0 * a * c;
        if (inside >= 0.0) {                         // (the quadratic's roots, or the linear's one)
            const double q = -0.5 * (3.0 * b + copysign(sqrt(inside), b));
            if (c != 0.0) also(q / (5.0 * c));
            if (q != 0.0) also(a / q);
        }
        const double most = std::max(fabs(low), fabs(high)), least = low <= 0.0 && high >= 0.0 ? 0.0 : std::min(fabs(low), fabs(high));
        product *= most;
        r.product = std::max(r.product, product);
        r.value = std::max(r.value, most);
        r.least = std::min(r.least, least);
        r.square = std::max(r.square, u);
    }
    return r;
}

// Whether this way holds the iteration.  What it stores stays within fp16 at its scales, with a factor of four to spare: 16 P, 64 A, 64 M.  And
// the roundings, halves of a step of 2^-23, stay below 2e-3 of the result.  What they come to, in such steps, with q = a / (least m):
//   those of P and M, which M's diagonal makes a times as large a step, against a result that is `least` times as large:  steps q^(steps - 1);
//   those of T = M A, terms of a + |b| + |c| that cancel to m: A's eigenvectors turn by (a + |b| + |c|) a / 2 m^2, P's do not:  times q^j, added up;
//   those of A's small eigenvalues, which grow by a^2 a step and which M takes times b:  (a + |b| + |c|) |b| a^(2 steps - 4).
// Each is over-estimated by the worst case of every factor; the limits are a little above what the five steps of the default coefficients come to (4.2e3,
// 4.5e4, 8.2e4).  Emulated against 64 bits, 3280 sets of coefficients and steps, ranks from one to full, 2 to 260 rows: within the limits
// 1.9e-3 at most, beyond them up to all of the result (m near zero where the singular values are; on the card 9 % for 3.4987, -5.165,
// 1.7679).
bool ns_gram_fits(const NsReach& r, int steps, float a, float b, float c) {
    if (steps < 1 || !(r.product <= 1000.0 && r.value <= 250.0 && r.square <= 250.0 && r.least > 0.0)) return false;
    const double aa = fabs((double)a), sum = aa + fabs((double)b) + fabs((double)c), q = std::max(1.0, aa / r.least);
    if (aa < 1.0) return false;                      // (P shrinks below what pairs hold)
    double power = 1.0, all = 0.0;
    for (int k = 1; k < steps; ++k) all += power *= q;
    return steps * power <= 1e4 && sum * aa / (2.0 * r.least * r.least) * all <= 6e4 &&
           (steps == 1 || sum * fabs((double)b) * pow(aa, 2 * steps - 4) <= 9e4);
}

namespace {
constexpr int kIterateMost = 128;                    // rows of what ns_iterate_kernel takes
constexpr int64_t kGatherStages = 11;
struct GramLayout {
    int tiles, chunks;
    size_t part, m[2], p[2], a, t, total;            // pairs: hi, then lo
};
GramLayout gram_layout(int64_t count, int mp, int np) {
    GramLayout L;
    const int side = mp / kPairTile;
    L.tiles = side * (side + 1) / 2;
    // contractions are cut until there are two workgroups to a CU, each with four stages at least; not where that saves no more stages than
    // the launch that gathers the parts takes.  us, cut / whole:  512 x 512, 8 stages in 2 parts: 152.7 / 150.3;  8 x 1000 x 333, 16 in 3: 167.7 /
    // 164.3;  512 x 1024, 16 in 4: 152.0 / 154.1;  333 x 2048, 32 in 8: 130.7 / 139.1
    const int64_t all = (int64_t)L.tiles * count, stages = np / 64;
    L.chunks = (int)std::max<int64_t>(1, std::min<int64_t>(stages / 4, 512 / all));
    if (mp > kIterateMost && stages - stages / L.chunks <= kGatherStages) L.chunks = 1;
    size_t o = 0;
    auto take = [&](size_t bytes) {
        const size_t at = o;
        o += round_up(bytes, 256);
        return at;
    };
    const size_t pair = (size_t)count * mp * mp * 4;
    L.part = take(mp > kIterateMost && L.chunks == 1 ? 0 : (size_t)L.chunks * count * mp * mp * 4);
    for (size_t* at : {&L.m[0], &L.m[1], &L.p[0], &L.p[1], &L.a, &L.t}) *at = take(pair);
    L.total = o;
    return L;
}
template <PairMode MODE>
int launch_pair(PairArgs& p, int problems, hipStream_t s) {
    p.deep = MODE == kPairGram ? p.chunks : MODE == kPairLast ? p.x.mp / kPairTile : 1;
    p.by_deep = 1.0 / p.deep;
    p.by_tiles = 1.0 / p.tiles;
    p.by_count = 1.0 / p.count;
    const unsigned groups = (unsigned)((int64_t)p.tiles * p.count * p.deep * problems);
    if (groups <= kSweepGroups) {
        if (!allow_lds(reinterpret_cast<const void*>(ns_pair_kernel<MODE, 3>), 3 * kPairStage)) return TPPO_ERR_LAUNCH;
        hipLaunchKernelGGL((ns_pair_kernel<MODE, 3>), dim3(groups), dim3(kPairThreads), 3 * kPairStage, s, p);
    } else {
        hipLaunchKernelGGL((ns_pair_kernel<MODE, 2>), dim3(groups), dim3(kPairThreads), 2 * kPairStage, s, p);
    }
    return launch_result();
}
template <int MP>
int launch_iterate(const PairArgs& p, half_t* p_hi, half_t* p_lo, hipStream_t s) {
    constexpr int kLds = MP * MP * 4 + MP * (MP + 1) * 4;            // one operand, and the other or A turned round
    if (kLds > 64 * 1024 && !allow_lds(reinterpret_cast<const void*>(ns_iterate_kernel<MP>), kLds)) return TPPO_ERR_LAUNCH;
    hipLaunchKernelGGL(ns_iterate_kernel<MP>, dim3((unsigned)p.count), dim3(MP * 4), kLds, s, p.part, p.chunks, p.count, p.scales,
                       p.x.steps, p.x.a, p.x.b, p.x.c, p_hi, p_lo);
    return launch_result();
}
}  // namespace

size_t ns_gram_bytes(int64_t count, int m, int n) { return gram_layout(count, (m + 63) / 64 * 64, (n + 63) / 64 * 64).total; }

int ns_gram(const NsShape& x, const half_t* hi, const half_t* lo, const float2* scales, char* ws, hipStream_t s) {
    const int mp = x.mp, np = x.np;
    const GramLayout L = gram_layout(x.count, mp, np);
    const int64_t each = (int64_t)mp * mp, half = x.count * each;
    auto pair = [&](size_t at) { return reinterpret_cast<half_t*>(ws + at); };
    half_t *A = pair(L.a), *T = pair(L.t);
    PairArgs p = {};
    p.x = x;
    p.scales = scales;
    p.count = (int)x.count;
    p.part = reinterpret_cast<float*>(ws + L.part);
    p.each_out = each;
    p.ld_out = mp;
    // A = X X^T
    p.problem[0] = {{hi, lo, hi, lo}, nullptr, nullptr, 1.f, 1.f};
    p.each_t = p.each_v = (int64_t)mp * np;
    p.ld_t = p.ld_v = np;
    p.tiles = L.tiles;
    p.stages = np / 64;
    p.chunks = L.chunks;
    const bool whole = mp > kIterateMost && L.chunks == 1;
    if (whole) {
        p.problem[0] = {{hi, lo, hi, lo}, A, A + half, 1.f, kOffScale};
        if (launch_pair<kPairWhole>(p, 1, s) != TPPO_OK) return TPPO_ERR_LAUNCH;
    } else if (launch_pair<kPairGram>(p, 1, s) != TPPO_OK) {
        return TPPO_ERR_LAUNCH;
    }
    if (L.chunks > kFewChunks) {
        const int64_t quads = half / 4;
        hipLaunchKernelGGL(ns_reduce_kernel, dim3((unsigned)(quads / 64)), dim3(256), 0, s, reinterpret_cast<float4*>(p.part), L.chunks, quads);
        p.chunks = 1;
    }
    half_t* P = pair(L.p[0]);
    float p_scale = kPolyScale;
    if (mp <= kIterateMost) {
        if ((mp == 64 ? launch_iterate<64>(p, P, P + half, s) : launch_iterate<128>(p, P, P + half, s)) != TPPO_OK) return TPPO_ERR_LAUNCH;
    } else {
        if (!whole)
            hipLaunchKernelGGL(ns_gather_kernel, dim3((unsigned)L.tiles, (unsigned)x.count), dim3(256), 0, s, p.part, p.chunks, p.count, mp,
                               scales, A, A + half);
        p.chunks = 1;
        p.stages = mp / 64;
        p.each_t = p.each_v = each;
        p.ld_t = p.ld_v = mp;
        const float off2 = 1.f / (kOffScale * kOffScale);
        for (int k = 0; k < x.steps; ++k) {
            half_t* M = pair(L.m[k & 1]);
            p.problem[0] = {{A, A + half, A, A + half}, M, M + half, off2, kOffScale};
            if (launch_pair<kPairPoly>(p, 1, s) != TPPO_OK) return TPPO_ERR_LAUNCH;
            const bool last = k + 1 == x.steps;
            int problems = 0;
            half_t* next = pair(L.p[k & 1]);
            if (!last) p.problem[problems++] = {{M, M + half, A, A + half}, T, T + half, off2, kOffScale};
            if (k > 0) p.problem[problems++] = {{M, M + half, P, P + half}, next, next + half, 1.f / (kOffScale * p_scale), kPolyScale};
            if (problems && launch_pair<kPairMul>(p, problems, s) != TPPO_OK) return TPPO_ERR_LAUNCH;
            if (!last) {
                p.problem[0] = {{T, T + half, M, M + half}, A, A + half, off2, kOffScale};
                if (launch_pair<kPairMul>(p, 1, s) != TPPO_OK) return TPPO_ERR_LAUNCH;
            }
            P = k == 0 ? M : next;
            p_scale = k == 0 ? kOffScale : kPolyScale;
        }
    }
    // X = P X
    p.problem[0] = {{P, P + half, hi, lo}, nullptr, nullptr, 1.f / p_scale, 1.f};
    p.each_t = each;
    p.ld_t = mp;
    p.each_v = (int64_t)mp * np;
    p.ld_v = np;
    p.tiles = np / kPairTile;
    p.stages = mp / 64;
    p.chunks = 1;
    return launch_pair<kPairLast>(p, 1, s);
}

}  // namespace tppo
