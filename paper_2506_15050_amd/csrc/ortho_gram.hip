// tppo_orthogonalize for matrices with a short side, m < kGramBelow: the iteration on X X^T alone.
//     X_k = P_k X_0 with P_k a polynomial of A_0 = X_0 X_0^T, and all of these m x m matrices are symmetric and commute:
//     M = a I + b A + c A A,   A <- M A M,   P <- M P;   at the end X = P X_0.
// X is read twice instead of twice a step, and what is left between is m x m: 6 m^2 n + 17 m^3 flop (5 steps, halves of symmetric
// results not counted) against 15 m^2 n + 5 m^3.
// Precision.  A holds squares of singular values, and its errors where they are small grow by a^2 a step.  So everything here is a pair of
// fp16, 22 bits, products are hi hi + (hi lo + lo hi) / 2048 with both sums in fp32, and results are taken from one side of the diagonal:
// emulated against 64 bits 1.3e-3 of the result's norm at worst (2 x 3, singular values 1 and 0.01), 5e-4 from 64 on.
#include "ortho.h"

namespace tppo {

constexpr float kPolyScale = 16.f;                   // of P, whose eigenvalues go up to a^steps
constexpr int kPairThreads = 256, kPairTile = 64, kPairStage = 4 * kPairTile * 128;

enum PairMode { kPairGram, kPairPoly, kPairMul, kPairLast };

// One product of pairs, out[t, v] = sum_k t_op[t, k] v_op[v, k] (kPairLast: v_op[k, v]).
struct PairProblem {
    const half_t *t_hi, *t_lo, *v_hi, *v_lo;
    half_t *out_hi, *out_lo;
    float in_scale, out_scale;                       // the sum times in_scale is the value; stored times out_scale
};
struct PairArgs {
    PairProblem problem[2];
    int64_t each_t, each_v, each_out;
    int ld_t, ld_v, ld_out;
    int tiles_t, tiles_v, tiles, stages, chunks;     // tiles: of one matrix; chunks: of the contraction (kPairGram)
    int count;
    float* part;                                     // kPairGram: [chunk][matrix][mp][mp], tiles on one side of the diagonal
    const float2* scales;
    NsShape x;
};

// tile `id` of those with v >= t
__device__ __forceinline__ void pair_tile_at(int id, int& t, int& v) {
    v = 0;
    while ((v + 1) * (v + 2) / 2 <= id) ++v;
    t = id - v * (v + 1) / 2;
}

// 64 x 64 tiles, four wavefronts of 32 x 32.  A stage holds 64 of K of both operands' halves, a quarter of it loaded by each wavefront.
template <PairMode MODE>
__global__ __launch_bounds__(kPairThreads, 2) void ns_pair_kernel(PairArgs p) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    constexpr bool kKMajor = MODE == kPairLast;
    int id = ns_by_xcd(blockIdx.x, gridDim.x);
    const int chunk = id % p.chunks;
    id /= p.chunks;
    const int tile = id % p.tiles;
    id /= p.tiles;
    const int mat = id % p.count;
    const PairProblem& q = p.problem[id / p.count];
    int tile_t, tile_v;
    if constexpr (MODE == kPairLast) {
        tile_v = tile / p.tiles_t;
        tile_t = tile - tile_v * p.tiles_t;
    } else {
        pair_tile_at(tile, tile_t, tile_v);
    }
    const int t0 = tile_t * kPairTile, v0 = tile_v * kPairTile;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wv = wave >> 1, wt = wave & 1, col = lane & 15, grp = lane >> 4;
    const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const int first = (int)((int64_t)p.stages * chunk / p.chunks), stages = (int)((int64_t)p.stages * (chunk + 1) / p.chunks) - first;

    // loader: wavefront 0 T's high halves, 1 T's low ones, 2 and 3 V's; lane l of transfer d has row d * 8 + l / 8, slot l % 8
    const bool on_v = wave >= 2;
    const half_t* base = wave == 0 ? q.t_hi : wave == 1 ? q.t_lo : wave == 2 ? q.v_hi : q.v_lo;
    const int ld = on_v ? p.ld_v : p.ld_t;
    const char* src = reinterpret_cast<const char*>(base + mat * (on_v ? p.each_v : p.each_t));
    int64_t row_step, k_step;
    const int row = lane >> 3;
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
        const unsigned dst = lds_base + slot * kPairStage + wave * 8192;
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            dma_16b_per_lane(from + chunk_at[d & 1], dst, d * 1024);
            from += row_step;
        }
    };
    f32x4 acc[2][2] = {}, cross[2][2] = {};
    issue(first, 0);
    for (int it = 0; it < stages; ++it) {
        __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
        __syncthreads();                             // this stage is there for everyone, and everyone has left the other one
        if (it + 1 < stages) issue(first + it + 1, (it + 1) & 1);
        const unsigned at = (it & 1) * kPairStage;
#pragma unroll
        for (int k32 = 0; k32 < 2; ++k32) {
            half8 t[2][2], v[2][2];                  // [hi, lo][block]
            const int c = k32 * 4 + grp;
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int rt = wt * 32 + b * 16 + col, rv = wv * 32 + b * 16 + col;
                    t[part][b] = *reinterpret_cast<const half8*>(smem + at + part * 8192 + rt * 128 + ((c ^ ns_swz(rt)) << 4));
                    if constexpr (kKMajor) v[part][b] = ns_k_major_frag<64>(lds_base + at + (2 + part) * 8192, wv * 2 + b, k32, lane);
                    else v[part][b] = *reinterpret_cast<const half8*>(smem + at + (2 + part) * 8192 + rv * 128 + ((c ^ ns_swz(rv)) << 4));
                }
#pragma unroll
            for (int vb = 0; vb < 2; ++vb)
#pragma unroll
                for (int tb = 0; tb < 2; ++tb) {
                    acc[vb][tb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[0][vb], t[0][tb], acc[vb][tb], 0, 0, 0);
                    cross[vb][tb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[0][vb], t[1][tb], cross[vb][tb], 0, 0, 0);
                    cross[vb][tb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[1][vb], t[0][tb], cross[vb][tb], 0, 0, 0);
                }
        }
    }
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
        const int t = t0 + wt * 32 + tb * 16 + col;
#pragma unroll
        for (int vb = 0; vb < 2; ++vb) {
            const int v = v0 + wv * 32 + vb * 16 + grp * 4;
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = fmaf(cross[vb][tb][e], 1.f / kLoScale, acc[vb][tb][e]);
            if constexpr (MODE == kPairGram) {
                *reinterpret_cast<float4*>(p.part + ((int64_t)chunk * p.count + mat) * p.each_out + (int64_t)t * p.ld_out + v) =
                    make_float4(x[0], x[1], x[2], x[3]);
            } else if constexpr (MODE == kPairLast) {
                const float by = q.in_scale * p.scales[mat].y;
                if (t < p.x.m)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (v + e < p.x.n) {
                            const int64_t to = p.x.transposed ? (int64_t)(v + e) * p.x.ld_out + t : (int64_t)t * p.x.ld_out + v + e;
                            p.x.out[mat * p.x.each_out + to] = ns_bf16(x[e] * by);
                        }
            } else {
                half_t *hi = q.out_hi + mat * p.each_out, *lo = q.out_lo + mat * p.each_out;
                half4 a_hi, a_lo;
                if constexpr (MODE == kPairPoly) {   // (t_op is A)
                    const int64_t at = mat * p.each_t + (int64_t)t * p.ld_t + v;
                    a_hi = *reinterpret_cast<const half4*>(q.t_hi + at);
                    a_lo = *reinterpret_cast<const half4*>(q.t_lo + at);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float y = x[e] * q.in_scale;
                    if constexpr (MODE == kPairPoly)
                        y = fmaf(p.x.c, y, fmaf(p.x.b * (1.f / kOffScale), fmaf((float)a_lo[e], 1.f / kLoScale, (float)a_hi[e]), t == v + e ? p.x.a : 0.f));
                    y *= q.out_scale;
                    const half_t h = (half_t)y, l = (half_t)((y - (float)h) * kLoScale);
                    if (t <= v + e) {
                        const int64_t to = (int64_t)t * p.ld_out + v + e, back = (int64_t)(v + e) * p.ld_out + t;
                        hi[to] = h;
                        lo[to] = l;
                        hi[back] = h;
                        lo[back] = l;
                    }
                }
            }
        }
    }
}

// A from the partial sums of its tiles, scaled, as pairs on both sides of the diagonal.
__global__ __launch_bounds__(256) void ns_gather_kernel(const float* part, int chunks, int count, int mp, const float2* scales, half_t* hi, half_t* lo) {
    const int mat = blockIdx.y, id = blockIdx.x * 256 + threadIdx.x;
    if (id >= mp * mp) return;
    const int t = id / mp, v = id - t * mp;
    if (t > v) return;
    float x = 0.f;
    for (int c = 0; c < chunks; ++c) x += part[((int64_t)c * count + mat) * mp * mp + id];
    x *= scales[mat].x * kOffScale;
    const half_t h = (half_t)x, l = (half_t)((x - (float)h) * kLoScale);
    const int64_t to = (int64_t)mat * mp * mp + id, back = (int64_t)mat * mp * mp + v * mp + t;
    hi[to] = h;
    lo[to] = l;
    hi[back] = h;
    lo[back] = l;
}

// All steps of one matrix of up to MP = 64 or 128 rows in one workgroup: two matrices in LDS, what becomes of them in registers (16 x 16
// blocks on one side of the diagonal, dealt out to the wavefronts).
constexpr int kIterWaves = 16;
template <int MP>
struct IterShape {
    static constexpr int kSide = MP / 16, kBlocks = kSide * (kSide + 1) / 2, kMine = (kBlocks + kIterWaves - 1) / kIterWaves;
    static constexpr int kRowBytes = MP * 2, kPieces = MP / 8, kHalf = MP * kRowBytes, kMatrix = 2 * kHalf, kLds = 2 * kMatrix;
    __device__ static __forceinline__ int at(int r, int c) {                                   // byte of piece c of row r
        const int swz = MP == 64 ? (r >> 1) & 7 : r & 15;
        return r * kRowBytes + ((c ^ swz) << 4);
    }
};
template <int MP>
__global__ __launch_bounds__(kIterWaves * 64) void ns_iterate_kernel(const float* part, int chunks, int count, const float2* scales, int steps,
                                                                     float a, float b, float c, half_t* p_hi, half_t* p_lo) {
    typedef IterShape<MP> S;
    constexpr int kMine = S::kMine;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    unsigned char *const U = smem, *const V = smem + S::kMatrix;
    const int mat = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;
    int bt[kMine], bv[kMine];
    bool there[kMine];
    f32x4 A[kMine], M[kMine], P[kMine];
    const float by = scales[mat].x;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int id = wave + i * kIterWaves;
        there[i] = id < S::kBlocks;
        pair_tile_at(there[i] ? id : 0, bt[i], bv[i]);
        A[i] = f32x4{0, 0, 0, 0};
        M[i] = P[i] = A[i];
        if (there[i]) {
            const int64_t at = ((int64_t)mat * MP + bt[i] * 16 + col) * MP + bv[i] * 16 + grp * 4;
#pragma unroll 4
            for (int k = 0; k < chunks; ++k) {
                const float4 x = *reinterpret_cast<const float4*>(part + (int64_t)k * count * MP * MP + at);
                A[i] += f32x4{x.x, x.y, x.z, x.w};
            }
            A[i] *= by;
        }
    }
    auto put = [&](unsigned char* to, const f32x4 (&x)[kMine], float scale) {
#pragma unroll
        for (int i = 0; i < kMine; ++i)
            if (there[i]) {
                const int t = bt[i] * 16 + col;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int v = bv[i] * 16 + grp * 4 + e;
                    const float y = x[i][e] * scale;
                    const half_t h = (half_t)y, l = (half_t)((y - (float)h) * kLoScale);
                    if (t <= v) {
                        const int one = S::at(t, v >> 3) + (v & 7) * 2, other = S::at(v, t >> 3) + (t & 7) * 2;
                        *reinterpret_cast<half_t*>(to + one) = h;
                        *reinterpret_cast<half_t*>(to + S::kHalf + one) = l;
                        *reinterpret_cast<half_t*>(to + other) = h;
                        *reinterpret_cast<half_t*>(to + S::kHalf + other) = l;
                    }
                }
            }
        __syncthreads();
    };
    auto product = [&](const unsigned char* v_op, const unsigned char* t_op, f32x4 (&out)[kMine], float scale) {
#pragma unroll
        for (int i = 0; i < kMine; ++i)
            if (there[i]) {
                f32x4 acc = {}, cross = {};
                const int rt = bt[i] * 16 + col, rv = bv[i] * 16 + col;
#pragma unroll
                for (int k32 = 0; k32 < MP / 32; ++k32) {
                    const int piece = k32 * 4 + grp;
                    const half8 th = *reinterpret_cast<const half8*>(t_op + S::at(rt, piece)), tl = *reinterpret_cast<const half8*>(t_op + S::kHalf + S::at(rt, piece));
                    const half8 vh = *reinterpret_cast<const half8*>(v_op + S::at(rv, piece)), vl = *reinterpret_cast<const half8*>(v_op + S::kHalf + S::at(rv, piece));
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(vh, th, acc, 0, 0, 0);
                    cross = __builtin_amdgcn_mfma_f32_16x16x32_f16(vh, tl, cross, 0, 0, 0);
                    cross = __builtin_amdgcn_mfma_f32_16x16x32_f16(vl, th, cross, 0, 0, 0);
                }
                out[i] = (cross * (1.f / kLoScale) + acc) * scale;
            }
    };
    constexpr float kOff = kOffScale, kPoly = kPolyScale;
    put(U, A, kOff);
    for (int step = 0; step < steps; ++step) {
        product(U, U, M, 1.f / (kOff * kOff));                       // A A, of A = U
#pragma unroll
        for (int i = 0; i < kMine; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                M[i][e] = fmaf(c, M[i][e], fmaf(b, A[i][e], bt[i] * 16 + col == bv[i] * 16 + grp * 4 + e ? a : 0.f));
        const bool last = step + 1 == steps;
        if (!(last && step == 0)) put(V, M, kOff);
        if (!last) {
            f32x4 T[kMine];
            product(V, U, T, 1.f / (kOff * kOff));                   // M A
            __syncthreads();
            put(U, T, kOff);
            product(V, U, A, 1.f / (kOff * kOff));                   // M A M
            __syncthreads();
        }
        if (step == 0) {
#pragma unroll
            for (int i = 0; i < kMine; ++i) P[i] = M[i];
        } else {
            put(U, P, kPoly);
            product(V, U, P, 1.f / (kOff * kPoly));                  // M P
            __syncthreads();
        }
        if (!last) put(U, A, kOff);
    }
#pragma unroll
    for (int i = 0; i < kMine; ++i)
        if (there[i]) {
            const int t = bt[i] * 16 + col;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int v = bv[i] * 16 + grp * 4 + e;
                const float y = P[i][e] * kPoly;
                const half_t h = (half_t)y, l = (half_t)((y - (float)h) * kLoScale);
                if (t <= v) {
                    const int64_t one = ((int64_t)mat * MP + t) * MP + v, other = ((int64_t)mat * MP + v) * MP + t;
                    p_hi[one] = h;
                    p_lo[one] = l;
                    p_hi[other] = h;
                    p_lo[other] = l;
                }
            }
        }
}

// Whether A, M and P stay within what pairs of fp16 hold at their scales, whatever singular values X begins with, and a^steps, by which
// errors of A grow against the result's, within the ten bits that are there for it.  (The polynomials are smooth: 64 points, and a factor
// of four to spare.)
bool ns_gram_fits(int steps, float a, float b, float c) {
    if (steps < 1) return false;
    double growth = 1.0;
    for (int k = 0; k < steps; ++k) growth *= fabs((double)a);
    if (!(growth <= 1000.0)) return false;
    for (int i = 0; i <= 64; ++i) {
        double l = (double)i / 64.0, p = 1.0;
        for (int k = 0; k < steps; ++k) {
            const double m = (double)a + l * ((double)b + l * (double)c);
            p *= m;
            l *= m * m;
            if (!(fabs(p) <= 1000.0) || !(fabs(m) <= 250.0) || !(l <= 250.0)) return false;
        }
    }
    return true;
}

namespace {
struct GramLayout {
    int tiles, chunks;
    size_t part, m[2], p[2], a, t, total;            // pairs: hi, then lo
};
GramLayout gram_layout(int64_t count, int mp, int np) {
    GramLayout L;
    const int side = mp / kPairTile;
    L.tiles = side * (side + 1) / 2;
    // contractions are cut until there are two workgroups to a CU, each with four stages at least
    const int64_t all = (int64_t)L.tiles * count, stages = np / 64;
    L.chunks = (int)std::max<int64_t>(1, std::min<int64_t>(stages / 4, 512 / all));
    size_t o = 0;
    auto take = [&](size_t bytes) {
        const size_t at = o;
        o += round_up(bytes, 256);
        return at;
    };
    const size_t pair = (size_t)count * mp * mp * 4;
    L.part = take((size_t)L.chunks * count * mp * mp * 4);
    for (size_t* at : {&L.m[0], &L.m[1], &L.p[0], &L.p[1], &L.a, &L.t}) *at = take(pair);
    L.total = o;
    return L;
}
template <PairMode MODE>
int launch_pair(PairArgs& p, int problems, hipStream_t s) {
    hipLaunchKernelGGL(ns_pair_kernel<MODE>, dim3((unsigned)(p.tiles * p.chunks * p.count * problems)), dim3(kPairThreads), 2 * kPairStage, s, p);
    return launch_result();
}
template <int MP>
int launch_iterate(const PairArgs& p, half_t* p_hi, half_t* p_lo, hipStream_t s) {
    if (IterShape<MP>::kLds > 64 * 1024 && !allow_lds(reinterpret_cast<const void*>(ns_iterate_kernel<MP>), IterShape<MP>::kLds))
        return TPPO_ERR_LAUNCH;
    hipLaunchKernelGGL(ns_iterate_kernel<MP>, dim3((unsigned)p.count), dim3(kIterWaves * 64), IterShape<MP>::kLds, s, p.part, p.chunks, p.count,
                       p.scales, p.x.steps, p.x.a, p.x.b, p.x.c, p_hi, p_lo);
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
    p.problem[0] = {hi, lo, hi, lo, nullptr, nullptr, 1.f, 1.f};
    p.each_t = p.each_v = (int64_t)mp * np;
    p.ld_t = p.ld_v = np;
    p.tiles = L.tiles;
    p.stages = np / 64;
    p.chunks = L.chunks;
    if (launch_pair<kPairGram>(p, 1, s) != TPPO_OK) return TPPO_ERR_LAUNCH;
    half_t* P = pair(L.p[0]);
    float p_scale = kPolyScale;
    if (mp <= 128) {
        if ((mp == 64 ? launch_iterate<64>(p, P, P + half, s) : launch_iterate<128>(p, P, P + half, s)) != TPPO_OK) return TPPO_ERR_LAUNCH;
    } else {
        hipLaunchKernelGGL(ns_gather_kernel, dim3((unsigned)((each + 255) / 256), (unsigned)x.count), dim3(256), 0, s, p.part, p.chunks, p.count, mp,
                           scales, A, A + half);
        p.chunks = 1;
        p.stages = mp / 64;
        p.each_t = p.each_v = each;
        p.ld_t = p.ld_v = mp;
        const float off2 = 1.f / (kOffScale * kOffScale);
        for (int k = 0; k < x.steps; ++k) {
            half_t* M = pair(L.m[k & 1]);
            p.problem[0] = {A, A + half, A, A + half, M, M + half, off2, kOffScale};
            if (launch_pair<kPairPoly>(p, 1, s) != TPPO_OK) return TPPO_ERR_LAUNCH;
            const bool last = k + 1 == x.steps;
            int problems = 0;
            half_t* next = pair(L.p[k & 1]);
            if (!last) p.problem[problems++] = {M, M + half, A, A + half, T, T + half, off2, kOffScale};
            if (k > 0) p.problem[problems++] = {M, M + half, P, P + half, next, next + half, 1.f / (kOffScale * p_scale), kPolyScale};
            if (problems && launch_pair<kPairMul>(p, problems, s) != TPPO_OK) return TPPO_ERR_LAUNCH;
            if (!last) {
                p.problem[0] = {T, T + half, M, M + half, A, A + half, off2, kOffScale};
                if (launch_pair<kPairMul>(p, 1, s) != TPPO_OK) return TPPO_ERR_LAUNCH;
            }
            P = k == 0 ? M : next;
            p_scale = k == 0 ? kOffScale : kPolyScale;
        }
    }
    // X = P X
    p.problem[0] = {P, P + half, hi, lo, nullptr, nullptr, 1.f / p_scale, 1.f};
    p.each_t = each;
    p.ld_t = mp;
    p.each_v = (int64_t)mp * np;
    p.ld_v = np;
    p.tiles_t = mp / kPairTile;
    p.tiles_v = np / kPairTile;
    p.tiles = p.tiles_t * p.tiles_v;
    p.stages = mp / 64;
    p.chunks = 1;
    return launch_pair<kPairLast>(p, 1, s);
}

}  // namespace tppo
