// tppo_layer_norm, tppo_layer_norm_backward: the trunk's last norm on the rows that the heads project, and its derivatives.
#include <algorithm>

#include "rows.h"

namespace tppo {

constexpr int kLnMaxH = 16384;
constexpr int kLnThreads = 256;
constexpr int64_t kLnMaxGroups = 1 << 20;

// Sum over the kLanes threads that share a row, of two numbers at once, in every one of them.  kLanes = 64: a wavefront, by data-parallel
// moves; more: a trip through LDS, in one of two places in turn, so that one barrier a sum is enough.
template <int kLanes>
__device__ __forceinline__ void row_sums(float& a, float& b, float2 (*place)[kLanes / kWave], int turn) {
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (kLanes > kWave) {
        constexpr int kWaves = kLanes / kWave;
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) place[turn][wave] = make_float2(a, b);
        __syncthreads();
        a = b = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float2 s = place[turn][w];
            a += s.x;
            b += s.y;
        }
    }
}

// Forward.  kLanes threads a row, kPieces pieces of 16 bytes for each, which stay in registers: the row is read once, the mean and then
// the sum of squared differences from it are taken from there (no difference of large numbers).
// Bound by memory: 77536 x 5120, bf16: 265 us, 6.0 TB/s, where a plain pass over as many streams reaches 6.2 to 6.4 (kept in the caches on
// the way, 275).  63 x 64: 3 us, the latency of a launch and two dependent loads.
template <class T, class W, int kLanes, int kPieces, bool RAGGED>
__global__ __launch_bounds__(kLnThreads) void layer_norm_kernel(
    const T* __restrict__ x, int64_t n_rows, int H, int64_t ld_x, const W* __restrict__ weight, const W* __restrict__ bias, float eps,
    const int32_t* __restrict__ rows, int64_t M, const int64_t* __restrict__ m_actual, T* __restrict__ y, int64_t ld_y,
    float* __restrict__ mean, float* __restrict__ rstd, int32_t* status) {
    constexpr int kN = Piece<T>::kN, kRowsAtOnce = kLnThreads / kLanes;
    __shared__ float2 place[2][kLanes / kWave];
    const int lane = threadIdx.x % kLanes, mine = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    const int64_t m_eff = m_actual ? min(M, *m_actual) : M;
    const int pieces = (H + kN - 1) / kN;
    const float each = 1.f / (float)H;
    auto is_own = [&](int i, int e) {
        const int c = lane + i * kLanes;
        return own<kN, RAGGED>(c, piece_start<kN, RAGGED>(c, H), e, H);
    };
    for (int64_t m = (int64_t)blockIdx.x * kRowsAtOnce + mine; m < m_eff; m += (int64_t)gridDim.x * kRowsAtOnce) {
        const int64_t want = rows ? (int64_t)rows[m] : m;
        const bool bad = want < 0 || want >= n_rows;
        const T* src = x + (bad ? 0 : want) * ld_x;
        Piece<T> p[kPieces];
        float sum = 0.f, none = 0.f;
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
            if (lane + i * kLanes < pieces) p[i] = piece_at<T, RAGGED, true>(src, piece_start<kN, RAGGED>(lane + i * kLanes, H), H);
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
            if (lane + i * kLanes < pieces)
#pragma unroll
                for (int e = 0; e < kN; ++e)
                    if (is_own(i, e)) sum += p[i].get(e);
        row_sums<kLanes>(sum, none, place, 0);
        const float mu = sum * each;
        float sq = 0.f;
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
            if (lane + i * kLanes < pieces)
#pragma unroll
                for (int e = 0; e < kN; ++e) {
                    const float d = p[i].get(e) - mu;
                    if (is_own(i, e)) sq = fmaf(d, d, sq);
                }
        row_sums<kLanes>(sq, none, place, 1);
        const float s = bad ? __builtin_nanf("") : 1.f / sqrtf(fmaf(sq, each, eps));
        T* dst = y + m * ld_y;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int c = lane + i * kLanes;
            if (c < pieces) {
                float w[kN], b[kN], out[kN];
                const int start = piece_start<kN, RAGGED>(c, H);
                get_piece<W, kN, RAGGED>(weight, start, H, w);
                if (bias) {
                    get_piece<W, kN, RAGGED>(bias, start, H, b);
                } else {
#pragma unroll
                    for (int e = 0; e < kN; ++e) b[e] = 0.f;
                }
#pragma unroll
                for (int e = 0; e < kN; ++e) out[e] = fmaf((p[i].get(e) - mu) * s, w[e], b[e]);
                put_piece<T, kN, RAGGED, true>(dst, start, H, out);
            }
        }
        if (lane == 0) {
            if (bad) set_status(status, TPPO_STATUS_BAD_ROW);
            if (mean) mean[m] = bad ? __builtin_nanf("") : mu;
            if (rstd) rstd[m] = s;
        }
    }
}

// Backward.  kLanes threads a row as above; the two sums of a row are taken together, and the next row is asked for before this one is
// worked on.  A thread's columns are the same in all of its rows, so it adds up their weights' derivatives in registers; the groups of a
// workgroup add theirs in LDS, and each workgroup leaves one row of partial sums, [2][H], which add_rows_kernel adds in a fixed order.
// Bound by memory: a call of 19384 x 5120, bf16 with fp32 grad_y: 152 us, 5.2 TB/s, 6 of them add_rows_kernel (without the next row asked for
// 187); 16416 x 1024, fp32: 45 us, 4.4 TB/s, 5 of them add_rows_kernel; 2513 x 1001, bf16: 13.5, two launches' latency.
// Wavefronts that a SIMD's 512 registers hold: a thread's weights and two sums for each of its columns, and two rows of both inputs.
template <class T, class G, int kPieces>
constexpr int backward_waves() {
    constexpr int kColumns = kPieces * Piece<T>::kN, kNeed = 3 * kColumns + 2 * kColumns * (int)(sizeof(T) + sizeof(G)) / 4 + 26;
    return 512 / kNeed < 1 ? 1 : 512 / kNeed < 4 ? 512 / kNeed : 4;
}
template <class T, class G, class O, int kLanes, int kPieces, bool RAGGED>
__global__ __launch_bounds__(kLanes < kLnThreads ? kLnThreads : kLanes, (backward_waves<T, G, kPieces>())) void layer_norm_backward_kernel(
    const G* __restrict__ grad_y, int64_t ld_gy, const T* __restrict__ x, int64_t n_rows, int H, int64_t ld_x,
    const void* __restrict__ weight, bool weight_f32, const float* __restrict__ mean, const float* __restrict__ rstd,
    const int32_t* __restrict__ rows, int64_t M, const int64_t* __restrict__ m_actual, O* __restrict__ grad_x, int64_t ld_gx,
    const int32_t* __restrict__ out_index, int64_t n_out, float* __restrict__ partial, int32_t* status) {
    constexpr int kThreads = kLanes < kLnThreads ? kLnThreads : kLanes;
    constexpr int kN = Piece<T>::kN, kRowsAtOnce = kThreads / kLanes, kQuads = kN / Piece<G>::kN;
    __shared__ float2 place[2][kLanes / kWave];
    __shared__ float gathered[kRowsAtOnce > 1 ? 2 * kLanes * kPieces * kN : 1];
    const int lane = threadIdx.x % kLanes, mine = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    const int64_t m_eff = m_actual ? min(M, *m_actual) : M, stride = (int64_t)gridDim.x * kRowsAtOnce;
    const int pieces = (H + kN - 1) / kN;
    const float each = 1.f / (float)H;
    auto there = [&](int i) { return lane + i * kLanes < pieces; };
    auto start = [&](int i) { return piece_start<kN, RAGGED>(lane + i * kLanes, H); };
    auto is_own = [&](int i, int e) { return own<kN, RAGGED>(lane + i * kLanes, start(i), e, H); };
    float w[kPieces][kN], gw[kPieces][kN], gb[kPieces][kN];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
#pragma unroll
        for (int e = 0; e < kN; ++e) w[i][e] = gw[i][e] = gb[i][e] = 0.f;
        if (there(i)) {
            if (sizeof(T) == 4 || weight_f32) get_piece<float, kN, RAGGED>(static_cast<const float*>(weight), start(i), H, w[i]);
            else if constexpr (sizeof(T) == 2) get_piece<uint16_t, kN, RAGGED>(static_cast<const uint16_t*>(weight), start(i), H, w[i]);
        }
    }
    struct Row {
        Piece<T> x[kPieces];
        Piece<G> g[kPieces][kQuads];
        float mu, s;
        bool bad;
    };
    auto index_of = [&](int64_t m) { return m < m_eff ? (rows ? (int64_t)rows[m] : m) : (int64_t)0; };
    auto fetch = [&](Row& r, int64_t m, int64_t want) {
        if (m >= m_eff) return;
        r.bad = want < 0 || want >= n_rows;
        const T* src = x + (r.bad ? 0 : want) * ld_x;
        const G* gsrc = grad_y + m * ld_gy;
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
            if (there(i)) {
                r.x[i] = piece_at<T, RAGGED, true>(src, start(i), H);
#pragma unroll
                for (int q = 0; q < kQuads; ++q) r.g[i][q] = piece_at<G, RAGGED, true>(gsrc, start(i) + q * Piece<G>::kN, H);
            }
        r.mu = mean[m];
        r.s = rstd[m];
    };
    int turn = 0;
    auto work = [&](const Row& r, int64_t m) {
        float c1 = 0.f, c2 = 0.f, s = r.s;
        auto gy = [&](int i, int e) { return r.g[i][e / Piece<G>::kN].get(e % Piece<G>::kN); };
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
            if (there(i) && !r.bad)
#pragma unroll
                for (int e = 0; e < kN; ++e) {
                    if (!is_own(i, e)) continue;
                    const float xh = (r.x[i].get(e) - r.mu) * s, g = gy(i, e) * w[i][e];
                    c1 += g;
                    c2 = fmaf(g, xh, c2);
                    gw[i][e] = fmaf(gy(i, e), xh, gw[i][e]);
                    gb[i][e] += gy(i, e);
                }
        row_sums<kLanes>(c1, c2, place, turn);
        turn ^= 1;
        if (r.bad) {
            s = __builtin_nanf("");
            if (lane == 0) set_status(status, TPPO_STATUS_BAD_ROW);
        }
        if (!grad_x) return;
        const int64_t to = out_index ? (int64_t)out_index[m] : m;
        if (to < 0 || to >= n_out) {
            if (lane == 0) set_status(status, TPPO_STATUS_BAD_ROW);
            return;
        }
        c1 *= each;
        c2 *= each;
        O* dst = grad_x + to * ld_gx;
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
            if (there(i)) {
                float out[kN];
#pragma unroll
                for (int e = 0; e < kN; ++e) {
                    const float xh = (r.x[i].get(e) - r.mu) * s;
                    out[e] = s * (fmaf(gy(i, e), w[i][e], -c1) - xh * c2);
                }
                put_piece<O, kN, RAGGED, true>(dst, start(i), H, out);
            }
    };
    int64_t m = (int64_t)blockIdx.x * kRowsAtOnce + mine;
    Row a, b;
    fetch(a, m, index_of(m));
    int64_t next = index_of(m + stride);
    for (; m < m_eff; m += 2 * stride) {
        fetch(b, m + stride, next);
        next = index_of(m + 2 * stride);
        work(a, m);
        if (m + stride >= m_eff) break;
        fetch(a, m + 2 * stride, next);
        next = index_of(m + 3 * stride);
        work(b, m + stride);
    }
    if (!partial) return;
    if constexpr (kRowsAtOnce > 1) {                                 // the groups, one after the other
        for (int k = 0; k < kRowsAtOnce; ++k) {
            if (mine == k)
#pragma unroll
                for (int i = 0; i < kPieces; ++i)
#pragma unroll
                    for (int e = 0; e < kN; ++e) {
                        float* at = gathered + 2 * ((i * kN + e) * kLanes + lane);
                        if (k > 0) {
                            gw[i][e] += at[0];
                            gb[i][e] += at[1];
                        }
                        at[0] = gw[i][e];
                        at[1] = gb[i][e];
                    }
            __syncthreads();
        }
        if (mine != kRowsAtOnce - 1) return;
    }
    float* to = partial + (int64_t)blockIdx.x * 2 * H;
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
        if (there(i)) {
            const int first = (lane + i * kLanes) * kN - start(i);
            put_piece<float, kN, RAGGED>(to, start(i), H, gw[i], first);
            put_piece<float, kN, RAGGED>(to + H, start(i), H, gb[i], first);
        }
}

// out[h] (+)= the sum of `count` rows' entry h: 64 columns a workgroup, four to a thread, its 64 rows of threads a 64th of the rows each,
// which are all asked for at once.  (A column to a thread, 16 parts of the rows: 512 rows of 2 x 5120 5.5 us.)
constexpr int kAddThreads = 1024, kAddColumns = 64, kAddParts = kAddThreads * 4 / kAddColumns;
__global__ __launch_bounds__(kAddThreads) void add_rows_kernel(const float* __restrict__ partial, int count, int H,
                                                               float* __restrict__ grad_weight, float* __restrict__ grad_bias,
                                                               int accumulate) {
    __shared__ float sums[kAddParts][kAddColumns + 4];
    const int at = (threadIdx.x & 15) * 4, part = threadIdx.x >> 4, h = blockIdx.x * kAddColumns + at;
    float* out = blockIdx.y ? grad_bias : grad_weight;
    if (!out) return;
    const float* from = partial + (blockIdx.y ? H : 0);
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    if (h < H)
#pragma unroll 8
        for (int r = part; r < count; r += kAddParts) {
            const Piece<float> x = piece_at<float, true>(from + (int64_t)r * 2 * H, h, H);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += x.get(e);
        }
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[part][at + e] = sum[e];
    __syncthreads();
    const int col = threadIdx.x & 63, share = threadIdx.x >> 6;      // 16 wavefronts add four parts each, the first one those
    float some = 0.f;
#pragma unroll
    for (int k = 0; k < kAddParts / 16; ++k) some += sums[share * (kAddParts / 16) + k][col];
    __syncthreads();
    sums[share][col] = some;
    __syncthreads();
    if (share == 0 && blockIdx.x * kAddColumns + col < H) {
        float all = 0.f;
#pragma unroll
        for (int k = 0; k < 16; ++k) all += sums[k][col];
        float* to = out + blockIdx.x * kAddColumns + col;
        *to = accumulate ? *to + all : all;
    }
}

// Workgroups of the backward kernel: as many as the chip holds at once, of no fewer than four rows each, and of two turns where a turn is a row to
// each of four wavefronts and there are more than 384 (a row of partial sums is written and read again for each workgroup, as much as one and a
// half to two rows are); and no more than take the same number of turns.  us, a call, one turn / two:  1001, bf16, 1025 rows: 11.0 / 11.4, 2048: 13.7 / 12.7,
// 4096: 19.8 / 15.7;  1024, fp32, 1025: 9.6 / 11.0, 2048: 11.2 / 11.3, 4096: 19.4 / 14.3;  four turns of a workgroup a row / three:  5120, bf16, 2513:
// 35.6 / 43.8.  512 workgroups whatever the size / so:  20000 x 3584, bf16: 112 / 90;  16416 x 1024, fp32: 51 / 46.
constexpr int64_t kLnPartials = 1024;
static int64_t backward_groups(int64_t M, int rows_at_once, int resident) {
    const int64_t few = rows_at_once > 1 ? 384 : 256, least = rows_at_once > 1 ? 2 * rows_at_once : 4;
    const int64_t most = std::min<int64_t>({kLnPartials, (int64_t)256 * resident, std::max<int64_t>(few, (M + least - 1) / least)});
    const int64_t groups = (M + rows_at_once - 1) / rows_at_once, turns = (groups + most - 1) / most;
    return (groups + turns - 1) / turns;
}

}  // namespace tppo

extern "C" int tppo_layer_norm(const void* x, int64_t n_rows, int64_t H, int64_t ld_x, tppo_dtype dt, const void* weight,
                               const void* bias, tppo_dtype dt_w, float eps, const int32_t* rows, int64_t M,
                               const int64_t* m_actual, void* y, int64_t ld_y, float* mean, float* rstd, int32_t* status,
                               void* stream) {
    using namespace tppo;
    for (tppo_dtype t : {dt, dt_w})
        if (t != TPPO_F32 && t != TPPO_BF16) return TPPO_ERR_DTYPE;
    if (dt == TPPO_F32 && dt_w != TPPO_F32) return TPPO_ERR_DTYPE;
    if (M < 0 || n_rows < 0 || H < 1 || H > kLnMaxH || ld_x < H || ld_y < H) return TPPO_ERR_SIZE;
    if (!(eps >= 0.f) || eps > 3.4e38f) return TPPO_ERR_PARAM;
    if (M == 0) return TPPO_OK;
    if (n_rows == 0 || (!rows && M > n_rows)) return TPPO_ERR_SIZE;
    if (!x || !weight || !y) return TPPO_ERR_NULL;
    const size_t size = dt == TPPO_F32 ? 4 : 2, size_w = dt_w == TPPO_F32 ? 4 : 2;
    if (!is_aligned(x, size) || !is_aligned(y, size) || !is_aligned(weight, size_w) || (bias && !is_aligned(bias, size_w)) ||
        !is_aligned(mean, 4) || !is_aligned(rstd, 4))
        return TPPO_ERR_PARAM;
    auto launch = [&](auto t, auto w, auto lanes, auto pieces, auto ragged) {
        typedef decltype(t) T;
        typedef decltype(w) W;
        constexpr int kLanes = decltype(lanes)::value, kPieces = decltype(pieces)::value;
        constexpr int64_t kRowsAtOnce = kLnThreads / kLanes;
        const int64_t want = (M + kRowsAtOnce - 1) / kRowsAtOnce;
        hipLaunchKernelGGL((layer_norm_kernel<T, W, kLanes, kPieces, decltype(ragged)::value>),
                           dim3((unsigned)(want < kLnMaxGroups ? want : kLnMaxGroups)), dim3(kLnThreads), 0,
                           static_cast<hipStream_t>(stream), static_cast<const T*>(x), n_rows, (int)H, ld_x,
                           static_cast<const W*>(weight), static_cast<const W*>(bias), eps, rows, M, m_actual, static_cast<T*>(y), ld_y,
                           mean, rstd, status);
    };
    auto typed = [&](auto t, auto w) {
        constexpr int kN = Piece<decltype(t)>::kN;
        const int pieces = (int)((H + kN - 1) / kN);
        auto sized = [&](auto ragged) {
            auto go = [&](auto lanes, auto k) { launch(t, w, lanes, k, ragged); };
            typedef std::integral_constant<int, 64> L64;
            typedef std::integral_constant<int, 256> L256;
            if (pieces <= 64) go(L64(), std::integral_constant<int, 1>());
            else if (pieces <= 128) go(L64(), std::integral_constant<int, 2>());
            else if (pieces <= 256) go(L64(), std::integral_constant<int, 4>());
            else if (pieces <= 512) go(L256(), std::integral_constant<int, 2>());
            else if (pieces <= 768) go(L256(), std::integral_constant<int, 3>());
            else if (pieces <= 1024) go(L256(), std::integral_constant<int, 4>());
            else if (pieces <= 2048) go(L256(), std::integral_constant<int, 8>());
            else if constexpr (kN == 4) go(L256(), std::integral_constant<int, 16>());      // (fp32 beyond 8192)
        };
        if (H % kN) sized(std::true_type());
        else sized(std::false_type());
    };
    if (dt == TPPO_F32) typed(float(), float());
    else if (dt_w == TPPO_F32) typed(uint16_t(), float());
    else typed(uint16_t(), uint16_t());
    return launch_result();
}

extern "C" size_t tppo_layer_norm_backward_workspace_bytes(int64_t M, int64_t H) {
    using namespace tppo;
    if (M <= 0 || H <= 0 || H > kLnMaxH) return 256;
    return round_up((size_t)std::min(M, kLnPartials) * 2 * H * sizeof(float), 256);
}

extern "C" int tppo_layer_norm_backward(const void* grad_y, int64_t ld_gy, tppo_dtype dt_gy, const void* x, int64_t n_rows, int64_t H,
                                        int64_t ld_x, tppo_dtype dt, const void* weight, tppo_dtype dt_w, const float* mean,
                                        const float* rstd, const int32_t* rows, int64_t M, const int64_t* m_actual, void* grad_x,
                                        int64_t ld_gx, tppo_dtype dt_gx, const int32_t* out_index, int64_t n_out, float* grad_weight,
                                        float* grad_bias, int32_t accumulate_w, void* workspace, size_t workspace_bytes,
                                        int32_t* status, void* stream) {
    using namespace tppo;
    for (tppo_dtype t : {dt, dt_w, dt_gy, dt_gx})
        if (t != TPPO_F32 && t != TPPO_BF16) return TPPO_ERR_DTYPE;
    if (dt == TPPO_F32 && (dt_gy != TPPO_F32 || dt_w != TPPO_F32 || (grad_x && dt_gx != TPPO_F32))) return TPPO_ERR_DTYPE;
    if (M < 0 || n_rows < 0 || H < 1 || H > kLnMaxH || ld_x < H || ld_gy < H || (grad_x && (ld_gx < H || n_out < 0))) return TPPO_ERR_SIZE;
    if (!grad_x && !grad_weight && !grad_bias) return TPPO_OK;
    const bool sums = grad_weight || grad_bias;
    if (M > 0) {
        if (n_rows == 0 || (!rows && M > n_rows) || (grad_x && !out_index && M > n_out)) return TPPO_ERR_SIZE;
        if (!grad_y || !x || !weight || !mean || !rstd) return TPPO_ERR_NULL;
        auto size = [](tppo_dtype t) { return t == TPPO_F32 ? (size_t)4 : (size_t)2; };
        if (!is_aligned(x, size(dt)) || !is_aligned(grad_y, size(dt_gy)) || !is_aligned(weight, size(dt_w)) || !is_aligned(mean, 4) ||
            !is_aligned(rstd, 4) || (grad_x && !is_aligned(grad_x, size(dt_gx))))
            return TPPO_ERR_PARAM;
    }
    if (!is_aligned(grad_weight, 4) || !is_aligned(grad_bias, 4)) return TPPO_ERR_PARAM;
    if (M > 0 && sums && (!workspace || !is_aligned(workspace, 256) || workspace_bytes < tppo_layer_norm_backward_workspace_bytes(M, H)))
        return TPPO_ERR_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    float* partial = sums ? static_cast<float*>(workspace) : nullptr;
    int64_t groups = 0;
    auto launch = [&](auto t, auto g, auto o, auto lanes, auto pieces, auto ragged) {
        typedef decltype(t) T;
        typedef decltype(g) G;
        typedef decltype(o) O;
        constexpr int kLanes = decltype(lanes)::value, kPieces = decltype(pieces)::value;
        constexpr int kThreads = kLanes < kLnThreads ? kLnThreads : kLanes;
        groups = backward_groups(M, kThreads / kLanes, std::max(1, backward_waves<T, G, kPieces>() * 4 * kWave / kThreads));
        hipLaunchKernelGGL((layer_norm_backward_kernel<T, G, O, kLanes, kPieces, decltype(ragged)::value>), dim3((unsigned)groups),
                           dim3(kThreads), 0, s, static_cast<const G*>(grad_y), ld_gy,
                           static_cast<const T*>(x), n_rows, (int)H, ld_x, weight, dt_w == TPPO_F32, mean, rstd, rows, M, m_actual,
                           static_cast<O*>(grad_x), ld_gx, out_index, n_out, partial, status);
    };
    auto typed = [&](auto t, auto g, auto o) {
        constexpr int kN = Piece<decltype(t)>::kN;
        const int pieces = (int)((H + kN - 1) / kN);
        auto sized = [&](auto ragged) {
            auto go = [&](auto lanes, auto k) { launch(t, g, o, lanes, k, ragged); };
            typedef std::integral_constant<int, 64> L64;
            typedef std::integral_constant<int, 256> L256;
            typedef std::integral_constant<int, 512> L512;
            if (pieces <= 64) go(L64(), std::integral_constant<int, 1>());
            else if (pieces <= 128) go(L64(), std::integral_constant<int, 2>());
            else if (pieces <= 256) go(L64(), std::integral_constant<int, 4>());
            else if (pieces <= 512) go(L256(), std::integral_constant<int, 2>());
            else if (pieces <= 768) go(L256(), std::integral_constant<int, 3>());
            else if (pieces <= 1024) go(L256(), std::integral_constant<int, 4>());
            else if (pieces <= 2048) go(L512(), std::integral_constant<int, 4>());
            else if constexpr (kN == 4) go(L512(), std::integral_constant<int, 8>());
        };
        if (H % kN) sized(std::true_type());
        else sized(std::false_type());
    };
    if (M > 0) {
        if (dt == TPPO_F32) typed(float(), float(), float());
        else if (dt_gy == TPPO_F32 && dt_gx == TPPO_F32) typed(uint16_t(), float(), float());
        else if (dt_gy == TPPO_F32) typed(uint16_t(), float(), uint16_t());
        else if (dt_gx == TPPO_F32) typed(uint16_t(), uint16_t(), float());
        else typed(uint16_t(), uint16_t(), uint16_t());
        if (hipGetLastError() != hipSuccess) return TPPO_ERR_LAUNCH;
    }
    if (sums && (M > 0 || !accumulate_w))
        hipLaunchKernelGGL(add_rows_kernel, dim3((unsigned)((H + kAddColumns - 1) / kAddColumns), 2), dim3(kAddThreads), 0, s, partial,
                           (int)groups, (int)H, grad_weight, grad_bias, accumulate_w);
    return launch_result();
}
