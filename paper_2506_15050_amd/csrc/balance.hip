// tppo_balance_loss, tppo_balance_loss_backward: the auxiliary loss of a mixture-of-experts router over the policy tokens, per-expert
// counts, and the derivative with respect to the router's logits.
//     p = softmax(logits),  f_e = counts_e / (k N),  P_e = sum_m p[m, e] / N,  loss = coefficient E sum_e f_e P_e
//     d loss / d logits[m, i] = coefficient E / N * p_i (f_i - sum_e f_e p_e)
// The p of a row add up to one, so f may be taken from its mean over the experts, d_e = (counts_e - total / E) / (k N): an even use,
// where all f_e are alike, loses no digits to the difference.
// Bound by memory: every logit is read once and, backward, every derivative written once.
#include "rows.h"

namespace tppo {

constexpr int kBlThreads = 256, kBlWaves = kBlThreads / kWave;
constexpr int kBlMaxE = 2048, kBlMaxK = 1024;
constexpr int64_t kBlMaxChoices = (int64_t)1 << 36;  // a workgroup's share of the choices is counted in 32 bits
constexpr int kBlGroups = 512;                       // workgroups of the rows' kernel at most: rows of partial sums
constexpr int kBlCounters = 64;                      // workgroups of the counting kernel at most

// Combined over the lanes that differ in the bits kFrom .. kTo / 2 of their number, in every one of them.
template <int kFrom, int kTo, class Op>
__device__ __forceinline__ float over_lanes(float x, Op op) {
    if constexpr (kFrom <= 1 && kTo > 1) x = op(x, dpp_move<0xB1, 0xF>(x));            // lanes 1 0 3 2
    if constexpr (kFrom <= 2 && kTo > 2) x = op(x, dpp_move<0x4E, 0xF>(x));            // 2 3 0 1
    if constexpr (kFrom <= 4 && kTo > 4) {
        float other = dpp_move<0x141, 0xF>(x);                                          // mirrored in 8: enough where a quad's lanes are alike
        if constexpr (kFrom > 1) other = dpp_move<0x1B, 0xF>(other);                    // each quad turned round again
        x = op(x, other);
    }
    if constexpr (kFrom <= 8 && kTo > 8) x = op(x, dpp_move<0x128, 0xF>(x));           // rotated by 8 in 16
    if constexpr (kFrom <= 16 && kTo > 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    if constexpr (kFrom <= 32 && kTo > 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return x;
}
struct Sum {
    __device__ float operator()(float a, float b) const { return a + b; }
};
struct Max {
    __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

// What the kernels share: the call's arrays and sizes.
struct Balance {
    const void* logits;
    int64_t n_rows, ld;
    int E;
    const int32_t* experts;
    int64_t k, ld_experts;
    const int32_t* rows;
    int64_t M;
    const int64_t* m_actual;
    float coefficient, scale;
    const int64_t* counts_in;
    int64_t denominator;
    void* grad;
    int64_t ld_grad;
    const int32_t* out_index;
    int64_t n_out;
    float* loss;
    int64_t* counts;
    float* mean_prob;
    float* part_p;                                   // [groups][E]
    int32_t* part_counts;                            // [counters][E]
    int groups, counters;
    int32_t* status;
    __device__ int64_t tokens() const { return m_actual ? max(min(M, *m_actual), (int64_t)0) : M; }
};

// This workgroup's share of the choices, token by token, into `seen` (LDS, E words, cleared here).
__device__ __forceinline__ void count_choices(const Balance& b, int64_t m_eff, int share, int shares, int* seen) {
    for (int e = threadIdx.x; e < b.E; e += kBlThreads) seen[e] = 0;
    __syncthreads();
    const int64_t per = (m_eff + shares - 1) / shares, from = share * per, to = min(from + per, m_eff);
    const int k = (int)b.k;
    for (int64_t i = threadIdx.x; i < (to - from) * k; i += kBlThreads) {
        const int64_t m = from + i / k, row = b.rows ? (int64_t)b.rows[m] : m;
        if (row < 0 || row >= b.n_rows) {
            set_status(b.status, TPPO_STATUS_BAD_ROW);
            continue;
        }
        const int e = b.experts[row * b.ld_experts + i % k];
        if (e >= 0 && e < b.E) atomicAdd(seen + e, 1);
        else if (e != -1) set_status(b.status, TPPO_STATUS_BAD_TARGET);
    }
    __syncthreads();
}

__global__ __launch_bounds__(kBlThreads) void balance_count_kernel(Balance b) {
    __shared__ int seen[kBlMaxE];
    count_choices(b, b.tokens(), blockIdx.x, b.counters, seen);
    for (int e = threadIdx.x; e < b.E; e += kBlThreads) b.part_counts[(int64_t)blockIdx.x * b.E + e] = seen[e];
}

// kLanes lanes a row, kPieces pieces of 16 bytes for each.  GRAD: counts are there already, and derivatives are written; otherwise the
// workgroup counts its part of the choices as well.
template <class T, int kLanes, int kPieces, bool RAGGED, bool GRAD>
__global__ __launch_bounds__(kBlThreads) void balance_rows_kernel(Balance b) {
    constexpr int kN = Piece<T>::kN, kRows = kBlThreads / kLanes;
    constexpr int kCols = kLanes * kPieces * kN;
    __shared__ float columns[kCols * kBlWaves];
    __shared__ int seen[GRAD ? 1 : kBlMaxE];
    const int lane = threadIdx.x % kLanes, mine = threadIdx.x / kLanes, E = b.E;
    const int64_t m_eff = b.tokens();
    const int pieces = (E + kN - 1) / kN;
    float d[kPieces][kN], total[kPieces][kN];
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
#pragma unroll
        for (int e = 0; e < kN; ++e) d[i][e] = total[i][e] = 0.f;
    float up = 0.f;
    if constexpr (GRAD) {
        const double n = (double)(b.denominator > 0 ? b.denominator : m_eff), each = 1.0 / ((double)b.k * n);
        up = (float)((double)b.scale * b.coefficient * E / n);
        // all counts, and their sum
        double sum = 0.0;
        for (int e = threadIdx.x; e < E; e += kBlThreads) {
            int64_t c = 0;
            if (b.counts_in) c = b.counts_in[e];
            else
                for (int g = 0; g < b.counters; ++g) c += b.part_counts[(int64_t)g * E + e];
            columns[e] = (float)((double)c * each);
            sum += (double)c;
        }
        __shared__ double sums[kBlWaves];
        sum = wave_prefix(sum);
        if ((threadIdx.x & 63) == 63) sums[threadIdx.x >> 6] = sum;
        __syncthreads();
        sum = 0.0;
#pragma unroll
        for (int w = 0; w < kBlWaves; ++w) sum += sums[w];
        const float mean = (float)(sum * each / E);
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                const int at = (lane + i * kLanes) * kN + e;
                d[i][e] = at < E ? columns[at] - mean : 0.f;
            }
        __syncthreads();
    } else {
        count_choices(b, m_eff, blockIdx.x, b.groups, seen);
        for (int e = threadIdx.x; e < E; e += kBlThreads) b.part_counts[(int64_t)blockIdx.x * E + e] = seen[e];
    }
    for (int64_t m = (int64_t)blockIdx.x * kRows + mine; m < m_eff; m += (int64_t)b.groups * kRows) {
        const int64_t want = b.rows ? (int64_t)b.rows[m] : m;
        const bool bad = want < 0 || want >= b.n_rows;
        const T* src = static_cast<const T*>(b.logits) + (bad ? 0 : want) * b.ld;
        float z[kPieces][kN], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int c = lane + i * kLanes;
            Piece<T> p;
            if (c < pieces) p = piece_at<T, RAGGED>(src, c, E, -INFINITY);
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                z[i][e] = c < pieces ? p.get(e) : -INFINITY;
                top = fmaxf(top, z[i][e]);
            }
        }
        top = over_lanes<1, kLanes>(top, Max());
        if (top == -INFINITY) top = 0.f;                             // nothing to choose from: every exp is 0
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                z[i][e] = __builtin_amdgcn_exp2f((z[i][e] - top) * 1.4426950408889634f);
                sum += z[i][e];
            }
        sum = over_lanes<1, kLanes>(sum, Sum());
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        float mean = 0.f;
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                z[i][e] *= inv;
                if (!bad) total[i][e] += z[i][e];
                if constexpr (GRAD) mean = fmaf(z[i][e], d[i][e], mean);
            }
        if (bad && lane == 0) set_status(b.status, TPPO_STATUS_BAD_ROW);
        if constexpr (GRAD) {
            mean = over_lanes<1, kLanes>(mean, Sum());
            const float by = bad ? __builtin_nanf("") : up;
            const int64_t to = b.out_index ? (int64_t)b.out_index[m] : m;
            if (to < 0 || to >= b.n_out) {
                if (lane == 0) set_status(b.status, TPPO_STATUS_BAD_ROW);
                continue;
            }
            T* dst = static_cast<T*>(b.grad) + to * b.ld_grad;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int c = lane + i * kLanes;
                if (c < pieces) {
                    float out[kN];
#pragma unroll
                    for (int e = 0; e < kN; ++e) out[e] = by * z[i][e] * (d[i][e] - mean);
                    put_piece<T, kN, RAGGED>(dst, c, E, out);
                }
            }
        }
    }
    // the wavefront's rows, then the workgroup's
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
#pragma unroll
        for (int e = 0; e < kN; ++e) {
            const float t = over_lanes<kLanes, 64>(total[i][e], Sum());
            if ((threadIdx.x & 63) < kLanes) columns[(threadIdx.x >> 6) * kCols + (lane + i * kLanes) * kN + e] = t;
        }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += kBlThreads) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < kBlWaves; ++w) t += columns[w * kCols + e];
        b.part_p[(int64_t)blockIdx.x * E + e] = t;
    }
}

// Counts, mean probabilities and the loss from the partial sums: one workgroup, a column to a thread of each of its parts.
constexpr int kBlLast = 1024;
__global__ __launch_bounds__(kBlLast) void balance_finish_kernel(Balance b) {
    __shared__ double shares[kBlLast];
    __shared__ long long chosen[kBlLast];
    const int E = b.E;
    const int64_t m_eff = b.tokens();
    const double n = (double)(b.denominator > 0 ? b.denominator : m_eff);
    int width = 1;
    while (width < E && width < kBlLast) width *= 2;
    const int parts = kBlLast / width, part = threadIdx.x / width, at = threadIdx.x % width;
    double loss = 0.0;
    for (int e0 = 0; e0 < E; e0 += width) {
        const int e = e0 + at;
        double p = 0.0;
        long long c = 0;
        if (e < E) {
            for (int g = part; g < b.groups; g += parts) p += (double)b.part_p[(int64_t)g * E + e];
            for (int g = part; g < b.counters; g += parts) c += b.part_counts[(int64_t)g * E + e];
        }
        shares[threadIdx.x] = p;
        chosen[threadIdx.x] = c;
        __syncthreads();
        if (part == 0 && e < E) {
            for (int s = 1; s < parts; ++s) {
                p += shares[s * width + at];
                c += chosen[s * width + at];
            }
            p = n > 0.0 ? p / n : 0.0;
            if (b.counts) b.counts[e] = c;
            if (b.mean_prob) b.mean_prob[e] = (float)p;
            const double all = (double)(b.counts_in ? b.counts_in[e] : c);
            if (n > 0.0) loss += all / ((double)b.k * n) * p;
        }
        __syncthreads();
    }
    loss = wave_prefix(loss);
    if ((threadIdx.x & 63) == 63) shares[threadIdx.x >> 6] = loss;
    __syncthreads();
    if (threadIdx.x == 0 && b.loss) {
        double all = 0.0;
        for (int w = 0; w < kBlLast / kWave; ++w) all += shares[w];
        *b.loss = (float)((double)b.coefficient * E * all);
    }
}

template <class T, bool GRAD>
static void launch_rows(const Balance& b, hipStream_t s) {
    constexpr int kN = Piece<T>::kN;
    const int pieces = (b.E + kN - 1) / kN;
    auto go = [&](auto lanes, auto n) {
        constexpr int kLanes = decltype(lanes)::value, kPieces = decltype(n)::value;
        if (b.E % kN) hipLaunchKernelGGL((balance_rows_kernel<T, kLanes, kPieces, true, GRAD>), dim3(b.groups), dim3(kBlThreads), 0, s, b);
        else hipLaunchKernelGGL((balance_rows_kernel<T, kLanes, kPieces, false, GRAD>), dim3(b.groups), dim3(kBlThreads), 0, s, b);
    };
    typedef std::integral_constant<int, 1> One;
    typedef std::integral_constant<int, 64> Wave;
    if (pieces <= 4) go(std::integral_constant<int, 4>(), One());
    else if (pieces <= 8) go(std::integral_constant<int, 8>(), One());
    else if (pieces <= 16) go(std::integral_constant<int, 16>(), One());
    else if (pieces <= 32) go(std::integral_constant<int, 32>(), One());
    else if (pieces <= 64) go(Wave(), One());
    else if (pieces <= 128) go(Wave(), std::integral_constant<int, 2>());
    else if (pieces <= 256) go(Wave(), std::integral_constant<int, 4>());
    else if constexpr (kN == 4) go(Wave(), std::integral_constant<int, 8>());
}

// Workgroups of the rows' kernel: as many as have a row to each group of lanes, up to kBlGroups.
static int row_groups(int64_t M, int64_t E, int per_piece) {
    const int64_t pieces = (E + per_piece - 1) / per_piece;
    int64_t lanes = 4;
    while (lanes < pieces && lanes < 64) lanes *= 2;
    const int64_t rows = kBlThreads / lanes, want = (M + rows - 1) / rows;
    return (int)(want < 1 ? 1 : want < kBlGroups ? want : kBlGroups);
}

static int check(const Balance& b, tppo_dtype dt) {
    if (dt != TPPO_F32 && dt != TPPO_BF16) return TPPO_ERR_DTYPE;
    if (b.M < 0 || b.M > INT32_MAX || b.n_rows < 0 || b.E < 1 || b.E > kBlMaxE || b.k < 1 || b.k > kBlMaxK || b.ld < b.E ||
        b.ld_experts < b.k || b.M * b.k > kBlMaxChoices)
        return TPPO_ERR_SIZE;
    if (!(b.coefficient - b.coefficient == 0.f) || !(b.scale - b.scale == 0.f)) return TPPO_ERR_PARAM;
    if (b.M > 0) {
        if (b.n_rows == 0 || (!b.rows && b.M > b.n_rows)) return TPPO_ERR_SIZE;
        if (!b.logits || !b.experts) return TPPO_ERR_NULL;
    }
    const size_t size = dt == TPPO_F32 ? 4 : 2;
    if (!is_aligned(b.logits, size) || !is_aligned(b.grad, size) || !is_aligned(b.experts, 4)) return TPPO_ERR_PARAM;
    return TPPO_OK;
}

static size_t part_bytes(int64_t E, int rows) { return round_up((size_t)rows * E * 4, 256); }

// The launches of a call; `grad`: with derivatives.
static int run_balance(Balance& b, tppo_dtype dt, bool grad, void* workspace, size_t workspace_bytes, hipStream_t s) {
    if (!workspace || !is_aligned(workspace, 256) || workspace_bytes < tppo_balance_loss_workspace_bytes(b.M, b.E))
        return TPPO_ERR_WORKSPACE;
    b.groups = row_groups(b.M, b.E, dt == TPPO_F32 ? 4 : 8);
    b.part_p = static_cast<float*>(workspace);
    b.part_counts = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + part_bytes(b.E, kBlGroups));
    if (grad) {
        const int64_t want = (b.M * b.k + 4 * kBlThreads - 1) / (4 * kBlThreads);
        b.counters = (int)(want < 1 ? 1 : want < kBlCounters ? want : kBlCounters);
        hipLaunchKernelGGL(balance_count_kernel, dim3(b.counters), dim3(kBlThreads), 0, s, b);
        if (dt == TPPO_F32) launch_rows<float, true>(b, s);
        else launch_rows<uint16_t, true>(b, s);
    } else {
        b.counters = b.groups;
        if (dt == TPPO_F32) launch_rows<float, false>(b, s);
        else launch_rows<uint16_t, false>(b, s);
    }
    hipLaunchKernelGGL(balance_finish_kernel, dim3(1), dim3(kBlLast), 0, s, b);
    return launch_result();
}

}  // namespace tppo

extern "C" size_t tppo_balance_loss_workspace_bytes(int64_t M, int64_t E) {
    using namespace tppo;
    (void)M;
    if (E < 1 || E > kBlMaxE) return 256;
    return 2 * part_bytes(E, kBlGroups);
}

extern "C" int tppo_balance_loss(const void* logits, int64_t n_rows, int64_t E, int64_t ld, tppo_dtype dt, const int32_t* experts,
                                 int64_t k, int64_t ld_experts, const int32_t* rows, int64_t M, const int64_t* m_actual,
                                 float coefficient, float* loss, int64_t* counts, float* mean_prob, void* workspace,
                                 size_t workspace_bytes, int32_t* status, void* stream) {
    using namespace tppo;
    if (E > kBlMaxE || E < 1) return TPPO_ERR_SIZE;
    Balance b = {};
    b.logits = logits; b.n_rows = n_rows; b.ld = ld; b.E = (int)E;
    b.experts = experts; b.k = k; b.ld_experts = ld_experts;
    b.rows = rows; b.M = M; b.m_actual = m_actual; b.coefficient = coefficient;
    b.loss = loss; b.counts = counts; b.mean_prob = mean_prob; b.status = status;
    const int rc = check(b, dt);
    if (rc != TPPO_OK) return rc;
    if (!loss && !counts && !mean_prob) return TPPO_OK;
    return run_balance(b, dt, false, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

extern "C" int tppo_balance_loss_backward(const void* logits, int64_t n_rows, int64_t E, int64_t ld, tppo_dtype dt,
                                          const int32_t* experts, int64_t k, int64_t ld_experts, const int32_t* rows, int64_t M,
                                          const int64_t* m_actual, float coefficient, float scale, const int64_t* counts_in,
                                          int64_t token_denominator, void* grad_logits, int64_t ld_grad, const int32_t* out_index,
                                          int64_t n_out, float* loss, int64_t* counts, float* mean_prob, void* workspace,
                                          size_t workspace_bytes, int32_t* status, void* stream) {
    using namespace tppo;
    if (E > kBlMaxE || E < 1) return TPPO_ERR_SIZE;
    Balance b = {};
    b.logits = logits; b.n_rows = n_rows; b.ld = ld; b.E = (int)E;
    b.experts = experts; b.k = k; b.ld_experts = ld_experts;
    b.rows = rows; b.M = M; b.m_actual = m_actual; b.coefficient = coefficient; b.scale = scale;
    b.counts_in = counts_in; b.denominator = token_denominator;
    b.grad = grad_logits; b.ld_grad = ld_grad; b.out_index = out_index; b.n_out = n_out;
    b.loss = loss; b.counts = counts; b.mean_prob = mean_prob; b.status = status;
    const int rc = check(b, dt);
    if (rc != TPPO_OK) return rc;
    if (token_denominator < 0 || ld_grad < E || n_out < 0 || (!out_index && M > n_out)) return TPPO_ERR_SIZE;
    if (M > 0 && !grad_logits) return TPPO_ERR_NULL;
    return run_balance(b, dt, true, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}
