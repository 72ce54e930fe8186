// tppo_balance_loss, tppo_balance_loss_backward: the auxiliary loss of a mixture-of-experts router over the policy tokens, per-expert
// counts, and the derivative with respect to the router's logits.
//     p = softmax(logits),  f_e = counts_e / (k N),  P_e = sum_m p[m, e] / N,  loss = coefficient E sum_e f_e P_e
//     d loss / d logits[m, i] = coefficient E / N * p_i (f_i - sum_e f_e p_e)
// The p of a row add up to one, so f may be taken from its mean over the experts, d_e = (counts_e - total / E) / (k N): an even use,
// where all f_e are alike, loses no digits to the difference.
// Bound by memory: every logit is read once and, backward, every derivative written once; and by two or three launches that wait for each
// other, 10 to 16 us whatever the size.  Backward of 77536 x 128, fp32: 30 us, of which the choices 6.5, the rows 17 (4.7 TB/s) and the
// finishing kernel 5;  2000 x 128: 16;  forward of 77536 x 256: 24.5, rows and choices 17, finishing 5.5;  146 x 8, all in one launch: 4.
#include "rows.h"

namespace tppo {

constexpr int kBlThreads = 512, kBlWaves = kBlThreads / kWave;
constexpr int kBlMaxE = 2048, kBlMaxK = 1024;
constexpr int64_t kBlMaxChoices = (int64_t)1 << 36;  // a workgroup's share of the choices is counted in 32 bits
constexpr int kBlGroups = 512;                       // workgroups of the rows' kernel at most: rows of partial sums
constexpr int kBlCounters = 128;                     // workgroups of the counting kernel at most

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
    double* part_loss;                               // by workgroup of the finishing kernel
    int32_t* arrived;                                // how many of those are done; cleared by the kernel before
    int groups, counters;
    int32_t* status;
    __device__ int64_t tokens() const { return m_actual ? max(min(M, *m_actual), (int64_t)0) : M; }
    __device__ double n_tokens(int64_t m_eff) const { return (double)(denominator > 0 ? denominator : m_eff); }
};

// This workgroup's share of the choices, a token to a thread and eight of its choices at a time, into `seen` (LDS, E words, cleared here).
// (A choice to a thread looked up its row for each and waited for both loads in turn: 620 000 choices 10.9 us.)
__device__ __forceinline__ void count_choices(const Balance& b, int64_t m_eff, int share, int shares, int* seen) {
    for (int e = threadIdx.x; e < b.E; e += blockDim.x) seen[e] = 0;
    __syncthreads();
    const int64_t per = (m_eff + shares - 1) / shares, from = share * per, to = min(from + per, m_eff);
    const int k = (int)b.k;
    int wrong = 0;
    for (int64_t m = from + threadIdx.x; m < to; m += blockDim.x) {
        const int64_t row = b.rows ? (int64_t)b.rows[m] : m;
        if (row < 0 || row >= b.n_rows) {
            wrong |= TPPO_STATUS_BAD_ROW;
            continue;
        }
        const int32_t* ids = b.experts + row * b.ld_experts;
        for (int j0 = 0; j0 < k; j0 += 8) {
            int e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = j0 + j < k ? ids[j0 + j] : -1;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (e[j] >= 0 && e[j] < b.E) atomicAdd(seen + e[j], 1);
                else if (e[j] != -1) wrong |= TPPO_STATUS_BAD_TARGET;
            }
        }
    }
    if (wrong) set_status(b.status, wrong);
    __syncthreads();
}

constexpr int kBlCountThreads = 1024;
__global__ __launch_bounds__(kBlCountThreads) void balance_count_kernel(Balance b) {
    __shared__ int seen[kBlMaxE];
    count_choices(b, b.tokens(), blockIdx.x, b.counters, seen);
    for (int e = threadIdx.x; e < b.E; e += kBlCountThreads) b.part_counts[(int64_t)blockIdx.x * b.E + e] = seen[e];
}

// A sum over the workgroup, in every thread (kBlThreads of them).
__device__ __forceinline__ double workgroup_sum(double x, double* place) {
    x = wave_prefix(x);
    if ((threadIdx.x & 63) == 63) place[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0;
#pragma unroll
    for (int w = 0; w < kBlWaves; ++w) x += place[w];
    __syncthreads();
    return x;
}

// kLanes lanes a row, kPieces pieces of 16 bytes for each, kAtOnce rows under way.  GRAD: derivatives are written, from counts that are
// there already; otherwise the workgroup counts its part of the choices as well (by workgroups of their own in the same launch: 77536 x 256
// 24.5 -> 28 us).  ONE: a single workgroup, which does all of the call.  Asking for a turn's rows before the one before is worked on gained
// nothing at 22 sizes: there are workgroups enough to cover for each other.
// Sums over a row are log2(kLanes) steps for 64 / kLanes rows side by side, so lanes are few and have several pieces as long as registers
// for the columns' sums and counts (2 kPieces kN) are no matter.
template <class T, int kLanes, int kPieces, bool RAGGED, bool GRAD, bool ONE>
__global__ __launch_bounds__(kBlThreads) void balance_rows_kernel(Balance b) {
    constexpr int kN = Piece<T>::kN, kRows = kBlThreads / kLanes, kAtOnce = kPieces * kN <= 16 ? 2 : 1;
    constexpr int kCols = kLanes * kPieces * kN;
    // the columns' sums wavefront by wavefront (in two turns where that is much)
    constexpr int kTurns = kCols * kBlWaves * 4 > 32768 ? 2 : 1, kPlaces = kBlWaves / kTurns;
    __shared__ __attribute__((aligned(8))) float columns[kCols * kPlaces > kBlMaxE ? kCols * kPlaces : kBlMaxE];
    static_assert(kBlThreads * sizeof(long long) <= sizeof(columns) && kCols * sizeof(long long) <= sizeof(columns), "all counts, or a part to a thread");
    __shared__ int seen[GRAD && !ONE ? 1 : kBlMaxE];
    __shared__ double sums[kBlWaves];
    const int lane = threadIdx.x % kLanes, mine = threadIdx.x / kLanes, E = b.E;
    const int64_t m_eff = b.tokens();
    const int pieces = (E + kN - 1) / kN;
    if (!ONE && blockIdx.x == 0 && threadIdx.x == 0) *b.arrived = 0;
    int starts[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) starts[i] = piece_start<kN, RAGGED>(lane + i * kLanes, E);
    float d[kPieces][kN], total[kPieces][kN];
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
#pragma unroll
        for (int e = 0; e < kN; ++e) d[i][e] = total[i][e] = 0.f;
    float up = 0.f;
    if constexpr (!GRAD || ONE) {
        count_choices(b, m_eff, blockIdx.x, b.groups, seen);
        if constexpr (!ONE)
            for (int e = threadIdx.x; e < E; e += kBlThreads) b.part_counts[(int64_t)blockIdx.x * E + e] = seen[e];
    }
    if constexpr (GRAD) {
        const double n = b.n_tokens(m_eff), each = 1.0 / ((double)b.k * n);
        up = (float)((double)b.scale * b.coefficient * E / n);
        // all counts, and their sum: a column to a thread, or its parts to several.  (A workgroup's counts are 32 bits, all of them together are
        // not; and they stay whole until their mean is known: rounded before that, counts of 3 x 10^7 one apart gave d wrong by 4 %.)
        long long* whole = reinterpret_cast<long long*>(columns);
        double sum = 0.0;
        if (b.counts_in || ONE) {
            for (int e = threadIdx.x; e < E; e += kBlThreads) {
                const long long c = b.counts_in ? (long long)b.counts_in[e] : (long long)seen[e];
                whole[e] = c;
                sum += (double)c;
            }
        } else {
            long long* parts = whole;
            const int width = E <= 64 ? 64 : E <= 128 ? 128 : E <= 256 ? 256 : kBlThreads, shares = kBlThreads / width;
            const int at = threadIdx.x % width, share = threadIdx.x / width;
            for (int e0 = 0; e0 < E; e0 += width) {
                long long c = 0;
                if (e0 + at < E)
#pragma unroll 16
                    for (int g = share; g < b.counters; g += shares) c += b.part_counts[(int64_t)g * E + e0 + at];
                if (shares > 1) {                                    // (then this is the only turn)
                    parts[threadIdx.x] = c;
                    __syncthreads();
                    if (share == 0)
                        for (int w = 1; w < shares; ++w) c += parts[w * width + at];
                    __syncthreads();
                }
                if (share == 0 && e0 + at < E) {
                    whole[e0 + at] = c;
                    sum += (double)c;
                }
            }
        }
        sum = workgroup_sum(sum, sums);
        const double mean = sum / E;
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                const int at = starts[i] + e;
                d[i][e] = lane + i * kLanes < pieces && at < E ? (float)(((double)whole[at] - mean) * each) : 0.f;
            }
        __syncthreads();
    }
    const int64_t stride = (int64_t)b.groups * kRows;
    for (int64_t m0 = (int64_t)blockIdx.x * kRows + mine; m0 < m_eff; m0 += stride * kAtOnce) {
        Piece<T> p[kAtOnce][kPieces];
        bool bad[kAtOnce];
#pragma unroll
        for (int a = 0; a < kAtOnce; ++a) {
            const int64_t m = min(m0 + a * stride, m_eff - 1);      // (beyond the end: the last one again, not used)
            const int64_t want = b.rows ? (int64_t)b.rows[m] : m;
            bad[a] = want < 0 || want >= b.n_rows;
            const T* src = static_cast<const T*>(b.logits) + (bad[a] ? 0 : want) * b.ld;
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                if (lane + i * kLanes < pieces) p[a][i] = piece_at<T, RAGGED>(src, starts[i], E);
        }
#pragma unroll
        for (int a = 0; a < kAtOnce; ++a) {
            const int64_t m = m0 + a * stride;
            if (m >= m_eff) break;
            float z[kPieces][kN], top = -INFINITY;
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
#pragma unroll
                for (int e = 0; e < kN; ++e) {
                    z[i][e] = lane + i * kLanes < pieces && own<kN, RAGGED>(lane + i * kLanes, starts[i], e, E) ? p[a][i].get(e) : -INFINITY;
                    top = fmaxf(top, z[i][e]);
                }
            top = over_lanes<1, kLanes>(top, Max());
            if (top == -INFINITY) top = 0.f;                         // nothing to choose from: every exp is 0
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
#pragma unroll
                for (int e = 0; e < kN; ++e) {
                    // (the product is rounded, half a step for each unit of distance from the top, of a p that is e to the minus that)
                    z[i][e] = __builtin_amdgcn_exp2f((z[i][e] - top) * 1.4426950408889634f);
                    sum += z[i][e];
                }
            sum = over_lanes<1, kLanes>(sum, Sum());
            const float inv = sum == 0.f || bad[a] ? 0.f : 1.f / sum;
            float mean = 0.f;
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
#pragma unroll
                for (int e = 0; e < kN; ++e) {
                    if (bad[a]) z[i][e] = 0.f;                       // (whatever row 0 holds)
                    z[i][e] *= inv;
                    total[i][e] += z[i][e];
                    if constexpr (GRAD) mean = fmaf(z[i][e], d[i][e], mean);
                }
            if (bad[a] && lane == 0) set_status(b.status, TPPO_STATUS_BAD_ROW);
            if constexpr (GRAD) {
                mean = over_lanes<1, kLanes>(mean, Sum());
                const float by = bad[a] ? __builtin_nanf("") : up;
                const int64_t to = b.out_index ? (int64_t)b.out_index[m] : m;
                if (to < 0 || to >= b.n_out) {
                    if (lane == 0) set_status(b.status, TPPO_STATUS_BAD_ROW);
                } else {
                    T* dst = static_cast<T*>(b.grad) + to * b.ld_grad;
#pragma unroll
                    for (int i = 0; i < kPieces; ++i) {
                        const int c = lane + i * kLanes;
                        if (c < pieces) {
                            float out[kN];
#pragma unroll
                            for (int e = 0; e < kN; ++e) out[e] = by * z[i][e] * (d[i][e] - mean);
                            put_piece<T, kN, RAGGED>(dst, starts[i], E, out, c * kN - starts[i]);
                        }
                    }
                }
            }
        }
    }
    // the wavefront's rows, then the workgroup's
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
#pragma unroll
        for (int e = 0; e < kN; ++e) total[i][e] = over_lanes<kLanes, 64>(total[i][e], Sum());
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int turn = kTurns - 1; turn >= 0; --turn) {                 // (the second half of the wavefronts first, then added to the first)
        if (wave / kPlaces == turn && (threadIdx.x & 63) < kLanes)
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
#pragma unroll
                for (int e = 0; e < kN; ++e) {
                    if (lane + i * kLanes >= pieces || !own<kN, RAGGED>(lane + i * kLanes, starts[i], e, E)) continue;
                    float* at = columns + (wave % kPlaces) * kCols + starts[i] + e;
                    *at = turn + 1 < kTurns ? *at + total[i][e] : total[i][e];
                }
        __syncthreads();
    }
    double loss = 0.0;
    const double n = b.n_tokens(m_eff);
    for (int e = threadIdx.x; e < E; e += kBlThreads) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < kPlaces; ++w) t += columns[w * kCols + e];
        if constexpr (ONE) {
            const double q = n > 0.0 ? (double)t / n : 0.0;
            if (b.counts) b.counts[e] = seen[e];
            if (b.mean_prob) b.mean_prob[e] = (float)q;
            if (n > 0.0) loss += (double)(b.counts_in ? b.counts_in[e] : (int64_t)seen[e]) / ((double)b.k * n) * q;
        } else {
            b.part_p[(int64_t)blockIdx.x * E + e] = t;
        }
    }
    if constexpr (ONE) {
        loss = workgroup_sum(loss, sums);
        if (threadIdx.x == 0 && b.loss) *b.loss = (float)((double)b.coefficient * E * loss);
    }
}

// Counts, mean probabilities and the loss from the partial sums: kBlColumns columns a workgroup, 32 threads to each.  The last workgroup to
// end adds up the losses of all, in their order.
constexpr int kBlLast = 1024, kBlColumns = 32, kBlShares = kBlLast / kBlColumns;
__global__ __launch_bounds__(kBlLast) void balance_finish_kernel(Balance b) {
    __shared__ double shares[kBlShares][kBlColumns + 1];
    __shared__ long long chosen[kBlShares][kBlColumns + 1];
    const int E = b.E, at = threadIdx.x % kBlColumns, share = threadIdx.x / kBlColumns, e = blockIdx.x * kBlColumns + at;
    double p = 0.0;
    long long c = 0;
    if (e < E) {
#pragma unroll 16
        for (int g = share; g < b.groups; g += kBlShares) p += (double)b.part_p[(int64_t)g * E + e];
#pragma unroll 16
        for (int g = share; g < b.counters; g += kBlShares) c += b.part_counts[(int64_t)g * E + e];
    }
    shares[share][at] = p;
    chosen[share][at] = c;
    __syncthreads();
    if (threadIdx.x >= kWave) return;
    double loss = 0.0;
    if (threadIdx.x < kBlColumns && e < E) {
        const double n = b.n_tokens(b.tokens());
#pragma unroll 8
        for (int s = 1; s < kBlShares; ++s) {
            p += shares[s][at];
            c += chosen[s][at];
        }
        p = n > 0.0 ? p / n : 0.0;
        if (b.counts) b.counts[e] = c;
        if (b.mean_prob) b.mean_prob[e] = (float)p;
        if (n > 0.0) loss = (double)(b.counts_in ? b.counts_in[e] : (int64_t)c) / ((double)b.k * n) * p;
    }
    loss = wave_prefix(loss);
    if (!b.loss) return;
    int last = 0;
    if (threadIdx.x == kWave - 1) {
        __hip_atomic_store(b.part_loss + blockIdx.x, loss, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __threadfence();
        last = atomicAdd(b.arrived, 1) + 1 == (int)gridDim.x;
    }
    if (__builtin_amdgcn_readlane(last, kWave - 1)) {
        __threadfence();
        static_assert(kBlMaxE / kBlColumns <= kWave, "a workgroup's loss to a lane");
        double all = threadIdx.x < gridDim.x ? __hip_atomic_load(b.part_loss + threadIdx.x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
        all = wave_prefix(all);
        if (threadIdx.x == kWave - 1) *b.loss = (float)((double)b.coefficient * E * all);
    }
}

// Lanes of a row for so many pieces: 4, 8 or 16, and 64 beyond 64 pieces.
static int lanes_of(int64_t pieces) { return pieces <= 4 ? 4 : pieces <= 8 ? 8 : pieces <= 64 ? 16 : 64; }
static int pieces_of_lane(int64_t pieces) {          // rounded up to a power of two, as launch_rows has them
    const int64_t each = (pieces + lanes_of(pieces) - 1) / lanes_of(pieces);
    return each <= 1 ? 1 : each <= 2 ? 2 : each <= 4 ? 4 : 8;
}

template <class T, bool GRAD>
static void launch_rows(const Balance& b, hipStream_t s) {
    constexpr int kN = Piece<T>::kN;
    const int pieces = (b.E + kN - 1) / kN;
    auto go = [&](auto lanes, auto n) {
        constexpr int kLanes = decltype(lanes)::value, kPieces = decltype(n)::value;
        auto launch = [&](auto ragged, auto one) {
            hipLaunchKernelGGL((balance_rows_kernel<T, kLanes, kPieces, decltype(ragged)::value, GRAD, decltype(one)::value>), dim3(b.groups),
                               dim3(kBlThreads), 0, s, b);
        };
        auto sized = [&](auto ragged) {
            if (b.groups == 1) launch(ragged, std::true_type());
            else launch(ragged, std::false_type());
        };
        if (b.E % kN) sized(std::true_type());
        else sized(std::false_type());
    };
    typedef std::integral_constant<int, 1> One;
    typedef std::integral_constant<int, 2> Two;
    typedef std::integral_constant<int, 4> Four;
    typedef std::integral_constant<int, 16> Row;
    typedef std::integral_constant<int, 64> Wave;
    if (pieces <= 4) go(Four(), One());
    else if (pieces <= 8) go(std::integral_constant<int, 8>(), One());
    else if (pieces <= 16) go(Row(), One());
    else if (pieces <= 32) go(Row(), Two());
    else if (pieces <= 64) go(Row(), Four());
    else if (pieces <= 128) go(Wave(), Two());
    else if (pieces <= 256) go(Wave(), Four());
    else if constexpr (kN == 4) go(Wave(), std::integral_constant<int, 8>());
}

// Workgroups of the rows' kernel: up to kBlGroups, as many as have rows for all their lanes; one alone where that has no more than
// kBlAlone pieces a thread and so many choices, whose work is less than the two or three launches that it does without.  Derivatives of 32
// columns a thread leave registers for one workgroup to a CU, and one round of those is the shorter: 512 / 256 workgroups, us:  8000 x 2048, fp32:
// 59.8 / 50.3, bf16: 50.0 / 41.0;  20000 x 512, bf16: 33.5 / 30.5;  where two fit:  10000 x 1024, fp32: 32.5 / 36.0.
constexpr int64_t kBlAlone = 8;
static int row_groups(int64_t M, int64_t k, int64_t E, int per_piece, bool grad) {
    const int64_t pieces = (E + per_piece - 1) / per_piece, rows = kBlThreads / lanes_of(pieces), want = (M + rows - 1) / rows;
    if (M * pieces <= kBlAlone * kBlThreads && M * k <= kBlAlone * kBlThreads) return 1;
    const int most = grad && pieces_of_lane(pieces) * per_piece >= 32 ? kBlGroups / 2 : kBlGroups;
    return (int)(want < 2 ? 2 : want < most ? want : most);
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
    b.groups = row_groups(b.M, b.k, b.E, dt == TPPO_F32 ? 4 : 8, grad);
    char* ws = static_cast<char*>(workspace);
    b.part_p = reinterpret_cast<float*>(ws);
    b.part_counts = reinterpret_cast<int32_t*>(ws + part_bytes(b.E, kBlGroups));
    b.part_loss = reinterpret_cast<double*>(ws + 2 * part_bytes(b.E, kBlGroups));
    b.arrived = reinterpret_cast<int32_t*>(b.part_loss + kBlMaxE / kBlColumns);
    b.counters = b.groups;
    if (grad) {
        if (b.groups > 1) {
            const int64_t want = (b.M + kBlCountThreads - 1) / kBlCountThreads;
            b.counters = (int)(want < 1 ? 1 : want < kBlCounters ? want : kBlCounters);
            hipLaunchKernelGGL(balance_count_kernel, dim3(b.counters), dim3(kBlCountThreads), 0, s, b);
        }
        if (dt == TPPO_F32) launch_rows<float, true>(b, s);
        else launch_rows<uint16_t, true>(b, s);
    } else {
        if (dt == TPPO_F32) launch_rows<float, false>(b, s);
        else launch_rows<uint16_t, false>(b, s);
    }
    if (b.groups > 1)
        hipLaunchKernelGGL(balance_finish_kernel, dim3((b.E + kBlColumns - 1) / kBlColumns), dim3(kBlLast), 0, s, b);
    return launch_result();
}

}  // namespace tppo

extern "C" size_t tppo_balance_loss_workspace_bytes(int64_t M, int64_t E) {
    using namespace tppo;
    (void)M;
    if (E < 1 || E > kBlMaxE) return 256;
    return 2 * part_bytes(E, kBlGroups) + round_up((kBlMaxE / kBlColumns) * sizeof(double) + sizeof(int32_t), 256);
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
