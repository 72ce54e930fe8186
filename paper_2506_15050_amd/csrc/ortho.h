// What the two ways of tppo_orthogonalize share (ortho.hip: products of X itself; ortho_gram.hip: of X X^T alone).
#pragma once
#include "head_tile.h"
#include "rows.h"

namespace tppo {

typedef _Float16 half_t;
typedef half_t half8 __attribute__((ext_vector_type(8)));
typedef half_t half4 __attribute__((ext_vector_type(4)));

// A pair of fp16: value = (hi + lo / kLoScale) / scale.  X is held times S (ortho.hip), m x m matrices times kOffScale.
constexpr float kLoScale = 2048.f, kOffScale = 64.f;

__device__ __forceinline__ int ns_swz(int r) { return (r >> 1) & 7; }

// K-major rows in LDS, as they lie in memory, pieces of 16 bytes exchanged: the 32 lanes that a transposing read serves at a time cover 8
// rows, {0 .. 3, 8 .. 11} + 4 h (mod 16), 32 bytes of each, and this spreads them over the 8 places of the 256-byte bank window.  Rows of
// 256 bytes begin at the same place all, rows of 128 or 384 in either half of the window by turns.
template <int COLUMNS>
__device__ __forceinline__ int ns_swz_k(int k) {
    static_assert(COLUMNS % 64 == 0, "pieces of 128 or 256 bytes are exchanged");
    if constexpr (COLUMNS % 128 == 0) return ((k & 3) | ((k >> 3) & 1) << 2) << 1;
    else return (((k >> 1) & 1) | ((k >> 3) & 1) << 1) << 1;
}
// the fragment of 16 columns `block` and 32 K rows from k32 * 32 on, of K-major rows that begin at LDS byte `at`
template <int COLUMNS>
__device__ __forceinline__ half8 ns_k_major_frag(unsigned at, int block, int k32, int lane) {
    typedef short s4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s4* lds_s4;
    constexpr int kRow = COLUMNS * 2;
    const int col = lane & 15, k = (lane >> 4) * 8 + (col >> 2);
    const unsigned from = at + k * kRow + ((2 * block + ((col & 3) >> 1)) ^ ns_swz_k<COLUMNS>(k)) * 16 + (col & 1) * 8 + k32 * 32 * kRow;
    const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(size_t)from);
    const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(size_t)(from + 4 * kRow));
    return __builtin_bit_cast(half8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

__device__ __forceinline__ uint16_t ns_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// eight values to a row of bf16 that has `left` more entries
__device__ __forceinline__ void put_whole_or_part(uint16_t* to, int left, const float (&x)[8]) {
    if (left >= 8) {
        put_piece<uint16_t, 8, false>(to, 0, 8, x);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) to[e] = ns_bf16(x[e]);
    }
}

// Consecutive numbers to the workgroups of an XCD, which go round-robin over the 8 (one more to the first `all` % 8 of them).
__device__ __forceinline__ int ns_by_xcd(int block, int all) {
    const int xcd = block & 7;
    return xcd * (all >> 3) + min(xcd, all & 7) + (block >> 3);
}

struct NsShape {
    int m, n, mp, np;                                // m <= n, and both rounded up to 64
    bool transposed;                                 // the caller's matrices are n x m
    int64_t count;
    int steps;
    float a, b, c;
    uint16_t* out;
    int64_t ld_out, each_out;
};

// What `steps` steps make of singular values s from 0 to 1: each multiplies them by m(l) = a + b l + c l l, l = s^2, which becomes
// g(l) = l m(l)^2.  Bounds over all of them, in every step: of the product of the |m|, of |m|, and of l.
struct NsReach {
    double product, value, least, square;            // product, largest and smallest |m|; largest l
};
NsReach ns_reach(int steps, float a, float b, float c);

// The way by X X^T (ortho_gram.hip): where it is the shorter, for m < kGramBelow at most, if the coefficients keep it within what fp16
// pairs hold.
constexpr int kGramBelow = 2048;
bool ns_gram_fits(const NsReach& reach, int steps, float a, float b, float c);
size_t ns_gram_bytes(int64_t count, int m, int n);
int ns_gram(const NsShape& x, const half_t* hi, const half_t* lo, const float2* scales, char* ws, hipStream_t s);

}  // namespace tppo
