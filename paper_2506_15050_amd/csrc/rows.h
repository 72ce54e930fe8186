// Rows of fp32 or bf16 in 16-byte pieces, for the kernels that take whole rows at any stride and address (layer norm, balance loss).
#pragma once
#include <type_traits>

#include "common.h"

namespace tppo {

// A piece of a row: 16 bytes, from any address that the type allows (the hardware takes vector accesses at any, across lines more slowly).
template <class T>
struct Piece;
template <>
struct Piece<float> {
    static constexpr int kN = 4;
    typedef float V __attribute__((ext_vector_type(4), aligned(4)));
    V v;
    __device__ __forceinline__ float get(int e) const { return v[e]; }
    __device__ __forceinline__ void set(int e, float x) { v[e] = x; }
};
template <>
struct Piece<uint16_t> {                             // bf16
    static constexpr int kN = 8;
    typedef uint32_t V __attribute__((ext_vector_type(4), aligned(2)));
    V v;
    __device__ __forceinline__ float get(int e) const {
        return __uint_as_float(e & 1 ? v[e >> 1] & 0xFFFF0000u : v[e >> 1] << 16);
    }
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

// two fp32 -> two bf16 in one instruction, round to nearest even
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{lo, hi}), b2));
}
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(uint16_t* p, float x) { *p = (uint16_t)two_bf16(x, 0.f); }

// Where piece c of a row of n begins.  RAGGED (n is no multiple of kN): the last one ends with the row, and its first elements are the one
// before's as well -- `own` says which are its own.
template <int kN, bool RAGGED>
__device__ __forceinline__ int piece_start(int c, int n) {
    return RAGGED ? min(c * kN, max(n - kN, 0)) : c * kN;
}
template <int kN, bool RAGGED>
__device__ __forceinline__ bool own(int c, int start, int e, int n) {
    return !RAGGED || (start + e >= c * kN && start + e < n);
}

// Elements start .. of a row of n; zeros beyond it.  (A row shorter than a piece, or a piece that passes its end: element by element.)
// STREAM: read once, and not kept in the caches for it.
template <class T, bool RAGGED, bool STREAM = false>
__device__ __forceinline__ Piece<T> piece_at(const T* row, int start, int n) {
    constexpr int kN = Piece<T>::kN;
    Piece<T> p;
    if (!RAGGED || start + kN <= n) {
        const typename Piece<T>::V* at = reinterpret_cast<const typename Piece<T>::V*>(row + start);
        p.v = STREAM ? __builtin_nontemporal_load(at) : *at;
    } else {
        if constexpr (kN == 4) {
#pragma unroll
            for (int e = 0; e < kN; ++e) p.v[e] = start + e < n ? row[start + e] : 0.f;
        } else {
#pragma unroll
            for (int e = 0; e < kN; e += 2) {
                const uint32_t lo = start + e < n ? row[start + e] : 0, hi = start + e + 1 < n ? row[start + e + 1] : 0;
                p.v[e >> 1] = lo | hi << 16;
            }
        }
    }
    return p;
}

// kIn values to elements start .. of a row of n of type T, those from `first` on.  (The last piece of a ragged row may write what the one
// before it writes too, the same: first = 0.)
template <class T, int kIn, bool RAGGED, bool STREAM = false>
__device__ __forceinline__ void put_piece(T* row, int start, int n, const float (&x)[kIn], int first = 0) {
    T* at = row + start;
    if (!RAGGED || (start + kIn <= n && first == 0)) {
        typedef typename Piece<T>::V V;
#pragma unroll
        for (int e = 0; e < kIn; e += Piece<T>::kN) {
            V v;
            if constexpr (sizeof(T) == 4) v = V{x[e], x[e + 1], x[e + 2], x[e + 3]};
            else v = V{two_bf16(x[e], x[e + 1]), two_bf16(x[e + 2], x[e + 3]), two_bf16(x[e + 4], x[e + 5]), two_bf16(x[e + 6], x[e + 7])};
            V* to = reinterpret_cast<V*>(at + e);
            if constexpr (STREAM) __builtin_nontemporal_store(v, to);
            else *to = v;
        }
    } else {
#pragma unroll
        for (int e = 0; e < kIn; ++e)
            if (e >= first && start + e < n) put(at + e, x[e]);
    }
}

// kOut values of type T from elements start .. of a row of n
template <class T, int kOut, bool RAGGED>
__device__ __forceinline__ void get_piece(const T* row, int start, int n, float (&x)[kOut]) {
    constexpr int kN = Piece<T>::kN;
#pragma unroll
    for (int q = 0; q < kOut / kN; ++q) {
        const Piece<T> p = piece_at<T, RAGGED>(row, start + q * kN, n);
#pragma unroll
        for (int e = 0; e < kN; ++e) x[q * kN + e] = p.get(e);
    }
}

// the wavefront's sum, in every lane
__device__ __forceinline__ float wave_sum(float x) {
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wave_prefix(x)), kWave - 1));
}

}  // namespace tppo
