// What the kernels of the 8-bit cache share: codes to and from numbers, and which request a workgroup works for.
#pragma once

#include "cart_common.h"

namespace cart {
namespace cache {

constexpr int BLOCK = CART_CACHE_BLOCK;

template <int FMT> struct Code;

template <> struct Code<CART_E4M3> {
    // the largest magnitude, 448 = 0.875 x 2^9: exponent, and the fraction bits of an fp32 number with that fraction
    static constexpr int MAX_EXP = 9;
    static constexpr uint32_t MAX_MANT = 0x600000u;
    // 4 codes as fp32
    static __device__ __forceinline__ void decode4(uint32_t w, float (&x)[4]) {
        const float2_v a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false), b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
        x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
    }
    // to nearest, half to even; never more than 448 here, so what the instruction does beyond does not matter
    static __device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true));
    }
};

template <> struct Code<CART_I8> {
    static constexpr int MAX_EXP = 7;                   // 127 = 0.9921875 x 2^7
    static constexpr uint32_t MAX_MANT = 0x7e0000u;
    static __device__ __forceinline__ void decode4(uint32_t w, float (&x)[4]) {
        x[0] = static_cast<float>(static_cast<int8_t>(w));
        x[1] = static_cast<float>(static_cast<int8_t>(w >> 8));
        x[2] = static_cast<float>(static_cast<int8_t>(w >> 16));
        x[3] = static_cast<float>(static_cast<int8_t>(w >> 24));
    }
    static __device__ __forceinline__ uint32_t byte(float x) { return static_cast<uint32_t>(static_cast<int>(__builtin_rintf(x))) & 255u; }
    static __device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
        return byte(a) | byte(b) << 8 | byte(c) << 16 | byte(d) << 24;
    }
};

// The smallest power of two, 2^-64 at least, that brings a magnitude into the codes' range; `bits`: the magnitude as
// fp32 bits (the order of the bits is that of the magnitudes, and a NaN is above them all).  NaN from 2^127 on: a code
// that is rounded up may stand for more than fp32 holds there.
template <int FMT>
__device__ __forceinline__ float scale_for(uint32_t bits) {
    if (bits >= 0x7f000000u) return __uint_as_float(0x7fc00000u);
    // bits = 1.mant x 2^(exp - 127) = (0.5 x 1.mant) x 2^(exp - 126)
    const int e = static_cast<int>(bits >> 23) - 126 - Code<FMT>::MAX_EXP + ((bits & 0x7fffffu) > Code<FMT>::MAX_MANT ? 1 : 0);
    return __uint_as_float(static_cast<uint32_t>((e < -64 ? -64 : e) + 127) << 23);
}

// Offset i of a packed batch, whatever the array holds.
__device__ __forceinline__ int offset_at(const int32_t* cu, int i, int T) {
    const int x = cu[i];
    return x < 0 ? 0 : x > T ? T : x;
}

// The request that place `at` of an axis belongs to on which request b begins at cu[b] / unit + pad b: the last one that
// begins there or before.  (Requests of n rows reach into n / unit + 2 units at most, wherever the first begins, and
// n / unit + 1 where it begins a unit, so with pad = 2 or 1 each has places enough, without a running sum of units.)
// All lanes of a wavefront call it; 64 requests are looked at in one trip to memory, and what the caller asks next of the one
// that is found -- its offsets, its entry of `first` (null: 0) -- comes with the last of them.
struct Request { int b, from, to, first; };
__device__ __forceinline__ Request request_of(const int32_t* cu, const int32_t* first, int B, int T, int unit_log2, int pad, int at, int lane) {
    int lo = 0, hi = B, step, k, c, f;
    do {
        step = (hi - lo + 63) >> 6;
        const int i = lo + lane * step, j = i < B ? i : B;
        c = offset_at(cu, j, T);
        f = first ? first[j < B ? j : B - 1] : 0;
        const int n = __builtin_popcountll(__ballot(i < hi && (c >> unit_log2) + static_cast<long>(pad) * i <= at));
        k = n > 0 ? n - 1 : 0;
        lo += k * step;
        hi = hi < lo + step ? hi : lo + step;
    } while (hi - lo > 1);
    Request r;
    r.b = lo;
    r.from = __shfl(c, k);
    r.to = __shfl(c, k < 63 ? k + 1 : 63);
    r.first = __shfl(f, k);
    if (step > 1 || k == 63) r.to = offset_at(cu, lo + 1, T);
    return r;
}

}  // namespace cache
}  // namespace cart
