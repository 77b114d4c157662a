// 8 neighbouring elements that start anywhere: the whole 16-byte pieces around them, which must lie in the tensor, and the values out of those.
// Two or three wide loads and some twenty selects instead of eight loads of an element each, whose addresses lie far apart in a warp.
#pragma once
#include <cstdint>
#include <cstring>
#include <cuda_bf16.h>

namespace bpt {

template <typename T> struct Any8;
template <> struct Any8<float> {
    static constexpr int kPieces = 3;
    uint4 q[kPieces];
    int s;              // elements between the first piece's start and the first element
    __device__ __forceinline__ void load(const float* at) {
        s = (int)((uintptr_t)at & 15) / 4;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) q[j] = __ldg((const uint4*)(at - s) + j);
    }
    __device__ __forceinline__ void get(float (&z)[8]) const {
        unsigned w[12];
        memcpy(w, q, sizeof(w));
#pragma unroll
        for (int j = 0; j < 11; ++j) w[j] = s & 1 ? w[j + 1] : w[j];
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = __uint_as_float(s & 2 ? w[j + 2] : w[j]);
    }
};
template <> struct Any8<__nv_bfloat16> {
    static constexpr int kPieces = 2;
    uint4 q[kPieces];
    int s;
    __device__ __forceinline__ void load(const __nv_bfloat16* at) {
        s = (int)((uintptr_t)at & 15) / 2;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) q[j] = __ldg((const uint4*)(at - s) + j);
    }
    __device__ __forceinline__ void get(float (&z)[8]) const {
        unsigned w[8];
        memcpy(w, q, sizeof(w));
#pragma unroll
        for (int j = 0; j < 7; ++j) w[j] = s & 2 ? w[j + 1] : w[j];
#pragma unroll
        for (int j = 0; j < 5; ++j) w[j] = s & 4 ? w[j + 2] : w[j];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const unsigned two = s & 1 ? __funnelshift_r(w[j], w[j + 1], 16) : w[j];
            z[2 * j] = __uint_as_float(two << 16);
            z[2 * j + 1] = __uint_as_float(two & 0xffff0000u);
        }
    }
};
// Whether the pieces around the 8 elements at `at` lie in a tensor of `n` elements at `base`.
template <typename T>
__device__ __forceinline__ bool any8_inside(const T* at, const T* base, long long n) {
    const char* first = (const char*)((uintptr_t)at & ~(uintptr_t)15);
    return first >= (const char*)base && first + 16 * Any8<T>::kPieces <= (const char*)(base + n);
}

}  // namespace bpt
