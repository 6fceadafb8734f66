// Rotation of a head's 16-byte granules to a position.
#pragma once

#include "device.h"

namespace treewy {

// Elements of 16 bytes, widened, and back (a bf16 rounds to nearest even).
template <typename T> struct Granule;
template <> struct Granule<__bf16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void wide(uint4 x, float *f) {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __builtin_bit_cast(float, w[i] << 16);
            f[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ uint4 narrow(const float *f) {
        return make_uint4(pack_bf2(f[0], f[1]), pack_bf2(f[2], f[3]), pack_bf2(f[4], f[5]), pack_bf2(f[6], f[7]));
    }
};
template <> struct Granule<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void wide(uint4 x, float *f) {
        f[0] = __builtin_bit_cast(float, x.x);
        f[1] = __builtin_bit_cast(float, x.y);
        f[2] = __builtin_bit_cast(float, x.z);
        f[3] = __builtin_bit_cast(float, x.w);
    }
    static __device__ __forceinline__ uint4 narrow(const float *f) {
        return make_uint4(__builtin_bit_cast(uint32_t, f[0]), __builtin_bit_cast(uint32_t, f[1]),
                          __builtin_bit_cast(uint32_t, f[2]), __builtin_bit_cast(uint32_t, f[3]));
    }
};

// Rows cos[p][i0 ..], sin[p][i0 ..] of one granule's pairs.
template <typename T> struct Angles {
    float c[Granule<T>::N], s[Granule<T>::N];
    __device__ __forceinline__ void load(const float *cos, const float *sin, int64_t row, int i0) {
#pragma unroll
        for (int i = 0; i < Granule<T>::N; i += 4) {
            const f32x4 a = *reinterpret_cast<const f32x4 *>(cos + row + i0 + i);
            const f32x4 b = *reinterpret_cast<const f32x4 *>(sin + row + i0 + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) c[i + j] = a[j], s[i + j] = b[j];
        }
    }
};

// The granule x of a pair's first half (or of its second, where `second`), y its partner: x c - y s, or x c + y s.
template <typename T> __device__ __forceinline__ uint4 rotated(uint4 x, uint4 y, const Angles<T> &a, bool second) {
    constexpr int N = Granule<T>::N;
    float f[N], g[N];
    Granule<T>::wide(x, f);
    Granule<T>::wide(y, g);
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = f[i] * a.c[i] + (second ? g[i] : -g[i]) * a.s[i];
    return Granule<T>::narrow(f);
}

// The same of bf16 granules as two bf16, x ~= hi + rest (16 bits).
__device__ __forceinline__ void rotated_split(uint4 x, uint4 y, const Angles<__bf16> &a, bool second, uint4 &hi, uint4 &rest) {
    float f[8], g[8];
    Granule<__bf16>::wide(x, f);
    Granule<__bf16>::wide(y, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = f[i] * a.c[i] + (second ? g[i] : -g[i]) * a.s[i];
    bf16x8 h, r;
    split8(f, h, r);
    hi = __builtin_bit_cast(uint4, h);
    rest = __builtin_bit_cast(uint4, r);
}

}  // namespace treewy
