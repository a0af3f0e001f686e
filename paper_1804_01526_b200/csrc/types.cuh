// Element types of the serving operators (int8.cu, kv4_*.cu): FP32, bfloat16 and binary16 in, the same out. Arithmetic is FP32.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace hbfp {
namespace {

inline int64_t dtype_bytes(int dt) { return dt == HBFP_F32 ? 4 : 2; }
inline bool dtype_ok(int dt) { return dt == HBFP_F32 || dt == HBFP_BF16 || dt == HBFP_F16; }

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <class T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

// Two FP32 values as a pair of 16-bit elements (the first in the low half).
__device__ __forceinline__ uint32_t pack_pair(float a, float b, const __nv_bfloat16*) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_pair(float a, float b, const __half*) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void unpack_pair(uint32_t w, float& a, float& b, const __nv_bfloat16*) {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xFFFF0000u);
}
__device__ __forceinline__ void unpack_pair(uint32_t w, float& a, float& b, const __half*) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    a = f.x;
    b = f.y;
}

// Eight neighbouring elements held in their own type.
template <class T>
struct Eight {
    uint4 raw[sizeof(T) / 2];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[i] = make_uint4(0u, 0u, 0u, 0u);
    }
    __device__ __forceinline__ void load(const T* p) {                     // 16-byte aligned
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
    }
    __device__ __forceinline__ void load_part(const T* p, int n) { load_between(p, 0, n); }      // any alignment, elements from n on zero
    __device__ __forceinline__ void load_between(const T* p, int from, int n) {       // the same, and those before `from`
        T e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = i >= from && i < n ? p[i] : from_f32<T>(0.f);
        uint32_t w[2 * sizeof(T)];
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(to_f32(e[i]));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack_pair(to_f32(e[2 * i]), to_f32(e[2 * i + 1]), p);
        }
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    }
    // Any alignment, all eight there: whole 16-byte words around them, shifted into place, where those lie within [from, to) (elsewhere as load_part).
    __device__ __forceinline__ void load_around(const T* p, const void* from, const void* to) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p), first = at & ~(uintptr_t)15;
        constexpr int Q = sizeof(T) / 2 + 1;                               // 16-byte words of the window
        if (first < reinterpret_cast<uintptr_t>(from) || first + 16 * Q > reinterpret_cast<uintptr_t>(to)) {
            load_part(p, 8);
            return;
        }
        uint32_t w[4 * Q];
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(first) + i);
            w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
        const uint32_t off = (uint32_t)(at & 15), half = (off & 2) * 8;
        constexpr int N = 4 * (Q - 1);
        uint32_t t[4 * Q];
#pragma unroll
        for (int i = 0; i < 4 * Q; ++i) t[i] = sizeof(T) == 4 || i + 1 == 4 * Q ? w[i] >> half : __funnelshift_r(w[i], w[i + 1 < 4 * Q ? i + 1 : i], half);
        uint32_t u[4 * Q];
#pragma unroll
        for (int i = 0; i < 4 * Q; ++i) u[i] = (off & 8) && i + 2 < 4 * Q ? t[i + 2 < 4 * Q ? i + 2 : i] : t[i];
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            uint32_t r[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) r[j] = (off & 4) ? u[4 * i + j + 1] : u[4 * i + j];
            raw[i] = make_uint4(r[0], r[1], r[2], r[3]);
        }
    }
    // The largest magnitude as the bit pattern of an FP32 number (16-bit types: patterns of magnitudes are ordered as their values are, two at a time).
    __device__ __forceinline__ uint32_t amax_bits() const {
        if constexpr (sizeof(T) == 4) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 2; ++i) m = max(max(m, max(raw[i].x & 0x7fffffffu, raw[i].y & 0x7fffffffu)), max(raw[i].z & 0x7fffffffu, raw[i].w & 0x7fffffffu));
            return m;
        } else {
            const uint32_t m = __vmaxu2(__vmaxu2(raw[0].x & 0x7fff7fffu, raw[0].y & 0x7fff7fffu), __vmaxu2(raw[0].z & 0x7fff7fffu, raw[0].w & 0x7fff7fffu));
            float a, b;
            unpack_pair(m, a, b, (const T*)nullptr);
            return max(__float_as_uint(a), __float_as_uint(b));
        }
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        if constexpr (sizeof(T) == 4) {
            const uint32_t w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
        } else {
            const uint32_t w[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) unpack_pair(w[i], v[2 * i], v[2 * i + 1], (const T*)nullptr);
        }
    }
};

// Four neighbouring elements held in their own type.
template <class T>
struct Four {
    uint32_t raw[sizeof(T)];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); ++i) raw[i] = 0u;
    }
    __device__ __forceinline__ void load(const T* p) {                     // aligned to four of them
        if constexpr (sizeof(T) == 4) {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(p));
            raw[0] = v.x; raw[1] = v.y; raw[2] = v.z; raw[3] = v.w;
        } else {
            const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
            raw[0] = v.x; raw[1] = v.y;
        }
    }
    __device__ __forceinline__ void load_each(const T* p) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) raw[i] = __float_as_uint(p[i]);
        } else {
            raw[0] = pack_pair(to_f32(p[0]), to_f32(p[1]), p);
            raw[1] = pack_pair(to_f32(p[2]), to_f32(p[3]), p);
        }
    }
    __device__ __forceinline__ void get(float (&v)[4]) const {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(raw[i]);
        } else {
            unpack_pair(raw[0], v[0], v[1], (const T*)nullptr);
            unpack_pair(raw[1], v[2], v[3], (const T*)nullptr);
        }
    }
};
// They leave; p must be aligned to four of them.
__device__ __forceinline__ void store_four(float* p, const float (&v)[4]) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
template <class T>
__device__ __forceinline__ void store_four(T* p, const float (&v)[4]) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_pair(v[0], v[1], p), pack_pair(v[2], v[3], p));
}
// Sixteen bytes; p must be 16-byte aligned.
__device__ __forceinline__ void store_piece(float* p, const float (&v)[4]) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
template <class T>
__device__ __forceinline__ void store_piece(T* p, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_pair(v[0], v[1], p), pack_pair(v[2], v[3], p), pack_pair(v[4], v[5], p), pack_pair(v[6], v[7], p));
}

}  // namespace
}  // namespace hbfp
