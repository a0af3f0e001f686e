// Conversion to 8-bit integers shared by the row quantiser (int8.cu) and by the product that converts its activations itself (int8_few.cu).
#pragma once

#include "tc_ptx.cuh"
#include "types.cuh"

namespace hbfp {
namespace {

// The scale of a row from its largest |x|, given as a bit pattern (so that NaN is larger than infinity, and infinity than any number).
__device__ __forceinline__ float scale_of(uint32_t amax_bits) { return __fdiv_rn(__uint_as_float(amax_bits), 127.0f); }

// How a row's values are divided by its scale: q = rint(x * inv) where the quotient is clear of the border between two whole numbers, by
// more than the error of x * inv (2^-23 of 127 at most). Next to a border (one value in 5000) the remainder x - q * s decides: one FMA, and
// exact there, since it is a multiple of half an ulp of s and no more than s / 2 and a little; the approximate quotient misses the right whole
// number by one at most.
struct Divider {
    float s, inv;
    bool small;              // inv is no normal number: the division is binary64's
    __device__ __forceinline__ explicit Divider(float scale) : s(scale), inv(0.f), small(false) {
        // An all-zero row, or one that holds an infinity or NaN: q = 0. (With the scale an infinity or NaN, every product of such a row is NaN.)
        if (!(s > 0.f) || s > 3.0e38f) s = 0.f;
        else if (s < 1.0e-37f) small = true;
        else inv = __frcp_rn(s);
    }
    __device__ __forceinline__ int exactly(float x) const {
        if (!(s > 0.f)) return 0;                            // (an infinity times 0 is no number)
        const float t = __fmaf_rn(x, inv, 12582912.0f);      // 1.5 * 2^23: rounds to the nearest whole number, halves to even
        const float r = __fmaf_rn(12582912.0f - t, s, x);
        int n = __float_as_int(t) - 0x4B400000;
        const float twice = fabsf(r) + fabsf(r);
        if (twice > s || (twice == s && (n & 1))) n += r > 0.f ? 1 : -1;
        return n;
    }
    // (a scale below 1e-37 is coarse: it may have been rounded down far)
    __device__ __forceinline__ int coarsely(float x) const { return max(-127, min(127, (int)rint((double)x / (double)s))); }
    __device__ __forceinline__ int operator()(float x) const { return small ? coarsely(x) : exactly(x); }
    __device__ __forceinline__ uint2 eight_coarsely(const float (&x)[8]) const {
        uint32_t w[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i >> 2] |= ((uint32_t)coarsely(x[i]) & 0xFFu) << (8 * (i & 3));
        return make_uint2(w[0], w[1]);
    }
    // Eight values as bytes (not where the scale is `small`).
    __device__ __forceinline__ uint2 eight(const float (&x)[8]) const {
        const uint64_t inv2 = pack2(__float_as_uint(inv), __float_as_uint(inv)), up = pack2(0x4B400000u, 0x4B400000u), minus = pack2(0xBF800000u, 0xBF800000u);
        float far = 0.f;
        uint32_t n[8];
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const uint64_t v = pack2(__float_as_uint(x[i]), __float_as_uint(x[i + 1]));
            const uint64_t t = ffma2(v, inv2, up), off = ffma2(v, inv2, ffma2(t, minus, up));        // up - t = -q
            float t0, t1, o0, o1;
            unpack2(t, t0, t1);
            unpack2(off, o0, o1);
            n[i] = __float_as_uint(t0);
            n[i + 1] = __float_as_uint(t1);
            asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(far) : "f"(fabsf(o0)), "f"(fabsf(o1)));
        }
        if (!(far < 0.4999f)) {                              // next to a border, or no number
#pragma unroll
            for (int i = 0; i < 8; ++i) n[i] = (uint32_t)exactly(x[i]);
        }
        // (the low byte of 1.5 * 2^23 + q is that of q)
        return make_uint2(__byte_perm(__byte_perm(n[0], n[1], 0x0040), __byte_perm(n[2], n[3], 0x0040), 0x5410),
                          __byte_perm(__byte_perm(n[4], n[5], 0x0040), __byte_perm(n[6], n[7], 0x0040), 0x5410));
    }
};

// A finished sum: scaled by its token and its channel, the bias added. All kernels round alike.
__device__ __forceinline__ float int8_result(int sum, float token, float channel, float bias) { return __fmaf_rn((float)sum * token, channel, bias); }

}  // namespace
}  // namespace hbfp
