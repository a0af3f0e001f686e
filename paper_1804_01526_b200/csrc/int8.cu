// Product in 8-bit integers with a scale for each token and each channel:
//   y[m][n] = sa[m] * sb[n] * sum_k qa[m][k] * qb[n][k]  (+ bias[n])
// qa and sa come from FP32, bfloat16 or binary16 activations, one scale per row (token): s = fl32(amax / 127),
// q = the whole number nearest to x / s, halves to even, decided on the exact quotient. qb and sb are the weights', one scale per
// output channel, converted once. The sum is an exact int32 (K < 2^17, so 128 * 128 * K < 2^31); it is converted to FP32, scaled
// and rounded to the result's type once.
#include <cuda.h>

#include "tc_ptx.cuh"
#include "types.cuh"

namespace hbfp {
namespace {

// ------------------------------------------------------------------------------ conversion

// The scale of a row from its largest |x|, given as a bit pattern (so that NaN is larger than infinity, and infinity than any number).
__device__ __forceinline__ float scale_of(uint32_t amax_bits) { return __fdiv_rn(__uint_as_float(amax_bits), 127.0f); }

// How a row's values are divided by its scale: q = rint(x * inv), and where x is next to the border between two whole numbers the
// remainder x - q * s decides (one FMA; next to a border it is a multiple of half an ulp of s and no more than s / 2 and a little,
// so it is exact, and an approximate quotient can miss the right whole number by one at most).
struct Divider {
    float s, inv;
    bool small;              // inv is no normal number: divide in binary64
    __device__ __forceinline__ explicit Divider(float scale) : s(scale), inv(0.f), small(false) {
        if (!(s > 0.f) || s > 3.0e38f) s = 0.f;              // an all-zero row, or one that holds an infinity or NaN: q = 0
        else if (s < 1.0e-37f) small = true;
        else inv = __frcp_rn(s);
    }
    __device__ __forceinline__ int operator()(float x) const {
        if (small) return max(-127, min(127, (int)rint((double)x / (double)s)));      // (such a scale is coarse: it may round down far)
        const float t = __fmaf_rn(x, inv, 12582912.0f);      // 1.5 * 2^23: rounds to the nearest whole number, halves to even
        const float q = t - 12582912.0f;
        const float r = __fmaf_rn(-q, s, x);
        int n = __float_as_int(t) - 0x4B400000;
        if (fabsf(r) + fabsf(r) >= s && s > 0.f && (fabsf(r) + fabsf(r) > s || (n & 1))) n += r > 0.f ? 1 : -1;
        return n;
    }
};

__device__ __forceinline__ uint32_t pack_bytes(int a, int b, int c, int d) {
    return __byte_perm(__byte_perm((uint32_t)a, (uint32_t)b, 0x0040), __byte_perm((uint32_t)c, (uint32_t)d, 0x0040), 0x5410);
}

// Rows of x [rows][k] to q [rows][pitch] (bytes beyond k zero) and scale [rows]. A CTA per row; the row stays in registers where it
// has up to KEEP * 8 values per thread, longer rows are read again (from L2). Bound by reading x and writing q.
constexpr int QR_KEEP = 4;
template <class T, int THREADS>
__global__ void __launch_bounds__(THREADS)
int8_rows_kernel(const T* __restrict__ x, int64_t k, int64_t ld, bool vec, int8_t* __restrict__ q, int64_t pitch, float* __restrict__ scale) {
    chain_start();
    const int64_t row = blockIdx.x;
    const T* src = x + row * ld;
    const int64_t pieces = pitch / 8;                        // of eight values; the row ends inside one of the last two
    float v[QR_KEEP][8];
    uint32_t am = 0;
    auto fetch = [&](int64_t i, float (&e)[8]) {
        const int64_t at = 8 * i;
        if (vec && at + 8 <= k) load8(src + at, e);
        else load8_part(src + at, (int)max((int64_t)0, min((int64_t)8, k - at)), e);
    };
#pragma unroll
    for (int u = 0; u < QR_KEEP; ++u) {
        const int64_t i = threadIdx.x + u * THREADS;
        if (i < pieces) fetch(i, v[u]);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) v[u][e] = 0.f;
    }
#pragma unroll
    for (int u = 0; u < QR_KEEP; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) am = max(am, __float_as_uint(v[u][e]) & 0x7fffffffu);
    for (int64_t i = threadIdx.x + QR_KEEP * THREADS; i < pieces; i += THREADS) {
        float w[8];
        fetch(i, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) am = max(am, __float_as_uint(w[e]) & 0x7fffffffu);
    }
    am = __reduce_max_sync(0xffffffffu, am);
    __shared__ uint32_t part[THREADS / 32];
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = am;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) am = max(am, part[w]);
    const float s = scale_of(am);
    if (threadIdx.x == 0) scale[row] = s;
    const Divider div(s);
    int8_t* dst = q + row * pitch;
    auto put = [&](int64_t i, const float (&e)[8]) {
        const uint32_t lo = pack_bytes(div(e[0]), div(e[1]), div(e[2]), div(e[3])), hi = pack_bytes(div(e[4]), div(e[5]), div(e[6]), div(e[7]));
        *reinterpret_cast<uint2*>(dst + 8 * i) = make_uint2(lo, hi);
    };
#pragma unroll
    for (int u = 0; u < QR_KEEP; ++u) {
        const int64_t i = threadIdx.x + u * THREADS;
        if (i < pieces) put(i, v[u]);
    }
    for (int64_t i = threadIdx.x + QR_KEEP * THREADS; i < pieces; i += THREADS) {
        float w[8];
        fetch(i, w);
        put(i, w);
    }
}

// Columns of x [k][cols] to q [cols][pitch] and scale [cols]: weights stored with the contraction down their rows, converted once.
// 32 columns per CTA: the largest values first, then tiles of 128 rows turned in shared memory.
template <class T>
__global__ void __launch_bounds__(256)
int8_columns_kernel(const T* __restrict__ x, int64_t k, int64_t cols, int64_t ld, int8_t* __restrict__ q, int64_t pitch, float* __restrict__ scale) {
    chain_start();
    __shared__ uint32_t top[8][32];
    __shared__ __align__(16) int8_t tile[32][144];           // rows of 144 bytes: 16-byte aligned, and no two columns in one bank group
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c0 = (int64_t)blockIdx.x * 32, c = c0 + lane;
    uint32_t am = 0;
    if (c < cols)
        for (int64_t r = warp; r < k; r += 8) am = max(am, __float_as_uint(to_f32(x[r * ld + c])) & 0x7fffffffu);
    top[warp][lane] = am;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) am = max(am, top[w][lane]);
    const float s = scale_of(am);
    if (warp == 0 && c < cols) scale[c] = s;
    const Divider div(s);
    for (int64_t r0 = 0; r0 < pitch; r0 += 128) {
        for (int r = warp; r < 128; r += 8) tile[lane][r] = c < cols && r0 + r < k ? (int8_t)div(to_f32(x[(r0 + r) * ld + c])) : (int8_t)0;
        __syncthreads();
        const int col = threadIdx.x >> 3, piece = threadIdx.x & 7;
        if (c0 + col < cols && r0 + 16 * piece < pitch)
            *reinterpret_cast<uint4*>(q + (c0 + col) * pitch + r0 + 16 * piece) = *reinterpret_cast<const uint4*>(&tile[col][16 * piece]);
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------ product

struct Int8Problem {
    int M, N, K;
    const float *sa, *sb, *bias;     // bias may be null
    void* y;
    int64_t ldy;
    int32_t* status;
};

// One 128 x NT tile per CTA: TMA fills stages of 128 bytes of K, one thread issues the MMAs, four warps read the finished int32 sums
// from tensor memory, scale them and store.
template <int NT>
struct I8Cfg {
    static constexpr int STAGE = (TILE_M + NT) * STAGE_K;
    static constexpr int STAGES = 5;
    static constexpr int SMEM = 1024 + STAGES * STAGE + 1024 + 8 * NT;
    static constexpr int THREADS = 192;
};

template <class T, int NT>
__global__ void __launch_bounds__(I8Cfg<NT>::THREADS)
int8_gemm_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, const Int8Problem p) {
    using C = I8Cfg<NT>;
    extern __shared__ unsigned char smem_dyn[];
    const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    unsigned char* sm = smem_dyn + (base - smem_u32(smem_dyn));
    const uint32_t full_bar = base + C::STAGES * C::STAGE, empty_bar = full_bar + 8 * C::STAGES, done_bar = empty_bar + 8 * C::STAGES;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sm + C::STAGES * C::STAGE + 16 * C::STAGES + 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    float* cols = reinterpret_cast<float*>(sm + C::STAGES * C::STAGE + 1024);         // [NT] channel scales, [NT] biases
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int m0 = blockIdx.y * TILE_M, n0 = blockIdx.x * NT;
    const int steps = (p.K + STAGE_K - 1) / STAGE_K;

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) { mbar_init(full_bar + 8 * s, 1); mbar_init(empty_bar + 8 * s, 1); }
        mbar_init(done_bar, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(NT) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    chain_start();

    if (warp == 0) {
        if (lane == 0) {
            uint32_t s = 0, ph = 0;
            int it = 0;
            for (; it < steps; ++it) {
                if (!mbar_wait(empty_bar + 8 * s, ph ^ 1, abort_flag, p.status, 171)) break;
                mbar_expect_tx(full_bar + 8 * s, C::STAGE);
                tma_load_2d(base + s * C::STAGE, &mapA, it * STAGE_K, m0, full_bar + 8 * s);
                tma_load_2d(base + s * C::STAGE + TILE_M * STAGE_K, &mapB, it * STAGE_K, n0, full_bar + 8 * s);
                if (++s == C::STAGES) { s = 0; ph ^= 1; }
            }
            // nothing of this CTA is in flight when it leaves
            for (int k = min(it, C::STAGES); k > 0; --k) {
                if (s == 0) { s = C::STAGES - 1; ph ^= 1; } else { --s; }
                mbar_wait(full_bar + 8 * s, ph, abort_flag, p.status, 172, false);
            }
        }
    } else if (warp == 1) {
        if (elect_one()) {
            uint32_t s = 0, ph = 0;
            for (int it = 0; it < steps; ++it) {
                if (!mbar_wait(full_bar + 8 * s, ph, abort_flag, p.status, 173)) break;
                tc_fence_after();
                const uint64_t a = smem_desc_sw128(base + s * C::STAGE), b = smem_desc_sw128(base + s * C::STAGE + TILE_M * STAGE_K);
#pragma unroll
                for (int q = 0; q < 4; ++q) tc_mma_i8(tmem_base, a + 2 * q, b + 2 * q, idesc_i8<NT>(), it > 0 || q > 0);
                tc_commit(empty_bar + 8 * s);
                if (++s == C::STAGES) { s = 0; ph ^= 1; }
            }
            tc_commit(done_bar);
            mbar_wait(done_bar, 0, abort_flag, p.status, 174, false);
        }
    } else {
        const int e = threadIdx.x - 64;
        for (int i = e; i < NT; i += 128) {
            cols[i] = n0 + i < p.N ? __ldg(p.sb + n0 + i) : 0.f;
            cols[NT + i] = p.bias && n0 + i < p.N ? __ldg(p.bias + n0 + i) : 0.f;
        }
        const int quarter = warp & 3, row = m0 + quarter * 32 + lane;
        const float sa = row < p.M ? __ldg(p.sa + row) : 0.f;
        asm volatile("bar.sync 1, 128;" ::: "memory");
        if (mbar_wait_warp(done_bar, 0, abort_flag, p.status, 175)) {
            tc_fence_after();
            T* dst = reinterpret_cast<T*>(p.y) + (int64_t)row * p.ldy + n0;
            const bool quad = (p.ldy & 3) == 0 && (reinterpret_cast<uintptr_t>(p.y) & (4 * sizeof(T) - 1)) == 0;
#pragma unroll
            for (int c = 0; c < NT; c += 32) {
                int v[32];
                tc_ld32(tmem_base + ((uint32_t)(quarter * 32) << 16) + c, v);
                tc_wait_ld();
                if (row < p.M)
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        float y[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) y[i] = __fmaf_rn((float)v[j + i] * sa, cols[c + j + i], cols[NT + c + j + i]);
                        if (quad && n0 + c + j + 4 <= p.N) store4(dst + c + j, y[0], y[1], y[2], y[3]);
                        else
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (n0 + c + j + i < p.N) dst[c + j + i] = from_f32<T>(y[i]);
                    }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(NT) : "memory");
    }
}

// A contraction of no terms: the bias, or zero.
template <class T>
__global__ void __launch_bounds__(256)
int8_no_terms_kernel(const float* __restrict__ bias, T* __restrict__ y, int64_t M, int64_t N, int64_t ldy) {
    chain_start();
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < M * N; i += (int64_t)gridDim.x * 256)
        y[i / N * ldy + i % N] = from_f32<T>(bias ? bias[i % N] : 0.f);
}

// ------------------------------------------------------------------------------ host side

template <class T>
int quantize_rows(const T* x, int64_t rows, int64_t k, int64_t ld, int8_t* q, int64_t pitch, float* scale, cudaStream_t st) {
    const bool vec = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && ld * sizeof(T) % 16 == 0;
    if (rows == 0) return HBFP_OK;
    const int64_t bytes = rows * k * (int64_t)sizeof(T);
    if (pitch / 8 <= 64 * QR_KEEP) launch_streamed(bytes, int8_rows_kernel<T, 64>, (unsigned)rows, 64, 0, st, x, k, ld, vec, q, pitch, scale);
    else launch_streamed(bytes, int8_rows_kernel<T, 256>, (unsigned)rows, 256, 0, st, x, k, ld, vec, q, pitch, scale);
    return launch_status();
}

template <class T>
int quantize_any(const T* x, int64_t d0, int64_t d1, int64_t ld, int axis, int8_t* q, int64_t pitch, float* scale, cudaStream_t st) {
    if (axis == 1) return quantize_rows(x, d0, d1, ld, q, pitch, scale, st);
    if (d1 == 0) return HBFP_OK;
    launch_streamed(d0 * d1 * (int64_t)sizeof(T), int8_columns_kernel<T>, (unsigned)((d1 + 31) / 32), 256, 0, st, x, d0, d1, ld, q, pitch, scale);
    return launch_status();
}

template <class T>
int product(const Int8Problem& p, const int8_t* a, int64_t lda, const int8_t* b, int64_t ldb, cudaStream_t st) {
    if (p.K == 0) {
        launch_chained(int8_no_terms_kernel<T>, (unsigned)(((int64_t)p.M * p.N + 255) / 256 < 148 * 8 ? ((int64_t)p.M * p.N + 255) / 256 : 148 * 8), 256, 0, st, p.bias,
                       static_cast<T*>(p.y), (int64_t)p.M, (int64_t)p.N, p.ldy);
        return launch_status();
    }
    constexpr int NT = 128;
    CUtensorMap mA, mB;
    int rc = make_map(&mA, a, p.K, p.M, lda, STAGE_K, TILE_M, true);
    if (!rc) rc = make_map(&mB, b, p.K, p.N, ldb, STAGE_K, NT, true);
    if (!rc) rc = allow_shared<int8_gemm_kernel<T, NT>>(I8Cfg<NT>::SMEM);
    if (rc) return rc;
    launch_chained(int8_gemm_kernel<T, NT>, dim3((p.N + NT - 1) / NT, (p.M + TILE_M - 1) / TILE_M), I8Cfg<NT>::THREADS, I8Cfg<NT>::SMEM, st, mA, mB, p);
    note_product(st);
    return launch_status();
}

}  // namespace

int64_t int8_pitch(int64_t k) { return round_up(k > 0 ? k : 1, 16); }

int launch_int8_quantize(const void* x, int dtype, int64_t d0, int64_t d1, int64_t ld, int axis, int8_t* q, int64_t pitch, float* scale, cudaStream_t st) {
    if (dtype == HBFP_F32) return quantize_any(static_cast<const float*>(x), d0, d1, ld, axis, q, pitch, scale, st);
    if (dtype == HBFP_BF16) return quantize_any(static_cast<const __nv_bfloat16*>(x), d0, d1, ld, axis, q, pitch, scale, st);
    return quantize_any(static_cast<const __half*>(x), d0, d1, ld, axis, q, pitch, scale, st);
}

int launch_int8_gemm(int64_t M, int64_t N, int64_t K, const int8_t* a, int64_t lda, const float* sa, const int8_t* b, int64_t ldb, const float* sb,
                     const float* bias, void* y, int dtype, int64_t ldy, cudaStream_t st) {
    Int8Problem p{(int)M, (int)N, (int)K, sa, sb, bias, y, ldy, device_status_word()};
    if (!p.status) return HBFP_ERR_CUDA;
    if (dtype == HBFP_F32) return product<float>(p, a, lda, b, ldb, st);
    if (dtype == HBFP_BF16) return product<__nv_bfloat16>(p, a, lda, b, ldb, st);
    return product<__half>(p, a, lda, b, ldb, st);
}

}  // namespace hbfp
