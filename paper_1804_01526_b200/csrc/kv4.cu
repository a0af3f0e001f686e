// Writing new tokens' keys and values into the 4-bit cache and reading values back (the attention itself: kv4_attend.cuh).
//
// The conversion is the library's own block floating point with 4-bit mantissas and blocks of 32 along the row (Eq. 1, nearest-even),
// stored two mantissas to a byte; exponents end at 120, where a value saturates at 7 * 2^120.
#include "kv4.cuh"
#include "quant_math.cuh"

namespace hbfp {
namespace {

// What the threads of a launch share of it: thread = one word (eight values) of one token's keys or values of one head, so that four
// neighbouring threads are a block and a warp's accesses are contiguous. Bound by reading and writing the rows once.
struct Kv4Where {
    int64_t token;
    int head, word, side;       // side 0: keys, 1: values
    int64_t row;                // row of the cache's arrays [pages * heads * page], or -1
};

// The r-th word from word i0 of the sequence's new tokens on (r < 256 + the words of a token, so 32 bits do).
__device__ __forceinline__ Kv4Where kv4_where(const Kv4Args& a, int64_t i0, int r, int b, const Kv4Seq& s) {
    const int words = a.dim / 8, per = 2 * a.heads * words;
    const int64_t t0 = i0 / per;                 // the same in all threads
    r += (int)(i0 - t0 * per);
    const int dt = r / per;
    r -= dt * per;
    Kv4Where w;
    const int line = r / words;
    w.word = r - line * words;
    w.side = line >= a.heads;
    w.head = line - w.side * a.heads;
    const int64_t t = t0 + dt, p = (int64_t)s.length - s.n + t;
    w.token = s.first + t;
    w.row = -1;
    if (p >= 0 && p < s.length) {
        const int64_t page = kv4_page(a, b, (int)p >> a.shift);
        if (page >= 0) w.row = ((page * a.heads + w.head) << a.shift) + ((int)p & (a.page - 1));
    }
    return w;
}

template <class T>
__global__ void __launch_bounds__(256)
kv4_append_kernel(const Kv4Args a, const T* __restrict__ k, Kv4Rows ks, const T* __restrict__ v, Kv4Rows vs, bool vec) {
    chain_start();
    const int b = blockIdx.y;
    const Kv4Seq s = kv4_seq(a, b);
    const int64_t total = (int64_t)s.n * 2 * a.heads * (a.dim / 8);
    // every lane of a warp stays for the shuffles
    for (int64_t i0 = (int64_t)blockIdx.x * 256; i0 < total; i0 += (int64_t)gridDim.x * 256) {
        Kv4Where w{};
        w.row = -1;
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = 0.f;
        if (i0 + threadIdx.x < total) {
            w = kv4_where(a, i0, threadIdx.x, b, s);
            const Kv4Rows st = w.side ? vs : ks;
            const T* src = (w.side ? v : k) + w.token * st.token + w.head * st.head + 8 * w.word;
            if (vec) load8(src, e);
            else load8_part(src, 8, e);
        }
        uint32_t am = amax8_bits(e);
        am = max(am, __shfl_xor_sync(0xffffffffu, am, 1));
        am = max(am, __shfl_xor_sync(0xffffffffu, am, 2));
        const int exp = min(block_exponent(am, 4, 0), KV4_MAX_EXP);
        if (w.row < 0) continue;
        uint32_t word = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) word |= (uint32_t)(round_rne(e[j], exp, 7) + 8) << (4 * (j >> 1) + 16 * (j & 1));
        reinterpret_cast<uint32_t*>(w.side ? a.v_mant : a.k_mant)[w.row * (a.dim / 8) + w.word] = word;
        if ((w.word & 3) == 0) (w.side ? a.v_exps : a.k_exps)[w.row * (a.dim / 32) + (w.word >> 2)] = (int8_t)exp;
    }
}

// The values of the last `count` positions of every sequence, FP32 [sequences * count][heads][dim]; zeros where there is no position.
__global__ void __launch_bounds__(256)
kv4_read_kernel(Kv4Args a, int count, float* __restrict__ k, float* __restrict__ v) {
    chain_start();
    const int b = blockIdx.y;
    a.starts = nullptr;
    a.most = count;
    const Kv4Seq s = kv4_seq(a, b);
    const int64_t total = (int64_t)count * 2 * a.heads * (a.dim / 8);
    for (int64_t i0 = (int64_t)blockIdx.x * 256; i0 + threadIdx.x < total; i0 += (int64_t)gridDim.x * 256) {
        const Kv4Where w = kv4_where(a, i0, threadIdx.x, b, s);
        uint32_t word = 0x88888888u;
        float two = 0.f;
        if (w.row >= 0) {
            word = reinterpret_cast<const uint32_t*>(w.side ? a.v_mant : a.k_mant)[w.row * (a.dim / 8) + w.word];
            two = pow2f(kv4_exponent((w.side ? a.v_exps : a.k_exps)[w.row * (a.dim / 32) + (w.word >> 2)]));
        }
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = (float)((int)((word >> (4 * (j >> 1) + 16 * (j & 1))) & 15u) - 8) * two;
        float* dst = (w.side ? v : k) + (w.token * a.heads + w.head) * a.dim + 8 * w.word;
        reinterpret_cast<float4*>(dst)[0] = make_float4(e[0], e[1], e[2], e[3]);
        reinterpret_cast<float4*>(dst)[1] = make_float4(e[4], e[5], e[6], e[7]);
    }
}

dim3 kv4_grid(const Kv4Args& a, int64_t tokens_each) {
    const int64_t words = tokens_each * 2 * a.heads * (a.dim / 8), blocks = (words + 255) / 256;
    return dim3((unsigned)(blocks < 4096 ? (blocks > 0 ? blocks : 1) : 4096), (unsigned)a.sequences);
}

template <class T>
int append(const Kv4Args& a, const T* k, Kv4Rows ks, const T* v, Kv4Rows vs, cudaStream_t st) {
    const uintptr_t mask = (uintptr_t)k | (uintptr_t)v | (uintptr_t)((ks.token | ks.head | vs.token | vs.head) * (int64_t)sizeof(T));
    launch_chained(kv4_append_kernel<T>, kv4_grid(a, a.most), 256, 0, st, a, k, ks, v, vs, (mask & 15) == 0);
    return launch_status();
}

}  // namespace

int launch_kv4_append(const Kv4Args& a, int dtype, const void* k, Kv4Rows ks, const void* v, Kv4Rows vs, cudaStream_t st) {
    if (a.sequences == 0 || a.tokens == 0) return HBFP_OK;
    if (dtype == HBFP_F32) return append(a, static_cast<const float*>(k), ks, static_cast<const float*>(v), vs, st);
    if (dtype == HBFP_BF16) return append(a, static_cast<const __nv_bfloat16*>(k), ks, static_cast<const __nv_bfloat16*>(v), vs, st);
    return append(a, static_cast<const __half*>(k), ks, static_cast<const __half*>(v), vs, st);
}

int launch_kv4_read(const Kv4Args& a, int count, float* k, float* v, cudaStream_t st) {
    if (a.sequences == 0 || count == 0) return HBFP_OK;
    launch_chained(kv4_read_kernel, kv4_grid(a, count), 256, 0, st, a, count, k, v);
    return launch_status();
}

}  // namespace hbfp
