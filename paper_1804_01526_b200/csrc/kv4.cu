// Writing new tokens' keys and values into the 4-bit cache and reading values back (the attention itself: kv4_attend.cuh).
//
// The conversion is the library's own block floating point with 4-bit mantissas and blocks of 32 along the row (Eq. 1, nearest-even),
// stored two mantissas to a byte; exponents end at 120, where a value saturates at 7 * 2^120.
#include <type_traits>

#include "kv4.cuh"
#include "quant_math.cuh"

namespace hbfp {
namespace {

// A thread takes a word (eight values) of one token's keys or values of one head, so that four neighbouring threads are a block of 32 and a
// warp's accesses are contiguous. A token's 2 * heads * D / 8 words fill the CTA, several times over or as a part of it, and the CTA goes through
// tokens, so that what a thread's word is is worked out once: with it found by division for every word, 8 prompts of 1024 tokens, 8 heads of
// 128 FP32 values (76 MB) took 27 us, so 19. Two tokens are on their way together.
constexpr int KV4_THREADS = 256, KV4_UNROLL = 2;

template <int D>
struct Kv4Words {
    static constexpr int WORDS = D / 8, NB = D / 32;
    int per, tokens, sub, first;      // words of a token, tokens of the CTA at a time, this thread's of them, its first word
    __device__ __forceinline__ explicit Kv4Words(int heads) {
        per = 2 * heads * WORDS;
        tokens = per < KV4_THREADS ? KV4_THREADS / per : 1;
        sub = per < KV4_THREADS ? (int)threadIdx.x / per : 0;
        first = (int)threadIdx.x - sub * per;
    }
    __device__ __forceinline__ bool idle() const { return sub >= tokens; }
};
// Row of the cache's arrays for a head of the token t of the sequence's new ones; -1: it has no place.
__device__ __forceinline__ int64_t kv4_row(const Kv4Args& a, int b, const Kv4Seq& s, int64_t t, int head) {
    const int64_t p = (int64_t)s.length - s.n + t;
    if (t >= s.n || p < 0 || p >= s.held) return -1;
    const int64_t page = kv4_page(a, b, (int)p >> a.shift);
    return page < 0 ? -1 : ((page * a.heads + head) << a.shift) + ((int)p & (a.page - 1));
}

template <int D, class T>
__global__ void __launch_bounds__(KV4_THREADS, 5)
kv4_append_kernel(const Kv4Args a, const T* __restrict__ k, Kv4Rows ks, const T* __restrict__ v, Kv4Rows vs, bool vec) {
    using W = Kv4Words<D>;
    chain_start();
    const int b = blockIdx.y;
    const Kv4Seq s = kv4_seq_unreported(a, b);
    const W w(a.heads);
    // every lane of a warp stays for the shuffles
    for (int64_t t0 = (int64_t)blockIdx.x * w.tokens; t0 < s.n; t0 += (int64_t)gridDim.x * w.tokens * KV4_UNROLL)
        for (int q0 = 0; q0 < w.per; q0 += KV4_THREADS) {
            const int q = q0 + w.first, line = q / W::WORDS, word = q - line * W::WORDS, side = line >= a.heads, head = line - side * a.heads;
            const bool mine = !w.idle() && q < w.per;
            const Kv4Rows st = side ? vs : ks;
            Eight<T> x[KV4_UNROLL];
            int64_t row[KV4_UNROLL];
#pragma unroll
            for (int u = 0; u < KV4_UNROLL; ++u) {
                const int64_t t = t0 + (int64_t)u * gridDim.x * w.tokens + w.sub;
                x[u].zero();
                if (mine && t < s.n) {
                    const T* src = (side ? v : k) + (s.first + t) * st.token + head * st.head + 8 * word;
                    if (vec) x[u].load(src);
                    else x[u].load_part(src, 8);
                }
            }
#pragma unroll
            for (int u = 0; u < KV4_UNROLL; ++u) row[u] = mine ? kv4_row(a, b, s, t0 + (int64_t)u * gridDim.x * w.tokens + w.sub, head) : -1;
#pragma unroll
            for (int u = 0; u < KV4_UNROLL; ++u) {
                float e[8];
                x[u].get(e);
                uint32_t am = amax8_bits(e);
                am = max(am, __shfl_xor_sync(0xffffffffu, am, 1));
                am = max(am, __shfl_xor_sync(0xffffffffu, am, 2));
                const int exp = min(block_exponent(am, 4, 0), KV4_MAX_EXP);
                if (row[u] < 0) continue;
                uint32_t m = 0;
                const float scale = pow2f(-exp);
#pragma unroll
                for (int i = 0; i < 4; ++i) {                                 // q + 8 is q with its top bit turned, in four bits
                    const uint32_t pair = round_rne_pair(e[2 * i], e[2 * i + 1], scale, qmax_pair(7), neg_qmax_pair(7));
                    m |= ((pair & 0x000F000Fu) ^ 0x00080008u) << (4 * i);
                }
                reinterpret_cast<uint32_t*>(side ? a.v_mant : a.k_mant)[row[u] * W::WORDS + word] = m;
                if ((word & 3) == 0) (side ? a.v_exps : a.k_exps)[row[u] * W::NB + (word >> 2)] = (int8_t)exp;
            }
        }
    kv4_report(a, s);
}

// The values of the last `count` positions of every sequence, FP32 [sequences * count][heads][dim]; zeros where there is no position.
template <int D>
__global__ void __launch_bounds__(KV4_THREADS, 5)
kv4_read_kernel(Kv4Args a, int count, float* __restrict__ k, float* __restrict__ v) {
    using W = Kv4Words<D>;
    chain_start();
    const int b = blockIdx.y;
    a.starts = nullptr;
    a.most = count;
    const Kv4Seq s = kv4_seq_unreported(a, b);
    const W w(a.heads);
    if (w.idle()) return;
    for (int64_t t0 = (int64_t)blockIdx.x * w.tokens; t0 < s.n; t0 += (int64_t)gridDim.x * w.tokens * KV4_UNROLL)
        for (int q = w.first; q < w.per; q += KV4_THREADS) {
            const int line = q / W::WORDS, word = q - line * W::WORDS, side = line >= a.heads, head = line - side * a.heads;
            uint32_t m[KV4_UNROLL];
            int exp[KV4_UNROLL];
            int64_t row[KV4_UNROLL];
#pragma unroll
            for (int u = 0; u < KV4_UNROLL; ++u) row[u] = kv4_row(a, b, s, t0 + (int64_t)u * gridDim.x * w.tokens + w.sub, head);
#pragma unroll
            for (int u = 0; u < KV4_UNROLL; ++u) {
                m[u] = 0x88888888u;                                           // zeros
                exp[u] = 0;
                if (row[u] >= 0) {
                    m[u] = reinterpret_cast<const uint32_t*>(side ? a.v_mant : a.k_mant)[row[u] * W::WORDS + word];
                    exp[u] = (side ? a.v_exps : a.k_exps)[row[u] * W::NB + (word >> 2)];
                }
            }
#pragma unroll
            for (int u = 0; u < KV4_UNROLL; ++u) {
                const int64_t t = t0 + (int64_t)u * gridDim.x * w.tokens + w.sub;
                if (t >= s.n) break;
                const float two = pow2f(kv4_exponent((int8_t)exp[u]));
                float e[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) e[j] = (float)((int)((m[u] >> (4 * (j >> 1) + 16 * (j & 1))) & 15u) - 8) * two;
                float* dst = (side ? v : k) + ((s.first + t) * a.heads + head) * D + 8 * word;
                asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "f"(e[0]), "f"(e[1]), "f"(e[2]), "f"(e[3]), "f"(e[4]), "f"(e[5]),
                             "f"(e[6]), "f"(e[7]) : "memory");
            }
        }
    kv4_report(a, s);
}

// CTAs of a sequence: one for what it takes at a time, several times as much for a CTA where that leaves the GPU its fill.
dim3 kv4_grid(const Kv4Args& a, int64_t tokens_each) {
    const int per = 2 * a.heads * (a.dim / 8), at_a_time = per < KV4_THREADS ? KV4_THREADS / per : 1;
    const int64_t blocks = (tokens_each + at_a_time - 1) / at_a_time, fill = (148 * 8 + a.sequences - 1) / a.sequences;
    const int64_t folded = (blocks + KV4_UNROLL - 1) / KV4_UNROLL, n = folded > fill ? folded : blocks < fill ? blocks : fill;
    return dim3((unsigned)(n < 1 ? 1 : n < 65536 ? n : 65536), (unsigned)a.sequences);
}

template <class F>
int for_dim(int dim, F f) {
    switch (dim) {
        case 64: return f(std::integral_constant<int, 64>());
        case 96: return f(std::integral_constant<int, 96>());
        case 128: return f(std::integral_constant<int, 128>());
    }
    return f(std::integral_constant<int, 256>());
}

template <class T>
int append(const Kv4Args& a, const T* k, Kv4Rows ks, const T* v, Kv4Rows vs, cudaStream_t st) {
    const uintptr_t mask = (uintptr_t)k | (uintptr_t)v | (uintptr_t)((ks.token | ks.head | vs.token | vs.head) * (int64_t)sizeof(T));
    return for_dim(a.dim, [&](auto d) {
        launch_chained(kv4_append_kernel<decltype(d)::value, T>, kv4_grid(a, a.most), KV4_THREADS, 0, st, a, k, ks, v, vs, (mask & 15) == 0);
        return launch_status();
    });
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
    return for_dim(a.dim, [&](auto d) {
        launch_chained(kv4_read_kernel<decltype(d)::value>, kv4_grid(a, count), KV4_THREADS, 0, st, a, count, k, v);
        return launch_status();
    });
}

}  // namespace hbfp
