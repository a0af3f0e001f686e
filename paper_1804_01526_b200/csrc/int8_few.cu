// 8-bit integer product of one to three tokens.
//
// Bound: reading the weights once (4096 x 4096: 17 MB, 2.6 us at the copy bandwidth) and, with so little to read, by the chain of latencies
// around it. A CTA takes 16 channels at a time and all of K, an eighth of it per warp: a lane loads 16 bytes of two channels at a time straight into
// MMA operand registers (the order of the values along an MMA's contraction is free as long as both operands agree), the first of them before
// anything else is known. The tokens lie in shared memory as bytes; every CTA converts them itself, which saves a launch. Sums of the warps are
// int32 and add up exactly. One token, 4096 x 4096, bfloat16: 5.6 us among others (cold 9.5), two 6.9, three 8.0; four
// took 10.8 when tried, where a conversion and int8_gemm_kernel take 8.5 to 9.2. (Tried for one token, when this kernel took 7.3: two launches with tiles of
// 128 x 128 13.0; conversion and tcgen05 MMAs in one launch, K split over a cluster, 12.9, most of it waits for the other CTAs.)
#include "int8.cuh"

namespace hbfp {
namespace {

constexpr int IF_WARPS = 8, IF_THREADS = 32 * IF_WARPS, IF_CHANNELS = 16, IF_AHEAD = 8, IF_TOKENS = 3;

struct FewInt8 {
    const void* x;
    int64_t ldx;
    const float* xs;                 // scales of tokens that were converted before
    int M, N, K, share;              // bytes of K of a warp, a multiple of 64
    int vec;                         // pieces of a token's row (eight values, 16 bytes of converted ones) are 16-byte aligned
    const int8_t* w;
    int64_t ldw;
    const float *ws, *bias;          // bias may be null
    void* y;
    int64_t ldy;
};

__device__ __forceinline__ void if_mma(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// X: type of the tokens (int8_t: converted before), T: of the result.
template <class X, class T>
__global__ void __launch_bounds__(IF_THREADS, 2)
int8_few_kernel(const FewInt8 p) {
    constexpr int ROWS = 8;                                                   // of the MMA's narrow operand
    extern __shared__ __align__(128) unsigned char sm[];
    __shared__ uint32_t top[ROWS];
    __shared__ float scale[ROWS];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int all = IF_WARPS * p.share, pitch = all + 64;                     // 64: rows start in different banks
    if (tid < ROWS) top[tid] = 0u;
    chain_start();

    // ---- weights: channels g and g + 8 of a tile, 16 bytes at 64 c + 16 t of the warp's share
    const int k0 = warp * p.share + 16 * t, chunks = p.share / 64, tiles = (p.N + IF_CHANNELS - 1) / IF_CHANNELS;
    uint4 a[IF_AHEAD], b[IF_AHEAD];
    auto load = [&](int tile, int c, uint4& u, uint4& v) {
        const int n = tile * IF_CHANNELS + g;
        const bool there = c < chunks && k0 + 64 * c < p.K;       // (what of the 16 bytes lies behind K meets a zero)
        const int8_t* at = p.w + (int64_t)n * p.ldw + k0 + 64 * c;
        u = v = make_uint4(0u, 0u, 0u, 0u);
        if (there && n < p.N) u = __ldg(reinterpret_cast<const uint4*>(at));
        if (there && n + 8 < p.N) v = __ldg(reinterpret_cast<const uint4*>(at + 8 * p.ldw));
    };
    int tile = blockIdx.x;
#pragma unroll
    for (int i = 0; i < IF_AHEAD; ++i) load(tile, i, a[i], b[i]);

    // ---- tokens as bytes
    if constexpr (sizeof(X) == 1) {
        const int8_t* x = static_cast<const int8_t*>(p.x);
        const int per = all / 16;
        for (int i = tid; i < ROWS * per; i += IF_THREADS) {
            const int r = i / per, k = 16 * (i - r * per);
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (r < p.M && k < p.K) {
                v = __ldg(reinterpret_cast<const uint4*>(x + (int64_t)r * p.ldx + k));
                if (k + 16 > p.K) {                                           // bytes behind the contraction may be anything
                    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int left = p.K - k - 4 * e;
                        w[e] = left <= 0 ? 0u : left >= 4 ? w[e] : w[e] & ((1u << (8 * left)) - 1u);
                    }
                    v = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            *reinterpret_cast<uint4*>(sm + r * pitch + k) = v;
        }
        if (tid < ROWS) scale[tid] = tid < p.M ? __ldg(p.xs + tid) : 0.f;
    } else {
        // A row after the other, 2048 values at a time: largest magnitude, then the bytes. (Compact loops: code that runs once is paid for by the line.)
        const X* x = static_cast<const X*>(p.x);
        __syncthreads();
        auto fetch = [&](int r, int k, Eight<X>& e) {
            const X* src = x + (int64_t)r * p.ldx + k;
            if (p.vec && k + 8 <= p.K) e.load(src);
            else e.load_part(src, p.K - k);
        };
#pragma unroll 1
        for (int r = 0; r < p.M; ++r) {
            uint32_t am = 0u;
#pragma unroll 2
            for (int k = 8 * tid; k < p.K; k += 8 * IF_THREADS) {
                Eight<X> e;
                fetch(r, k, e);
                am = max(am, e.amax_bits());
            }
            am = __reduce_max_sync(0xffffffffu, am);
            if (lane == 0) atomicMax(top + r, am);
        }
        __syncthreads();
        if (tid < ROWS) scale[tid] = scale_of(top[tid]);
#pragma unroll 1
        for (int r = 0; r < p.M; ++r) {
            const Divider div(scale_of(top[r]));
#pragma unroll 2
            for (int k = 8 * tid; k < all; k += 8 * IF_THREADS) {
                uint2 q = make_uint2(0u, 0u);
                if (k < p.K) {
                    Eight<X> e;
                    float f[8];
                    fetch(r, k, e);
                    e.get(f);
                    q = div.small ? div.eight_coarsely(f) : div.eight(f);
                }
                *reinterpret_cast<uint2*>(sm + r * pitch + k) = q;
            }
        }
        for (int i = tid; i < (ROWS - p.M) * (all / 16); i += IF_THREADS) {
            const int r = p.M + i / (all / 16), k = 16 * (i % (all / 16));
            *reinterpret_cast<uint4*>(sm + r * pitch + k) = make_uint4(0u, 0u, 0u, 0u);
        }
    }
    __syncthreads();

    const int col = tid & 15;                                                 // this thread's channel of a tile's results
    const unsigned char* xs = sm + g * pitch + k0;
    int* sums = reinterpret_cast<int*>(sm + ROWS * pitch);                    // [warp][token][channel]
    for (; tile < tiles; tile += gridDim.x) {
        const int n = tile * IF_CHANNELS + col;
        float ws = 0.f, bias = 0.f;
        if (n < p.N && tid < 16 * IF_TOKENS) {
            ws = __ldg(p.ws + n);
            if (p.bias) bias = __ldg(p.bias + n);
        }
        int acc[4] = {0, 0, 0, 0};
#pragma unroll 1
        for (int c = 0; c < chunks; c += IF_AHEAD) {
            const bool last = c + IF_AHEAD >= chunks;                         // then the next tile's first bytes follow
#pragma unroll
            for (int i = 0; i < IF_AHEAD; ++i) {
                if (c + i < chunks) {
                    const uint4 q = *reinterpret_cast<const uint4*>(xs + 64 * (c + i));
                    if_mma(acc, a[i].x, b[i].x, a[i].y, b[i].y, q.x, q.y);
                    if_mma(acc, a[i].z, b[i].z, a[i].w, b[i].w, q.z, q.w);
                }
                if (!last) load(tile, c + i + IF_AHEAD, a[i], b[i]);
                else if (tile + gridDim.x < tiles) load(tile + gridDim.x, i, a[i], b[i]);
            }
        }
        // columns 2 t and 2 t + 1 of the accumulators are tokens: the lanes t = 0 and 1 hold those there are
        if (t < 2)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[(warp * 4 + 2 * t + (e & 1)) * IF_CHANNELS + g + 8 * (e >> 1)] = acc[e];
        __syncthreads();
        const int r = tid >> 4;
        if (r < p.M && n < p.N) {
            int sum = 0;
#pragma unroll
            for (int w = 0; w < IF_WARPS; ++w) sum += sums[(w * 4 + r) * IF_CHANNELS + col];
            static_cast<T*>(p.y)[(int64_t)r * p.ldy + n] = from_f32<T>(int8_result(sum, scale[r], ws, bias));
        }
        __syncthreads();
    }
}

int if_share(int64_t K) { return (int)((K + 64 * IF_WARPS - 1) / (64 * IF_WARPS)) * 64; }
int if_smem(int share) { return 8 * (IF_WARPS * share + 64) + IF_WARPS * 4 * IF_CHANNELS * 4; }
constexpr int IF_SMEM_LIMIT = 112 * 1024;                                     // two CTAs of an SM

template <class X, class T>
int if_launch(const FewInt8& p, cudaStream_t st) {
    if (const int rc = allow_shared<int8_few_kernel<X, T>>(IF_SMEM_LIMIT)) return rc;
    const int tiles = (p.N + IF_CHANNELS - 1) / IF_CHANNELS, ctas = 2 * sm_count();
    launch_chained(int8_few_kernel<X, T>, dim3((unsigned)(tiles < ctas ? tiles : ctas)), IF_THREADS, if_smem(p.share), st, p);
    return launch_status();
}
template <class T>
int if_launch_x(int a_dtype, const FewInt8& p, cudaStream_t st) {
    if (a_dtype == HBFP_I8) return if_launch<int8_t, T>(p, st);
    if (a_dtype == HBFP_F32) return if_launch<float, T>(p, st);
    if (a_dtype == HBFP_BF16) return if_launch<__nv_bfloat16, T>(p, st);
    return if_launch<__half, T>(p, st);
}

}  // namespace

bool int8_few_eligible(int64_t M, int64_t K) { return M >= 1 && M <= IF_TOKENS && K >= 1 && if_smem(if_share(K)) <= IF_SMEM_LIMIT; }

int launch_int8_few(int64_t M, int64_t N, int64_t K, const void* a, int a_dtype, int64_t lda, const float* sa, const int8_t* w, int64_t ldw, const float* sw,
                    const float* bias, void* y, int dtype, int64_t ldy, cudaStream_t st) {
    FewInt8 p{};
    p.x = a;
    p.ldx = lda;
    p.xs = sa;
    p.M = (int)M;
    p.N = (int)N;
    p.K = (int)K;
    p.share = if_share(K);
    p.vec = a_dtype != HBFP_I8 && (reinterpret_cast<uintptr_t>(a) & 15) == 0 && lda * dtype_bytes(a_dtype) % 16 == 0;
    p.w = w;
    p.ldw = ldw;
    p.ws = sw;
    p.bias = bias;
    p.y = y;
    p.ldy = ldy;
    if (dtype == HBFP_F32) return if_launch_x<float>(a_dtype, p, st);
    if (dtype == HBFP_BF16) return if_launch_x<__nv_bfloat16>(a_dtype, p, st);
    return if_launch_x<__half>(a_dtype, p, st);
}

}  // namespace hbfp
