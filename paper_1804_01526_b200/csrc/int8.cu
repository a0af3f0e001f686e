// Product in 8-bit integers with a scale for each token and each channel:
//   y[m][n] = sa[m] * sb[n] * sum_k qa[m][k] * qb[n][k]  (+ bias[n])
// qa and sa come from FP32, bfloat16 or binary16 activations, one scale per row (token): s = fl32(amax / 127),
// q = the whole number nearest to x / s, halves to even, decided on the exact quotient. qb and sb are the weights', one scale per
// output channel, converted once. The sum is an exact int32 (K < 2^17, so 128 * 128 * K < 2^31); it is converted to FP32, scaled
// and rounded to the result's type once.
#include <cuda.h>

#include "int8.cuh"

namespace hbfp {
namespace {

// ------------------------------------------------------------------------------ conversion

// Rows of x [rows][k] to q [rows][pitch] (bytes beyond k zero) and scale [rows]. GROUP threads take a row (a warp needs no barrier); it stays
// in their registers, in its own type, up to KEEP * 8 values each, longer rows are read again (from L2). Bound by reading x and writing q:
// 8192 x 8192 FP32 49 us, 6.8 TB/s.
constexpr int QR_KEEP = 4;
template <class T, int GROUP>
__global__ void __launch_bounds__(GROUP > 256 ? GROUP : 256, GROUP > 256 ? 2 : 4)
int8_rows_kernel(const T* __restrict__ x, int64_t rows, int64_t k, int64_t ld, bool vec, int8_t* __restrict__ q, int64_t pitch, float* __restrict__ scale) {
    chain_start();
    constexpr int THREADS = GROUP > 256 ? GROUP : 256;
    const int me = threadIdx.x % GROUP;
    const int64_t row = (int64_t)blockIdx.x * (THREADS / GROUP) + threadIdx.x / GROUP;
    if (GROUP <= 32 && row >= rows) return;                          // (whole warps; with larger groups they stay for the barrier)
    const bool in = row < rows;
    const T* src = x + (in ? row : 0) * ld;
    const int pieces = in ? (int)(pitch / 8) : 0, whole = (int)(k / 8);      // of eight values; those behind k are zeros, as many as the pitch has
    Eight<T> v[QR_KEEP];
    const T* const end = x + (rows - 1) * ld + k;
    auto fetch = [&](int i, Eight<T>& e) {
        if (i >= whole) e.load_part(src + 8 * (int64_t)i, (int)(k - 8 * (int64_t)i));
        else if (vec) e.load(src + 8 * (int64_t)i);
        else e.load_around(src + 8 * (int64_t)i, x, end);
    };
#pragma unroll
    for (int u = 0; u < QR_KEEP; ++u) {
        const int i = me + u * GROUP;
        v[u].zero();
        if (i < pieces) fetch(i, v[u]);
    }
    uint32_t am = 0;
#pragma unroll
    for (int u = 0; u < QR_KEEP; ++u) am = max(am, v[u].amax_bits());
    for (int i = me + QR_KEEP * GROUP; i < pieces; i += GROUP) {
        Eight<T> w;
        fetch(i, w);
        am = max(am, w.amax_bits());
    }
    am = __reduce_max_sync(0xffffffffu, am);
    if (GROUP > 32) {
        constexpr int W = GROUP / 32;
        __shared__ uint32_t part[THREADS / 32];
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = am;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) am = max(am, part[threadIdx.x / GROUP * W + w]);
    }
    if (!in) return;
    const float s = scale_of(am);
    if (me == 0) scale[row] = s;
    const Divider div(s);
    int8_t* dst = q + row * pitch;
    if (div.small) {
        for (int64_t i = me; i < pitch; i += GROUP) dst[i] = i < k ? (int8_t)div.coarsely(to_f32(src[i])) : (int8_t)0;
        return;
    }
    auto put = [&](int i, const Eight<T>& e) {
        float f[8];
        e.get(f);
        *reinterpret_cast<uint2*>(dst + 8 * (int64_t)i) = div.eight(f);
    };
#pragma unroll
    for (int u = 0; u < QR_KEEP; ++u) {
        const int i = me + u * GROUP;
        if (i < pieces) put(i, v[u]);
    }
    for (int i = me + QR_KEEP * GROUP; i < pieces; i += GROUP) {
        Eight<T> w;
        fetch(i, w);
        put(i, w);
    }
}

// The same for rows that start at any element (a contraction that is no whole number of 16 bytes, a slice): the pieces loaded are those
// between 16-byte borders, so that a row's loads are whole words, read once; the row is moved into place as bytes, eight of a piece and the
// next one's from the neighbouring lane. Rows that GROUP threads hold, pitch / 8 + 1 pieces.
// (a turn more than above: 1023 values are 129 pieces)
template <int GROUP> constexpr int QS_KEEP = GROUP > 256 ? QR_KEEP : QR_KEEP + 1;
template <class T, int GROUP>
__global__ void __launch_bounds__(GROUP > 256 ? GROUP : 256, GROUP > 256 ? 2 : sizeof(T) == 4 ? 3 : 4)
int8_shifted_rows_kernel(const T* __restrict__ x, int64_t rows, int64_t k, int64_t ld, int8_t* __restrict__ q, int64_t pitch, float* __restrict__ scale) {
    chain_start();
    constexpr int KEEP = QS_KEEP<GROUP>, THREADS = GROUP > 256 ? GROUP : 256, WARPS = GROUP / 32;
    __shared__ uint32_t part[THREADS / 32];
    __shared__ uint2 edge[KEEP][THREADS / 32];                    // the first piece of every warp
    const int me = threadIdx.x % GROUP, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warp0 = warp / WARPS * WARPS;
    const int64_t row = (int64_t)blockIdx.x * (THREADS / GROUP) + threadIdx.x / GROUP;
    if (GROUP <= 32 && row >= rows) return;                          // (whole warps; with larger groups they stay for the barriers)
    const bool in = row < rows;
    const T* src = x + (in ? row : 0) * ld;
    const int shift = (int)((reinterpret_cast<uintptr_t>(src) & 15) / sizeof(T)), n = (int)k, pieces = (int)(pitch / 8);
    Eight<T> v[KEEP];
#pragma unroll
    for (int u = 0; u < KEEP; ++u) {
        const int e0 = 8 * (me + u * GROUP) - shift;                 // piece's first element
        v[u].zero();
        if (in && e0 >= 0 && e0 + 8 <= n) v[u].load(src + e0);
        else if (in && e0 < n && e0 > -8) v[u].load_between(src + e0, -e0, n - e0);
    }
    uint32_t am = 0;
#pragma unroll
    for (int u = 0; u < KEEP; ++u) am = max(am, v[u].amax_bits());
    am = __reduce_max_sync(0xffffffffu, am);
    if (GROUP > 32) {
        if (lane == 0) part[warp] = am;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WARPS; ++w) am = max(am, part[warp0 + w]);
    }
    const float s = scale_of(am);
    if (in && me == 0) scale[row] = s;
    const Divider div(s);
    int8_t* dst = q + (in ? row : 0) * pitch;
    uint2 b[KEEP];
#pragma unroll
    for (int u = 0; u < KEEP; ++u) {
        b[u] = make_uint2(0u, 0u);
        if (u * GROUP <= pieces) {                                   // (turns behind the row are passed over)
            float f[8];
            v[u].get(f);
            b[u] = div.eight(f);
        }
        if (GROUP > 32 && lane == 0) edge[u][warp] = b[u];
    }
    if (GROUP > 32) __syncthreads();
    if (!in) return;
    if (div.small) {
        for (int64_t i = me; i < pitch; i += GROUP) dst[i] = i < k ? (int8_t)div.coarsely(to_f32(src[i])) : (int8_t)0;
        return;
    }
    const uint32_t bits = 8u * (shift & 3);
#pragma unroll
    for (int u = 0; u < KEEP; ++u) {
        // the piece after: the next lane's, of the last lane the next warp's first, of the last warp the first's of the next turn
        const int un = u + 1 < KEEP ? u + 1 : u;                  // (behind the last turn there is nothing)
        uint2 next = make_uint2(__shfl_down_sync(0xffffffffu, b[u].x, 1), __shfl_down_sync(0xffffffffu, b[u].y, 1));
        if constexpr (GROUP > 32) {
            if (lane == 31) next = warp + 1 < warp0 + WARPS ? edge[u][warp + 1] : edge[un][warp0];
        } else {
            const uint32_t nx = __shfl_sync(0xffffffffu, b[un].x, 0), ny = __shfl_sync(0xffffffffu, b[un].y, 0);
            if (lane == 31) next = make_uint2(nx, ny);
        }
        const uint32_t w0 = shift & 4 ? b[u].y : b[u].x, w1 = shift & 4 ? next.x : b[u].y, w2 = shift & 4 ? next.y : next.x;
        const int i = me + u * GROUP;
        if (i < pieces) *reinterpret_cast<uint2*>(dst + 8 * (int64_t)i) = make_uint2(__funnelshift_r(w0, w1, bits), __funnelshift_r(w1, w2, bits));
    }
}

// Columns of x [k][cols] to q [cols][pitch] and scale [cols]: weights stored with the contraction down their rows, converted once.
// 32 columns per CTA: the largest values first, then tiles of 128 rows turned in shared memory. Reads twice, with few CTAs: 4096 x 4096 FP32 139 us.
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
    int tma_out;                     // the result has a tensor map
    int a_rows, stages, off_boxes;   // int8_gemm_kernel
};

// The way of a finished tile out of a warp: 32 rows (lane = row) x 128 bytes of the result at a time, scaled, the bias added and rounded, in
// shared memory (16-byte piece j of row r at piece j ^ (r & 7), the swizzle of the tensor map: no two lanes meet in a bank), from where the
// copy engine stores it. Stored by the lanes themselves, 32 bytes of 32 rows an instruction, the FP32 result
// of 4096 x 4096 x 1024 took 30.6 us where the product without its stores takes 15.4. A result whose pitch or place is not a multiple of 16
// bytes is copied out along its rows.
constexpr int I8_BOX = 32 * 128;
// The copy engine cuts a box off at the matrix's last row, but along the rows only at the next 16 bytes behind N: where N does not end on such a
// border, boxes that go beyond it (`stop`) are copied out too.
struct Int8Out {
    const CUtensorMap* map;      // null: no tensor map can be made
    void* y;
    int64_t ldy;
    int M, N, stop;
};
template <class T>
__device__ __forceinline__ int int8_stop(int N) { return N % (16 / (int)sizeof(T)) == 0 ? 0x7fffffff : N; }
// Half of a box for 16-bit types, all of it for FP32: columns j0 .. j0 + 31 of it.
template <class T>
__device__ __forceinline__ void int8_fill_box(unsigned char* box, int j0, const int (&v)[32], float sa, const float* sb, const float* bias) {
    constexpr int V = 16 / sizeof(T);
    const int lane = threadIdx.x & 31;
    unsigned char* line = box + lane * 128;
#pragma unroll
    for (int j = 0; j < 32; j += V) {
        float o[V];
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 s = *reinterpret_cast<const float4*>(sb + j + i), b = *reinterpret_cast<const float4*>(bias + j + i);
            o[i] = int8_result(v[j + i], sa, s.x, b.x);
            o[i + 1] = int8_result(v[j + i + 1], sa, s.y, b.y);
            o[i + 2] = int8_result(v[j + i + 2], sa, s.z, b.z);
            o[i + 3] = int8_result(v[j + i + 3], sa, s.w, b.w);
        }
        store_piece(reinterpret_cast<T*>(line + ((((j0 + j) / V) ^ (lane & 7)) << 4)), o);
    }
}
// The box leaves; it may be filled again after int8_box_free.
template <class T, int COLS = 128 / (int)sizeof(T)>
__device__ __forceinline__ void int8_send_box(const Int8Out& out, unsigned char* box, int row0, int col0) {
    const int lane = threadIdx.x & 31;
    if (out.map && col0 + COLS <= out.stop) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0 && row0 < out.M && col0 < out.N) {
            asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
                         ::"l"(reinterpret_cast<uint64_t>(out.map)), "r"(smem_u32(box)), "r"(col0), "r"(row0) : "memory");
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
        return;
    }
    __syncwarp();
    T* y = reinterpret_cast<T*>(out.y);
    const int rows = min(32, out.M - row0);
    for (int r = 0; r < rows; ++r)
#pragma unroll
        for (int c = lane; c < COLS; c += 32) {
            const int at = c * (int)sizeof(T);
            if (col0 + c < out.N) y[(int64_t)(row0 + r) * out.ldy + col0 + c] = *reinterpret_cast<const T*>(box + r * 128 + (((at >> 4) ^ (r & 7)) << 4) + (at & 15));
        }
}
__device__ __forceinline__ void int8_box_free() {
    asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
}

// One 128 x NT tile per CTA: TMA fills stages of 128 bytes of K, one thread issues the MMAs, four warps read the finished int32 sums
// from tensor memory, scale them and store. For products of few tiles, which a narrow NT spreads over the SMs, and which are bound by the
// latency of what is in flight: a stage holds only the tokens that there are (`a_rows`, a multiple of eight: the MMA's other rows are whatever lies
// behind, and are not stored), so that 24 tokens and 32 channels have 150 KB on the way.
// Two columns of 128 bytes of K a stage: a commit and a look at a barrier for eight MMAs (17 tokens x 4096 x 4096: one column 12.0 us, two 9.7, four 10.2).
constexpr int I8_STAGES = 8, I8_COLUMNS = 2, I8_STAGE_BYTES = 160 * 1024;
template <int NT>
struct I8Cfg {
    static constexpr int THREADS = 192;
    static constexpr int SMEM = 1024 + I8_STAGE_BYTES + (TILE_M * STAGE_K) + 4 * I8_BOX + 1024 + 8 * NT;       // at most
    static int stages(int a_rows) { const int n = I8_STAGE_BYTES / (I8_COLUMNS * (a_rows + NT) * STAGE_K); return n < I8_STAGES ? n : I8_STAGES; }
    // (behind the last stage the MMA still reads what its rows would be)
    static int tiles(int a_rows) { return stages(a_rows) * I8_COLUMNS * (a_rows + NT) * STAGE_K + (TILE_M - a_rows) * STAGE_K; }
    static int smem(int a_rows) { return 1024 + tiles(a_rows) + 4 * I8_BOX + 1024 + 8 * NT; }
};

template <class T, int NT>
__global__ void __launch_bounds__(I8Cfg<NT>::THREADS)
int8_gemm_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, const __grid_constant__ CUtensorMap mapY, const Int8Problem p) {
    extern __shared__ unsigned char smem_dyn[];
    const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    unsigned char* sm = smem_dyn + (base - smem_u32(smem_dyn));
    // [stages][NT channels, tokens], boxes on their way out, barriers, [NT] channel scales and [NT] biases
    const int stages = p.stages;
    const uint32_t column = (uint32_t)(p.a_rows + NT) * STAGE_K, stage = I8_COLUMNS * column;
    unsigned char* boxes = sm + p.off_boxes;
    const uint32_t full_bar = base + p.off_boxes + 4 * I8_BOX, empty_bar = full_bar + 8 * I8_STAGES, done_bar = empty_bar + 8 * I8_STAGES;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(boxes + 4 * I8_BOX + 16 * I8_STAGES + 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    float* cols = reinterpret_cast<float*>(boxes + 4 * I8_BOX + 1024);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int m0 = blockIdx.y * TILE_M, n0 = blockIdx.x * NT;
    const int steps = (p.K + I8_COLUMNS * STAGE_K - 1) / (I8_COLUMNS * STAGE_K);

    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) { mbar_init(full_bar + 8 * s, 1); mbar_init(empty_bar + 8 * s, 1); }
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
                if (!mbar_wait_soon(empty_bar + 8 * s, ph ^ 1, abort_flag, p.status, 171)) break;
                mbar_expect_tx(full_bar + 8 * s, stage);
#pragma unroll
                for (int c = 0; c < I8_COLUMNS; ++c) {                        // (a column behind K is zeros)
                    tma_load_2d(base + s * stage + c * column, &mapB, (I8_COLUMNS * it + c) * STAGE_K, n0, full_bar + 8 * s);
                    tma_load_2d(base + s * stage + c * column + NT * STAGE_K, &mapA, (I8_COLUMNS * it + c) * STAGE_K, m0, full_bar + 8 * s);
                }
                if (++s == stages) { s = 0; ph ^= 1; }
            }
            // nothing of this CTA is in flight when it leaves
            for (int k = min(it, stages); k > 0; --k) {
                if (s == 0) { s = stages - 1; ph ^= 1; } else { --s; }
                mbar_wait_soon(full_bar + 8 * s, ph, abort_flag, p.status, 172, false);
            }
        }
    } else if (warp == 1) {
        if (elect_one()) {
            uint32_t s = 0, ph = 0;
            for (int it = 0; it < steps; ++it) {
                if (!mbar_wait_soon(full_bar + 8 * s, ph, abort_flag, p.status, 173)) break;
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < I8_COLUMNS; ++c) {
                    const uint64_t b = smem_desc_sw128(base + s * stage + c * column), a = smem_desc_sw128(base + s * stage + c * column + NT * STAGE_K);
#pragma unroll
                    for (int q = 0; q < 4; ++q) tc_mma_i8(tmem_base, a + 2 * q, b + 2 * q, idesc_i8<NT>(), it > 0 || c > 0 || q > 0);
                }
                tc_commit(empty_bar + 8 * s);
                if (++s == stages) { s = 0; ph ^= 1; }
            }
            tc_commit(done_bar);
            mbar_wait_soon(done_bar, 0, abort_flag, p.status, 174, false);
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
        if (mbar_wait_warp_soon(done_bar, 0, abort_flag, p.status, 175)) {
            tc_fence_after();
            constexpr int BOX = NT < 128 / (int)sizeof(T) ? NT : 128 / (int)sizeof(T);       // 32 columns of 16 bits fill half of a box: copied out
            const Int8Out out{p.tma_out && BOX * sizeof(T) == 128 ? &mapY : nullptr, p.y, p.ldy, p.M, p.N, int8_stop<T>(p.N)};
            unsigned char* box = boxes + (warp - 2) * I8_BOX;
#pragma unroll
            for (int c = 0; c < NT; c += 32) {
                int v[32];
                tc_ld32(tmem_base + ((uint32_t)(quarter * 32) << 16) + c, v);
                tc_wait_ld();
                if (c % BOX == 0) int8_box_free();
                int8_fill_box<T>(box, c % BOX, v, sa, cols + c, cols + NT + c);
                if ((c + 32) % BOX == 0) int8_send_box<T, BOX>(out, box, m0 + quarter * 32, n0 + c + 32 - BOX);
            }
            asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(NT) : "memory");
    }
}

// ---- Two SMs per 256 x NT tile, for products of many tiles. Each CTA of a pair brings its own 128 rows of tokens and half of the
// channels' rows, so a byte from L2 takes part in twice the products of the kernel above, which is bound by that (8192 cube 545 us).
// Persistent: a pair goes through its share of the tiles, the finished tile is read, scaled and stored by eight warps of each CTA while
// the MMAs fill the next accumulator of tensor memory. (16 384 operations per clock and SM: 16 KB + NT / 2 * 128 bytes per stage.)
template <int NT>
struct I8Pair {
    static constexpr int A_BYTES = TILE_M * STAGE_K, B_BYTES = NT / 2 * STAGE_K, STAGE = A_BYTES + B_BYTES;
    static constexpr int STAGES = NT == 256 ? 5 : 7, GROUPS = TMEM_COLS / NT;
    static constexpr int EPI_WARPS = 8, COLS = NT / 2, THREADS = 64 + 32 * EPI_WARPS;      // two warps per lane quarter, half the columns each
    static constexpr int SCALES = EPI_WARPS * 2 * COLS * 4;       // per epilogue warp: channel scales, biases
    static constexpr int SMEM = 1024 + STAGES * STAGE + EPI_WARPS * I8_BOX + SCALES + 1024;
    static_assert(SMEM <= 232448, "shared memory");
};
template <int NT>
__device__ __forceinline__ constexpr uint32_t idesc_i8_two() {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(NT >> 3) << 17) | ((uint32_t)(2 * TILE_M >> 4) << 24);
}

// Tile `w` of the traversal: groups of eight tile rows sweep across the channels, so that their panels are shared in L2.
__device__ __forceinline__ void pair_tile(int w, int tiles_m, int tiles_n, int& m, int& n) {
    constexpr int G = 8;
    const int per = G * tiles_n, group = w / per, first = group * G, size = min(G, tiles_m - first), within = w - group * per;
    n = within / size;
    m = first + (within - n * size);
}

template <class T, int NT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(I8Pair<NT>::THREADS, 1)
int8_pair_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, const __grid_constant__ CUtensorMap mapY, const Int8Problem p,
                 int tiles_m, int tiles_n) {
    using C = I8Pair<NT>;
    extern __shared__ unsigned char smem_dyn[];
    const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    unsigned char* sm = smem_dyn + (base - smem_u32(smem_dyn));
    float* scales = reinterpret_cast<float*>(sm + C::STAGES * C::STAGE + C::EPI_WARPS * I8_BOX);
    constexpr int BARS = C::STAGES * C::STAGE + C::EPI_WARPS * I8_BOX + C::SCALES;
    const uint32_t full_bar = base + BARS;                   // leader: tiles of both CTAs landed
    const uint32_t empty_bar = full_bar + 8 * C::STAGES;     // local: the MMAs have read the stage
    const uint32_t tfull_bar = empty_bar + 8 * C::STAGES;    // local: accumulator complete
    const uint32_t tempty_bar = tfull_bar + 8 * C::GROUPS;   // leader: accumulator read by the warps of both CTAs
    const uint32_t done_bar = tempty_bar + 8 * C::GROUPS;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sm + BARS + 16 * C::STAGES + 16 * C::GROUPS + 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int cluster = (int)cluster_id_x(), nclusters = (int)cluster_count_x(), total = tiles_m * tiles_n;
    const int steps = (p.K + STAGE_K - 1) / STAGE_K;

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) { mbar_init(full_bar + 8 * s, 1); mbar_init(empty_bar + 8 * s, 1); }
        for (int g = 0; g < C::GROUPS; ++g) { mbar_init(tfull_bar + 8 * g, 1); mbar_init(tempty_bar + 8 * g, 2 * C::EPI_WARPS); }
        mbar_init(done_bar, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_barrier();            // both CTAs' barriers and tensor memory exist before anyone signals across
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    chain_start();

    if (warp == 0) {
        if (lane == 0) {
            const uint32_t leader_full = map_to_rank(full_bar, 0);
            uint32_t s = 0, ph = 0, it = 0;
            bool ok = true;
            for (int w = cluster; ok && w < total; w += nclusters) {
                int tm, tn;
                pair_tile(w, tiles_m, tiles_n, tm, tn);
                const int my_m = tm * 2 * TILE_M + (int)rank * TILE_M, my_n = tn * NT + (int)rank * (NT / 2);
                for (int k = 0; k < steps; ++k, ++it) {
                    if (!mbar_wait_soon(empty_bar + 8 * s, ph ^ 1, abort_flag, p.status, 181)) { ok = false; break; }
                    if (rank == 0) mbar_expect_tx(full_bar + 8 * s, 2u * C::STAGE);
                    const uint32_t at = base + s * C::STAGE;
                    tma_load_2d_pair(at, &mapA, k * STAGE_K, my_m, leader_full + 8 * s, L2_EVICT_LAST);
                    tma_load_2d_pair(at + C::A_BYTES, &mapB, k * STAGE_K, my_n, leader_full + 8 * s, L2_EVICT_NORMAL);
                    if (++s == C::STAGES) { s = 0; ph ^= 1; }
                }
            }
            // the leader waits for the tiles of both CTAs that nobody may have waited for
            if (rank == 0)
                for (uint32_t back = min(it, (uint32_t)C::STAGES); back > 0; --back) {
                    if (s == 0) { s = C::STAGES - 1; ph ^= 1; } else { --s; }
                    mbar_wait_soon(full_bar + 8 * s, ph, abort_flag, p.status, 182, false);
                }
        }
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            uint32_t s = 0, ph = 0, g = 0, gph = 1;
            bool ok = true;
            for (int w = cluster; ok && w < total; w += nclusters) {
                if (!mbar_wait_soon(tempty_bar + 8 * g, gph, abort_flag, p.status, 183)) break;
                tc_fence_after();
                for (int k = 0; k < steps; ++k) {
                    if (!mbar_wait_soon(full_bar + 8 * s, ph, abort_flag, p.status, 184)) { ok = false; break; }
                    tc_fence_after();
                    const uint64_t a = smem_desc_sw128(base + s * C::STAGE), b = smem_desc_sw128(base + s * C::STAGE + C::A_BYTES);
#pragma unroll
                    for (int q = 0; q < 4; ++q) tc_mma_i8_pair(tmem_base + g * NT, a + 2 * q, b + 2 * q, idesc_i8_two<NT>(), k > 0 || q > 0);
                    tc_commit_pair(empty_bar + 8 * s, 3);
                    if (++s == C::STAGES) { s = 0; ph ^= 1; }
                }
                if (ok) tc_commit_pair(tfull_bar + 8 * g, 3);
                if (++g == C::GROUPS) { g = 0; gph ^= 1; }
            }
            tc_commit_pair(done_bar, 1);
            mbar_wait_soon(done_bar, 0, abort_flag, p.status, 185, false);
        }
    } else {
        const int e = warp - 2, quarter = warp & 3, half = e >> 2;
        float* sb = scales + e * 2 * C::COLS;
        unsigned char* box = sm + C::STAGES * C::STAGE + e * I8_BOX;
        const uint32_t tempty_leader = map_to_rank(tempty_bar, 0);
        const Int8Out out{p.tma_out ? &mapY : nullptr, p.y, p.ldy, p.M, p.N, int8_stop<T>(p.N)};
        constexpr int BOX = 128 / sizeof(T);
        uint32_t g = 0, gph = 0;
        for (int w = cluster; w < total; w += nclusters) {
            int tm, tn;
            pair_tile(w, tiles_m, tiles_n, tm, tn);
            const int row = tm * 2 * TILE_M + (int)rank * TILE_M + quarter * 32 + lane, n0 = tn * NT + half * C::COLS;
            __syncwarp();
            for (int i = lane; i < C::COLS; i += 32) {
                sb[i] = n0 + i < p.N ? __ldg(p.sb + n0 + i) : 0.f;
                sb[C::COLS + i] = p.bias && n0 + i < p.N ? __ldg(p.bias + n0 + i) : 0.f;
            }
            const float sa = row < p.M ? __ldg(p.sa + row) : 0.f;
            __syncwarp();
            if (!mbar_wait_warp_soon(tfull_bar + 8 * g, gph, abort_flag, p.status, 186)) break;
            tc_fence_after();
            const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + g * NT + half * C::COLS;
            constexpr int CH = 32;
            int v[2][CH];
            tc_ld32(taddr, v[0]);
#pragma unroll
            for (int c = 0; c < C::COLS; c += CH) {
                tc_wait_ld();
                if (c + CH < C::COLS) tc_ld32(taddr + c + CH, v[(c / CH + 1) & 1]);
                else {
                    // all of the accumulator is in registers: it is handed back before the last columns are scaled
                    tc_fence_before();
                    mbar_arrive_cluster_elect(tempty_leader + 8 * g);
                }
                const int(&x)[CH] = v[(c / CH) & 1];
                if (c % BOX == 0) int8_box_free();
                int8_fill_box<T>(box, c % BOX, x, sa, sb + c, sb + C::COLS + c);
                if ((c + CH) % BOX == 0) int8_send_box<T>(out, box, row - lane, n0 + c + CH - BOX);
            }
            if (++g == C::GROUPS) { g = 0; gph ^= 1; }
        }
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    // neither CTA leaves while the other can still signal its barriers
    tc_fence_before();
    __syncthreads();
    cluster_barrier();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
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
    auto launch = [&](auto kernel, int group) {
        const int threads = group > 256 ? group : 256, per = threads / group;
        launch_streamed(bytes, kernel, (unsigned)((rows + per - 1) / per), threads, 0, st, x, rows, k, ld, vec, q, pitch, scale);
    };
    // as few threads as keep the row in registers
    // Rows off 16-byte borders go by their aligned pieces (int8_shifted_rows_kernel / int8_rows_kernel, which loads around each of its own): 4736 x 8607 FP32 38.1 / 65.2 us,
    // 8192 x 8191 bfloat16 59.0 / 71.1, 630 x 9732 binary16 6.2 / 8.6, 64 x 4095 FP32 3.1 / 3.6. Not where the piece more is a second turn for little:
    // 16384 x 250 bfloat16 9.4 / 8.2.
    const int64_t shifted = pitch / 8 + 1;
    if (!vec && pitch > 256 && shifted <= 512 * QS_KEEP<512>) {
        auto launch_shifted = [&](auto kernel, int group) {
            const int threads = group > 256 ? group : 256, per = threads / group;
            launch_streamed(bytes, kernel, (unsigned)((rows + per - 1) / per), threads, 0, st, x, rows, k, ld, q, pitch, scale);
        };
        if (shifted <= 32 * QS_KEEP<32>) launch_shifted(int8_shifted_rows_kernel<T, 32>, 32);
        else if (shifted <= 128 * QS_KEEP<128>) launch_shifted(int8_shifted_rows_kernel<T, 128>, 128);
        else if (shifted <= 256 * QS_KEEP<256>) launch_shifted(int8_shifted_rows_kernel<T, 256>, 256);
        else launch_shifted(int8_shifted_rows_kernel<T, 512>, 512);
        return launch_status();
    }
    if (pitch <= 32 * 8 * QR_KEEP) launch(int8_rows_kernel<T, 32>, 32);
    else if (pitch <= 128 * 8 * QR_KEEP) launch(int8_rows_kernel<T, 128>, 128);
    else if (pitch <= 256 * 8 * QR_KEEP) launch(int8_rows_kernel<T, 256>, 256);
    else launch(int8_rows_kernel<T, 512>, 512);
    return launch_status();
}

template <class T>
int quantize_any(const T* x, int64_t d0, int64_t d1, int64_t ld, int axis, int8_t* q, int64_t pitch, float* scale, cudaStream_t st) {
    if (axis == 1) return quantize_rows(x, d0, d1, ld, q, pitch, scale, st);
    if (d1 == 0) return HBFP_OK;
    launch_streamed(d0 * d1 * (int64_t)sizeof(T), int8_columns_kernel<T>, (unsigned)((d1 + 31) / 32), 256, 0, st, x, d0, d1, ld, q, pitch, scale);
    return launch_status();
}

// Tensor map of the result in boxes of 32 rows x 128 bytes, where its pitch and place allow one. It counts elements: a column's byte can lie
// past 2^31, where the copy engine's coordinates end.
template <class T>
int map_result(Int8Problem& p, CUtensorMap* m) {
    p.tma_out = p.ldy * (int64_t)sizeof(T) % 16 == 0 && (reinterpret_cast<uintptr_t>(p.y) & 15) == 0;
    if (!p.tma_out) { *m = CUtensorMap{}; return HBFP_OK; }
    return make_map(m, p.y, p.N, p.M, p.ldy * sizeof(T), 128 / sizeof(T), 32, true, sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_UINT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16);
}

template <class T, int NT>
int launch_pair(Int8Problem p, const int8_t* a, int64_t lda, const int8_t* b, int64_t ldb, cudaStream_t st) {
    using C = I8Pair<NT>;
    CUtensorMap mA, mB, mY;
    int rc = make_map(&mA, a, p.K, p.M, lda, STAGE_K, TILE_M, true);
    if (!rc) rc = make_map(&mB, b, p.K, p.N, ldb, STAGE_K, NT / 2, true);
    if (!rc) rc = map_result<T>(p, &mY);
    if (!rc) rc = allow_shared<int8_pair_kernel<T, NT>>(C::SMEM);
    if (rc) return rc;
    const int tiles_m = (p.M + 2 * TILE_M - 1) / (2 * TILE_M), tiles_n = (p.N + NT - 1) / NT;
    const int64_t tiles = (int64_t)tiles_m * tiles_n;
    if (tiles >= (1ll << 30)) return HBFP_ERR_UNSUPPORTED;
    // pairs that can be resident at once: the tiles are dealt out by their number
    static std::atomic<int> resident[MAX_DEVICES];
    const int dev = current_device();
    if (dev < 0) return HBFP_ERR_CUDA;
    int pairs = resident[dev].load(std::memory_order_acquire);
    if (!pairs) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(2 * (unsigned)sm_count());
        cfg.blockDim = dim3(C::THREADS);
        cfg.dynamicSmemBytes = C::SMEM;
        HBFP_CUDA_OK(cudaOccupancyMaxActiveClusters(&pairs, int8_pair_kernel<T, NT>, &cfg));
        if (pairs < 1) return HBFP_ERR_CUDA;
        resident[dev].store(pairs, std::memory_order_release);
    }
    launch_chained(int8_pair_kernel<T, NT>, dim3(2 * (unsigned)(tiles < pairs ? tiles : pairs)), C::THREADS, C::SMEM, st, mA, mB, mY, p, tiles_m, tiles_n);
    note_product(st);
    return launch_status();
}
// Enough 256 x 128 tiles to give every pair of SMs one.
bool pair_eligible(int64_t M, int64_t N) { return M > 128 && (M + 255) / 256 * ((N + 127) / 128) >= 74; }

template <class T, int NT>
int launch_tiles(Int8Problem p, const int8_t* a, int64_t lda, const int8_t* b, int64_t ldb, cudaStream_t st) {
    using C = I8Cfg<NT>;
    p.a_rows = p.M < TILE_M ? (p.M + 7) / 8 * 8 : TILE_M;
    p.stages = C::stages(p.a_rows);
    p.off_boxes = C::tiles(p.a_rows);
    CUtensorMap mA, mB, mY;
    int rc = make_map(&mA, a, p.K, p.M, lda, STAGE_K, p.a_rows, true);
    if (!rc) rc = make_map(&mB, b, p.K, p.N, ldb, STAGE_K, NT, true);
    if (!rc) rc = map_result<T>(p, &mY);
    if (!rc) rc = allow_shared<int8_gemm_kernel<T, NT>>(C::SMEM);
    if (rc) return rc;
    launch_chained(int8_gemm_kernel<T, NT>, dim3((p.N + NT - 1) / NT, (p.M + TILE_M - 1) / TILE_M), C::THREADS, C::smem(p.a_rows), st, mA, mB, mY, p);
    note_product(st);
    return launch_status();
}

template <class T>
int product(Int8Problem p, const int8_t* a, int64_t lda, const int8_t* b, int64_t ldb, cudaStream_t st) {
    if (p.K == 0) {
        launch_chained(int8_no_terms_kernel<T>, (unsigned)(((int64_t)p.M * p.N + 255) / 256 < 148 * 8 ? ((int64_t)p.M * p.N + 255) / 256 : 148 * 8), 256, 0, st, p.bias,
                       static_cast<T*>(p.y), (int64_t)p.M, (int64_t)p.N, p.ldy);
        return launch_status();
    }
    if (pair_eligible(p.M, p.N)) {
        // 128 channels where the tiles fill the pairs that much better (such a tile takes 0.6 of the time of one of 256: 4096 cube 53.1 / 46.7 us
        // in 7 rounds of the one and 4 of the other)
        const int64_t tiles = (int64_t)((p.M + 255) / 256) * ((p.N + 255) / 256), halves = (int64_t)((p.M + 255) / 256) * ((p.N + 127) / 128);
        if ((halves + 73) / 74 * 6 < (tiles + 73) / 74 * 10) return launch_pair<T, 128>(p, a, lda, b, ldb, st);
        return launch_pair<T, 256>(p, a, lda, b, ldb, st);
    }
    // channels of a tile: as many as leave the SMs a tile each
    const int64_t tiles_m = (p.M + TILE_M - 1) / TILE_M;
    if (tiles_m * ((p.N + 127) / 128) >= 100) return launch_tiles<T, 128>(p, a, lda, b, ldb, st);
    if (tiles_m * ((p.N + 63) / 64) >= 100) return launch_tiles<T, 64>(p, a, lda, b, ldb, st);
    return launch_tiles<T, 32>(p, a, lda, b, ldb, st);
}

}  // namespace

// Rows of whole lines of memory for activations that a product converts itself.
int64_t int8_pitch(int64_t k) { return round_up(k > 0 ? k : 1, k < 128 ? 16 : 128); }

int launch_int8_quantize(const void* x, int dtype, int64_t d0, int64_t d1, int64_t ld, int axis, int8_t* q, int64_t pitch, float* scale, cudaStream_t st) {
    if (dtype == HBFP_F32) return quantize_any(static_cast<const float*>(x), d0, d1, ld, axis, q, pitch, scale, st);
    if (dtype == HBFP_BF16) return quantize_any(static_cast<const __nv_bfloat16*>(x), d0, d1, ld, axis, q, pitch, scale, st);
    return quantize_any(static_cast<const __half*>(x), d0, d1, ld, axis, q, pitch, scale, st);
}

int launch_int8_gemm(int64_t M, int64_t N, int64_t K, const int8_t* a, int64_t lda, const float* sa, const int8_t* b, int64_t ldb, const float* sb,
                     const float* bias, void* y, int dtype, int64_t ldy, cudaStream_t st) {
    Int8Problem p{(int)M, (int)N, (int)K, sa, sb, bias, y, ldy, device_status_word(), 0, 0, 0, 0};
    if (!p.status) return HBFP_ERR_CUDA;
    if (dtype == HBFP_F32) return product<float>(p, a, lda, b, ldb, st);
    if (dtype == HBFP_BF16) return product<__nv_bfloat16>(p, a, lda, b, ldb, st);
    return product<__half>(p, a, lda, b, ldb, st);
}

}  // namespace hbfp
