// Attention of many query rows (prompts) over the 4-bit cache on the fifth-generation tensor cores.
//
// A CTA takes 128 rows, or two tiles of 128 where a query is one bfloat16 part (of at most 128 values), of one sequence and KV head: rows = queries
// times the query heads of the KV head. Keys come in tiles of 128 (64 of a 256-wide head). Four warps unpack a tile's keys and values to bfloat16 (exact, see kv4_attend.cuh)
// into swizzled shared memory, once for all rows; one thread issues S = Q K^T and O += P V; a warpgroup per row tile holds a row per thread:
// it reads the scores from tensor memory, keeps the row's maximum and sum in FP32, and writes the probabilities back to tensor memory as the
// bfloat16 operand of the second product (which takes it from there; V's tile is the operand with the values contiguous, keys down its rows).
// With two row tiles the MMAs of one run while the other's softmax does; probabilities then lie in the place of their scores. Where the row
// tiles do not fill the GPU, the CTAs of a cluster share a tile's keys and join their results through shared memory.
//
// Queries and probabilities have as many bfloat16 parts as their type has bits (1, 2 or 3 as in kv4_attend.cuh), each an MMA of its own.
// The maximum is only moved, and O rescaled, when a row's scores exceed it by more than 2^8 (a published technique): probabilities up to 2^8 lose nothing in FP32 and
// bfloat16, and the sum is divided out with the same maximum.
//
// Bound: per 128 keys and 256 rows 2048 cycles of MMA (bfloat16, 128 wide) and as many of exponentials.
#include <cuda.h>

#include <atomic>

#include "kv4_attend.cuh"

namespace hbfp {
namespace {

constexpr float KP_SLACK = 8.0f;
constexpr int KP_SPLITS = 8;                       // CTAs of a cluster at most

template <int D, int NP> struct KpCfg {
    static constexpr int QT = NP == 1 && D <= 128 ? 2 : 1;                 // row tiles of a CTA
    static constexpr int KEYS = D <= 128 ? 128 : 64;                       // keys of a tile
    static constexpr int STAGES = D == 256 && NP == 2 ? 1 : 2;             // tiles of keys, and of values
    static constexpr int ROWS = 128 * QT, HALVES = (D + 63) / 64;          // (96: the last half of the second column of 64 stays unused)
    static constexpr int TILE = HALVES * 16384;                            // 128 rows of D bfloat16, 128-byte columns swizzled
    static constexpr int COLUMN = KEYS * 128, KTILE = HALVES * COLUMN;     // the same of keys or values
    static constexpr int SOFT_WARPS = 4 * QT, FILL_WARPS = 4, THREADS = 32 * (SOFT_WARPS + FILL_WARPS + 4);      // the last four: one issues the MMAs
    // registers by role, out of what the launch has (512 x 128 or 384 x 168)
    static constexpr int REGS_SOFT = QT == 2 ? 168 : 232, REGS_FILL = QT == 2 ? 96 : 120, REGS_MMA = 56;
    static constexpr int REGS_LAUNCH = QT == 2 ? 128 : 168;
    static_assert(65536 / THREADS / 8 * 8 == REGS_LAUNCH, "registers of the launch");
    static_assert(32 * (SOFT_WARPS * REGS_SOFT + FILL_WARPS * REGS_FILL + 4 * REGS_MMA) <= THREADS * REGS_LAUNCH - 512, "register split");
    static_assert(REGS_SOFT >= REGS_LAUNCH && REGS_FILL <= REGS_LAUNCH && REGS_MMA <= REGS_LAUNCH, "setmaxnreg.dec takes no number above the launch's, .inc none below");
    static constexpr int OFF_K = QT * NP * TILE, OFF_V = OFF_K + STAGES * KTILE, OFF_BAR = OFF_V + STAGES * KTILE;
    static constexpr int SMEM = 1024 + OFF_BAR + 512;
    static_assert(SMEM <= 232448, "shared memory");
    static constexpr int OP = D + 4;                                       // FP32 of a row of a share of the keys; behind the rows their maxima and sums
    static_assert(ROWS * (OP * 4 + 8) <= OFF_BAR, "shares");
    // columns of tensor memory
    static constexpr int S_COL = 0, O_COL = D == 256 ? 256 : 128 * QT, P_COL = QT == 2 ? 0 : D == 256 ? 64 : 256;     // scores and results of tile t: + 128 t; parts of P: + 64 p
};

__device__ __forceinline__ void kp_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// The same with A in tensor memory (two neighbours along K to a column).
__device__ __forceinline__ void kp_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// FP32 accumulator, bfloat16 operands, M = 128; B_MN: the columns of B are contiguous, not its contraction.
template <int N, bool B_MN>
__device__ __forceinline__ constexpr uint32_t kp_idesc() {
    return (1u << 4) | (1u << 7) | (1u << 10) | (B_MN ? 1u << 16 : 0u) | ((uint32_t)(N >> 3) << 17) | (8u << 24);
}
// Descriptor of a tile whose columns are contiguous: 64 of them (128 bytes, swizzled) by 8 rows of the contraction an atom, atoms 1024 bytes
// apart along the contraction and COLUMN along the columns.
template <int COLUMN>
__device__ __forceinline__ uint64_t kp_desc_mn(uint32_t addr) {
    return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)(COLUMN >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

// One word of eight values as 16 bytes of bfloat16.
__device__ __forceinline__ uint4 kp_unpack(uint32_t w, uint32_t scale, uint32_t offset) {
    return make_uint4(ka_value(w, scale, offset), ka_value(w >> 4, scale, offset), ka_value(w >> 8, scale, offset), ka_value(w >> 12, scale, offset));
}

// What the rows of a warp see of 32 neighbouring keys: all of them, none, or (bits) some, each row its own. Only the keys around the diagonal, a
// window's edge or a missing page are looked at one by one; with one code for all, the tests cost a whole tile as much as its arithmetic.
enum Seen : int { SEEN_NONE, SEEN_SOME, SEEN_ALL };
struct KpSight {
    int first, last;         // limits of the warp's first and last row
    int limit, window;       // this row's: key p is seen where p <= limit and limit - p < window
    int missing;             // groups of sixteen of the tile that are not there
    __device__ __forceinline__ Seen look(int pos, int c) const {
        const int p = pos + c, gone = missing >> (c >> 4) & 3;
        if (gone == 0 && p + 31 <= first && last - p < window) return SEEN_ALL;
        if (gone == 3 || p > last || first - (p + 31) >= window) return SEEN_NONE;
        return SEEN_SOME;
    }
    __device__ __forceinline__ uint32_t bits(int pos, int c) const {
        const int p = pos + c, to = limit + 1 - p, from = limit - p - window + 1;        // columns [from, to)
        uint32_t b = to <= 0 ? 0u : to >= 32 ? 0xFFFFFFFFu : (1u << to) - 1u;
        b &= from <= 0 ? 0xFFFFFFFFu : from >= 32 ? 0u : 0xFFFFFFFFu << from;
        const int gone = missing >> (c >> 4) & 3;
        if (gone & 1) b &= 0xFFFF0000u;
        if (gone & 2) b &= 0x0000FFFFu;
        return b;
    }
};
// The largest of a row's scores in tensor memory (columns sc ..), WHOLE: of all of the tile.
__device__ __forceinline__ float kp_max32(const uint32_t (&x)[32], float top) {
    float other = -INFINITY;
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
        asm("max.f32 %0, %0, %1, %2;" : "+f"(top) : "f"(__uint_as_float(x[i])), "f"(__uint_as_float(x[i + 1])));
        asm("max.f32 %0, %0, %1, %2;" : "+f"(other) : "f"(__uint_as_float(x[i + 2])), "f"(__uint_as_float(x[i + 3])));
    }
    return fmaxf(top, other);
}
template <int KEYS>
__device__ __forceinline__ float kp_top(uint32_t sc, const KpSight& sight, int pos, bool whole) {
    float top = -INFINITY;
    if (whole) {
        uint32_t v[2][32];
        tc_ld32(sc, v[0]);
#pragma unroll
        for (int c = 0; c < KEYS; c += 32) {
            tc_wait_ld();
            if (c + 32 < KEYS) tc_ld32(sc + c + 32, v[(c / 32 + 1) & 1]);
            top = kp_max32(v[c / 32 & 1], top);
        }
        return top;
    }
#pragma unroll 1
    for (int c = 0; c < KEYS; c += 32) {
        const Seen how = sight.look(pos, c);
        if (how == SEEN_NONE) continue;
        uint32_t v[32];
        tc_ld32(sc + c, v);
        tc_wait_ld();
        if (how == SEEN_SOME) {
            const uint32_t bits = sight.bits(pos, c);
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (!(bits >> i & 1)) v[i] = 0xFF800000u;
        }
        top = kp_max32(v, top);
    }
    return top;
}
// Its probabilities 2^(score * scale2 - m), as parts, to tensor memory (columns pc .., 64 a part); their sum is added to `sum`.
template <int NP, bool SOME>
__device__ __forceinline__ void kp_exp32(uint32_t sc, uint32_t pc, uint64_t k2, uint64_t m2, uint32_t bits, uint64_t (&sum)[2]) {
    uint32_t v[32], x[NP][16];
    tc_ld32(sc, v);
    tc_wait_ld();
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
        float e0, e1;
        unpack2(ffma2(pack2(v[i], v[i + 1]), k2, m2), e0, e1);
        e0 = ka_exp2(e0);
        e1 = ka_exp2(e1);
        if (SOME) {
            if (!(bits >> i & 1)) e0 = 0.f;
            if (!(bits >> (i + 1) & 1)) e1 = 0.f;
        }
        sum[i / 2 & 1] = fadd2(sum[i / 2 & 1], pack2(__float_as_uint(e0), __float_as_uint(e1)));
        uint32_t parts[NP];
        ka_parts<NP>(e0, e1, parts);
#pragma unroll
        for (int p = 0; p < NP; ++p) x[p][i / 2] = parts[p];
    }
#pragma unroll
    for (int p = 0; p < NP; ++p) tc_st16(pc + 64 * p, x[p]);
}
template <int NP, int KEYS>
__device__ __forceinline__ float kp_probabilities(uint32_t sc, uint32_t pc, float scale2, float m, const KpSight& sight, int pos, bool whole) {
    const uint64_t k2 = pack2(__float_as_uint(scale2), __float_as_uint(scale2)), m2 = pack2(__float_as_uint(-m), __float_as_uint(-m));
    uint64_t sum[2] = {0ull, 0ull};
    if (whole) {
#pragma unroll
        for (int c = 0; c < KEYS; c += 32) kp_exp32<NP, false>(sc + c, pc + c / 2, k2, m2, 0u, sum);
    } else {
#pragma unroll 1
        for (int c = 0; c < KEYS; c += 32) {
            const Seen how = sight.look(pos, c);
            if (how == SEEN_NONE) {
                uint32_t zero[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) zero[i] = 0u;
#pragma unroll
                for (int p = 0; p < NP; ++p) tc_st16(pc + 64 * p + c / 2, zero);
            } else if (how == SEEN_SOME) {
                kp_exp32<NP, true>(sc + c, pc + c / 2, k2, m2, sight.bits(pos, c), sum);
            } else {
                kp_exp32<NP, false>(sc + c, pc + c / 2, k2, m2, 0u, sum);
            }
        }
    }
    float s0, s1;
    unpack2(fadd2(sum[0], sum[1]), s0, s1);
    return s0 + s1;
}

// SHARE: clusters of `splits` CTAs share a row tile's keys.
template <int D, int NP, class T, bool SHARE>
__global__ void __launch_bounds__(KpCfg<D, NP>::THREADS, 1)
kv4_prompt_kernel(const Kv4Attend a, int splits) {
    using C = KpCfg<D, NP>;
    extern __shared__ unsigned char smem_dyn[];
    const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    unsigned char* sm = smem_dyn + (base - smem_u32(smem_dyn));
    const uint32_t bars = base + C::OFF_BAR;
    const uint32_t kfull = bars, vfull = bars + 16, kempty = bars + 32, vempty = bars + 48, sfull = bars + 64, pfull = bars + 80, odone = bars + 96, done = bars + 112, qfull = bars + 120;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sm + C::OFF_BAR + 128);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    volatile int* holes = reinterpret_cast<volatile int*>(tmem_slot + 4);        // [4 tiles][4 warps]: groups of sixteen keys that are not there
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    // the tiles with the most keys first
    const int rank = SHARE ? blockIdx.x % splits : 0, item = SHARE ? blockIdx.x / splits : blockIdx.x;
    const int h = item % a.c.heads, b = item / a.c.heads, tile = gridDim.y - 1 - blockIdx.y;
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(kfull + 8 * i, C::FILL_WARPS);
            mbar_init(vfull + 8 * i, C::FILL_WARPS);
            mbar_init(kempty + 8 * i, 1);
            mbar_init(vempty + 8 * i, 1);
            mbar_init(sfull + 8 * i, 1);
            mbar_init(pfull + 8 * i, 4);
            mbar_init(odone + 8 * i, 1);
        }
        mbar_init(done, 1);
        mbar_init(qfull, C::SOFT_WARPS);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    constexpr int MMA_WARP = C::SOFT_WARPS + C::FILL_WARPS;
    if (warp == MMA_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    chain_start();

    const Kv4Seq seq = kv4_seq(a.c, b);
    const int all = seq.n * a.group, r0 = tile * C::ROWS, rows = min(C::ROWS, all - r0);
    if (rows > 0) {
        const int first = seq.length - seq.n;                              // position of the first query
        // keys [lo, hi): hi of the last row, lo of the first; tiles of keys for each row tile
        const int hi = max(0, min(seq.held, first + (r0 + rows - 1) / a.group + 1));
        int lo = a.window ? max(0, first + r0 / a.group - a.window + 1) & ~15 : 0;
        int n[C::QT], most = 0;
#pragma unroll
        for (int t = 0; t < C::QT; ++t) {
            const int last = min(r0 + 128 * t + 127, r0 + rows - 1);
            const int hi_t = 128 * t < rows ? max(0, min(seq.held, first + last / a.group + 1)) : 0;
            n[t] = hi_t > lo ? (hi_t - lo + C::KEYS - 1) / C::KEYS : 0;
            most = max(most, n[t]);
        }
        if (SHARE) {
            const int j0 = (int)((int64_t)most * rank / splits), j1 = (int)((int64_t)most * (rank + 1) / splits);
            lo += j0 * C::KEYS;
            most = j1 - j0;
#pragma unroll
            for (int t = 0; t < C::QT; ++t) n[t] = max(0, min(n[t] - j0, most));
        }
        const float flip = a.scale2 < 0.f ? -1.f : 1.f, scale2 = fabsf(a.scale2);

        if (warp >= C::SOFT_WARPS && warp < MMA_WARP) {
            asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::REGS_FILL));
            // ------------------------------------------------------------ unpacking: a quarter of a tile's keys per warp, a block of 32 values a lane and load
            constexpr int NBLK = D / 32, WIDE = NBLK < 4 ? (NBLK + 1) / 2 * 2 : 4, TURNS = (NBLK + 3) / 4;      // blocks of a row, of it in a load, loads of a row
            constexpr int MINE = C::KEYS / 4, KPL = 32 / WIDE, LOADS = MINE / KPL * TURNS;                    // keys of a warp, of a load; loads
            const int w = warp - C::SOFT_WARPS, blk = (lane >> 3) % WIDE, sub = (lane & 7) + 8 * ((lane >> 3) / WIDE);
            const bool there = NBLK % WIDE == 0 || blk < NBLK;
            uint4 kr[LOADS], vr[LOADS];
            int ke[LOADS], ve[LOADS];
            int64_t row[MINE / 16];
            int gone = 0;
            auto find = [&](int j) {
                gone = 0;
#pragma unroll
                for (int g = 0; g < MINE / 16; ++g) {
                    const int p = lo + j * C::KEYS + MINE * w + 16 * g;
                    row[g] = -1;
                    if (j < most && p < hi) {
                        const int64_t page = kv4_page(a.c, b, p >> a.c.shift);
                        if (page >= 0) row[g] = ((page * a.c.heads + h) << a.c.shift) + (p & (a.c.page - 1));
                        else gone |= 1 << g;
                    } else {                                                 // behind hi, where a row's own position can lie (a length beyond the page table);
                        gone |= 1 << g;                                      // (one test for both cases: other registers, 2 x 2048 tokens 180 -> 184 us)
                    }
                }
            };
            auto load = [&](const uint8_t* mant, const int8_t* exps, uint4 (&m)[LOADS], int (&e)[LOADS]) {
#pragma unroll
                for (int u = 0; u < LOADS; ++u) {
                    const int key = KPL * (u / TURNS) + sub, block = blk + 4 * (u % TURNS);      // of the warp's
                    const int64_t at = MINE == 16 || key < 16 ? row[0] : row[MINE / 16 - 1];
                    m[u] = make_uint4(0u, 0u, 0u, 0u);
                    e[u] = 0;
                    if (at >= 0 && there) {
                        const int64_t line = at + (key & 15);
                        m[u] = __ldg(reinterpret_cast<const uint4*>(mant + line * (D / 2)) + block);
                        e[u] = __ldg(exps + line * NBLK + block);
                    }
                }
            };
            auto store = [&](unsigned char* to, const uint4 (&m)[LOADS], const int (&e)[LOADS]) {
#pragma unroll
                for (int u = 0; u < LOADS; ++u) {
                    const int key = MINE * w + KPL * (u / TURNS) + sub, block = blk + 4 * (u % TURNS), x = kv4_exponent((int8_t)e[u]);
                    const uint32_t scale = ka_scale(x, x), offset = ka_offset(scale);
                    const uint32_t words[4] = {m[u].x, m[u].y, m[u].z, m[u].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int c = 4 * block + i;
                        if (there) *reinterpret_cast<uint4*>(to + (c >> 3) * C::COLUMN + key * 128 + (((c & 7) ^ (key & 7)) << 4)) = kp_unpack(words[i], scale, offset);
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            };
            find(0);
            load(a.c.k_mant, a.c.k_exps, kr, ke);
            load(a.c.v_mant, a.c.v_exps, vr, ve);
            for (int j = 0; j < most; ++j) {
                const int s = j % C::STAGES;
                const uint32_t ph = (uint32_t)((j / C::STAGES) & 1) ^ 1u;
                if (!mbar_wait_warp_soon(kempty + 8 * s, ph, abort_flag, a.c.status, 191)) break;
                if (lane == 0) holes[(j & 3) * 4 + w] = gone;
                store(sm + C::OFF_K + s * C::KTILE, kr, ke);
                if (lane == 0) mbar_arrive(kfull + 8 * s);
                find(j + 1);
                load(a.c.k_mant, a.c.k_exps, kr, ke);
                if (!mbar_wait_warp_soon(vempty + 8 * s, ph, abort_flag, a.c.status, 192)) break;
                store(sm + C::OFF_V + s * C::KTILE, vr, ve);
                if (lane == 0) mbar_arrive(vfull + 8 * s);
                load(a.c.v_mant, a.c.v_exps, vr, ve);
            }
            if (SHARE) cluster_barrier();                             // as the softmax's below
        } else if (warp >= MMA_WARP) {
            asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::REGS_MMA));
            // ------------------------------------------------------------ MMAs
            if (warp == MMA_WARP && elect_one()) {
                auto scores = [&](int t, int j) {
                    const uint32_t d = tmem + C::S_COL + 128 * t, kt = base + C::OFF_K + j % C::STAGES * C::KTILE;
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p)
#pragma unroll
                        for (int i = 0; i < D / 16; ++i) {
                            const uint32_t column = (uint32_t)(i >> 2), off = (uint32_t)(i & 3) * 32u;
                            kp_mma(d, smem_desc_sw128(base + (t * NP + p) * C::TILE + column * 16384u + off), smem_desc_sw128(kt + column * C::COLUMN + off), kp_idesc<C::KEYS, false>(), p < NP - 1 || i > 0);
                        }
                };
                auto values = [&](int t, int j) {
                    const uint32_t d = tmem + C::O_COL + 128 * t, pt = tmem + C::P_COL + 128 * t, vt = base + C::OFF_V + j % C::STAGES * C::KTILE;
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p)
#pragma unroll
                        for (int i = 0; i < C::KEYS / 16; ++i)
                            kp_mma_ts(d, pt + 64 * p + 8 * i, kp_desc_mn<C::COLUMN>(vt + i * 2048), kp_idesc<D, true>(), j > 0 || p < NP - 1 || i > 0);
                };
                bool ok = most == 0 || (mbar_wait_soon(qfull, 0, abort_flag, a.c.status, 189) && mbar_wait_soon(kfull, 0, abort_flag, a.c.status, 193));
                if (ok && most > 0) {
                    tc_fence_after();
#pragma unroll
                    for (int t = 0; t < C::QT; ++t)
                        if (n[t] > 0) {
                            scores(t, 0);
                            tc_commit(sfull + 8 * t);
                        }
                    tc_commit(kempty);
                }
                for (int j = 0; ok && j < most; ++j) {
                    const int s = j % C::STAGES, s1 = (j + 1) % C::STAGES;
                    if (!mbar_wait_soon(vfull + 8 * s, (uint32_t)((j / C::STAGES) & 1), abort_flag, a.c.status, 194)) { ok = false; break; }
                    if (j + 1 < most && !mbar_wait_soon(kfull + 8 * s1, (uint32_t)(((j + 1) / C::STAGES) & 1), abort_flag, a.c.status, 195)) { ok = false; break; }
#pragma unroll
                    for (int t = 0; t < C::QT; ++t) {
                        if (!ok || j >= n[t]) continue;
                        if (!mbar_wait_soon(pfull + 8 * t, (uint32_t)(j & 1), abort_flag, a.c.status, 196)) { ok = false; continue; }
                        tc_fence_after();
                        values(t, j);
                        if (j + 1 < n[t]) {
                            scores(t, j + 1);
                            tc_commit(sfull + 8 * t);
                        } else {
                            tc_commit(odone + 8 * t);
                        }
                    }
                    if (!ok) break;
                    tc_commit(vempty + 8 * s);
                    if (j + 1 < most) tc_commit(kempty + 8 * s1);
                }
                tc_commit(done);
                mbar_wait_soon(done, 0, abort_flag, a.c.status, 197, false);
            }
            __syncwarp();
            if (SHARE) cluster_barrier();
        } else {
            // ------------------------------------------------------------ softmax: a row per thread
            const int t = warp >> 2, quarter = warp & 3, r = 128 * t + quarter * 32 + lane;
            const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16), sc = lanes + C::S_COL + 128 * t, oc = lanes + C::O_COL + 128 * t, pc = lanes + C::P_COL + 128 * t;
            asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::REGS_SOFT));
            // The queries first, in parts (a negative scale is a negative query). A warp brings its own 32 rows: a lane knows where one of them is, all
            // lanes load it. (A row looked up per 16 bytes: 6 us a CTA.)
            const int own = r0 + r, own_query = own / a.group, own_head = h * a.group + own - own_query * a.group;
            constexpr int CPR = D / 8, RPL = 32 / CPR;                      // pieces of eight values of a row, rows of a load
            {
                const bool vec = ((reinterpret_cast<uintptr_t>(a.q) | (uintptr_t)((a.qs.token | a.qs.head) * (int64_t)sizeof(T))) & 15) == 0;
                const int64_t own_at = (seq.first + own_query) * a.qs.token + own_head * a.qs.head;
                const int c = lane % CPR, sub = lane / CPR, row0 = 32 * quarter;
                auto put = [&](int k, const Eight<T>& e) {
                    const int line = row0 + k * RPL + sub;
                    unsigned char* at = sm + t * C::TILE + (c >> 3) * 16384 + line * 128 + (((c & 7) ^ (line & 7)) << 4);
                    if constexpr (NP == 1) {
                        const uint32_t sign = flip < 0.f ? 0x80008000u : 0u;
                        *reinterpret_cast<uint4*>(at) = make_uint4(e.raw[0].x ^ sign, e.raw[0].y ^ sign, e.raw[0].z ^ sign, e.raw[0].w ^ sign);
                    } else {
                        float f[8];
                        e.get(f);
                        uint32_t x[4][NP];
#pragma unroll
                        for (int j = 0; j < 4; ++j) ka_parts<NP>(flip * f[2 * j], flip * f[2 * j + 1], x[j]);
#pragma unroll
                        for (int p = 0; p < NP; ++p) *reinterpret_cast<uint4*>(at + p * C::TILE) = make_uint4(x[0][p], x[1][p], x[2][p], x[3][p]);
                    }
                };
                constexpr int UNR = 32 / RPL < 16 ? 32 / RPL : 16;
#pragma unroll 1
                for (int k0 = 0; k0 < 32 / RPL; k0 += UNR) {
                    Eight<T> e[UNR];
                    if (vec) {
#pragma unroll
                        for (int k = 0; k < UNR; ++k) {
                            const int line = (k0 + k) * RPL + sub;
                            const int64_t at = __shfl_sync(0xffffffffu, own_at, line);
                            e[k].zero();
                            if ((32 % CPR == 0 || sub < RPL) && 128 * t + row0 + line < rows) e[k].load(reinterpret_cast<const T*>(a.q) + at + 8 * c);
                        }
                    } else {
#pragma unroll
                        for (int k = 0; k < UNR; ++k) {
                            const int line = (k0 + k) * RPL + sub;
                            const int64_t at = __shfl_sync(0xffffffffu, own_at, line);
                            e[k].zero();
                            if ((32 % CPR == 0 || sub < RPL) && 128 * t + row0 + line < rows) e[k].load_part(reinterpret_cast<const T*>(a.q) + at + 8 * c, 8);
                        }
                    }
#pragma unroll
                    for (int k = 0; k < UNR; ++k)
                        if (32 % CPR == 0 || sub < RPL) put(k0 + k, e[k]);
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(qfull);

            const int limit = r < rows ? first + own_query : first + (r0 + rows - 1) / a.group, window = a.window ? a.window : 1 << 30;
            // rows of this warp: the first's limit and the last's, for a look at whole tiles
            const int limit0 = __reduce_min_sync(0xffffffffu, limit), limit1 = __reduce_max_sync(0xffffffffu, limit);
            float m = -INFINITY, l = 0.f;
            bool ok = true;
            const int mine = t == 0 ? n[0] : n[C::QT - 1];
            for (int j = 0; j < mine; ++j) {
                if (!mbar_wait_warp_soon(sfull + 8 * t, (uint32_t)(j & 1), abort_flag, a.c.status, 198)) { ok = false; break; }
                tc_fence_after();
                const int pos = lo + j * C::KEYS;
                constexpr int G = C::KEYS / 64;
                const int missing = holes[(j & 3) * 4] | holes[(j & 3) * 4 + 1] << G | holes[(j & 3) * 4 + 2] << 2 * G | holes[(j & 3) * 4 + 3] << 3 * G;
                const KpSight sight{limit0, limit1, limit, window, missing};
                const bool whole = pos + C::KEYS - 1 <= limit0 && limit1 - pos < window && missing == 0;
                const float top = kp_top<C::KEYS>(sc, sight, pos, whole);
                const float top2 = top == -INFINITY ? top : top * scale2;
                const bool move = top2 > m + KP_SLACK || (m == -INFINITY && top2 != -INFINITY);
                if (__any_sync(0xffffffffu, move)) {
                    const float f = move ? ka_exp2(m - top2) : 1.f;        // m = -inf: 0
                    if (move) m = top2;
                    l *= f;
                    if (j > 0) {
#pragma unroll
                        for (int c = 0; c < D; c += 32) {
                            uint32_t v[32];
                            tc_ld32(oc + c, v);
                            tc_wait_ld();
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
                            tc_st32(oc + c, v);
                        }
                        tc_wait_st();
                    }
                }
                const float m_use = m == -INFINITY ? 0.f : m;
                l += kp_probabilities<NP, C::KEYS>(sc, pc, scale2, m_use, sight, pos, whole);
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(pfull + 8 * t);
            }
            // ---- the row's result
            if (ok && mine > 0) ok = mbar_wait_warp_soon(odone + 8 * t, 0, abort_flag, a.c.status, 199);
            if constexpr (SHARE) {
                // This CTA's share of the row to shared memory (all of the MMAs that read keys, values and queries have ended), joined with those of the
                // cluster's other CTAs, a share of the elements by each.
                asm volatile("bar.sync 1, %0;" ::"n"(32 * C::SOFT_WARPS) : "memory");
                float* const os = reinterpret_cast<float*>(sm);
                float2* const ml = reinterpret_cast<float2*>(os + C::ROWS * C::OP);
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < D; c += 32) {
                    uint32_t v[32];
                    if (ok && mine > 0) {
                        tc_ld32(oc + c, v);
                        tc_wait_ld();
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = 0u;
                    }
#pragma unroll
                    for (int i = 0; i < 32; i += 4) *reinterpret_cast<uint4*>(os + r * C::OP + c + i) = make_uint4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                }
                ml[r] = make_float2(m, l);
                cluster_barrier();
                const uint32_t os_at = smem_u32(os), ml_at = smem_u32(ml);
                const bool vec = ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)((a.os.token | a.os.head) * (int64_t)sizeof(T))) & 15) == 0;
                for (int i = rank * 32 * C::SOFT_WARPS + threadIdx.x; i < rows * (D / 4); i += splits * 32 * C::SOFT_WARPS) {
                    const int line = i / (D / 4), d = 4 * (i - line * (D / 4));
                    float top = -INFINITY, sum = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
                    float2 x[KP_SPLITS];
                    float4 o[KP_SPLITS];
#pragma unroll
                    for (int sp = 0; sp < KP_SPLITS; ++sp)
                        if (sp < splits) {
                            x[sp] = ka_shared2(map_to_rank(ml_at + line * 8, sp));
                            o[sp] = ka_shared4(map_to_rank(os_at + (line * C::OP + d) * 4, sp));
                            top = fmaxf(top, x[sp].x);
                        }
                    if (top == -INFINITY) top = 0.f;
#pragma unroll
                    for (int sp = 0; sp < KP_SPLITS; ++sp)
                        if (sp < splits) {
                            const float f = ka_exp2(x[sp].x - top);
                            sum += f * x[sp].y;
                            y[0] += f * o[sp].x; y[1] += f * o[sp].y; y[2] += f * o[sp].z; y[3] += f * o[sp].w;
                        }
                    const float inv = sum > 0.f ? __frcp_rn(sum) : 0.f;    // a row that sees no key: zeros
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = sum == 0.f ? 0.f : y[e] * inv;
                    const int query = (r0 + line) / a.group, head = h * a.group + r0 + line - query * a.group;
                    T* const dst = reinterpret_cast<T*>(a.out) + (seq.first + query) * a.os.token + head * a.os.head + d;
                    if (vec) {
                        store_four(dst, y);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) dst[e] = from_f32<T>(y[e]);
                    }
                }
            } else if (ok) {
                tc_fence_after();
                const float inv = l > 0.f ? __frcp_rn(l) : 0.f;            // a row that sees no key: zeros
                // Through shared memory, in the place of the queries (all MMAs that read them have ended), out along the rows: 16 bytes of 32
                // rows an instruction took 2 us.
                constexpr int V = 16 / sizeof(T), PIECES = D / V, LINE = (PIECES + 7) / 8 * 128, RPS = 32 / PIECES > 0 ? 32 / PIECES : 1;
                unsigned char* area = sm + (t * 4 + quarter) * 32 * LINE;
                // (a tile without a key has no MMAs to wait for, but its other warps may still be bringing queries)
                if (mine == 0) asm volatile("bar.sync %0, 128;" ::"r"(2 + t) : "memory");
#pragma unroll
                for (int c = 0; c < D; c += 32) {
                    uint32_t v[32];
                    if (mine > 0) {
                        tc_ld32(oc + c, v);
                        tc_wait_ld();
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = 0u;
                    }
#pragma unroll
                    for (int i = 0; i < 32; i += V) {
                        float y[V];
#pragma unroll
                        for (int k = 0; k < V; ++k) y[k] = l == 0.f ? 0.f : __uint_as_float(v[i + k]) * inv;
                        store_piece(reinterpret_cast<T*>(area + lane * LINE + ((((c + i) / V) ^ (lane & 7)) << 4)), y);
                    }
                }
                __syncwarp();
                const bool vec = ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)((a.os.token | a.os.head) * (int64_t)sizeof(T))) & 15) == 0;
                const int64_t own_out = (seq.first + own_query) * a.os.token + own_head * a.os.head;
                const int row0 = 128 * t + 32 * quarter;
#pragma unroll 4
                for (int k = 0; k < 32; k += RPS) {
                    const int line = k + lane / PIECES % RPS;
                    const int64_t at = __shfl_sync(0xffffffffu, own_out, line);
                    if (row0 + line >= rows || (PIECES < 32 && lane / PIECES >= RPS)) continue;
#pragma unroll
                    for (int c = lane % PIECES; c < PIECES; c += 32) {
                        const uint4 y = *reinterpret_cast<const uint4*>(area + line * LINE + ((c ^ (line & 7)) << 4));
                        T* dst = reinterpret_cast<T*>(a.out) + at + c * V;
                        if (vec) {
                            *reinterpret_cast<uint4*>(dst) = y;
                        } else {
                            const T* e = reinterpret_cast<const T*>(&y);
#pragma unroll
                            for (int i = 0; i < V; ++i) dst[i] = e[i];
                        }
                    }
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (SHARE && rows > 0) cluster_barrier();                         // nobody reads this CTA's share any more
    if (warp == MMA_WARP) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
    }
}

// CTAs that share the keys of a row tile: as many as the GPU has room for, where each has a tile of keys. 32 tokens of 4 x 8 heads of 128 (bfloat16)
// behind 16384 keys 263 us with one CTA a row tile, so 43; 1024 keys 22.6 / 12.1, with two tiles of keys each at least 13.9. (A table with room for more
// than there is: 100 keys 8.5 / 11.8.)
template <int D, int NP, class T>
int kp_splits(const Kv4Attend& a, int64_t tiles, int* splits) {
    using C = KpCfg<D, NP>;
    static std::atomic<int> resident[MAX_DEVICES][4];                      // clusters of 1, 2, 4, 8
    const int dev = current_device();
    if (dev < 0) return HBFP_ERR_CUDA;
    const int64_t ctas = tiles * a.c.heads * a.c.sequences, keys = kv4_keys(a);
    *splits = 1;
    for (int i = 1; (1 << i) <= KP_SPLITS && keys >= (128ll << i) && (ctas << i) <= sm_count(); ++i) {
        int room = resident[dev][i].load(std::memory_order_acquire);
        if (!room) {
            cudaLaunchConfig_t cfg = {};
            cudaLaunchAttribute at[1];
            at[0].id = cudaLaunchAttributeClusterDimension;
            at[0].val.clusterDim.x = 1 << i; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
            cfg.gridDim = dim3(1 << i);
            cfg.blockDim = dim3(C::THREADS);
            cfg.dynamicSmemBytes = C::SMEM;
            cfg.attrs = at;
            cfg.numAttrs = 1;
            HBFP_CUDA_OK(cudaOccupancyMaxActiveClusters(&room, kv4_prompt_kernel<D, NP, T, true>, &cfg));
            if (room < 1) return HBFP_ERR_CUDA;
            resident[dev][i].store(room, std::memory_order_release);
        }
        if (ctas > room) break;
        *splits = 1 << i;
    }
    return HBFP_OK;
}

template <int D, int NP, class T>
int kp_launch(const Kv4Attend& a, cudaStream_t st) {
    using C = KpCfg<D, NP>;
    const int64_t rows = (int64_t)a.c.most * a.group, tiles = (rows + C::ROWS - 1) / C::ROWS;
    int splits = 1;
    int rc = allow_shared<kv4_prompt_kernel<D, NP, T, false>>(C::SMEM);
    if (!rc) rc = allow_shared<kv4_prompt_kernel<D, NP, T, true>>(C::SMEM);
    if (!rc) rc = kp_splits<D, NP, T>(a, tiles, &splits);
    if (rc) return rc;
    launch_chained_clusters(splits > 1 ? kv4_prompt_kernel<D, NP, T, true> : kv4_prompt_kernel<D, NP, T, false>, splits, dim3((unsigned)(a.c.heads * a.c.sequences * splits), (unsigned)tiles), C::THREADS, C::SMEM, st, true, a, splits);
    note_product(st);
    return launch_status();
}
template <int NP, class T>
int kp_launch_dim(const Kv4Attend& a, cudaStream_t st) {
    if (a.c.dim == 64) return kp_launch<64, NP, T>(a, st);
    if (a.c.dim == 96) return kp_launch<96, NP, T>(a, st);
    if constexpr (NP < 3)
        if (a.c.dim == 256) return kp_launch<256, NP, T>(a, st);
    return kp_launch<128, NP, T>(a, st);
}

}  // namespace

// More rows than the widest tile of the kernel of few rows (32, of a 256-wide head 16), which reads the keys once for each such tile but spreads any
// number of tiles over all SMs, where a row tile here is no more than a cluster's. An SM's time for a key, of such a tile there and of a CTA's rows
// here, in ns: 128 wide 13 / 18 (bfloat16), 19 / 24 (binary16), 24 / 37 (FP32); 96 wide 13 / 19, 18 / 24, 23 / 34; 256 wide 18 / 30, 23 / 61. Up to 8192
// keys (1024 where the ratio is above two, 256 wide binary16) it is the launches that count, one here. Measured, 8 heads, bfloat16, few / here: 40 rows of 128 in 32 sequences with 4096 keys 179 / 145 us, in one
// with 4096 20.5 / 16.5, with 32768 53 / 76; 96 rows 273 / 145, 21.6 / 17.7, 74 / 77. 512 rows of 32 sequences with 2048 keys, 96 wide 641 / 167, 256 wide
// 1813 / 422. FP32 queries of 256 have no room in shared memory.
bool kv4_prompt_eligible(const Kv4Attend& a, int dtype) {
    const bool wide = a.c.dim == 256;
    const int64_t rows = (int64_t)a.c.most * a.group, each = dtype == HBFP_BF16 && !wide ? 256 : 128, few = wide ? 16 : 32;
    const int64_t items = (int64_t)a.c.heads * a.c.sequences;
    if ((wide && dtype == HBFP_F32) || rows <= few || (rows + 127) / 128 > 65535 || items > (1ll << 27)) return false;
    constexpr int64_t SMS = 148;
    const int64_t ctas = (rows + each - 1) / each * items, waves = (ctas + SMS - 1) / SMS;
    const int64_t ratio = !wide ? 14 : dtype == HBFP_BF16 ? 17 : 27;       // of the two times, in tenths
    int splits = 1;
    while (splits < KP_SPLITS && ctas * splits * 2 <= SMS) splits *= 2;
    return kv4_keys(a) <= (ratio < 20 ? 8192 : 1024) || ratio * SMS * waves <= 10 * splits * items * ((rows + few - 1) / few);
}

int launch_kv4_prompt(const Kv4Attend& a, int dtype, cudaStream_t st) {
    if (dtype == HBFP_F32) return kp_launch_dim<3, float>(a, st);
    if (dtype == HBFP_BF16) return kp_launch_dim<1, __nv_bfloat16>(a, st);
    return kp_launch_dim<2, __half>(a, st);
}

}  // namespace hbfp
