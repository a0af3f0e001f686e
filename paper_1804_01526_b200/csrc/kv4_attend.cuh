// Attention of a few query rows over the 4-bit cache, with warp-level bfloat16 MMAs.
//
// For one sequence and one KV head the rows are the call's queries times the query heads that share the head. Scores are computed
// transposed, S^T = K Q^T (16 keys x 8 rows an MMA), and so is the result, O^T = V^T P^T: both wide operands come from the cache, a
// lane's share of a key or value row is a run of words that it loads with one instruction and unpacks in registers, and eight rows
// fill the narrow side, where the usual order would pad a single token's rows to sixteen. The order of the 16 values along an MMA's
// contraction is free as long as both operands agree, so the unpacked pairs need no shuffling; scores become the second product's
// operand by one 8 x 8 transpose (movmatrix).
//
// A cached value, nibble * 2^s, is a bfloat16 exactly: (128 + nibble) is put together with one logical instruction (a published technique) and
// fma(128 + nibble, 2^s, -136 * 2^s) rounds nothing. Queries and probabilities are split into as many bfloat16 parts as their type
// has bits (1 for bfloat16, 2 for binary16, 3 for FP32: of a query nothing is left, of a probability 2^-8, 2^-16, 2^-24), so
// products are exact and sums FP32. Softmax in base 2, running maximum and sum in FP32.
//
// Bound: reading the cache, dim / 2 + dim / 32 bytes per key and head and as much for values. Warps take 64 keys each in turn (32 where
// a tile has more than eight rows, 16 of a 256-wide head) and keep their own maximum and sum; the CTA joins them once at the end of its keys. Keys, values and exponents of a warp's
// next chunks come by bulk copies into its own ring of shared memory (rows of a page and head are one run of memory), issued by one
// lane, so that a warp has its next chunks in flight without a register or an address for them (64 keys at a time with 12 warps an SM 94.6 us for
// 64 sequences of up to 8192 tokens, 32 with 16 warps 97.4; one sequence of 131072 in binary16 52.4 / 57.8).
//
// Split. Sequences differ in length and the host does not know the lengths, so a launch with long keys has as many CTAs as the GPU
// holds at a time and each takes an equal share of all units (a chunk for each warp, of one sequence, head and row tile), found by adding up the
// lengths itself. A tile whose keys end up in several CTAs leaves FP32 parts (at most two a CTA) that a second launch joins in
// ascending order: the same result every time.
#pragma once

#include <atomic>

#include "kv4.cuh"
#include "tc_ptx.cuh"

namespace hbfp {

struct Kv4Attend {
    Kv4Args c;
    const void* q;
    Kv4Rows qs;
    void* out;
    Kv4Rows os;
    int group;              // query heads of a KV head
    int window;             // 0: none
    float scale2;           // scale * log2(e)
    int tiles;              // row tiles of a sequence at most
    float* partial;         // split launches: [2 * CTAs][rows of a tile][dim], then [2 * CTAs][rows][2] (maximum, sum)
    int ctas;
};

// Keys that a sequence's rows see at most, of what the host knows (whole chunks of 64 from the window's edge on).
inline int64_t kv4_keys(const Kv4Attend& a) {
    const int64_t cap = (int64_t)a.c.table_pages << a.c.shift, near = (int64_t)a.window + a.c.most + 63;
    return a.window && near < cap ? near : cap;
}

int launch_kv4_attend_f32(const Kv4Attend& a, cudaStream_t st, size_t* bytes);
int launch_kv4_attend_bf16(const Kv4Attend& a, cudaStream_t st, size_t* bytes);
int launch_kv4_attend_f16(const Kv4Attend& a, cudaStream_t st, size_t* bytes);
// Many rows (kv4_prompt.cu); no workspace.
bool kv4_prompt_eligible(const Kv4Attend& a, int dtype);
int launch_kv4_prompt(const Kv4Attend& a, int dtype, cudaStream_t st);

namespace {

constexpr int KA_WARPS = 4, KA_THREADS = 32 * KA_WARPS, KA_SPLITS = 8;      // KA_SPLITS: CTAs of a cluster at most

template <int D, int NT> struct KaDim {
    static constexpr int NB = D / 32;                      // blocks of a row; words of a key row that a lane takes
    static constexpr int VW = (D + 63) / 64;               // words of a value row that a lane takes (96: as 128, the last lanes none)
    static constexpr int CH = D > 128 ? 16 : NT == 1 ? 64 : 32;      // keys of a warp at a time
    static constexpr int UNIT = CH * KA_WARPS;             // keys of a CTA at a time
    static constexpr int STEPS = D / 16;                   // MMA steps along a key row
    static constexpr int KE = D == 128 || D == 64 ? 1 : 2; // exponents of a lane's key words
    // a chunk in shared memory: keys, values, exponents of the keys, of the values
    static constexpr int MANT = CH * D / 2, EXPS = CH * NB, CHUNK = 2 * (MANT + EXPS), STAGES = CH == 64 ? 2 : 3;
    static_assert(MANT % 16 == 0 && EXPS % 16 == 0, "bulk copies");
};
template <int D, int NP, int NT> struct KaShared {                      // queries; the rings, then the warps' results in their place; maxima and sums; barriers
    static constexpr int Q = NP * NT * KaDim<D, NT>::STEPS * 256, OP = D + 4;
    static constexpr int RING = KA_WARPS * KaDim<D, NT>::STAGES * KaDim<D, NT>::CHUNK, O = KA_WARPS * 8 * NT * OP * 4;
    static constexpr int ML = Q + (RING > O ? RING : O), BAR = ML + (KA_WARPS + 1) * 8 * NT * 8, BYTES = BAR + KA_WARPS * KaDim<D, NT>::STAGES * 8 + 16;
};

__device__ __forceinline__ void ka_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint2 b) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b.x), "r"(b.y));
}
__device__ __forceinline__ uint32_t ka_transpose(uint32_t v) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}
// 2^s of two neighbours as a pair of bfloat16 ((s + 127) << 7 in each half), and -136 * 2^s
__device__ __forceinline__ uint32_t ka_scale(int s0, int s1) { return (uint32_t)(s0 * 0x80 + (s1 * 0x800000 + 0x3F803F80)); }
__device__ __forceinline__ uint32_t ka_offset(uint32_t scale) {
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(scale), "r"(0xC308C308u));
    return d;
}
// The pair of values whose nibbles are the low four bits of w's halfwords.
__device__ __forceinline__ uint32_t ka_value(uint32_t w, uint32_t scale, uint32_t offset) {
    uint32_t d, n;
    asm("lop3.b32 %0, %1, 0x000F000F, 0x43004300, 0xEA;" : "=r"(n) : "r"(w));
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(n), "r"(scale), "r"(offset));
    return d;
}
// The parts of two FP32 values as pairs of bfloat16: the first the values rounded, each later one what is left.
template <int NP>
__device__ __forceinline__ void ka_parts(float a, float b, uint32_t (&d)[NP]) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        d[i] = pack_pair(a, b, (const __nv_bfloat16*)nullptr);
        a -= __uint_as_float(d[i] << 16);
        b -= __uint_as_float(d[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ float ka_exp2(float x) {
    float d;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(x));
    return d;
}

template <int N>
__device__ __forceinline__ void ka_load_words(uint32_t at, uint32_t (&w)[N]) {      // from shared memory
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3]) : "r"(at + 4 * i));
    } else if constexpr (N == 2) {
        asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[i]) : "r"(at + 4 * i));
    }
}
__device__ __forceinline__ int ka_load_byte(uint32_t at) {
    int v;
    asm volatile("ld.shared.s8 %0, [%1];" : "=r"(v) : "r"(at));
    return v;
}
// size bytes of global memory to shared memory, counted on the barrier; all of them multiples of 16
__device__ __forceinline__ void ka_copy(uint32_t dst, const void* src, uint32_t size, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(size), "r"(bar) : "memory");
}

// From the shared memory of any CTA of the cluster.
__device__ __forceinline__ float2 ka_shared2(uint32_t at) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ float4 ka_shared4(uint32_t at) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}

// A warp's ring: its barriers and which phase each is in.
struct KaRing {
    uint32_t bars, phases;
    volatile int* abort_flag;
};

// The keys [lo, hi) that the rows of a tile see, lo rounded down to a whole chunk.
struct KaRange { int lo, hi; };

// Row tile `tile` of (sequence b, head h): keys [lo, hi), result into `out` (slot < 0) or as a part. splits: the CTAs of a cluster have a share of the
// tile's keys each and join them here.
template <int D, int NP, int NT, class T>
__device__ __forceinline__ void ka_tile(const Kv4Attend& a, int b, const Kv4Seq& seq, int h, int tile, KaRange range, int slot, int splits, unsigned char* sm, KaRing& ring) {
    using C = KaDim<D, NT>;
    constexpr int RT = 8 * NT, MT = C::CH / 16, TILES = 4 * C::VW;        // TILES: 16-row tiles of V^T
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int rows = min(RT, seq.n * a.group - tile * RT), r0 = tile * RT;
    const float flip = a.scale2 < 0.f ? -1.f : 1.f, scale2 = fmaxf(fabsf(a.scale2), 1.4e-45f);      // a negative scale is a negative query; 0 times an unseen -inf would be NaN
    uint2* qs = reinterpret_cast<uint2*>(sm);                             // [NP][NT][STEPS][32]
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");          // (copies follow where results were written)
    __syncthreads();                                                      // the tile before is through with shared memory
    // ---- the ring. Lanes 0 to 3 each ask for one of a chunk's arrays (keys, values, their exponents); every lane knows the page of the
    // chunk after the last one asked for. gone: which sixteens of each stage's chunk are not there.
    const uint32_t base = smem_u32(sm) + KaShared<D, NP, NT>::Q + warp * C::STAGES * C::CHUNK;
    constexpr int GROUPS = C::CH / 16, ALL = (1 << GROUPS) - 1;
    const int mine = lane & 3;
    const uint32_t line = mine < 2 ? D / 2 : C::NB, to_mine = (mine & 1) * (mine < 2 ? C::MANT : C::EXPS) + (mine < 2 ? 0 : 2 * C::MANT);
    const int64_t page_bytes = ((int64_t)a.c.heads << a.c.shift) * line;
    const char* const array = reinterpret_cast<const char*>(mine == 0 ? (const void*)a.c.k_mant : mine == 1 ? (const void*)a.c.v_mant : mine == 2 ? (const void*)a.c.k_exps
                                                                                                                                       : (const void*)a.c.v_exps) +
                              ((int64_t)h << a.c.shift) * line;
    // a chunk in pages of fewer rows: a page for each of its pieces
    const int piece = min(C::CH, a.c.page), pieces = C::CH / piece, groups = piece / 16;
    auto page_of = [&](int p) { return p < range.hi ? (int)kv4_page(a.c, b, p >> a.c.shift) : -1; };
    auto ask = [&](int p, int id, int stage) {
        const uint32_t at = base + stage * C::CHUNK + to_mine, bar = ring.bars + 8 * stage;
        int ids[GROUPS], keys = 0, gone = 0;
#pragma unroll
        for (int i = 0; i < GROUPS; ++i)
            if (i < pieces) {
                ids[i] = i == 0 ? id : page_of(p + i * piece);
                if (ids[i] >= 0) keys += piece;
                else gone |= ((1 << groups) - 1) << (i * groups);
            }
        if (lane == 0) mbar_expect_tx(bar, (uint32_t)keys * (2 * (D / 2 + C::NB)));
        __syncwarp();
        if (lane < 4)
#pragma unroll
            for (int i = 0; i < GROUPS; ++i)
                if (i < pieces && ids[i] >= 0)
                    ka_copy(at + i * piece * line, array + ids[i] * page_bytes + (uint32_t)((p + i * piece) & (a.c.page - 1)) * line, piece * line, bar);
        return gone;
    };
    const int start = range.lo + warp * C::CH;
    int gone = 0;
#pragma unroll
    for (int i = 0; i < C::STAGES - 1; ++i) {
        const int p = start + i * C::UNIT;
        if (p < range.hi) gone |= ask(p, page_of(p), i) << (GROUPS * i);
    }
    int next_id = page_of(start + (C::STAGES - 1) * C::UNIT);
    // ---- the queries, while the first keys come
    const bool vec_q = ((reinterpret_cast<uintptr_t>(a.q) | (uintptr_t)((a.qs.token | a.qs.head) * (int64_t)sizeof(T))) & (4 * sizeof(T) - 1)) == 0;
    constexpr int QUERIES = NT * C::STEPS * 32, AHEAD = QUERIES >= 4 * KA_THREADS ? 4 : (QUERIES + KA_THREADS - 1) / KA_THREADS;      // asked for together
#pragma unroll 1
    for (int i0 = threadIdx.x; i0 < QUERIES; i0 += AHEAD * KA_THREADS) {
        Four<T> e[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int i = i0 + k * KA_THREADS, l = i & 31, step = (i >> 5) % C::STEPS, nt = (i >> 5) / C::STEPS, r = 8 * nt + (l >> 2);
            e[k].zero();
            if (i < QUERIES && r < rows) {
                const int query = (r0 + r) / a.group, gh = (r0 + r) - query * a.group;
                const T* src = reinterpret_cast<const T*>(a.q) + (seq.first + query) * a.qs.token + (h * a.group + gh) * a.qs.head + ((l & 3) * C::NB + (step >> 1)) * 8 + 4 * (step & 1);
                if (vec_q) e[k].load(src);
                else e[k].load_each(src);
            }
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int i = i0 + k * KA_THREADS;
            if (QUERIES % (AHEAD * KA_THREADS) && i >= QUERIES) break;
            float f[4];
            e[k].get(f);
            uint32_t x[NP], y[NP];
            ka_parts<NP>(flip * f[0], flip * f[1], x);
            ka_parts<NP>(flip * f[2], flip * f[3], y);
#pragma unroll
            for (int p = 0; p < NP; ++p) qs[p * QUERIES + i] = make_uint2(x[p], y[p]);
        }
    }
    // positions of this lane's rows (columns 2 t and 2 t + 1 of every eight): keys up to there are seen
    int limit[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) limit[nt][c] = seq.length - seq.n + (r0 + min(8 * nt + 2 * t + c, rows - 1)) / a.group;
    const int first_limit = seq.length - seq.n + r0 / a.group, last_limit = seq.length - seq.n + (r0 + rows - 1) / a.group;
    const int window = a.window ? a.window : 1 << 30;
    __syncthreads();

    float o[TILES][NT][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int i = 0; i < TILES; ++i)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][nt][e] = 0.f;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) { m[nt][c] = -INFINITY; l[nt][c] = 0.f; }

    // row of this lane's keys g and g + 8 in the chunk: neighbours are swapped in every other pair, so that neither the keys' nor the values'
    // accesses meet in a bank more than twice
    const int gk = g ^ ((g >> 1) & 1), ke0 = (t * C::NB) >> 2, ve0 = (g * C::VW) >> 2;
    const bool has_value = D % 64 == 0 || g * C::VW < D / 8;
    int stage = 0;
    bool ok = true;
    int pos = start;
    for (; pos < range.hi; pos += C::UNIT) {
        {
            const int p = pos + (C::STAGES - 1) * C::UNIT, to = stage == 0 ? C::STAGES - 1 : stage - 1;
            if (p < range.hi) {
                gone = (gone & ~(ALL << (GROUPS * to))) | ask(p, next_id, to) << (GROUPS * to);
                next_id = page_of(p + C::UNIT);
            }
        }
        const int missing = gone >> (GROUPS * stage) & ALL;
        ok = mbar_wait_warp_soon(ring.bars + 8 * stage, ring.phases >> stage & 1, ring.abort_flag, a.c.status, 187);
        if (!ok) break;
        ring.phases ^= 1u << stage;
        const uint32_t at = base + stage * C::CHUNK;
        const bool whole = pos + C::CH <= range.hi && pos + C::CH - 1 <= first_limit && last_limit - pos < window && missing == 0;
        if (!whole) {
            // rows that nobody appended may hold any exponent: brought into range, so that a probability of zero leaves nothing of them
            for (int i = lane; i < 2 * C::EXPS / 4; i += 32) {
                uint32_t e;
                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(e) : "r"(at + 2 * C::MANT + 4 * i));
                e = __vmins4(__vmaxs4(e, 0xC1C1C1C1u), (uint32_t)KV4_MAX_EXP * 0x01010101u);
                asm volatile("st.shared.b32 [%0], %1;" ::"r"(at + 2 * C::MANT + 4 * i), "r"(e) : "memory");
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the next copy to this place comes after
            __syncwarp();
        }
        uint32_t kw[MT][2][C::NB];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) ka_load_words<C::NB>(at + (16 * i + 8 * hh + gk) * (D / 2) + t * C::NB * 4, kw[i][hh]);
        // ---- S^T = K Q^T
        float s[MT][NT][4];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[i][nt][e] = 0.f;
        uint32_t sc[MT][2][C::KE], of[MT][2][C::KE];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int hh = 0; hh < 2; ++hh)
#pragma unroll
                for (int e = 0; e < C::KE; ++e) {
                    const int x = ka_load_byte(at + 2 * C::MANT + (16 * i + 8 * hh + gk) * C::NB + min(ke0 + e, C::NB - 1));
                    sc[i][hh][e] = ka_scale(x, x);
                    of[i][hh][e] = ka_offset(sc[i][hh][e]);
                }
#pragma unroll
        for (int j = 0; j < C::NB; ++j) {
            // which of the lane's exponents: all words in one block, or (256) four in each, or (96) split by lane
            uint32_t scj[MT][2], ofj[MT][2];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const bool second = C::KE == 2 && ((t * C::NB + j) >> 2) != ke0;
                    scj[i][hh] = second ? sc[i][hh][C::KE - 1] : sc[i][hh][0];
                    ofj[i][hh] = second ? of[i][hh][C::KE - 1] : of[i][hh][0];
                }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint32_t f[MT][4];
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    f[i][0] = ka_value(kw[i][0][j] >> (8 * u), scj[i][0], ofj[i][0]);
                    f[i][1] = ka_value(kw[i][1][j] >> (8 * u), scj[i][1], ofj[i][1]);
                    f[i][2] = ka_value(kw[i][0][j] >> (8 * u + 4), scj[i][0], ofj[i][0]);
                    f[i][3] = ka_value(kw[i][1][j] >> (8 * u + 4), scj[i][1], ofj[i][1]);
                }
#pragma unroll
                for (int p = NP - 1; p >= 0; --p)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const uint2 q = qs[((p * NT + nt) * C::STEPS + 2 * j + u) * 32 + lane];
#pragma unroll
                        for (int i = 0; i < MT; ++i) ka_mma(s[i][nt], f[i][0], f[i][1], f[i][2], f[i][3], q);
                    }
            }
        }

        // ---- softmax in base 2: this lane holds keys gk and gk + 8 of every sixteen for its rows
        if (!whole)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int p = pos + 16 * i + gk + 8 * (e >> 1);
                        if ((missing >> i & 1) || p >= range.hi || p > limit[nt][e & 1] || limit[nt][e & 1] - p >= window) s[i][nt][e] = -INFINITY;
                    }
        float top[NT][2];
        bool grows = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float x = fmaxf(s[0][nt][c], s[0][nt][c + 2]);
#pragma unroll
                for (int i = 1; i < MT; ++i) x = fmaxf(x, fmaxf(s[i][nt][c], s[i][nt][c + 2]));
                top[nt][c] = x = x * scale2;
                grows |= x > m[nt][c];
            }
        if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float x = fmaxf(m[nt][c], top[nt][c]);
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
                    const float f = x == -INFINITY ? 0.f : ka_exp2(m[nt][c] - x);
                    m[nt][c] = x;
                    l[nt][c] *= f;
#pragma unroll
                    for (int i = 0; i < TILES; ++i) { o[i][nt][c] *= f; o[i][nt][c + 2] *= f; }
                }
        }
        uint2 pb[MT][NT][NP];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float m0 = m[nt][0] == -INFINITY ? 0.f : m[nt][0], m1 = m[nt][1] == -INFINITY ? 0.f : m[nt][1];
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                float x0[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x0[e] = ka_exp2(__fmaf_rn(s[i][nt][e], scale2, e & 1 ? -m1 : -m0));
                const float p0 = x0[0], p1 = x0[1], p2 = x0[2], p3 = x0[3];
                l[nt][0] += p0 + p2;
                l[nt][1] += p1 + p3;
                uint32_t x[NP], y[NP];
                ka_parts<NP>(p0, p1, x);
                ka_parts<NP>(p2, p3, y);
#pragma unroll
                for (int p = 0; p < NP; ++p) pb[i][nt][p] = make_uint2(ka_transpose(x[p]), ka_transpose(y[p]));
            }
        }
        // ---- O^T += V^T P^T
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            uint32_t vw[4][C::VW];
            int ve[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = 2 * t + (j & 1), key = 16 * i + (r ^ ((r >> 1) & 1)) + 8 * (j >> 1);
                if (has_value) {
                    ka_load_words<C::VW>(at + C::MANT + key * (D / 2) + g * C::VW * 4, vw[j]);
                    ve[j] = ka_load_byte(at + 2 * C::MANT + C::EXPS + key * C::NB + ve0);
                } else {
#pragma unroll
                    for (int e = 0; e < C::VW; ++e) vw[j][e] = 0;
                    ve[j] = 0;
                }
            }
            const uint32_t s01 = ka_scale(ve[0], ve[1]), s23 = ka_scale(ve[2], ve[3]);
            const uint32_t o01 = ka_offset(s01), o23 = ka_offset(s23);
#pragma unroll
            for (int w = 0; w < C::VW; ++w) {
                const uint32_t x01 = __byte_perm(vw[0][w], vw[1][w], 0x5410), y01 = __byte_perm(vw[0][w], vw[1][w], 0x7632);
                const uint32_t x23 = __byte_perm(vw[2][w], vw[3][w], 0x5410), y23 = __byte_perm(vw[2][w], vw[3][w], 0x7632);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t f0 = ka_value(x01 >> (4 * e), s01, o01), f1 = ka_value(y01 >> (4 * e), s01, o01);
                    const uint32_t f2 = ka_value(x23 >> (4 * e), s23, o23), f3 = ka_value(y23 >> (4 * e), s23, o23);
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) ka_mma(o[4 * w + e][nt], f0, f1, f2, f3, pb[i][nt][p]);
                }
            }
        }
        __syncwarp();                                                      // all lanes are through with the chunk
        stage = stage == C::STAGES - 1 ? 0 : stage + 1;
    }
    // (given up: what was asked for lands before the CTA leaves)
    if (!ok)
        for (int i = 0; i < C::STAGES; ++i) mbar_wait_soon(ring.bars + 8 * i, ring.phases >> i & 1, ring.abort_flag, a.c.status, 188, false);

    // ---- the warps' parts joined
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], d);
    __syncthreads();                                                      // all are through with their rings
    constexpr int OP = KaShared<D, NP, NT>::OP;
    float* os = reinterpret_cast<float*>(sm + KaShared<D, NP, NT>::Q);    // [KA_WARPS][RT][OP]
    float2* ml = reinterpret_cast<float2*>(sm + KaShared<D, NP, NT>::ML);      // [KA_WARPS][RT]
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
            const int d = (C::VW * g + (i >> 2)) * 8 + 2 * (i & 3);
            if (D % 64 == 0 || d < D) {
                float* at = os + (warp * RT + 8 * nt + 2 * t) * OP + d;
                *reinterpret_cast<float2*>(at) = make_float2(o[i][nt][0], o[i][nt][2]);
                *reinterpret_cast<float2*>(at + OP) = make_float2(o[i][nt][1], o[i][nt][3]);
            }
        }
        if (g == 0)
#pragma unroll
            for (int c = 0; c < 2; ++c) ml[warp * RT + 8 * nt + 2 * t + c] = make_float2(m[nt][c], l[nt][c]);
    }
    __syncthreads();
    // the warps' results of one element of four, and in a cluster then the CTAs' (each CTA's lie where its first warp's were)
    const int rank = splits > 1 ? (int)cluster_ctarank() : 0;
    float2* const joined = ml + KA_WARPS * RT;                            // [RT]
    auto join = [&](int r, int d, float& top, float& sum, float (&v)[4]) {
        top = -INFINITY;
        sum = 0.f;
        v[0] = v[1] = v[2] = v[3] = 0.f;
#pragma unroll
        for (int w = 0; w < KA_WARPS; ++w) top = fmaxf(top, ml[w * RT + r].x);
        const float use = top == -INFINITY ? 0.f : top;                   // (no key seen, or scores that are no numbers: these stay so)
#pragma unroll
        for (int w = 0; w < KA_WARPS; ++w) {
            const float2 x = ml[w * RT + r];
            const float f = ka_exp2(x.x - use);
            const float4 y = *reinterpret_cast<const float4*>(os + (w * RT + r) * OP + d);
            sum += f * x.y;
            v[0] += f * y.x; v[1] += f * y.y; v[2] += f * y.z; v[3] += f * y.w;
        }
    };
    if (splits > 1) {
        for (int i = threadIdx.x; i < rows * (D / 4); i += KA_THREADS) {
            const int r = i / (D / 4), d = 4 * (i - r * (D / 4));
            float top, sum, v[4];
            join(r, d, top, sum, v);
            *reinterpret_cast<float4*>(os + r * OP + d) = make_float4(v[0], v[1], v[2], v[3]);
            if (d == 0) joined[r] = make_float2(top, sum);
        }
        __syncthreads();
        cluster_barrier();
    }
    const uint32_t os_at = smem_u32(os), joined_at = smem_u32(joined);
    const bool vec_out = ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)((a.os.token | a.os.head) * (int64_t)sizeof(T))) & (4 * sizeof(T) - 1)) == 0;
    for (int i = rank * KA_THREADS + threadIdx.x; i < rows * (D / 4); i += splits * KA_THREADS) {
        const int r = i / (D / 4), d = 4 * (i - r * (D / 4));
        float top = -INFINITY, sum = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
        if (splits == 1) {
            join(r, d, top, sum, v);
        } else {
            float2 x[KA_SPLITS];
            float4 y[KA_SPLITS];
#pragma unroll
            for (int sp = 0; sp < KA_SPLITS; ++sp)
                if (sp < splits) {
                    x[sp] = ka_shared2(map_to_rank(joined_at + r * 8, sp));
                    y[sp] = ka_shared4(map_to_rank(os_at + (r * OP + d) * 4, sp));
                    top = fmaxf(top, x[sp].x);
                }
            if (top == -INFINITY) top = 0.f;
#pragma unroll
            for (int sp = 0; sp < KA_SPLITS; ++sp)
                if (sp < splits) {
                    const float f = ka_exp2(x[sp].x - top);
                    sum += f * x[sp].y;
                    v[0] += f * y[sp].x; v[1] += f * y[sp].y; v[2] += f * y[sp].z; v[3] += f * y[sp].w;
                }
        }
        if (slot >= 0) {
            float* part = a.partial + ((int64_t)slot * RT + r) * D + d;
            *reinterpret_cast<float4*>(part) = make_float4(v[0], v[1], v[2], v[3]);
            if (d == 0) reinterpret_cast<float2*>(a.partial + (int64_t)2 * a.ctas * RT * D)[(int64_t)slot * RT + r] = make_float2(top, sum);
            continue;
        }
        const float inv = sum > 0.f ? __frcp_rn(sum) : 0.f;               // a row that sees no key: zeros
        const int query = (r0 + r) / a.group, gh = (r0 + r) - query * a.group;
        T* dst = reinterpret_cast<T*>(a.out) + (seq.first + query) * a.os.token + (h * a.group + gh) * a.os.head + d;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] *= inv;
        if (vec_out) {
            store_four(dst, v);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) dst[e] = from_f32<T>(v[e]);
        }
    }
}

template <int D, int NP, int NT>
__device__ __forceinline__ KaRing ka_ring(unsigned char* sm) {
    using S = KaShared<D, NP, NT>;
    constexpr int STAGES = KaDim<D, NT>::STAGES;
    volatile int* flag = reinterpret_cast<volatile int*>(sm + S::BAR + KA_WARPS * STAGES * 8);
    const uint32_t bars = smem_u32(sm + S::BAR);
    if (threadIdx.x == 0) {
        for (int i = 0; i < KA_WARPS * STAGES; ++i) mbar_init(bars + 8 * i, 1);
        *flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    return KaRing{bars + (threadIdx.x >> 5) * STAGES * 8, 0u, flag};
}

__device__ __forceinline__ KaRange ka_range(const Kv4Attend& a, const Kv4Seq& s, int first_query, int last_query) {
    KaRange r;
    const int base = s.length - s.n;
    r.hi = max(0, min(s.held, base + last_query + 1));
    r.lo = a.window ? max(0, base + first_query - a.window + 1) & ~63 : 0;
    return r;
}

// A tile per CTA, or per cluster of `splits` CTAs: short keys, or tiles enough.
template <int D, int NP, int NT, class T>
__global__ void __launch_bounds__(KA_THREADS, NT == 1 && D <= 128 ? 3 : 2)
kv4_attend_kernel(const Kv4Attend a, int splits) {
    extern __shared__ __align__(128) unsigned char sm[];
    KaRing ring = ka_ring<D, NP, NT>(sm);
    chain_start();
    const int b = blockIdx.z, h = blockIdx.y, tile = blockIdx.x / splits, rank = blockIdx.x % splits;
    const Kv4Seq s = kv4_seq(a.c, b);
    constexpr int RT = 8 * NT, UNIT = KaDim<D, NT>::UNIT;
    if (tile * RT >= s.n * a.group) return;                               // (all of a cluster alike)
    const int last = min((tile + 1) * RT, s.n * a.group) - 1;
    KaRange r = ka_range(a, s, tile * RT / a.group, last / a.group);
    const int units = (max(0, r.hi - r.lo) + UNIT - 1) / UNIT, u0 = units * rank / splits, u1 = units * (rank + 1) / splits;
    r = KaRange{r.lo + u0 * UNIT, min(r.hi, r.lo + u1 * UNIT)};
    ka_tile<D, NP, NT, T>(a, b, s, h, tile, r, -1, splits, sm, ring);
    if (splits > 1) cluster_barrier();                                    // nobody reads this CTA's results any more
}

// The units of a sequence's tiles (all alike) and how many tiles it has.
template <int D, int NT>
__device__ __forceinline__ int2 ka_units(const Kv4Attend& a, const Kv4Seq& s) {
    const KaRange r = ka_range(a, s, 0, s.n - 1);
    const int tiles = (s.n * a.group + 8 * NT - 1) / (8 * NT) * a.c.heads;
    return make_int2(max(1, (r.hi - r.lo + KaDim<D, NT>::UNIT - 1) / KaDim<D, NT>::UNIT), tiles);
}
// Units of all sequences, of those before each thread's share of them and of its own, by all threads of the CTA.
template <int D, int NT, int WARPS>
__device__ __forceinline__ void ka_scan(const Kv4Attend& a, int& total, int& before, int& own, int& b0, int& b1) {
    __shared__ int sums[WARPS];
    const int per = (a.c.sequences + 32 * WARPS - 1) / (32 * WARPS);
    b0 = min(a.c.sequences, (int)threadIdx.x * per);
    b1 = min(a.c.sequences, b0 + per);
    own = 0;
    for (int b = b0; b < b1; ++b) {
        const int2 u = ka_units<D, NT>(a, kv4_seq(a.c, b));
        own += u.x * u.y;
    }
    int x = own;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, d);
        if ((threadIdx.x & 31) >= d) x += y;
    }
    if ((threadIdx.x & 31) == 31) sums[threadIdx.x >> 5] = x;
    __syncthreads();
    total = 0;
    before = x - own;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
        if (w < (int)(threadIdx.x >> 5)) before += sums[w];
        total += sums[w];
    }
}

template <int D, int NP, int NT, class T>
__global__ void __launch_bounds__(KA_THREADS, NT == 1 && D <= 128 ? 3 : 2)
kv4_attend_split_kernel(const Kv4Attend a) {
    extern __shared__ __align__(128) unsigned char sm[];
    __shared__ int found[2];
    KaRing ring = ka_ring<D, NP, NT>(sm);
    chain_start();
    int total, before, own, b0, b1;
    ka_scan<D, NT, KA_WARPS>(a, total, before, own, b0, b1);
    const int ctas = min(a.ctas, total), cta = blockIdx.x;
    if (cta >= ctas) return;
    int u = (int)((int64_t)total * cta / ctas);
    const int end = (int)((int64_t)total * (cta + 1) / ctas);
    if (u >= before && u < before + own) {
        int b = b0;
        for (; b + 1 < b1; ++b) {
            const int2 x = ka_units<D, NT>(a, kv4_seq(a.c, b));
            if (u < before + x.x * x.y) break;
            before += x.x * x.y;
        }
        found[0] = b;
        found[1] = u - before;
    }
    __syncthreads();
    int b = found[0], at = found[1];
    while (u < end && b < a.c.sequences) {
        const Kv4Seq s = kv4_seq(a.c, b);
        const int2 x = ka_units<D, NT>(a, s);
        const KaRange all = ka_range(a, s, 0, s.n - 1);
        while (u < end && at < x.x * x.y) {
            const int item = at / x.x, within = at - item * x.x, take = min(x.x - within, end - u);
            const int tile = item / a.c.heads, h = item - tile * a.c.heads;
            KaRange r;
            r.lo = all.lo + within * KaDim<D, NT>::UNIT;
            r.hi = min(all.hi, r.lo + take * KaDim<D, NT>::UNIT);
            const int slot = take == x.x ? -1 : 2 * cta + (within == 0);
            ka_tile<D, NP, NT, T>(a, b, s, h, tile, r, slot, 1, sm, ring);
            at += take;
            u += take;
        }
        ++b;
        at = 0;
    }
}

// The parts of the tiles that were split, joined in ascending order of their keys. A CTA takes `each` rows of a tile, one after the
// other; groups of dim / 4 threads share a row's parts, and their sums are added up in the order of the groups.
constexpr int KJ_THREADS = 256;
template <int D, int NT, class T>
__global__ void __launch_bounds__(KJ_THREADS)
kv4_join_kernel(const Kv4Attend a, int each) {
    constexpr int RT = 8 * NT, LANES = D / 4, GROUPS = KJ_THREADS / LANES;
    __shared__ int found[2];
    __shared__ float4 sums[GROUPS][LANES];
    __shared__ float weights[GROUPS];
    chain_start();
    const int b = blockIdx.z, h = blockIdx.y, tile = blockIdx.x / (RT / each), row0 = blockIdx.x % (RT / each) * each;
    int total, before, own, b0, b1;
    ka_scan<D, NT, KJ_THREADS / 32>(a, total, before, own, b0, b1);
    const Kv4Seq s = kv4_seq(a.c, b);
    const int2 x = ka_units<D, NT>(a, s);
    const int item = tile * a.c.heads + h;
    if (item >= x.y) return;
    if (b >= b0 && b < b1) {
        for (int c = b0; c < b; ++c) {
            const int2 y = ka_units<D, NT>(a, kv4_seq(a.c, c));
            before += y.x * y.y;
        }
        found[0] = before;
    }
    __syncthreads();
    const int64_t ctas = min(a.ctas, total);
    const int first = found[0] + item * x.x;
    const int c0 = (int)(((int64_t)(first + 1) * ctas - 1) / total), c1 = (int)(((int64_t)(first + x.x) * ctas - 1) / total);
    if (c0 == c1) return;
    const int rows = min(RT, s.n * a.group - tile * RT), group = threadIdx.x / LANES, d = 4 * (threadIdx.x % LANES), lane = threadIdx.x & 31;
    const float2* ml = reinterpret_cast<const float2*>(a.partial + (int64_t)2 * a.ctas * RT * D);
    auto place = [&](int c, int r) { return (int64_t)(2 * c + (c == c0)) * RT + r; };
    auto add = [&](int c, int r, float top, float& sum, float4& v) {
        const float2 y = ml[place(c, r)];
        const float4 w = *reinterpret_cast<const float4*>(a.partial + place(c, r) * D + d);
        const float f = ka_exp2(y.x - top);
        sum += f * y.y;
        v.x += f * w.x; v.y += f * w.y; v.z += f * w.z; v.w += f * w.w;
    };
    auto store = [&](int r, float sum, const float4& v) {
        const float inv = sum > 0.f ? __frcp_rn(sum) : 0.f;
        const int query = (tile * RT + r) / a.group, gh = tile * RT + r - query * a.group;
        T* dst = reinterpret_cast<T*>(a.out) + (s.first + query) * a.os.token + (h * a.group + gh) * a.os.head + d;
        dst[0] = from_f32<T>(v.x * inv);
        dst[1] = from_f32<T>(v.y * inv);
        dst[2] = from_f32<T>(v.z * inv);
        dst[3] = from_f32<T>(v.w * inv);
    };
    if (c1 - c0 < 8) {
        // few parts: a row per group
        if (group < GROUPS)
            for (int r = row0 + group; r < min(rows, row0 + each); r += GROUPS) {
                float top = -INFINITY, sum = 0.f;
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                for (int c = c0; c <= c1; ++c) top = fmaxf(top, ml[place(c, r)].x);
                if (top == -INFINITY) top = 0.f;
#pragma unroll 4
                for (int c = c0; c <= c1; ++c) add(c, r, top, sum, v);
                store(r, sum, v);
            }
        return;
    }
    for (int r = row0; r < min(rows, row0 + each); ++r) {
        float top = -INFINITY;
        for (int c = c0 + lane; c <= c1; c += 32) top = fmaxf(top, ml[place(c, r)].x);
#pragma unroll
        for (int k = 1; k < 32; k <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
        float sum = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (top == -INFINITY) top = 0.f;
        if (group < GROUPS) {
#pragma unroll 4
            for (int c = c0 + group; c <= c1; c += GROUPS) add(c, r, top, sum, v);
        }
        __syncthreads();                                                  // the row before has been stored
        if (group < GROUPS) {
            sums[group][threadIdx.x % LANES] = v;
            if (d == 0) weights[group] = sum;
        }
        __syncthreads();
        if (group == 0) {
#pragma unroll
            for (int k = 1; k < GROUPS; ++k) {
                const float4 w = sums[k][threadIdx.x];
                sum += weights[k];
                v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
            }
            store(r, sum, v);
        }
    }
}

// ------------------------------------------------------------------------------ host side

// With `bytes` the workspace is asked for and nothing is launched.
template <int D, int NP, int NT, class T>
int ka_launch(Kv4Attend a, cudaStream_t st, size_t* bytes) {
    constexpr int SMEM = KaShared<D, NP, NT>::BYTES;
    static std::atomic<int> resident[MAX_DEVICES];
    const int dev = current_device();
    if (dev < 0) return HBFP_ERR_CUDA;
    int ctas = resident[dev].load(std::memory_order_acquire);
    if (!ctas) {
        int rc = allow_shared<kv4_attend_kernel<D, NP, NT, T>>(SMEM);
        if (!rc) rc = allow_shared<kv4_attend_split_kernel<D, NP, NT, T>>(SMEM);
        if (rc) return rc;
        int per = 0;
        HBFP_CUDA_OK(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kv4_attend_split_kernel<D, NP, NT, T>, KA_THREADS, SMEM));
        if (per < 1) return HBFP_ERR_CUDA;
        ctas = per * sm_count();
        resident[dev].store(ctas, std::memory_order_release);
    }
    constexpr int RT = 8 * NT;
    const int64_t keys = kv4_keys(a);
    a.tiles = (int)(((int64_t)a.c.most * a.group + RT - 1) / RT);
    const int64_t items = (int64_t)a.tiles * a.c.heads * a.c.sequences, units = (keys + KaDim<D, NT>::UNIT - 1) / KaDim<D, NT>::UNIT;
    const dim3 grid((unsigned)a.tiles, (unsigned)a.c.heads, (unsigned)a.c.sequences);
    // Clusters share a tile's keys while that leaves a CTA two units and the GPU has room for twice the CTAs.
    int splits = 1;
    while (splits < KA_SPLITS && keys > 256 * splits && items * splits * 2 <= ctas) splits *= 2;
    // A launch more and the parts' way through memory pay where what is left to a CTA is long and the tiles do not fill the GPU.
    const bool split = keys > 1536 * splits && items * splits < 2 * (int64_t)ctas && items * units < (1ll << 30);
    if (bytes) {
        *bytes = split ? (size_t)2 * ctas * RT * (D + 2) * sizeof(float) : 0;
        return HBFP_OK;
    }
    if (!split) {
        launch_chained_clusters(kv4_attend_kernel<D, NP, NT, T>, splits, dim3(grid.x * splits, grid.y, grid.z), KA_THREADS, SMEM, st, true, a, splits);
        return launch_status();
    }
    a.ctas = ctas;
    launch_chained(kv4_attend_split_kernel<D, NP, NT, T>, dim3((unsigned)ctas), KA_THREADS, SMEM, st, a);
    // Tiles of many parts each: a CTA per row. (25 sequences of 1856 keys, 28 rows of 8 heads, bfloat16: 6400 CTAs for one or two parts a tile
    // took 26 us, 800 take 11.)
    const int each = items * 8 <= ctas ? 1 : 8;
    launch_chained(kv4_join_kernel<D, NT, T>, dim3(grid.x * (RT / each), grid.y, grid.z), KJ_THREADS, 0, st, a, each);
    return launch_status();
}

// Row tiles of 8, 16 or 32 (a 256-wide head: 16, its accumulators take twice the registers).
template <int D, int NP, class T>
int ka_launch_rows(const Kv4Attend& a, cudaStream_t st, size_t* bytes) {
    const int64_t rows = (int64_t)a.c.most * a.group;
    if (rows <= 8) return ka_launch<D, NP, 1, T>(a, st, bytes);
    if constexpr (D <= 128)
        if (rows > 16) return ka_launch<D, NP, 4, T>(a, st, bytes);
    return ka_launch<D, NP, 2, T>(a, st, bytes);
}
template <int NP, class T>
int ka_launch_dim(const Kv4Attend& a, cudaStream_t st, size_t* bytes) {
    switch (a.c.dim) {
        case 64: return ka_launch_rows<64, NP, T>(a, st, bytes);
        case 96: return ka_launch_rows<96, NP, T>(a, st, bytes);
        case 128: return ka_launch_rows<128, NP, T>(a, st, bytes);
        case 256: return ka_launch_rows<256, NP, T>(a, st, bytes);
    }
    return HBFP_ERR_UNSUPPORTED;
}

}  // namespace
}  // namespace hbfp
