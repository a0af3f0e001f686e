// Key/value cache held in 4-bit block floating point: the arrays, the tokens of a batch, and what the kernels of kv4.cu and
// kv4_attend.cuh share.
//
// A page holds `page` tokens of every head. A row of `dim` values is dim / 32 blocks; value = (nibble - 8) * 2^s. A 32-bit word holds
// eight consecutive values, value 2 i in nibble i and value 2 i + 1 in nibble i + 4: masked with 0x000F000F, a word shifted by 4 i
// gives the neighbours 2 i and 2 i + 1 in the low bits of two halfwords, where they become a pair of bfloat16 by one logical
// instruction and one FMA (pair_value).
#pragma once

#include "types.cuh"

namespace hbfp {

constexpr int STATUS_PAGE = 1001;         // device status: a page number outside the cache
constexpr int STATUS_TOKENS = 1002;       // device status: a length beyond the page table, or starts out of order
constexpr int KV4_MAX_EXP = 120;          // 136 * 2^s, the offset of a pair, is a finite bfloat16 up to here

// Element strides of a [token][head][dim] tensor; dim has stride one.
struct Kv4Rows {
    int64_t token, head;
};

struct Kv4Args {
    uint8_t *k_mant, *v_mant;
    int8_t *k_exps, *v_exps;
    int64_t pages;
    int heads, dim, page, shift;          // page = 1 << shift, at least 16
    const int32_t* table;                 // [sequences][table_ld]
    int64_t table_ld;
    int table_pages, sequences;
    const int32_t* lengths;
    const int32_t* starts;                // [sequences + 1], or null: tokens / sequences each
    int64_t tokens;
    int most;                             // tokens of a sequence at most
    int32_t* status;
};

namespace {

struct Kv4Seq {
    int64_t first;      // its first row among the call's tokens
    int n, length;      // tokens of this call, tokens in the cache when they are in it
    int held;           // those of them that the page table has room for: the rest has no place, its positions stay what they are
    bool bad;           // one of the numbers was out of range
};

// The numbers come from the caller's device memory: whatever they are, a row lies within the call's tokens and a position below `held` within
// the table. (Not reported here: a branch on the length would keep loads that do not need it waiting.)
__device__ __forceinline__ Kv4Seq kv4_seq_unreported(const Kv4Args& a, int b) {
    Kv4Seq s;
    bool bad = false;
    if (a.starts) {
        const int64_t lo = __ldg(a.starts + b), hi = __ldg(a.starts + b + 1);
        s.first = lo;
        s.n = 0;
        if (lo < 0 || hi < lo || hi > a.tokens || hi - lo > a.most) bad = true;
        else s.n = (int)(hi - lo);
    } else {
        s.n = a.most;
        s.first = (int64_t)b * a.most;
    }
    const int cap = (int)((int64_t)a.table_pages << a.shift);             // (below 2^30)
    const int len = __ldg(a.lengths + b);
    s.length = (uint32_t)len < 1u << 30 ? len : 0;                         // positions have 30 bits: a longer sequence counts as an empty one
    s.held = min(s.length, cap);
    s.bad = bad || len > cap;
    return s;
}
__device__ __forceinline__ void kv4_report(const Kv4Args& a, const Kv4Seq& s) {
    if (s.bad) atomicCAS(a.status, 0, STATUS_TOKENS);
}
__device__ __forceinline__ Kv4Seq kv4_seq(const Kv4Args& a, int b) {
    const Kv4Seq s = kv4_seq_unreported(a, b);
    kv4_report(a, s);
    return s;
}

// The page that holds position p (0 <= p < held) of sequence b; -1 for a number that is no page of the cache.
__device__ __forceinline__ int64_t kv4_page(const Kv4Args& a, int b, int index) {
    const int id = __ldg(a.table + (int64_t)b * a.table_ld + index);
    if (id < 0 || id >= a.pages) {
        atomicCAS(a.status, 0, STATUS_PAGE);
        return -1;
    }
    return id;
}

// An exponent byte as the kernels take it: within what kv4_append writes, also where a page was never written.
__device__ __forceinline__ int kv4_exponent(int8_t e) { return min(max((int)e, -63), KV4_MAX_EXP); }

}  // namespace
}  // namespace hbfp
