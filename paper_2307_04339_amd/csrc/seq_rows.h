// Device-side reading of the sequence arrays: every value is clamped, so that none leads outside a buffer.
#pragma once

#include "elastic_common.h"
#include "seq_args.h"

namespace miriam {

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }

__device__ __forceinline__ int seq_len(const SeqArgs &q, int64_t s) {
    return clampi(q.kv_len[s], 0, q.table ? q.page * q.max_pages : 0x3fffffff);
}

// f over the values of the lanes up to and with this one, 0 being neutral to it; six data-parallel moves.
template <class T, class F>
__device__ __forceinline__ T upto_lane(T v, F f) {
    auto from = [&](auto ctrl, auto rows) {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
    };
    v = f(v, from(ActTag<0x111>{}, ActTag<0xf>{}));  // 1, 2, 4 and 8 lanes back in each row of 16
    v = f(v, from(ActTag<0x112>{}, ActTag<0xf>{}));
    v = f(v, from(ActTag<0x114>{}, ActTag<0xf>{}));
    v = f(v, from(ActTag<0x118>{}, ActTag<0xf>{}));
    v = f(v, from(ActTag<0x142>{}, ActTag<0xa>{}));  // the last lane of rows 0 and 2 to rows 1 and 3
    v = f(v, from(ActTag<0x143>{}, ActTag<0xc>{}));  // lane 31 to rows 2 and 3
    return v;
}
__device__ __forceinline__ int upto_sum(int v) {
    return upto_lane(v, [](int a, int b) { return a + b; });
}
__device__ __forceinline__ int all_sum(int v) { return __builtin_amdgcn_readlane(upto_sum(v), kWave - 1); }
__device__ __forceinline__ int all_max(int v) {  // of values >= 0
    return __builtin_amdgcn_readlane(upto_lane(v, [](int a, int b) { return a > b ? a : b; }), kWave - 1);
}
__device__ __forceinline__ float all_sum(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, upto_lane(v, [](float a, float b) { return a + b; })), kWave - 1));
}

// Loads and stores past the caches.  (The empty statements keep the compiler from merging them with ordinary ones in
// the other branch of a condition, which makes both ordinary.)
template <class T>
__device__ __forceinline__ u32x4 ld_past(const T *p) {
    asm volatile("");
    const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
    asm volatile("");
    return v;
}
template <class T>
__device__ __forceinline__ void st_past(T *p, const u32x4 &v) {
    asm volatile("");
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(p));
    asm volatile("");
}

// Sequence of packed row `row` (uniform over the wave): the number of sequences that end at or before it, found
// by all lanes at once, and its position; -1 for a row that belongs to none.
__device__ __forceinline__ int find_seq(const SeqArgs &q, int row, int lane, int &pos) {
    int s = 0;
    for (int64_t i0 = 0; i0 < q.seqs; i0 += kWave) {
        const int64_t i = i0 + lane;
        const bool past = i < q.seqs && q.q_start[i + 1] <= row;
        const int n = __builtin_popcountll(__ballot(past));
        s += n;
        if (n < kWave) break;
    }
    if (s >= q.seqs) return -1;
    const int q0 = clampi(q.q_start[s], 0, (int)q.tokens), q1 = clampi(q.q_start[s + 1], 0, (int)q.tokens);
    if (row < q0 || row >= q1) return -1;
    pos = seq_len(q, s) - (q1 - q0) + (row - q0);
    return s;
}

// Element offset, without the head's, of the place of the token at `pos` of sequence s; -1 if it has none.
__device__ __forceinline__ int64_t cache_place(const SeqArgs &q, int s, int pos) {
    if (pos < 0) return -1;
    const int p = (int)fdiv((uint32_t)pos, q.fd_page);
    if (p >= q.max_pages) return -1;
    const int id = q.table[s * q.ldt + p];
    if (id < 0 || id >= q.pages) return -1;
    return id * q.sp + (int64_t)(pos - p * q.page) * q.st;
}

}  // namespace miriam
