// Device-side reading of the sequence arrays: every value is clamped, so that none leads outside a buffer.
#pragma once

#include "elastic_common.h"
#include "seq_args.h"

namespace miriam {

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }

__device__ __forceinline__ int seq_len(const SeqArgs &q, int64_t s) {
    return clampi(q.kv_len[s], 0, q.table ? q.page * q.max_pages : 0x3fffffff);
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
