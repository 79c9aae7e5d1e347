// Attention over a paged cache: what its two kernels share.
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = 2^(c q . k_j - m),  c = scale * log2(e),  m the running maximum
//
// in one pass over the keys: when the maximum rises from m to m', the sums so far are multiplied by 2^(m - m').
// Scores, maxima and sums are fp32.  Products run on the matrix cores with the keys as their rows, S^T = K Q^T
// and O^T = V^T P^T, so that a lane owns one query row: its maximum, its sum and its factor need no broadcast,
// and the scores leave the first product in the layout in which the second takes them, if the contraction
// index over the keys is numbered accordingly (it may be, as any order of the keys gives the same sum).
//
// The reference m need not be the maximum itself: it is raised only where the maximum is more than kRise (8) above it,
// so the sums are seldom multiplied (for every other step of 64 random keys otherwise); P is then at most 2^8.
// fp16: P is 2^kShift times larger (the sum as well, so it cancels): values down to 2^-20 of 2^m are then normal
// fp16 numbers, and 2^(8 + 6) is one too.
#pragma once

#include "igemm.h"
#include "seq_rows.h"

namespace miriam {

template <class T> constexpr float kShift = 0.0f;
template <> inline constexpr float kShift<half_t> = 6.0f;
constexpr float kRise = 8.0f;
// The maximum of a row is -inf where it sees no key, and at least this where it does: scores that are all -inf give 0 / 0,
// as the definition has it, and no keys give zeros.
constexpr float kLowest = -3.402823466e+38f;

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;
typedef __attribute__((address_space(3))) char *lds_char;

// 16 bytes of zeros: where keys that are not there are read.
static __device__ __attribute__((aligned(64))) uint32_t g_no_key[16];

// New tokens and keys of a sequence, for an op's batch.
struct SeqView {
    int q0, n;       // first packed row, rows (at most max_q)
    int pos0;        // position of the first
    int len;         // keys
    int begin, end;  // keys that any of the rows may see
};
__device__ __forceinline__ SeqView seq_view(const AttendArgs &a, int64_t s) {
    SeqView v;
    v.q0 = clampi(a.sq.q_start[s], 0, (int)a.sq.tokens);
    const int full = clampi(a.sq.q_start[s + 1], v.q0, (int)a.sq.tokens) - v.q0;
    v.len = seq_len(a.sq, s);
    v.pos0 = v.len - full;
    v.n = full < a.max_q ? full : a.max_q;
    v.end = a.causal ? clampi(v.pos0 + v.n, 0, v.len) : v.len;
    v.begin = a.window > 0 ? clampi(v.pos0 - a.window + 1, 0, v.end) : 0;
    return v;
}

// Element offset of key j (without the head's), -1 where there is none.
__device__ __forceinline__ int64_t key_place(const AttendArgs &a, int64_t s, const SeqView &v, int j) {
    return j >= v.begin && j < v.end ? cache_place(a.sq, (int)s, j) : -1;
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// Factors of partial results are at least the smallest number, so that an infinity among them stays one (0 times
// infinity is none) however much smaller than the others' their maximum is.
constexpr float kLeast = 0x1p-149f;
__device__ __forceinline__ float part_factor(float m, float top) { return fmaxf(exp2_(m - top), kLeast); }

// What a row's sums are multiplied by at last, m being its maximum.
__device__ __forceinline__ float one_over(float l, float m) { return m == -INFINITY ? 0.0f : 1.0f / l; }

// Two 32-bit floats rounded to T, packed.
template <class T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    typedef T t2 __attribute__((ext_vector_type(2)));
    typedef float f2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{a, b}), t2));
}
template <class T>
__device__ __forceinline__ float unpack(uint32_t w, int hi) {
    return TypeOps<T>::to_f(__builtin_bit_cast(T, (uint16_t)(hi ? w >> 16 : w & 0xffffu)));
}

// s + the two 16-bit values of w.
template <class T>
__device__ __forceinline__ float add2(uint32_t w, float s) {
    if constexpr (__is_same(T, half_t)) {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, w), __builtin_bit_cast(h2, 0x3c003c00u), s, false);
    } else {
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(b2, w), __builtin_bit_cast(b2, 0x3f803f80u), s, false);
    }
}

// Whether any of the eight 16-bit values is an infinity or a NaN.
template <class T>
__device__ __forceinline__ bool not_finite(const u32x4 &v) {
    constexpr uint32_t M = sizeof(T) == 2 && __is_same(T, half_t) ? 0x7c00u : 0x7f80u;
    bool r = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) r |= ((v[i] & M) == M) | ((v[i] >> 16 & M) == M);
    return r;
}

// Bits of the keys kb .. kb + 63 that the row at `pos` sees.
__device__ __forceinline__ uint64_t seen_keys(const AttendArgs &a, int kb, int pos) {
    auto upto = [](int n) -> uint64_t { return n >= 63 ? ~0ull : n < 0 ? 0ull : (2ull << n) - 1; };  // bits 0 .. n
    uint64_t w = ~0ull;
    if (a.causal) w = upto(pos - kb);
    if (a.window > 0) w &= ~upto(pos - a.window - kb);
    return w;
}

// Values of keys that some of the rows do not see.  Their probability is 0 for those rows, but 0 times an
// infinity or a NaN is no 0: such values are added to the outputs of the rows that see them by themselves (no
// probability but 0 makes another of them), and taken out of the product.
template <class T>
__device__ __forceinline__ u32x4 only_finite(u32x4 v) {
    constexpr uint32_t M = __is_same(T, half_t) ? 0x7c00u : 0x7f80u;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] &= ((v[i] & M) == M ? 0u : 0xffffu) | ((v[i] >> 16 & M) == M ? 0u : 0xffff0000u);
    return v;
}
template <class T>
__device__ __forceinline__ float not_finite_of(uint32_t w, int hi, bool seen) {
    constexpr uint32_t M = __is_same(T, half_t) ? 0x7c00u : 0x7f80u;
    return seen && ((hi ? w >> 16 : w) & M) == M ? unpack<T>(w, hi) : 0.0f;
}

// Whether the row at `pos` sees key j of its sequence.
__device__ __forceinline__ bool sees(const AttendArgs &a, int pos, int j) {
    return (!a.causal || j <= pos) && (a.window <= 0 || j > pos - a.window);
}
// And where every row sees such a value?  An infinity makes its output one however small its probability, but in
// the products it may have met a 0, or the two numbers of a probability, which may differ in sign.  Outputs that are not
// finite are therefore made once more, of such values alone: add(key, its offset in the cache) for each key of
// [j0, j1) that is there, j0 >= 0.  Rare, so nothing is done for speed but to pass over absent pages.
template <class F>
__device__ __forceinline__ void each_key(const AttendArgs &a, int s, int j0, int j1, F &&add) {
#pragma unroll 1
    for (int j = j0; j < j1; ++j) {
        const int64_t o = cache_place(a.sq, s, j);
        if (o >= 0) add(j, o);
        else j = ((int)fdiv((uint32_t)j, a.sq.fd_page) + 1) * a.sq.page - 1;
    }
}
// Whether any of the values is an infinity or a NaN.
template <int N, class V>
__device__ __forceinline__ bool has_not_finite(const V &v) {
    f32x4 t = {0.0f, 0.0f, 0.0f, 0.0f};  // 0 times such a value is NaN
#pragma unroll
    for (int i = 0; i < N; ++i) t[i % 4] = __builtin_fmaf(v[i], 0.0f, t[i % 4]);
    const float s = (t[0] + t[1]) + (t[2] + t[3]);
    return s != s;
}

// Cache policy of a buffer access with agent-scope coherence.
constexpr int kAgent = 16;

}  // namespace miriam
