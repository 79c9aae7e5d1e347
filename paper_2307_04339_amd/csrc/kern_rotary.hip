// Elastic kernel of the rotary positions and the append to the paged cache.
//
// Pair j of a head of the token at position p is turned by the angle p f_j.  The angle in turns, p f_j / (2 pi),
// is held in 64 bits: the product's rounding error is recovered by a fused multiply-add and whole turns are
// dropped before anything is rounded to fp32, so that 2^20 positions cost 2^-32 of a turn (in fp32 the angle
// itself would be off by 0.06 radians there).  What is left, an eighth of a turn at most beside a multiple of a
// quarter, goes into the power series of sine and cosine, cut where the next term is below 2^-25.
//
// What bounds it: HBM, every value read and written once (8192 tokens of 48 heads of 128 bf16: 40 us, 5.1 TB/s past the
// caches, where a plain copy reaches 4.9; 128 tokens: 5 us, hardly more than a launch).  A lane keeps its place in the head over all heads of
// its token, so a row's angles are computed once per wave; loads of four rounds over the heads are in flight
// at once.  Few tokens: a row's heads are divided among several waves (RotaryArgs::parts).
#include "seq_rows.h"

namespace miriam {

// sin and cos of 2 pi * pos * f, f = freq / (2 pi) in turns per position.
__device__ __forceinline__ void turn(int pos, double f, float &sn, float &cs) {
    const double p = (double)pos, hi = p * f, lo = __builtin_fma(p, f, -hi);
    const double r = (hi - __builtin_rint(hi)) + lo;      // within half a turn
    const double q = __builtin_rint(4.0 * r);             // quarters
    const float x = (float)(__builtin_fma(-0.25, q, r) * 6.283185307179586477);  // |x| <= pi / 4
    const float u = x * x;
    // x^13 / 13! and x^12 / 12! are below 7e-12 and 1.2e-10 here
    float s = __builtin_fmaf(u, -2.5052108e-08f, 2.7557319e-06f);
    s = __builtin_fmaf(s, u, -1.9841270e-04f);
    s = __builtin_fmaf(s, u, 8.3333333e-03f);
    s = __builtin_fmaf(s, u, -1.6666667e-01f);
    s = __builtin_fmaf(s * u, x, x);
    float c = __builtin_fmaf(u, -2.7557319e-07f, 2.4801587e-05f);
    c = __builtin_fmaf(c, u, -1.3888889e-03f);
    c = __builtin_fmaf(c, u, 4.1666667e-02f);
    c = __builtin_fmaf(c, u, -0.5f);
    c = __builtin_fmaf(c, u, 1.0f);
    const int k = (int)q & 3;
    const float a = (k & 1) ? c : s, b = (k & 1) ? s : c;
    sn = (k & 2) ? -a : a;
    cs = (k == 1 || k == 2) ? -b : b;
}

// V values of an item's half.
template <class T, int V>
struct Piece {
    T e[V];
};
template <class T, int V, bool PAST>
__device__ __forceinline__ Piece<T, V> ld_piece(const T *p) {
    Piece<T, V> v;
    if constexpr (V == 1) v.e[0] = *p;
    else if constexpr (PAST) v = __builtin_bit_cast(Piece<T, V>, ld_past(p));
    else v = __builtin_bit_cast(Piece<T, V>, *reinterpret_cast<const u32x4 *>(p));
    return v;
}
template <class T, int V>
__device__ __forceinline__ void st_piece(T *p, const Piece<T, V> &v, int past) {
    if constexpr (V == 1) *p = v.e[0];
    else if (past) st_past(p, __builtin_bit_cast(u32x4, v));
    else *reinterpret_cast<u32x4 *>(p) = __builtin_bit_cast(u32x4, v);
}

template <class T, int V, int P>
__global__ __launch_bounds__(kWave * P) void rotary_kernel(RotaryArgs a, Shard sh) {
    const int pw = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int lane = threadIdx.x % kWave;
    const int64_t G = gridDim.x;
    const int64_t rank = a.past ? blockIdx.x : wg_rank(blockIdx.x, G);
    const int HT = a.heads + 2 * a.kv_heads, turned = a.heads + a.kv_heads;
    int iter = 0;
    for (int64_t t = sh.begin + rank; t < sh.begin + sh.len; t += G, ++iter) {
        trace_tile(sh, t, iter);
        for (int slot = 0; slot < kLogicalWaves / P; ++slot) {
            const int lam = slot * P + pw;
            trace_wave(sh, t, lam, pw, slot);
            const int64_t u = t * kLogicalWaves + lam;
            if (u >= a.sq.tokens * a.parts) continue;
            const int64_t row = fdiv((uint32_t)u, a.fd_parts);
            const int part = (int)(u - row * a.parts);
            int pos = 0;
            const int s = find_seq(a.sq, (int)row, lane, pos);
            if (s < 0) continue;
            const int64_t place = a.kv_heads > 0 ? cache_place(a.sq, s, pos) : -1;
            const T *xr = static_cast<const T *>(a.x) + row * a.ldx;
            T *yr = static_cast<T *>(a.y) + row * a.ldy;
            T *kr = static_cast<T *>(a.k) + place, *vr = static_cast<T *>(a.v) + place;
            for (int c0 = 0; c0 < a.items; c0 += kWave) {
                const int ic = a.items - c0 < kWave ? a.items - c0 : kWave;  // items of a head in this pass
                const int at_once = kWave / ic;                             // heads of a round
                const int ho = lane / ic, item = c0 + lane - ho * ic;
                const int rounds = (HT + at_once - 1) / at_once;
                const int r0 = (int)((int64_t)part * rounds / a.parts), r1 = (int)((int64_t)(part + 1) * rounds / a.parts);
                if (r0 >= r1) continue;
                const bool on = ho < at_once, turns = on && item < a.rot_items;
                // the two vectors of the item: a turned item's pairs lie across them (half layout) or in them
                int p0, p1;
                if (turns && !a.interleaved) {
                    p0 = item * V;
                    p1 = p0 + a.rot / 2;
                } else {
                    p0 = 2 * V * item;
                    p1 = p0 + V;
                }
                const bool two = p1 < a.d;  // (an odd head's last value stands alone)
                auto in = [&](int r) { return on && r < r1 && r * at_once + ho < HT; };
                constexpr int NB = 4;
                Piece<T, V> v0[NB], v1[NB];
                auto fetch = [&](int r, auto past) {
                    constexpr bool PAST = decltype(past)::value != 0;
#pragma unroll
                    for (int i = 0; i < NB; ++i)
                        if (in(r + i)) {
                            const T *src = xr + (int64_t)((r + i) * at_once + ho) * a.d;
                            v0[i] = ld_piece<T, V, PAST>(src + p0);
                            if (two) v1[i] = ld_piece<T, V, PAST>(src + p1);
                        }
                };
                auto load = [&](int r) {
                    if (V > 1 && a.past) fetch(r, ActTag<1>{});
                    else fetch(r, ActTag<0>{});
                };
                load(r0);
                float sn[V], cs[V];
                if (turns) {
                    double f[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) f[e] = a.freq[item * V + e];
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        turn(pos, f[e] * 0.15915494309189533577, sn[e], cs[e]);
                        sn[e] *= a.scale;
                        cs[e] *= a.scale;
                    }
                }
                for (int r = r0; r < r1; r += NB) {
#pragma unroll
                    for (int i = 0; i < NB; ++i) {
                        if (!in(r + i)) continue;
                        const int h = (r + i) * at_once + ho;
                        if (turns && h < turned) {
                            auto pair = [&](T &ta, T &tb, int e) {
                                const float x = TypeOps<T>::to_f(ta), y = TypeOps<T>::to_f(tb);
                                // (held in 32 bits: where the compiler made one instruction of the sum and its rounding
                                // to fp16, in some of the unrolled copies only, some results differed by a step)
                                float ra = __builtin_fmaf(x, cs[e], -(y * sn[e])), rb = __builtin_fmaf(y, cs[e], x * sn[e]);
                                asm("" : "+v"(ra), "+v"(rb));
                                ta = TypeOps<T>::from_f(ra);
                                tb = TypeOps<T>::from_f(rb);
                            };
                            if (V == 1 || !a.interleaved) {
#pragma unroll
                                for (int e = 0; e < V; ++e) pair(v0[i].e[e], v1[i].e[e], e);
                            } else if constexpr (V > 1) {
#pragma unroll
                                for (int e = 0; e < V / 2; ++e) {
                                    pair(v0[i].e[2 * e], v0[i].e[2 * e + 1], e);
                                    pair(v1[i].e[2 * e], v1[i].e[2 * e + 1], V / 2 + e);
                                }
                            }
                        }
                        T *dst = h < a.heads ? yr + (int64_t)h * a.d
                                 : h < turned ? kr + (int64_t)(h - a.heads) * a.sq.sh : vr + (int64_t)(h - turned) * a.sq.sh;
                        if (h < a.heads || place >= 0) {
                            st_piece<T, V>(dst + p0, v0[i], a.past);
                            if (two) st_piece<T, V>(dst + p1, v1[i], a.past);
                        }
                    }
                    if (r + NB < r1) load(r + NB);
                }
            }
        }
    }
}

template <class T, int V>
static void rotary_table(const void *out[3]) {
    out[0] = reinterpret_cast<const void *>(&rotary_kernel<T, V, 1>);
    out[1] = reinterpret_cast<const void *>(&rotary_kernel<T, V, 2>);
    out[2] = reinterpret_cast<const void *>(&rotary_kernel<T, V, 4>);
}

template <class T>
static int rotary_table_v(bool vec, const void *out[3]) {
    if (vec) rotary_table<T, 16 / sizeof(T)>(out);
    else rotary_table<T, 1>(out);
    return 0;
}

int rotary_kernels(int dtype, bool vec, const void *out[3]) {
    switch (dtype) {
    case 0: return rotary_table_v<float>(vec, out);
    case 1: return rotary_table_v<half_t>(vec, out);
    case 2: return rotary_table_v<bf16_t>(vec, out);
    default: return -1;
    }
}

}  // namespace miriam
