// Elastic kernel of the norms around a block: with u = N_post(x), gated,
//   h = residual + scale * u,   y = h,   z = N_pre(h),
// N(v) = (v - mean) / sqrt(mean((v - mean)^2) + eps) * weight + bias, the mean 0 for RMS norm.
//
// What bounds it: HBM, every row read and written once (8192 rows of 4096 bf16 with residual and both outputs:
// 53 us, 5.1 TB/s past the caches, where a plain copy reaches 4.9).  Reading the weights once for four rows, or before the sums are known, changed nothing.  So a row
// stays in registers between its passes: one logical wave's for short rows, and the four of a tile's for longer
// ones, whose sums meet in LDS.  Rows beyond 32 vectors per lane (16384 16-bit values) are read again for each
// pass, and so are all rows of the second kind in blocks of 64 and 128, where one wave would have to hold what two
// or four do.
//
// Rows are whole 16-byte vectors, at any alignment with RAG, and a rest of less than one, an element of which
// the first lanes hold besides.  Sums are fp32: each lane's own values in order, the wave's lanes in the fixed
// order of wave_sum, then the four waves' in order; the same operations whether a row is kept or read again,
// so results do not depend on the physical block (hence no contraction by the compiler).
#include "memops.h"
#include "seq_rows.h"

#pragma clang fp contract(off)

namespace miriam {

enum Gate { GATE_NONE = 0, GATE_CHANNEL = 1, GATE_ROWS = 2, GATE_SILU = 3, GATE_SIGMOID = 4 };

// Gate value of a row gate; 1 / (1 + e^-g) has no overflow: e^-g = inf gives 0.
__device__ __forceinline__ float gate_value(int kind, float g) {
    if (kind == GATE_ROWS) return g;
    const float s = 1.0f / (1.0f + expf(-g));
    return kind == GATE_SIGMOID ? s : g * s;
}

// N values of a row as they are stored; N = 1: one element.
template <class T, int N, bool RAG>
struct Held {
    Vec16<T> p;
    template <bool PAST = false>
    __device__ __forceinline__ void load(const T *src) {
        if constexpr (N == 1) p.e[0] = *src;
        else if constexpr (RAG) p = ld_loose(src);
        else if constexpr (PAST) p.u = ld_past(src);
        else p = ld_vec(src);
    }
    __device__ __forceinline__ float at(int e) const { return TypeOps<T>::to_f(p.e[e]); }
};
template <class T, int N, bool RAG>
__device__ __forceinline__ void put_row(T *dst, const float (&v)[N], int past) {
    if constexpr (N == 1) {
        st_f(dst, v[0]);
    } else {
        Vec16<T> o;
#pragma unroll
        for (int e = 0; e < N; ++e) o.e[e] = TypeOps<T>::from_f(v[e]);
        if constexpr (RAG) st_loose(dst, o);
        else if (past) st_past(dst, o.u);
        else st_vec(dst, o);
    }
}

// v = (v - mean) * rstd * w + b at column j.
template <int N, bool RAG>
__device__ __forceinline__ void norm_apply(float (&v)[N], int64_t j, const float *w, const float *b, float mean, float rstd) {
    float c[N];
    ld_cols<N, RAG>(w + j, N, c);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = (v[e] - mean) * rstd * c[e];
    if (b) {
        ld_cols<N, RAG>(b + j, N, c);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] += c[e];
    }
}
// Gate, scale and residual at column j.
template <int N, bool RAG, class H>
__device__ __forceinline__ void norm_join(const NormArgs &a, float (&u)[N], int64_t j, const H &r, const H &g) {
    if (a.gate_kind == GATE_CHANNEL) {
        float c[N];
        ld_cols<N, RAG>(static_cast<const float *>(a.gate) + j, N, c);
#pragma unroll
        for (int e = 0; e < N; ++e) u[e] *= c[e];
    } else if (a.gate_kind != GATE_NONE) {
#pragma unroll
        for (int e = 0; e < N; ++e) u[e] *= gate_value(a.gate_kind, g.at(e));
    }
#pragma unroll
    for (int e = 0; e < N; ++e) u[e] = a.res ? __builtin_fmaf(a.scale, u[e], r.at(e)) : a.scale * u[e];
}
// s and the values, c times as large; the squares of c (v - mean), cmean being c mean.
template <int N>
__device__ __forceinline__ float norm_add(float s, const float (&v)[N], float c) {
#pragma unroll
    for (int e = 0; e < N; ++e) s += v[e] * c;
    return s;
}
template <int N>
__device__ __forceinline__ float norm_square(float s, const float (&v)[N], float c, float cmean) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float d = __builtin_fmaf(v[e], c, -cmean);
        s = __builtin_fmaf(d, d, s);
    }
    return s;
}
// Mean and 1 / sqrt(variance + eps) of a row.  sums(c, cmean) sets the mean of c v and returns that of (c (v - mean))^2.
// A row whose sums leave fp32 is summed once more, its values 2^-80 as large: the largest ones' squares are 2^96 then, and
// what vanishes beside those that left it is below 2^-46.
template <class F>
__device__ __forceinline__ void norm_stats(const NormArgs &a, F &&sums, float &mean, float &rstd) {
    constexpr float kSmall = 0x1p-80f;
    const float var = sums(1.0f, mean);
    rstd = 1.0f / sqrtf(var + a.eps);
    if (__builtin_expect(!(var < INFINITY), 0)) {
        const float small = sums(kSmall, mean);
        mean *= 1.0f / kSmall;
        rstd = kSmall / sqrtf(small + a.eps * kSmall * kSmall);
    }
}

// WR: logical waves per row; NR: vectors of V values per lane that are kept (0: the row is read again for each
// pass).  NR > 0 holds one logical wave per physical one: WR = 1, or P = 4.
template <class T, int V, bool RAG, int WR, int NR, int P>
__global__ __launch_bounds__(kWave * P) void norm_kernel(NormArgs a, Shard sh) {
    static_assert(NR == 0 || WR == 1 || P == kLogicalWaves, "a physical wave keeps one logical wave's values");
    constexpr int SL = WR == 1 ? 1 : kLogicalWaves / P;  // logical waves of one row that a physical wave runs
    typedef Held<T, V, RAG> Piece;
    typedef Held<T, 1, RAG> One;
    __shared__ float sums[2][4];
    const int pw = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int lane = threadIdx.x % kWave;
    const int64_t G = gridDim.x;
    const int64_t rank = a.past ? blockIdx.x : wg_rank(blockIdx.x, G);
    constexpr int64_t step = (int64_t)WR * kWave * V;
    const float inv_n = 1.0f / (float)a.n;
    const int64_t whole = RAG ? a.n / V * V : a.n;  // the rest: one element of the row's first lanes
    const bool rows_gate = a.gate_kind > GATE_CHANNEL;
    // mean over the row from its lanes' sums (divided by n first), in LDS over its four logical waves: two places in
    // turn, as a wave is at most one meeting ahead of another's reads
    int turn = 0;
    auto row_mean = [&](const float (&part)[SL]) {
        if constexpr (WR == 1) {
            return wave_sum(part[0] * inv_n);
        } else {
            float *p = sums[turn & 1];
            ++turn;
#pragma unroll
            for (int s = 0; s < SL; ++s) {
                const float w = wave_sum(part[s] * inv_n);
                if (lane == 0) p[s * P + pw] = w;
            }
            __syncthreads();
            return ((p[0] + p[1]) + p[2]) + p[3];
        }
    };

    int iter = 0;
    for (int64_t t = sh.begin + rank; t < sh.begin + sh.len; t += G, ++iter) {
        trace_tile(sh, t, iter);
        for (int s0 = 0; s0 < kLogicalWaves / P; s0 += SL) {
#pragma unroll
            for (int s = 0; s < SL; ++s) trace_wave(sh, t, (s0 + s) * P + pw, pw, s0 + s);
            const int64_t row = WR == 1 ? t * kLogicalWaves + s0 * P + pw : t;
            if (row >= a.rows) continue;  // (one wave per row only: nothing is met)
            const T *xr = static_cast<const T *>(a.x) + row * a.ldx;
            const T *rr = static_cast<const T *>(a.res) + row * a.ldr;
            const T *gr = static_cast<const T *>(a.gate) + row * a.ldg;
            T *yr = static_cast<T *>(a.y) + row * a.ldy;
            T *zr = static_cast<T *>(a.z) + row * a.ldz;
            // first column of the lane in slot s; its element of the rest
            auto col0 = [&](int s) { return (int64_t)((WR == 1 ? 0 : (s0 + s) * P + pw) * kWave + lane) * V; };
            const int64_t jt = whole + lane;
            const bool rest = RAG && jt < a.n && (WR == 1 || s0 * P + pw == 0);
            if constexpr (NR > 0) {
                float v[NR][V], vt[1];
                Piece r[NR], g[NR];
                One rt, gt;
                auto each = [&](auto &&f) {
#pragma unroll
                    for (int i = 0; i < NR; ++i) {
                        const int64_t j = col0(0) + i * step;
                        if (j < whole) f(i, j);
                    }
                };
                {
                    Piece x[NR];
                    One xt;
                    auto fetch = [&](auto past) {
                        constexpr bool PAST = decltype(past)::value != 0;
                        each([&](int i, int64_t j) {
                            x[i].template load<PAST>(xr + j);
                            if (a.res) r[i].template load<PAST>(rr + j);
                            if (rows_gate) g[i].template load<PAST>(gr + j);
                        });
                    };
                    if (!RAG && a.past) fetch(ActTag<1>{});
                    else fetch(ActTag<0>{});
                    if (rest) {
                        xt.load(xr + jt);
                        if (a.res) rt.load(rr + jt);
                        if (rows_gate) gt.load(gr + jt);
                        vt[0] = xt.at(0);
                    }
                    each([&](int i, int64_t) {
#pragma unroll
                        for (int e = 0; e < V; ++e) v[i][e] = x[i].at(e);
                    });
                }
                auto sums = [&](float c, float &cmean) __attribute__((always_inline)) {
                    float part[1] = {0.0f};
                    cmean = 0.0f;
                    if (a.layer) {
                        each([&](int i, int64_t) { part[0] = norm_add(part[0], v[i], c); });
                        if (rest) part[0] = norm_add(part[0], vt, c);
                        cmean = row_mean(part);
                        part[0] = 0.0f;
                    }
                    each([&](int i, int64_t) { part[0] = norm_square(part[0], v[i], c, cmean); });
                    if (rest) part[0] = norm_square(part[0], vt, c, cmean);
                    return row_mean(part);
                };
                float mean, rstd;
                if (a.post) {
                    norm_stats(a, sums, mean, rstd);
                    each([&](int i, int64_t j) { norm_apply<V, RAG>(v[i], j, a.post, a.post_bias, mean, rstd); });
                    if (rest) norm_apply<1, RAG>(vt, jt, a.post, a.post_bias, mean, rstd);
                }
                each([&](int i, int64_t j) {
                    norm_join<V, RAG>(a, v[i], j, r[i], g[i]);
                    if (a.y) put_row<T, V, RAG>(yr + j, v[i], a.past);
                });
                if (rest) {
                    norm_join<1, RAG>(a, vt, jt, rt, gt);
                    if (a.y) put_row<T, 1, RAG>(yr + jt, vt, a.past);
                }
                if (a.z) {
                    norm_stats(a, sums, mean, rstd);
                    each([&](int i, int64_t j) {
                        norm_apply<V, RAG>(v[i], j, a.pre, a.pre_bias, mean, rstd);
                        put_row<T, V, RAG>(zr + j, v[i], a.past);
                    });
                    if (rest) {
                        norm_apply<1, RAG>(vt, jt, a.pre, a.pre_bias, mean, rstd);
                        put_row<T, 1, RAG>(zr + jt, vt, a.past);
                    }
                }
            } else {
                float m1 = 0.0f, r1 = 1.0f, m2 = 0.0f, r2 = 1.0f;
                // the block's values at column j, and h
                auto load = [&](auto &v, int64_t j) {
                    constexpr int N = sizeof(v) / sizeof(float);
                    Held<T, N, RAG> x;
                    x.load(xr + j);
#pragma unroll
                    for (int e = 0; e < N; ++e) v[e] = x.at(e);
                };
                auto joined = [&](auto &v, int64_t j) {
                    constexpr int N = sizeof(v) / sizeof(float);
                    Held<T, N, RAG> r, g;
                    load(v, j);
                    if (a.res) r.load(rr + j);
                    if (rows_gate) g.load(gr + j);
                    if (a.post) norm_apply<N, RAG>(v, j, a.post, a.post_bias, m1, r1);
                    norm_join<N, RAG>(a, v, j, r, g);
                };
                auto sums = [&](auto &&get, float c, float &cmean) __attribute__((always_inline)) {
                    float part[SL] = {}, total = 0.0f;
                    cmean = 0.0f;
                    float v[V], vt[1];
                    for (int pass = a.layer ? 0 : 1; pass < 2; ++pass) {
#pragma unroll
                        for (int s = 0; s < SL; ++s) {
                            part[s] = 0.0f;
                            for (int64_t j = col0(s); j < whole; j += step) {
                                get(v, j);
                                part[s] = pass == 0 ? norm_add(part[s], v, c) : norm_square(part[s], v, c, cmean);
                            }
                            if (rest && s == 0) {
                                get(vt, jt);
                                part[s] = pass == 0 ? norm_add(part[s], vt, c) : norm_square(part[s], vt, c, cmean);
                            }
                        }
                        total = row_mean(part);
                        if (pass == 0) cmean = total;
                    }
                    return total;
                };
                auto stats = [&](auto &&get, float &mean, float &rstd) {
                    norm_stats(a, [&](float c, float &cmean) { return sums(get, c, cmean); }, mean, rstd);
                };
                if (a.post) stats(load, m1, r1);
                if (a.z) stats(joined, m2, r2);
                auto finish = [&](auto &v, int64_t j) {
                    constexpr int N = sizeof(v) / sizeof(float);
                    joined(v, j);
                    if (a.y) put_row<T, N, RAG>(yr + j, v, a.past);
                    if (a.z) {
                        norm_apply<N, RAG>(v, j, a.pre, a.pre_bias, m2, r2);
                        put_row<T, N, RAG>(zr + j, v, a.past);
                    }
                };
                float v[V], vt[1];
                for (int s = 0; s < SL; ++s)
                    for (int64_t j = col0(s); j < whole; j += step) finish(v, j);
                if (rest) finish(vt, jt);
            }
        }
    }
}

template <class T, bool RAG, int WR, int NR>
static void norm_table(const void *out[3]) {
    constexpr int V = 16 / sizeof(T), NS = WR == 1 ? NR : 0;  // blocks of 64 and 128
    out[0] = reinterpret_cast<const void *>(&norm_kernel<T, V, RAG, WR, NS, 1>);
    out[1] = reinterpret_cast<const void *>(&norm_kernel<T, V, RAG, WR, NS, 2>);
    out[2] = reinterpret_cast<const void *>(&norm_kernel<T, V, RAG, WR, NR, 4>);
}

template <class T, bool RAG>
static int norm_table_form(int form, const void *out[3]) {
    switch (form) {
    case NORM_WAVE1: norm_table<T, RAG, 1, 1>(out); return 0;
    case NORM_WAVE2: norm_table<T, RAG, 1, 2>(out); return 0;
    case NORM_TILE1: norm_table<T, RAG, 4, 1>(out); return 0;
    case NORM_TILE2: norm_table<T, RAG, 4, 2>(out); return 0;
    case NORM_TILE4: norm_table<T, RAG, 4, 4>(out); return 0;
    case NORM_TILE8: norm_table<T, RAG, 4, 8>(out); return 0;
    case NORM_LONG: norm_table<T, RAG, 4, 0>(out); return 0;
    default: return -1;
    }
}

template <class T>
static int norm_table_t(int form, bool vec, const void *out[3]) {
    return vec ? norm_table_form<T, false>(form, out) : norm_table_form<T, true>(form, out);
}

int norm_kernels(int dtype, int form, bool vec, const void *out[3]) {
    switch (dtype) {
    case 0: return norm_table_t<float>(form, vec, out);
    case 1: return norm_table_t<half_t>(form, vec, out);
    case 2: return norm_table_t<bf16_t>(form, vec, out);
    default: return -1;
    }
}

}  // namespace miriam
