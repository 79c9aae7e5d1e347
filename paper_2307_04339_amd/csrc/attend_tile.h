// Attention over a paged cache for many query rows: tiles of 128 rows, bound by the matrix cores.
//
// A row is a (token, head of the group) pair, so the heads that share a cache head share its keys and values
// in LDS, and a tile of a group of heads is short along the tokens, which wastes less at the causal edge.  Each
// logical wave owns 32 rows: queries, running maximum, sum and the 32 x dp output stay in its registers.  64
// keys and values at a time come by LDS-DMA into one of two stages while the other is used; their places in
// the cache are looked up a step earlier by one wave.  One meeting per step.
//
// Tiles of one cache head are consecutive, so a die's tiles share its L2's keys, and run from a sequence's last
// rows to its first: the longest first.  With fewer than two tiles per CU a tile's keys are divided among
// `splits` tiles, the last of which joins their partial results in order.
#pragma once

#include "attend.h"
#include "igemm_dma.h"

namespace miriam {

template <class T, int DP, int P>
struct TileKernel {
    static constexpr int NJ = DP / 16;        // 16-value steps of a key
    static constexpr int ND = DP / 32;        // 32-value tiles of the output
    static constexpr int CPR = DP / 8;        // 16-byte pieces of a row
    static constexpr int RPL = kWave / CPR;   // rows per load
    static constexpr int NLD = kTileKeys / RPL;  // loads per stage of keys (and of values)
    static constexpr int STAGE = 2 * kTileKeys * DP * 2;
    static constexpr int PL0 = 2 * STAGE, MASK0 = PL0 + 2 * kTileKeys * 8, LDS_BYTES = MASK0 + 16;
    // pieces are exchanged so that what a read takes from several rows lies on different banks
    static constexpr __device__ int kswz(int r) { return DP == 64 ? (r >> 1) & 7 : r & 15; }
    static constexpr __device__ int vswz(int r) { return DP == 64 ? ((r >> 1) & 1) << 2 : (r & 3) << 2; }
};

template <class T, int DP, int P>
__global__ __launch_bounds__(kWave * P, DP > 128 ? 1 : 2) void attend_tile_kernel(AttendArgs a, Shard sh) {
    typedef TileKernel<T, DP, P> K_;
    typedef Mfma<T, 32> MF;
    typedef typename MF::op_t op_t;
    typedef typename MF::acc_t acc_t;
    constexpr int NJ = K_::NJ, ND = K_::ND, CPR = K_::CPR, RPL = K_::RPL, NLD = K_::NLD;
    __shared__ __attribute__((aligned(1024))) char smem[K_::LDS_BYTES];
    __shared__ int s_last;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    const int tid = threadIdx.x;
    const int pw = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int lane = tid % kWave, hx = lane >> 5, xl = lane & 31;
    int64_t *const places = reinterpret_cast<int64_t *>(smem + K_::PL0);      // [2][64]
    uint64_t *const masks = reinterpret_cast<uint64_t *>(smem + K_::MASK0);   // [2]
    const T *const X = static_cast<const T *>(a.x);
    T *const Y = static_cast<T *>(a.y);
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(a.work, (short)0, (int)a.work_bytes, 0x00020000);
    const int64_t G = gridDim.x;
    const int64_t rank = wg_rank(blockIdx.x, G);
    const int seqs = (int)a.sq.seqs, g = a.group;
    const int outputs = (int)(a.T / a.splits), per_head = outputs / a.kv_heads;

    int iter = 0;
    for (int64_t t = sh.begin + rank; t < sh.begin + sh.len; t += G, ++iter) {
        trace_tile(sh, t, iter);
        for (int slot = 0; slot < kLogicalWaves / P; ++slot) trace_wave(sh, t, slot * P + pw, pw, slot);
        const int out = (int)fdiv((uint32_t)t, a.fd_splits), split = (int)t - out * a.splits;
        const int hk = out / per_head;
        int qi = out - hk * per_head;
        // the qi-th of all sequences' row tiles
        int s = -1;
        for (int base = 0; base < seqs; base += kWave) {
            int n = 0;
            if (base + lane < seqs) n = (seq_view(a, base + lane).n * g + kTileRows - 1) / kTileRows;
            int upto = n;
#pragma unroll
            for (int o = 1; o < kWave; o <<= 1) {
                const int v = __shfl_up(upto, o);
                upto += lane >= o ? v : 0;
            }
            const int all = __builtin_amdgcn_readlane(upto, kWave - 1);
            if (qi < all) {
                const int i = __builtin_popcountll(__ballot(upto <= qi));
                s = base + i;
                qi = __builtin_amdgcn_readlane(upto, i) - 1 - qi;  // a sequence's last rows first
                break;
            }
            qi -= all;
        }
        if (s < 0) continue;
        const SeqView sv = seq_view(a, s);
        const int row0 = qi * kTileRows, rows = sv.n * g - row0 < kTileRows ? sv.n * g - row0 : kTileRows;
        // keys that the tile's rows may see, in steps of 64, and this split's share
        SeqView tv = sv;
        int tile_lo, tile_hi;  // positions of the tile's first and last row
        {
            const int t0 = (int)fdiv((uint32_t)row0, a.fd_group), t1 = (int)fdiv((uint32_t)(row0 + rows - 1), a.fd_group);
            tile_lo = sv.pos0 + t0;
            tile_hi = sv.pos0 + t1;
            tv.end = a.causal ? clampi(sv.pos0 + t1 + 1, 0, sv.len) : sv.len;
            tv.begin = a.window > 0 ? clampi(sv.pos0 + t0 - a.window + 1, 0, tv.end) : 0;
        }
        const int lo = tv.begin / kTileKeys, nb = tv.end > tv.begin ? (tv.end + kTileKeys - 1) / kTileKeys - lo : 0;
        const int b0 = lo + (int)((int64_t)split * nb / a.splits), b1 = lo + (int)((int64_t)(split + 1) * nb / a.splits);
        const T *const kh = static_cast<const T *>(a.k) + (int64_t)hk * a.sq.sh, *const vh = static_cast<const T *>(a.v) + (int64_t)hk * a.sq.sh;

        auto look_up = [&](int b) -> int64_t { return b < b1 ? key_place(a, s, tv, b * kTileKeys + lane) : -1; };
        auto place = [&](int64_t pl, int buf) {
            const uint64_t there = __ballot(pl >= 0);
            places[buf * kTileKeys + lane] = pl;
            if (lane == 0) masks[buf] = there;
        };
        // loads of the step whose places are in `buf` into stage `buf`
        auto load = [&](int buf) {
#pragma unroll
            for (int i = 0; i < NLD / P; ++i) {
                const int q = i * P + pw, r = q * RPL + lane / CPR;
                const int64_t o = places[buf * kTileKeys + r];
                const int dk = ((lane % CPR) ^ K_::kswz(r)) * 8, dv = ((lane % CPR) ^ K_::vswz(r)) * 8;
                const T *none = reinterpret_cast<const T *>(g_no_key);
                lds_dma16(o >= 0 && dk < a.d ? kh + o + dk : none, lds0 + (uint32_t)(buf * K_::STAGE + q * 1024));
                lds_dma16(o >= 0 && dv < a.d ? vh + o + dv : none, lds0 + (uint32_t)(buf * K_::STAGE + kTileKeys * DP * 2 + q * 1024));
            }
        };

        for (int slot = 0; slot < kLogicalWaves / P; ++slot) {
            const int lam = slot * P + pw;
            const int wr0 = row0 + 32 * lam, wrows = row0 + rows - wr0;  // the wave's first row, and how many (may be <= 0)
            const int r = wr0 + xl, tok = (int)fdiv((uint32_t)r, a.fd_group);
            const int pos = sv.pos0 + tok;
            const int pos_lo = sv.pos0 + (int)fdiv((uint32_t)wr0, a.fd_group);
            const int pos_hi = wrows > 0 ? sv.pos0 + (int)fdiv((uint32_t)(wr0 + (wrows < 32 ? wrows : 32) - 1), a.fd_group) : pos_lo;
            u32x4 q[NJ];
            {
                const T *qr = X + (int64_t)(sv.q0 + tok) * a.ldx + (int64_t)(hk * g + r - tok * g) * a.d;
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    const int d = 16 * j + 8 * hx;
                    const T *src = xl < wrows && d < a.d ? qr + d : reinterpret_cast<const T *>(g_no_key);
                    q[j] = *reinterpret_cast<const u32x4 *>(src);
                }
            }
            acc_t acc[ND];
            float m = -INFINITY, l = 0.0f;
#pragma unroll
            for (int i = 0; i < ND; ++i) acc[i] = acc_t{};

            // one step on stage `buf`; edge: some rows do not see some of its keys
            auto step = [&](int b, int buf, uint64_t there, bool edge) __attribute__((always_inline)) {
                const char *const ks = smem + buf * K_::STAGE;
                const uint32_t vs = lds0 + (uint32_t)(buf * K_::STAGE + kTileKeys * DP * 2);
                acc_t sc[2];
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    sc[kt] = acc_t{};
                    const int kr = 32 * kt + xl;
#pragma unroll
                    for (int j = 0; j < NJ; ++j) {
                        const u32x4 k = *reinterpret_cast<const u32x4 *>(ks + kr * (DP * 2) + (((2 * j + hx) ^ K_::kswz(kr)) << 4));
                        sc[kt] = MF::run(__builtin_bit_cast(op_t, k), __builtin_bit_cast(op_t, q[j]), sc[kt]);
                    }
                }
                // lane: row xl, keys 64 b + 32 kt + 8 (i / 4) + 4 hx + i % 4
                // key 32 kt + 8 (i / 4) + 4 hx + i % 4 is bit 8 (i / 4) + i % 4 of seen[kt]
                if (edge) {
                    const uint64_t w = (there & seen_keys(a, b * kTileKeys, pos)) >> (4 * hx);
                    const uint32_t seen[2] = {(uint32_t)w, (uint32_t)(w >> 32)};
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                        for (int i = 0; i < 16; ++i) sc[kt][i] = seen[kt] & (1u << (8 * (i / 4) + i % 4)) ? sc[kt][i] : -INFINITY;
                }
                float top = -INFINITY;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[kt][i]);
                {
                    const uint32_t u = __builtin_bit_cast(uint32_t, top);
                    const auto s32 = __builtin_amdgcn_permlane32_swap(u, u, false, false);
                    top = fmaxf(__builtin_bit_cast(float, (uint32_t)s32[0]), __builtin_bit_cast(float, (uint32_t)s32[1]));
                }
                const float m1 = fmaxf(m, top * a.scale), ms = m1 == -INFINITY ? 0.0f : m1;
                const float alpha = m == -INFINITY ? 1.0f : exp2_(m - ms);  // (nothing to lower before the first key)
                m = m1;
                if (__ballot(alpha != 1.0f)) {
                    l *= alpha;
#pragma unroll
                    for (int i = 0; i < ND; ++i) acc[i] *= alpha;
                }
                u32x4 p[2][2];
                const float sub = ms - kShift<T>;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float p0 = exp2_(__builtin_fmaf(sc[kt][2 * i], a.scale, -sub)), p1 = exp2_(__builtin_fmaf(sc[kt][2 * i + 1], a.scale, -sub));
                        l += p0 + p1;
                        p[kt][i / 4][i % 4] = pack2<T>(p0, p1);
                    }
                const int vrow = 4 * hx + ((lane >> 2) & 3), vpc = ((lane >> 3) & 2) | ((lane >> 1) & 1);
                // eight keys of the lane's value in output tile i: those of step u of key tile kt
                auto value = [&](int kt, int u, int i) __attribute__((always_inline)) {
                    u32x4 v;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int vr = 32 * kt + 16 * u + 8 * j + vrow;
                        const uint32_t at = vs + (uint32_t)(vr * (DP * 2)) + (uint32_t)((((4 * i + vpc) ^ K_::vswz(vr)) << 4) + ((lane & 1) << 3));
                        const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)at));
                        v[2 * j] = x[0];
                        v[2 * j + 1] = x[1];
                    }
                    return v;
                };
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int i = 0; i < ND; ++i)
                            acc[i] = MF::run(__builtin_bit_cast(op_t, value(kt, u, i)), __builtin_bit_cast(op_t, p[kt][u]), acc[i]);
            };
            // infinities and NaN among the step's values, before its product
            auto take_apart = [&](int kb, int buf, uint64_t there) __attribute__((always_inline)) {
                char *const vb = smem + buf * K_::STAGE + kTileKeys * DP * 2;
                int bad = 0;
#pragma unroll 1
                for (int i = pw; i < NLD; i += P) bad |= not_finite<T>(*reinterpret_cast<const u32x4 *>(vb + i * 1024 + lane * 16));
                if (!__syncthreads_or(bad)) return;
                const uint64_t seen = there & seen_keys(a, kb, pos);
#pragma unroll 1
                for (int j = 0; j < kTileKeys; ++j) {
                    const bool in = (seen >> j) & 1;
#pragma unroll
                    for (int i = 0; i < ND; ++i)
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const u32x2 w = *reinterpret_cast<const u32x2 *>(vb + j * (DP * 2) + (((4 * i + c) ^ K_::vswz(j)) << 4) + 8 * hx);
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[i][4 * c + e] += not_finite_of<T>(w[e >> 1], e & 1, in);
                        }
                }
                __syncthreads();
#pragma unroll 1
                for (int i = pw; i < NLD; i += P) {
                    u32x4 *const at = reinterpret_cast<u32x4 *>(vb + i * 1024 + lane * 16);
                    *at = only_finite<T>(*at);
                }
                __syncthreads();
            };

            if (b0 < b1) {
                int64_t pl = -1;
                __syncthreads();  // the previous round's stages and places are free
                if (pw == 0) {
                    place(look_up(b0), 0);
                    pl = look_up(b0 + 1);
                }
                __syncthreads();
                load(0);
                if (pw == 0) place(pl, 1);
                for (int b = b0; b < b1; ++b) {
                    const int buf = (b - b0) & 1;
                    // this step's loads have arrived, the next one's places are written, and every wave is
                    // done with the stage that the next one's loads go to
                    wait_vmcnt<0>();
                    __syncthreads();
                    const uint64_t there_ = masks[buf];
                    if (b + 1 < b1) load(buf ^ 1);
                    if (pw == 0) pl = look_up(b + 2);
                    const uint64_t there = ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(there_ >> 32)) << 32) |
                                           (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)there_);
                    const int kb = b * kTileKeys;
                    // (the same for all waves: what the tile's first and last rows do not all see)
                    if ((a.causal && kb + kTileKeys - 1 > tile_lo) || (a.window > 0 && kb <= tile_hi - a.window)) take_apart(kb, buf, there);
                    const bool none = wrows <= 0 || (a.causal && kb > pos_hi) || (a.window > 0 && kb + kTileKeys - 1 <= pos_lo - a.window);
                    if (!none) {
                        const bool edge = ~there != 0 || (a.causal && kb + kTileKeys - 1 > pos_lo) || (a.window > 0 && kb <= pos_hi - a.window);
                        step(b, buf, there, edge);
                    }
                    // places and mask of the step after the next: everyone has read those of this one
                    if (b + 2 < b1) {
                        __syncthreads();
                        if (pw == 0) place(pl, buf);
                    }
                }
            }
            // ---- the row's sum over both halves of the keys, then the output
            {
                const uint32_t u = __builtin_bit_cast(uint32_t, l);
                const auto s32 = __builtin_amdgcn_permlane32_swap(u, u, false, false);
                l = __builtin_bit_cast(float, (uint32_t)s32[0]) + __builtin_bit_cast(float, (uint32_t)s32[1]);
            }
            if (a.splits <= 1) {
                const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;  // no key: zeros
                T *yr = Y + (int64_t)(sv.q0 + tok) * a.ldy + (int64_t)(hk * g + r - tok * g) * a.d;
                if (xl < wrows) {
#pragma unroll
                    for (int i = 0; i < ND; ++i)
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const int d = 32 * i + 8 * c + 4 * hx;
                            if (d >= a.d) continue;
                            u32x2 w;
                            w[0] = pack2<T>(acc[i][4 * c] * inv, acc[i][4 * c + 1] * inv);
                            w[1] = pack2<T>(acc[i][4 * c + 2] * inv, acc[i][4 * c + 3] * inv);
                            *reinterpret_cast<u32x2 *>(yr + d) = w;
                        }
                }
            } else {
                // partial result, device-coherent: another die's tile may join it
                const uint32_t at = (uint32_t)t * (uint32_t)(attend_partial(false, DP) * 4), pr = (uint32_t)(32 * lam + xl);
                if (xl < wrows) {
#pragma unroll
                    for (int i = 0; i < ND; ++i)
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const uint32_t d = (uint32_t)(32 * i + 8 * c + 4 * hx);
                            const f32x4 o = {acc[i][4 * c], acc[i][4 * c + 1], acc[i][4 * c + 2], acc[i][4 * c + 3]};
                            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, o), rw, (int)(at + (pr * DP + d) * 4u), 0, kAgent);
                        }
                    if (hx == 0) {
                        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, m), rw, (int)(at + (kTileRows * DP + pr) * 4u), 0, kAgent);
                        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, l), rw, (int)(at + (kTileRows * (DP + 1) + pr) * 4u), 0, kAgent);
                    }
                }
            }
        }
        if (a.splits > 1) {
            // the partial result's stores complete before the arrival is counted
            __builtin_amdgcn_s_waitcnt(0);
            __syncthreads();
            if (tid == 0) {
                const int prev = __hip_atomic_fetch_add(a.counters + out, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                s_last = prev == a.splits - 1;
                if (s_last) __hip_atomic_store(a.counters + out, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (s_last) {
                const int n4 = a.d / 4;
                for (int i = tid; i < rows * n4; i += kWave * P) {
                    const int r = i / n4, d4 = (i - r * n4) * 4;
                    float m = -INFINITY, l = 0.0f;
                    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
                    for (int w = 0; w < a.splits; ++w) {
                        const uint32_t at = (uint32_t)(out * a.splits + w) * (uint32_t)(attend_partial(false, DP) * 4);
                        const f32x4 ow = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, (int)(at + (uint32_t)(r * DP + d4) * 4u), 0, kAgent));
                        const float mw = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rw, (int)(at + (uint32_t)(kTileRows * DP + r) * 4u), 0, kAgent));
                        const float lw = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rw, (int)(at + (uint32_t)(kTileRows * (DP + 1) + r) * 4u), 0, kAgent));
                        const float top = fmaxf(m, mw), ms = top == -INFINITY ? 0.0f : top, f0 = exp2_(m - ms), f = exp2_(mw - ms);
                        m = top;
                        l = __builtin_fmaf(f, lw, l * f0);
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(f, ow[e], o[e] * f0);
                    }
                    const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
                    const int tok = (int)fdiv((uint32_t)(row0 + r), a.fd_group);
                    T *yr = Y + (int64_t)(sv.q0 + tok) * a.ldy + (int64_t)(hk * g + row0 + r - tok * g) * a.d + d4;
                    u32x2 w;
                    w[0] = pack2<T>(o[0] * inv, o[1] * inv);
                    w[1] = pack2<T>(o[2] * inv, o[3] * inv);
                    *reinterpret_cast<u32x2 *>(yr) = w;
                }
            }
            __syncthreads();  // s_last is free
        }
    }
}

template <class T, int DP>
inline void tile_table(const void *out[3], int *lds) {
    out[0] = reinterpret_cast<const void *>(&attend_tile_kernel<T, DP, 1>);
    out[1] = reinterpret_cast<const void *>(&attend_tile_kernel<T, DP, 2>);
    out[2] = reinterpret_cast<const void *>(&attend_tile_kernel<T, DP, 4>);
    *lds = TileKernel<T, DP, 4>::LDS_BYTES;
}

}  // namespace miriam
