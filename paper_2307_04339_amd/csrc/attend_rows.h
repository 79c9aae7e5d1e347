// Attention over a paged cache for few query rows per cache head (up to 16: single tokens of a group of heads,
// short drafts): bound by reading the caches.
//
// Work is divided by what there is on the device, not by sequences: the blocks of 128 keys of all sequences
// and cache heads form one list, of which every tile takes an equal run, so a batch of very different lengths
// keeps all CUs busy to the end.  Where a tile's run ends inside a cache head's list, it leaves a partial
// result (maximum, sum, unnormalised output); the last tile to arrive joins a head's partial results in the
// tiles' order.  The runs depend on the lengths and the op's tile count alone.
//
// A logical wave walks every block's 32 keys of its own by itself: keys go from memory straight into the
// matrix instructions' operands, 64 contiguous bytes of 16 keys per load, values through the wave's own LDS,
// out of which ds_read_b64_tr_b16 reads them transposed; the next 32 keys' loads go out as soon as the registers
// of these are free, and their places in the cache are looked up one step earlier still.  The waves meet once per
// run to join their results.
//
// Measured: 48 sequences of 200 to 8000 keys, 32 heads over 8 cache heads of 128: 105 us, 4.8 TB/s (a copy 4.9); two
// of 100k to 131k keys, 16 heads over 2: 57 us, 4.0 TB/s, of which some 10 to find the work and to join 256 partial
// results per head in two stages; one token behind 128 keys 7.5 us, where a launch takes 4 and each of 12 of the 256 CUs
// then reads lengths, page, keys and values one after the other, for two blocks.
//
// P is the sum of two 16-bit numbers (its rounding and the rest), which keeps the output at the
// rounding of its own type and costs matrix instructions that wait for memory anyway.
#pragma once

#include "attend.h"

namespace miriam {

template <class T, int DP, int P>
struct RowsKernel {
    static constexpr int NKD = DP / 32;        // 32-value steps of a key
    static constexpr int ND = DP / 16;         // 16-value tiles of the output
    static constexpr int CPR = DP / 8;         // 16-byte pieces of a row
    static constexpr int RPL = kWave / CPR;    // rows per load of values
    static constexpr int NV = 32 / RPL;        // loads per 32 values
    static constexpr int LDO = DP + 4;         // row of partial outputs
    static constexpr int V_BYTES = 32 * DP * 2;
    static constexpr int O0 = P * V_BYTES, M0 = O0 + kLogicalWaves * 16 * LDO * 4, L0 = M0 + kLogicalWaves * 16 * 4;
    static constexpr int P0 = L0 + kLogicalWaves * 16 * 4, LDS_BYTES = P0 + P * 32 * 8;
};

template <class T, int DP, int P>
__global__ __launch_bounds__(kWave * P, DP > 128 ? 1 : 2) void attend_rows_kernel(AttendArgs a, Shard sh) {
    constexpr int kJoin = 16;  // partial results joined at once
    typedef RowsKernel<T, DP, P> K_;
    typedef Mfma<T, 16> MF;
    typedef typename MF::op_t op_t;
    constexpr int NKD = K_::NKD, ND = K_::ND, CPR = K_::CPR, RPL = K_::RPL, NV = K_::NV, LDO = K_::LDO;
    __shared__ __attribute__((aligned(1024))) char smem[K_::LDS_BYTES];
    __shared__ int s_last;
    const int tid = threadIdx.x;
    const int pw = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int lane = tid % kWave, rl = lane % 16, grp = lane / 16;
    float *const part_o = reinterpret_cast<float *>(smem + K_::O0);
    float *const part_m = reinterpret_cast<float *>(smem + K_::M0);
    float *const part_l = reinterpret_cast<float *>(smem + K_::L0);
    int64_t *const places = reinterpret_cast<int64_t *>(smem + K_::P0) + pw * 32;
    char *const vlds = smem + pw * K_::V_BYTES;
    const uint32_t vaddr = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)vlds;
    const T *const X = static_cast<const T *>(a.x);
    const T *const KC = static_cast<const T *>(a.k);
    const T *const VC = static_cast<const T *>(a.v);
    T *const Y = static_cast<T *>(a.y);
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(a.work, (short)0, (int)a.work_bytes, 0x00020000);
    const int64_t G = gridDim.x;
    const int64_t rank = wg_rank(blockIdx.x, G);
    const int seqs = (int)a.sq.seqs, heads = a.kv_heads, g = a.group;

    // 64 sequences from `base` on, one per lane: its view, the blocks of one of its cache heads (one where there are
    // rows but no keys, to write their zeros), their places in the list, and the places up to and with them.
    SeqView view;
    int base = 0, blocks = 0, mine = 0, upto = 0;
    auto blocks_of = [&](const SeqView &v) {
        const int n = (v.end + kRowKeys - 1) / kRowKeys - v.begin / kRowKeys;
        return v.n <= 0 ? 0 : n > 0 ? n : 1;
    };
    auto look = [&](int from) {
        base = from;
        view = SeqView{};
        if (base + lane < seqs) view = seq_view(a, base + lane);
        blocks = blocks_of(view);
    };
    // All blocks, and each tile's share.  While there are tiles enough for runs of two blocks that do not cross
    // from one head into the next, these are taken (a head's list then counts as even): two blocks take little
    // longer than one, and most heads of short sequences need no joining.
    int total = 0, share = 0, ahead = 0;  // ahead: places up to and with the lane's part of the sequences
    bool even = false;
    const int per = (seqs + kWave - 1) / kWave;  // sequences of a lane's part (300 of 300 keys, one cache head: 41 us, 64 after 64: 61)
    if (a.splits > 1) {
        int sum = 0, pairs = 0;
        if (per == 1) {
            look(0);  // (they stay)
            sum = blocks;
            pairs = (blocks + 1) / 2;
        } else {
            for (int s = lane * per; s < (lane + 1) * per && s < seqs; ++s) {
                const int n = blocks_of(seq_view(a, s));
                sum += n;
                pairs += (n + 1) / 2;
            }
        }
        const int all_pairs = all_sum(pairs) * heads;
        total = all_sum(sum) * heads;
        even = all_pairs <= (int)a.T;
        if (even) total = 2 * all_pairs;
        share = even ? 2 : (total + (int)a.T - 1) / (int)a.T;
        ahead = upto_sum((even ? 2 * pairs : sum) * heads);
    }
    auto list = [&]() {
        mine = (even ? (blocks + 1) & ~1 : blocks) * heads;
        upto = upto_sum(mine);
    };
    auto view_of = [&](int i) {  // of the 64's i-th
        SeqView v;
        v.q0 = __builtin_amdgcn_readlane(view.q0, i);
        v.n = __builtin_amdgcn_readlane(view.n, i);
        v.pos0 = __builtin_amdgcn_readlane(view.pos0, i);
        v.len = __builtin_amdgcn_readlane(view.len, i);
        v.begin = __builtin_amdgcn_readlane(view.begin, i);
        v.end = __builtin_amdgcn_readlane(view.end, i);
        return v;
    };

    // A partial result into `slot` of the workspace, by device-coherent stores: another die's tile may join it.
    auto keep = [&](int slot, int r, int d4, const f32x4 &o, float m, float l) {
        const uint32_t at = (uint32_t)slot * (uint32_t)(attend_partial(16, DP) * 4);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, o), rw, (int)(at + (uint32_t)(r * DP + d4) * 4u), 0, kAgent);
        if (d4 == 0) {
            __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, m), rw, (int)(at + (uint32_t)(16 * DP + r) * 4u), 0, kAgent);
            __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, l), rw, (int)(at + (uint32_t)(16 * DP + 16 + r) * 4u), 0, kAgent);
        }
    };
    // Whether this tile is the last of n to arrive at `counter`; its stores are complete before it is counted.
    auto arrive = [&](int32_t *counter, int n) {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (tid == 0) {
            const int prev = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s_last = prev == n - 1;
            if (s_last) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        return s_last != 0;
    };
    // Partial results slot_of(0 .. n - 1) joined in order, 16 loads in flight; done(row, d, o, m, l) for each piece.
    auto join = [&](int rows, int n, auto &&slot_of, auto &&done) __attribute__((always_inline)) {
        const int n4 = a.d / 4;
        for (int i = tid; i < rows * n4; i += kWave * P) {
            const int r = i / n4, d4 = (i - r * n4) * 4;
            float m = -INFINITY, l = 0.0f;
            f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int w = 0; w < n; w += kJoin) {
                f32x4 ow[kJoin];
                float mw[kJoin], lw[kJoin];
#pragma unroll
                for (int q = 0; q < kJoin; ++q) {
                    const uint32_t at = (uint32_t)slot_of(w + q < n ? w + q : n - 1) * (uint32_t)(attend_partial(16, DP) * 4);
                    ow[q] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, (int)(at + (uint32_t)(r * DP + d4) * 4u), 0, kAgent));
                    mw[q] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rw, (int)(at + (uint32_t)(16 * DP + r) * 4u), 0, kAgent));
                    lw[q] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rw, (int)(at + (uint32_t)(16 * DP + 16 + r) * 4u), 0, kAgent));
                }
                float top = m;
#pragma unroll
                for (int q = 0; q < kJoin; ++q) top = fmaxf(top, mw[q]);
                const float ms = top == -INFINITY ? 0.0f : top, f0 = part_factor(m, ms);
                m = top;
                l *= f0;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] *= f0;
#pragma unroll
                for (int q = 0; q < kJoin; ++q) {
                    if (w + q >= n) continue;
                    const float f = part_factor(mw[q], ms);
                    l = __builtin_fmaf(f, lw[q], l);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(f, ow[q][e], o[e]);
                }
            }
            done(r, d4, o, m, l);
        }
    };

    // One run: blocks [b0, b1) of the nb of cache head hk of sequence s, the first of which is block `first`
    // of the sequence; tiles w0 .. w1 share the head.
    auto run = [&](int64_t t, int s, const SeqView &sv, int hk, int b0, int b1, int w0, int w1) __attribute__((always_inline)) {
        const int rows = sv.n * g;
        const int first = sv.begin / kRowKeys;
        const T *const kh = KC + (int64_t)hk * a.sq.sh, *const vh = VC + (int64_t)hk * a.sq.sh;
        for (int slot = 0; slot < kLogicalWaves / P; ++slot) {
            const int lam = slot * P + pw;
            // queries: row rl of the group's n * g, values 32 j + 8 grp ..
            u32x4 q[NKD];
            const int tok = (int)fdiv((uint32_t)rl, a.fd_group);
            const int pos = sv.pos0 + tok;
            {
                const T *qr = X + (int64_t)(sv.q0 + tok) * a.ldx + (int64_t)(hk * g + rl - tok * g) * a.d;
#pragma unroll
                for (int j = 0; j < NKD; ++j) {
                    const int d = 32 * j + 8 * grp;
                    const T *src = rl < rows && d < a.d ? qr + d : reinterpret_cast<const T *>(g_no_key);
                    q[j] = *reinterpret_cast<const u32x4 *>(src);
                }
            }
            u32x4 kr[2][NKD], vr[NV];
            uint32_t there = 0;  // keys of kr and vr that are there
            f32x4 acc[ND];
            float m = -INFINITY, l = 0.0f;
#pragma unroll
            for (int i = 0; i < ND; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            auto key0 = [&](int b) { return (first + b) * kRowKeys + lam * 32; };
            auto look_up = [&](int b) -> int64_t { return b < b1 ? key_place(a, s, sv, key0(b) + (lane & 31)) : -1; };
            // the places of the next 32 keys, -1 for those that are not there
            auto place = [&](int64_t pl) {
                there = (uint32_t)__ballot(pl >= 0);
                if (lane < 32) places[lane] = pl;
                __builtin_amdgcn_wave_barrier();
            };
            auto load_keys = [&]() {
#pragma unroll
                for (int jt = 0; jt < 2; ++jt) {
                    const int64_t o = places[16 * jt + rl];
#pragma unroll
                    for (int j = 0; j < NKD; ++j) {
                        const int d = 32 * j + 8 * grp;
                        const T *src = o >= 0 && d < a.d ? kh + o + d : reinterpret_cast<const T *>(g_no_key);
                        kr[jt][j] = *reinterpret_cast<const u32x4 *>(src);
                    }
                }
            };
            auto load_values = [&]() {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int64_t o = places[i * RPL + lane / CPR];
                    const int d = (lane % CPR) * 8;
                    const T *src = o >= 0 && d < a.d ? vh + o + d : reinterpret_cast<const T *>(g_no_key);
                    vr[i] = *reinterpret_cast<const u32x4 *>(src);
                }
            };
            place(look_up(b0));
            load_keys();
            load_values();
            int64_t pl = look_up(b0 + 1);
            for (int b = b0; b < b1; ++b) {
                const int kb = key0(b);
                const uint32_t here = there;
                const bool more = b + 1 < b1;
                __builtin_amdgcn_wave_barrier();
                if (more) {
                    place(pl);
                    pl = look_up(b + 2);
                }
                // values to LDS, 32-byte pieces exchanged by the row's lowest bits so that 8 rows of one piece
                // lie on different banks
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int r = i * RPL + lane / CPR, f = DP == 64 ? (r >> 1) & 3 : r & 7;
                    *reinterpret_cast<u32x4 *>(vlds + r * (DP * 2) + (((lane % CPR) ^ (f << 1)) << 4)) = vr[i];
                }
                const bool edge = sv.n > 1 && ((a.causal && kb + 31 > sv.pos0) || (a.window > 0 && kb <= sv.pos0 + sv.n - 1 - a.window));
                // key 16 jt + 4 grp + e: bit 16 jt + e of seen
                const uint32_t row_seen = edge ? here & (uint32_t)seen_keys(a, kb, pos) : here, seen = row_seen >> (4 * grp);
                if (edge) {
                    bool bad = false;
#pragma unroll
                    for (int i = 0; i < NV; ++i) bad |= not_finite<T>(vr[i]);
                    if (__ballot(bad)) {
                        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
                        for (int j = 0; j < 32; ++j) {
                            const bool in = (row_seen >> j) & 1;
                            const int f = DP == 64 ? (j >> 1) & 3 : j & 7;
#pragma unroll
                            for (int i = 0; i < ND; ++i) {
                                const u32x2 w = *reinterpret_cast<const u32x2 *>(vlds + j * (DP * 2) + (((2 * i + (grp >> 1)) ^ (f << 1)) << 4) + 8 * (grp & 1));
#pragma unroll
                                for (int e = 0; e < 4; ++e) acc[i][e] += not_finite_of<T>(w[e >> 1], e & 1, in);
                            }
                        }
                        __builtin_amdgcn_wave_barrier();
#pragma unroll
                        for (int i = 0; i < NV; ++i) {
                            const int r = i * RPL + lane / CPR, f = DP == 64 ? (r >> 1) & 3 : r & 7;
                            *reinterpret_cast<u32x4 *>(vlds + r * (DP * 2) + (((lane % CPR) ^ (f << 1)) << 4)) = only_finite<T>(vr[i]);
                        }
                    }
                }
                if (more) load_values();
                f32x4 sc[2];
#pragma unroll
                for (int jt = 0; jt < 2; ++jt) {
                    sc[jt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int j = 0; j < NKD; ++j)
                        sc[jt] = MF::run(__builtin_bit_cast(op_t, kr[jt][j]), __builtin_bit_cast(op_t, q[j]), sc[jt]);
                }
                if (more) load_keys();
                // lane: row rl, keys kb + 16 jt + 4 grp + e
                float top = -INFINITY;
#pragma unroll
                for (int jt = 0; jt < 2; ++jt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        sc[jt][e] = seen & (1u << (16 * jt + e)) ? sc[jt][e] * a.scale : -INFINITY;
                        top = fmaxf(top, sc[jt][e]);
                    }
                {
                    const uint32_t u = __builtin_bit_cast(uint32_t, top);
                    const auto s16 = __builtin_amdgcn_permlane16_swap(u, u, false, false);
                    top = fmaxf(__builtin_bit_cast(float, (uint32_t)s16[0]), __builtin_bit_cast(float, (uint32_t)s16[1]));
                    const uint32_t w = __builtin_bit_cast(uint32_t, top);
                    const auto s32 = __builtin_amdgcn_permlane32_swap(w, w, false, false);
                    top = fmaxf(__builtin_bit_cast(float, (uint32_t)s32[0]), __builtin_bit_cast(float, (uint32_t)s32[1]));
                }
                const float m1 = fmaxf(m, top), ms = m1 == -INFINITY ? 0.0f : m1;
                const float alpha = m == -INFINITY ? 1.0f : exp2_(m - ms);  // (nothing to lower before the first key)
                m = m1;
                if (__ballot(alpha != 1.0f)) {
                    l *= alpha;
#pragma unroll
                    for (int i = 0; i < ND; ++i) acc[i] *= alpha;
                }
                u32x4 hi, lo;
#pragma unroll
                for (int jt = 0; jt < 2; ++jt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float p0 = exp2_(sc[jt][2 * h] - (ms - kShift<T>)), p1 = exp2_(sc[jt][2 * h + 1] - (ms - kShift<T>));
                        l += p0 + p1;
                        const uint32_t w = pack2<T>(p0, p1);
                        hi[2 * jt + h] = w;
                        lo[2 * jt + h] = pack2<T>(p0 - unpack<T>(w, 0), p1 - unpack<T>(w, 1));
                    }
                // lane l of a group of 16 reads 8 bytes of row 4 grp + (l & 15) / 4 at columns 4 (l & 3) of the 16,
                // and holds four rows of column l & 15 then
                const uint32_t va = vaddr + (uint32_t)((lane & 1) << 3);
                const int vr = 4 * grp + ((lane >> 2) & 3), vf = DP == 64 ? (vr >> 1) & 3 : vr & 7;
#pragma unroll
                for (int i = 0; i < ND; ++i) {
                    u32x4 v;
#pragma unroll
                    for (int jt = 0; jt < 2; ++jt) {
                        const uint32_t at = va + (uint32_t)((vr + 16 * jt) * (DP * 2)) + (uint32_t)((((2 * i) ^ (vf << 1)) | ((lane >> 1) & 1)) << 4);
                        const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)at));
                        v[2 * jt] = x[0];
                        v[2 * jt + 1] = x[1];
                    }
                    acc[i] = MF::run(__builtin_bit_cast(op_t, v), __builtin_bit_cast(op_t, hi), acc[i]);
                    acc[i] = MF::run(__builtin_bit_cast(op_t, v), __builtin_bit_cast(op_t, lo), acc[i]);
                }
            }
            // the row's sum over the four groups of keys
            l += __shfl_xor(l, 16);
            l += __shfl_xor(l, 32);
            if (grp == 0) {
                part_m[lam * 16 + rl] = m;
                part_l[lam * 16 + rl] = l;
            }
#pragma unroll
            for (int i = 0; i < ND; ++i) *reinterpret_cast<f32x4 *>(part_o + (lam * 16 + rl) * LDO + 16 * i + 4 * grp) = acc[i];
        }
        __syncthreads();
        // ---- the four logical waves' results, in order
        const bool whole = w0 == w1;
        const int slot0 = (int)t * 2 + (t == w0 ? 1 : 0);
        auto put = [&](int r, int d4, const f32x4 &o, float m, float l) {
            const int tok = (int)fdiv((uint32_t)r, a.fd_group);
            T *yr = Y + (int64_t)(sv.q0 + tok) * a.ldy + (int64_t)(hk * g + r - tok * g) * a.d + d4;
            const float inv = one_over(l, m);
            u32x2 w;
            w[0] = pack2<T>(o[0] * inv, o[1] * inv);
            w[1] = pack2<T>(o[2] * inv, o[3] * inv);
            *reinterpret_cast<u32x2 *>(yr) = w;
        };
        const int n4 = a.d / 4;
        for (int i = tid; i < rows * n4; i += kWave * P) {
            const int r = i / n4, d4 = (i - r * n4) * 4;
            float m = part_m[r];
#pragma unroll
            for (int w = 1; w < kLogicalWaves; ++w) m = fmaxf(m, part_m[w * 16 + r]);
            const float ms = m == -INFINITY ? 0.0f : m;
            f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
            float l = 0.0f;
#pragma unroll
            for (int w = 0; w < kLogicalWaves; ++w) {
                const float f = exp2_(part_m[w * 16 + r] - ms);
                const f32x4 ow = *reinterpret_cast<const f32x4 *>(part_o + (w * 16 + r) * LDO + d4);
                l = __builtin_fmaf(f, part_l[w * 16 + r], l);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(f, ow[e], o[e]);
            }
            // outputs that are not finite, and sums of 0 (no keys, or scores of -inf): see each_key
            if (__builtin_expect(!(l > 0.0f) || has_not_finite<4>(o), 0)) {
                const int pos = sv.pos0 + (int)fdiv((uint32_t)r, a.fd_group), j0 = (first + b0) * kRowKeys, j1 = (first + b1) * kRowKeys;
                f32x4 only = {0.0f, 0.0f, 0.0f, 0.0f};
                each_key(a, s, j0 > sv.begin ? j0 : sv.begin, j1 < sv.end ? j1 : sv.end, [&](int j, int64_t at) {
                    if (!sees(a, pos, j)) return;
                    m = fmaxf(m, kLowest);
                    const u32x2 v = *reinterpret_cast<const u32x2 *>(vh + at + d4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) only[e] += not_finite_of<T>(v[e >> 1], e & 1, true);
                });
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = only[e] == 0.0f ? o[e] : only[e];
            }
            if (whole) put(r, d4, o, m, l);
            else keep(slot0, r, d4, o, m, l);
        }
        if (!whole) {
            const int n = w1 - w0 + 1;
            int32_t *const heads_done = a.counters + (int64_t)s * heads + hk;
            auto slot_of = [&](int w) { return w * 2 + (w == w0 ? 1 : 0); };
            // Up to 16 partial results are joined by their last tile; more in two stages, 16 consecutive ones into a
            // place (and with a counter) of the first one's, then those.
            if (n <= kJoin) {
                if (arrive(heads_done, n)) join(rows, n, [&](int i) { return slot_of(w0 + i); }, put);
            } else {
                const int first_tile = w0 + ((int)t - w0) / kJoin * kJoin, here = w1 - first_tile + 1 < kJoin ? w1 - first_tile + 1 : kJoin;
                const int groups = (n + kJoin - 1) / kJoin, place = slot_of(first_tile), second = 2 * (int)a.T;
                if (arrive(a.counters + (int64_t)seqs * heads + place, here)) {
                    join(rows, here, [&](int i) { return slot_of(first_tile + i); }, [&](int r, int d4, const f32x4 &o, float m, float l) { keep(second + place, r, d4, o, m, l); });
                    if (arrive(heads_done, groups)) join(rows, groups, [&](int i) { return second + slot_of(w0 + i * kJoin); }, put);
                }
            }
        }
        __syncthreads();  // the partial results in LDS are free
    };

    int iter = 0;
    for (int64_t t = sh.begin + rank; t < sh.begin + sh.len; t += G, ++iter) {
        trace_tile(sh, t, iter);
        for (int slot = 0; slot < kLogicalWaves / P; ++slot) trace_wave(sh, t, slot * P + pw, pw, slot);
        if (a.splits <= 1) {
            // one tile per sequence and cache head
            const int s = (int)fdiv((uint32_t)t, a.fd_kv);
            look(s / kWave * kWave);
            const int nb = __builtin_amdgcn_readlane(blocks, s % kWave);
            if (nb > 0) run(t, s, view_of(s % kWave), (int)t - s * heads, 0, nb, 0, 0);
            continue;
        }
        int at = (int)t * share;
        const int stop = at + share < total ? at + share : total;
        if (at >= stop) continue;
        // the sequence of place `at`
        int before = 0;  // places before the 64
        if (per > 1) {
            const int p = __builtin_popcountll(__ballot(ahead <= at));
            before = p > 0 ? __builtin_amdgcn_readlane(ahead, p - 1) : 0;
            look(p * per);
        } else if (base != 0) {
            look(0);
        }
        for (list(); base < seqs; list()) {
            const int all = __builtin_amdgcn_readlane(upto, kWave - 1);
            if (before + all > at) break;
            before += all;
            look(base + kWave);
        }
        int i = __builtin_popcountll(__ballot(before + upto <= at));
        while (at < stop && base < seqs) {
            const int nbs = __builtin_amdgcn_readlane(mine, i);
            if (nbs > 0) {
                const int from = before + __builtin_amdgcn_readlane(upto, i) - nbs, nb = nbs / heads;
                const int real = __builtin_amdgcn_readlane(blocks, i);  // (all places but perhaps the last)
                const SeqView sv = view_of(i);
                int hk = (at - from) / nb;
                while (hk < heads && at < stop) {
                    const int h0 = from + hk * nb, b0 = at - h0;
                    const int b1 = stop - h0 < nb ? stop - h0 : nb;
                    run(t, base + i, sv, hk, b0, b1 < real ? b1 : real, h0 / share, (h0 + nb - 1) / share);
                    at = h0 + b1;
                    ++hk;
                }
            }
            if (++i >= kWave && at < stop) {
                before += __builtin_amdgcn_readlane(upto, kWave - 1);
                i = 0;
                look(base + kWave);
                list();
            }
        }
    }
}

template <class T, int DP>
inline void rows_table(const void *out[3], int *lds) {
    out[0] = reinterpret_cast<const void *>(&attend_rows_kernel<T, DP, 1>);
    out[1] = reinterpret_cast<const void *>(&attend_rows_kernel<T, DP, 2>);
    out[2] = reinterpret_cast<const void *>(&attend_rows_kernel<T, DP, 4>);
    *lds = RowsKernel<T, DP, 4>::LDS_BYTES;
}

}  // namespace miriam
