// Attention over a paged cache for many query rows: tiles of 128 rows, bound by the matrix cores and by what they
// are fed from LDS.
//
// A row is a (token, head of the group) pair, so the heads that share a cache head share its keys and values
// in LDS, and a tile of a group of heads is short along the tokens, which wastes less at the causal edge.  Each
// logical wave owns 32 rows: queries, running maximum, sum and output stay in its registers.  64 keys and values
// at a time come by LDS-DMA into one of two stages while the other is used; the page table is read
// a step earlier still.  One meeting per step.
//
// Where a load's rows (4 of 256 bytes) always lie in one page, its base is scalar and the lanes' offsets never
// change (UNI); otherwise every lane finds its row by itself.
//
// Row tiles of one cache head are consecutive, so a die's tiles share its L2's keys, and run from a sequence's
// last rows to its first: the longest first.  Every tile finds out by itself how the batch, as it is on the device,
// is divided (some microseconds, with row tiles across the lanes):
//  - Many row tiles, none of them longer than twice what each of the 2 x CUs workgroups that run at once gets:
//    a tile each, as the hardware hands them out.
//  - Fewer row tiles than such workgroups, of like lengths (a chunk behind a long context): every row tile is cut
//    into about equal pieces, at the same keys for all row tiles of a sequence, which then share them in L2
//    (512 tokens behind 16k: 178 us then, in equal runs of the list below 205).
//  - Otherwise (single tokens beside chunks): the steps of all row tiles form a list of which every tile takes an
//    equal run (20 sequences of 1 to 400 tokens: 61 us then, in pieces 70, by a fixed division of every row tile 86).
//    As a second row tile's start and the joining cost more than a few steps, a run's end that lies within a third
//    of a run of a row tile's is moved there.
// A row tile that ends up in several tiles is joined by the last of them to arrive, in their order.
//
// Probabilities are rounded once, to T, as the matrix instructions take them, and the sum that divides the output is
// that of the rounded ones (fp32), so a row's weights still add up to one.  Each weight is then off by half a step of T at
// most, and an output of values of both signs by about as much as its own rounding: against 64 bits 0.0024 of its size
// in bf16 and 0.00026 in fp16, where rounding the output alone gives 0.0017 and 0.00020.  The two numbers per probability
// of the kernel for few rows give that here, too, but take half of the products again where these bound it: whole
// prompts 679 -> 858 us, a chunk behind 16k 174 -> 220, the 20 sequences 55 -> 62.
//
// Measured, with that division and loads whose addresses the lanes work out: 4 prompts of 4096 tokens, 32 heads of
// 128: 640 to 720 us by box and its clock, 760 to 860 TFLOP/s of the products that are needed (a wave's vector and
// matrix instructions together keep a SIMD busy for 85% of that, and neither their order nor their waves' priorities
// matter: the clock falls under them); a chunk of 512 tokens behind 16k 160 to 175 us; the 20 sequences (heads of 80)
// 53 us, of which 5 to find the work, 8 for starts and outputs of row tiles and 11 for joining.
#pragma once

#include "attend.h"
#include "tile_regs.h"

namespace miriam {

// DP: a row in LDS; DE: values of it that the products take, as many 32s as a head has (heads of 80, the 20 sequences
// above: 53 us with 96, 57 with 128).
template <class T, int DP, int P, int DE>
struct TileKernel {
    static constexpr int NJ = DE / 16;        // 16-value steps of a key
    static constexpr int ND = DE / 32;        // 32-value tiles of the output
    static constexpr int CPR = DP / 8;        // 16-byte pieces of a row
    static constexpr int RPL = kWave / CPR;   // rows per load
    static constexpr int NLD = kTileKeys / RPL;  // loads per stage of keys (and of values)
    static constexpr int HALF = kTileKeys * DP * 2;  // a stage of keys or of values
    static constexpr int LDS_BYTES = 4 * HALF;
    static constexpr int NI = NLD / P;        // loads of a wave
    static constexpr int PARTS = LDS_BYTES / (kTileRows * 8);  // partial results that can be joined
    // loads q of a wave whose rows are swizzled differently: q mod 4 (DP = 128), 2 (64), 8 (256)
    static constexpr int CYC = DP == 64 ? 2 : DP == 128 ? 4 : 8, NSW = CYC / P > 0 ? CYC / P : 1;
    // pieces are exchanged so that what a read takes from several rows lies on different banks
    static constexpr __device__ int kswz(int r) { return DP == 64 ? (r >> 1) & 7 : r & 15; }
    static constexpr __device__ int vswz(int r) { return DP == 64 ? ((r >> 1) & 1) << 2 : (r & 3) << 2; }
};

template <class T, int DP, int P, bool UNI, int DE>
__global__ __launch_bounds__(kWave * P, DP > 128 ? 1 : 2) void attend_tile_kernel(AttendArgs a, Shard sh) {
    typedef TileKernel<T, DP, P, DE> K_;
    typedef Mfma<T, 32> MF;
    typedef typename MF::op_t op_t;
    typedef typename MF::acc_t acc_t;
    constexpr int NJ = K_::NJ, ND = K_::ND, CPR = K_::CPR, RPL = K_::RPL, NLD = K_::NLD;
    __shared__ __attribute__((aligned(1024))) char smem[K_::LDS_BYTES];
    __shared__ int s_last, s_ahead[kWave];
    lds_char const lsmem = (lds_char)smem;
    // where the lane reads the values of output tile i in a stage, and the keys of step j: the swizzles go by the
    // lane alone
    const int xkey = (threadIdx.x % kWave) & 31, xhalf = (threadIdx.x % kWave) >> 5;
    int vat[ND], kat[NJ];
    {
        const int l = threadIdx.x % kWave, vrow = 4 * xhalf + ((l >> 2) & 3), vpc = ((l >> 3) & 2) | ((l >> 1) & 1);
#pragma unroll
        for (int i = 0; i < ND; ++i) vat[i] = vrow * (DP * 2) + (((4 * i + vpc) ^ K_::vswz(vrow)) << 4) + ((l & 1) << 3);
#pragma unroll
        for (int j = 0; j < NJ; ++j) kat[j] = xkey * (DP * 2) + (((2 * j + xhalf) ^ K_::kswz(xkey)) << 4);
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    const int tid = threadIdx.x;
    const int pw = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int lane = tid % kWave, hx = lane >> 5, xl = lane & 31;
    const T *const X = static_cast<const T *>(a.x);
    T *const Y = static_cast<T *>(a.y);
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(a.work, (short)0, (int)a.work_bytes, 0x00020000);
    const int64_t G = gridDim.x;
    const int64_t rank = wg_rank(blockIdx.x, G);
    const int seqs = (int)a.sq.seqs, g = a.group;

    // 64 sequences from `base` on, one per lane, and their row tiles
    SeqView view;
    int base = -1, ntiles = 0;
    auto look = [&](int from) {
        if (from == base) return;
        base = from;
        view = SeqView{};
        if (base + lane < seqs) view = seq_view(a, base + lane);
        ntiles = (view.n * g + kTileRows - 1) / kTileRows;
    };
    auto at_lane = [&](const SeqView &of, int i) {
        SeqView v;
        v.q0 = __builtin_amdgcn_readlane(of.q0, i);
        v.n = __builtin_amdgcn_readlane(of.n, i);
        v.pos0 = __builtin_amdgcn_readlane(of.pos0, i);
        v.len = __builtin_amdgcn_readlane(of.len, i);
        v.begin = v.end = 0;
        return v;
    };
    // keys that the rows of row tile q may see, and the positions of its first and last row
    struct Span {
        int begin, end, lo, hi;
    };
    auto span = [&](const SeqView &v, int q) {
        const int row0 = q * kTileRows, last = v.n * g < row0 + kTileRows ? v.n * g - 1 : row0 + kTileRows - 1;
        Span p;
        p.lo = v.pos0 + (int)fdiv((uint32_t)row0, a.fd_group);
        p.hi = v.pos0 + (int)fdiv((uint32_t)last, a.fd_group);
        p.end = a.causal ? clampi(p.hi + 1, 0, v.len) : v.len;
        p.begin = a.window > 0 ? clampi(p.lo - a.window + 1, 0, p.end) : 0;
        return p;
    };
    auto steps = [&](const Span &p) {  // one where there are no keys, to write the rows' zeros
        return p.end > p.begin ? (p.end + kTileKeys - 1) / kTileKeys - p.begin / kTileKeys : 1;
    };
    // row tiles of a cache head, the longest sequence's steps, and at least half of all; a lane goes through its part
    // of the sequences, so that a tile need not look through all of them again (1000 sequences of 128 tokens, 12
    // heads of 64: 438 us, 64 sequences after 64 twice 581)
    const int per = (seqs + kWave - 1) / kWave;
    int J = 0, longest = 0;
    float half = 0.0f;
    {
        auto add = [&](const SeqView &v) {
            const int nt = (v.n * g + kTileRows - 1) / kTileRows;
            const int n = nt > 0 && v.end > v.begin ? (v.end + kTileKeys - 1) / kTileKeys - v.begin / kTileKeys : 0;
            J += nt;
            longest = longest > n ? longest : n;
            half += 0.5f * (float)n * (float)nt;
        };
        if (per == 1) {
            look(0);  // (they stay)
            add(view);
        } else {
            for (int s = lane * per; s < (lane + 1) * per && s < seqs; ++s) add(seq_view(a, s));
        }
        const int ahead = upto_sum(J);  // row tiles up to and with the lane's part
        if (pw == 0) s_ahead[lane] = ahead;
        J = __builtin_amdgcn_readlane(ahead, kWave - 1);
        longest = all_max(longest);
        half = all_sum(half);
        __syncthreads();
    }
    // where to look for row tile j: the first sequence of its part, and the row tiles before that
    auto part_of = [&](int j, int &from, int &before) {
        from = before = 0;
        if (per > 1) {
            const int ahead = s_ahead[lane], p = __builtin_popcountll(__ballot(ahead <= j));
            from = p * per;
            before = p > 0 ? __builtin_amdgcn_readlane(ahead, p - 1) : 0;
        }
    };
    // row tiles 64 c .. 64 c + 63 of a cache head, one per lane: whose, which of its, and its steps (0: none)
    struct Chunk {
        int s, qi, n;
        SeqView v;
    };
    auto chunk = [&](int c) {
        Chunk r = {};
        const int want = c * kWave + lane;
        int from, before;
        for (part_of(c * kWave, from, before); from < seqs; from += kWave) {
            look(from);
            const int upto = upto_sum(ntiles), all = __builtin_amdgcn_readlane(upto, kWave - 1);
            int i = 0;  // sequences of these that end at or before it
#pragma unroll
            for (int o = kWave / 2; o > 0; o >>= 1) i += __shfl(upto, i + o - 1) <= want - before ? o : 0;
            SeqView v = view;
            v.q0 = __shfl(view.q0, i);
            v.n = __shfl(view.n, i);
            v.pos0 = __shfl(view.pos0, i);
            v.len = __shfl(view.len, i);
            const int end = __shfl(upto, i);
            if (want >= before && want - before < all) {
                r.s = from + i;
                r.qi = end - 1 - (want - before);  // a sequence's last rows first
                r.v = v;
                r.n = steps(span(v, r.qi));
            }
            before += all;
            if (before > c * kWave + kWave - 1) break;
        }
        return r;
    };
    const bool many = J * a.kv_heads >= 4 * a.runs && (float)longest * (float)a.runs <= 2.0f * half * (float)a.kv_heads;
    // (more row tiles than rows can have: starts that overlap; no tile may then wait for another's part)
    const bool list = a.splits > 1 && J <= a.tiles && !__builtin_amdgcn_readfirstlane(many);
    if (J > a.tiles) J = a.tiles;
    // Places of the list: a row tile's steps, or with unit > 0 its pieces of about `unit` steps.  Of a cache head,
    // and of tile k: [start(k), start(k + 1))
    int unit = 0, head_places = 0, runs = 1, near = 1;
    auto places = [&](int n) { return unit == 0 || n == 0 ? n : n < unit ? 1 : (n + unit / 2) / unit; };
    const int chunks = (J + kWave - 1) / kWave;
    Chunk ch = {};
    int have = -1;
    auto get = [&](int c) {
        if (c != have) ch = chunk(have = c);
    };
    int biggest = 0;  // piece
    auto count = [&]() {
        head_places = biggest = 0;
        for (int c = chunks - 1; c >= 0; --c) {
            get(c);
            const int n = places(ch.n), m = all_max(n > 0 ? (ch.n + n - 1) / n : 0);
            head_places += all_sum(n);
            biggest = biggest > m ? biggest : m;
        }
    };
    if (list) {
        // runs and pieces of four steps at least, and as many as the parts of a row tile that can be joined need
        const int room = (longest + K_::PARTS - 3) / (K_::PARTS - 2), least = room > 4 ? room : 4;
        count();
        const int all = head_places * a.kv_heads, each = all / a.runs;
        if (J * a.kv_heads <= a.runs) {
            unit = each > least ? each : least;
            count();
            // (fewer pieces than there are workgroups to take them, of equal lengths)
            if (head_places * a.kv_heads > a.runs || 4 * biggest > 5 * unit) unit = 0;
            runs = head_places * a.kv_heads;
        }
        if (unit == 0) {
            head_places = all / a.kv_heads;
            runs = all / least;
            runs = runs < 1 ? 1 : runs < a.runs ? runs : a.runs;
            near = all / runs / 3;
            near = near > 1 ? near : 1;
        }
    }
    const int total = head_places * a.kv_heads;
    const Runs division = runs_of(total, runs);

    int iter = 0;
    for (int64_t t = sh.begin + rank; t < sh.begin + sh.len; t += G, ++iter) {
        trace_tile(sh, t, iter);
        for (int slot = 0; slot < kLogicalWaves / P; ++slot) trace_wave(sh, t, slot * P + pw, pw, slot);
        // ---- where the tile begins: row tile j of cache head hk, which is row tile qi of sequence s; in the list
        // place `inside` of it, and place `at` of all
        int at = 0, stop = 1, hk, j, s = -1, qi = 0, inside = 0;
        if (list) {
            if (t >= runs) continue;
            at = division.start((int)t);
            stop = division.start((int)t + 1);
            hk = at / head_places;
            inside = at - hk * head_places;
            j = 0;
        } else {
            if (t >= (int64_t)J * a.kv_heads) continue;
            hk = (int)t / J;
            j = (int)t - hk * J;
        }
        SeqView sv;
        if (list) {
            for (int c = 0; c < chunks && s < 0; ++c) {
                get(c);
                const int upto = upto_sum(places(ch.n)), here = __builtin_amdgcn_readlane(upto, kWave - 1);
                if (inside < here) {
                    const int i = __builtin_popcountll(__ballot(upto <= inside));
                    inside -= i > 0 ? __builtin_amdgcn_readlane(upto, i - 1) : 0;
                    j = c * kWave + i;
                    s = __builtin_amdgcn_readlane(ch.s, i);
                    qi = __builtin_amdgcn_readlane(ch.qi, i);
                    sv = at_lane(ch.v, i);
                } else {
                    inside -= here;
                }
            }
        } else {
            int from, before;
            for (part_of(j, from, before); from < seqs && s < 0; from += kWave) {
                look(from);
                const int upto = upto_sum(ntiles), all = __builtin_amdgcn_readlane(upto, kWave - 1);
                if (j - before < all) {
                    const int i = __builtin_popcountll(__ballot(upto <= j - before));
                    s = from + i;
                    qi = __builtin_amdgcn_readlane(upto, i) - 1 - (j - before);
                    sv = at_lane(view, i);
                }
                before += all;
            }
        }
        // (what the next tile looks up anew: it is not to hold registers through this one's work)
        ch = Chunk{};
        view = SeqView{};
        ntiles = 0;
        have = base = -1;
        if (s < 0) continue;
        // ---- its pieces of row tiles, one after another.  A run ends inside a row tile only if that leaves `near`
        // steps or more on both sides; nearer ends are moved to the row tile's.
        auto onward = [&]() {  // to the next row tile of the list
            inside = 0;
            ++j;
            if (--qi < 0) {
                do {
                    if (++s == seqs) {
                        s = 0;
                        j = 0;
                        ++hk;
                    }
                    sv = seq_view(a, s);
                } while (sv.n <= 0 && hk < a.kv_heads);
                qi = (sv.n * g + kTileRows - 1) / kTileRows - 1;
            }
        };
        if (list && unit == 0 && inside > 0) {
            const int nb = steps(span(sv, qi));
            if (inside < near) {
                at -= inside;
                inside = 0;
            } else if (nb - inside < near) {
                at += nb - inside;
                onward();
            }
        }
        while (at < stop && hk < a.kv_heads && j < J) {
        const Span tv = span(sv, qi);
        const int tile_lo = tv.lo, tile_hi = tv.hi;
        const int row0 = qi * kTileRows, rows = sv.n * g - row0 < kTileRows ? sv.n * g - row0 : kTileRows;
        const int lo = tv.begin / kTileKeys, nb = steps(tv), out = hk * J + j;
        int skip = inside, take = nb - inside, w0 = (int)t, w1 = (int)t;  // steps of this piece; the tiles that share the row tile
        if (list && unit > 0) {
            const int n = places(nb);
            skip = (int)((int64_t)nb * inside / n);
            take = (int)((int64_t)nb * (inside + 1) / n) - skip;
            w0 = (int)t - inside;
            w1 = w0 + n - 1;
        } else if (list) {
            const int h0 = at - inside, e = stop - h0;  // where the row tile begins, and the run ends in it
            if (e < nb && e < near) break;
            if (e < nb && nb - e >= near) take = e - inside;
            // the runs that share it: those around the starts that lie in it; start(k) >= v from k = ceil(v runs / total) on
            auto from = [&](int v) { return (int)(((int64_t)v * runs + total - 1) / total); };
            const int k0 = from(h0 + near), k1 = from(h0 + nb - near + 1) - 1;
            if (nb >= 2 * near && k1 >= k0) {
                w0 = k0 - 1;
                w1 = k1;
            }
        }
        const int b0 = lo + skip, b1 = tv.end > tv.begin ? b0 + take : b0;
        auto slot_at = [&](int w) { return (uint32_t)(2 * w + (w == w0 ? 1 : 0)) * (uint32_t)(attend_partial(kTileRows, DP) * 4); };  // run w's partial result
        const T *const kh = static_cast<const T *>(a.k) + (int64_t)hk * a.sq.sh, *const vh = static_cast<const T *>(a.v) + (int64_t)hk * a.sq.sh;

        // Page-table entries of a step: UNI: of load `mine`, so that a wave's i-th load is that of its lane i P; else
        // of the lane's rows and of key `lane`.
        constexpr int NE = UNI ? 1 : K_::NI + 1;
        const int mine = ((lane & ~(P - 1)) | ((lane + pw) & (P - 1))) % NLD;
        const int32_t *const pages = a.sq.table + s * a.sq.ldt;
        struct Entry {
            int32_t id[NE], slot[NE];
        };
        auto fetch = [&](int b, Entry &n) {
            auto entry = [&](int j, int i) {
                n.id[i] = -1;
                n.slot[i] = 0;
                if (b < b1 && j < tv.end && (UNI ? j + RPL > tv.begin : j >= tv.begin)) {
                    const uint32_t pg = fdiv((uint32_t)j, a.sq.fd_page);
                    n.slot[i] = j - (int)pg * a.sq.page;
                    if (pg < (uint32_t)a.sq.max_pages) n.id[i] = pages[pg];
                }
            };
            if constexpr (UNI) {
                entry(b * kTileKeys + mine * RPL, 0);
            } else {
#pragma unroll
                for (int i = 0; i < K_::NI; ++i) entry(b * kTileKeys + (i * P + pw) * RPL + lane / CPR, i);
                entry(b * kTileKeys + lane, K_::NI);
            }
        };
        // Where a step's keys and values lie (byte offsets, -1: nowhere; UNI: and how many bytes from there on), and
        // which of its keys are there.
        struct Where {
            int64_t off[UNI ? 1 : K_::NI];
            uint32_t bytes;
            uint64_t there;
        };
        auto resolve = [&](int b, const Entry &n) {
            Where w;
            w.bytes = 0;
            if constexpr (UNI) {
                const bool ok = (uint32_t)n.id[0] < (uint32_t)a.sq.pages;
                w.off[0] = ((uint64_t)(uint32_t)n.id[0] * (uint64_t)a.sq.sp + (uint64_t)(uint32_t)n.slot[0] * (uint64_t)a.sq.st) * 2;
                // rows up to the last key
                w.bytes = ok ? (uint32_t)clampi(tv.end - (b * kTileKeys + mine * RPL), 0, RPL) * ((uint32_t)a.sq.st * 2u) : 0u;
                const uint64_t groups = __ballot(ok);
                constexpr uint64_t ALL = (1ull << NLD) - 1;
                w.there = ~0ull;
                if ((groups & ALL) != ALL || b * kTileKeys < tv.begin || (b + 1) * kTileKeys > tv.end) {
                    const int j = b * kTileKeys + lane, q = lane / RPL, at = (q & ~(P - 1)) | ((q - pw) & (P - 1));
                    w.there = __ballot(((groups >> at) & 1) && j >= tv.begin && j < tv.end);
                }
            } else {
#pragma unroll
                for (int i = 0; i < K_::NI; ++i) {
                    const bool ok = n.id[i] >= 0 && n.id[i] < a.sq.pages;
                    w.off[i] = ok ? (n.id[i] * a.sq.sp + (int64_t)n.slot[i] * a.sq.st) * 2 : -1;
                }
                w.there = __ballot(n.id[K_::NI] >= 0 && n.id[K_::NI] < a.sq.pages);
            }
            return w;
        };
        // the lane's byte offsets within a load's rows
        uint32_t ko[K_::NSW], vo[K_::NSW];
        {
            const int rr = lane / CPR;
#pragma unroll
            for (int w = 0; w < K_::NSW; ++w) {
                const int r = (w * P + pw) * RPL + rr, row = UNI ? rr * (int)a.sq.st : 0;
                const int dk = ((lane % CPR) ^ K_::kswz(r)) * 8, dv = ((lane % CPR) ^ K_::vswz(r)) * 8;
                ko[w] = dk < a.d ? (uint32_t)((row + dk) * 2) : kOutOfRange;
                vo[w] = dv < a.d ? (uint32_t)((row + dv) * 2) : kOutOfRange;
            }
        }
        // loads of step b's keys or values (from `base`) into the stage at LDS byte `dst`; at: the lane's offsets
        auto load = [&](int b, const Where &w, const T *base, const uint32_t (&at)[K_::NSW], uint32_t dst) {
#pragma unroll
            for (int i = 0; i < K_::NI; ++i) {
                const int q = i * P + pw;
                if constexpr (UNI) {
                    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)w.off[0], i * P), hi = (uint32_t)__builtin_amdgcn_readlane((int)(w.off[0] >> 32), i * P);
                    const uint32_t bytes = (uint32_t)__builtin_amdgcn_readlane((int)w.bytes, i * P);
                    buf_dma16(at[i % K_::NSW], make_rsrc(reinterpret_cast<const char *>(base) + (((uint64_t)hi << 32) | lo), bytes), 0u, dst + (uint32_t)(q * 1024));
                } else {
                    const uint32_t d = at[i % K_::NSW];
                    const bool ok = w.off[i] >= 0 && d != kOutOfRange;
                    lds_dma16(ok ? reinterpret_cast<const char *>(base) + w.off[i] + d : reinterpret_cast<const char *>(g_no_key), dst + (uint32_t)(q * 1024));
                }
            }
        };
        // keys: stages 0 and 1, values: stages 2 and 3 of kTileKeys rows each
        auto stage = [&](int i) { return (uint32_t)(i * K_::HALF); };

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

            // The step's work in pieces.  The next step's scores are formed before this step's are turned into
            // probabilities, so that the vector units start on those while the matrix cores still work on these;
            // beside the products with the values they look for the next scores' maximum.  (Powers beside every
            // product of the next scores instead: 2% slower.)  Operands are read from LDS three pieces ahead.
            constexpr int NQ = 2 * NJ, NP = 4 * ND, NW = 16, LA = 3;  // operands of the scores and of the values, pairs of scores of a lane
            struct Scores {
                acc_t s[2];
            };
            u32x4 op[LA + 1], p[2][2];
            float top, low, sub;  // low: what top is at least, once scaled
            lds_char kst, vst;
            auto read = [&](auto n_) __attribute__((always_inline)) {
                constexpr int n = decltype(n_)::value;
                if constexpr (n < NQ) {
                    op[n % (LA + 1)] = *(__attribute__((address_space(3))) u32x4 *)(kst + kat[n % NJ] + n / NJ * 32 * (DP * 2));
                } else if constexpr (n < NQ + NP) {
                    // eight keys of the lane's value in output tile i: those of step u of key tile kt
                    constexpr int i = (n - NQ) % ND, u = (n - NQ) / ND % 2, kt = (n - NQ) / ND / 2;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(vst + vat[i] + (32 * kt + 16 * u + 8 * j) * (DP * 2))));
                        op[n % (LA + 1)][2 * j] = x[0];
                        op[n % (LA + 1)][2 * j + 1] = x[1];
                    }
                }
            };
            auto score = [&](auto n_, Scores &z) __attribute__((always_inline)) {
                constexpr int n = decltype(n_)::value, kt = n / NJ;
                z.s[kt] = MF::run(__builtin_bit_cast(op_t, op[n % (LA + 1)]), __builtin_bit_cast(op_t, q[n % NJ]), n % NJ == 0 ? acc_t{} : z.s[kt]);
            };
            auto product = [&](auto n_) __attribute__((always_inline)) {
                constexpr int n = decltype(n_)::value, i = n % ND, u = n / ND % 2, kt = n / ND / 2;
                acc[i] = MF::run(__builtin_bit_cast(op_t, op[(NQ + n) % (LA + 1)]), __builtin_bit_cast(op_t, p[kt][u]), acc[i]);
            };
            // probabilities of pair w of the lane's scores, in the order in which the products take them
            auto power = [&](auto w_, const Scores &z) __attribute__((always_inline)) {
                constexpr int w = decltype(w_)::value, kt = w / 8, i = w % 8;
                const float p0 = exp2_(__builtin_fmaf(z.s[kt][2 * i], a.scale, -sub)), p1 = exp2_(__builtin_fmaf(z.s[kt][2 * i + 1], a.scale, -sub));
                p[kt][i / 4][i % 4] = pack2<T>(p0, p1);
                l = add2<T>(p[kt][i / 4][i % 4], l);
            };
            auto largest = [&](auto w_, const Scores &z) __attribute__((always_inline)) {
                constexpr int w = decltype(w_)::value, kt = w / 8, i = w % 8;
                top = fmaxf(fmaxf(z.s[kt][2 * i], z.s[kt][2 * i + 1]), top);
            };
            // scores of keys that a row does not see; lane: row xl, key 32 kt + 8 (i / 4) + 4 hx + i % 4
            auto mask = [&](int b, uint64_t there, Scores &z) __attribute__((always_inline)) {
                const uint64_t all = there & seen_keys(a, b * kTileKeys, pos), w = all >> (4 * hx);
                if (all == 0) low = -INFINITY;
                const uint32_t seen[2] = {(uint32_t)w, (uint32_t)(w >> 32)};
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) z.s[kt][i] = seen[kt] & (1u << (8 * (i / 4) + i % 4)) ? z.s[kt][i] : -INFINITY;
            };
            // the reference that the next probabilities are relative to
            auto raise = [&]() __attribute__((always_inline)) {
                const uint32_t u = __builtin_bit_cast(uint32_t, top);
                const auto s32 = __builtin_amdgcn_permlane32_swap(u, u, false, false);
                top = fmaxf(fmaxf(__builtin_bit_cast(float, (uint32_t)s32[0]), __builtin_bit_cast(float, (uint32_t)s32[1])) * a.scale, low);
                if (__ballot(top > m + kRise)) {  // (-inf: the first key raises it)
                    const float m1 = top > m + kRise ? top : m;
                    const float alpha = m == m1 || m == -INFINITY ? 1.0f : exp2_(m - m1);  // (nothing to lower before the first key)
                    m = m1;
                    l *= alpha;
#pragma unroll
                    for (int i = 0; i < ND; ++i) acc[i] *= alpha;
                }
                sub = (m == -INFINITY ? 0.0f : m) - kShift<T>;
            };
            auto edge = [&](int b, uint64_t there) {  // some rows do not see some of its keys
                const int kb = b * kTileKeys;
                return ~there != 0 || (a.causal && kb + kTileKeys - 1 > pos_lo) || (a.window > 0 && kb <= pos_hi - a.window);
            };
            // The products of step b, whose scores are z, beside the scores of step b + 1 into zn.  One path for all
            // steps (a branch around it costs registers, and the tile's other waves would wait all the same): scores
            // of keys that are not there or that no row sees are masked, so their probabilities are 0 and the
            // maximum goes without them, and their values are finite (see take_apart).
            auto step = [&](int b, Scores &z, Scores &zn, uint64_t there1, int odd) __attribute__((always_inline)) {
                kst = lsmem + stage(odd ^ 1);
                vst = lsmem + stage(2 + odd);
                top = -INFINITY;
                static_for<LA>([&](auto n) { read(n); });
                static_for<NQ>([&](auto n) {
                    read(ActTag<decltype(n)::value + LA>{});
                    score(n, zn);
                    __builtin_amdgcn_sched_barrier(0);
                });
                low = kLowest;
                if (edge(b + 1, there1)) mask(b + 1, there1, zn);
                static_for<NW>([&](auto w) { power(w, z); });
                static_for<NP>([&](auto n_) {
                    constexpr int n = decltype(n_)::value, w0 = n * NW / NP, w1 = (n + 1) * NW / NP;
                    read(ActTag<NQ + n + LA>{});
                    product(n_);
                    static_for<w1 - w0>([&](auto w) { largest(ActTag<w0 + decltype(w)::value>{}, zn); });
                    __builtin_amdgcn_sched_barrier(0);
                });
                raise();
            };
            // scores of the first step
            auto first = [&](int b, Scores &zn, uint64_t there1) __attribute__((always_inline)) {
                kst = lsmem + stage(0);
                top = -INFINITY;
                static_for<LA>([&](auto n) { read(n); });
                static_for<NQ>([&](auto n) {
                    if constexpr (decltype(n)::value + LA < NQ) read(ActTag<decltype(n)::value + LA>{});
                    score(n, zn);
                    __builtin_amdgcn_sched_barrier(0);
                });
                low = kLowest;
                if (edge(b, there1)) mask(b, there1, zn);
                static_for<NW>([&](auto w) { largest(w, zn); });
                raise();
            };
            // infinities and NaN among the step's values, before its product
            auto take_apart = [&](int kb, int vst, uint64_t there) __attribute__((always_inline)) {
                char *const vb = smem + stage(vst);
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
                Scores za, zb;
                Entry e, e1;
                fetch(b0, e);
                fetch(b0 + 1, e1);
                Where w0 = resolve(b0, e), wn = resolve(b0 + 1, e1);
                uint64_t here = w0.there;  // keys of the step that are there
                __syncthreads();  // the previous round's stages are free
                load(b0, w0, kh, ko, lds0 + stage(0));
                load(b0, w0, vh, vo, lds0 + stage(2));
                w0 = wn;
                if (b0 + 1 < b1) load(b0 + 1, w0, kh, ko, lds0 + stage(1));
                fetch(b0 + 2, e);
                wait_vmcnt<0>();
                __syncthreads();
                first(b0, za, here);
                // step b's keys lie in stage b - b0 mod 2, its values in the like one.  Loads in flight during its
                // products: keys of step b + 2, values of step b + 1, which w0 places.
                auto turn = [&](int b, Scores &z, Scores &zn, int odd) __attribute__((always_inline)) {
                    // step b + 1's keys and step b's values have arrived, and every wave is done with what the
                    // loads to come overwrite
                    wait_vmcnt<0>();
                    __syncthreads();
                    const Where w1 = resolve(b + 2, e);
                    if (b + 2 < b1) load(b + 2, w1, kh, ko, lds0 + stage(odd));
                    if (b + 1 < b1) load(b + 1, w0, vh, vo, lds0 + stage(2 + (odd ^ 1)));
                    fetch(b + 3, e);
                    const int kb = b * kTileKeys;
                    // (the same for all waves: what the tile's first and last rows do not all see)
                    if ((a.causal && kb + kTileKeys - 1 > tile_lo) || (a.window > 0 && kb <= tile_hi - a.window)) take_apart(kb, 2 + odd, here);
                    step(b, z, zn, w0.there, odd);
                    here = w0.there;
                    w0 = w1;
                };
                for (int b = b0;;) {
                    turn(b, za, zb, 0);
                    if (++b >= b1) break;
                    turn(b, zb, za, 1);
                    if (++b >= b1) break;
                }
            }
#pragma unroll
            for (int i = 0; i < ND; ++i) {  // see each_key
                if (__builtin_expect(__ballot(xl < wrows && has_not_finite<16>(acc[i])) == 0, 1)) continue;
                acc_t only = {};
                const int j0 = b0 * kTileKeys, j1 = b1 * kTileKeys;
                each_key(a, s, j0 > tv.begin ? j0 : tv.begin, j1 < tv.end ? j1 : tv.end, [&](int j, int64_t o) {
                    const bool in = sees(a, pos, j);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int d = 32 * i + 8 * c + 4 * hx;
                        if (d >= a.d) continue;
                        const u32x2 w = *reinterpret_cast<const u32x2 *>(vh + o + d);
#pragma unroll
                        for (int e = 0; e < 4; ++e) only[4 * c + e] += not_finite_of<T>(w[e >> 1], e & 1, in);
                    }
                });
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][e] = only[e] == 0.0f ? acc[i][e] : only[e];
            }
            // ---- the rows' sums over both halves of the keys, then the output
            {
                const uint32_t u = __builtin_bit_cast(uint32_t, l);
                const auto s32 = __builtin_amdgcn_permlane32_swap(u, u, false, false);
                l = __builtin_bit_cast(float, (uint32_t)s32[0]) + __builtin_bit_cast(float, (uint32_t)s32[1]);
                if (xl >= wrows) {
                } else if (w0 == w1) {
                    const float inv = one_over(l, m);
                    T *yr = Y + (int64_t)(sv.q0 + tok) * a.ldy + (int64_t)(hk * g + r - tok * g) * a.d;
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
                } else {
                    // partial result as the lanes hold it, device-coherent: another die's tile may join it
                    const uint32_t at = slot_at((int)t), pr = (uint32_t)(32 * lam + xl);
#pragma unroll
                    for (int i = 0; i < ND; ++i)
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            if (32 * i + 8 * c >= a.d) continue;
                            const f32x4 o = {acc[i][4 * c], acc[i][4 * c + 1], acc[i][4 * c + 2], acc[i][4 * c + 3]};
                            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, o), rw, (int)(at + (uint32_t)(((lam * ND + i) * 4 + c) * kWave + lane) * 16u), 0, kAgent);
                        }
                    if (hx == 0) {
                        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, m), rw, (int)(at + (kTileRows * DP + pr) * 4u), 0, kAgent);
                        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, l), rw, (int)(at + (kTileRows * (DP + 1) + pr) * 4u), 0, kAgent);
                    }
                }
            }
        }
        if (w0 != w1) {
            // the partial result's stores complete before the arrival is counted
            const int parts = w1 - w0 + 1;
            __builtin_amdgcn_s_waitcnt(0);
            __syncthreads();
            if (tid == 0) {
                const int prev = __hip_atomic_fetch_add(a.counters + out, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                s_last = prev == parts - 1;
                if (s_last) __hip_atomic_store(a.counters + out, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (s_last) {
                // each part's maxima and sums, then its share of each row's sum, in LDS (the stages are free); then
                // the outputs, the loads of several pieces in flight
                float *const weight = reinterpret_cast<float *>(smem), *const sums = weight + K_::PARTS * kTileRows;  // [parts][kTileRows]
#pragma unroll 8
                for (int i = tid; i < parts * kTileRows; i += kWave * P) {
                    const int w = i / kTileRows, r = i % kTileRows;
                    const uint32_t from = slot_at(w0 + w) + (uint32_t)(kTileRows * DP + r) * 4u;
                    weight[i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rw, (int)from, 0, kAgent));
                    sums[i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rw, (int)(from + kTileRows * 4u), 0, kAgent));
                }
                __syncthreads();
                for (int r = tid; r < rows; r += kWave * P) {
                    float top = -INFINITY, all = 0.0f;
                    for (int w = 0; w < parts; ++w) top = fmaxf(top, weight[w * kTileRows + r]);
                    const float ms = top == -INFINITY ? 0.0f : top;
                    for (int w = 0; w < parts; ++w) {
                        const float f = part_factor(weight[w * kTileRows + r], ms);
                        weight[w * kTileRows + r] = f;
                        all = __builtin_fmaf(f, sums[w * kTileRows + r], all);
                    }
                    const float inv = one_over(all, top);
                    for (int w = 0; w < parts; ++w) weight[w * kTileRows + r] = fmaxf(weight[w * kTileRows + r] * inv, kLeast);
                }
                __syncthreads();
                // piece i of a partial result: values 32 (i / 256 % ND) + 8 (i / 64 % 4) + 4 (i / 32 % 2) .. of row
                // 32 (i / (256 ND)) + i % 32
                constexpr int step = kWave * P, NB = 8;
                for (int i0 = tid; i0 < (rows + 31) / 32 * (256 * ND); i0 += NB * step) {
                    f32x4 o[NB];
#pragma unroll
                    for (int j = 0; j < NB; ++j) o[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                    auto row_of = [&](int j) { return 32 * ((i0 + j * step) / (256 * ND)) + (i0 + j * step) % 32; };
                    auto col_of = [&](int j) { return 32 * ((i0 + j * step) / 256 % ND) + 8 * ((i0 + j * step) / 64 % 4) + 4 * ((i0 + j * step) / 32 % 2); };
#pragma unroll 2
                    for (int w = 0; w < parts; ++w) {
                        f32x4 ow[NB];
#pragma unroll
                        for (int j = 0; j < NB; ++j)  // (rows and values that are not there lie in the workspace, too)
                            ow[j] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, (int)(slot_at(w0 + w) + (uint32_t)(i0 + j * step) * 16u), 0, kAgent));
#pragma unroll
                        for (int j = 0; j < NB; ++j) {
                            const float f = weight[w * kTileRows + row_of(j)];
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[j][e] = __builtin_fmaf(f, ow[j][e], o[j][e]);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < NB; ++j) {
                        const int rj = row_of(j), d = col_of(j);
                        if (rj >= rows || d >= a.d) continue;
                        const int tok = (int)fdiv((uint32_t)(row0 + rj), a.fd_group);
                        T *yr = Y + (int64_t)(sv.q0 + tok) * a.ldy + (int64_t)(hk * g + row0 + rj - tok * g) * a.d + d;
                        u32x2 w;
                        w[0] = pack2<T>(o[j][0], o[j][1]);
                        w[1] = pack2<T>(o[j][2], o[j][3]);
                        *reinterpret_cast<u32x2 *>(yr) = w;
                    }
                }
            }
            __syncthreads();  // s_last is free
        }
        at += list && unit == 0 ? take : 1;
        if (at < stop) onward();
        }
    }
}

template <class T, int DP, bool UNI, int DE>
inline void tile_table_u(const void *out[3], int *lds) {
    out[0] = reinterpret_cast<const void *>(&attend_tile_kernel<T, DP, 1, UNI, DE>);
    out[1] = reinterpret_cast<const void *>(&attend_tile_kernel<T, DP, 2, UNI, DE>);
    out[2] = reinterpret_cast<const void *>(&attend_tile_kernel<T, DP, 4, UNI, DE>);
    *lds = TileKernel<T, DP, 4, DE>::LDS_BYTES;
}
// uni: a load's 512 / dp rows lie in one page (the page a multiple of them) and span less than 2^31 bytes
template <class T, int DP, int DE = DP>
inline void tile_table(bool uni, const void *out[3], int *lds) {
    if (uni) tile_table_u<T, DP, true, DE>(out, lds);
    else tile_table_u<T, DP, false, DE>(out, lds);
}

}  // namespace miriam
