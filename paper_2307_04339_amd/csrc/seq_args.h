// Kernel argument blocks of the operators over packed token rows, passed by value.
#pragma once

#include "kargs.h"

namespace miriam {

// Ops that move more than this read and write their rows past the caches: nothing would be left in L2 (8 x 4 MB) for
// a reader anyway, and lines that are used once no longer take places from others; and their tiles go over the dies
// in turn, so that all memory channels are busy at once.  With buffers that the last-level cache does not hold: norms
// of 8192 rows of 4096 69 -> 53 us (outputs alone 63, tiles in turn 60), positions of 8192 tokens of 48 heads of
// 128 49 -> 40 us (47, 45).  Where it does hold them, the limit matters little either way: norms and then a reader of both
// outputs 50.4 -> 49.2 us at 134 MB, 27.7 -> 28.9 at 67 MB, 21.4 -> 19.8 at 34 MB.
constexpr double kPastBytes = 32e6;

// The norms around a block.
struct NormArgs {
    const void *x, *res, *gate;                      // res, gate: null = none
    void *y, *z;                                     // either may be null
    const float *post, *post_bias, *pre, *pre_bias;  // null = none
    int64_t rows, n, ldx, ldr, ldg, ldy, ldz;
    float scale, eps;
    int32_t gate_kind;                               // miriam_gate
    int32_t layer;                                   // 1: layer norm, 0: RMS norm
    int32_t past;                                    // rows are read and written past the caches (see kPastBytes)
};

// What a row is divided into: one logical wave holding 1 or 2 vectors per lane; a tile's four logical waves
// holding 1, 2, 4 or 8; or the tile's four reading the row again for each pass.
enum NormForm { NORM_WAVE1 = 0, NORM_WAVE2 = 1, NORM_TILE1 = 2, NORM_TILE2 = 3, NORM_TILE4 = 4, NORM_TILE8 = 5, NORM_LONG = 6 };
constexpr int norm_regs(int form) {
    return form == NORM_WAVE1 || form == NORM_TILE1 ? 1 : form == NORM_WAVE2 || form == NORM_TILE2 ? 2 : form == NORM_TILE4 ? 4 : form == NORM_TILE8 ? 8 : 0;
}

// Sequences of packed rows over a paged cache (device arrays, clamped where they are read).
struct SeqArgs {
    const int32_t *q_start, *kv_len, *table;
    int64_t tokens, seqs, ldt;
    int64_t sp, sh, st;       // cache strides
    int32_t page, pages, max_pages;
    FastDiv fd_page;
};

struct RotaryArgs {
    const void *x;
    void *y, *k, *v;          // k, v: null without a cache
    const double *freq;
    SeqArgs sq;
    int64_t ldx, ldy;
    int32_t heads, kv_heads, d, rot;
    int32_t interleaved;
    int32_t items, rot_items; // vector pairs per head, and those of them that are turned
    int32_t past;             // rows are read and written past the caches (see kPastBytes)
    int32_t parts;            // logical waves per row
    FastDiv fd_parts;         // division by it
    float scale;
};

struct AttendArgs {
    const void *x;
    void *y;
    const void *k, *v;
    SeqArgs sq;
    int64_t ldx, ldy;
    int32_t heads, kv_heads, group, d;  // group = query heads per cache head
    FastDiv fd_group, fd_kv;  // division by group and kv_heads
    int32_t max_q, window, causal;
    float scale;              // times log2(e): the exponentials are powers of two
    int32_t splits;           // 1: every output is finished by one tile, 2: tiles may share one
    int64_t T;
    int32_t runs, tiles;      // many rows: tiles that share the list of all steps; row tiles of a cache head, at most
    float *work;              // partial results
    uint32_t work_bytes;
    int32_t *counters;        // arrivals per output; back to 0 once a pass over the op completes
};

constexpr int kRowKeys = 128;    // keys of a block of the kernel for few query rows: 32 for each logical wave
constexpr int kTileRows = 128;   // query rows of a tile of the kernel for many: 32 for each logical wave
constexpr int kTileKeys = 64;    // and its keys per step
// Runs that share a list of places: run k begins at floor(k places / runs).  (Without new tokens there are neither
// places nor runs, and nothing to divide.)
struct Runs {
    int runs, run, more;
    constexpr int start(int k) const { return k * run + k * more / runs; }
};
constexpr Runs runs_of(int places, int runs) {
    const int run = runs > 0 ? places / runs : 0;
    return {runs, run, places - run * runs};
}

// fp32 values of a partial result: rows x (dp values, maximum, sum)
constexpr int64_t attend_partial(int rows, int dp) { return (int64_t)rows * (dp + 2); }

}  // namespace miriam
