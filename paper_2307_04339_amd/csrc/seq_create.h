// Operators over packed token rows: validation of their descriptors, tile spaces and kernel choice.  Part of
// ops.cpp, whose helpers it uses.
#pragma once

namespace miriam {

static bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// Rows of `n` elements of `es` bytes, `rows` of them `ld` elements apart.
struct Rows {
    const void *p;
    int64_t rows, n, ld;
    int es;
};

// Whether two sets of rows share memory.  Rows of the same stride are compared by column, so that columns of
// their own in one buffer are apart.
static bool overlap(const Rows &a, const Rows &b) {
    if (!a.p || !b.p || a.rows < 1 || b.rows < 1) return false;
    const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
    const uintptr_t a1 = a0 + (uintptr_t)(((a.rows - 1) * a.ld + a.n) * a.es), b1 = b0 + (uintptr_t)(((b.rows - 1) * b.ld + b.n) * b.es);
    if (a1 <= b0 || b1 <= a0) return false;
    if (a.ld * a.es != b.ld * b.es) return true;
    const int64_t ld = a.ld * a.es, off = (int64_t)((b0 + (uintptr_t)ld * 2 - a0 % (uintptr_t)ld) % (uintptr_t)ld);
    // b's columns begin `off` bytes behind a's, modulo the stride
    return off < a.n * a.es || off + b.n * b.es > ld;
}

constexpr int64_t kMost = (int64_t)1 << 30;  // rows, heads x values of a row, pages: indices stay in 32 bits

// Sequence arrays and caches of ROTARY (with a cache) and ATTENTION.
static int check_seqs(const miriam_seq_desc &d, SeqArgs &q, bool cache) {
    if (d.tokens < 1 || d.seqs < 1 || d.tokens >= kMost || d.seqs >= kMost) return einval("tokens and seqs must be >= 1 and below 2^30");
    if (!d.q_start || !d.kv_len) return einval("q_start and kv_len are required");
    if (!aligned(d.q_start, 4) || !aligned(d.kv_len, 4) || !aligned(d.page_table, 4)) return einval("q_start, kv_len and page_table must be 4-byte aligned");
    q.q_start = d.q_start;
    q.kv_len = d.kv_len;
    q.tokens = d.tokens;
    q.seqs = d.seqs;
    q.table = nullptr;
    q.page = q.pages = q.max_pages = 1;
    q.fd_page = make_fastdiv(1);
    if (!cache) return MIRIAM_OK;
    if (!d.k_cache || !d.v_cache || !d.page_table) return einval("k_cache, v_cache and page_table are required");
    if (d.page < 1 || d.pages < 1 || d.max_pages < 1 || d.page >= kMost || d.pages >= kMost || d.max_pages >= kMost ||
        d.page * d.max_pages >= kMost)
        return einval("page, pages and max_pages must be >= 1, and page * max_pages below 2^30");
    q.ldt = d.ldt > 0 ? d.ldt : d.max_pages;
    if (q.ldt < d.max_pages || q.ldt > ((int64_t)1 << 58) / d.seqs) return einval("page table: row stride too small or too large");
    if (d.cache_page < 1 || d.cache_head < 1 || d.cache_token < 1) return einval("cache strides must be >= 1");
    if (d.page > 1 && d.cache_token < d.head_dim) return einval("cache: token stride smaller than a head");
    constexpr int64_t far = (int64_t)1 << 58;  // bytes of a cache stay below 2^62
    if (d.cache_page > far / d.pages || d.cache_head > far / std::max<int64_t>(d.kv_heads, 1) || d.cache_token > far / d.page)
        return einval("cache strides are too large");
    q.table = d.page_table;
    q.sp = d.cache_page;
    q.sh = d.cache_head;
    q.st = d.cache_token;
    q.page = (int32_t)d.page;
    q.pages = (int32_t)d.pages;
    q.max_pages = (int32_t)d.max_pages;
    q.fd_page = make_fastdiv((uint32_t)d.page);
    return MIRIAM_OK;
}

// A cache from its first value to its last (with the other one in between where they are interleaved).
static Rows cache_span(const miriam_seq_desc &d, const void *p, int es) {
    const int64_t n = (d.pages - 1) * d.cache_page + (d.kv_heads - 1) * d.cache_head + (d.page - 1) * d.cache_token + d.head_dim;
    return {p, 1, n, n, es};
}

// Whether rows that are stored share memory with the arrays of the batch.
static bool over_batch(const miriam_seq_desc &d, const SeqArgs &q, const Rows &out) {
    return overlap({q.q_start, 1, q.seqs + 1, q.seqs + 1, 4}, out) || overlap({q.kv_len, 1, q.seqs, q.seqs, 4}, out) ||
           overlap({q.table, q.seqs, d.max_pages, q.ldt, 4}, out);
}

// Dimensions of a cache, by their steps (those of one entry, which step nowhere, first).
struct CacheDims {
    struct {
        int64_t step, n;
    } dim[3];
};
static CacheDims cache_dims(const miriam_seq_desc &d) {
    CacheDims c = {{{d.cache_page, d.pages}, {d.cache_head, d.kv_heads}, {d.cache_token, d.page}}};
    for (auto &m : c.dim)
        if (m.n < 2) m.step = 0;
    std::sort(c.dim, c.dim + 3, [](const auto &a, const auto &b) { return a.step < b.step; });
    return c;
}

// Whether each dimension steps past all that the ones of shorter steps reach: every place of the cache is its own then.
static bool own_places(const CacheDims &c, int64_t head_dim) {
    int64_t reach = head_dim;
    for (const auto &m : c.dim) {
        if (m.n < 2) continue;
        if (m.step < reach) return false;
        reach += (m.n - 1) * m.step;
    }
    return true;
}

// Whether two such caches, `apart` values from one to the other, share a place: whether apart is a sum of steps and of
// less than a head.  What is left for the shorter steps is less than the longest one, so only the two multiples of that
// next to `apart` may be among them.
static bool share_places(const CacheDims &c, int64_t head_dim, int64_t apart, int dims = 3) {
    if (dims == 0) return apart < head_dim && -apart < head_dim;
    const auto &m = c.dim[dims - 1];
    if (m.n < 2) return share_places(c, head_dim, apart, dims - 1);
    const int64_t q = apart / m.step - (apart % m.step < 0 ? 1 : 0);  // floor
    for (int64_t k = q; k <= q + 1; ++k)
        if (k < m.n && -k < m.n && share_places(c, head_dim, apart - k * m.step, dims - 1)) return true;
    return false;
}

// The heads of a descriptor.
static int check_heads(const miriam_seq_desc &d) {
    if (d.heads < 1 || d.kv_heads < 0 || d.head_dim < 1 || d.heads >= kMost || d.kv_heads >= kMost || d.head_dim >= kMost ||
        (d.heads + 2 * d.kv_heads) > kMost / d.head_dim)
        return einval("heads and head_dim must be >= 1, kv_heads >= 0, and a row below 2^30 values");
    return MIRIAM_OK;
}

static int create_norm(miriam_op *op) {
    const miriam_seq_desc &d = op->sd;
    NormArgs &a = op->nm;
    std::memset(&a, 0, sizeof(a));
    const int es = d.dtype == MIRIAM_F32 ? 4 : 2, V = 16 / es;
    if (d.tokens < 1 || d.n < 1 || d.tokens >= kMost || d.n >= kMost) return einval("block norm: tokens and n must be >= 1 and below 2^30");
    if (d.flags & ~MIRIAM_SEQ_LAYER_NORM) return einval("block norm: unknown flag");
    if (d.gate_kind < MIRIAM_GATE_NONE || d.gate_kind > MIRIAM_GATE_SIGMOID) return einval("block norm: unknown gate");
    if ((d.gate_kind != MIRIAM_GATE_NONE) != (d.gate != nullptr)) return einval("block norm: a gate and its kind go together");
    if (!d.x) return einval("block norm: x is required");
    if (!d.y && !d.z) return einval("block norm: y or z is required");
    if ((d.z != nullptr) != (d.pre != nullptr)) return einval("block norm: z and pre go together");
    if ((d.post_bias && !d.post) || (d.pre_bias && !d.pre)) return einval("block norm: a bias without its weights");
    if (!(d.eps >= 0.0f) || !std::isfinite(d.eps)) return einval("block norm: eps must be >= 0");
    if (!std::isfinite(d.scale)) return einval("block norm: scale must be finite");
    const bool rows_gate = d.gate_kind > MIRIAM_GATE_CHANNEL;
    a.x = d.x; a.res = d.residual; a.gate = d.gate; a.y = d.y; a.z = d.z;
    a.post = d.post; a.post_bias = d.post_bias; a.pre = d.pre; a.pre_bias = d.pre_bias;
    a.rows = d.tokens; a.n = d.n;
    a.ldx = d.ldx > 0 ? d.ldx : d.n;
    a.ldr = d.ldr > 0 ? d.ldr : d.n;
    a.ldg = d.ldg > 0 ? d.ldg : d.n;
    a.ldy = d.ldy > 0 ? d.ldy : d.n;
    a.ldz = d.ldz > 0 ? d.ldz : d.n;
    if (std::min({a.ldx, a.ldr, a.ldg, a.ldy, a.ldz}) < d.n || std::max({a.ldx, a.ldr, a.ldg, a.ldy, a.ldz}) >= kMost)
        return einval("block norm: row stride too small or too large");
    a.scale = d.scale; a.eps = d.eps; a.gate_kind = d.gate_kind;
    a.layer = (d.flags & MIRIAM_SEQ_LAYER_NORM) ? 1 : 0;
    for (const void *p : {d.x, d.residual, rows_gate ? d.gate : nullptr, (const void *)d.y, (const void *)d.z})
        if (!aligned(p, (uintptr_t)es)) return einval("block norm: rows must be aligned to their type");
    for (const void *p : {(const void *)d.post, (const void *)d.post_bias, (const void *)d.pre, (const void *)d.pre_bias, rows_gate ? nullptr : d.gate})
        if (!aligned(p, 4)) return einval("block norm: weights must be 4-byte aligned");
    const Rows ins[3] = {{a.x, a.rows, a.n, a.ldx, es}, {a.res, a.rows, a.n, a.ldr, es}, {rows_gate ? a.gate : nullptr, a.rows, a.n, a.ldg, es}};
    const Rows y{a.y, a.rows, a.n, a.ldy, es}, z{a.z, a.rows, a.n, a.ldz, es};
    for (const Rows &in : ins)
        if (overlap(in, y) || overlap(in, z)) return einval("block norm: an output overlaps an input");
    for (const float *w : {d.post, d.post_bias, d.pre, d.pre_bias, rows_gate ? nullptr : static_cast<const float *>(d.gate)})
        if (overlap({w, 1, a.n, a.n, 4}, y) || overlap({w, 1, a.n, a.n, 4}, z)) return einval("block norm: an output overlaps weights");
    if (overlap(y, z)) return einval("block norm: y and z overlap");
    // 16-byte vectors, or pieces at any alignment with the last one by element
    const bool vec = d.n % V == 0 && a.ldx % V == 0 && aligned(a.x, 16) && (!a.res || (a.ldr % V == 0 && aligned(a.res, 16))) &&
                     (!rows_gate || (a.ldg % V == 0 && aligned(a.gate, 16))) && (!a.y || (a.ldy % V == 0 && aligned(a.y, 16))) &&
                     (!a.z || (a.ldz % V == 0 && aligned(a.z, 16)));
    // (a rest of less than a vector is held besides: 777 rows of 2050 fp32 in two vectors of a lane 11.4 us, in four 15.4)
    const int64_t wave = (int64_t)kWave * V, held = vec ? d.n : d.n / V * V;
    const int form = d.n <= wave ? NORM_WAVE1 : d.n <= 2 * wave ? NORM_WAVE2 : held <= 4 * wave ? NORM_TILE1 : held <= 8 * wave ? NORM_TILE2
                     : held <= 16 * wave ? NORM_TILE4 : held <= 32 * wave ? NORM_TILE8 : NORM_LONG;
    op->T = form <= NORM_WAVE2 ? cdiv(a.rows, kLogicalWaves) : a.rows;
    op->lds_bytes = form <= NORM_WAVE2 ? 0 : 64;
    if (norm_kernels(d.dtype, form, vec, op->kern) != 0) return einval("block norm: no kernel for this dtype");
    const double e = (double)a.rows * a.n;
    op->flops = 12.0 * e;
    op->bytes = es * e * (1.0 + (a.res ? 1 : 0) + (rows_gate ? 1 : 0) + (a.y ? 1 : 0) + (a.z ? 1 : 0)) +
                4.0 * a.n * ((a.post ? 1 : 0) + (a.post_bias ? 1 : 0) + (a.pre ? 1 : 0) + (a.pre_bias ? 1 : 0) + (a.gate && !rows_gate ? 1 : 0));
    a.past = op->bytes > kPastBytes;
    return MIRIAM_OK;
}

static int create_rotary(miriam_op *op) {
    const miriam_seq_desc &d = op->sd;
    RotaryArgs &a = op->ro;
    std::memset(&a, 0, sizeof(a));
    const int es = d.dtype == MIRIAM_F32 ? 4 : 2, V = 16 / es;
    int rc = check_heads(d);
    if (rc) return rc;
    if (d.flags & ~MIRIAM_SEQ_INTERLEAVED) return einval("rotary: unknown flag");
    if (!d.x || !d.y) return einval("rotary: x and y are required");
    if (d.rot < 0 || d.rot % 2 != 0 || d.rot > d.head_dim) return einval("rotary: rot must be even and at most head_dim");
    if (d.rot > 0 && (!d.freq || !aligned(d.freq, 8))) return einval("rotary: freq (8-byte aligned) is required");
    if (!std::isfinite(d.scale)) return einval("rotary: scale must be finite");
    rc = check_seqs(d, a.sq, d.kv_heads > 0);
    if (rc) return rc;
    const int64_t width = (d.heads + 2 * d.kv_heads) * d.head_dim;
    a.x = d.x; a.y = d.y; a.freq = d.freq;
    if (d.kv_heads > 0) {
        a.k = d.k_cache;
        a.v = d.v_cache;
    }
    a.ldx = d.ldx > 0 ? d.ldx : width;
    a.ldy = d.ldy > 0 ? d.ldy : d.heads * d.head_dim;
    if (a.ldx < width || a.ldy < d.heads * d.head_dim || std::max(a.ldx, a.ldy) >= kMost) return einval("rotary: row stride too small or too large");
    for (const void *p : {a.x, (const void *)a.y, (const void *)a.k, (const void *)a.v})
        if (!aligned(p, (uintptr_t)es)) return einval("rotary: x, y and the caches must be aligned to their type");
    const Rows x{a.x, d.tokens, width, a.ldx, es}, y{a.y, d.tokens, d.heads * d.head_dim, a.ldy, es};
    const Rows freq{d.rot > 0 ? a.freq : nullptr, 1, d.rot / 2, d.rot / 2, 8};
    if (overlap(x, y)) return einval("rotary: y overlaps x");
    if (over_batch(d, a.sq, y) || overlap(freq, y)) return einval("rotary: y overlaps q_start, kv_len, page_table or freq");
    if (d.kv_heads > 0) {
        const Rows k = cache_span(d, a.k, es), v = cache_span(d, a.v, es);
        if (a.k == a.v) return einval("rotary: both caches are one");
        // (two stores to one place would leave either)
        const uintptr_t ka = (uintptr_t)a.k, va = (uintptr_t)a.v, bytes = ka < va ? va - ka : ka - va;
        const CacheDims dims = cache_dims(d);
        if (!own_places(dims, d.head_dim)) return einval("rotary: places of a cache overlap (each stride must step past what the shorter ones reach)");
        if (share_places(dims, d.head_dim, (int64_t)std::min<uintptr_t>(bytes / (uintptr_t)es, (uintptr_t)1 << 62)))
            return einval("rotary: places of the two caches overlap");
        if (overlap(x, k) || overlap(x, v) || overlap(y, k) || overlap(y, v)) return einval("rotary: x or y overlaps a cache");
        for (const Rows &c : {k, v})
            if (over_batch(d, a.sq, c) || overlap(freq, c)) return einval("rotary: a cache overlaps q_start, kv_len, page_table or freq");
    }
    a.heads = (int32_t)d.heads; a.kv_heads = (int32_t)d.kv_heads; a.d = (int32_t)d.head_dim; a.rot = (int32_t)d.rot;
    a.interleaved = (d.flags & MIRIAM_SEQ_INTERLEAVED) ? 1 : 0;
    a.scale = d.scale;
    // items of two 16-byte vectors where the head and its turned part are whole items and every row is
    // aligned, else of two elements (an odd head's last value is an item of its own)
    const bool vec = d.head_dim % (2 * V) == 0 && d.rot % (2 * V) == 0 && a.ldx % V == 0 && a.ldy % V == 0 && aligned(a.x, 16) && aligned(a.y, 16) &&
                     (d.kv_heads == 0 || (aligned(a.k, 16) && aligned(a.v, 16) && a.sq.sp % V == 0 && a.sq.sh % V == 0 && a.sq.st % V == 0));
    const int v = vec ? V : 1;
    a.items = (int32_t)cdiv(d.head_dim, 2 * v);
    a.rot_items = (int32_t)(d.rot / (2 * v));
    // a row goes to as many logical waves as it has batches of four rounds over its heads, and while there are
    // fewer waves than the chip holds, to more
    const int64_t at_once = std::max<int64_t>(1, kWave / std::min<int64_t>(a.items, kWave));
    const int64_t rounds = cdiv(d.heads + 2 * d.kv_heads, at_once);
    a.parts = (int32_t)std::min<int64_t>(rounds, std::max<int64_t>(cdiv(rounds, 8), cdiv((int64_t)device_cus() * 8, d.tokens)));
    a.fd_parts = make_fastdiv((uint32_t)a.parts);
    op->T = cdiv(d.tokens * a.parts, kLogicalWaves);
    if (d.tokens * a.parts >= (int64_t)INT32_MAX) return einval("rotary: too large for 32-bit tile indexing");
    op->lds_bytes = 0;
    if (rotary_kernels(d.dtype, vec, op->kern) != 0) return einval("rotary: no kernel for this dtype");
    op->flops = 3.0 * (double)d.tokens * (double)(d.heads + d.kv_heads) * (double)d.rot;
    op->bytes = 2.0 * es * (double)d.tokens * (double)width;
    a.past = op->bytes > kPastBytes;
    return MIRIAM_OK;
}

static int create_attention(miriam_op *op) {
    const miriam_seq_desc &d = op->sd;
    AttendArgs &a = op->at;
    std::memset(&a, 0, sizeof(a));
    if (d.dtype == MIRIAM_F32) return einval("attention: needs fp16/bf16");
    int rc = check_heads(d);
    if (rc) return rc;
    if (d.flags & ~MIRIAM_SEQ_CAUSAL) return einval("attention: unknown flag");
    if (!d.x || !d.y) return einval("attention: x and y are required");
    if (d.kv_heads < 1 || d.heads % d.kv_heads != 0) return einval("attention: heads must be a multiple of kv_heads");
    if (d.head_dim % 8 != 0 || d.head_dim > 256) return einval("attention: head_dim must be a multiple of 8, at most 256");
    if (!std::isfinite(d.scale) || !(d.scale > 0.0f)) return einval("attention: scale must be positive and finite");
    if (d.window < 0 || d.max_q < 0) return einval("attention: window and max_q must be >= 0");
    rc = check_seqs(d, a.sq, true);
    if (rc) return rc;
    if (d.tokens * (d.heads / d.kv_heads) >= kMost) return einval("attention: too large for 32-bit row indexing");
    const int64_t width = d.heads * d.head_dim;
    a.x = d.x; a.y = d.y; a.k = d.k_cache; a.v = d.v_cache;
    a.ldx = d.ldx > 0 ? d.ldx : width;
    a.ldy = d.ldy > 0 ? d.ldy : width;
    if (std::min(a.ldx, a.ldy) < width || std::max(a.ldx, a.ldy) >= kMost) return einval("attention: row stride too small or too large");
    if (!aligned(a.x, 16) || !aligned(a.y, 16) || !aligned(a.k, 16) || !aligned(a.v, 16) || a.ldx % 8 != 0 || a.ldy % 8 != 0 ||
        a.sq.sp % 8 != 0 || a.sq.sh % 8 != 0 || a.sq.st % 8 != 0)
        return einval("attention: x, y and the caches must be 16-byte aligned, their strides multiples of 8");
    const Rows y{a.y, d.tokens, width, a.ldy, 2};
    if (overlap({a.x, d.tokens, width, a.ldx, 2}, y)) return einval("attention: y overlaps x");
    if (overlap(y, cache_span(d, a.k, 2)) || overlap(y, cache_span(d, a.v, 2))) return einval("attention: y overlaps a cache");
    if (over_batch(d, a.sq, y)) return einval("attention: y overlaps q_start, kv_len or page_table");
    a.heads = (int32_t)d.heads; a.kv_heads = (int32_t)d.kv_heads; a.group = (int32_t)(d.heads / d.kv_heads); a.d = (int32_t)d.head_dim;
    a.fd_group = make_fastdiv((uint32_t)a.group);
    a.fd_kv = make_fastdiv((uint32_t)a.kv_heads);
    a.max_q = (int32_t)(d.max_q > 0 ? std::min(d.max_q, d.tokens) : d.tokens);
    a.window = (int32_t)std::min<int64_t>(d.window, kMost);
    a.causal = (d.flags & MIRIAM_SEQ_CAUSAL) ? 1 : 0;
    a.scale = (float)((double)d.scale * 1.4426950408889634074);
    if (!std::isfinite(a.scale)) return einval("attention: scale is too large");
    const bool rows = (int64_t)a.max_q * a.group <= 16;
    const int dp = d.head_dim <= 64 ? 64 : d.head_dim <= 128 ? 128 : 256;
    const int64_t cus = device_cus(), part = attend_partial(rows ? 16 : kTileRows, dp) * 4, keys = d.page * d.max_pages;
    int64_t outputs;  // outputs that several tiles may share
    int64_t slots;    // partial results in the workspace
    if (rows) {
        // every tile takes an equal share of all sequences' blocks of keys, as they are on the device: two
        // tiles per CU, fewer where even full caches have no more blocks
        outputs = d.seqs * d.kv_heads;
        if (outputs >= kMost || outputs > kMost / cdiv(keys, kRowKeys)) return einval("attention: too large for 32-bit block indexing");
        op->T = std::min<int64_t>(2 * cus, outputs * cdiv(keys, kRowKeys));
        if (op->noalloc) op->T = std::min<int64_t>(op->T, (int64_t)(kScratchBytes - kScratchCounters) / (4 * part));
        slots = 4 * op->T;  // two per tile, and as many for joining in two stages
        a.splits = (int32_t)std::min<int64_t>(op->T, 2);
    } else {
        // a tile for every 128 query rows that there may be, and two per CU at least, which share the steps of a
        // smaller batch
        if (keys >= (int64_t)1 << 26) return einval("attention: page * max_pages must be below 2^26 for more than 16 query rows per cache head");
        const int64_t qt = std::min(d.tokens * a.group / kTileRows + d.seqs, d.seqs * cdiv((int64_t)a.max_q * a.group, kTileRows));
        if (qt >= kMost / d.kv_heads) return einval("attention: too large for 32-bit tile indexing");
        outputs = qt * d.kv_heads;
        a.tiles = (int32_t)qt;
        // (as many as runs of four steps of full caches, and in the device scratch as have room)
        int64_t runs = std::min<int64_t>(2 * cus, cdiv(outputs * cdiv(keys, kTileKeys), 4));
        if (op->noalloc) runs = std::min<int64_t>(runs, (int64_t)(kScratchBytes - kScratchCounters) / (2 * part));
        a.runs = (int32_t)runs;
        op->T = std::max(outputs, runs);
        slots = 2 * runs;
        a.splits = runs > 1 && cdiv(keys, kTileKeys) > 4 ? 2 : 1;
    }
    if (a.splits > 1) {
        // counters of the outputs, and for few rows of the first stage of joining
        const int64_t wbytes = slots * part, counters = outputs + (rows ? 2 * op->T : 0);
        const int wr = alloc_workspace(op, (size_t)wbytes, (size_t)(counters * 4), false);
        if (wr < 0) return wr;
        if (wr == 0) {
            a.splits = 1;
        } else {
            a.work = static_cast<float *>(op->work);
            a.work_bytes = (uint32_t)wbytes;
            a.counters = static_cast<int32_t *>(op->counters);
        }
    }
    if (a.splits == 1) op->T = outputs;
    if (op->T >= (int64_t)INT32_MAX) return einval("attention: too large for 32-bit tile indexing");
    a.T = op->T;
    // many rows: the rows of one load (512 / dp keys) always in one page
    const bool f16 = d.dtype == MIRIAM_F16, uni = d.page % (512 / dp) == 0 && d.cache_token < ((int64_t)1 << 26);
    if ((rows ? (f16 ? attend_rows_kernels_f16(dp, op->kern, &op->lds_bytes) : attend_rows_kernels_bf16(dp, op->kern, &op->lds_bytes))
              : (f16 ? attend_tile_kernels_f16(a.d, uni, op->kern, &op->lds_bytes) : attend_tile_kernels_bf16(a.d, uni, op->kern, &op->lds_bytes))) != 0)
        return einval("attention: no kernel for this dtype");
    // at full capacity
    op->flops = 4.0 * (double)d.tokens * (double)width * (double)keys;
    op->bytes = 4.0 * (double)d.tokens * (double)width + 4.0 * (double)d.seqs * (double)keys * (double)(d.kv_heads * d.head_dim);
    return MIRIAM_OK;
}

static int create_seq(miriam_op *op) {
    const miriam_seq_desc &d = op->sd;
    if (d.dtype < MIRIAM_F32 || d.dtype > MIRIAM_BF16) return einval("unknown dtype");
    switch (d.kind) {
    case MIRIAM_OP_BLOCK_NORM: op->family = FAM_NORM; return create_norm(op);
    case MIRIAM_OP_ROTARY: op->family = FAM_ROTARY; return create_rotary(op);
    case MIRIAM_OP_ATTENTION: op->family = FAM_ATTEND; return create_attention(op);
    default: return einval("unknown op kind");
    }
}

static void *seq_args(const miriam_op *op) {
    switch (op->family) {
    case FAM_NORM: return const_cast<NormArgs *>(&op->nm);
    case FAM_ROTARY: return const_cast<RotaryArgs *>(&op->ro);
    default: return const_cast<AttendArgs *>(&op->at);
    }
}

}  // namespace miriam
