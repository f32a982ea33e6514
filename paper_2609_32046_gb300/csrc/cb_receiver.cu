// C-ABI of the receiver's side (declared in include/cacheback.h): rotary positions, rows held in 4
// bits, attention over them.  Validation and launch plumbing.
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "cb_ctx.cuh"

using namespace cbk;

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 31;
constexpr int64_t kMaxPos = (int64_t)1 << 40;

// A dimension of a strided array: `count` steps of `stride` elements.
struct Dim {
    int64_t count, stride;
};

// Strides are positive multiples of 8 where the dimension has more than one entry.
bool strides_ok(const Dim* dims, int n) {
    for (int i = 0; i < n; ++i)
        if (dims[i].count > 1 && !stride_ok(dims[i].stride)) return false;
    return true;
}

// No two rows of `row` elements share memory: every dimension steps over all that the shorter strides span.
bool rows_apart(Dim* dims, int n, int64_t row) {
    for (int i = 0; i < n; ++i)
        for (int j = i + 1; j < n; ++j)
            if (dims[j].stride < dims[i].stride) { const Dim t = dims[i]; dims[i] = dims[j]; dims[j] = t; }
    int64_t span = row;
    for (int i = 0; i < n; ++i) {
        if (dims[i].count <= 1) continue;
        if (dims[i].stride < span) return false;
        span += (dims[i].count - 1) * dims[i].stride;
    }
    return true;
}

// Elements from the first to behind the last of a strided array (0 where it is empty); -1 where that passes 2^60.
int64_t span_of(const Dim* dims, int n, int64_t row) {
    int64_t span = row;
    for (int i = 0; i < n; ++i) {
        if (dims[i].count <= 0) return 0;
        if (dims[i].count == 1) continue;
        if (dims[i].stride > ((int64_t)1 << 60) / dims[i].count) return -1;
        span += (dims[i].count - 1) * dims[i].stride;
        if (span > ((int64_t)1 << 60)) return -1;
    }
    return span;
}

int log2_of(int32_t page_size) {
    int sh = 0;
    while ((1 << sh) < page_size) ++sh;
    return sh;
}

cb_status check_page_fields(cb_ctx* ctx, DevicePtrs& ptrs, const int32_t* pages, int32_t page_size, int64_t n_pages, const char* what, int i) {
    if (page_size < 1 || page_size > 65536 || (page_size & (page_size - 1)) != 0)
        return fail(ctx, CB_EINVAL, "%s[%d].page_size = %d is not a power of two in [1, 65536]", what, i, page_size);
    if (n_pages < 1) return fail(ctx, CB_EINVAL, "%s[%d].n_pages must be at least 1", what, i);
    return ptrs.check(pages, "pages", i, 4);
}

// The most rows of a cache: positions are counted in 32 bits, a few tiles past the last one too.
constexpr int64_t kMaxHeld = kMaxRows - 4096;

cb_status check_packed(cb_ctx* ctx, DevicePtrs& ptrs, const cb_packed& p, int i, int64_t most = kMaxHeld) {
    const int d = ctx->cfg.head_dim;
    if (p.T < 0 || p.T > most)
        return fail(ctx, CB_ESHAPE, "caches[%d].T = %lld not in [0, %lld]", i, (long long)p.T, (long long)most);
    cb_status st;
    if (p.length && (st = ptrs.check(p.length, "caches.length", i, 4))) return st;
    if (p.T == 0) return CB_OK;
    const int scale_align = d == 128 ? 8 : 4;
    if ((st = ptrs.check(p.k, "caches.k", i))) return st;
    if ((st = ptrs.check(p.v, "caches.v", i))) return st;
    if ((st = ptrs.check(p.k_scale, "caches.k_scale", i, scale_align))) return st;
    if ((st = ptrs.check(p.v_scale, "caches.v_scale", i, scale_align))) return st;
    auto ok = [d](int64_t s) { return s > 0 && s % d == 0 && s / d < kMaxRows * 16; };
    if (!ok(p.s_layer) || !ok(p.s_head) || !ok(p.s_pos))
        return fail(ctx, CB_EINVAL, "caches[%d]: strides must be positive multiples of head_dim", i);
    if (p.pages) {
        if (!ok(p.s_page)) return fail(ctx, CB_EINVAL, "caches[%d].s_page must be a positive multiple of head_dim", i);
        if ((st = check_page_fields(ctx, ptrs, p.pages, p.page_size, p.n_pages, "caches", i))) return st;
        if (p.n_pages > kMaxRows || p.s_page / d > kMaxRows / p.n_pages ||
            p.s_pos / d > kMaxRows / p.page_size ||
            (p.n_pages - 1) * (p.s_page / d) + (p.page_size - 1) * (p.s_pos / d) >= kMaxRows)
            return fail(ctx, CB_ESHAPE, "caches[%d]: the pages of a layer and head span 2^31 rows or more", i);
    } else if (p.s_pos / d > kMaxRows / p.T) {
        return fail(ctx, CB_ESHAPE, "caches[%d]: the rows of a layer and head span 2^31 rows or more", i);
    }
    return CB_OK;
}

PackedRows packed_rows(const cb_packed& p, int d) {
    PackedRows r{};
    r.code[0] = static_cast<uint8_t*>(p.k);
    r.code[1] = static_cast<uint8_t*>(p.v);
    r.scale[0] = static_cast<uint16_t*>(p.k_scale);
    r.scale[1] = static_cast<uint16_t*>(p.v_scale);
    r.s_layer = p.s_layer / d;
    r.s_head = p.s_head / d;
    r.s_pos = p.s_pos / d;
    if (p.pages) {
        r.pages = p.pages;
        r.s_page = p.s_page / d;
        r.n_pages = p.n_pages;
        r.shift = log2_of(p.page_size);
    }
    return r;
}

// The frequencies of a cb_rope as turns of 2^64, and what cosine and sine are multiplied by.  Base powers are
// successive products (a powl each took 120 us of host time); kept with the context for the next call.
cb_status rope_table(cb_ctx* ctx, const cb_rope& p, int dims) {
    RopeTable& t = ctx->rope;
    if (t.dims == dims && std::memcmp(&t.key, &p, sizeof p) == 0) return CB_OK;
    if (!(std::isfinite(p.base) && p.base > 1.0)) return fail(ctx, CB_EINVAL, "rope base must be finite and > 1");
    if (p.scaling < 0 || p.scaling > 2) return fail(ctx, CB_EINVAL, "rope scaling %d not in 0..2", p.scaling);
    if (p.scaling && !(std::isfinite(p.factor) && p.factor >= 1.0))
        return fail(ctx, CB_EINVAL, "rope factor must be finite and >= 1");
    if (!(std::isfinite(p.attention) && p.attention >= 0.0))
        return fail(ctx, CB_EINVAL, "rope attention must be finite and >= 0");
    double lo = 0, hi = 1, gain = p.attention > 0 ? p.attention : 1.0;
    if (p.scaling == 2) {
        const double fast = p.beta_fast == 0 ? 32.0 : p.beta_fast, slow = p.beta_slow == 0 ? 1.0 : p.beta_slow;
        if (p.original < 1 || !(std::isfinite(fast) && slow > 0 && fast > slow))
            return fail(ctx, CB_EINVAL, "rope original must be >= 1 and beta_fast > beta_slow > 0");
        const double per = dims / (2 * std::log(p.base)), full = (double)p.original / (2 * 3.14159265358979323846);
        lo = std::floor(per * std::log(full / fast));
        hi = std::ceil(per * std::log(full / slow));
        lo = lo > 0 ? lo : 0;
        hi = hi < dims - 1 ? hi : dims - 1;
        if (hi <= lo) hi = lo + 0.001;
        if (p.attention == 0) gain = 0.1 * std::log(p.factor) + 1.0;
    }
    const long double ratio = powl((long double)p.base, -2.0L / dims);
    long double f = 1.0L / 6.283185307179586476925286766559L;
    for (int k = 0; k < dims / 2; ++k, f *= ratio) {
        long double g = f;
        if (p.scaling == 1) g = f / p.factor;
        if (p.scaling == 2) {
            const double w = (k - lo) / (hi - lo), c = w < 0 ? 0 : w > 1 ? 1 : w;
            g = f * (1.0L - c) + f / p.factor * c;
        }
        t.turns[k] = (uint64_t)ldexpl(g, 64);
    }
    t.gain = (float)gain;
    t.key = p;
    t.dims = dims;
    return CB_OK;
}

cb_status rotary_impl(cb_ctx* ctx, int32_t n, const cb_vectors* sets, const cb_rope* rope, cudaStream_t strm) {
    const int d = ctx->cfg.head_dim;
    if (n < 1) return fail(ctx, CB_ESHAPE, "n = %d < 1", n);
    if (!sets || !rope) return fail(ctx, CB_EINVAL, "sets or rope is NULL");
    if (rope->style != 0 && rope->style != 1) return fail(ctx, CB_EINVAL, "rope style %d not 0 or 1", rope->style);
    if (rope->inverse != 0 && rope->inverse != 1) return fail(ctx, CB_EINVAL, "rope inverse must be 0 or 1");
    if (rope->dims < 0 || rope->dims > d || rope->dims % 16)
        return fail(ctx, CB_EINVAL, "rope dims %d not a multiple of 16 up to %d", rope->dims, d);
    DeviceGuard dg(ctx->device);
    DevicePtrs ptrs(ctx);
    if (!dg.ok) return fail(ctx, CB_ECUDA, "cannot select device %d", ctx->device);
    const int dims = rope->dims ? rope->dims : d;
    cb_status st;
    if ((st = rope_table(ctx, *rope, dims))) return st;
    std::vector<int32_t> some;
    for (int i = 0; i < n; ++i) {
        const cb_vectors& v = sets[i];
        if (v.n_layers < 0 || v.n_heads < 0 || v.n_tokens < 0 || v.n_tokens >= kMaxRows ||
            (int64_t)v.n_layers * v.n_heads >= ((int64_t)1 << 24))
            return fail(ctx, CB_ESHAPE, "sets[%d]: counts are negative or too large", i);
        if (v.n_layers == 0 || v.n_heads == 0 || v.n_tokens == 0) continue;
        Dim in[3] = {{v.n_layers, v.s_layer}, {v.n_tokens, v.s_tok}, {v.n_heads, v.s_head}};
        Dim out[3] = {{v.n_layers, v.o_layer}, {v.n_tokens, v.o_tok}, {v.n_heads, v.o_head}};
        if (!strides_ok(in, 3) || !strides_ok(out, 3))
            return fail(ctx, CB_EINVAL, "sets[%d]: strides must be positive multiples of 8", i);
        const int64_t si = span_of(in, 3, d), so = span_of(out, 3, d);
        if (si < 0 || so < 0) return fail(ctx, CB_EINVAL, "sets[%d]: strides are too large", i);
        const bool same = v.x == v.y && (v.n_layers == 1 || v.s_layer == v.o_layer) &&
                          (v.n_tokens == 1 || v.s_tok == v.o_tok) && (v.n_heads == 1 || v.s_head == v.o_head);
        const char *x = static_cast<const char*>(v.x), *y = static_cast<const char*>(v.y);
        if (!same && x < y + 2 * so && y < x + 2 * si)
            return fail(ctx, CB_EINVAL, "sets[%d]: y overlaps x and is not x itself", i);
        if (!rows_apart(out, 3, d)) return fail(ctx, CB_EINVAL, "sets[%d]: vectors of y overlap", i);
        if ((st = ptrs.check(v.x, "sets.x", i)) || (st = ptrs.check(v.y, "sets.y", i))) return st;
        if (v.pos && (st = ptrs.check(v.pos, "sets.pos", i, 4))) return st;
        if (!v.pos && (v.pos0 < -kMaxPos || v.pos0 > kMaxPos - v.n_tokens))
            return fail(ctx, CB_EINVAL, "sets[%d].pos0 is not within +-2^40", i);
        some.push_back(i);
    }
    for (size_t b0 = 0; b0 < some.size(); b0 += kMaxBatch) {
        RotaryBatch b;
        std::memset(&b, 0, sizeof b);
        b.n = (int32_t)(some.size() - b0 < (size_t)kMaxBatch ? some.size() - b0 : kMaxBatch);
        b.dims = dims;
        b.gain = ctx->rope.gain;
        b.sine_gain = rope->inverse ? -b.gain : b.gain;
        std::memcpy(b.turns, ctx->rope.turns, sizeof b.turns);
        for (int k = 0; k < b.n; ++k) {
            const cb_vectors& v = sets[some[b0 + k]];
            RotarySet& s = b.s[k];
            s.x = static_cast<const uint16_t*>(v.x);
            s.y = static_cast<uint16_t*>(v.y);
            s.pos = v.pos;
            s.pos0 = v.pos0;
            s.n_tokens = v.n_tokens;
            s.n_layers = v.n_layers;
            s.n_heads = v.n_heads;
            s.s_layer = v.s_layer; s.s_tok = v.s_tok; s.s_head = v.s_head;
            s.o_layer = v.o_layer; s.o_tok = v.o_tok; s.o_head = v.o_head;
        }
        const cudaError_t e = launch_rotary(b, d, rope->style, strm, ctx->num_sms);
        if (e != cudaSuccess) return fail(ctx, CB_ECUDA, "rotary launch failed: %s", cudaGetErrorString(e));
    }
    return CB_OK;
}

cb_status pack_impl(cb_ctx* ctx, int32_t n, const cb_kv* senders, const int32_t* const* idx, const int64_t* count,
                    const cb_packed* caches, const int64_t* offset, const int32_t* const* rows, int32_t layer,
                    int32_t n_layers, cudaStream_t strm) {
    const cb_config& c = ctx->cfg;
    if (n < 1 || n > c.max_senders) return fail(ctx, CB_ESHAPE, "n = %d not in [1, %d]", n, c.max_senders);
    if (!senders || !count || !caches) return fail(ctx, CB_EINVAL, "senders, count or caches is NULL");
    if (layer < 0 || n_layers < 1 || n_layers > c.n_layers - layer)
        return fail(ctx, CB_ESHAPE, "layers [%d, %d) not in [0, %d)", layer, layer + n_layers, c.n_layers);
    DeviceGuard dg(ctx->device);
    DevicePtrs ptrs(ctx);
    if (!dg.ok) return fail(ctx, CB_ECUDA, "cannot select device %d", ctx->device);
    std::vector<const void*> kdev(n), vdev(n);
    cb_status st;
    for (int i = 0; i < n; ++i) {
        const cb_kv& s = senders[i];
        const bool by_row = rows && rows[i];
        if ((st = check_packed(ctx, ptrs, caches[i], i))) return st;
        if (count[i] < 0 || count[i] >= kMaxRows) return fail(ctx, CB_EBUDGET, "count[%d] = %lld", i, (long long)count[i]);
        if (count[i] == 0) continue;
        if (s.T < 1 || s.T > c.max_positions)
            return fail(ctx, CB_ESHAPE, "senders[%d].T = %lld not in [1, %lld]", i, (long long)s.T,
                        (long long)c.max_positions);
        if (!(idx && idx[i]) && count[i] > s.T)
            return fail(ctx, CB_EBUDGET, "count[%d] = %lld above senders[%d].T without idx", i, (long long)count[i], i);
        if (!by_row && (!offset || offset[i] < 0 || count[i] > caches[i].T || offset[i] > caches[i].T - count[i]))
            return fail(ctx, CB_EBUDGET, "sender %d: rows from offset on exceed caches[%d].T = %lld", i, i,
                        (long long)caches[i].T);
        if (by_row && caches[i].T == 0) return fail(ctx, CB_EBUDGET, "caches[%d] has no rows", i);
        if (!stride_ok(s.s_layer) || !stride_ok(s.s_head) || !stride_ok(s.s_pos) || s.s_pos < c.head_dim)
            return fail(ctx, CB_EINVAL, "senders[%d]: strides must be positive multiples of 8 (s_pos >= d)", i);
        if ((st = check_source_ptr(ctx, s.k, "senders.k", i, 16, &kdev[i]))) return st;
        if ((st = check_source_ptr(ctx, s.v, "senders.v", i, 16, &vdev[i]))) return st;
        if (s.pages) {
            if (!stride_ok(s.s_page)) return fail(ctx, CB_EINVAL, "senders[%d].s_page must be a positive multiple of 8", i);
            if ((st = check_page_fields(ctx, ptrs, s.pages, s.page_size, s.n_pages, "senders", i))) return st;
        }
        if (idx && idx[i] && (st = ptrs.check(idx[i], "idx", i, 4))) return st;
        if (by_row && (st = ptrs.check(rows[i], "rows", i, 4))) return st;
    }
    for (int b0 = 0; b0 < n; b0 += kMaxPackBatch) {
        PackBatch b;
        std::memset(&b, 0, sizeof b);
        b.n = n - b0 < kMaxPackBatch ? n - b0 : kMaxPackBatch;
        b.n_layers = n_layers;
        b.n_kv_heads = c.n_kv_heads;
        b.layer = layer;
        b.err = ctx->err;
        for (int k = 0; k < b.n; ++k) {
            const int i = b0 + k;
            const cb_kv& s = senders[i];
            PackSender& d = b.s[k];
            d.count = count[i];
            if (d.count == 0) continue;
            d.src[0] = static_cast<const uint16_t*>(kdev[i]);
            d.src[1] = static_cast<const uint16_t*>(vdev[i]);
            d.ks_l = s.s_layer; d.ks_h = s.s_head; d.ks_p = s.s_pos;
            if (s.pages) d.pm = PageMap{s.pages, s.s_page, s.n_pages, log2_of(s.page_size)};
            d.T = s.T;
            d.idx = idx ? idx[i] : nullptr;
            d.rows = rows ? rows[i] : nullptr;
            d.dst_off = d.rows ? 0 : offset[i];
            d.dst_T = caches[i].T;
            d.held = packed_rows(caches[i], c.head_dim);
        }
        const cudaError_t e = launch_pack(b, c.head_dim, strm, ctx->num_sms);
        if (e != cudaSuccess) return fail(ctx, CB_ECUDA, "pack launch failed: %s", cudaGetErrorString(e));
    }
    return CB_OK;
}

cb_status unpack_impl(cb_ctx* ctx, int32_t n, const cb_packed* caches, const int32_t* const* idx, const int64_t* count,
                      void* k_out, void* v_out, int64_t out_capacity, const int64_t* out_offset, int64_t o_layer,
                      int64_t o_head, cudaStream_t strm) {
    const cb_config& c = ctx->cfg;
    if (n < 1 || n > c.max_senders) return fail(ctx, CB_ESHAPE, "n = %d not in [1, %d]", n, c.max_senders);
    if (!caches || !count || !out_offset) return fail(ctx, CB_EINVAL, "caches, count or out_offset is NULL");
    if (out_capacity < 0 || out_capacity >= kMaxRows) return fail(ctx, CB_EINVAL, "out_capacity not in [0, 2^31)");
    if (!stride_ok(o_head) || !stride_ok(o_layer) || o_head < out_capacity * c.head_dim ||
        o_layer / c.n_kv_heads < o_head)
        return fail(ctx, CB_EINVAL, "output strides must be multiples of 8 and not overlap rows");
    DeviceGuard dg(ctx->device);
    DevicePtrs ptrs(ctx);
    if (!dg.ok) return fail(ctx, CB_ECUDA, "cannot select device %d", ctx->device);
    cb_status st;
    if ((st = ptrs.check(k_out, "k_out", 0))) return st;
    if ((st = ptrs.check(v_out, "v_out", 0))) return st;
    for (int i = 0; i < n; ++i) {
        if ((st = check_packed(ctx, ptrs, caches[i], i))) return st;
        if (count[i] < 0 || count[i] >= kMaxRows) return fail(ctx, CB_EBUDGET, "count[%d] = %lld", i, (long long)count[i]);
        const bool by_idx = idx && idx[i];
        if (count[i] > 0 && (caches[i].T == 0 || (!by_idx && count[i] > caches[i].T)))
            return fail(ctx, CB_EBUDGET, "count[%d] = %lld above caches[%d].T", i, (long long)count[i], i);
        if (out_offset[i] < 0 || out_offset[i] > out_capacity - count[i])
            return fail(ctx, CB_EBUDGET, "cache %d: rows exceed out_capacity %lld", i, (long long)out_capacity);
        if (count[i] > 0 && by_idx && (st = ptrs.check(idx[i], "idx", i, 4))) return st;
    }
    for (int b0 = 0; b0 < n; b0 += kMaxPackBatch) {
        PackBatch b;
        std::memset(&b, 0, sizeof b);
        b.n = n - b0 < kMaxPackBatch ? n - b0 : kMaxPackBatch;
        b.n_layers = c.n_layers;
        b.n_kv_heads = c.n_kv_heads;
        b.out[0] = static_cast<uint16_t*>(k_out);
        b.out[1] = static_cast<uint16_t*>(v_out);
        b.o_layer = o_layer;
        b.o_head = o_head;
        b.err = ctx->err;
        for (int k = 0; k < b.n; ++k) {
            PackSender& d = b.s[k];
            d.count = count[b0 + k];
            if (d.count == 0) continue;
            d.T = caches[b0 + k].T;
            d.idx = idx ? idx[b0 + k] : nullptr;
            d.dst_off = out_offset[b0 + k];
            d.held = packed_rows(caches[b0 + k], c.head_dim);
        }
        const cudaError_t e = launch_unpack(b, c.head_dim, strm, ctx->num_sms);
        if (e != cudaSuccess) return fail(ctx, CB_ECUDA, "unpack launch failed: %s", cudaGetErrorString(e));
    }
    return CB_OK;
}

cb_status attend_impl(cb_ctx* ctx, int32_t layer, int32_t n, const cb_packed* caches, const cb_attend_query* queries,
                      int32_t causal, int64_t window, cudaStream_t strm) {
    const cb_config& c = ctx->cfg;
    const int d = c.head_dim;
    if (n < 1 || n > c.max_senders) return fail(ctx, CB_ESHAPE, "n = %d not in [1, %d]", n, c.max_senders);
    if (layer < 0 || layer >= c.n_layers) return fail(ctx, CB_ESHAPE, "layer %d not in [0, %d)", layer, c.n_layers);
    if (!caches || !queries) return fail(ctx, CB_EINVAL, "caches or queries is NULL");
    if (causal != 0 && causal != 1) return fail(ctx, CB_EINVAL, "causal must be 0 or 1");
    if (window < 0 || (window && !causal)) return fail(ctx, CB_EINVAL, "window must be >= 0, and 0 unless causal");
    DeviceGuard dg(ctx->device);
    DevicePtrs ptrs(ctx);
    if (!dg.ok) return fail(ctx, CB_ECUDA, "cannot select device %d", ctx->device);
    cb_status st;
    std::vector<int32_t> some;
    std::vector<Written> outs, lses;
    for (int i = 0; i < n; ++i) {
        const cb_attend_query& q = queries[i];
        if ((st = check_packed(ctx, ptrs, caches[i], i, c.max_positions < kMaxHeld ? c.max_positions : kMaxHeld))) return st;
        if (q.m < 0 || q.m > c.max_query_tokens)
            return fail(ctx, CB_ESHAPE, "queries[%d].m = %d not in [0, %d]", i, q.m, c.max_query_tokens);
        if (q.m == 0) continue;
        Dim in[2] = {{q.m, q.s_tok}, {c.n_q_heads, q.s_head}}, out[2] = {{q.m, q.o_tok}, {c.n_q_heads, q.o_head}};
        if (!strides_ok(in, 2) || !strides_ok(out, 2))
            return fail(ctx, CB_EINVAL, "queries[%d]: strides must be positive multiples of 8", i);
        const int64_t rows = (int64_t)q.m * c.n_q_heads, span = span_of(out, 2, d);
        if (span_of(in, 2, d) < 0 || span < 0 || !rows_apart(out, 2, d))
            return fail(ctx, CB_EINVAL, "queries[%d]: strides are too large, or rows of out overlap", i);
        if ((st = ptrs.check(q.q, "queries.q", i)) || (st = ptrs.check(q.out, "queries.out", i)))
            return st;
        if (q.lse && (st = ptrs.check(q.lse, "queries.lse", i, 4))) return st;
        // (units of work are counted in 32 bits)
        if ((caches[i].T / 128 + 2) * c.n_kv_heads * ((int64_t)q.m * ctx->G / 128 + 1) > ((int64_t)1 << 31) / kMaxBatch)
            return fail(ctx, CB_ESHAPE, "sequence %d: too many positions, heads and query tokens for one launch", i);
        const uintptr_t at = reinterpret_cast<uintptr_t>(q.out), e = reinterpret_cast<uintptr_t>(q.lse);
        outs.push_back(Written{at, at + 2 * (uintptr_t)span, span == rows * d});
        if (e) lses.push_back(Written{e, e + 4 * (uintptr_t)rows, true});
        some.push_back(i);
    }
    if (some.empty()) return CB_OK;
    if (written_twice(outs) || written_twice(lses))
        return fail(ctx, CB_EINVAL, "two sequences write the same rows of out or lse");
    if ((st = attend_scratch(ctx, strm))) return st;
    for (size_t b0 = 0; b0 < some.size(); b0 += kMaxBatch) {
        AttendBatch b;
        std::memset(&b, 0, sizeof b);
        b.n = (int32_t)(some.size() - b0 < (size_t)kMaxBatch ? some.size() - b0 : kMaxBatch);
        b.n_q_heads = c.n_q_heads;
        b.n_kv_heads = c.n_kv_heads;
        b.G = ctx->G;
        b.scale_log2e = ctx->scale * 1.4426950408889634f;
        b.causal = causal;
        b.window = window;
        b.err = ctx->err;
        b.part = ctx->attend_part;
        b.part_ml = ctx->attend_ml;
        b.tickets = ctx->attend_tickets;
        b.cuts = ctx->attend_cuts;
        b.wait_ns = (uint64_t)ctx->wait_ns;
        b.stall = ctx->stall_attend;
        for (int k = 0; k < b.n; ++k) {
            const cb_packed& p = caches[some[b0 + k]];
            const cb_attend_query& q = queries[some[b0 + k]];
            AttendSeq& s = b.s[k];
            s.kv = packed_rows(p, d);
            for (int x = 0; x < 2 && p.T; ++x) {
                s.kv.code[x] += layer * s.kv.s_layer * (d / 2);
                s.kv.scale[x] += layer * s.kv.s_layer * (d / 32);
            }
            b.span[k].T = p.T;
            b.span[k].length = p.length;
            b.span[k].m = q.m;
            s.q = static_cast<const uint16_t*>(q.q);
            s.out = static_cast<uint16_t*>(q.out);
            s.lse = q.lse;
            s.s_tok = q.s_tok; s.s_head = q.s_head;
            s.o_tok = q.o_tok; s.o_head = q.o_head;
        }
        const cudaError_t e = launch_attend(b, d, strm, ctx->num_sms);
        ctx->stall_attend = b.stall;
        if (e != cudaSuccess) return fail(ctx, CB_ECUDA, "attend launch failed: %s", cudaGetErrorString(e));
    }
    return CB_OK;
}

// The body of an entry point: the context checked, no exception past the C boundary.
template <typename F>
cb_status entry(cb_ctx* ctx, const char* name, F body) {
    NvtxRange nr(name);
    if (!ctx) return fail(nullptr, CB_EINVAL, "ctx is NULL");
    try {
        ctx->last_error.clear();
        return body();
    } catch (const std::bad_alloc&) {
        return CB_ENOMEM;
    } catch (...) {
        return CB_EINVAL;
    }
}

}  // namespace

extern "C" {

cb_status cb_rotary(cb_ctx* ctx, int32_t n, const cb_vectors* sets, const cb_rope* rope, void* stream) {
    return entry(ctx, "cb_rotary", [&] { return rotary_impl(ctx, n, sets, rope, static_cast<cudaStream_t>(stream)); });
}

cb_status cb_pack(cb_ctx* ctx, int32_t n, const cb_kv* senders, const int32_t* const* idx, const int64_t* count,
                  const cb_packed* caches, const int64_t* offset, const int32_t* const* rows, int32_t layer,
                  int32_t n_layers, void* stream) {
    return entry(ctx, "cb_pack", [&] {
        return pack_impl(ctx, n, senders, idx, count, caches, offset, rows, layer, n_layers,
                         static_cast<cudaStream_t>(stream));
    });
}

cb_status cb_unpack(cb_ctx* ctx, int32_t n, const cb_packed* caches, const int32_t* const* idx, const int64_t* count,
                    void* k_out, void* v_out, int64_t out_capacity, const int64_t* out_offset, int64_t o_layer,
                    int64_t o_head, void* stream) {
    return entry(ctx, "cb_unpack", [&] {
        return unpack_impl(ctx, n, caches, idx, count, k_out, v_out, out_capacity, out_offset, o_layer, o_head,
                           static_cast<cudaStream_t>(stream));
    });
}

cb_status cb_attend(cb_ctx* ctx, int32_t layer, int32_t n, const cb_packed* caches, const cb_attend_query* queries,
                    int32_t causal, int64_t window, void* stream) {
    return entry(ctx, "cb_attend", [&] {
        return attend_impl(ctx, layer, n, caches, queries, causal, window, static_cast<cudaStream_t>(stream));
    });
}

}  // extern "C"
