// C-ABI of the receiver's side (declared in include/cacheback.h): rotary positions, rows held in 4
// bits, attention over them.  Validation and launch plumbing.
#include <cmath>
#include <cstddef>
#include <cstring>
#include <new>
#include <utility>
#include <vector>

#include "cb_ctx.cuh"
#include "cb_weigh.cuh"

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

// The same from a layer on.
PackedRows packed_layer(const cb_packed& p, int d, int32_t layer) {
    PackedRows r = packed_rows(p, d);
    for (int x = 0; x < 2 && p.T; ++x) {
        r.code[x] += layer * r.s_layer * (d / 2);
        r.scale[x] += layer * r.s_layer * (d / 32);
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

// Bits of the m tokens of a sequence.
cb_status check_tree(cb_ctx* ctx, DevicePtrs& ptrs, const cb_tree& t, int32_t m, int i) {
    if (!t.seen) return CB_OK;
    if (m > 1 && (t.s_row < (m + 31) / 32 || t.s_row > kMaxRows))
        return fail(ctx, CB_EINVAL, "trees[%d].s_row = %lld words for %d tokens", i, (long long)t.s_row, m);
    return ptrs.check(t.seen, "trees.seen", i, 4);
}

void set_trees(AttendBatch&, int, const cb_tree*) {}
void set_trees(AttendTreeBatch& b, int k, const cb_tree* t) { b.tree[k] = TreeBits{t->seen, t->s_row}; }

// (units of work are counted in 32 bits)
bool too_much_work(const cb_ctx* ctx, int64_t T, int32_t m) {
    return (T / 128 + 2) * ctx->cfg.n_kv_heads * ((int64_t)m * ctx->G / 128 + 1) > ((int64_t)1 << 31) / kMaxBatch;
}

// Batch: AttendBatch, or AttendTreeBatch with trees.
template <class Batch>
cb_status attend_impl(cb_ctx* ctx, int32_t layer, int32_t n, const cb_packed* caches, const cb_attend_query* queries,
                      const cb_tree* trees, int32_t causal, int64_t window, cudaStream_t strm) {
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
        if (trees && (st = check_tree(ctx, ptrs, trees[i], q.m, i))) return st;
        if (too_much_work(ctx, caches[i].T, q.m))
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
        Batch b;
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
            s.kv = packed_layer(p, d, layer);
            b.span[k].T = p.T;
            b.span[k].length = p.length;
            b.span[k].m = q.m;
            s.q = static_cast<const uint16_t*>(q.q);
            s.out = static_cast<uint16_t*>(q.out);
            s.lse = q.lse;
            s.s_tok = q.s_tok; s.s_head = q.s_head;
            s.o_tok = q.o_tok; s.o_head = q.o_head;
            if (trees) set_trees(b, k, trees + some[b0 + k]);
        }
        const cudaError_t e = launch_attend(b, d, strm, ctx->num_sms);
        ctx->stall_attend = b.stall;
        if (e != cudaSuccess) return fail(ctx, CB_ECUDA, "attend launch failed: %s", cudaGetErrorString(e));
    }
    return CB_OK;
}

// fp32 arrays [n_layers][n_heads][rows] with unit steps over the rows: the elements they span, or -1 where rows overlap
// or the strides are too large.
int64_t weights_span(int64_t n_layers, int64_t s_layer, int64_t n_heads, int64_t s_head, int64_t rows) {
    Dim dims[2] = {{n_layers, s_layer}, {n_heads, s_head}};
    for (const Dim& x : dims)
        if (x.count > 1 && x.stride <= 0) return -1;
    const int64_t span = span_of(dims, 2, rows);
    return span < 0 || !rows_apart(dims, 2, rows) ? -1 : span;
}

bool touch(const void* a, int64_t bytes_a, const void* b, int64_t bytes_b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + (uintptr_t)bytes_b && y < x + (uintptr_t)bytes_a;
}

cb_status weigh_impl(cb_ctx* ctx, int32_t layer, int32_t n, const cb_packed* caches, const cb_weigh_query* queries,
                     const cb_tree* trees, int32_t causal, int64_t window, float decay, cudaStream_t strm) {
    const cb_config& c = ctx->cfg;
    const int d = c.head_dim;
    if (n < 1 || n > c.max_senders) return fail(ctx, CB_ESHAPE, "n = %d not in [1, %d]", n, c.max_senders);
    if (layer < 0 || layer >= c.n_layers) return fail(ctx, CB_ESHAPE, "layer %d not in [0, %d)", layer, c.n_layers);
    if (!caches || !queries) return fail(ctx, CB_EINVAL, "caches or queries is NULL");
    if (causal != 0 && causal != 1) return fail(ctx, CB_EINVAL, "causal must be 0 or 1");
    if (window < 0 || (window && !causal)) return fail(ctx, CB_EINVAL, "window must be >= 0, and 0 unless causal");
    if (trees && (!causal || window)) return fail(ctx, CB_EINVAL, "trees go with causal = 1 and window = 0");
    if (!(decay >= 0.f && decay <= 1.f)) return fail(ctx, CB_EINVAL, "decay must be within 0 .. 1");
    DeviceGuard dg(ctx->device);
    DevicePtrs ptrs(ctx);
    if (!dg.ok) return fail(ctx, CB_ECUDA, "cannot select device %d", ctx->device);
    cb_status st;
    std::vector<int32_t> some;
    std::vector<Written> written;
    for (int i = 0; i < n; ++i) {
        const cb_weigh_query& q = queries[i];
        if ((st = check_packed(ctx, ptrs, caches[i], i, c.max_positions < kMaxHeld ? c.max_positions : kMaxHeld))) return st;
        if (q.m < 0 || q.m > c.max_query_tokens)
            return fail(ctx, CB_ESHAPE, "queries[%d].m = %d not in [0, %d]", i, q.m, c.max_query_tokens);
        if (q.fresh < 0) return fail(ctx, CB_EINVAL, "queries[%d].fresh is negative", i);
        const int64_t T = caches[i].T;
        if (q.m == 0 || T == 0) continue;
        Dim in[2] = {{q.m, q.s_tok}, {c.n_q_heads, q.s_head}};
        if (!strides_ok(in, 2) || span_of(in, 2, d) < 0)
            return fail(ctx, CB_EINVAL, "queries[%d]: strides must be positive multiples of 8, and not too large", i);
        if ((st = ptrs.check(q.q, "queries.q", i)) || (st = ptrs.check(q.lse, "queries.lse", i, 4)) ||
            (st = ptrs.check(q.weights, "queries.weights", i, 4)) ||
            (q.before && (st = ptrs.check(q.before, "queries.before", i, 4))))
            return st;
        const int64_t span = weights_span(1, 0, c.n_kv_heads, q.w_head, T);
        const int64_t had = q.before ? weights_span(1, 0, c.n_kv_heads, q.b_head, T) : 0;
        if (span < 0 || had < 0) return fail(ctx, CB_EINVAL, "queries[%d]: rows of weights overlap, or the strides are too large", i);
        const bool same = q.before == q.weights && (c.n_kv_heads == 1 || q.b_head == q.w_head);
        if (q.before && !same && touch(q.weights, 4 * span, q.before, 4 * had))
            return fail(ctx, CB_EINVAL, "queries[%d]: weights overlap before and are not before itself", i);
        if (trees && (st = check_tree(ctx, ptrs, trees[i], q.m, i))) return st;
        if (too_much_work(ctx, T, q.m))
            return fail(ctx, CB_ESHAPE, "sequence %d: too many positions, heads and query tokens for one launch", i);
        const uintptr_t at = reinterpret_cast<uintptr_t>(q.weights);
        written.push_back(Written{at, at + 4 * (uintptr_t)span, span == T * c.n_kv_heads});
        some.push_back(i);
    }
    if (some.empty()) return CB_OK;
    if (written_twice(written)) return fail(ctx, CB_EINVAL, "two sequences write the same weights");
    // (sorted by now, or in order) what one sequence writes is not what another reads
    for (const int32_t i : some) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(queries[i].before);
        if (!at || queries[i].before == queries[i].weights) continue;
        const auto x = std::lower_bound(written.begin(), written.end(), at, [](const Written& a, uintptr_t b) { return a.lo < b; });
        if (x != written.end() && x->lo == at)
            return fail(ctx, CB_EINVAL, "queries[%d].before is another sequence's weights", i);
    }
    for (size_t b0 = 0; b0 < some.size(); b0 += kMaxBatch) {
        WeighBatch b;
        std::memset(&b, 0, sizeof b);
        b.n = (int32_t)(some.size() - b0 < (size_t)kMaxBatch ? some.size() - b0 : kMaxBatch);
        b.n_q_heads = c.n_q_heads;
        b.n_kv_heads = c.n_kv_heads;
        b.G = ctx->G;
        b.scale_log2e = ctx->scale * 1.4426950408889634f;
        b.err = ctx->err;
        b.wait_ns = (uint64_t)ctx->wait_ns;
        // (a weight is 2^(f z - l'): where f z and l' are far from 0 and their difference is not, f's rounding is taken from it by
        // an l' that has the same)
        const double log2e = (double)b.scale_log2e / (c.softmax_scale > 0.f ? (double)c.softmax_scale : 1.0 / std::sqrt((double)d));
        b.lse_log2e = (float)log2e;
        b.lse_log2e_lo = (float)(log2e - (double)b.lse_log2e);
        b.stall = ctx->stall_weigh;
        b.sees = causal;
        b.sees_window = window < kNoWindow ? (int32_t)window : 0;
        b.decay = decay;
        for (int k = 0; k < b.n; ++k) {
            const int i = some[b0 + k];
            const cb_weigh_query& q = queries[i];
            AttendSeq& s = b.s[k];
            WeighSeq& w = b.w[k];
            s.kv = packed_layer(caches[i], d, layer);
            s.q = static_cast<const uint16_t*>(q.q);
            s.s_tok = q.s_tok; s.s_head = q.s_head;
            b.span[k].T = caches[i].T;
            b.span[k].length = caches[i].length;
            b.span[k].m = q.m;
            w.lse = q.lse;
            w.before = q.before;
            w.weights = q.weights;
            w.b_head = q.b_head; w.w_head = q.w_head;
            w.fresh = q.fresh < kMaxRows ? q.fresh : kMaxRows;
            if (trees) w.tree = TreeBits{trees[i].seen, trees[i].s_row};
        }
        const cudaError_t e = launch_weigh(b, d, strm, ctx->num_sms);
        ctx->stall_weigh = b.stall;
        if (e != cudaSuccess) return fail(ctx, CB_ECUDA, "weigh launch failed: %s", cudaGetErrorString(e));
    }
    return CB_OK;
}

// Caches whose rows a call moves: nothing that one part writes may be another's.  What can be seen of that on the host: the
// same codes under the same block table, or rows of unpaged caches that overlap.
struct Places {
    std::vector<Written> codes;
    std::vector<std::pair<uintptr_t, uintptr_t>> paged;     // codes and table of every cache written
    std::vector<std::pair<uintptr_t, uintptr_t>> read, written;   // the same of those read and of all written, entry by entry
    std::vector<Written> weights, idx;
    std::vector<PartOf> weights_from, weights_to;             // weights that move: where they are read, and `weights` again
    std::vector<uintptr_t> lengths, left;                   // numbers that are read, and lengths that are written

    // An entry's rows: from a cache, to a cache.
    void add(const cb_packed& from, const cb_packed& p, int d, const cb_config& c) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p.k);
        read.emplace_back(reinterpret_cast<uintptr_t>(from.k), reinterpret_cast<uintptr_t>(from.pages));
        written.emplace_back(at, reinterpret_cast<uintptr_t>(p.pages));
        if (p.pages) {
            paged.emplace_back(at, reinterpret_cast<uintptr_t>(p.pages));
            return;
        }
        Dim dims[3] = {{c.n_layers, p.s_layer}, {c.n_kv_heads, p.s_head}, {p.T, p.s_pos}};
        const int64_t span = span_of(dims, 3, d), rows = c.n_layers * c.n_kv_heads * p.T;
        codes.push_back(Written{at, at + (uintptr_t)(span / 2), span == rows * d});
    }
    bool clash() {
        std::sort(paged.begin(), paged.end());
        for (size_t i = 1; i < paged.size(); ++i)
            if (paged[i] == paged[i - 1]) return true;
        std::sort(left.begin(), left.end());
        for (size_t i = 1; i < left.size(); ++i)
            if (left[i] == left[i - 1]) return true;
        // what one entry writes is not what another reads
        auto sorted = read;
        std::sort(sorted.begin(), sorted.end());
        for (size_t i = 0; i < written.size(); ++i) {
            const auto all = std::equal_range(sorted.begin(), sorted.end(), written[i]);
            if (all.second - all.first > (read[i] == written[i] ? 1 : 0)) return true;
        }
        return written_twice(codes) || written_twice(weights) || written_twice(idx) || read_and_written(weights_from, weights_to);
    }
    // A length that is written is also another cache's, or a count, which is read.  `own`: the length that each cache has and
    // the one it writes.
    bool lengths_clash(const std::vector<std::pair<uintptr_t, uintptr_t>>& own) {
        std::sort(lengths.begin(), lengths.end());
        for (const auto& x : own) {
            if (!x.second) continue;
            const auto all = std::equal_range(lengths.begin(), lengths.end(), x.second);
            if (all.second - all.first > (x.second == x.first ? 1 : 0)) return true;
        }
        return false;
    }
};

cb_status move_all(cb_ctx* ctx, std::vector<MoveSeq>& seqs, int32_t n_layers, cudaStream_t strm) {
    bool later = false;
    for (const MoveSeq& m : seqs) later |= m.left_later != 0;
    for (int pass = 0; pass < (later ? 2 : 1); ++pass)      // rows, then lengths
        for (size_t b0 = 0; b0 < seqs.size(); b0 += kMaxPackBatch) {
            MoveBatch b;
            std::memset(&b, 0, sizeof b);
            b.n = (int32_t)(seqs.size() - b0 < (size_t)kMaxPackBatch ? seqs.size() - b0 : kMaxPackBatch);
            b.n_layers = n_layers;
            b.n_kv_heads = ctx->cfg.n_kv_heads;
            b.err = ctx->err;
            for (int k = 0; k < b.n; ++k) b.s[k] = seqs[b0 + k];
            const cudaError_t e = pass ? launch_left(b, strm) : launch_move(b, ctx->cfg.head_dim, strm, ctx->num_sms);
            if (e != cudaSuccess) return fail(ctx, CB_ECUDA, "move launch failed: %s", cudaGetErrorString(e));
        }
    return CB_OK;
}

cb_status evict_impl(cb_ctx* ctx, int32_t layer, int32_t n_layers, int32_t n, const cb_packed* caches, const cb_packed* into,
                     const cb_eviction* evictions, cudaStream_t strm) {
    const cb_config& c = ctx->cfg;
    const int d = c.head_dim;
    if (n < 1 || n > c.max_senders) return fail(ctx, CB_ESHAPE, "n = %d not in [1, %d]", n, c.max_senders);
    if (!caches || !evictions) return fail(ctx, CB_EINVAL, "caches or evictions is NULL");
    if (layer < 0 || n_layers < 1 || n_layers > c.n_layers - layer)
        return fail(ctx, CB_ESHAPE, "layers [%d, %d) not in [0, %d)", layer, layer + n_layers, c.n_layers);
    DeviceGuard dg(ctx->device);
    DevicePtrs ptrs(ctx);
    if (!dg.ok) return fail(ctx, CB_ECUDA, "cannot select device %d", ctx->device);
    cb_status st;
    std::vector<MoveSeq> moves;
    std::vector<RankSeq> ranks;
    std::vector<std::pair<uintptr_t, uintptr_t>> lengths;
    Places places;
    const int64_t lists = (int64_t)n_layers * c.n_kv_heads;
    for (int i = 0; i < n; ++i) {
        const cb_packed& p = caches[i];
        const cb_eviction& e = evictions[i];
        if ((st = check_packed(ctx, ptrs, p, i))) return st;
        if (e.keep < 0 || e.keep >= kMaxRows || e.first < 0 || e.last < 0)
            return fail(ctx, CB_ESHAPE, "evictions[%d]: keep, first and last must be in [0, 2^31)", i);
        if (e.first > e.keep || e.last > e.keep - e.first)
            return fail(ctx, CB_EBUDGET, "evictions[%d]: first + last above keep = %lld", i, (long long)e.keep);
        if (e.length && (st = ptrs.check(e.length, "evictions.length", i, 4))) return st;
        const bool other = into && into[i].k != p.k;
        const cb_packed& to = into ? into[i] : p;
        if (into && (st = check_packed(ctx, ptrs, to, i))) return st;
        if (into && !other && std::memcmp(&to, &p, offsetof(cb_packed, length)) != 0)
            return fail(ctx, CB_EINVAL, "into[%d] has the codes of caches[%d] but is not the same cache", i, i);
        if (to.T < (e.keep < p.T ? e.keep : p.T))
            return fail(ctx, CB_EBUDGET, "into[%d].T = %lld has no room for %lld rows", i, (long long)to.T, (long long)e.keep);
        if (p.T > 0 && e.keep > 0) {
            if ((st = ptrs.check(e.weights, "evictions.weights", i, 4)) || (st = ptrs.check(e.idx, "evictions.idx", i, 4)) ||
                (e.weights_to && (st = ptrs.check(e.weights_to, "evictions.weights_to", i, 4))))
                return st;
            const int64_t rows = e.keep < p.T ? e.keep : p.T;
            const int64_t span = weights_span(n_layers, e.w_layer, c.n_kv_heads, e.w_head, p.T);
            const int64_t span_to = e.weights_to ? weights_span(n_layers, e.t_layer, c.n_kv_heads, e.t_head, rows) : 0;
            if (span < 0 || span_to < 0)
                return fail(ctx, CB_EINVAL, "evictions[%d]: rows of weights overlap, or the strides are too large", i);
            const bool same = e.weights == e.weights_to && (n_layers == 1 || e.w_layer == e.t_layer) &&
                              (c.n_kv_heads == 1 || e.w_head == e.t_head);
            if (e.weights_to && (other ? touch(e.weights, 4 * span, e.weights_to, 4 * span_to) : !same))
                return fail(ctx, CB_EINVAL, "evictions[%d]: weights move as the rows do, in place or to memory of their own", i);
            const uintptr_t w = reinterpret_cast<uintptr_t>(e.weights_to);
            if (w) {
                const uintptr_t from = reinterpret_cast<uintptr_t>(e.weights);
                places.weights.push_back(Written{w, w + 4 * (uintptr_t)span_to, span_to == lists * rows});
                places.weights_to.push_back(PartOf{places.weights.back(), i});
                places.weights_from.push_back(PartOf{{from, from + 4 * (uintptr_t)span, span == lists * p.T}, i});
            }
            places.add(p, to, d, c);
        }
        places.lengths.push_back(reinterpret_cast<uintptr_t>(p.length));
        if (e.length) places.left.push_back(reinterpret_cast<uintptr_t>(e.length));
        lengths.emplace_back(reinterpret_cast<uintptr_t>(p.length), reinterpret_cast<uintptr_t>(e.length));
        MoveSeq m{};
        m.count = e.keep;
        m.T = p.T;
        m.length = p.length;
        m.left = e.length;
        m.drafted = -1;
        if (e.keep > 0 && e.idx) {                     // (of an empty cache -1 everywhere: its weights are not read)
            if (p.T == 0 && (st = ptrs.check(e.idx, "evictions.idx", i, 4))) return st;
            const uintptr_t x = reinterpret_cast<uintptr_t>(e.idx);
            places.idx.push_back(Written{x, x + 4 * (uintptr_t)(lists * e.keep), true});
            RankSeq r{};
            r.weights = e.weights;
            r.w_layer = e.w_layer; r.w_head = e.w_head;
            r.T = p.T;
            r.length = p.length;
            r.keep = e.keep; r.first = e.first; r.last = e.last;
            r.idx = e.idx;
            ranks.push_back(r);
        }
        if (p.T > 0 && e.keep > 0) {
            m.from = packed_layer(p, d, layer);
            m.to = packed_layer(to, d, layer);
            m.w = e.weights_to ? e.weights : nullptr;
            m.w_to = e.weights_to;
            m.w_layer = e.w_layer; m.w_head = e.w_head;
            m.t_layer = e.t_layer; m.t_head = e.t_head;
            m.idx = e.idx;
            m.idx_list = e.keep;
            m.in_place = !other;
        } else {
            m.count = 0;
        }
        moves.push_back(m);
    }
    if (places.clash() || places.lengths_clash(lengths)) return fail(ctx, CB_EINVAL, "two parts of the call write the same memory");
    for (size_t b0 = 0; b0 < ranks.size(); b0 += kMaxBatch) {
        RankBatch b;
        std::memset(&b, 0, sizeof b);
        b.n = (int32_t)(ranks.size() - b0 < (size_t)kMaxBatch ? ranks.size() - b0 : kMaxBatch);
        b.n_layers = n_layers;
        b.n_kv_heads = c.n_kv_heads;
        for (int k = 0; k < b.n; ++k) b.s[k] = ranks[b0 + k];
        const cudaError_t e = launch_rank(b, strm);
        if (e != cudaSuccess) return fail(ctx, CB_ECUDA, "rank launch failed: %s", cudaGetErrorString(e));
    }
    return move_all(ctx, moves, n_layers, strm);
}

cb_status keep_impl(cb_ctx* ctx, int32_t n, const cb_packed* caches, const cb_kept* kept, cudaStream_t strm) {
    const cb_config& c = ctx->cfg;
    const int d = c.head_dim;
    if (n < 1 || n > c.max_senders) return fail(ctx, CB_ESHAPE, "n = %d not in [1, %d]", n, c.max_senders);
    if (!caches || !kept) return fail(ctx, CB_EINVAL, "caches or kept is NULL");
    DeviceGuard dg(ctx->device);
    DevicePtrs ptrs(ctx);
    if (!dg.ok) return fail(ctx, CB_ECUDA, "cannot select device %d", ctx->device);
    cb_status st;
    std::vector<MoveSeq> moves;
    std::vector<std::pair<uintptr_t, uintptr_t>> lengths;
    Places places;
    for (int i = 0; i < n; ++i) {
        const cb_packed& p = caches[i];
        const cb_kept& e = kept[i];
        if ((st = check_packed(ctx, ptrs, p, i))) return st;
        if (e.drafted < 0 || e.drafted > p.T || e.count < 0 || e.count > e.drafted)
            return fail(ctx, CB_EBUDGET, "kept[%d]: count = %lld of %lld drafted rows of a cache of %lld", i, (long long)e.count,
                        (long long)e.drafted, (long long)p.T);
        if (e.length && (st = ptrs.check(e.length, "kept.length", i, 4))) return st;
        if (e.n_kept && (st = ptrs.check(e.n_kept, "kept.n_kept", i, 4))) return st;
        places.lengths.push_back(reinterpret_cast<uintptr_t>(p.length));
        places.lengths.push_back(reinterpret_cast<uintptr_t>(e.n_kept));
        if (e.length) places.left.push_back(reinterpret_cast<uintptr_t>(e.length));
        lengths.emplace_back(reinterpret_cast<uintptr_t>(p.length), reinterpret_cast<uintptr_t>(e.length));
        MoveSeq m{};
        m.T = p.T;
        m.length = p.length;
        m.left = e.length;
        m.drafted = e.drafted;
        m.n_kept = e.n_kept;
        m.left_later = e.length && e.length == p.length;
        m.in_place = 1;
        if (e.count > 0) {
            if ((st = ptrs.check(e.idx, "kept.idx", i, 4)) || (e.weights && (st = ptrs.check(e.weights, "kept.weights", i, 4))))
                return st;
            if (e.weights) {
                const int64_t span = weights_span(c.n_layers, e.w_layer, c.n_kv_heads, e.w_head, p.T);
                if (span < 0) return fail(ctx, CB_EINVAL, "kept[%d]: rows of weights overlap, or the strides are too large", i);
                const uintptr_t w = reinterpret_cast<uintptr_t>(e.weights);
                places.weights.push_back(Written{w, w + 4 * (uintptr_t)span, span == (int64_t)c.n_layers * c.n_kv_heads * p.T});
            }
            places.add(p, p, d, c);
            m.count = e.count;
            m.from = m.to = packed_rows(p, d);
            m.w = e.weights;
            m.w_to = e.weights;
            m.w_layer = m.t_layer = e.w_layer;
            m.w_head = m.t_head = e.w_head;
            m.idx = e.idx;
        }
        moves.push_back(m);
    }
    if (places.clash() || places.lengths_clash(lengths)) return fail(ctx, CB_EINVAL, "two parts of the call write the same memory");
    return move_all(ctx, moves, c.n_layers, strm);
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
        return attend_impl<AttendBatch>(ctx, layer, n, caches, queries, nullptr, causal, window, static_cast<cudaStream_t>(stream));
    });
}

cb_status cb_attend_tree(cb_ctx* ctx, int32_t layer, int32_t n, const cb_packed* caches, const cb_attend_query* queries,
                         const cb_tree* trees, void* stream) {
    return entry(ctx, "cb_attend_tree", [&] {
        if (!trees) return fail(ctx, CB_EINVAL, "trees is NULL");
        return attend_impl<AttendTreeBatch>(ctx, layer, n, caches, queries, trees, 1, 0, static_cast<cudaStream_t>(stream));
    });
}

cb_status cb_weigh(cb_ctx* ctx, int32_t layer, int32_t n, const cb_packed* caches, const cb_weigh_query* queries,
                   const cb_tree* trees, int32_t causal, int64_t window, float decay, void* stream) {
    return entry(ctx, "cb_weigh", [&] {
        return weigh_impl(ctx, layer, n, caches, queries, trees, causal, window, decay, static_cast<cudaStream_t>(stream));
    });
}

cb_status cb_evict(cb_ctx* ctx, int32_t layer, int32_t n_layers, int32_t n, const cb_packed* caches, const cb_packed* into,
                   const cb_eviction* evictions, void* stream) {
    return entry(ctx, "cb_evict", [&] {
        return evict_impl(ctx, layer, n_layers, n, caches, into, evictions, static_cast<cudaStream_t>(stream));
    });
}

cb_status cb_keep(cb_ctx* ctx, int32_t n, const cb_packed* caches, const cb_kept* kept, void* stream) {
    return entry(ctx, "cb_keep", [&] { return keep_impl(ctx, n, caches, kept, static_cast<cudaStream_t>(stream)); });
}

}  // extern "C"
