// What the kernels of cb_attend share: the rows a query tile sees, packed words as numbers, and the
// last step of an output row.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "cb_receiver.cuh"
#include "cb_sm100_attend.cuh"

namespace cbk {

using sm100::ex2;

constexpr uint32_t kTopScaleBits = 0x4600u;   // 2^13 as bf16, the largest scale

constexpr int kUnit = 128;                    // positions of one unit of work
constexpr int kMaxPairs = kMaxBatch * 16;     // most (sequence, row tile) pairs of a launch: 1024 tokens x 4 heads in tiles of 256 rows

// Query rows of partial results a context holds for each SM: two parts of 256 rows.
constexpr int kPartRowsPerSm = 512;

// Rows in the cache.
__device__ __forceinline__ int64_t attend_length(const AttendSpan& s) {
    if (!s.length) return s.T;
    const int64_t l = *s.length;
    return l < 0 ? 0 : l < s.T ? l : s.T;
}

// Positions [lo, hi) that some row of a tile sees; those from all_to_here on and before all_from_here are
// seen by every row of it.
struct Reach {
    int64_t lo, hi, all_to_here, all_from_here;
};
__device__ __forceinline__ Reach attend_reach(const AttendBatch& b, const AttendSpan& s, int64_t L, int tile, int tile_rows) {
    const int first = tile * tile_rows, last = min(first + tile_rows, s.m * b.G) - 1;
    Reach x{0, L, 0, L};
    if (b.causal) {
        const int64_t p0 = L - s.m + first / b.G, p1 = L - s.m + last / b.G;
        x.hi = max((int64_t)0, min(L, p1 + 1));
        x.all_from_here = p0 + 1;
        if (b.window) {
            x.lo = min(x.hi, max((int64_t)0, p0 - b.window + 1)) & ~(int64_t)31;
            x.all_to_here = p1 - b.window + 1;
        }
    }
    return x;
}

// The work is cut into units of 128 positions of one pair (sequence, row tile) and one or more KV heads,
// and every block takes an equal run of them: whatever the lengths are, which the kernel reads itself, no
// block has more than one unit more than another.  A run is made of segments, each of one pair and head;
// only the first and the last may hold a part of their positions, and leave a partial result in slot
// 2 * block (the first) or 2 * block + 1.  A tile that sees no position has one unit, which writes its
// zeros.
//   k_attend_tc: `heads` = all KV heads, ordered by pair, head and position;
//   k_attend_few: `heads` = 1, ordered by pair and position: as many blocks as there are KV heads share a
//     run, a head each, so that rows of neighbouring heads, which a position-major cache keeps side by side,
//     are read at about the same time (blocks ordered by head read 1.8 times the bytes of a paged cache).

// (The number of units is below 2^31.)

// (What runs once a block or segment is rolled up: fetching the code cost more than running it.)

// Sequence of pair p.
__device__ __forceinline__ int attend_seq_of(const AttendBatch& b, int p) {
    if (b.pairs == b.n) return p;         // (a tile each)
    int i = 0;
#pragma unroll 1
    for (int step = kMaxBatch / 2; step; step /= 2)
        if (i + step < b.n && b.span[i + step].pair0 <= p) i += step;
    return i;
}

// Units of pair p.
__device__ __forceinline__ int attend_units_of(const AttendBatch& b, int tile_rows, int p) {
    const AttendSpan& s = b.span[attend_seq_of(b, p)];
    const Reach x = attend_reach(b, s, attend_length(s), p - s.pair0, tile_rows);
    const int u = (int)((x.hi - x.lo + kUnit - 1) / kUnit);
    return u > 0 ? u : 1;
}

// Units of the pairs before each pair, into shared memory: pre[0..pairs].  Whole block.
__device__ __forceinline__ void attend_units(const AttendBatch& b, int tile_rows, int* pre) {
    const bool few = b.pairs <= 32;                    // the first warp alone, out of registers
    if (!few) {
#pragma unroll 1
        for (int p = threadIdx.x; p < b.pairs; p += blockDim.x) pre[p + 1] = attend_units_of(b, tile_rows, p);
        __syncthreads();
    }
    if (threadIdx.x < 32) {
        int before = 0;
#pragma unroll 1
        for (int p0 = 0; p0 < b.pairs; p0 += 32) {
            const int p = p0 + threadIdx.x;
            int u = p >= b.pairs ? 0 : few ? attend_units_of(b, tile_rows, p) : pre[p + 1];
#pragma unroll
            for (int k = 1; k < 32; k *= 2) {
                const int y = __shfl_up_sync(0xFFFFFFFFu, u, k);
                if (threadIdx.x >= k) u += y;
            }
            if (p < b.pairs) pre[p + 1] = before + u;
            before += __shfl_sync(0xFFFFFFFFu, u, 31);
        }
        if (threadIdx.x == 0) pre[0] = 0;
    }
    __syncthreads();
}

// How units are dealt out: the first `more` of the blocks have each + 1, the others each.
struct Runs {
    int units, blocks, each, more;
};
__device__ __forceinline__ Runs attend_runs(int units, int grid) {
    Runs r;
    r.units = units;
    r.blocks = min(grid, units);
    r.each = units / r.blocks;
    r.more = units - r.each * r.blocks;
    return r;
}
// First unit of a block's run, and the block whose run holds unit u.
__device__ __forceinline__ int attend_run(const Runs& r, int block) { return block * r.each + min(block, r.more); }
__device__ __forceinline__ int attend_block(const Runs& r, int u) {
    const int wide = r.more * (r.each + 1);
    return u < wide ? u / (r.each + 1) : r.more + (u - wide) / r.each;
}

// A segment of a run, in shared memory: registers hold what the loops need all the time.
struct Segment {
    int64_t begin;            // its first position
    int64_t at;               // position of the sequence's token 0, from `begin` on
    const uint8_t* code[2];   // K and V from the head on
    const uint16_t* scale[2];
    const int32_t* pages;
    int32_t first, units;     // units of its (pair, head): the first one's number, how many
    int32_t n;                // units of the segment
    int32_t len;              // positions
    int32_t all_to, all_from; // those from all_to on and before all_from are seen by every row of the tile
    int32_t seq, g, row0, rows;   // the tile's first query row, and how many there are
    uint32_t s_pos, s_page, n_pages, shift, mask;
};

// The (pair, head) that holds unit u: its first unit and their number.
struct Item {
    int first, units, seq, tile, g;
};
__device__ __forceinline__ Item attend_item(const AttendBatch& b, const int* pre, int heads, int u) {
    Item x;
    int p = 0;
#pragma unroll 1
    for (int step = kMaxPairs / 2; step; step /= 2)
        if (p + step < b.pairs && pre[p + step] * heads <= u) p += step;
    x.units = pre[p + 1] - pre[p];
    x.g = heads == 1 ? 0 : (u - pre[p] * heads) / x.units;
    x.first = pre[p] * heads + x.g * x.units;
    x.seq = attend_seq_of(b, p);
    x.tile = p - b.span[x.seq].pair0;
    return x;
}

// The segment that begins with unit u of a run that ends at `end` (one thread); its head counts from g0.
__device__ __forceinline__ void attend_segment(const AttendBatch& b, const int* pre, int heads, int g0, int u, int end,
                                               int head_dim, int tile_rows, Segment* x) {
    Item item = attend_item(b, pre, heads, u);
    item.g += g0;
    const AttendSeq& s = b.s[item.seq];
    const AttendSpan& a = b.span[item.seq];
    const int64_t L = attend_length(a);
    const Reach r = attend_reach(b, a, L, item.tile, tile_rows);
    x->first = item.first;
    x->units = item.units;
    x->n = min(end - u, item.units - (u - item.first));
    x->begin = r.lo + (int64_t)(u - item.first) * kUnit;
    x->at = L - a.m - x->begin;
    const int64_t len = min(r.hi - x->begin, (int64_t)x->n * kUnit);
    x->len = (int)len;
    x->all_to = (int)max((int64_t)0, min(r.all_to_here - x->begin, len));
    x->all_from = (int)max((int64_t)0, min(r.all_from_here - x->begin, len));
    x->seq = item.seq;
    x->g = item.g;
    x->row0 = item.tile * tile_rows;
    x->rows = min(tile_rows, a.m * b.G - x->row0);
    const int64_t head = (int64_t)item.g * s.kv.s_head;
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {
        x->code[k] = s.kv.code[k] + head * (head_dim / 2);
        x->scale[k] = s.kv.scale[k] + head * (head_dim / 32);
    }
    x->pages = s.kv.pages;
    x->s_pos = (uint32_t)s.kv.s_pos;
    x->s_page = (uint32_t)s.kv.s_page;
    x->n_pages = (uint32_t)min(s.kv.n_pages, (int64_t)0x7FFFFFFF);
    x->shift = s.kv.shift;
    x->mask = (1u << s.kv.shift) - 1;
}

// The block-table entry of position t of the segment, read ahead of the copies that need it, and the row of
// position t from it (counted from the head's base, by 32-bit products: offsets are below 2^31): -1 where
// there is none, behind the segment's end or for a bad entry.
__device__ __forceinline__ uint32_t segment_page(const Segment& x, int t) {
    return x.pages && t < x.len ? (uint32_t)__ldg(x.pages + (((uint32_t)x.begin + (uint32_t)t) >> x.shift)) : 0u;
}
__device__ __forceinline__ int segment_row(const Segment& x, int t, uint32_t page, uint32_t* err) {
    const uint32_t p = (uint32_t)x.begin + (uint32_t)t;
    if (t >= x.len) return -1;
    if (!x.pages) return (int)(p * x.s_pos);
    if (page >= x.n_pages) {
        atomicOr(err, kErrPageIndex);
        return -1;
    }
    return (int)(page * x.s_page + (p & x.mask) * x.s_pos);
}

// Copies of 16, 8 or 4 bytes into shared memory (small ones without `there` read nothing and write zeros).
__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
template <int N>
__device__ __forceinline__ void copy_small(uint32_t to, const void* from, bool there) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(to), "l"(from), "n"(N), "r"(there ? N : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A scale's bits, or those of 0 where it is none.
__device__ __forceinline__ uint32_t checked_scale(uint32_t s, uint32_t& bad) {
    if (s > kTopScaleBits) {
        bad = 1;
        return 0;
    }
    return s;
}

// Two bf16 scales as a pair of fp16 ones (exact within 2^-20 .. 2^13).
__device__ __forceinline__ uint32_t f16_scales(uint32_t lo, uint32_t hi) {
    const __half2 h = __floats2half2_rn(__uint_as_float(lo << 16), __uint_as_float(hi << 16));
    return reinterpret_cast<const uint32_t&>(h);
}

// Pairs of nibbles (j, j + 4), j = 0..3, of a word as numbers c * s, exactly, by one fma each: setting bits
// makes u = c + 8 the number 128 + 4 u (bf16, the nibble at bit 2), 1024 + 4 u or 1024 + 64 u (fp16, at bits
// 2 and 6: two shifts serve four pairs), and
//   (128 + 4 u) (s / 4) - 40 s = (1024 + 4 u) (s / 4) - 264 s = (1024 + 64 u) (s / 64) - 24 s = c s.
// 40 s has 8 significant bits (a bf16 number), 264 s and 24 s have 11 and 7 (fp16 numbers); with the
// nibble at bit 0 they would have 10 and 13, and the bias a subtraction of its own.
__device__ __forceinline__ void values_bf16(uint32_t word, uint32_t s2, uint32_t (&out)[4]) {
    const __nv_bfloat162 s = reinterpret_cast<const __nv_bfloat162&>(s2);
    const __nv_bfloat162 a = __hmul2(s, __floats2bfloat162_rn(0.25f, 0.25f)), b = __hmul2(s, __floats2bfloat162_rn(-40.f, -40.f));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t x = ((j == 0 ? word << 2 : word >> (4 * j - 2)) & 0x003C003Cu) | 0x43004300u;
        const __nv_bfloat162 p = __hfma2(reinterpret_cast<const __nv_bfloat162&>(x), a, b);
        out[j] = reinterpret_cast<const uint32_t&>(p);
    }
}
// NEAR: every s is within 2^-14 .. 2^7, where s / 64 and 264 s are fp16 numbers.  Otherwise c by one fma
// and its product with s by another instruction.
template <bool NEAR>
__device__ __forceinline__ void values_f16(uint32_t word, uint32_t s2, uint32_t (&out)[4]) {
    const __half2 s = reinterpret_cast<const __half2&>(s2);
#pragma unroll
    for (int k = 0; k < 2; ++k) {           // the nibble at bit 2, at bit 6
        const __half2 u = __float2half2_rn(k ? 0.015625f : 0.25f), w = __float2half2_rn(k ? -24.f : -264.f);
        const __half2 a = NEAR ? __hmul2(s, u) : u, b = NEAR ? __hmul2(s, w) : w;
#pragma unroll
        for (int j = k; j < 4; j += 2) {
            const uint32_t x = ((j < 2 ? word << 2 : word >> 6) & (k ? 0x03C003C0u : 0x003C003Cu)) | 0x64006400u;
            const __half2 c = __hfma2(reinterpret_cast<const __half2&>(x), a, b), p = NEAR ? c : __hmul2(c, s);
            out[j] = reinterpret_cast<const uint32_t&>(p);
        }
    }
}

// One of the four pairs alone, for any scale.
__device__ __forceinline__ uint32_t value_f16(uint32_t word, int j, __half2 s) {
    const bool high = j & 1;
    const uint32_t x = ((j < 2 ? word << 2 : word >> 6) & (high ? 0x03C003C0u : 0x003C003Cu)) | 0x64006400u;
    const __half2 c = __hfma2(reinterpret_cast<const __half2&>(x), __float2half2_rn(high ? 0.015625f : 0.25f),
                              __float2half2_rn(high ? -24.f : -264.f));
    const __half2 p = __hmul2(c, s);
    return reinterpret_cast<const uint32_t&>(p);
}

// Four elements of an output row and the row's log-sum-exp, from sums of weights exp2(z - M).
template <int D>
__device__ __forceinline__ void attend_write(const AttendBatch& b, const AttendSeq& s, int g, int row, int d, float4 y,
                                             float M, float l) {
    const int r = row / b.G, h = g * b.G + row % b.G;
    const float f = l == 0.f ? 0.f : 1.f / l;     // (no row seen: 0; NaN stays NaN)
    const __nv_bfloat162 lo = __floats2bfloat162_rn(y.x * f, y.y * f), hi = __floats2bfloat162_rn(y.z * f, y.w * f);
    *reinterpret_cast<uint2*>(s.out + (int64_t)r * s.o_tok + (int64_t)h * s.o_head + d) =
        make_uint2(reinterpret_cast<const uint32_t&>(lo), reinterpret_cast<const uint32_t&>(hi));
    if (d == 0 && s.lse)
        s.lse[(int64_t)r * b.n_q_heads + h] = l == 0.f ? -INFINITY : (M + log2f(l)) * 0.6931471805599453f;
}

// Adds a part's four elements and its sum, times f.
__device__ __forceinline__ void add_part(float4& y, float& l, const float4& v, float f, float sum) {
    y.x = fmaf(v.x, f, y.x); y.y = fmaf(v.y, f, y.y); y.z = fmaf(v.z, f, y.z); y.w = fmaf(v.w, f, y.w);
    l = fmaf(sum, f, l);
}

// Four elements of a row from n parts, in order, N at a time: parts are slots slot0 + skip, slot0 + step,
// slot0 + 2 step ...
struct Joined {
    float4 y;
    float M, l;
};
template <int D, int N>
__device__ __forceinline__ Joined attend_join_row(const AttendBatch& b, int64_t slot0, int skip, int step, int n, int tile_rows,
                                                  int r, int d) {
    Joined j{make_float4(0.f, 0.f, 0.f, 0.f), -INFINITY, 0.f};
#pragma unroll 1
    for (int k0 = 0; k0 < n; k0 += N) {
        float2 x[N];
        float4 v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int k = k0 + i;
            const int64_t at = (slot0 + (k ? k * step : skip)) * tile_rows + r;
            x[i] = make_float2(-INFINITY, 0.f);
            v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (k < n) {
                x[i] = __ldcg(b.part_ml + at);
                v[i] = __ldcg(reinterpret_cast<const float4*>(b.part + at * D + d));
            }
        }
        float top = j.M;
#pragma unroll
        for (int i = 0; i < N; ++i) top = fmaxf(top, x[i].x);
        const float f = j.M == -INFINITY ? 0.f : exp2f(j.M - top);
        j.y.x *= f; j.y.y *= f; j.y.z *= f; j.y.w *= f;
        j.l *= f;
        j.M = top;
#pragma unroll
        for (int i = 0; i < N; ++i)
            add_part(j.y, j.l, v[i], x[i].x == -INFINITY ? 0.f : exp2f(x[i].x - j.M), x[i].y);
    }
    return j;
}

// A window that no cache and its tokens reach across (fewer than 2^31 rows and 1024 tokens): larger ones are
// taken for this one, so that neither sums of rows, tokens and window nor their differences leave 64 bits.
constexpr int64_t kFarWindow = (int64_t)1 << 32;

// Host side, shared by the launchers: row tiles of every sequence, and the most units there can be.
int64_t attend_pairs(AttendBatch& b, int tile_rows);
cudaError_t launch_attend_tc(AttendBatch& b, int head_dim, cudaStream_t st, int num_sms);

}  // namespace cbk
