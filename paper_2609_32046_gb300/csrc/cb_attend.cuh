// What the kernels of cb_attend share: the rows a query tile sees, packed words as numbers, and the
// last step of an output row.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "cb_internal.cuh"
#include "cb_sm100.cuh"

namespace cbk {

using sm100::ex2;

constexpr uint32_t kTopScaleBits = 0x4600u;   // 2^13 as bf16, the largest scale

// Query rows of partial results a context holds for each SM: 16 parts of 16 rows, or two of 128.
constexpr int kPartRowsPerSm = 256;

// Rows in the cache.
__device__ __forceinline__ int64_t attend_length(const AttendSeq& s) {
    if (!s.length) return s.T;
    const int64_t l = *s.length;
    return l < 0 ? 0 : l < s.T ? l : s.T;
}

// Positions [begin, end) of one part that some row of a tile sees; those from all_to_here on and before
// all_from_here are seen by every row of the tile.
struct Span {
    int64_t begin, end, all_to_here, all_from_here;
};
__device__ __forceinline__ Span attend_span(const AttendBatch& b, const AttendSeq& s, int64_t L, int first_row,
                                            int last_row, int part, int granule) {
    int64_t lo = 0, hi = L;
    Span x;
    x.all_to_here = 0;
    x.all_from_here = L;
    if (b.causal) {
        const int64_t p0 = L - s.m + first_row / b.G, p1 = L - s.m + last_row / b.G;
        hi = min(L, p1 + 1);
        x.all_from_here = p0 + 1;
        if (b.window) {
            lo = max((int64_t)0, p0 - b.window + 1) & ~(int64_t)31;
            x.all_to_here = p1 - b.window + 1;
        }
    }
    const int64_t span = hi > lo ? hi - lo : 0;
    int64_t each = (span + s.splits - 1) / s.splits;
    each = (each + granule - 1) / granule * granule;
    x.begin = lo + part * each;
    x.end = min(hi, x.begin + each);
    if (x.end < x.all_from_here) x.all_from_here = x.end;
    return x;
}

// The most positions a tile of the sequence may read (host: from T, the bound of the length).
inline int64_t attend_reach(const AttendBatch& b, const AttendSeq& s) {
    const int64_t w = b.causal && b.window ? b.window + s.m : s.T;
    return s.T < w ? s.T : w;
}

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
// makes u = c + 8 the number 128 + 4 u (bf16, the nibble at bit 2) or 1024 + 16 u (fp16, at bit 4), and
//   (128 + 4 u) (s / 4) - 40 s = (1024 + 16 u) (s / 16) - 72 s = c s.
// 40 s and 72 s have 8 and 9 significant bits: bf16 and fp16 numbers.  With the nibble at bit 0 they would
// have 10 (136 s) and 13 (1032 s), and the bias a subtraction of its own.
__device__ __forceinline__ uint32_t nibbles_at(uint32_t word, int shift, uint32_t mask, uint32_t bits) {
    return ((shift >= 0 ? word << (shift >= 0 ? shift : 0) : word >> (shift < 0 ? -shift : 0)) & mask) | bits;
}
__device__ __forceinline__ void values_bf16(uint32_t word, uint32_t s2, uint32_t (&out)[4]) {
    const __nv_bfloat162 s = reinterpret_cast<const __nv_bfloat162&>(s2);
    const __nv_bfloat162 a = __hmul2(s, __floats2bfloat162_rn(0.25f, 0.25f)), b = __hmul2(s, __floats2bfloat162_rn(-40.f, -40.f));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t x = nibbles_at(word, 2 - 4 * j, 0x003C003Cu, 0x43004300u);
        const __nv_bfloat162 p = __hfma2(reinterpret_cast<const __nv_bfloat162&>(x), a, b);
        out[j] = reinterpret_cast<const uint32_t&>(p);
    }
}
// NEAR: every s is 0 or within 2^-16 .. 2^9, where s / 16 and 72 s are fp16 numbers.  Otherwise c by one fma
// and its product with s by another instruction.
template <bool NEAR>
__device__ __forceinline__ void values_f16(uint32_t word, uint32_t s2, uint32_t (&out)[4]) {
    const __half2 s = reinterpret_cast<const __half2&>(s2);
    const __half2 u = __floats2half2_rn(0.0625f, 0.0625f), w = __floats2half2_rn(-72.f, -72.f);
    const __half2 a = NEAR ? __hmul2(s, u) : u, b = NEAR ? __hmul2(s, w) : w;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t x = nibbles_at(word, 4 - 4 * j, 0x00F000F0u, 0x64006400u);
        const __half2 c = __hfma2(reinterpret_cast<const __half2&>(x), a, b), p = NEAR ? c : __hmul2(c, s);
        out[j] = reinterpret_cast<const uint32_t&>(p);
    }
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

// Host side, shared by the launchers.
bool attend_plan(AttendBatch& b, int tile_rows, int64_t blocks, int64_t least, int num_sms);
cudaError_t attend_join(const AttendBatch& b, int head_dim, int tile_rows, cudaStream_t st);
cudaError_t launch_attend_tc(AttendBatch& b, int head_dim, cudaStream_t st, int num_sms);

}  // namespace cbk
