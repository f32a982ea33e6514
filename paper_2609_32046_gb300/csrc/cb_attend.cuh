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

// Pairs of nibbles (j, j + 4), j = 0..3, of a word as numbers c * s: 128 + u (bf16) or 1024 + u (fp16)
// by setting bits, less the bias is c, exactly; so is the product.
__device__ __forceinline__ void values_bf16(uint32_t word, uint32_t s2, uint32_t (&out)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t x = ((word >> (4 * j)) & 0x000F000Fu) | 0x43004300u;
        const __nv_bfloat162 c = __hsub2(reinterpret_cast<const __nv_bfloat162&>(x), __floats2bfloat162_rn(136.f, 136.f));
        const __nv_bfloat162 p = __hmul2(c, reinterpret_cast<const __nv_bfloat162&>(s2));
        out[j] = reinterpret_cast<const uint32_t&>(p);
    }
}
__device__ __forceinline__ void values_f16(uint32_t word, uint32_t s2, uint32_t (&out)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t x = ((word >> (4 * j)) & 0x000F000Fu) | 0x64006400u;
        const __half2 c = __hsub2(reinterpret_cast<const __half2&>(x), __floats2half2_rn(1032.f, 1032.f));
        const __half2 p = __hmul2(c, reinterpret_cast<const __half2&>(s2));
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
