// Rotary embedding of query and key vectors: pair k of a head turns by position * f_k, over the
// whole head or its first `dims` elements, pairs as halves or interleaved, frequencies stretched for
// long contexts (the three scalings of cb_rope), forwards or transposed.
//
// Angles: F_k = f_k / (2 pi) * 2^64 (host, long double), position * F_k modulo 2^64 is the angle in
// turns, exact to 2^-64 of a turn a position; its top 32 bits give the angle in [-pi, pi), whose sine
// and cosine come from the hardware approximations (absolute error near 2^-21, far below the bf16
// rounding of the result).
#include <cmath>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "cb_internal.cuh"

namespace cbk {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// A unit is 16 elements of a row, two 16-byte pieces: 8 pairs (8u .. 8u + 7) of the rotary part, whose
// halves are dims / 2 apart (STYLE 0) or which lie side by side (STYLE 1), or 16 elements behind it.
// Block: one token of one set, D / 16 units of 256 / (D / 16) rows (layer, head) at a time; a thread
// keeps its unit's eight sines and cosines for all rows it walks, so that the special-function unit
// works once a token and not once a head.
// Grid: x = token (and slice of the rows, innermost), y = set.
template <int D, int STYLE>
__global__ void __launch_bounds__(kThreads) k_rotary(const __grid_constant__ RotaryBatch b, int slices) {
    constexpr int U = D / 16, LANES = kThreads / U;
    const RotarySet& s = b.s[blockIdx.y];
    const int64_t r = blockIdx.x / (unsigned)slices;
    if (r >= s.n_tokens) return;
    const int u = threadIdx.x % U;
    const bool turn = u * 16 < b.dims;
    if (!turn && s.x == s.y) return;                       // in place: nothing to do behind the rotary part
    const int e0 = turn && STYLE == 0 ? u * 8 : u * 16;    // the unit's two pieces
    const int e1 = turn && STYLE == 0 ? u * 8 + b.dims / 2 : u * 16 + 8;
    float c[8], n[8];
    if (turn) {
        const int64_t pos = s.pos ? (int64_t)__ldg(s.pos + r) : s.pos0 + r;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint64_t turns = (uint64_t)pos * b.turns[u * 8 + k];
            const float a = (float)(int32_t)(uint32_t)(turns >> 32) * 1.4629180792671596e-09f;   // 2 pi / 2^32
            c[k] = __cosf(a) * b.gain;
            n[k] = __sinf(a) * b.sine_gain;
        }
    }
    const int rows = s.n_layers * s.n_heads;
    const int step = LANES * slices;
    for (int q0 = (int)(blockIdx.x % (unsigned)slices) * LANES + threadIdx.x / U; q0 < rows; q0 += step * kUnroll) {
        uint4 va[kUnroll], vb[kUnroll];
        uint16_t* out[kUnroll];
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            const int q = q0 + i * step;
            if (q >= rows) break;
            const int l = q / s.n_heads, h = q - l * s.n_heads;
            const uint16_t* x = s.x + l * s.s_layer + r * s.s_tok + h * s.s_head;
            out[i] = s.y + l * s.o_layer + r * s.o_tok + h * s.o_head;
            va[i] = *reinterpret_cast<const uint4*>(x + e0);
            vb[i] = *reinterpret_cast<const uint4*>(x + e1);
        }
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            if (q0 + i * step >= rows) break;
            if (turn) {
                uint32_t a[4] = {va[i].x, va[i].y, va[i].z, va[i].w}, w[4] = {vb[i].x, vb[i].y, vb[i].z, vb[i].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (STYLE == 0) {        // a: first elements of pairs 2j, 2j + 1; w: their second ones
                        const float a0 = lo_f(a[j]), a1 = hi_f(a[j]), w0 = lo_f(w[j]), w1 = hi_f(w[j]);
                        a[j] = pack_bf16(a0 * c[2 * j] - w0 * n[2 * j], a1 * c[2 * j + 1] - w1 * n[2 * j + 1]);
                        w[j] = pack_bf16(w0 * c[2 * j] + a0 * n[2 * j], w1 * c[2 * j + 1] + a1 * n[2 * j + 1]);
                    } else {                 // a: pair j; w: pair 4 + j
                        const float a0 = lo_f(a[j]), a1 = hi_f(a[j]), w0 = lo_f(w[j]), w1 = hi_f(w[j]);
                        a[j] = pack_bf16(a0 * c[j] - a1 * n[j], a1 * c[j] + a0 * n[j]);
                        w[j] = pack_bf16(w0 * c[4 + j] - w1 * n[4 + j], w1 * c[4 + j] + w0 * n[4 + j]);
                    }
                }
                va[i] = make_uint4(a[0], a[1], a[2], a[3]);
                vb[i] = make_uint4(w[0], w[1], w[2], w[3]);
            }
            *reinterpret_cast<uint4*>(out[i] + e0) = va[i];
            *reinterpret_cast<uint4*>(out[i] + e1) = vb[i];
        }
    }
}

}  // namespace

cudaError_t launch_rotary(const RotaryBatch& b, int head_dim, int style, cudaStream_t st, int num_sms) {
    int64_t tokens = 0, rows = 0;
    for (int i = 0; i < b.n; ++i) {
        const int64_t q = (int64_t)b.s[i].n_layers * b.s[i].n_heads;
        tokens = b.s[i].n_tokens > tokens ? b.s[i].n_tokens : tokens;
        rows = q > rows ? q : rows;
    }
    if (tokens == 0 || rows == 0) return cudaSuccess;
    // enough blocks for eight an SM where there are few tokens, at least one pass of rows a block
    const int64_t lanes = kThreads / (head_dim / 16), most = (rows + lanes - 1) / lanes;
    int64_t slices = ((int64_t)num_sms * 8 + tokens * b.n - 1) / (tokens * b.n);
    slices = slices < most ? slices : most;
    const dim3 grid((unsigned)(tokens * slices), (unsigned)b.n);
    if (head_dim == 128) {
        if (style == 0) k_rotary<128, 0><<<grid, kThreads, 0, st>>>(b, (int)slices);
        else k_rotary<128, 1><<<grid, kThreads, 0, st>>>(b, (int)slices);
    } else {
        if (style == 0) k_rotary<64, 0><<<grid, kThreads, 0, st>>>(b, (int)slices);
        else k_rotary<64, 1><<<grid, kThreads, 0, st>>>(b, (int)slices);
    }
    return cudaGetLastError();
}

}  // namespace cbk
