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

#include "cb_receiver.cuh"

namespace cbk {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 3;          // vectors a thread has in flight
constexpr int kMaxTokens = 8;       // tokens a block takes at a time

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Tokens a block takes at a time: enough vectors (layer, head) for kUnroll a thread.
__host__ __device__ __forceinline__ int tokens_at_once(int rows, int lanes) {
    const int n = (kUnroll * lanes + rows - 1) / rows;
    return n < 1 ? 1 : n < kMaxTokens ? n : kMaxTokens;
}

// Where two pairs' numbers stand: the same place of eight units in eight different banks.
__device__ __forceinline__ int place(int q) { return q ^ ((q >> 3) & 3); }

// A unit is 16 elements of a vector, two 16-byte pieces: 8 pairs (8u .. 8u + 7) of the rotary part, whose
// halves are dims / 2 apart (STYLE 0) or which lie side by side (STYLE 1), or 16 elements behind it.
// A block takes up to eight tokens of a set at a time: their sines and cosines go to shared memory, one a
// thread, and D / 16 units of 256 / (D / 16) vectors in turn read them there.  (With every thread working out
// the eight of its unit, 24 vectors a token left the special-function unit more to do than memory: 6001
// tokens x 8 layers x 24 heads, d = 64, 91 us.)
// Bound by HBM: those 295 MB now take 48 us, 6.1 TB/s; 16384 tokens x 4 layers x 40 heads of 128, 1.3 GB, 195 us, 6.9 TB/s;
// the 47 MB of a short question 10.7 us, 4.4 TB/s, of which starting and ending a kernel of three waves take a part.
// Three vectors a thread and four blocks an SM: two and five take 10.3, 51 and 194 us, two and six 11.4, 54 and 212,
// four and three 12.1, 51 and 197.
// Grid: x = token group (and slice of its vectors, innermost), y = set.
template <int D, int STYLE>
__global__ void __launch_bounds__(kThreads, 4) k_rotary(const __grid_constant__ RotaryBatch b, int slices) {
    constexpr int U = D / 16, LANES = kThreads / U;
    __shared__ float4 turn_of[2][kMaxTokens][D / 4];     // cosine, sine of two pairs, at place()
    const RotarySet& s = b.s[blockIdx.y];
    const int u = threadIdx.x % U;
    const bool turn = u * 16 < b.dims;
    const int e0 = turn && STYLE == 0 ? u * 8 : u * 16;    // the unit's two pieces
    const int e1 = turn && STYLE == 0 ? u * 8 + b.dims / 2 : u * 16 + 8;
    const bool idle = !turn && s.x == s.y;                 // in place: nothing to do behind the rotary part
    const int H = s.n_heads, NL = s.n_layers, rows = NL * H, many = tokens_at_once(rows, LANES);
    const int pairs = b.dims / 2, step = LANES * slices;
    const int dt = step / rows, dl = step % rows / H, dh = step % rows % H;      // a step's tokens, layers, heads
    int buffer = 0;
    for (int64_t t0 = (int64_t)(blockIdx.x / (unsigned)slices) * many; t0 < s.n_tokens;
         t0 += (int64_t)(gridDim.x / (unsigned)slices) * many, buffer ^= 1) {
        const int n = (int)min((int64_t)many, s.n_tokens - t0);
        const int first = (int)(blockIdx.x % (unsigned)slices) * LANES + threadIdx.x / U;
        int t = idle ? n : first / rows, l = first % rows / H, h = first % rows % H;
        uint4 va[kUnroll], vb[kUnroll];
        uint16_t* out[kUnroll];
        int at[kUnroll];
        auto load = [&]() {
#pragma unroll
            for (int i = 0; i < kUnroll; ++i) {
                at[i] = -1;
                if (t < n) {
                    const int64_t r = t0 + t;
                    const uint16_t* x = s.x + l * s.s_layer + r * s.s_tok + h * s.s_head;
                    out[i] = s.y + l * s.o_layer + r * s.o_tok + h * s.o_head;
                    va[i] = *reinterpret_cast<const uint4*>(x + e0);
                    vb[i] = *reinterpret_cast<const uint4*>(x + e1);
                    at[i] = t;
                }
                h += dh;
                l += dl;
                t += dt;
                if (h >= H) { h -= H; ++l; }
                if (l >= NL) { l -= NL; ++t; }
            }
        };
        load();               // (the first vectors are on their way while the sines are worked out)
        for (int i = threadIdx.x; i < n * pairs; i += kThreads) {
            const int t = i / pairs, k = i - t * pairs;
            const int64_t pos = s.pos ? (int64_t)__ldg(s.pos + t0 + t) : s.pos0 + t0 + t;
            const uint64_t turns = (uint64_t)pos * b.turns[k];
            const float a = (float)(int32_t)(uint32_t)(turns >> 32) * 1.4629180792671596e-09f;   // 2 pi / 2^32
            reinterpret_cast<float2*>(&turn_of[buffer][t][place(k / 2)])[k % 2] = make_float2(__cosf(a) * b.gain, __sinf(a) * b.sine_gain);
        }
        __syncthreads();      // (a buffer is written again two turns later, behind the next turn's barrier)
        while (at[0] >= 0) {
#pragma unroll
            for (int i = 0; i < kUnroll; ++i) {
                if (at[i] < 0) continue;
                if (turn) {
                    float4 f[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) f[j] = turn_of[buffer][at[i]][place(4 * u + j)];
                    uint32_t a[4] = {va[i].x, va[i].y, va[i].z, va[i].w}, w[4] = {vb[i].x, vb[i].y, vb[i].z, vb[i].w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (STYLE == 0) {        // a: first elements of pairs 2j, 2j + 1; w: their second ones
                            const float4 c = f[j];
                            const float a0 = lo_f(a[j]), a1 = hi_f(a[j]), w0 = lo_f(w[j]), w1 = hi_f(w[j]);
                            a[j] = pack_bf16(a0 * c.x - w0 * c.y, a1 * c.z - w1 * c.w);
                            w[j] = pack_bf16(w0 * c.x + a0 * c.y, w1 * c.z + a1 * c.w);
                        } else {                 // a: pairs 0..3 of the unit, w: 4..7; word j is one pair
                            const float4 c = f[j / 2], g = f[2 + j / 2];
                            const float ca = j & 1 ? c.z : c.x, na = j & 1 ? c.w : c.y, cw = j & 1 ? g.z : g.x, nw = j & 1 ? g.w : g.y;
                            const float a0 = lo_f(a[j]), a1 = hi_f(a[j]), w0 = lo_f(w[j]), w1 = hi_f(w[j]);
                            a[j] = pack_bf16(a0 * ca - a1 * na, a1 * ca + a0 * na);
                            w[j] = pack_bf16(w0 * cw - w1 * nw, w1 * cw + w0 * nw);
                        }
                    }
                    va[i] = make_uint4(a[0], a[1], a[2], a[3]);
                    vb[i] = make_uint4(w[0], w[1], w[2], w[3]);
                }
                __stcs(reinterpret_cast<uint4*>(out[i] + e0), va[i]);
                __stcs(reinterpret_cast<uint4*>(out[i] + e1), vb[i]);
            }
            load();
        }
    }
}

}  // namespace

cudaError_t launch_rotary(const RotaryBatch& b, int head_dim, int style, cudaStream_t st, int num_sms) {
    const int lanes = kThreads / (head_dim / 16);
    int64_t groups = 0, most = 1;
    for (int i = 0; i < b.n; ++i) {
        const int rows = b.s[i].n_layers * b.s[i].n_heads, many = tokens_at_once(rows, lanes);
        const int64_t g = (b.s[i].n_tokens + many - 1) / many, k = ((int64_t)rows * many + lanes - 1) / lanes;
        groups = g > groups ? g : groups;
        most = k > most ? k : most;
    }
    // slices where there are few groups, so that eight blocks an SM have work, each a pass of vectors at least
    const int64_t full = (int64_t)num_sms * 8;
    int64_t slices = (full + groups * b.n - 1) / (groups * b.n);
    slices = slices < most ? slices : most;
    const int64_t cap = full * 4 / slices > 1 ? full * 4 / slices : 1;
    const dim3 grid((unsigned)((groups < cap ? groups : cap) * slices), (unsigned)b.n);
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
