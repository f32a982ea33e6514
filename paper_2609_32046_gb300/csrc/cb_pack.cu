// K/V rows held in 4 bits: packing selected rows into a message or cache (k_pack) and restoring
// packed rows as bf16 (k_unpack).
//
// A group of 32 elements takes the scale s = the smallest number of 5 significant bits >= max|x| / 7
// (within 2^-20 .. 2^13) and the codes c = x / s rounded to whole numbers, halves away from zero.
// c has 3 bits, so c * s has 8: a bf16 number exactly, and an fp16 number in that range of s.
//
// Both are exact in 32-bit arithmetic.  max|x| and 7 s have 8 significant bits, so the quotient
// max|x| / 7 is a number of 5 bits or at least 2^-8 of itself away from one: the product with 1 / 7, both
// rounded down and off by less than 2^-21, is rounded up to the same number.  x / s is a whole number
// and a half, or 2^-12 away from one: the product with a number between 1 / s and (1 + 2^-19) / s lies on
// the right side, and where x / s is a whole number and a half it is not below.  (The reciprocal
// approximation's error is below 2^-22: times 1 + 2^-21 it is such a number.)
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "cb_attend.cuh"
#include "cb_receiver.cuh"

namespace cbk {
namespace {

constexpr int kThreads = 256;
constexpr int kRows = 4;                 // rows a thread has in flight
constexpr float kSeventh = 0.142857134342193603515625f;   // the fp32 number below 1 / 7
constexpr uint32_t kLargest = 0x4760u;   // 7 * 2^13 as bf16

__device__ __forceinline__ uint4 ld_stream(const uint4* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}

__device__ __forceinline__ void st_stream(uint4* p, uint4 v) {
    asm volatile("st.global.cs.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
                 : "memory");
}

// Largest magnitude of eight bf16 values, as bits: their order is that of the numbers, with infinity
// and NaN above all of them.
__device__ __forceinline__ uint32_t top_bits(const uint32_t (&w)[4]) {
    uint32_t a = __vmaxu2(__vmaxu2(w[0] & 0x7FFF7FFFu, w[1] & 0x7FFF7FFFu),
                          __vmaxu2(w[2] & 0x7FFF7FFFu, w[3] & 0x7FFF7FFFu));
    return max(a & 0xFFFFu, a >> 16);
}

// NaN becomes 0, what lies above the largest value that can be held becomes that value.
__device__ __forceinline__ uint32_t held_range(uint32_t w) {
    uint32_t r = 0;
#pragma unroll
    for (int h = 0; h < 32; h += 16) {
        const uint32_t x = (w >> h) & 0xFFFFu, a = x & 0x7FFFu;
        r |= (a > 0x7F80u ? 0u : a > kLargest ? (x & 0x8000u) | kLargest : x) << h;
    }
    return r;
}

// Codes of eight elements as the word a cache holds: nibble i / 2 + 4 (i % 2) is c + 8 of element i.
// |x| / s + 1/2 is added to 2^22, where a float's last bit is worth 1/2, rounding down: bits 1..3 are the
// whole number.  Signs are gathered one a nibble (n), and 8 - c = (7 - c) + 1 = (c ^ 7) + 1.
__device__ __forceinline__ uint32_t code_word(const uint32_t (&w)[4], float r) {
    uint32_t m = 0, n = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t b0 = __float_as_uint(__fmaf_rz(fabsf(__uint_as_float(w[j] << 16)), r, 4194304.5f));
        const uint32_t b1 = __float_as_uint(__fmaf_rz(fabsf(__uint_as_float(w[j] & 0xFFFF0000u)), r, 4194304.5f));
        const uint32_t p = __byte_perm(b0, b1, 0x5410);
        m |= (j == 0 ? p >> 1 : p << (4 * j - 1)) & (0x00070007u << (4 * j));
        n |= (w[j] >> (15 - 4 * j)) & (0x00010001u << (4 * j));
    }
    return (m ^ (n * 7u)) + (0x88888888u - n * 7u);
}

// Rows of a block's tile.  One thread a row looks up the index, the block tables and the bounds; the 8 or 16 threads
// that move it read the result.
constexpr uint32_t kNone = 0xFFFFFFFFu;

// Where row j of a sender comes from (elements from the segment's base on) and goes to (its row in the cache, which
// are below 2^31; kNone: it does not).
struct __align__(16) PackRow {
    int64_t from;
    uint32_t to;
};
__device__ __forceinline__ PackRow pack_row(const PackBatch& bt, const PackSender& sd, int64_t j) {
    PackRow r{0, kNone};
    if (j >= sd.count) return r;
    const int64_t t = sd.idx ? (int64_t)__ldg(sd.idx + j) : j;
    const int64_t at = sd.rows ? (int64_t)__ldg(sd.rows + j) : sd.dst_off + j;
    if (t < 0 || t >= sd.T) {
        atomicOr(bt.err, kErrCompactIndex);
        return r;
    }
    if (at < 0 || at >= sd.dst_T) {
        atomicOr(bt.err, kErrPackRow);
        return r;
    }
    const int64_t from = row_offset(sd.pm, sd.ks_p, t), to = packed_row(sd.held, at);
    if (from < 0 || to < 0) {
        atomicOr(bt.err, kErrPageIndex);
        return r;
    }
    r.from = from;
    r.to = (uint32_t)to;
    return r;
}

// The row of the cache that row j of the output comes from, and j; kNone: zeros, and nothing to restore.
__device__ __forceinline__ uint2 unpack_row(const PackBatch& bt, const PackSender& sd, int64_t j) {
    if (j >= sd.count) return make_uint2(kNone, kNone);
    const int64_t t = sd.idx ? (int64_t)__ldg(sd.idx + j) : j;
    if (t < 0 || t >= sd.T) {
        atomicOr(bt.err, kErrCompactIndex);
        return make_uint2(kNone, kNone);
    }
    const int64_t from = packed_row(sd.held, t);
    if (from < 0) atomicOr(bt.err, kErrPageIndex);
    return make_uint2(from < 0 ? kNone : (uint32_t)from, (uint32_t)j);
}

// Grid: x = (K or V, layer, head) segment, y = sender, z = slice of the segment's rows.
// A thread takes 8 elements (16 bytes) of four rows of a tile; the four threads of a group each work out the
// scale of one of the four rows and hand it round, two rows' largest values to a word.
// Bound by instructions and by its bytes (2 read and 9/16 written an element) alike: 2048 of 8192 positions of 36 layers x
// 8 heads of 128 take 72 us, 5.3 TB/s; with every thread looking up its own rows and two exchanges a row it was 116.
// Five blocks an SM: four take 75 us, six 79.
template <int D>
__global__ void __launch_bounds__(kThreads, 5) k_pack(const __grid_constant__ PackBatch bt) {
    constexpr int CH = D / 8;              // threads a row
    constexpr int ROWS = kThreads / CH, TILE = ROWS * kRows;
    __shared__ PackRow where[2][TILE];
    const PackSender& sd = bt.s[blockIdx.y];
    const int seg = blockIdx.x;
    const int g = seg % bt.n_kv_heads;
    const int l = (seg / bt.n_kv_heads) % bt.n_layers;
    const int kv = seg / (bt.n_kv_heads * bt.n_layers);
    const int ch = threadIdx.x % CH, mine = threadIdx.x & 3;
    const uint16_t* src = sd.src[kv] + (int64_t)l * sd.ks_l + (int64_t)g * sd.ks_h + ch * 8;
    const int64_t base = (int64_t)(bt.layer + l) * sd.held.s_layer + (int64_t)g * sd.held.s_head;
    uint8_t* code = sd.held.code[kv] + base * (D / 2) + ch * 4;
    uint16_t* scale = sd.held.scale[kv] + base * (D / 32) + ch / 4;
    int buffer = 0;
    int64_t jb = (int64_t)blockIdx.z * TILE;
    if (threadIdx.x < TILE) where[0][threadIdx.x] = pack_row(bt, sd, jb + threadIdx.x);
    for (; jb < sd.count; jb += (int64_t)gridDim.z * TILE, buffer ^= 1) {
        __syncthreads();
        uint32_t w[kRows][4];
        uint32_t to[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const PackRow r = where[buffer][u * ROWS + threadIdx.x / CH];
            to[u] = r.to;
            w[u][0] = w[u][1] = w[u][2] = w[u][3] = 0;
            if (r.to == kNone) continue;
            const uint4 v = ld_stream(reinterpret_cast<const uint4*>(src + r.from));
            w[u][0] = v.x; w[u][1] = v.y; w[u][2] = v.z; w[u][3] = v.w;
        }
        // the next tile's rows while these are on their way
        if (threadIdx.x < TILE)
            where[buffer ^ 1][threadIdx.x] = pack_row(bt, sd, jb + (int64_t)gridDim.z * TILE + threadIdx.x);
        uint32_t a01 = top_bits(w[0]) | (top_bits(w[1]) << 16), a23 = top_bits(w[2]) | (top_bits(w[3]) << 16);
        const uint32_t both = __vmaxu2(a01, a23);
        if (__any_sync(0xFFFFFFFFu, max(both & 0xFFFFu, both >> 16) > kLargest)) {
            bool bad = false;
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                bad |= top_bits(w[u]) > kLargest;
#pragma unroll
                for (int k = 0; k < 4; ++k) w[u][k] = held_range(w[u][k]);
            }
            if (bad) atomicOr(bt.err, kErrPackValue);
            a01 = top_bits(w[0]) | (top_bits(w[1]) << 16);
            a23 = top_bits(w[2]) | (top_bits(w[3]) << 16);
        }
#pragma unroll
        for (int x = 1; x <= 2; x *= 2) {
            a01 = __vmaxu2(a01, __shfl_xor_sync(0xFFFFFFFFu, a01, x));
            a23 = __vmaxu2(a23, __shfl_xor_sync(0xFFFFFFFFu, a23, x));
        }
        const uint32_t a = mine & 2 ? a23 : a01;
        const float top = __uint_as_float(mine & 1 ? a & 0xFFFF0000u : a << 16);
        float s = __uint_as_float((__float_as_uint(__fmul_rz(top, kSeventh)) + 0x7FFFFu) & ~0x7FFFFu);
        s = fminf(fmaxf(s, 9.5367431640625e-07f), 8192.f);
        float inv;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
        inv = fmaf(inv, 4.76837158203125e-07f, inv);
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const float r = __shfl_sync(0xFFFFFFFFu, inv, u, 4), su = __shfl_sync(0xFFFFFFFFu, s, u, 4);
            if (to[u] == kNone) continue;
            *reinterpret_cast<uint32_t*>(code + (uint64_t)to[u] * (D / 2)) = code_word(w[u], r);
            if (mine == 0) scale[(uint64_t)to[u] * (D / 32)] = (uint16_t)(__float_as_uint(su) >> 16);
        }
    }
}

// The same grid and tiles; a thread restores 8 elements of each of four rows: the same
// 2048 positions back in 63 us, 6.1 TB/s (1.8 GB through pages and back: six blocks an SM 144 us, five 151).
template <int D>
__global__ void __launch_bounds__(kThreads, 6) k_unpack(const __grid_constant__ PackBatch bt) {
    constexpr int CH = D / 8;
    constexpr int ROWS = kThreads / CH, TILE = ROWS * kRows;
    __shared__ uint2 where[2][TILE];
    const PackSender& sd = bt.s[blockIdx.y];
    const int seg = blockIdx.x;
    const int g = seg % bt.n_kv_heads;
    const int l = (seg / bt.n_kv_heads) % bt.n_layers;
    const int kv = seg / (bt.n_kv_heads * bt.n_layers);
    const int ch = threadIdx.x % CH;
    const int64_t base = (int64_t)l * sd.held.s_layer + (int64_t)g * sd.held.s_head;
    const uint8_t* code = sd.held.code[kv] + base * (D / 2) + ch * 4;
    const uint16_t* scale = sd.held.scale[kv] + base * (D / 32) + ch / 4;
    uint16_t* dst = bt.out[kv] + (int64_t)l * bt.o_layer + (int64_t)g * bt.o_head + sd.dst_off * D + ch * 8;
    int buffer = 0;
    int64_t jb = (int64_t)blockIdx.z * TILE;
    if (threadIdx.x < TILE) where[0][threadIdx.x] = unpack_row(bt, sd, jb + threadIdx.x);
    for (; jb < sd.count; jb += (int64_t)gridDim.z * TILE, buffer ^= 1) {
        __syncthreads();
        uint32_t w[kRows], s[kRows];
        uint32_t to[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const uint2 r = where[buffer][u * ROWS + threadIdx.x / CH];
            to[u] = r.y;
            w[u] = 0x88888888u;
            s[u] = 0;
            if (r.x == kNone) continue;
            w[u] = __ldg(reinterpret_cast<const uint32_t*>(code + (uint64_t)r.x * (D / 2)));
            s[u] = __ldg(scale + (uint64_t)r.x * (D / 32));
        }
        if (threadIdx.x < TILE)
            where[buffer ^ 1][threadIdx.x] = unpack_row(bt, sd, jb + (int64_t)gridDim.z * TILE + threadIdx.x);
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            if (to[u] == kNone) continue;
            if (s[u] > kTopScaleBits) {
                atomicOr(bt.err, kErrPackScale);
                s[u] = 0;
            }
            uint32_t v[4];
            values_bf16(w[u], s[u] * 0x10001u, v);
            st_stream(reinterpret_cast<uint4*>(dst + (uint64_t)to[u] * D), make_uint4(v[0], v[1], v[2], v[3]));
        }
    }
}

// Slices of the rows: about 24 blocks an SM over the batch, at least one tile each.
dim3 grid_of(const PackBatch& b, int head_dim, int num_sms) {
    int64_t most = 0;
    for (int i = 0; i < b.n; ++i) most = b.s[i].count > most ? b.s[i].count : most;
    const int segs = 2 * b.n_layers * b.n_kv_heads;
    const int64_t pass = (int64_t)(kThreads / (head_dim / 8)) * kRows;
    int64_t slices = ((int64_t)num_sms * 24) / ((int64_t)segs * b.n);
    const int64_t need = (most + pass - 1) / pass;
    if (slices > need) slices = need;
    if (slices < 1) slices = 1;
    if (slices > 65535) slices = 65535;
    return dim3((unsigned)segs, (unsigned)b.n, (unsigned)(most ? slices : 0));
}

}  // namespace

cudaError_t launch_pack(const PackBatch& b, int head_dim, cudaStream_t st, int num_sms) {
    const dim3 grid = grid_of(b, head_dim, num_sms);
    if (grid.z == 0) return cudaSuccess;
    if (head_dim == 128) k_pack<128><<<grid, kThreads, 0, st>>>(b);
    else k_pack<64><<<grid, kThreads, 0, st>>>(b);
    return cudaGetLastError();
}

cudaError_t launch_unpack(const PackBatch& b, int head_dim, cudaStream_t st, int num_sms) {
    const dim3 grid = grid_of(b, head_dim, num_sms);
    if (grid.z == 0) return cudaSuccess;
    if (head_dim == 128) k_unpack<128><<<grid, kThreads, 0, st>>>(b);
    else k_unpack<64><<<grid, kThreads, 0, st>>>(b);
    return cudaGetLastError();
}

}  // namespace cbk
