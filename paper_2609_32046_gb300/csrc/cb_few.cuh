// Logits of few query rows (token, head of the group) by mma.sync, for the kernels of cb_attend and cb_weigh: packed
// keys in shared memory, 32 positions a warp.  Keys are the operand with 16 rows, so that a group's few query
// rows fill the one with 8.
#pragma once

#include <cstdint>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "cb_attend.cuh"

namespace cbk {

constexpr int kStep = 32;                // positions a warp takes at a time

// D (16 x 8) += A (16 x 16) B (16 x 8), fp32 sums.
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// 32 positions of a warp in shared memory: codes of K, of V (rows of D / 2 bytes), scales of K, of V
// (PLANES = 2), or of K alone.
// Thread (gid, tig) = (lane / 4, lane % 4) reads of K the quarter tig of the rows of its two operand rows,
// of V the eighth gid of four rows.  Operand row r of 16 positions is position place(r), so that those four
// are 4 i + tig: with the codes' places below both reads meet every bank once.
__device__ __forceinline__ int place(int r) { return (r & 8) + ((r >> 1) & 3) + 4 * (r & 1); }
template <int D, int PLANES = 2>
struct Stage {
    static constexpr int kCodes = kStep * D / 2, kScales = kStep * D / 16, kBytes = PLANES * (kCodes + kScales);
    // Byte of piece p (16 bytes) of a row's codes.
    static __device__ __forceinline__ uint32_t at(int row, int p) {
        if (D == 128) return (row >> 1) * 128 + ((row ^ (row >> 2)) & 1) * 64 + ((p ^ (row & 2)) << 4);
        return (row >> 2) * 128 + (((row & 3) ^ ((row >> 1) & 2)) << 5) + (p << 4);
    }
};

template <int BYTES> struct Piece;
template <> struct Piece<16> { using T = uint4; };
template <> struct Piece<8> { using T = uint2; };
template <> struct Piece<4> { using T = uint32_t; };
__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ uint32_t word_of(const uint2& v, int i) { return i == 0 ? v.x : v.y; }
__device__ __forceinline__ uint32_t word_of(const uint32_t& v, int) { return v; }

// Logits of 16 positions, S^T = K Q^T: operand rows are the positions row0 + place(r) of the stage.
template <int D, int NT, bool NEAR, int PLANES = 2>
__device__ __forceinline__ void score_keys(const uint8_t* stage, int row0, const uint32_t (&q)[NT][D / 32][4], float (&z)[NT][4]) {
    constexpr int KW = D / 32;            // words of K a thread takes of a row
    using S = Stage<D, PLANES>;
    using T = typename Piece<D / 8>::T;
    const int lane = threadIdx.x & 31, tig = lane & 3;
    const int ra = row0 + place(lane >> 2), rb = ra + 8;
    const T ca = *reinterpret_cast<const T*>(stage + S::at(ra, tig * (D / 8) / 16) + tig * (D / 8) % 16);
    const T cb = *reinterpret_cast<const T*>(stage + S::at(rb, tig * (D / 8) / 16) + tig * (D / 8) % 16);
    const uint16_t* sc = reinterpret_cast<const uint16_t*>(stage + PLANES * S::kCodes) + tig * (D / 32) / 4;
    const uint32_t xa = sc[ra * (D / 32)], xb = sc[rb * (D / 32)];
    const uint32_t sa = f16_scales(xa, xa), sb = f16_scales(xb, xb);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) z[nt][0] = z[nt][1] = z[nt][2] = z[nt][3] = 0.f;
#pragma unroll
    for (int w = 0; w < KW; ++w) {
        uint32_t u[4], v[4];
        values_f16<NEAR>(word_of(ca, w), sa, u);
        values_f16<NEAR>(word_of(cb, w), sb, v);
        const uint32_t a0[4] = {u[0], v[0], u[1], v[1]}, a1[4] = {u[2], v[2], u[3], v[3]};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            mma_f16(z[nt], a0, q[nt][w][0], q[nt][w][1]);
            mma_f16(z[nt], a1, q[nt][w][2], q[nt][w][3]);
        }
    }
}

// Query rows row0 + 8 nt + gid of head group g (of `rows`; zeros behind them): the elements that the thread's pieces
// of K hold, and the factors that make logits (log2 domain) of the products of columns 2 tig and 2 tig + 1.
// Queries become fp16 numbers times a power of two that takes a row's largest element to 2^14 .. 2^15:
// elements down to 2^-29 of it exactly (a bf16 number has 8 bits), smaller ones to 2^-39 of it.
// Rows that `there` does not know are zeros too.
struct EveryRow {
    __device__ __forceinline__ bool operator()(int) const { return true; }
};
template <int D, int NT, class There = EveryRow>
__device__ __forceinline__ void load_queries(const AttendBatch& b, const AttendSeq& s, int g, int row0, int rows,
                                             uint32_t (&q)[NT][D / 32][4], float (&zs)[NT][2], const There& there = There()) {
    constexpr int KW = D / 32;            // words of K a thread holds of a row
    const int lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int row = row0 + nt * 8 + gid;
        const uint16_t* qp = s.q + (int64_t)(row / b.G) * s.s_tok + (int64_t)(g * b.G + row % b.G) * s.s_head + tig * (D / 4);
        uint32_t top = 0;
#pragma unroll
        for (int w = 0; w < KW; ++w) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (row < rows && there(row)) v = __ldg(reinterpret_cast<const uint4*>(qp + w * 8));
            q[nt][w][0] = v.x; q[nt][w][1] = v.y; q[nt][w][2] = v.z; q[nt][w][3] = v.w;
#pragma unroll
            for (int k = 0; k < 4; ++k) top = __vmaxu2(top, q[nt][w][k] & 0x7FFF7FFFu);
        }
        top = max(top & 0xFFFFu, top >> 16) >> 7;       // exponent of the largest
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const uint32_t e = min(max(top, 15u), 253u);    // 2^(141 - e): of normal numbers on both sides
        // (never 0, which times a masked row's -infinity would be NaN: logits are below 2^38, and 2^-88 is none either)
        const float up = __uint_as_float((268u - e) << 23);
        const float down = fmaxf(__uint_as_float((e - 14u) << 23) * b.scale_log2e, 1.17549435e-38f);
#pragma unroll
        for (int w = 0; w < KW; ++w)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                q[nt][w][k] = pack_f16(__uint_as_float(q[nt][w][k] << 16) * up, __uint_as_float(q[nt][w][k] & 0xFFFF0000u) * up);
        zs[nt][0] = __shfl_sync(0xFFFFFFFFu, down, 8 * tig);
        zs[nt][1] = __shfl_sync(0xFFFFFFFFu, down, 8 * tig + 4);
    }
}

}  // namespace cbk
