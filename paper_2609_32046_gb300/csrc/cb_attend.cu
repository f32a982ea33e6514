// Attention of query tokens over a cache held in 4 bits (cb_attend): few query rows a KV head
// (k_attend_few), the joining of partial results (k_attend_join), and the choice between the kernels.
//
//   out = sum_t p_t v_t / sum_t p_t,   p_t = exp2(z_t - M),   z_t = scale * log2(e) * <q, k_t>
//
// in one pass over the rows with a running M.  A packed value c * s is a bf16 number and an fp16
// number exactly, so products of queries and keys (bf16) and of weights and values (fp16) round
// nothing of the cache; weights are rounded to fp16, 2^-12 of each.
#include <cmath>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "cb_attend.cuh"
#include "cb_internal.cuh"

namespace cbk {
namespace {

constexpr int kWarps = 4;
constexpr int kStep = 32;                // positions a warp takes at a time
constexpr int kStages = 2;               // of them in shared memory
// Weights are exp2(z - top + 14): up to 2^14, so that fp16 holds those down to 2^-28 of the largest as
// normal numbers and to 2^-38 at all, and 32-bit sums stay in range.
constexpr float kWeightBits = 14.f;

// D (16 x 8) += A (16 x 16) B (16 x 8), fp32 sums.
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Copies of 16, 8 or 4 bytes into shared memory (nothing read and zeros written without `there`).
__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}
template <int N>
__device__ __forceinline__ void copy_small(uint32_t to, const void* from, bool there) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(to), "l"(from), "n"(N), "r"(there ? N : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// 32 positions of a warp in shared memory: codes of K, of V (rows of D / 2 bytes), scales of K, of V.
// Thread (gid, tig) = (lane / 4, lane % 4) reads of K the quarter tig of the rows of its two operand rows,
// of V the eighth gid of four rows.  Operand row r of 16 positions is position place(r), so that those four
// are 4 i + tig: with the codes' places below both reads meet every bank once.
__device__ __forceinline__ int place(int r) { return (r & 8) + ((r >> 1) & 3) + 4 * (r & 1); }
template <int D>
struct Stage {
    static constexpr int kCodes = kStep * D / 2, kScales = kStep * D / 16, kBytes = 2 * (kCodes + kScales);
    // Byte of piece p (16 bytes) of a row's codes.
    static __device__ __forceinline__ uint32_t at(int row, int p) {
        if (D == 128) return (row >> 1) * 128 + ((row ^ (row >> 2)) & 1) * 64 + ((p ^ (row & 2)) << 4);
        return (row >> 2) * 128 + (((row & 3) ^ ((row >> 1) & 2)) << 5) + (p << 4);
    }
};

// The row of position t0 + lane from the head's base on: -1 where there is none (from `end` on, or a bad
// block-table entry).
__device__ __forceinline__ int row_of_lane(const PackedRows& p, int64_t t0, int64_t end, uint32_t* err) {
    const int64_t t = t0 + (threadIdx.x & 31);
    if (t >= end) return -1;
    const int64_t r = packed_row(p, t);
    if (r < 0) atomicOr(err, kErrPageIndex);
    return (int)r;
}

struct Bases {
    const uint8_t *k, *v;
    const uint16_t *ks, *vs;
};

template <int D>
__device__ __forceinline__ void copy_stage(uint32_t to, const Bases& x, int mine) {
    constexpr int P = D / 32;             // pieces of a row's codes
    constexpr int N = 32 / P;             // rows a copy of the warp takes
    using S = Stage<D>;
    const int lane = threadIdx.x & 31, p = lane % P;
#pragma unroll
    for (int i = 0; i < 32 / N; ++i) {
        const int row = lane / P + i * N;
        const int r = __shfl_sync(0xFFFFFFFFu, mine, row);
        const int64_t off = (int64_t)(r < 0 ? 0 : r) * (D / 2) + p * 16;
        copy16(to + S::at(row, p), x.k + off, r >= 0);
        copy16(to + S::kCodes + S::at(row, p), x.v + off, r >= 0);
    }
    const int64_t off = (int64_t)(mine < 0 ? 0 : mine) * (D / 32);
    copy_small<D / 16>(to + 2 * S::kCodes + lane * (D / 16), x.ks + off, mine >= 0);
    copy_small<D / 16>(to + 2 * S::kCodes + S::kScales + lane * (D / 16), x.vs + off, mine >= 0);
}

// Looks a lane's scales over (its row's, K's and V's): what is none becomes 0.  True where every scale of V
// in the warp's rows is 0 or within 2^-16 .. 2^9, where values_f16_near applies.
template <int D>
__device__ __forceinline__ bool look_over(uint8_t* stage, uint32_t* err) {
    constexpr int W = D / 64;             // words of two scales in a row
    uint32_t* ks = reinterpret_cast<uint32_t*>(stage + 2 * Stage<D>::kCodes) + (threadIdx.x & 31) * W;
    uint32_t* vs = ks + Stage<D>::kScales / 4;
    uint32_t top = 0, high = 0, low = 0xFFFFFFFFu;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        top = __vmaxu2(top, ks[i]);
        high = __vmaxu2(high, vs[i]);
        low = __vminu2(low, __vsub2(vs[i], 0x00010001u));          // (0 becomes the largest)
    }
    top = __vmaxu2(top, high);
    if (__any_sync(0xFFFFFFFFu, max(top & 0xFFFFu, top >> 16) > kTopScaleBits)) {
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            ks[i] = checked_scale(ks[i] & 0xFFFFu, bad) | checked_scale(ks[i] >> 16, bad) << 16;
            vs[i] = checked_scale(vs[i] & 0xFFFFu, bad) | checked_scale(vs[i] >> 16, bad) << 16;
        }
        if (bad) atomicOr(err, kErrPackScale);
        __syncwarp();
    }
    const bool near = max(high & 0xFFFFu, high >> 16) <= 0x4400u && min(low & 0xFFFFu, low >> 16) >= 0x377Fu;
    return __all_sync(0xFFFFFFFFu, near);
}

template <int BYTES> struct Piece;
template <> struct Piece<16> { using T = uint4; };
template <> struct Piece<8> { using T = uint2; };
template <> struct Piece<4> { using T = uint32_t; };
__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ uint32_t word_of(const uint2& v, int i) { return i == 0 ? v.x : v.y; }
__device__ __forceinline__ uint32_t word_of(const uint32_t& v, int) { return v; }

// O^T += V^T P^T of 16 positions (rows row0 .. row0 + 15 of the stage).
template <int D, int NT, bool NEAR>
__device__ __forceinline__ void add_values(const uint8_t* stage, int row0, const uint32_t (&p)[NT][2], float (&o)[NT][D / 16][4]) {
    constexpr int VW = D / 64;            // words of V a thread takes of a row
    using S = Stage<D>;
    const int lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
    typename Piece<D / 16>::T c[4];
    uint32_t s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = row0 + 4 * i + tig;
        c[i] = *reinterpret_cast<const typename Piece<D / 16>::T*>(stage + S::kCodes + S::at(row, gid * (D / 16) / 16) +
                                                                  gid * (D / 16) % 16);
        s[i] = *reinterpret_cast<const uint16_t*>(stage + 2 * S::kCodes + S::kScales + row * (D / 16) + gid * (D / 32) / 8 * 2);
    }
    const uint32_t s01 = f16_scales(s[0], s[1]), s89 = f16_scales(s[2], s[3]);
#pragma unroll
    for (int w = 0; w < VW; ++w) {
        // pairs of positions, element by element: low halves hold elements 0, 2, 4, 6, high ones 1, 3, 5, 7
        const uint32_t a = word_of(c[0], w), a1 = word_of(c[1], w), a8 = word_of(c[2], w), a9 = word_of(c[3], w);
        uint32_t u[4], v[4], u8[4], v8[4];
        values_f16<NEAR>(__byte_perm(a, a1, 0x5410), s01, u);
        values_f16<NEAR>(__byte_perm(a, a1, 0x7632), s01, v);
        values_f16<NEAR>(__byte_perm(a8, a9, 0x5410), s89, u8);
        values_f16<NEAR>(__byte_perm(a8, a9, 0x7632), s89, v8);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t f[4] = {u[j], v[j], u8[j], v8[j]};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_f16(o[nt][4 * w + j], f, p[nt][0], p[nt][1]);
        }
    }
}

template <int D, int NT>
constexpr int few_smem() {
    constexpr int stages = kWarps * kStages * Stage<D>::kBytes, join = kWarps * 8 * NT * (D * 4 + 8);
    return stages > join ? stages : join;
}

// Grid: x = part of the positions, y = (KV head, row tile), z = sequence.  A block takes 8 NT query
// rows (token, head of the group) of one KV head over one part; its four warps take 32 positions in
// turn, each with its own copies, running maximum and sums, and join at the end.
//   S^T [16 positions][8 rows] = K Q^T: keys are the operand with 16 rows, so that a group's few
//     query rows fill the one with 8;
//   O^T [D][8 rows] += V^T P^T, with P^T turned by movmatrix from S^T's layout.
template <int D, int NT>
__global__ void __launch_bounds__(kWarps * 32) k_attend_few(const __grid_constant__ AttendBatch b, int tiles_max) {
    constexpr int KW = D / 32;            // words of K a thread holds of a row
    constexpr int ROWS = 8 * NT;
    using S = Stage<D>;
    extern __shared__ __align__(128) uint8_t smem[];
    const AttendSeq& s = b.s[blockIdx.z];
    const int g = blockIdx.y / tiles_max, tile = blockIdx.y % tiles_max;
    if (tile >= s.tiles || (int)blockIdx.x >= s.splits) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gid = lane >> 2, tig = lane & 3;
    const int R = s.m * b.G, row0 = tile * ROWS;
    const int64_t L = attend_length(s);
    const Span span = attend_span(b, s, L, row0, min(row0 + ROWS, R) - 1, blockIdx.x, kWarps * kStep);

    const int64_t head = (int64_t)g * s.kv.s_head;
    const Bases from{s.kv.code[0] + head * (D / 2), s.kv.code[1] + head * (D / 2), s.kv.scale[0] + head * (D / 32),
                     s.kv.scale[1] + head * (D / 32)};
    uint8_t* stages = smem + warp * kStages * S::kBytes;
    const uint32_t to = sm100::smem_u32(stages);

    // the copies run kStages tiles of 32 ahead, the block-table entries one more
    int64_t t0 = span.begin + warp * kStep, ahead = t0;
    int mine = row_of_lane(s.kv, ahead, span.end, b.err);
#pragma unroll
    for (int i = 0; i < kStages; ++i) {
        if (span.begin < span.end) copy_stage<D>(to + i * S::kBytes, from, mine);   // (an empty cache may have no memory)
        copy_commit();
        ahead += kWarps * kStep;
        mine = row_of_lane(s.kv, ahead, span.end, b.err);
    }

    // query rows of column gid: the elements that the thread's pieces of K hold
    uint32_t q[NT][KW][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int row = row0 + nt * 8 + gid;
        const uint16_t* qp = s.q + (int64_t)(row / b.G) * s.s_tok + (int64_t)(g * b.G + row % b.G) * s.s_head + tig * (D / 4);
#pragma unroll
        for (int w = 0; w < KW; ++w) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (row < R) v = __ldg(reinterpret_cast<const uint4*>(qp + w * 8));
            q[nt][w][0] = v.x; q[nt][w][1] = v.y; q[nt][w][2] = v.z; q[nt][w][3] = v.w;
        }
    }

    float o[NT][D / 16][4], top[NT][2], sum[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
        top[nt][0] = top[nt][1] = -INFINITY;
        sum[nt][0] = sum[nt][1] = 0.f;
    }

    for (int turn = 0; t0 < span.end; t0 += kWarps * kStep) {
        uint8_t* st = stages + turn * S::kBytes;
        copy_wait<kStages - 1>();
        __syncwarp();
        const bool near = look_over<D>(st, b.err);

        float z[2][NT][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int ra = 16 * i + place(gid), rb = ra + 8;       // operand rows gid and gid + 8
            const auto ca = *reinterpret_cast<const typename Piece<D / 8>::T*>(st + S::at(ra, tig * (D / 8) / 16) + tig * (D / 8) % 16);
            const auto cb = *reinterpret_cast<const typename Piece<D / 8>::T*>(st + S::at(rb, tig * (D / 8) / 16) + tig * (D / 8) % 16);
            const uint16_t* sc = reinterpret_cast<const uint16_t*>(st + 2 * S::kCodes);
            const uint32_t sa = sc[ra * (D / 32) + tig * (D / 32) / 4] * 0x10001u, sb = sc[rb * (D / 32) + tig * (D / 32) / 4] * 0x10001u;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) z[i][nt][0] = z[i][nt][1] = z[i][nt][2] = z[i][nt][3] = 0.f;
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                uint32_t u[4], v[4];
                values_bf16(word_of(ca, w), sa, u);
                values_bf16(word_of(cb, w), sb, v);
                const uint32_t a0[4] = {u[0], v[0], u[1], v[1]}, a1[4] = {u[2], v[2], u[3], v[3]};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mma_bf16(z[i][nt], a0, q[nt][w][0], q[nt][w][1]);
                    mma_bf16(z[i][nt], a1, q[nt][w][2], q[nt][w][3]);
                }
            }
        }
        // positions 16 i + place(gid) (elements 0, 1) and + 8 (2, 3), columns 2 tig and 2 tig + 1
        const bool edge = t0 + kStep > span.all_from_here || t0 < span.all_to_here;
        if (edge) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t at = L - s.m + (row0 + nt * 8 + 2 * tig + h) / b.G;     // position of the column's token
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int64_t t = t0 + 8 * k + place(gid);
                        if (t >= span.end || (b.causal && (t > at || (b.window && t <= at - b.window))))
                            z[k / 2][nt][2 * (k % 2) + h] = -INFINITY;
                    }
                }
        }
        float high[NT][2];
        bool grow = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                high[nt][h] = b.scale_log2e * fmaxf(fmaxf(z[0][nt][h], z[0][nt][2 + h]), fmaxf(z[1][nt][h], z[1][nt][2 + h]));
                grow |= high[nt][h] > top[nt][h];
            }
        if (__any_sync(0xFFFFFFFFu, grow)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float y = fmaxf(high[nt][h], top[nt][h]);
#pragma unroll
                    for (int k = 4; k <= 16; k *= 2) y = fmaxf(y, __shfl_xor_sync(0xFFFFFFFFu, y, k));
                    const float f = y == -INFINITY ? 1.f : exp2f(top[nt][h] - y);
                    top[nt][h] = y;
                    sum[nt][h] *= f;
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        o[nt][i][h] *= f;
                        o[nt][i][2 + h] *= f;
                    }
                }
        }
        uint32_t p[2][NT][2];             // weights as the second product's operand
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float m0 = top[nt][0] == -INFINITY ? 0.f : kWeightBits - top[nt][0];
            const float m1 = top[nt][1] == -INFINITY ? 0.f : kWeightBits - top[nt][1];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float y0 = ex2(fmaf(z[i][nt][2 * e], b.scale_log2e, m0));
                    const float y1 = ex2(fmaf(z[i][nt][2 * e + 1], b.scale_log2e, m1));
                    sum[nt][0] += y0;
                    sum[nt][1] += y1;
                    p[i][nt][e] = transpose8(pack_f16(y0, y1));
                }
        }
        if (near) {
            add_values<D, NT, true>(st, 0, p[0], o);
            add_values<D, NT, true>(st, 16, p[1], o);
        } else {
            add_values<D, NT, false>(st, 0, p[0], o);
            add_values<D, NT, false>(st, 16, p[1], o);
        }
        __syncwarp();
        copy_stage<D>(to + turn * S::kBytes, from, mine);
        copy_commit();
        ahead += kWarps * kStep;
        mine = row_of_lane(s.kv, ahead, span.end, b.err);
        turn = turn + 1 == kStages ? 0 : turn + 1;
    }
    copy_wait<0>();
    __syncthreads();

    // join the warps: every warp's sums relative to the largest M
    float* sh_o = reinterpret_cast<float*>(smem);                            // [warp][row][D]
    float* sh_m = sh_o + kWarps * ROWS * D;                                  // [warp][row]
    float* sh_l = sh_m + kWarps * ROWS;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float l = sum[nt][h];
#pragma unroll
            for (int k = 4; k <= 16; k *= 2) l += __shfl_xor_sync(0xFFFFFFFFu, l, k);
            if (gid == 0) {
                sh_m[warp * ROWS + nt * 8 + 2 * tig + h] = top[nt][h] - kWeightBits;
                sh_l[warp * ROWS + nt * 8 + 2 * tig + h] = l;
            }
        }
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = nt * 8 + 2 * tig + h;
            float M = sh_m[r];
#pragma unroll
            for (int w = 1; w < kWarps; ++w) M = fmaxf(M, sh_m[w * ROWS + r]);
            const float f = top[nt][h] == -INFINITY ? 0.f : exp2f(top[nt][h] - kWeightBits - M);
            // elements (D / 8) gid + 2 i (register h) and + 2 i + 1 (register 2 + h)
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
                *reinterpret_cast<float2*>(sh_o + (warp * ROWS + r) * D + gid * (D / 8) + 2 * i) =
                    make_float2(o[nt][i][h] * f, o[nt][i][2 + h] * f);
        }
    __syncthreads();
    const bool whole = s.splits == 1;
    const int64_t slot = s.slot0 + ((int64_t)g * s.tiles + tile) * s.splits + blockIdx.x;
    for (int e = threadIdx.x; e < ROWS * (D / 4); e += kWarps * 32) {
        const int r = e / (D / 4), d = (e % (D / 4)) * 4, row = row0 + r;
        if (row >= R) break;
        float M = sh_m[r];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) M = fmaxf(M, sh_m[w * ROWS + r]);
        float l = 0.f;
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float m = sh_m[w * ROWS + r];
            l += m == -INFINITY ? 0.f : sh_l[w * ROWS + r] * exp2f(m - M);
            const float4 v = *reinterpret_cast<const float4*>(sh_o + (w * ROWS + r) * D + d);
            y.x += v.x; y.y += v.y; y.z += v.z; y.w += v.w;
        }
        if (whole) {
            attend_write<D>(b, s, g, row, d, y, M, l);
        } else {
            *reinterpret_cast<float4*>(b.part + (slot * ROWS + r) * D + d) = y;
            if (d == 0) b.part_ml[slot * ROWS + r] = make_float2(M, l);
        }
    }
}

// A warp a query row: the parts' sums relative to the largest M, part by part in order.
template <int D>
__global__ void __launch_bounds__(128) k_attend_join(const __grid_constant__ AttendBatch b, int tile_rows) {
    const AttendSeq& s = b.s[blockIdx.y];
    const int R = s.m * b.G;
    const int at = blockIdx.x * 4 + (threadIdx.x >> 5);
    if (s.splits == 1 || at >= R * b.n_kv_heads) return;
    const int g = at / R, row = at % R, tile = row / tile_rows, r = row % tile_rows, lane = threadIdx.x & 31;
    const int64_t slot = s.slot0 + ((int64_t)g * s.tiles + tile) * s.splits;
    const float2* ml = b.part_ml + slot * tile_rows + r;
    float M = -INFINITY;
    for (int k = lane; k < s.splits; k += 32) M = fmaxf(M, ml[(int64_t)k * tile_rows].x);
#pragma unroll
    for (int k = 16; k; k /= 2) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, k));
    float l = 0.f;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    const float* part = b.part + (slot * tile_rows + r) * D + lane * 4;
#pragma unroll 4
    for (int k = 0; k < s.splits; ++k) {
        const float2 x = ml[(int64_t)k * tile_rows];
        const float f = x.x == -INFINITY ? 0.f : exp2f(x.x - M);
        l += x.y * f;
        if (lane * 4 < D) {
            const float4 v = *reinterpret_cast<const float4*>(part + (int64_t)k * tile_rows * D);
            y.x += v.x * f; y.y += v.y * f; y.z += v.z * f; y.w += v.w * f;
        }
    }
    if (lane * 4 < D) attend_write<D>(b, s, g, row, lane * 4, y, M, l);
}

template <int D, int NT>
cudaError_t launch_few(const AttendBatch& b, dim3 grid, int tiles, cudaStream_t st) {
    static_assert(few_smem<D, NT>() <= 48 * 1024, "more needs the function's attribute set");
    k_attend_few<D, NT><<<grid, kWarps * 32, few_smem<D, NT>(), st>>>(b, tiles);
    return cudaGetLastError();
}

}  // namespace

int64_t attend_part_rows(int num_sms) { return (int64_t)num_sms * kPartRowsPerSm; }

// Parts of every sequence's positions, so that about `blocks` blocks of tile_rows query rows run, each
// over at least `least` positions; false where the partial results do not fit.
bool attend_plan(AttendBatch& b, int tile_rows, int64_t blocks, int64_t least, int num_sms) {
    double all = 0;
    for (int i = 0; i < b.n; ++i) {
        AttendSeq& s = b.s[i];
        s.tiles = (s.m * b.G + tile_rows - 1) / tile_rows;
        all += (double)attend_reach(b, s) * s.tiles * b.n_kv_heads;
    }
    int64_t slots = 0;
    for (int i = 0; i < b.n; ++i) {
        AttendSeq& s = b.s[i];
        const int64_t reach = attend_reach(b, s);
        int64_t k = all > 0 ? (int64_t)((double)reach * blocks / all) : 1;
        const int64_t most = (reach + least - 1) / least;
        k = k < most ? k : most;
        k = k > 1 ? k : 1;
        s.splits = (int32_t)k;
        s.slot0 = (int32_t)slots;
        if (k > 1) slots += k * s.tiles * b.n_kv_heads;
        if (slots * tile_rows > attend_part_rows(num_sms)) return false;
    }
    return true;
}

cudaError_t attend_join(const AttendBatch& b, int head_dim, int tile_rows, cudaStream_t st) {
    int rows = 0;
    for (int i = 0; i < b.n; ++i)
        if (b.s[i].splits > 1) rows = b.s[i].m > rows ? b.s[i].m : rows;
    if (rows == 0) return cudaSuccess;
    const dim3 grid((unsigned)((rows * b.G * b.n_kv_heads + 3) / 4), (unsigned)b.n);
    if (head_dim == 128) k_attend_join<128><<<grid, 128, 0, st>>>(b, tile_rows);
    else k_attend_join<64><<<grid, 128, 0, st>>>(b, tile_rows);
    return cudaGetLastError();
}

cudaError_t launch_attend(AttendBatch& b, int head_dim, cudaStream_t st, int num_sms) {
    int rows = 0;
    for (int i = 0; i < b.n; ++i) rows = b.s[i].m > rows ? b.s[i].m : rows;
    rows *= b.G;
    if (rows == 0) return cudaSuccess;
    if (rows > 16) return launch_attend_tc(b, head_dim, st, num_sms);
    const int tile_rows = rows <= 8 ? 8 : 16;
    for (int64_t blocks = (int64_t)num_sms * 4; !attend_plan(b, tile_rows, blocks, kWarps * kStep, num_sms); blocks /= 2) {}
    int splits = 1, tiles = 1;
    for (int i = 0; i < b.n; ++i) {
        splits = b.s[i].splits > splits ? b.s[i].splits : splits;
        tiles = b.s[i].tiles > tiles ? b.s[i].tiles : tiles;
    }
    const dim3 grid((unsigned)splits, (unsigned)(b.n_kv_heads * tiles), (unsigned)b.n);
    cudaError_t e = head_dim == 128 ? (tile_rows == 8 ? launch_few<128, 1>(b, grid, tiles, st) : launch_few<128, 2>(b, grid, tiles, st))
                                    : (tile_rows == 8 ? launch_few<64, 1>(b, grid, tiles, st) : launch_few<64, 2>(b, grid, tiles, st));
    if (e == cudaSuccess) e = attend_join(b, head_dim, tile_rows, st);
    return e;
}

}  // namespace cbk
