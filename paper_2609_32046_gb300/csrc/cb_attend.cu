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

template <int BYTES> struct Piece;
template <> struct Piece<16> { using T = uint4; };
template <> struct Piece<8> { using T = uint2; };
template <> struct Piece<4> { using T = uint32_t; };
__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ uint32_t word_of(const uint2& v, int i) { return i == 0 ? v.x : v.y; }
__device__ __forceinline__ uint32_t word_of(const uint32_t& v, int) { return v; }

// What a thread reads of 32 positions.  Lane (gid, tig) = (lane / 4, lane % 4): of the rows gid,
// gid + 8, .. the quarter tig of K (whole words of 8 elements of one group), of the rows 2 tig,
// 2 tig + 1, 2 tig + 8, .. the eighth gid of V.
template <int D>
struct Tile {
    typename Piece<D / 8>::T k[4];
    typename Piece<D / 16>::T v[8];
    uint32_t ks[4], vs[8];
};

// Rows from `base` to the 32 positions from t0 on, the one of position t0 + lane: -1 where there is
// none (from `end` on, or a bad block-table entry).
__device__ __forceinline__ int row_of_lane(const PackedRows& p, int64_t t0, int64_t end, uint32_t* err) {
    const int64_t t = t0 + (threadIdx.x & 31);
    if (t >= end) return -1;
    const int64_t r = packed_row(p, t);
    if (r < 0) atomicOr(err, kErrPageIndex);
    return (int)r;
}

template <int D>
__device__ __forceinline__ void load_tile(Tile<D>& x, const uint8_t* k, const uint8_t* v, const uint16_t* ks,
                                          const uint16_t* vs, int mine) {
    const int lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = __shfl_sync(0xFFFFFFFFu, mine, gid + 8 * i);
        x.ks[i] = 0;
        x.k[i] = {};
        if (r >= 0) {
            x.k[i] = __ldg(reinterpret_cast<const typename Piece<D / 8>::T*>(k + (int64_t)r * (D / 2) + tig * (D / 8)));
            x.ks[i] = __ldg(ks + (int64_t)r * (D / 32) + tig * (D / 32) / 4);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = __shfl_sync(0xFFFFFFFFu, mine, 16 * (i / 4) + 8 * ((i / 2) % 2) + 2 * tig + i % 2);
        x.vs[i] = 0;
        x.v[i] = {};
        if (r >= 0) {
            x.v[i] = __ldg(reinterpret_cast<const typename Piece<D / 16>::T*>(v + (int64_t)r * (D / 2) + gid * (D / 16)));
            x.vs[i] = __ldg(vs + (int64_t)r * (D / 32) + gid * (D / 32) / 8);
        }
    }
}

// Grid: x = part of the positions, y = (KV head, row tile), z = sequence.  A block takes 8 NT query
// rows (token, head of the group) of one KV head over one part; its four warps take 32 positions in
// turn, each with its own running maximum and sums, and join at the end.
//   S^T [16 positions][8 rows] = K Q^T: keys are the operand with 16 rows, so that a group's few
//     query rows fill the one with 8;
//   O^T [D][8 rows] += V^T P^T, with P^T turned by movmatrix from S^T's layout.
template <int D, int NT>
__global__ void __launch_bounds__(kWarps * 32) k_attend_few(const __grid_constant__ AttendBatch b, int tiles_max) {
    constexpr int KW = D / 32;            // words of K a thread holds of a row
    constexpr int VW = D / 64;            // words of V
    constexpr int ROWS = 8 * NT;
    const AttendSeq& s = b.s[blockIdx.z];
    const int g = blockIdx.y / tiles_max, tile = blockIdx.y % tiles_max;
    if (tile >= s.tiles || (int)blockIdx.x >= s.splits) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gid = lane >> 2, tig = lane & 3;
    const int R = s.m * b.G, row0 = tile * ROWS;
    const int64_t L = attend_length(s);
    const Span span = attend_span(b, s, L, row0, min(row0 + ROWS, R) - 1, blockIdx.x, kWarps * kStep);

    const int64_t head = (int64_t)g * s.kv.s_head;
    const uint8_t* kc = s.kv.code[0] + head * (D / 2);
    const uint8_t* vc = s.kv.code[1] + head * (D / 2);
    const uint16_t* ksc = s.kv.scale[0] + head * (D / 32);
    const uint16_t* vsc = s.kv.scale[1] + head * (D / 32);

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

    uint32_t bad = 0;
    Tile<D> x;
    int64_t t0 = span.begin + warp * kStep;
    int mine = t0 < span.end ? row_of_lane(s.kv, t0, span.end, b.err) : -1;
    int next = t0 + kWarps * kStep < span.end ? row_of_lane(s.kv, t0 + kWarps * kStep, span.end, b.err) : -1;
    if (t0 < span.end) load_tile<D>(x, kc, vc, ksc, vsc, mine);
    for (; t0 < span.end; t0 += kWarps * kStep) {
        const Tile<D> c = x;
        mine = next;
        if (t0 + kWarps * kStep < span.end) load_tile<D>(x, kc, vc, ksc, vsc, mine);
        if (t0 + 2 * kWarps * kStep < span.end) next = row_of_lane(s.kv, t0 + 2 * kWarps * kStep, span.end, b.err);

        float z[2][NT][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) z[i][nt][0] = z[i][nt][1] = z[i][nt][2] = z[i][nt][3] = 0.f;
            const uint32_t s0 = checked_scale(c.ks[2 * i], bad) * 0x10001u, s1 = checked_scale(c.ks[2 * i + 1], bad) * 0x10001u;
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                uint32_t u[4], v[4];
                values_bf16(word_of(c.k[2 * i], w), s0, u);
                values_bf16(word_of(c.k[2 * i + 1], w), s1, v);
                const uint32_t a0[4] = {u[0], v[0], u[1], v[1]}, a1[4] = {u[2], v[2], u[3], v[3]};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mma_bf16(z[i][nt], a0, q[nt][w][0], q[nt][w][1]);
                    mma_bf16(z[i][nt], a1, q[nt][w][2], q[nt][w][3]);
                }
            }
        }
        // rows 16 i + gid (elements 0, 1) and 16 i + gid + 8 (2, 3), columns 2 tig and 2 tig + 1
        const bool edge = t0 + kStep > span.all_from_here || t0 < span.all_to_here;
        float high[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t at = L - s.m + (row0 + nt * 8 + 2 * tig + h) / b.G;     // position of the column's token
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float& y = z[i][nt][2 * e + h];
                        y *= b.scale_log2e;
                        if (edge) {
                            const int64_t t = t0 + 16 * i + 8 * e + gid;
                            if (t >= span.end || (b.causal && (t > at || (b.window && t <= at - b.window)))) y = -INFINITY;
                        }
                    }
                high[nt][h] = fmaxf(fmaxf(z[0][nt][h], z[0][nt][2 + h]), fmaxf(z[1][nt][h], z[1][nt][2 + h]));
            }
        bool grow = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) grow |= high[nt][0] > top[nt][0] || high[nt][1] > top[nt][1];
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
            const float m0 = top[nt][0] == -INFINITY ? 0.f : top[nt][0] - kWeightBits;
            const float m1 = top[nt][1] == -INFINITY ? 0.f : top[nt][1] - kWeightBits;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float y0 = ex2(z[i][nt][2 * e] - m0), y1 = ex2(z[i][nt][2 * e + 1] - m1);
                    sum[nt][0] += y0;
                    sum[nt][1] += y1;
                    p[i][nt][e] = transpose8(pack_f16(y0, y1));
                }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t s01 = f16_scales(checked_scale(c.vs[4 * i], bad), checked_scale(c.vs[4 * i + 1], bad));
            const uint32_t s89 = f16_scales(checked_scale(c.vs[4 * i + 2], bad), checked_scale(c.vs[4 * i + 3], bad));
#pragma unroll
            for (int w = 0; w < VW; ++w) {
                // pairs of positions, element by element: low halves hold elements 0, 2, 4, 6, high ones 1, 3, 5, 7
                const uint32_t a = word_of(c.v[4 * i], w), a1 = word_of(c.v[4 * i + 1], w);
                const uint32_t a8 = word_of(c.v[4 * i + 2], w), a9 = word_of(c.v[4 * i + 3], w);
                uint32_t u[4], v[4], u8[4], v8[4];
                values_f16(__byte_perm(a, a1, 0x5410), s01, u);
                values_f16(__byte_perm(a, a1, 0x7632), s01, v);
                values_f16(__byte_perm(a8, a9, 0x5410), s89, u8);
                values_f16(__byte_perm(a8, a9, 0x7632), s89, v8);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t f[4] = {u[j], v[j], u8[j], v8[j]};
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_f16(o[nt][4 * w + j], f, p[i][nt][0], p[i][nt][1]);
                }
            }
        }
    }
    if (bad) atomicOr(b.err, kErrPackScale);

    // join the warps: every warp's sums relative to the largest M
    __shared__ float sh_o[kWarps][ROWS][D];
    __shared__ float sh_m[kWarps][ROWS], sh_l[kWarps][ROWS];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float l = sum[nt][h];
#pragma unroll
            for (int k = 4; k <= 16; k *= 2) l += __shfl_xor_sync(0xFFFFFFFFu, l, k);
            if (gid == 0) {
                sh_m[warp][nt * 8 + 2 * tig + h] = top[nt][h] - kWeightBits;
                sh_l[warp][nt * 8 + 2 * tig + h] = l;
            }
        }
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = nt * 8 + 2 * tig + h;
            float M = sh_m[0][r];
#pragma unroll
            for (int w = 1; w < kWarps; ++w) M = fmaxf(M, sh_m[w][r]);
            const float f = top[nt][h] == -INFINITY ? 0.f : exp2f(top[nt][h] - kWeightBits - M);
            // elements (D / 8) gid + 2 i (register h) and + 2 i + 1 (register 2 + h)
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
                *reinterpret_cast<float2*>(&sh_o[warp][r][gid * (D / 8) + 2 * i]) =
                    make_float2(o[nt][i][h] * f, o[nt][i][2 + h] * f);
        }
    __syncthreads();
    const bool whole = s.splits == 1;
    const int64_t slot = s.slot0 + ((int64_t)g * s.tiles + tile) * s.splits + blockIdx.x;
    for (int e = threadIdx.x; e < ROWS * (D / 4); e += kWarps * 32) {
        const int r = e / (D / 4), d = (e % (D / 4)) * 4, row = row0 + r;
        if (row >= R) break;
        float M = sh_m[0][r];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) M = fmaxf(M, sh_m[w][r]);
        float l = 0.f;
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float m = sh_m[w][r];
            l += m == -INFINITY ? 0.f : sh_l[w][r] * exp2f(m - M);
            const float4 v = *reinterpret_cast<const float4*>(&sh_o[w][r][d]);
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
    if (head_dim == 128) {
        if (tile_rows == 8) k_attend_few<128, 1><<<grid, kWarps * 32, 0, st>>>(b, tiles);
        else k_attend_few<128, 2><<<grid, kWarps * 32, 0, st>>>(b, tiles);
    } else {
        if (tile_rows == 8) k_attend_few<64, 1><<<grid, kWarps * 32, 0, st>>>(b, tiles);
        else k_attend_few<64, 2><<<grid, kWarps * 32, 0, st>>>(b, tiles);
    }
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) e = attend_join(b, head_dim, tile_rows, st);
    return e;
}

}  // namespace cbk
