// Attention of query tokens over a cache held in 4 bits (cb_attend): few query rows a KV head
// (k_attend_few), and the choice between the kernels.
//
//   out = sum_t p_t v_t / sum_t p_t,   p_t = exp2(z_t - M),   z_t = scale * log2(e) * <q, k_t>
//
// in one pass over the rows with a running M.  A packed value c * s is a bf16 number and an fp16
// number exactly, so products of queries and keys (bf16) and of weights and values (fp16) round
// nothing of the cache.  Weights are rounded to fp16 for their product with the values, which is off by at most
// 2^-11 of each, an eighth of what rounding an output to bf16 may cost; their sum takes them unrounded, in
// fp32.  Errors against 64 bits: those of the rounded output, + 0.05% here and + 0.6% in k_attend_tc.
#include <cmath>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "cb_attend.cuh"
#include "cb_few.cuh"
#include "cb_receiver.cuh"

namespace cbk {
namespace {

constexpr int kWarps = 4;
constexpr int kStages = 2;               // of them in shared memory
// Weights are exp2(z - top + 14): up to 2^14, so that fp16 holds those down to 2^-28 of the largest as
// normal numbers and to 2^-38 at all, and 32-bit sums stay in range.
constexpr float kWeightBits = 14.f;

__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// Copies 32 positions; mine: the row of this lane's.  The codes of a position that has none are some row's: its
// scales are zeros.
template <int D>
__device__ __forceinline__ void copy_stage(uint32_t to, const Segment& x, int mine) {
    constexpr int P = D / 32;             // pieces of a row's codes
    constexpr int N = 32 / P;             // rows a copy of the warp takes
    using S = Stage<D>;
    const int lane = threadIdx.x & 31, p = lane % P;
    const uint32_t row = max(mine, 0);
    const uint8_t *k = x.code[0] + p * 16, *v = x.code[1] + p * 16;
#pragma unroll
    for (int i = 0; i < 32 / N; ++i) {
        const int at = lane / P + i * N;
        const uint64_t off = (uint64_t)__shfl_sync(0xFFFFFFFFu, row, at) * (D / 2);
        copy16(to + S::at(at, p), k + off);
        copy16(to + S::kCodes + S::at(at, p), v + off);
    }
    const uint64_t off = (uint64_t)row * (D / 16);
    copy_small<D / 16>(to + 2 * S::kCodes + lane * (D / 16), reinterpret_cast<const uint8_t*>(x.scale[0]) + off, mine >= 0);
    copy_small<D / 16>(to + 2 * S::kCodes + S::kScales + lane * (D / 16), reinterpret_cast<const uint8_t*>(x.scale[1]) + off,
                       mine >= 0);
}

// Looks a lane's scales over (its row's, K's and V's): what is none becomes 0.  True where every scale of the
// warp's rows is within 2^-14 .. 2^7 (values_f16's NEAR).
template <int D>
__device__ __forceinline__ bool look_over(uint8_t* stage, uint32_t* err) {
    constexpr int W = D / 64;             // words of two scales in a row
    uint32_t* ks = reinterpret_cast<uint32_t*>(stage + 2 * Stage<D>::kCodes) + (threadIdx.x & 31) * W;
    uint32_t* vs = ks + Stage<D>::kScales / 4;
    uint32_t top = __vmaxu2(ks[0], vs[0]), low = __vminu2(ks[0], vs[0]);
    if (W > 1) {
        top = __vmaxu2(top, __vmaxu2(ks[W - 1], vs[W - 1]));
        low = __vminu2(low, __vminu2(ks[W - 1], vs[W - 1]));
    }
    // (a bf16 number's bits above 2^7's or below 2^-14's)
    const bool far = max(top & 0xFFFFu, top >> 16) > 0x4300u || min(low & 0xFFFFu, low >> 16) < 0x3880u;
    if (!__any_sync(0xFFFFFFFFu, far)) return true;
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        ks[i] = checked_scale(ks[i] & 0xFFFFu, bad) | checked_scale(ks[i] >> 16, bad) << 16;
        vs[i] = checked_scale(vs[i] & 0xFFFFu, bad) | checked_scale(vs[i] >> 16, bad) << 16;
    }
    if (bad) atomicOr(err, kErrPackScale);
    __syncwarp();
    return false;
}

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

// Blocks an SM holds: 120 registers a thread, or 168.
template <int D, int NT>
constexpr int few_blocks() { return D == 128 && NT == 2 ? 3 : kFewBlocksPerSm; }

// True in the last of n blocks to come here, which then sees what the others wrote.  Whole block.
__device__ __forceinline__ bool last_of(int32_t* ticket, int n, int* last) {
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        *last = atomicAdd(ticket, 1) == n - 1;
        if (*last) *ticket = 0;
    }
    __syncthreads();
    if (*last) __threadfence();
    return *last;
}

// attend_join_row for all of a tile's rows, by the whole block: the same sums in the same order, but what a row's parts are
// multiplied by is worked out once a row, eight lanes a row and part each, and not by every thread of the row again (16
// parts of 16 rows: 10 us that way).  sh: room for ROWS rows' factors.
template <int D, int ROWS, class Done>
__device__ __forceinline__ void join_parts(const AttendBatch& b, float* sh, int64_t slot0, int skip, int step, int n, int rows, Done done) {
    constexpr int kParts = 8;
    static_assert(kWarps * 32 >= ROWS * kParts, "");
    const int turns = (n + kParts - 1) / kParts;
    float* part_f = sh;                                  // [row][part]: factor of a part
    float* turn_f = part_f + ROWS * turns * kParts;      // [row][eight parts]: factor of what was there before them
    float2* ends = reinterpret_cast<float2*>(turn_f + ROWS * turns + (ROWS * turns & 1));
    {
        const int r = threadIdx.x / kParts, i = threadIdx.x % kParts;
        float M = -INFINITY, l = 0.f;
        for (int k0 = 0; k0 < n; k0 += kParts) {
            const int k = k0 + i;
            float2 x = make_float2(-INFINITY, 0.f);
            if (k < n && r < rows) x = __ldcg(b.part_ml + (slot0 + (k ? k * step : skip)) * ROWS + r);
            float top = fmaxf(M, x.x);
#pragma unroll
            for (int y = 1; y < kParts; y *= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, y));
            const float f = M == -INFINITY ? 0.f : exp2f(M - top), p = x.x == -INFINITY ? 0.f : exp2f(x.x - top);
            l *= f;
            M = top;
#pragma unroll
            for (int y = 0; y < kParts; ++y)
                l = fmaf(__shfl_sync(0xFFFFFFFFu, x.y, y, kParts), __shfl_sync(0xFFFFFFFFu, p, y, kParts), l);
            if (r < ROWS) {
                part_f[r * turns * kParts + k] = p;
                if (i == 0) turn_f[r * turns + k0 / kParts] = f;
            }
        }
        if (i == 0 && r < ROWS) ends[r] = make_float2(M, l);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < rows * (D / 4); e += kWarps * 32) {
        const int r = e / (D / 4), d = (e % (D / 4)) * 4;
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
        float nothing = 0.f;
#pragma unroll 2
        for (int t = 0; t < turns; ++t) {
            float4 v[kParts];
#pragma unroll
            for (int i = 0; i < kParts; ++i) {
                const int k = t * kParts + i;
                v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (k < n) v[i] = __ldcg(reinterpret_cast<const float4*>(b.part + ((slot0 + (k ? k * step : skip)) * ROWS + r) * D + d));
            }
            const float f = turn_f[r * turns + t];
            y.x *= f; y.y *= f; y.z *= f; y.w *= f;
#pragma unroll
            for (int i = 0; i < kParts; ++i) add_part(y, nothing, v[i], part_f[(r * turns + t) * kParts + i], 0.f);
        }
        done(r, d, y, ends[r].x, ends[r].y);
    }
}

// A block takes its run of units (cb_attend.cuh), 8 NT query rows (token, head of the group) of one KV head
// at a time; its four warps take 32 positions in turn, each with its own copies, running maximum and
// sums, and join at a segment's end.  The last block to leave a part of an item joins the parts, block by
// block in order.
//   S^T [16 positions][8 rows] = K Q^T (cb_few.cuh);
//   O^T [D][8 rows] += V^T P^T, with P^T turned by movmatrix from S^T's layout.
//
// Bound by the instructions that turn codes into numbers (half-rate logic and the fp16 fma: some 870 a warp for 32
// positions), and for one sequence by the joins.  48 sequences in pages, 8 KV heads of 128: 83 us, 3.2 TB/s; one
// token over 65536 positions 33 us, 2.3 TB/s.  Rows read straight into registers took 291 and 163 us; a third
// stage of copies 87 us and 34 us.
template <int D, int NT, class Batch>
__global__ void __launch_bounds__(kWarps * 32, few_blocks<D, NT>()) k_attend_few(const __grid_constant__ Batch b) {
    constexpr int KW = D / 32;            // words of K a thread holds of a row
    constexpr int ROWS = 8 * NT;
    using S = Stage<D>;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int pre[kMaxBatch + 1];
    __shared__ Segment x;
    __shared__ int last;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gid = lane >> 2, tig = lane & 3;
    attend_units(b, ROWS, pre);
    const int g = blockIdx.x % b.n_kv_heads, run = blockIdx.x / b.n_kv_heads;
    const Runs runs = attend_runs(pre[b.pairs], gridDim.x / b.n_kv_heads);
    if (run >= runs.blocks) return;
    const int run0 = attend_run(runs, run), run1 = attend_run(runs, run + 1);
    uint8_t* stages = smem + warp * kStages * S::kBytes;
    const uint32_t to = sm100::smem_u32(stages);
    for (int unit = run0; unit < run1;) {
        if (threadIdx.x == 0) attend_segment(b, pre, 1, g, unit, run1, D, ROWS, &x);
        __syncthreads();
        // the copies run kStages tiles of 32 ahead, the block-table entries one more
        int t0 = warp * kStep, ahead = t0;
        uint32_t page = segment_page(x, ahead + lane);
#pragma unroll
        for (int i = 0; i < kStages; ++i) {
            if (ahead < x.len) copy_stage<D>(to + i * S::kBytes, x, segment_row(x, ahead + lane, page, b.err));
            copy_commit();
            ahead += kWarps * kStep;
            page = segment_page(x, ahead + lane);
        }

        uint32_t q[NT][KW][4];
        float zs[NT][2];                  // factor of the logits of columns 2 tig and 2 tig + 1
        load_queries<D, NT>(b, b.s[x.seq], g, 0, x.rows, q, zs);               // (one row tile: at most 16 rows)

        float o[NT][D / 16][4], top[NT][2], sum[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < D / 16; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
            top[nt][0] = top[nt][1] = -INFINITY;
            sum[nt][0] = sum[nt][1] = 0.f;
        }

        for (int turn = 0; t0 < x.len; t0 += kWarps * kStep) {
            uint8_t* st = stages + turn * S::kBytes;
            copy_wait<kStages - 1>();
            __syncwarp();
            const bool near = look_over<D>(st, b.err);
            float z[2][NT][4];
            if (near) {
                score_keys<D, NT, true>(st, 0, q, z[0]);
                score_keys<D, NT, true>(st, 16, q, z[1]);
            } else {
                score_keys<D, NT, false>(st, 0, q, z[0]);
                score_keys<D, NT, false>(st, 16, q, z[1]);
            }
            // positions 16 i + place(gid) (elements 0, 1) and + 8 (2, 3), columns 2 tig and 2 tig + 1
            if (t0 + kStep > x.all_from || t0 < x.all_to) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int64_t at = x.at + (nt * 8 + 2 * tig + h) / b.G;       // position of the column's token
                        if constexpr (Batch::kTrees) {
                            const TreeBits& tree = b.tree[x.seq];
                            if (tree.seen) {
                                // (columns behind the last token's read that one's bits; nothing is made of them)
                                const int m = b.span[x.seq].m, r = min((int)(at - x.at), m - 1);
                                const uint32_t bits = tree_bits(tree.seen + r * tree.s_row, (m + 31) / 32, t0 - x.at);
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    if (t0 + 8 * k + place(gid) >= x.len || !(bits >> (8 * k + place(gid)) & 1u))
                                        z[k / 2][nt][2 * (k % 2) + h] = -INFINITY;
                                continue;
                            }
                        }
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int t = t0 + 8 * k + place(gid);
                            if (t >= x.len || (b.causal && (t > at || (b.window && t <= at - b.window))))
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
                    high[nt][h] = zs[nt][h] * fmaxf(fmaxf(z[0][nt][h], z[0][nt][2 + h]), fmaxf(z[1][nt][h], z[1][nt][2 + h]));
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
                        const float y0 = ex2(fmaf(z[i][nt][2 * e], zs[nt][0], m0));
                        const float y1 = ex2(fmaf(z[i][nt][2 * e + 1], zs[nt][1], m1));
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
            if (ahead < x.len) copy_stage<D>(to + turn * S::kBytes, x, segment_row(x, ahead + lane, page, b.err));
            copy_commit();
            ahead += kWarps * kStep;
            page = segment_page(x, ahead + lane);
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
                const int r = nt * 8 + 2 * tig + h;
                if (gid == 0) {
                    sh_m[warp * ROWS + r] = top[nt][h] - kWeightBits;
                    sh_l[warp * ROWS + r] = l;
                }
                // elements (D / 8) gid + 2 i (register h) and + 2 i + 1 (register 2 + h)
                if (r < x.rows) {
#pragma unroll
                    for (int i = 0; i < D / 16; ++i)
                        *reinterpret_cast<float2*>(sh_o + (warp * ROWS + r) * D + gid * (D / 8) + 2 * i) =
                            make_float2(o[nt][i][h], o[nt][i][2 + h]);
                }
            }
        __syncthreads();
        const AttendSeq& s = b.s[x.seq];
        const bool whole = x.n == x.units;
        const int64_t slot = 2 * (int64_t)blockIdx.x + (unit == run0 ? 0 : 1);
        for (int e = threadIdx.x; e < x.rows * (D / 4); e += kWarps * 32) {
            const int r = e / (D / 4), d = (e % (D / 4)) * 4;
            float M = sh_m[r], l = 0.f;
#pragma unroll
            for (int w = 1; w < kWarps; ++w) M = fmaxf(M, sh_m[w * ROWS + r]);
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float m = sh_m[w * ROWS + r];
                add_part(y, l, *reinterpret_cast<const float4*>(sh_o + (w * ROWS + r) * D + d), m == -INFINITY ? 0.f : exp2f(m - M),
                         sh_l[w * ROWS + r]);
            }
            if (whole) {
                attend_write<D>(b, s, g, r, d, y, M, l);
            } else {
                *reinterpret_cast<float4*>(b.part + (slot * ROWS + r) * D + d) = y;
                if (d == 0) b.part_ml[slot * ROWS + r] = make_float2(M, l);
            }
        }
        if (!whole) {
            // n parts, from run b0 on, in groups of `size`, about the root of their number.  (Loads that the last
            // block waits for: 76 parts a head joined at once took 11 us of one token's 38 over 65536 positions, in
            // two steps 6; 16 parts took 0.8 us longer in two.  Both before join_parts.)
            const int b0 = attend_block(runs, x.first), n = attend_block(runs, x.first + x.units - 1) - b0 + 1;
            int size = 16;
            while (size * size < n) size += 8;
            const int groups = (n + size - 1) / size, group = (run - b0) / size, head = b0 + group * size;
            const int skip = attend_run(runs, b0) == x.first ? 0 : 1;          // of the first run's two slots
            const int of_group = group == 0 ? skip : 0;
            const int members = min(size, n - group * size);
            const int64_t group0 = 2 * ((int64_t)head * b.n_kv_heads + g);     // its first block's slots
            float* sh = reinterpret_cast<float*>(smem);
            auto write = [&](int r, int d, float4 y, float M, float l) { attend_write<D>(b, s, g, r, d, y, M, l); };
            if (last_of(b.tickets + group0 + of_group, members, &last)) {
                if (groups == 1) {
                    join_parts<D, ROWS>(b, sh, group0, of_group, 2 * b.n_kv_heads, members, x.rows, write);
                } else {
                    join_parts<D, ROWS>(b, sh, group0, of_group, 2 * b.n_kv_heads, members, x.rows, [&](int r, int d, float4 y, float M, float l) {
                        const int64_t at = (2 * (int64_t)gridDim.x + group0 + of_group) * ROWS + r;
                        *reinterpret_cast<float4*>(b.part + at * D + d) = y;
                        if (d == 0) b.part_ml[at] = make_float2(M, l);
                    });
                    const int64_t item0 = (int64_t)b0 * b.n_kv_heads + g;
                    if (last_of(b.tickets + 2 * gridDim.x + item0, groups, &last))
                        join_parts<D, ROWS>(b, sh, 2 * ((int64_t)gridDim.x + item0), skip, 2 * size * b.n_kv_heads, groups, x.rows, write);
                }
            }
        }
        unit += x.n;
        __syncthreads();
    }
}

template <int D, int NT, class Batch>
cudaError_t launch_few(const Batch& b, int64_t units, int num_sms, cudaStream_t st) {
    // as many runs as leave no block waiting, one at least
    const int64_t most = num_sms * few_blocks<D, NT>() / b.n_kv_heads, all = units / b.n_kv_heads;
    const int64_t runs = all < most ? all : most;
    const int blocks = (int)(runs > 1 ? runs : 1) * b.n_kv_heads;
    static_assert(few_smem<D, NT>() <= 46 * 1024, "more needs the function's attribute set");
    k_attend_few<D, NT, Batch><<<blocks, kWarps * 32, few_smem<D, NT>(), st>>>(b);
    return cudaGetLastError();
}

}  // namespace

int64_t attend_part_rows(int num_sms) { return (int64_t)num_sms * kPartRowsPerSm; }

int64_t attend_pairs(AttendBatch& b, int tile_rows) {
    int64_t units = 0;
    b.pairs = 0;
    b.window = b.window < kFarWindow ? b.window : kFarWindow;
    for (int i = 0; i < b.n; ++i) {
        AttendSpan& s = b.span[i];
        const int tiles = (s.m * b.G + tile_rows - 1) / tile_rows;
        const int64_t w = b.causal && b.window ? b.window + s.m : s.T, reach = s.T < w ? s.T : w;
        s.pair0 = b.pairs;
        b.pairs += tiles;
        units += tiles * b.n_kv_heads * (reach / kUnit + 2);
    }
    return units;
}

template <class Batch>
static cudaError_t launch_by_rows(Batch& b, int head_dim, cudaStream_t st, int num_sms) {
    int rows = 0;
    for (int i = 0; i < b.n; ++i) rows = b.span[i].m > rows ? b.span[i].m : rows;
    rows *= b.G;
    if (rows == 0) return cudaSuccess;
    // Up to 16 rows a KV head (token, head of its group) their sums stay in a warp's registers, above that the tcgen05
    // kernel takes over.  8 KV heads of 128, 2048 / 16384 positions: 8 rows 11.2 / 19.5 us here and 17.8 / 35.0 us
    // there, 16 rows 15.7 / 24.6 and 18.1 / 35.2 us.
    // The rule goes by the longest of the call's sequences.  What one of many rows costs the others, 47 decoding
    // sequences in pages (4 rows each, 8 KV heads of 128; 86 us by themselves) with one of m tokens, in one call / in
    // two: m = 2 88 / 106 us, 4 111 / 116, 16 240 / 111, 64 288 / 118, 1024 398 / 207.
    if (rows > 16) return launch_attend_tc(b, head_dim, st, num_sms);
    // (With the join as it was, 8 rows in a tile of 16: 13.4 / 22.3 us; 4 rows 10.2 / 17.1 in one of 8, 10.8 / 18.4 in one of 16.)
    const int tile_rows = rows <= 8 ? 8 : 16;
    const int64_t units = attend_pairs(b, tile_rows);
    if (head_dim == 128)
        return tile_rows == 8 ? launch_few<128, 1>(b, units, num_sms, st) : launch_few<128, 2>(b, units, num_sms, st);
    return tile_rows == 8 ? launch_few<64, 1>(b, units, num_sms, st) : launch_few<64, 2>(b, units, num_sms, st);
}

cudaError_t launch_attend(AttendBatch& b, int head_dim, cudaStream_t st, int num_sms) {
    return launch_by_rows(b, head_dim, st, num_sms);
}
cudaError_t launch_attend(AttendTreeBatch& b, int head_dim, cudaStream_t st, int num_sms) {
    return launch_by_rows(b, head_dim, st, num_sms);
}

}  // namespace cbk
