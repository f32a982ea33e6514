// Attention weights gathered by the rows of a 4-bit cache (cb_weigh):
//
//   w_t = decay * w_t + sum over query rows (token, head of the group) that see t of exp2(z_t - lse * log2(e)),
//   z_t = scale * log2(e) * <q, k_t>
//
// Products are exact (a packed key is an fp16 number and a bf16 number), sums are fp32.
#include <cmath>
#include <cstdint>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "cb_few.cuh"
#include "cb_weigh.cuh"

namespace cbk {
namespace {

constexpr int kWarps = 4;
constexpr int kStages = 2;
constexpr int kBlocksPerSm = 5;          // (48 sequences' weights: 4 blocks 55 us, 5 53, 6 54.4, 7 64)

// Copies 32 positions' keys; mine: the row of this lane's.  The codes of a position that has none are some row's: its
// scales are zeros.
template <int D>
__device__ __forceinline__ void copy_keys(uint32_t to, const Segment& x, int mine) {
    constexpr int P = D / 32;             // pieces of a row's codes
    constexpr int N = 32 / P;             // rows a copy of the warp takes
    using S = Stage<D, 1>;
    const int lane = threadIdx.x & 31, p = lane % P;
    const uint32_t row = max(mine, 0);
#pragma unroll
    for (int i = 0; i < 32 / N; ++i) {
        const int at = lane / P + i * N;
        copy16(to + S::at(at, p), x.code[0] + (uint64_t)__shfl_sync(0xFFFFFFFFu, row, at) * (D / 2) + p * 16);
    }
    copy_small<D / 16>(to + S::kCodes + lane * (D / 16),
                       reinterpret_cast<const uint8_t*>(x.scale[0]) + (uint64_t)row * (D / 16), mine >= 0);
}

// Looks a lane's scales over: what is none becomes 0.  True where every scale of the warp's rows is within
// 2^-14 .. 2^7 (values_f16's NEAR).
template <int D>
__device__ __forceinline__ bool look_over_keys(uint8_t* stage, uint32_t* err) {
    constexpr int W = D / 64;             // words of two scales in a row
    uint32_t* ks = reinterpret_cast<uint32_t*>(stage + Stage<D, 1>::kCodes) + (threadIdx.x & 31) * W;
    const uint32_t top = __vmaxu2(ks[0], ks[W - 1]), low = __vminu2(ks[0], ks[W - 1]);
    const bool far = max(top & 0xFFFFu, top >> 16) > 0x4300u || min(low & 0xFFFFu, low >> 16) < 0x3880u;
    if (!__any_sync(0xFFFFFFFFu, far)) return true;
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) ks[i] = checked_scale(ks[i] & 0xFFFFu, bad) | checked_scale(ks[i] >> 16, bad) << 16;
    if (bad) atomicOr(err, kErrPackScale);
    __syncwarp();
    return false;
}

// Up to 16 query rows a KV head.  A block takes its run of units (cb_attend.cuh); its four warps take 32 positions in turn,
// each with its own copies.  S^T [16 positions][8 rows] = K Q^T (cb_few.cuh), the rows' weights are added up over a quad's
// lanes, and every position's sum is written by one lane: nothing to join.
//
// Bound, as k_attend_few's half of the keys is, by some 570 instructions a warp for 32 positions (64 of them conversions and 140
// masks and shifts of codes) and by what they wait for one another, with 20 warps an SM: issue slots 59%, logic pipe 48%, none
// is full. 48 sequences in pages, 8 KV heads of 128, 4 rows: 53 us, 2.8 TB/s, where the bytes take 22; one token over 2048
// positions 5.3 us.
template <int D, int NT>
__global__ void __launch_bounds__(kWarps * 32, kBlocksPerSm) k_weigh_few(const __grid_constant__ WeighBatch b) {
    using S = Stage<D, 1>;
    __shared__ __align__(128) uint8_t smem[kWarps * kStages * S::kBytes];
    __shared__ int pre[kMaxBatch + 1];
    __shared__ Segment x;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gid = lane >> 2, tig = lane & 3;
    attend_units(b, kWeighRows, pre);
    const int g = blockIdx.x % b.n_kv_heads, run = blockIdx.x / b.n_kv_heads;
    const Runs runs = attend_runs(pre[b.pairs], gridDim.x / b.n_kv_heads);
    if (run >= runs.blocks) return;
    const int run0 = attend_run(runs, run), run1 = attend_run(runs, run + 1);
    uint8_t* stages = smem + warp * kStages * S::kBytes;
    const uint32_t to = sm100::smem_u32(stages);
    for (int unit = run0; unit < run1;) {
        if (threadIdx.x == 0) attend_segment(b, pre, 1, g, unit, run1, D, kWeighRows, &x);
        __syncthreads();
        const WeighSeq& w = b.w[x.seq];
        const WeighRows rows(b, x);
        // positions before `low` no token sees; those before `all_to` and from `all_from` on not every one does
        const bool windowed = rows.causal && rows.window && !rows.tree;
        const int low = windowed ? max(0, rows.at - rows.window + 1) : 0, len = x.len;
        const int all_to = windowed ? rows.at + rows.m - rows.window : 0;
        const int all_from = rows.tree ? rows.at : rows.causal ? rows.at + 1 : len;
        float* to_w = w.weights + (int64_t)g * w.w_head + x.begin;
        const float* from_w = w.before + (int64_t)g * w.b_head + x.begin;
        const int had = w.before ? min(len, rows.fresh) : 0;
        int t0 = warp * kStep, ahead = t0;
        uint32_t page = segment_page(x, ahead + lane);
#pragma unroll
        for (int i = 0; i < kStages; ++i) {
            if (ahead < len && ahead + kStep > low) copy_keys<D>(to + i * S::kBytes, x, segment_row(x, ahead + lane, page, b.err));
            copy_commit();
            ahead += kWarps * kStep;
            page = segment_page(x, ahead + lane);
        }
        uint32_t q[NT][D / 32][4];
        // of columns 2 tig and 2 tig + 1: factor of the logits, -lse * log2(e), and 2^(what its rounding left out)
        float zs[NT][2], nl[NT][2], rest[NT][2];
        load_queries<D, NT>(b, b.s[x.seq], g, 0, x.rows, q, zs, [&](int row) { return isfinite(rows.lse(w, g, row)); });
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = nt * 8 + 2 * tig + h;
                const float lse = row < x.rows ? rows.lse(w, g, row) : INFINITY;
                const float l = lse * -b.lse_log2e;
                nl[nt][h] = isfinite(lse) ? l : -INFINITY;
                // (2^x = 1 + x ln 2 for an x of 2^-20: nearer than the approximation of exp2 is)
                rest[nt][h] = isfinite(lse) ? fmaf(fmaf(lse, -b.lse_log2e, -l) - lse * b.lse_log2e_lo, 0.6931471805599453f, 1.f) : 0.f;
            }
        for (int turn = 0; t0 < len; t0 += kWarps * kStep) {
            uint8_t* st = stages + turn * S::kBytes;
            const int own = t0 + 8 * tig + place(gid);          // the position whose sum this lane writes
            const float before = own < had ? from_w[own] : 0.f;
            copy_wait<kStages - 1>();
            __syncwarp();
            float s[4] = {};                                    // of positions t0 + 8 k + place(gid)
            if (t0 + kStep > low) {
                const bool near = look_over_keys<D>(st, b.err), edge = t0 + kStep > min(len, all_from) || t0 < all_to;
                float z[2][NT][4];
                if (near) {
                    score_keys<D, NT, true, 1>(st, 0, q, z[0]);
                    score_keys<D, NT, true, 1>(st, 16, q, z[1]);
                } else {
                    score_keys<D, NT, false, 1>(st, 0, q, z[0]);
                    score_keys<D, NT, false, 1>(st, 16, q, z[1]);
                }
                if (edge) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t bits = rows.seen(w, (nt * 8 + 2 * tig + h) / b.G, t0);
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                if (!(bits >> (8 * k + place(gid)) & 1u)) z[k / 2][nt][2 * (k % 2) + h] = -INFINITY;
                        }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        s[k] = fmaf(ex2(fmaf(z[k / 2][nt][2 * (k % 2)], zs[nt][0], nl[nt][0])), rest[nt][0],
                                    fmaf(ex2(fmaf(z[k / 2][nt][2 * (k % 2) + 1], zs[nt][1], nl[nt][1])), rest[nt][1], s[k]));
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                s[k] += __shfl_xor_sync(0xFFFFFFFFu, s[k], 1);
                s[k] += __shfl_xor_sync(0xFFFFFFFFu, s[k], 2);
            }
            const float sum = tig == 0 ? s[0] : tig == 1 ? s[1] : tig == 2 ? s[2] : s[3];
            if (own < len) to_w[own] = fmaf(b.decay, before, sum);
            __syncwarp();
            if (ahead < len && ahead + kStep > low) copy_keys<D>(to + turn * S::kBytes, x, segment_row(x, ahead + lane, page, b.err));
            copy_commit();
            ahead += kWarps * kStep;
            page = segment_page(x, ahead + lane);
            turn = turn + 1 == kStages ? 0 : turn + 1;
        }
        copy_wait<0>();
        unit += x.n;
        __syncthreads();
    }
}

template <int D, int NT>
cudaError_t launch_few(const WeighBatch& b, int64_t units, int num_sms, cudaStream_t st) {
    const int64_t most = num_sms * kBlocksPerSm / b.n_kv_heads, all = units / b.n_kv_heads;
    const int64_t runs = all < most ? all : most;
    k_weigh_few<D, NT><<<(int)(runs > 1 ? runs : 1) * b.n_kv_heads, kWarps * 32, 0, st>>>(b);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_weigh(WeighBatch& b, int head_dim, cudaStream_t st, int num_sms) {
    int rows = 0;
    for (int i = 0; i < b.n; ++i) rows = b.span[i].m > rows ? b.span[i].m : rows;
    rows *= b.G;
    if (rows == 0) return cudaSuccess;
    // 8 KV heads of 128, 2048 / 16384 positions: 8 rows 5.7 / 8.4 us here and 8.4 / 16.0 us on tcgen05, 16 rows 7.3 / 10.2 and
    // 8.4 / 15.9 us; 20 rows, a third tile of them here, 8.6 / 15.9 us there.  48 sequences of 2048 / 6000 positions (graphs, 7 us
    // of them not the kernel's): 4 rows 32 / 67 us here and 65 / 147 there, 16 rows 38 / 81 and 67 / 149.
    // The rule goes by the longest of the call's sequences: 47 tokens and one sequence of 5 take 65 / 149 us in one call, 44 / 81 in
    // two, so a server calls for them apart.
    if (rows > 16) return launch_weigh_tc(b, head_dim, st, num_sms);
    const int64_t units = attend_pairs(b, kWeighRows);
    if (head_dim == 128)
        return rows <= 8 ? launch_few<128, 1>(b, units, num_sms, st) : launch_few<128, 2>(b, units, num_sms, st);
    return rows <= 8 ? launch_few<64, 1>(b, units, num_sms, st) : launch_few<64, 2>(b, units, num_sms, st);
}

}  // namespace cbk
