// What the kernels of cb_weigh share: what a segment's tokens see, and the weights of its rows.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "cb_attend.cuh"

namespace cbk {

constexpr int kWeighRows = 4096;    // query rows of a sequence and KV head at most: one row tile for all

// Positions are counted from the segment's beginning: 32 bits hold them, and their sums with tokens and windows (a window that
// reaches past every cache is none).
constexpr int64_t kNoWindow = (int64_t)0x7FFFF000;

struct WeighRows {
    int at;                 // of token 0
    int window;             // 0: none
    int fresh;              // rows from here on have gathered nothing
    int m, len, G, n_q_heads;
    bool causal, tree;
    int64_t begin;

    __device__ __forceinline__ WeighRows(const WeighBatch& b, const Segment& x)
        : at((int)x.at), window(b.sees_window), m(b.span[x.seq].m), len(x.len), G(b.G), n_q_heads(b.n_q_heads), causal(b.sees != 0),
          tree(b.w[x.seq].tree.seen != nullptr), begin(x.begin) {
        fresh = (int)(x.at + m - b.w[x.seq].fresh);
    }

    // Of the 32 positions from t0 on, those that a token sees, as bits.  (Tokens behind the last: some.)
    __device__ __forceinline__ uint32_t seen(const WeighSeq& w, int token, int t0) const {
        int lo = t0, hi = len;                              // positions [lo, hi)
        uint32_t bits = 0xFFFFFFFFu;
        if (tree) {
            bits = tree_bits(w.tree.seen + min(token, m - 1) * w.tree.s_row, (m + 31) / 32, t0 - at);
        } else if (causal) {
            hi = min(hi, at + token + 1);
            if (window) lo = max(lo, at + token - window + 1);
        }
        if (hi <= lo || lo >= t0 + 32) return 0;
        const int a = lo - t0, n = min(32, hi - t0);        // bits a .. n - 1
        return bits & (0xFFFFFFFFu << a) & (0xFFFFFFFFu >> (32 - n));
    }
    // The log-sum-exp of a query row (token, head of the group).
    __device__ __forceinline__ float lse(const WeighSeq& w, int g, int row) const {
        return __ldg(w.lse + (int64_t)(row / G) * n_q_heads + g * G + row % G);
    }
    // What row t had gathered.
    __device__ __forceinline__ float before(const WeighSeq& w, int g, int t) const {
        return w.before && t < min(len, fresh) ? w.before[(int64_t)g * w.b_head + begin + t] : 0.f;
    }
};

cudaError_t launch_weigh_tc(WeighBatch& b, int head_dim, cudaStream_t st, int num_sms);

}  // namespace cbk
