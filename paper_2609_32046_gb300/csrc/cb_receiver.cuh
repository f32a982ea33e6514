// What the receiver's side (rotary positions, rows held in 4 bits, attention over them) hands from the host to its
// kernels.  Apart from cb_internal.cuh, which the score kernels are built and profiled with.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "cb_internal.cuh"

namespace cbk {

// Bits of the error word that cb_sync_status reads, beside cb_internal.cuh's.
constexpr uint32_t kErrPackValue = 32u;    // cb_pack: a value that is not finite or above 7 * 2^13
constexpr uint32_t kErrPackScale = 64u;    // cb_attend, cb_unpack: a scale outside [0, 2^13]
constexpr uint32_t kErrPackRow = 128u;     // cb_pack: a destination row outside [0, T)

// Rotary embedding of sets of vectors (cb_rotary).
struct RotarySet {
    const uint16_t* x;
    uint16_t* y;
    const int32_t* pos;       // or null: pos0 + token
    int64_t pos0;
    int64_t n_tokens;
    int64_t s_layer, s_tok, s_head;
    int64_t o_layer, o_tok, o_head;
    int32_t n_layers, n_heads;
};

struct RotaryBatch {
    int32_t n;
    int32_t dims;             // rotary part of the head
    float gain, sine_gain;    // what cosine and sine are multiplied by
    uint64_t turns[64];       // f_k / (2 pi) * 2^64
    RotarySet s[kMaxBatch];
};

// Rows held in 4 bits (cb_packed).  Offsets of rows count rows of head_dim elements: below 2^31.
struct PackedRows {
    uint8_t* code[2];         // K, V
    uint16_t* scale[2];
    int64_t s_layer, s_head, s_pos;   // in rows
    const int32_t* pages;     // block table, or null
    int64_t s_page, n_pages;
    int32_t shift;            // log2(page_size)
};

// Rows from the (l, g) base of a packed cache to position t's row; -1 for a bad block-table entry.
__device__ __forceinline__ int64_t packed_row(const PackedRows& p, int64_t t) {
    if (!p.pages) return t * p.s_pos;
    const int32_t page = __ldg(p.pages + (t >> p.shift));
    if (page < 0 || page >= p.n_pages) return -1;
    return (int64_t)page * p.s_page + (t & ((int64_t(1) << p.shift) - 1)) * p.s_pos;
}

struct PackSender {
    const uint16_t* src[2];   // K, V (cb_pack)
    int64_t ks_l, ks_h, ks_p;
    PageMap pm;
    int64_t T;                // rows of the source
    const int32_t* idx;       // or null: row j
    const int32_t* rows;      // cb_pack: destination rows, or null: dst_off + j
    int64_t count;
    int64_t dst_off;
    int64_t dst_T;            // cb_pack: rows of the destination
    PackedRows held;
};

constexpr int kMaxPackBatch = 32;
struct PackBatch {
    int32_t n;
    int32_t n_layers, n_kv_heads, layer;
    uint16_t* out[2];         // cb_unpack
    int64_t o_layer, o_head;
    uint32_t* err;
    PackSender s[kMaxPackBatch];
};

// One sequence of cb_attend.
struct AttendSeq {
    PackedRows kv;            // bases at the call's layer
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    int64_t s_tok, s_head, o_tok, o_head;
};

// What decides a sequence's share of the work, apart from the rest: every block reads it of all sequences.
struct AttendSpan {
    int64_t T;
    const int32_t* length;    // or null
    int32_t m;
    int32_t pair0;            // row tiles of the sequences before
};

// An item (row tile, head) of k_attend_tc that several blocks' runs share: the parts' blocks are block, block + 1 ...
struct AttendCut {
    int32_t seq, g, row0, rows;
    int32_t parts;            // 0: none
    int32_t block, skip;      // skip: which of the first block's two slots
};

struct AttendBatch {
    static constexpr bool kTrees = false;
    int32_t n;
    int32_t n_q_heads, n_kv_heads, G;
    float scale_log2e;
    int32_t causal;
    int64_t window;           // 0: none
    uint32_t* err;
    float* part;              // partial outputs [slot][rows of a tile][d]
    float2* part_ml;          // their (maximum, sum) [slot][rows of a tile]
    int32_t* tickets;         // kFewTickets a block of k_attend_few, zero between calls
    AttendCut* cuts;          // one a block of k_attend_tc
    int32_t pairs;            // row tiles of all sequences
    int32_t stall;            // failure-detection test: one wait of k_attend_tc that nothing completes; 0 once it ran
    uint64_t wait_ns;
    AttendSpan span[kMaxBatch];
    AttendSeq s[kMaxBatch];
};

// What tokens see of one another's rows (cb_tree), sequence by sequence.
struct TreeBits {
    const uint32_t* seen;     // or null: each those up to itself
    int64_t s_row;
};

// cb_attend_tree: `causal` is 1 and `window` 0.
struct AttendTreeBatch : AttendBatch {
    static constexpr bool kTrees = true;
    TreeBits tree[kMaxBatch];
};

// cb_weigh.  The work is planned as that of tokens that see every row (AttendBatch: causal and window are 0): what
// they see is `sees` (causal), `sees_window` and `tree`.
struct WeighSeq {
    const float* lse;
    const float* before;      // or null
    float* weights;
    int64_t b_head, w_head;
    int64_t fresh;            // rows at the end whose `before` is not read
    TreeBits tree;
};
struct WeighBatch : AttendBatch {
    int32_t sees;
    int32_t sees_window;      // 0: none
    float decay;
    float lse_log2e, lse_log2e_lo;   // scale_log2e / scale, in two parts: log2(e) as the logits' factor has it
    WeighSeq w[kMaxBatch];
};

// cb_evict: the rows of one cache that stay.
struct RankSeq {
    const float* weights;
    int64_t w_layer, w_head;
    int64_t T;
    const int32_t* length;    // or null
    int64_t keep, first, last;
    int32_t* idx;             // [layer][head][keep]
};
struct RankBatch {
    int32_t n;
    int32_t n_layers, n_kv_heads;
    RankSeq s[kMaxBatch];
};

// Rows that move within a cache or into another (cb_evict, cb_keep): row base + j of `to` becomes row base + idx[j]
// of `from`, and so do their weights.
struct MoveSeq {
    PackedRows from, to;      // bases at the call's first layer
    const float* w;           // or null
    float* w_to;
    int64_t w_layer, w_head, t_layer, t_head;
    const int32_t* idx;
    int64_t idx_list;         // entries of a (layer, head); 0: all have the same
    int64_t count;            // entries at most (of lists of their own -1 is none)
    const int32_t* n_kept;    // or null: entries that count
    int64_t T;                // rows of `from`
    const int32_t* length;    // or null
    int64_t drafted;          // base = rows - drafted; -1: 0
    int32_t* left;            // or null: receives base + entries (lists of their own: min(rows, count))
    int32_t left_later;       // not before every group has read `length`
    int32_t in_place;
};
struct MoveBatch {
    int32_t n;
    int32_t n_layers, n_kv_heads;
    uint32_t* err;
    MoveSeq s[kMaxPackBatch];
};

cudaError_t launch_rotary(const RotaryBatch& b, int head_dim, int style, cudaStream_t st, int num_sms);
cudaError_t launch_pack(const PackBatch& b, int head_dim, cudaStream_t st, int num_sms);
cudaError_t launch_unpack(const PackBatch& b, int head_dim, cudaStream_t st, int num_sms);
// Fills in pair0 and pairs, bounds window, launches, and clears stall where the kernel that has it ran.
cudaError_t launch_attend(AttendBatch& b, int head_dim, cudaStream_t st, int num_sms);
cudaError_t launch_attend(AttendTreeBatch& b, int head_dim, cudaStream_t st, int num_sms);
// Fills in pair0 and pairs, and launches.
cudaError_t launch_weigh(WeighBatch& b, int head_dim, cudaStream_t st, int num_sms);
// How k_rank takes a batch: blocks of a list, keys of a block at most, and whether its shared memory holds them all (where it
// does not, there are kRankCluster).
constexpr int kRankKeys = 24 * 1024;         // keys of a block's slice held in shared memory at most (96 KB)
constexpr int kRankCluster = 8;
struct RankPlan {
    int blocks;
    int64_t slice;
    bool held;
};
RankPlan rank_plan(const RankBatch& b);
cudaError_t launch_rank(const RankBatch& b, cudaStream_t st);
cudaError_t launch_move(const MoveBatch& b, int head_dim, cudaStream_t st, int num_sms);
cudaError_t launch_left(const MoveBatch& b, cudaStream_t st);     // those that are left_later, behind every launch_move of a call
// Query rows of partial results that launch_attend may use on num_sms SMs.
int64_t attend_part_rows(int num_sms);
constexpr int kFewBlocksPerSm = 4;   // blocks of k_attend_few an SM holds at most
constexpr int kFewTickets = 3;       // tickets for each: groups of parts that begin in it (two), items that do

}  // namespace cbk
