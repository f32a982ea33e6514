// What the roles of a tcgen05 kernel over packed rows share: bounded waits on one another and the layout of operands.
// Ctl is a kernel's control block in shared memory, of which `abort` and `wait_ns` are used here.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "cb_internal.cuh"
#include "cb_sm100_attend.cuh"

namespace cbk {

constexpr uint32_t kPollNs = 1000000u;
constexpr uint64_t kDrainNs = 1000000000ull;

__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

// Bounded wait: false when it gave up or another role did (bits 8 + tag of the error word name the wait).
// (Inline: a call would have to do with the registers of every role.)  SLEEP: nanoseconds between looks.
template <int SLEEP, class Ctl>
__device__ __forceinline__ bool poll(uint64_t* bar, uint32_t parity, Ctl* c, uint32_t* err, int tag) {
    const uint64_t t0 = now_ns();
    do {
        if (SLEEP ? sm100::mbar_try_wait(bar, parity) : sm100::mbar_try_wait_hint(bar, parity, kPollNs)) return true;
        if (SLEEP) __nanosleep(SLEEP);
        if (*reinterpret_cast<volatile int*>(&c->abort)) return false;
    } while (now_ns() - t0 <= c->wait_ns);
    *reinterpret_cast<volatile int*>(&c->abort) = 1;
    atomicOr(err, kErrTimeout | (1u << (8 + tag)));
    return false;
}
template <int SLEEP = 0, class Ctl>
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, Ctl* c, uint32_t* err, int tag) {
    return sm100::mbar_try_wait(bar, parity) || poll<SLEEP>(bar, parity, c, err, tag);
}
// The same for a whole warp, which stays together whatever its lanes saw.
template <int SLEEP = 0, class Ctl>
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, Ctl* c, uint32_t* err, int tag) {
    return __all_sync(0xFFFFFFFFu, wait<SLEEP>(bar, parity, c, err, tag));
}
__device__ __forceinline__ void drain(uint64_t* bar, uint32_t parity) {
    const uint64_t t0 = now_ns();
    while (!sm100::mbar_try_wait(bar, parity))
        if (now_ns() - t0 > kDrainNs) return;
}

__device__ __forceinline__ uint64_t desc(uint32_t lo, uint32_t hi) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"(hi));
    return d;
}

// A 16-byte piece of a K-major operand with 128-byte rows (64 elements a block): row, piece 0..7 of block.
__device__ __forceinline__ uint32_t piece(int block, int rows, int row, int p) {
    return (uint32_t)(block * rows * 128 + row * 128 + ((p ^ (row & 7)) << 4));
}

__device__ __forceinline__ void st_piece(uint8_t* base, uint32_t at, const uint32_t (&w)[4]) {
    *reinterpret_cast<uint4*>(base + at) = make_uint4(w[0], w[1], w[2], w[3]);
}

}  // namespace cbk
