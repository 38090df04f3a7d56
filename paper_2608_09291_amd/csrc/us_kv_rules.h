// What the attention kernels decide by whole numbers alone. Used by the kernels
// on the device and by host tests; the including file provides __host__ and
// __device__ (the HIP runtime, or empty definitions in a host build).
#ifndef UNIONSPARSE_US_KV_RULES_H
#define UNIONSPARSE_US_KV_RULES_H

#include <stdint.h>

namespace us_kv {

struct Mask {
    int32_t causal, window;
    // Keys [lo, hi) that query i of n of a sequence of len tokens sees. Both grow with i.
    __host__ __device__ void range(int i, int n, int len, int &lo, int &hi) const {
        lo = 0;
        hi = len;
        if (causal) {
            const int at = len - n + i;
            hi = at < 0 ? 0 : at + 1;
            lo = window > 0 && at >= window ? at - window + 1 : 0;             // (no window is too wide for 32 bits)
        }
    }
};

// How a prompt workgroup passes the blocks of a row tile through its LDS stages:
// block i lies in stage i % stages, keys and values apart. Ahead of step 0 the
// first blocks are staged, then a barrier, then block 0's scores are taken. Step
// i takes the scores of block i + 1 and the values of block i, then stages later
// ones (also past the last block, where nothing takes them any more).
struct StageOrder {
    int stages;
    __host__ __device__ constexpr int ahead() const { return stages == 4 ? 1 : 0; }
    __host__ __device__ constexpr int first_keys() const { return 2 + ahead(); }          // staged ahead of step 0
    __host__ __device__ constexpr int first_values() const { return 1 + ahead(); }
    __host__ __device__ constexpr int puts_keys(int i) const { return i + 2 + ahead(); }  // by step i
    __host__ __device__ constexpr int puts_values(int i) const { return i + 1 + ahead(); }
    // With four stages a barrier serves two steps, and comes after the even ones: step 1 stages over block 0's
    // keys, and with the barrier of step 0 every wavefront has taken their scores by then. With two stages it
    // is step 0 that does, hence the barrier after those scores.
    __host__ __device__ constexpr bool barrier_after_first() const { return ahead() == 0; }
    __host__ __device__ constexpr bool barrier_after(int i) const { return ahead() == 0 || i % 2 == 0; }
};

}  // namespace us_kv

#endif  // UNIONSPARSE_US_KV_RULES_H
