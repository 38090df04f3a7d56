// Rows that are not simply those of a sequence over all of its keys: a token's
// over a list of blocks, and those of a group of sequences over the blocks that
// they have in common. What the tables say is bounded here, as in us_kv_common.h.
#ifndef UNIONSPARSE_US_KV_OTHERS_H
#define UNIONSPARSE_US_KV_OTHERS_H

#include "us_kv_attend.h"

namespace us_kv {

enum Kind { kWhole, kChosen, kPart, kShared, kRest };

// The last of n ascending numbers that is at most x, or -1, 64 probes at a time: one load for up to 64
// numbers, three for 2^18. By whole wavefronts, with the same arguments in every lane.
__device__ inline int last_at_most(const int32_t *p, int n, int x) {
    const int lane = threadIdx.x & 63;
    int lo = 0, size = n;
    for (;;) {
        const int step = (size + 63) / 64;
        const bool most = lane * step < size && p[lo + lane * step] <= x;
        const int k = __builtin_popcountll(__builtin_amdgcn_ballot_w64(most));
        if (k == 0) return lo - 1;
        lo += (k - 1) * step;
        if (step <= 1) return lo;
        size = min(step, size - (k - 1) * step);
    }
}

// A group's sequences [first, last), their token rows, and the keys that they have in common.
struct Group {
    int first, last, r0, n, cut, number;

    // Keys of the group's that row t sees: none if it is no row of its sequences.
    __device__ int sees(const Seqs &s, const Mask &mask, int t) const {
        int b = t;
        if (s.starts) {
            b = first;
            for (int e = last; e - b > 1;) {
                const int mid = (b + e) >> 1;
                if (s.starts[mid] <= t) b = mid;
                else e = mid;
            }
        }
        if (b < first || b >= last) return 0;
        int r, rows, lo, hi;
        s.rows(b, r, rows);
        if (t < r || t - r >= rows) return 0;
        mask.range(t - r, rows, s.len(b), lo, hi);
        return min(hi, cut);
    }
};

struct Others {
    int32_t batch;
    const int32_t *chosen;                                 // tokens x heads x top
    int32_t top;
    const int32_t *group_starts, *shared;
    int32_t groups, max_group, max_shared;
    // Of kPart: how the keys behind the common ones are split, the workgroups of a launch that take common ones,
    // and whether the last to end joins.
    Split own;
    int32_t pre_groups, inside;
    int32_t pre_shift;                                     // log2 of the rows of a tile over common ones

    // The sequence and position of row t; whether it is a row of the call.
    __device__ bool place(const Seqs &s, int t, int &b, int &at) const {
        b = s.starts ? last_at_most(s.starts, batch, t) : t < batch ? t : -1;
        if (b < 0) return false;
        int r, n;
        s.rows(b, r, n);
        if (t < r || t - r >= n) return false;
        at = s.len(b) - n + (t - r);
        return true;
    }
    // Whether the groups are in order: each sequence is then in one of them at most, and a launch's workgroups
    // agree on which. (Where they are not, nothing is in common.) By whole wavefronts, as the next two.
    __device__ bool ordered() const {
        const int lane = threadIdx.x & 63;
        uint64_t down = 0;
        for (int i = lane; i - lane < groups; i += 64)
            down |= __builtin_amdgcn_ballot_w64(i < groups && group_starts[min(i, groups - 1)] > group_starts[min(i, groups - 1) + 1]);
        return down == 0;
    }
    __device__ Group group(const Seqs &s, int g) const {
        Group x = group_at(s, g);
        if (!ordered()) x.cut = x.n = 0;
        return x;
    }
    __device__ Group group_at(const Seqs &s, int g) const {
        Group x;
        x.number = g;
        x.first = min(max(group_starts[g], 0), batch);
        x.last = min(max(group_starts[g + 1], x.first), (int)min((int64_t)batch, (int64_t)x.first + max_group));
        x.cut = (int)min((int64_t)min(max(shared[g], 0), max_shared) * kBlock, (int64_t)s.max_len);
        x.r0 = s.starts ? s.starts[x.first] : x.first;
        const int64_t n = (int64_t)(s.starts ? s.starts[x.last] : x.last) - x.r0;
        x.n = x.r0 < 0 || x.r0 >= s.tokens
                  ? 0
                  : (int)min(min(max(n, (int64_t)0), (int64_t)max_group * s.max_new), (int64_t)s.tokens - x.r0);
        return x;
    }
    // The group of sequence b; one that has nothing in common for a sequence of none.
    __device__ Group group_of(const Seqs &s, int b) const {
        const int g = last_at_most(group_starts, groups, b);
        if (g >= 0 && ordered()) {
            const Group x = group_at(s, g);
            if (b >= x.first && b < x.last) return x;
        }
        return Group{b, b + 1, 0, 0, 0, 0};
    }
};

}  // namespace us_kv

#endif  // UNIONSPARSE_US_KV_OTHERS_H
