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

// A group's sequences [first, last), their token rows, and the keys that they have in common. A lane has the
// first row, the number of rows and the length of a sequence of the first 64.
struct Group {
    int first, last, r0, n, cut, number;
    int my_r0, my_n, my_len;

    // Keys of the group's that row t sees: none if it is no row of its sequences. By whole wavefronts.
    __device__ int sees(const Seqs &s, const Mask &mask, int t) const {
        int r, rows, len, lo, hi;
        if (last - first <= 64) {
            int at = 0;                                    // the last that begins at t or before
#pragma unroll
            for (int step = 32; step > 0; step >>= 1) {
                const int r1 = __shfl(my_r0, at + step, 64);
                at = at + step < last - first && r1 <= t ? at + step : at;
            }
            r = __shfl(my_r0, at, 64);
            rows = __shfl(my_n, at, 64);
            len = __shfl(my_len, at, 64);
        } else {
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
            s.rows(b, r, rows);
            len = s.len(b);
        }
        if (t < r || t - r >= rows) return 0;
        mask.range(t - r, rows, len, lo, hi);
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
    // What all of a launch's workgroups read of the groups; by whole wavefronts. Up to 64 groups come in one
    // load, a lane each. Whether they are in order: each sequence is then in one of them at most, and the
    // workgroups agree on which. (Where they are not, nothing is in common.)
    struct Table {
        int start, end, shared;                            // this lane's
        bool ordered;
    };
    __device__ Table table() const {
        const int lane = threadIdx.x & 63;
        Table t;
        t.start = group_starts[min(lane, groups)];
        t.end = group_starts[min(lane + 1, groups)];
        t.shared = shared[min(lane, groups - 1)];
        uint64_t down = __builtin_amdgcn_ballot_w64(t.start > t.end);
        for (int i = lane + 64; i - lane < groups; i += 64)
            down |= __builtin_amdgcn_ballot_w64(i < groups && group_starts[min(i, groups - 1)] > group_starts[min(i, groups - 1) + 1]);
        t.ordered = down == 0;
        return t;
    }
    // Group g's sequences and keys in common.
    __device__ Group sequences(const Seqs &s, const Table &t, int g) const {
        int a, z, c;
        if (groups <= 64) {
            a = __builtin_amdgcn_readlane(t.start, g);
            z = __builtin_amdgcn_readlane(t.end, g);
            c = __builtin_amdgcn_readlane(t.shared, g);
        } else {
            a = group_starts[g];
            z = group_starts[g + 1];
            c = shared[g];
        }
        Group x;
        x.number = g;
        x.first = min(max(a, 0), batch);
        x.last = min(max(z, x.first), (int)min((int64_t)batch, (int64_t)x.first + max_group));
        x.cut = t.ordered ? (int)min((int64_t)min(max(c, 0), max_shared) * kBlock, (int64_t)s.max_len) : 0;
        return x;
    }
    // And their rows.
    __device__ void rows_of(const Seqs &s, Group &x) const {
        const int b = x.first + (threadIdx.x & 63);
        int next = b + 1;
        x.my_r0 = b;
        x.my_n = x.my_len = 0;
        if (b < x.last) {
            if (s.starts) {
                x.my_r0 = s.starts[b];
                next = s.starts[b + 1];
            }
            x.my_len = s.len(b);
        }
        x.r0 = __builtin_amdgcn_readlane(x.my_r0, 0);
        int end = x.last;
        if (s.starts) end = x.last - x.first <= 64 ? __builtin_amdgcn_readlane(next, max(x.last - x.first - 1, 0)) : s.starts[x.last];
        if (b < x.last) x.my_n = s.bounded(x.my_r0, next - x.my_r0);
        const int64_t n = x.first < x.last ? (int64_t)end - x.r0 : 0;
        x.n = x.r0 < 0 || x.r0 >= s.tokens
                  ? 0
                  : (int)min(min(max(n, (int64_t)0), (int64_t)max_group * s.max_new), (int64_t)s.tokens - x.r0);
    }
    __device__ Group group(const Seqs &s, int g) const {
        Group x = sequences(s, table(), g);
        rows_of(s, x);
        return x;
    }
    // The group of sequence b, without its rows; one that has nothing in common for a sequence of none.
    __device__ Group group_of(const Seqs &s, int b) const {
        const Table t = table();
        const int g = groups <= 64 ? __builtin_popcountll(__builtin_amdgcn_ballot_w64((int)(threadIdx.x & 63) < groups && t.start <= b)) - 1
                                   : last_at_most(group_starts, groups, b);
        if (g >= 0) {
            const Group x = sequences(s, t, g);
            if (b >= x.first && b < x.last) return x;
        }
        return Group{b, b + 1, 0, 0, 0, 0, 0, 0, 0};
    }
};

}  // namespace us_kv

#endif  // UNIONSPARSE_US_KV_OTHERS_H
