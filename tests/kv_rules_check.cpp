// Host check of what the attention kernels decide by whole numbers
// (us_kv_rules.h): the same inline functions the kernels use, compiled for the
// host. Run by tests/test_kv_rules_host.py; prints "ok" or the first failing case.
#define __host__
#define __device__
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <initializer_list>
#include "us_kv_rules.h"

using namespace us_kv;

// Wavefronts run freely between two barriers: what one reads must have been staged before the last
// barrier, and nothing is staged over what another may read between the same two.
struct Slots {
    int block[8], put[8], read[8];                         // block that a stage holds; interval of the last access
    Slots() {
        for (int s = 0; s < 8; ++s) block[s] = put[s] = read[s] = -1;
    }
    bool stage(int b, int stages, int interval) {
        const int s = b % stages;
        const bool ok = read[s] < interval && put[s] < interval;
        block[s] = b;
        put[s] = interval;
        return ok;
    }
    bool take(int b, int stages, int interval) {
        const int s = b % stages;
        read[s] = interval;
        return block[s] == b && put[s] < interval;
    }
};

static bool stages_are_sound(int stages, int count) {
    const StageOrder o{stages};
    Slots k, v;
    int interval = 0;
    bool ok = true;
    for (int z = 0; z < o.first_keys(); ++z) ok = k.stage(z, stages, interval) && ok;
    for (int z = 0; z < o.first_values(); ++z) ok = v.stage(z, stages, interval) && ok;
    ++interval;
    ok = k.take(0, stages, interval) && ok;
    if (o.barrier_after_first()) ++interval;
    for (int i = 0; i < count && ok; ++i) {
        if (i + 1 < count) ok = k.take(i + 1, stages, interval) && ok;
        ok = v.take(i, stages, interval) && ok;
        ok = k.stage(o.puts_keys(i), stages, interval) && ok;
        ok = v.stage(o.puts_values(i), stages, interval) && ok;
        if (!ok) std::printf("FAIL stages=%d count=%d: step %d\n", stages, count, i);
        if (o.barrier_after(i)) ++interval;
    }
    return ok;
}

static int stages() {
    for (int n : {2, 4})
        for (int count = 1; count <= 40; ++count)
            if (!stages_are_sound(n, count)) return 1;
    return 0;
}

// The keys that a query sees, against the definition in 64 bits: positions up to its own, the last `window` of them.
static int masks() {
    const int lens[] = {0, 1, 2, 50, 64, 4000, 1 << 28}, counts[] = {1, 2, 80, 5000, 1 << 25};
    const int windows[] = {0, 1, 2, 49, 50, 64, 4001, 1 << 28, INT32_MAX - 2, INT32_MAX - 1, INT32_MAX};
    for (int len : lens)
        for (int n : counts)
            for (int window : windows)
                for (int causal = window ? 1 : 0; causal <= 1; ++causal)
                    for (int i : {0, 1, n / 2, n - 2, n - 1}) {
                        if (i < 0 || i >= n) continue;
                        const int64_t at = (int64_t)len - n + i;
                        int64_t from = causal && window ? at - window + 1 : 0, end = causal ? at + 1 : len;
                        from = from < 0 ? 0 : from;
                        end = end < 0 ? 0 : end;
                        int lo, hi;
                        Mask{causal, window}.range(i, n, len, lo, hi);
                        if (lo != from || hi != end) {
                            std::printf("FAIL len=%d n=%d window=%d causal=%d i=%d: [%d, %d)\n", len, n, window, causal, i, lo, hi);
                            return 1;
                        }
                    }
    return 0;
}

int main(int argc, char **argv) {
    int r = 1;
    if (argc == 2 && !std::strcmp(argv[1], "stages")) r = stages();
    if (argc == 2 && !std::strcmp(argv[1], "masks")) r = masks();
    if (r == 0) std::printf("ok\n");
    return r;
}
