// Host check of the place of a sequence's rows among its group's (us_kv_rules.h): the inline function that the
// kernels of shared attention index partial rows by. Run by tests/test_kv_groups_host.py; prints "ok" or the
// first failing case.
#define __host__
#define __device__
#include <cstdint>
#include <cstdio>
#include <initializer_list>
#include "us_kv_rules.h"

int main() {
    const int32_t at[] = {INT32_MIN, INT32_MIN + 1, -4000, -1, 0, 1, 5, 63, 4000, 1 << 25, INT32_MAX - 1, INT32_MAX};
    const int32_t rows[] = {0, 1, 17, 300, 1 << 25};
    for (int32_t r0 : at)
        for (int32_t first : at)
            for (int32_t G : {1, 3, 71, 65535})
                for (int32_t row : rows)
                    for (int32_t end : rows) {
                        const __int128 want = ((__int128)r0 - first) * G + row;
                        const int got = us_kv::place_of(r0, first, G, row, end);
                        if (got != (want >= 0 && want < end ? (int)want : -1)) {
                            std::printf("FAIL r0=%d first=%d G=%d row=%d end=%d: %d\n", r0, first, G, row, end, got);
                            return 1;
                        }
                    }
    std::printf("ok\n");
    return 0;
}
