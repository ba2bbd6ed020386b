// The division and the row lookup of the paged cache (csrc/moa_kv_device.h), on the host.  Run by test_kv_rows.py.
#include "moa_kv_device.h"

#include <stdio.h>

#include <random>
#include <vector>

int main()
{
    std::mt19937 g(1);
    long bad = 0;
    auto check = [&](uint32_t n, uint32_t d) { bad += moa::FastDiv(d)(n) != n / d; };
    for (uint32_t d = 1; d < 3000; ++d)
        for (uint32_t q : {0u, 1u, 2u, 1000u, 0x7fffffffu / d})
            for (int e = -1; e <= 1; ++e) {
                const int64_t n = (int64_t)q * d + e;
                if (n >= 0 && n <= 0x7fffffff) check((uint32_t)n, d);
            }
    for (int s = 0; s < 31; ++s)
        for (int e = -1; e <= 1; ++e) {
            const int64_t d = (1ll << s) + e;
            if (d < 1) continue;
            for (int i = 0; i < 2000; ++i) check(g() & 0x7fffffffu, (uint32_t)d);
            check(0x7fffffffu, (uint32_t)d);
        }
    for (int i = 0; i < 2000000; ++i) check(g() & 0x7fffffffu, (g() & 0x7fffffffu) >> (g() % 31) | 1u);
    if (bad) printf("%ld wrong quotients\n", bad);

    // pages that do not exist give no row, whatever their number; all others one inside the pool
    const int32_t ids[] = {0, 9, 10, -1, INT32_MIN, INT32_MAX, 1 << 30, 4};
    std::vector<int32_t> table(ids, ids + 8), len(2, 0);
    moa_kv_cache_t c = {MOA_BF16, 3, 64, 2, 10, 7, 4, (void *)256, (void *)256, table.data(), len.data(), nullptr, nullptr, nullptr};
    const moa::KvDev d(c, nullptr);
    for (int b = 0; b < 2; ++b)
        for (int h = 0; h < 3; ++h)
            for (int s = 0; s < d.cap; ++s) {
                const int id = ids[b * 4 + s / 7], want = id >= 0 && id < 10 ? (id * 3 + h) * 7 + s % 7 : -1;
                if (d.row(b, h, s) != want || want >= 10 * 3 * 7) {
                    printf("row(%d, %d, %d) = %d, not %d\n", b, h, s, d.row(b, h, s), want);
                    ++bad;
                }
            }
    puts(bad ? "failed" : "ok");
    return bad != 0;
}
