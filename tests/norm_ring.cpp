// norm_ring() for every row length that the resident norm kernel takes: its blocks have to be on the SM at once.
#include <cstdio>

#include "../paper_1908_11263_gb300/csrc/block_internal.h"

int main()
{
    using namespace qnn;
    int fails = 0, rows = 0;
    const int kinds[4][2] = {{2, 0}, {2, 2}, {2, 4}, {4, 4}};  // bytes of an element of x and of the residual
    for (const auto &kind : kinds)
        for (int d = 8; d <= 16384; d += 8, ++rows) {
            const NormRing r = norm_ring(d, d * kind[0], d * kind[1]);
            const unsigned stage = d * (kind[0] + kind[1]);
            const unsigned block = (kNormStatic + r.smem + 127) / 128 * 128 + 1024;  // what a block takes of an SM's 228 KB
            const bool taken = r.stages >= 2;
            bool ok = r.per_sm >= 1 && r.threads % 32 == 0 && r.threads >= 64 && r.threads <= 1024 && r.threads * 16 >= d &&
                      r.per_sm * r.threads <= 1024 && r.stages <= 4 && r.smem == r.stages * stage;
            if (taken) ok = ok && r.per_sm * block <= 228 * 1024 && r.smem <= kNormRoom;
            if (!taken) ok = ok && r.per_sm == 1 && 2 * stage > kNormRoom;  // left to the other kernel for want of room only
            if (!ok) {
                ++fails;
                std::printf("d=%d bytes %d+%d: %d blocks of %u bytes (%d stages), %d threads\n", d, kind[0], kind[1], r.per_sm, block,
                            r.stages, r.threads);
            }
        }
    std::printf("rows=%d fails=%d\n", rows, fails);
    return fails != 0;
}
