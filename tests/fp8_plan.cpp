// Goes over the plans of the 8-bit layer's host side (fp8_plan.h).
#include <cstdio>
#include <cstdlib>
#include "fp8_plan.h"

using namespace slim;

static int g_seen[9];

static void fail(const char* what, int b, int d_out, int groups, const Fp8Plan& p) {
    std::printf("%s: %d tokens, %d rows, %d groups: kernel %d, %d CTAs\n", what, b, d_out, groups, (int)p.kernel, p.ctas);
    std::exit(1);
}

int main() {
    // what a B200 holds at once, and a part of one
    const int full[4][4] = {{296, 148, 74, 32}, {296, 148, 74, 32}, {148, 74, 37, 16}, {148, 74, 37, 16}};
    const int part[4][4] = {{8, 4, 2, 1}, {8, 4, 2, 1}, {4, 2, 1, 1}, {4, 2, 1, 1}};
    const int tokens[] = {1, 2, 15, 16, 17, 32, 33, 64, 65, 100, 128, 129, 200, 256, 257, 333, 600, 1000, 2048, 4096, 65536, 8388481, 2147483647};
    const int rows[] = {1, 16, 127, 128, 129, 512, 1000, 1024, 4096, 5504, 8192, 13824, 28672, 128256, 2147483647};
    const int columns[] = {1, 2, 3, 4, 14, 16, 32, 64, 108, 224, 1000, 16777216};
    for (int half = 0; half < 2; ++half)
        for (int b : tokens)
            for (int n : rows)
                for (int g : columns) {
                    const auto& clusters = half ? part : full;
                    const Fp8Plan p = fp8_plan(b, n, g, half ? 4 : 148, half ? 2 : 74, clusters);
                    ++g_seen[p.kernel];
                    const bool cluster = p.kernel <= FP8_CLUSTER_128;
                    if (p.ctas != 1 && p.ctas != 2 && p.ctas != 4 && p.ctas != 8) fail("no power of two", b, n, g, p);
                    if (!cluster && p.ctas != 1) fail("a cluster of a kernel without", b, n, g, p);
                    if (p.ctas > g) fail("a CTA without columns", b, n, g, p);
                    const int most[4] = {16, 32, 64, 128};
                    if ((b <= 16) != (p.kernel == FP8_CLUSTER_16) || (b <= 32 && p.kernel > FP8_CLUSTER_32) || (b <= 64 && !cluster)) fail("another kernel than few tokens have", b, n, g, p);
                    if (cluster && p.ctas > 1) {
                        const int i = p.ctas == 2 ? 1 : p.ctas == 4 ? 2 : 3;
                        const long long tiles = (long long)((n + 127ll) / 128) * ((b + most[p.kernel] - 1ll) / most[p.kernel]);
                        if (tiles > clusters[p.kernel][i]) fail("more clusters than are resident", b, n, g, p);
                    }
                    if (cluster && (b + most[p.kernel] - 1ll) / most[p.kernel] > 65535) fail("a grid too high", b, n, g, p);
                }
    for (int k = 0; k < 9; ++k)
        if (!g_seen[k]) { std::printf("no call reaches kernel %d\n", k); return 1; }
    std::printf("ok\n");
}
