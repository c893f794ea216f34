// Which kernel serves a call of the 8-bit layer (fwd_fp8.cu), as plain C++: the host's side of it, and what the tests go over.
//
// Up to 64 tokens a cluster has 128 rows and cuts the columns: the weight's stream has to be spread over the SMs, and the tokens are the
// MMA's columns, so that no row of it is empty.  The kernels differ in the tile that a CTA, a cluster or a pair has, and from 33 tokens on the
// call takes the one with the shortest time by the longer of
//     fixed + rounds of tiles * groups of 128 columns in a tile's walk * time of a group
//         (rounds * all of it where a CTA ends with its tile, in a cluster)
//     and the tiles' bytes at the 11.7 TB/s that the SMs together got from the L2,
// with the fixed times and times of a group below (ns), fitted to 57 measured sizes (weights in rotation): its choice was the fastest or within
// 1 % of it on 50 of them, and at most 9 % slower.  Some measured, us (tokens, columns -> rows; c: a cluster's tokens, r: a CTA's rows, p: a pair's):
//     40, 8192 -> 1024    c32 6.3, c64 6.9, c128 7.6, r32 17.7
//     64, 5120 -> 13824   c64 16.5, r128 16.8, c32 19.0, c128 20.6, r64 24.0, r32 31.8
//     100, 4096 -> 1024   c32 5.6, c64 6.9, c128 8.2, r32 10.1, r64 10.8, p128 10.9, r128 12.0, p256 15.5
//     100, 8192 -> 8192   r64 20.0, p128 20.5, c128 21.1, c64 21.4, r128 22.3, c32 24.4, p256 27.8, r32 33.6
//     231, 8192 -> 1024   c32 10.0, c64 10.1, c128 12.7, r32 17.9, p128 18.4, r64 18.9, r128 21.0, p256 27.0
//     333, 8192 -> 1024   c128 13.1, c32 14.1, c64 14.4, r32 18.2, p128 18.5, r64 19.0, r128 21.1, p256 27.1
//     4000, 512 -> 512    r128 4.2, r64 4.8, p128 5.2, p256 5.8, r32 6.4, c128 7.5, c32 8.8, c64 9.7
//     333, 8192 -> 8192   p256 31.4, p128 37.5, r128 41.3, r64 52.4, c128 64.2, r32 94.1
//     600, 8192 -> 8192   p128 53.8, p256 59.9, r128 60.7, r64 84.7, r32 140
#pragma once
#include <cmath>

namespace slim {

enum Fp8Kernel { FP8_CLUSTER_16, FP8_CLUSTER_32, FP8_CLUSTER_64, FP8_CLUSTER_128, FP8_ROWS_32, FP8_ROWS_64, FP8_ROWS_128, FP8_PAIR_128, FP8_PAIR_256 };

struct Fp8Plan {
    Fp8Kernel kernel;
    int ctas;              // of a cluster
};

// CTAs that cut the columns of a tile: as many as are resident at once for all tiles, with four groups of columns each at least (their
// exchange takes half a microsecond: 512 -> 512, 8 tokens 3.2 us with two CTAs, 2.7 with one; 1728 -> 5120, one token 5.1 with four, 5.0 with two).
// clusters[i]: clusters of 2^i CTAs resident at once.
inline int fp8_cluster_ctas(long long tiles, int groups, const int (&clusters)[4]) {
    int i = 3;
    while (i > 0 && (tiles > clusters[i] || groups < (4 << i))) --i;
    return 1 << i;
}

// clusters: of the kernel for up to 16, 32, 64 and 128 tokens.
inline Fp8Plan fp8_plan(int b, int d_out, int groups, int sms, int pairs, const int (&clusters)[4][4]) {
    auto up = [](long long a, long long n) { return (a + n - 1) / n; };
    const long long blocks = up(d_out, 128);
    if (b <= 32) return {b <= 16 ? FP8_CLUSTER_16 : FP8_CLUSTER_32, fp8_cluster_ctas(blocks, groups, clusters[b <= 16 ? 0 : 1])};
    // (times are doubles: those of the largest sizes pass 2^63 ns)
    auto feed = [](long long tiles, int groups, int tokens, int rows) { return std::floor((double)tiles * groups * (tokens + rows) * 128 / 11700); };
    Fp8Plan best = {FP8_PAIR_256, 1};
    double least = HUGE_VAL;
    struct Cluster { Fp8Kernel kernel; int tokens; long long alone, together, group; };      // (fixed times of one CTA and of several)
    const Cluster cuts[] = {{FP8_CLUSTER_32, 32, 2250, 3750, 360}, {FP8_CLUSTER_64, 64, 3000, 5000, 300}, {FP8_CLUSTER_128, 128, 4500, 6500, 450}};
    for (const Cluster& k : cuts) {
        const long long parts = up(b, k.tokens), tiles = blocks * parts;
        const int (&resident)[4] = clusters[k.kernel - FP8_CLUSTER_16];
        const int ctas = fp8_cluster_ctas(tiles, groups, resident);
        const long long rounds = up(tiles, resident[ctas == 1 ? 0 : ctas == 2 ? 1 : ctas == 4 ? 2 : 3]);
        const double walk = (double)rounds * ((ctas > 1 ? k.together : k.alone) + up(groups, ctas) * k.group), bytes = feed(tiles, groups, k.tokens, 128);
        const double cost = walk > bytes ? walk : bytes;
        if (cost < least && parts <= 65535) { least = cost; best = {k.kernel, ctas}; }       // (the grid has a row for each part of the tokens)
    }
    if (b <= 64) return best;
    struct Tile { Fp8Kernel kernel; int tokens, rows; long long fixed, group; };
    const Tile kinds[] = {{FP8_ROWS_32, 128, 32, 2400, 240}, {FP8_ROWS_64, 128, 64, 2500, 255}, {FP8_ROWS_128, 128, 128, 3000, 300},
                          {FP8_PAIR_128, 256, 128, 3500, 270}, {FP8_PAIR_256, 256, 256, 4300, 420}};
    for (const Tile& k : kinds) {
        const long long n = up(b, k.tokens) * up(d_out, k.rows);
        const double walk = k.fixed + (double)up(n, k.tokens == 256 ? pairs : sms) * groups * k.group, bytes = k.fixed + feed(n, groups, k.tokens, k.rows);
        const double cost = walk > bytes ? walk : bytes;
        if (cost < least) { least = cost; best = {k.kernel, 1}; }
    }
    return best;
}

}  // namespace slim
