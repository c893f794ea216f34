// Which kernel serves a call of the 8-bit layer (fwd_fp8.cu), as plain C++: the host's side of it, and what the tests go over.
//
// Up to 64 tokens a cluster has 128 rows and cuts the columns: the weight's stream has to be spread over the SMs, and the tokens are the
// MMA's columns, so that no row of it is empty.  Above, the kernels differ in the tile that a CTA or a pair has, and the call takes the one
// with the shortest time by
//     fixed + the longer of  rounds of tiles * groups of 128 columns in a tile's walk * time of a group
//                       and  the tiles' bytes at the 11.7 TB/s that the SMs together got from the L2,
// with the measured fixed times and times of a group below (ns, weights in rotation).  Measured against it, us (tokens, columns -> rows):
//     100, 8192 -> 8192   tiles of 64 rows 20.1, cluster 20.2, pairs of 128 rows 20.7, 128 rows 22.3, pairs of 256 28.4, 32 rows 33.7
//     100, 5120 -> 13824  128 rows 17.1, cluster 20.3, pairs of 256 20.8, 64 rows 24.4, pairs of 128 24.4, 32 rows 31.7
//     333, 8192 -> 1024   cluster 12.9, 32 rows 18.8, pairs of 128 19.1, 64 rows 19.6, 128 rows 21.1, pairs of 256 27.6
//     333, 8192 -> 8192   pairs of 256 31.4, pairs of 128 37.5, 128 rows 41.3, 64 rows 52.4, cluster 64.2, 32 rows 94.1
//     600, 8192 -> 8192   pairs of 128 rows 53.8, pairs of 256 59.9, 128 rows 60.7, 64 rows 84.7, 32 rows 140
//     4000, 512 -> 512    128 rows 4.2, 64 rows 5.0, pairs of 128 5.3, pairs of 256 5.9, 32 rows 6.6
#pragma once

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
    if (b <= 64) {
        const int i = b <= 16 ? 0 : b <= 32 ? 1 : 2;
        return {(Fp8Kernel)(FP8_CLUSTER_16 + i), fp8_cluster_ctas(blocks, groups, clusters[i])};
    }
    const long long tiles = blocks * up(b, 128);
    const int ctas = fp8_cluster_ctas(tiles, groups, clusters[3]);
    Fp8Plan best = {FP8_CLUSTER_128, ctas};          // (its grid has a row for 128 tokens)
    long long least = up(b, 128) > 65535 ? (1ll << 62) : (ctas > 1 ? 6500 : 3000) + up(tiles, clusters[3][ctas == 1 ? 0 : ctas == 2 ? 1 : ctas == 4 ? 2 : 3]) * up(groups, ctas) * 440;
    struct Tile { Fp8Kernel kernel; int tokens, rows; long long fixed, group; };
    const Tile kinds[] = {{FP8_ROWS_32, 128, 32, 3200, 230}, {FP8_ROWS_64, 128, 64, 3200, 250}, {FP8_ROWS_128, 128, 128, 3000, 300},
                          {FP8_PAIR_128, 256, 128, 3500, 270}, {FP8_PAIR_256, 256, 256, 4300, 420}};
    for (const Tile& k : kinds) {
        const long long n = up(b, k.tokens) * up(d_out, k.rows);
        const long long walk = up(n, k.tokens == 256 ? pairs : sms) * groups * k.group, feed = (long long)((double)n * groups * (k.tokens + k.rows) * 128 / 11700);
        const long long cost = k.fixed + (walk > feed ? walk : feed);
        if (cost < least) { least = cost; best = {k.kernel, 1}; }
    }
    return best;
}

}  // namespace slim
