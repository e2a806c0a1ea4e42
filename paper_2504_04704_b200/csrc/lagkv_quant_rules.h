// Which kernel a call of the attention over caches in 8 bits takes: rules over sizes that the host knows.  Host code that needs no GPU.
#pragma once
#include <cstdint>

namespace lagkv {

// Query rows of the units that a call takes, by the least of
//     base + passes * kv_heads * (S_cap + begin) * (row + D / 128 * channels + (capped ? cap : 0)) * 1e-6 us,
// where `passes` is how many units read a KV head, and beginning a unit costs as much as `begin` rows.  The numbers are fitted to
// the times of all four units (256 channels: 8 and 16 only) in 1540 calls of 4 to 256 query rows to a KV head over 8 x 256 to
// 16 x 8 x 8192 and 3 x 2 x 100000 rows, 64 to 256 channels, both formats, with and without a cap; its choice takes 0.4 % longer than
// the best one on average, 3 % of the calls lose more than 5 %, none more than 20.  Some of the times, in us, int8:
//     KV heads x rows, channels, query rows    8       16       32      128
//     1 x 8 x 256      128        16          9.5     10.6     11.7     14.1
//     16 x 8 x 8192    128        16         87.4     60.8     81.8    106.2
//     6 x 4 x 16411    128        20         52.9     47.0     40.3     53.7
//     6 x 4 x 16411    64         35         55.7     43.9     45.5     44.4
//     the same, capped                       63.5     52.9     58.3     88.5
//     6 x 4 x 16411    128        35         80.8     63.6     64.8     53.3
//     the same, capped                       88.9     72.6     78.2     96.7
//     16 x 8 x 8192    128        64        325.2    220.0    173.1    117.4
//     the same, capped                      350.3    241.5    194.2    234.4
//     64 x 8 x 512     128        35         90.3     78.0     80.2     50.5
// Units of 256 rows (int8) read K and V once for two of 128, but have two groups of helpers only and leave CTAs idle where there are
// few heads: 256 query rows of 128 channels over 2 x 8 x 131072 rows in 336 us against 346, 8 x 8 x 32768 343 and 356, 16 x 8 x 16384
// 357 and 367, but 1 x 8 x 131072 187 and 187, 1 x 8 x 32768 71 and 64, 16 x 8 x 8192 213 and 212 (e4m3, 2 x 8 x 131072 rows under
// half as many: 234 and 205: not built).
inline int quant_unit_rows(int64_t kv_heads, int D, bool int8, int query_rows, int64_t S_cap, bool capped) {
    if (int8 && query_rows > 128 && D <= 128 && S_cap >= 16384 && kv_heads * S_cap >= 1500000) return 256;
    struct Cost {
        int rows;
        double base, row, channels, cap, begin;
    };
    static const Cost costs[4] = {
        {8, 9.3, 7.3, 27.5, 3.4, 448},
        {16, 10.7, 8.0, 38.7, 4.8, 488},
        {32, 13.3, 18.7, 42.8, 15.0, 496},
        {128, 19.3, 54.3, 41.6, 93.8, 200},
    };
    int best = 0;
    double least = 0.0;
    for (const Cost& c : costs) {
        if (D > 128 && c.rows > 16) break;
        const double passes = (query_rows + c.rows - 1) / c.rows, rows = double(kv_heads) * (double(S_cap) + c.begin) * 1e-6;
        const double time = c.base + passes * rows * (c.row + D / 128.0 * c.channels + (capped ? c.cap : 0.0));
        if (best == 0 || time < least) {
            best = c.rows;
            least = time;
        }
    }
    return best;
}

// CTAs of a unit's cluster, where a call of units of 8 or 16 query rows takes that form (1: it does not): one launch instead of two,
// and every unit gets the same CTAs whatever its length.  In us, int8, 128 channels, 4 query rows to a KV head, without and in clusters
// of 4, 8, 16:
//     1 x 8 heads x 256 rows   7.9   6.2   6.2   7.5      4 x 8 x 256    8.5   6.5   7.0  20.4
//     1 x 8 x 1216             9.1   8.1   7.4   7.9      4 x 8 x 1216  10.4   8.6   8.6  20.8
//     1 x 8 x 4096            11.1  13.0   9.6   9.4      4 x 8 x 4096  14.0  13.5  11.7  25.7
//     1 x 8 x 20000           17.3  41.3  23.9  19.9      8 x 8 x 256    9.1   7.1  12.9
//     1 x 4 x 1216             8.7   8.1   7.3   6.8      8 x 8 x 1216  12.5   9.9  15.7
// So: as long as all clusters are on the GPU at once (`fits`: of each size, as the runtime says for the kernel and the device; 0:
// none), and up to 640 rows a CTA, above which equal shares of all rows win.  More than four clusters of 16 begin later.  Over one
// to 64 heads, 64 to 10240 rows and 64 to 256 channels the size taken is 0.1 % behind the best one on average.
constexpr int kClusterSizes = 3, kClusterCtas[kClusterSizes] = {4, 8, 16};
inline int quant_cluster_ctas(int64_t units, int64_t S_cap, const int (&fits)[kClusterSizes]) {
    const int most[kClusterSizes] = {256, 256, 128};  // CTAs in all that were measured as worth it on 148 SMs
    const double base[kClusterSizes] = {6.0, 6.3, 6.6}, each[kClusterSizes] = {0.0, 0.0, 0.0133};  // us; and for each CTA from the 65th on
    int best = 1;
    double least = 0.0;
    for (int i = 0; i < kClusterSizes; ++i) {
        const double rows = double(S_cap) / kClusterCtas[i];
        if (units > fits[i] || units * kClusterCtas[i] > most[i] || rows > 640.0) continue;
        const double more = double(units * kClusterCtas[i] - 64), time = base[i] + (more > 0.0 ? each[i] * more : 0.0) + rows * 7e-3;
        if (best > 1 && time >= least) continue;
        best = kClusterCtas[i];
        least = time;
    }
    return best;
}

}  // namespace lagkv
