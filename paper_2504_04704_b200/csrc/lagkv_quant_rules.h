// Which kernel a call of the attention over caches in 8 bits takes: rules over sizes that the host knows.  Host code that needs no GPU.
#pragma once
#include <cstdint>

namespace lagkv {

// Query rows of the units that a call takes, by the least of
//     base + passes * kv_heads * (S_cap + begin) * (row + D / 128 * channels + (capped ? cap : 0)) * 1e-6 us,
// where `passes` is how many units read a KV head, and beginning a unit costs as much as `begin` rows.  The numbers are fitted to
// the times of all four units (256 channels: 8 and 16 only) in 1540 calls of 4 to 256 query rows to a KV head over 8 x 256 to 16 x 8 x 8192
// and 3 x 2 x 100000 rows, 64 to 256 channels, both formats, with and without a cap; its choice takes 0.4 % longer than the best one on average,
// 3 % of the calls lose more than 5 %, none more than 20.  Some of the times, in us, int8:
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
// Units of 256 rows (int8) read K and V once for two of 128, but have two groups of helpers only and leave CTAs idle where there are few heads: 256 query
// rows of 128 channels over 2 x 8 x 131072 rows in 336 us against 346, 8 x 8 x 32768 343 and 356, 16 x 8 x 16384 357 and 367, but 1 x 8 x 131072 187 and 187,
// 1 x 8 x 32768 71 and 64, 16 x 8 x 8192 213 and 212 (e4m3, 2 x 8 x 131072 rows under half as many: 234 and 205: not built).
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

}  // namespace lagkv
