// Attention kernels for fp8 caches, every head_dim.
#include "lagkv_attend_tables.h"

namespace lagkv {
namespace {
const AttendEntry kTable[] = {LAGKV_ATTEND_ENTRIES(2)};
}  // namespace

int attend_fp8_kernels(const AttendEntry** table) {
    *table = kTable;
    return int(sizeof(kTable) / sizeof(kTable[0]));
}
}  // namespace lagkv
