// Attention kernels for caches held in 8 bits as e4m3 codes, every head_dim.
#include "lagkv_attend_quant_tables.h"

namespace lagkv {
namespace {
const AttendEntry kTable[] = {LAGKV_QUANT_ENTRIES(FORM_E4M3)};
}  // namespace

int attend_e4m3_kernels(const AttendEntry** table) {
    *table = kTable;
    return int(sizeof(kTable) / sizeof(kTable[0]));
}
}  // namespace lagkv
