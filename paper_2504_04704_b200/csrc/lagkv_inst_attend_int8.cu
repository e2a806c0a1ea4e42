// Attention kernels for caches held in 8 bits as int8 codes, every head_dim.
#include "lagkv_attend_quant_tables.h"

namespace lagkv {
namespace {
const AttendEntry kTable[] = {LAGKV_QUANT_ENTRIES(FORM_INT8), LAGKV_QUANT_WIDE_ENTRY(64, FORM_INT8, 2),
                               LAGKV_QUANT_WIDE_ENTRY(96, FORM_INT8, 2), LAGKV_QUANT_WIDE_ENTRY(128, FORM_INT8, 2)};
}  // namespace

int attend_int8_kernels(const AttendEntry** table) {
    *table = kTable;
    return int(sizeof(kTable) / sizeof(kTable[0]));
}
}  // namespace lagkv
