// Table of the compiled attention kernels over caches in 8 bits (one translation unit per code format).
#pragma once
#include "lagkv_attend_quant_kernels.cuh"
#include "lagkv_attend_quant_wide_kernel.cuh"
#include "lagkv_attend_tables.h"

namespace lagkv {

// dtype: the code format
int attend_int8_kernels(const AttendEntry** table);
int attend_e4m3_kernels(const AttendEntry** table);

#define LAGKV_QUANT_ENTRY(D, FORM, NQ) \
    { D, FORM, QuantGeo<D, FORM, NQ>::MR, false, size_t(QuantGeo<D, FORM, NQ>::MR) * (D + 2), QuantGeo<D, FORM, NQ>::NT, \
      QuantGeo<D, FORM, NQ>::CTAS, size_t(QuantGeo<D, FORM, NQ>::SMEM), \
      reinterpret_cast<const void*>(&lagkv_attend_quant_kernel<D, FORM, NQ, false>), \
      reinterpret_cast<const void*>(&lagkv_attend_quant_merge_kernel<D, FORM, NQ>), kMergeWarps, kMergeWarps * 32, \
      reinterpret_cast<const void*>(&lagkv_attend_quant_kernel<D, FORM, NQ, true>) }
#define LAGKV_QUANT_WIDE_ENTRY(D, FORM, MT) \
    { D, FORM, MT * kWideTile, true, size_t(QuantWideGeo<D, FORM, MT>::PSIZE), QuantWideGeo<D, FORM, MT>::NT, 1, \
      size_t(QuantWideGeo<D, FORM, MT>::SMEM), reinterpret_cast<const void*>(&lagkv_attend_quant_wide_kernel<D, FORM, MT>), \
      reinterpret_cast<const void*>(&lagkv_attend_quant_join_kernel<D, FORM, MT>), kJoinRows, kJoinThreads }
#define LAGKV_QUANT_ENTRIES(FORM) \
    LAGKV_QUANT_ENTRY(64, FORM, 1), LAGKV_QUANT_ENTRY(64, FORM, 2), LAGKV_QUANT_ENTRY(64, FORM, 4), \
    LAGKV_QUANT_ENTRY(96, FORM, 1), LAGKV_QUANT_ENTRY(96, FORM, 2), LAGKV_QUANT_ENTRY(96, FORM, 4), \
    LAGKV_QUANT_ENTRY(128, FORM, 1), LAGKV_QUANT_ENTRY(128, FORM, 2), LAGKV_QUANT_ENTRY(128, FORM, 4), \
    LAGKV_QUANT_ENTRY(256, FORM, 1), LAGKV_QUANT_ENTRY(256, FORM, 2), \
    LAGKV_QUANT_WIDE_ENTRY(64, FORM, 1), LAGKV_QUANT_WIDE_ENTRY(96, FORM, 1), LAGKV_QUANT_WIDE_ENTRY(128, FORM, 1)

}  // namespace lagkv
