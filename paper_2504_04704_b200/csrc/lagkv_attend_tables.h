// Table of the compiled attention kernels (one translation unit per storage format).
#pragma once
#include "lagkv_attend_kernels.cuh"

namespace lagkv {

typedef void (*attend_kernel_t)(const AttendParams);

struct AttendEntry {
    int D, dtype;
    int rows;     // query rows of a unit
    int threads, ctas_per_sm;
    size_t smem;
    attend_kernel_t fn;
};

// each returns the number of entries and sets *table
int attend_bf16_kernels(const AttendEntry** table);
int attend_fp16_kernels(const AttendEntry** table);
int attend_fp8_kernels(const AttendEntry** table);

#define LAGKV_ATTEND_ENTRY(D, DT, MT) \
    { D, DT, AttendGeo<D, DT, MT>::MR, AttendGeo<D, DT, MT>::NT, AttendGeo<D, DT, MT>::CTAS, \
      size_t(AttendGeo<D, DT, MT>::SMEM), &lagkv_attend_kernel<D, DT, MT> }
#define LAGKV_ATTEND_ENTRIES(DT) \
    LAGKV_ATTEND_ENTRY(64, DT, 1), LAGKV_ATTEND_ENTRY(96, DT, 1), LAGKV_ATTEND_ENTRY(128, DT, 1), \
    LAGKV_ATTEND_ENTRY(256, DT, 1), LAGKV_ATTEND_ENTRY(64, DT, 2), LAGKV_ATTEND_ENTRY(96, DT, 2), \
    LAGKV_ATTEND_ENTRY(128, DT, 2)

}  // namespace lagkv
