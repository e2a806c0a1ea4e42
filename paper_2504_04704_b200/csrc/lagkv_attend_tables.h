// Table of the compiled attention kernels (one translation unit per storage format).
#pragma once
#include "lagkv_attend_kernels.cuh"
#include "lagkv_attend_wide_kernel.cuh"

namespace lagkv {

struct AttendEntry {
    int D, dtype;
    int rows;     // query rows of a unit
    bool wide;    // tensor memory kernel: whole sequences only, no block choice
    size_t partial_words;  // floats of one partial result
    int threads, ctas_per_sm;
    size_t smem;
    const void* fn;
    const void* join;  // launched behind it, for the units that several CTAs share, and the rows that a CTA takes
    int join_rows, join_threads;
    const void* cluster = nullptr;  // the form with a cluster of CTAs for each unit, if there is one
};

// each returns the number of entries and sets *table
int attend_bf16_kernels(const AttendEntry** table);
int attend_fp16_kernels(const AttendEntry** table);
int attend_fp8_kernels(const AttendEntry** table);

#define LAGKV_ATTEND_ENTRY(D, DT, MT) \
    { D, DT, AttendGeo<D, DT, MT>::MR, false, size_t(AttendGeo<D, DT, MT>::MR) * (D + 2), AttendGeo<D, DT, MT>::NT, \
      AttendGeo<D, DT, MT>::CTAS, \
      size_t(AttendGeo<D, DT, MT>::SMEM), reinterpret_cast<const void*>(&lagkv_attend_kernel<D, DT, MT>), \
      reinterpret_cast<const void*>(&lagkv_attend_merge_kernel<D, DT, MT>), kMergeWarps, kMergeWarps * 32 }
#define LAGKV_WIDE_ENTRY(D, DT, MT) \
    { D, DT, MT * kWideTile, true, size_t(WideGeo<D, DT, MT>::PSIZE), WideGeo<D, DT, MT>::NT, 1, \
      size_t(WideGeo<D, DT, MT>::SMEM), reinterpret_cast<const void*>(&lagkv_attend_wide_kernel<D, DT, MT>), \
      reinterpret_cast<const void*>(&lagkv_attend_join_kernel<D, DT, MT>), kJoinRows, kJoinThreads }
#define LAGKV_ATTEND_ENTRIES(DT) \
    LAGKV_ATTEND_ENTRY(64, DT, 1), LAGKV_ATTEND_ENTRY(96, DT, 1), LAGKV_ATTEND_ENTRY(128, DT, 1), \
    LAGKV_ATTEND_ENTRY(256, DT, 1), LAGKV_ATTEND_ENTRY(64, DT, 2), LAGKV_ATTEND_ENTRY(96, DT, 2), \
    LAGKV_ATTEND_ENTRY(128, DT, 2), LAGKV_WIDE_ENTRY(64, DT, 1), LAGKV_WIDE_ENTRY(96, DT, 1), LAGKV_WIDE_ENTRY(128, DT, 1), \
    LAGKV_WIDE_ENTRY(64, DT, 2), LAGKV_WIDE_ENTRY(96, DT, 2), LAGKV_WIDE_ENTRY(128, DT, 2)

}  // namespace lagkv
