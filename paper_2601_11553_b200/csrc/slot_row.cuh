// Where a prompt's slot lies in the pools.
#pragma once
#include "kernels.h"
#include "ptx.cuh"

namespace pc {

// Pool row of a prompt's slot, or -1 when it lies outside the pool.
__device__ __forceinline__ int64_t slot_row(const int32_t* page_table, int pt_stride, const int32_t* start, int64_t n_slots,
                                            int b, int slot) {
  const int64_t r = page_table ? static_cast<int64_t>(ld_dep_s32(page_table + static_cast<size_t>(b) * pt_stride + slot / PAGE_TOKENS)) * PAGE_TOKENS + slot % PAGE_TOKENS
                               : static_cast<int64_t>(ld_dep_s32(start + b)) + slot;
  return r >= 0 && r < n_slots ? r : -1;
}

}  // namespace pc
