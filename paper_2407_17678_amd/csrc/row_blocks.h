// Internal: the kept blocks of one row of a head's mask as the decode kernels walk them, in closed form or from a layout's lists.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "kernels.h"

namespace s2 {

// Kept blocks of block row i, in ascending order, as (stripe run, local run), or as a list.
struct RowBlocks {
  int first_stripe, n_stripe, stride, local_lo, count;
  const int32_t* cols;  // caller-supplied pattern: the row's list; nullptr = closed form
  __device__ int block(int n) const {
    const int striped = first_stripe + n * stride, local = local_lo + (n - n_stripe);
    if (cols) return load_const<int32_t>(cols + n);
    return n < n_stripe ? striped : local;
  }
  // the same for an n that is a lane's own
  __device__ int block_of_lane(int n) const {
    const int striped = first_stripe + n * stride, local = local_lo + (n - n_stripe);
    if (cols) return cols[n];
    return n < n_stripe ? striped : local;
  }
};

template <class PARAMS>
__device__ inline RowBlocks row_blocks(const PARAMS& p, int head, int i) {
  RowBlocks r;
  r.stride = p.stride;
  r.first_stripe = 0;
  r.n_stripe = 0;
  r.cols = nullptr;
  r.local_lo = 0;
  if (p.row_ptr) {
    const int32_t lo = load_const<int32_t>(p.row_ptr + (int64_t)head * p.num_blocks + i);
    r.cols = p.col_idx + lo;
    r.count = load_const<int32_t>(p.row_ptr + (int64_t)head * p.num_blocks + i + 1) - lo;
    return r;
  }
  if (p.dense) {
    r.local_lo = 0;
    r.count = i + 1;
    return r;
  }
  r.local_lo = max(0, i - p.local_blocks + 1);
  if (p.stride > 0) {
    const int o = p.head_index_base + head - (p.head_index_base + head) / p.by_stride * p.stride;
    const int lo = p.window_blocks > 0 ? max(0, i - p.window_blocks + 1) : 0;
    int first = o;
    if (lo > o) first = o + (lo - o + p.stride - 1) / p.by_stride * p.stride;
    if (first < r.local_lo) {
      r.first_stripe = first;
      r.n_stripe = (r.local_lo - 1 - first) / p.by_stride + 1;
    }
  }
  r.count = r.n_stripe + (i - r.local_lo + 1);
  return r;
}

// Whether row i keeps block j, a lane's own.  With lists, n is where j is likely to be in row i's: the rows of neighbouring tokens differ in few
// places, so that the search goes from there in steps that double, and then halves.
template <class PARAMS>
__device__ inline bool row_keeps(const PARAMS& p, const RowBlocks& rb, int head, int i, int j, int n) {
  if (rb.cols) {
    int lo = min(max(n, 0), rb.count - 1), hi = lo;  // (a row keeps its own block: count > 0)
    const int at = rb.cols[lo];
    if (at == j) return true;
    if (at > j) {
      for (int step = 1; lo > 0 && rb.cols[lo] > j; step *= 2) {
        hi = lo;
        lo = max(lo - step, 0);
      }
    } else {
      for (int step = 1; hi < rb.count - 1 && rb.cols[hi] < j; step *= 2) {
        lo = hi;
        hi = min(hi + step, rb.count - 1);
      }
    }
    while (lo < hi) {  // (the last entry <= j)
      const int mid = (lo + hi + 1) / 2;
      if (rb.cols[mid] > j)
        hi = mid - 1;
      else
        lo = mid;
    }
    return rb.cols[lo] == j;
  }
  if (j > i) return false;
  if (p.dense || i - j < p.local_blocks) return true;
  if (p.stride <= 0 || (p.window_blocks > 0 && i - j >= p.window_blocks)) return false;
  const int g = p.head_index_base + head, o = g - g / p.by_stride * p.stride, back = j - o;
  return back >= 0 && back - back / p.by_stride * p.stride == 0;
}

}  // namespace s2
