// Block tables of a paged cache for a step (section 4.1: a head's blocks that no later query attends are evicted), on the GPU from the lengths of the requests.
//
// For every (sequence, head, block) j of a table: to be held iff j * S < lens + new and a query at a position >= from can attend it, that is iff row
// r = from div S of the mask keeps j or j >= r (a later row of section 4.2's mask keeps no earlier block that row r does not), or, with a layout, iff the last row
// that keeps j is r or later.  Held and not to be held: its page is the next one at the end of the ring of free pages.  To be held, not held, and
// its first token new: it takes the next page from the ring's beginning.  "Next" is by (sequence, head, block), so that the result depends on
// the lengths and the tables alone: pages are numbered by counting, not by whoever comes first.
//
// Two launches: the first counts what every (sequence, head) gives up and takes, and sums the new tokens of 256 sequences at a time; in the second
// a workgroup adds up the counts before its own (at most kGroups numbers) and moves the pages.  Pages that are given up lie beyond those that were free before, so that
// taking and giving never meet in the ring, in place too.
//
// It reads and writes 4 bytes an entry, and takes what two dependent launches and their trips to memory take: for 64 sequences x 32 heads x 512 blocks, a table of 4 MB, 5.4 and 7.7 us
// (0.9 TB/s of 11 MB), for 11 x 7 short lines 3.4 and 4.8.  One launch would have each workgroup count what is before it, or wait for others.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kernels.h"
#include "row_blocks.h"

namespace s2 {

namespace {

using i32x2 = __attribute__((ext_vector_type(2))) int;
using i32x4 = __attribute__((ext_vector_type(4))) int;

constexpr int kThreadsPlan = 256, kWaves = kThreadsPlan / 64;
constexpr int kGroups = 1024;  // workgroups over the tables, about: so many counts are added up by each of them

// A sequence as the step finds it.
struct Seq {
  int len, end, row;  // tokens before and after it (as far as the table has room for), row that the first query is in
};
__device__ __forceinline__ Seq seq_of(int len, int fresh, int from, const KvPlanParams& p) {
  Seq s;
  s.len = min(max(len, 0), p.max_len);
  s.end = fresh < 0 ? 0 : s.len + min(fresh, p.max_len - s.len);
  s.row = min(max(from, 0), p.max_len - 1) >> p.block_shift;
  return s;
}

// What becomes of block j of (sequence, head) h, whose entry is `page`; 64 blocks at a time.
struct Fate {
  bool held, needed, taken;  // it has a page; it is to have one; it is to take one
};
__device__ __forceinline__ Fate fate_of(const KvPlanParams& p, const Seq& s, const RowBlocks& rb, int h, int j, int page) {
  const int S = 1 << p.block_shift;
  Fate f;
  f.held = page >= 0 && page < p.num_pages;
  f.needed = j < (s.end + S - 1) >> p.block_shift;  // (max_len is below 2^31 - S)
  if (p.last_row)
    f.needed = f.needed && p.last_row[(int64_t)h * p.num_blocks + j] >= s.row;
  else
    f.needed = f.needed && (j >= s.row || row_keeps(p, rb, h, s.row, j, 0));
  f.taken = f.needed && !f.held && j >= (s.len + S - 1) >> p.block_shift;
  return f;
}

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
  for (int i = 1; i < 64; i *= 2) x += __shfl_xor(x, i, 64);
  return x;
}
// The sums of N numbers over a workgroup (to all its threads).
template <int N>
__device__ __forceinline__ void group_sums(int64_t (&x)[N], int64_t (*parts)[kWaves]) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
#pragma unroll
    for (int i = 1; i < 64; i *= 2) x[k] += __shfl_xor(x[k], i, 64);
    if ((threadIdx.x & 63) == 0) parts[k][threadIdx.x >> 6] = x[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) {
    x[k] = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) x[k] += parts[k][i];
  }
}

// kAtOnce times 64 entries of a line from j0 on, a lane's; -1 behind the line's end.  (48 sequences x 32 heads x 543 blocks: 5.7 and 8.2 us; loaded one after the other, with the counts, up to 7.6 and 10.4.)
constexpr int kAtOnce = 8;
__device__ __forceinline__ void load_entries(const int32_t* line, int j0, int max_blocks, int lane, int (&to)[kAtOnce]) {
#pragma unroll
  for (int k = 0; k < kAtOnce; ++k) {
    const int j = j0 + 64 * k + lane;
    to[k] = line[min(j, max_blocks - 1)];
    if (j >= max_blocks) to[k] = -1;
  }
}

__global__ __launch_bounds__(kThreadsPlan) void kv_plan_count_kernel(const KvPlanParams p) {
  __shared__ int64_t parts[1][kWaves];
  __shared__ int counts[kWaves][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if ((int)blockIdx.x >= p.groups) {  // 256 sequences
    const int block = blockIdx.x - p.groups, b = block * kThreadsPlan + tid;
    int64_t fresh[1] = {0};
    if (b < p.nseq) {
      const int len = p.lens[b], n = p.new_lens[b];
      const Seq s = seq_of(len, n, p.query_from ? p.query_from[b] : len, p);
      int* const to = p.ws_seq + 4 * (int64_t)b;
      to[0] = s.len;
      to[1] = s.end;
      to[2] = s.row;
      to[3] = max(n, 0);
      fresh[0] = max(n, 0);
    }
    group_sums(fresh, parts);
    if (tid == 0) p.ws_fresh[block] = fresh[0];
    if (block == 0 && tid == 0) {
      const int first = p.free_state[0], count = min(max(p.free_state[1], 0), p.num_pages);
      p.ws_state[0] = first >= 0 && first < p.num_pages ? first : 0;
      p.ws_state[1] = count;
    }
    return;
  }
  int freed = 0, taken = 0;  // of all my pairs, a lane's part
  for (int i = 0; i < p.pairs_each; ++i) {
    const int64_t pair = ((int64_t)blockIdx.x * kWaves + wave) * p.pairs_each + i;
    if (pair >= p.pairs) break;
    const int32_t* const line = p.table + pair * p.max_blocks;
    int page[kAtOnce];
    load_entries(line, 0, p.max_blocks, lane, page);
    const int b = (int)pair / p.by_heads, h = (int)pair - b * p.heads;
    const int len = load_const<int32_t>(p.lens + b);
    const Seq s = seq_of(len, load_const<int32_t>(p.new_lens + b), p.query_from ? load_const<int32_t>(p.query_from + b) : len, p);
    const RowBlocks rb{};
    int f0 = 0, t0 = 0;
    for (int j0 = 0;;) {
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        if (j0 + 64 * k >= p.max_blocks) break;
        const int j = j0 + 64 * k + lane;
        const bool is = j < p.max_blocks;
        const Fate f = fate_of(p, s, rb, h, is ? j : 0, page[k]);
        f0 += __popcll(__ballot(is && f.held && !f.needed));
        t0 += __popcll(__ballot(is && f.taken));
      }
      j0 += 64 * kAtOnce;
      if (j0 >= p.max_blocks) break;
      load_entries(line, j0, p.max_blocks, lane, page);
    }
    if (lane == 0) {
      p.ws_pair[2 * pair] = f0;
      p.ws_pair[2 * pair + 1] = t0;
    }
    freed += f0;
    taken += t0;
  }
  if (lane == 0) {
    counts[wave][0] = freed;
    counts[wave][1] = taken;
  }
  __syncthreads();
  if (tid < 2) {
    int sum = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += counts[w][tid];
    p.ws_group[2 * blockIdx.x + tid] = sum;
  }
}

// What all groups before `group` give up and take.
__device__ __forceinline__ void before_group(const KvPlanParams& p, int group, int64_t (*parts)[kWaves], int64_t& freed, int64_t& taken) {
  int64_t sums[2] = {0, 0};
#pragma unroll 4
  for (int i = threadIdx.x; i < group; i += kThreadsPlan) {
    const i32x2 of = reinterpret_cast<const i32x2*>(p.ws_group)[i];
    sums[0] += of[0];
    sums[1] += of[1];
  }
  group_sums(sums, parts);
  freed = sums[0];
  taken = sums[1];
}

__global__ __launch_bounds__(kThreadsPlan) void kv_plan_move_kernel(const KvPlanParams p) {
  __shared__ int64_t parts[2][kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int first = p.ws_state[0], count = p.ws_state[1];
  const int room = p.num_pages - count;  // pages that the ring has room for (more than are held only if an entry names a page twice)
  int item = blockIdx.x;
  auto slot = [&](int64_t at) {  // of the ring, at < 2 num_pages
    return at >= p.num_pages ? at - p.num_pages : at;
  };
  if (item < p.groups) {
    const int64_t pair0 = (int64_t)item * kWaves * p.pairs_each, mine = pair0 + (int64_t)wave * p.pairs_each;
    int page[kAtOnce];
    load_entries(p.table + min(mine, p.pairs - 1) * p.max_blocks, 0, p.max_blocks, lane, page);
    // (all of these loads before the wavefronts wait for each other)
    int f0 = 0, t0 = 0;  // of the wavefronts before mine
    for (int64_t i = pair0 + lane; i < min(mine, (int64_t)p.pairs); i += 64) {
      const i32x2 of = reinterpret_cast<const i32x2*>(p.ws_pair)[i];
      f0 += of[0];
      t0 += of[1];
    }
    i32x4 seq = reinterpret_cast<const i32x4*>(p.ws_seq)[(int)min(mine, p.pairs - 1) / p.by_heads];
    int64_t freed, taken;
    before_group(p, item, parts, freed, taken);
    if (item == p.groups - 1 && tid == 0) {
      const int64_t f = min(freed + p.ws_group[2 * item], (int64_t)room), t = min(taken + p.ws_group[2 * item + 1], (int64_t)count);
      p.new_state[0] = (int)slot(first + t);
      p.new_state[1] = (int)(count - t + f);
    }
    freed += wave_sum(f0);
    taken += wave_sum(t0);
    int without = 0;
    for (int i = 0; i < p.pairs_each; ++i) {
      const int64_t pair = mine + i;
      if (pair >= p.pairs) break;
      const int b = (int)pair / p.by_heads, h = (int)pair - b * p.heads;
      if (i > 0) seq = reinterpret_cast<const i32x4*>(p.ws_seq)[b];
      const Seq s{seq[0], seq[1], seq[2]};
      const RowBlocks rb{};
      const int32_t* const line = p.table + pair * p.max_blocks;
      int32_t* const to = p.new_table + pair * p.max_blocks;
      if (i > 0) load_entries(line, 0, p.max_blocks, lane, page);
      for (int j0 = 0;;) {
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
          if (j0 + 64 * k >= p.max_blocks) break;
          const int j = j0 + 64 * k + lane;
          const bool is = j < p.max_blocks;
          const Fate f = fate_of(p, s, rb, h, is ? j : 0, page[k]);
          const uint64_t gives = __ballot(is && f.held && !f.needed), takes = __ballot(is && f.taken);
          const uint64_t below = ((uint64_t)1 << lane) - 1;
          int now = f.needed ? page[k] : -1;
          if (gives) {  // (in most lines of a step none, or one chunk's: 8.3 -> 7.7 us)
            const int64_t at = freed + __popcll(gives & below);
            if ((gives >> lane & 1) && at < room) p.new_ring[slot((int64_t)first + count + at)] = page[k];
            freed += __popcll(gives);
          }
          if (takes) {
            const int64_t at = taken + __popcll(takes & below);
            if (takes >> lane & 1) now = at < count ? p.ring[slot(first + at)] : -1;
            without += (int)min(max(taken + __popcll(takes) - max(taken, (int64_t)count), (int64_t)0), (int64_t)64);
            taken += __popcll(takes);
          }
          if (is && (p.apart || now != page[k])) to[j] = now;
        }
        j0 += 64 * kAtOnce;
        if (j0 >= p.max_blocks) break;
        load_entries(line, j0, p.max_blocks, lane, page);
      }
    }
    if (p.short_of && lane == 0 && without > 0) atomicAdd(p.short_of, without);
    return;
  }
  item -= p.groups;
  if (item < p.nseq) {  // a sequence's rows
    if (!p.cu_new && !p.positions && !p.seq_lens) return;
    int64_t sums[1] = {0};
    for (int i = tid; i < item / kThreadsPlan; i += kThreadsPlan) sums[0] += p.ws_fresh[i];
    const int in_block = item / kThreadsPlan * kThreadsPlan + tid;
    if (in_block < item) sums[0] += p.ws_seq[4 * (int64_t)in_block + 3];
    group_sums(sums, parts);
    const int64_t before = sums[0];
    const int len = p.ws_seq[4 * (int64_t)item], end = p.ws_seq[4 * (int64_t)item + 1], fresh = p.ws_seq[4 * (int64_t)item + 3];
    constexpr int64_t kMost = 0x7fffffff;
    if (tid == 0) {
      if (p.cu_new) {
        if (item == 0) p.cu_new[0] = 0;
        p.cu_new[item + 1] = (int)min(before + fresh, kMost);
      }
      if (p.seq_lens) p.seq_lens[item] = end;
    }
    if (!p.positions) return;
    const int64_t rows = min((int64_t)fresh, p.num_rows - before);
    for (int64_t i = tid; i < rows; i += kThreadsPlan) p.positions[before + i] = (int)min(len + i, kMost);
    return;
  }
  item -= p.nseq;  // entries of the ring that no page is written to
  const int64_t i0 = (int64_t)item * kRingEach + tid;
  int entry[kRingEach / kThreadsPlan];
#pragma unroll
  for (int k = 0; k < kRingEach / kThreadsPlan; ++k) entry[k] = p.ring[min(i0 + k * kThreadsPlan, (int64_t)p.num_pages - 1)];
  int64_t freed, taken;
  before_group(p, p.groups, parts, freed, taken);
  freed = min(freed, (int64_t)room);
#pragma unroll
  for (int k = 0; k < kRingEach / kThreadsPlan; ++k) {
    const int64_t i = i0 + k * kThreadsPlan, from_tail = i - slot((int64_t)first + count);
    if (i < p.num_pages && (from_tail < 0 ? from_tail + p.num_pages : from_tail) >= freed) p.new_ring[i] = entry[k];
  }
}

}  // namespace

void plan_groups(KvPlanParams& p) {
  p.pairs_each = (int)((p.pairs + (int64_t)kGroups * kWaves - 1) / ((int64_t)kGroups * kWaves));
  p.groups = (int)((p.pairs + (int64_t)p.pairs_each * kWaves - 1) / ((int64_t)p.pairs_each * kWaves));
}

hipError_t launch_kv_plan(const KvPlanParams& params, hipStream_t stream) {
  KvPlanParams p = params;
  p.by_heads = fast_div(p.heads);
  p.by_stride = fast_div(p.stride > 0 ? p.stride : 1);
  hipLaunchKernelGGL(kv_plan_count_kernel, dim3(p.groups + (p.nseq + kThreadsPlan - 1) / kThreadsPlan), dim3(kThreadsPlan), 0, stream, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int ring = p.new_ring == p.ring ? 0 : (int)(((int64_t)p.num_pages + kRingEach - 1) / kRingEach);
  hipLaunchKernelGGL(kv_plan_move_kernel, dim3(p.groups + p.nseq + ring), dim3(kThreadsPlan), 0, stream, p);
  return hipGetLastError();
}

}  // namespace s2
