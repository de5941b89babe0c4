// C ABI of libs2attn.so: argument validation, the layout handle's device copies, and dispatch to
// the kernels.  See include/s2attn.h for the contract of every entry point.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>
#include <initializer_list>
#include <limits>
#include <new>

#include "../../include/s2attn.h"
#include "config.h"
#include "kernels.h"
#include "layout.h"

namespace {

thread_local int g_last_hip_error = 0;

inline bool hip_ok(hipError_t e) {
  if (e == hipSuccess) return true;
  g_last_hip_error = (int)e;
  return false;
}

bool upload(const std::vector<int32_t>& host, int32_t** dev) {
  *dev = nullptr;
  const size_t bytes = (host.empty() ? 1 : host.size()) * sizeof(int32_t);
  if (!hip_ok(hipMalloc(reinterpret_cast<void**>(dev), bytes))) return false;
  if (host.empty()) return true;
  return hip_ok(hipMemcpy(*dev, host.data(), host.size() * sizeof(int32_t), hipMemcpyHostToDevice));
}

bool upload_tiles(s2::TileList& t) {
  return upload(t.ptr, &t.d_ptr) && upload(t.ent, &t.d_ent) && upload(t.rec, &t.d_rec);
}

void free_tiles(s2::TileList& t) {
  if (t.d_ptr) (void)hipFree(t.d_ptr);
  if (t.d_ent) (void)hipFree(t.d_ent);
  if (t.d_rec) (void)hipFree(t.d_rec);
  t.d_ptr = t.d_ent = t.d_rec = nullptr;
}

void free_device_copies(s2_layout* L) {
  free_tiles(L->q_tiles);
  free_tiles(L->kv_tiles);
  if (L->d_row_ptr) (void)hipFree(L->d_row_ptr);
  if (L->d_col_idx) (void)hipFree(L->d_col_idx);
  if (L->d_last_row) (void)hipFree(L->d_last_row);
  if (L->d_dq_units) (void)hipFree(L->d_dq_units);
  if (L->d_kv_split_codes) (void)hipFree(L->d_kv_split_codes);
  L->d_row_ptr = L->d_col_idx = L->d_last_row = L->d_dq_units = L->d_kv_split_codes = nullptr;
}

s2::DevTiles dev_tiles(const s2::TileList& t) {
  s2::DevTiles d;
  d.ptr = t.d_ptr;
  d.ent = t.d_ent;
  d.rec = t.d_rec;
  d.tiles_per_head = t.tiles_per_head;
  d.group = t.group;
  return d;
}

// The lists the row-tile and key-tile kernels walk.
void set_tiles(s2::AttnParams& p, const s2_layout* L) {
  p.q_tiles = dev_tiles(L->q_tiles);
  p.kv_tiles = dev_tiles(L->kv_tiles);
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// The split partials of s2_attn_decode_static live here instead of in a caller's workspace: device
// memory that belongs to the loaded library, one copy per GPU at that GPU's own address, held
// until the process ends.  In host code the array's name is only a handle for
// hipGetSymbolAddress; the address found there, kept per device, is what the kernels are given.
constexpr size_t kStaticScratchBytes = S2_DECODE_STATIC_SCRATCH_BYTES;
__device__ __align__(256) unsigned char scratch[kStaticScratchBytes];

constexpr int kScratchMaxDevices = 64;
std::atomic<void*> g_scratch_ptr[kScratchMaxDevices];  // zero-initialised: not looked up yet

// Address of `scratch` on the current device, or nullptr (the hipError_t is kept for
// s2_last_hip_error).  The first call on a device asks the runtime; later calls read the slot.
void* scratch_on_current_device() {
  int dev = -1;
  if (!hip_ok(hipGetDevice(&dev))) return nullptr;
  if (dev < 0 || dev >= kScratchMaxDevices) {
    g_last_hip_error = (int)hipErrorInvalidDevice;
    return nullptr;
  }
  void* ptr = g_scratch_ptr[dev].load(std::memory_order_acquire);
  if (ptr) return ptr;
  if (!hip_ok(hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch))) || !ptr) return nullptr;
  g_scratch_ptr[dev].store(ptr, std::memory_order_release);  // racing threads store the same address
  return ptr;
}

// Shape / alignment checks shared by forward and backward.  `need_bwd` also checks the
// gradient tensors.
int check_tensors(const s2_tensors* t, bool need_bwd, float scale) {
  if (!t) return S2_ERR_NULL;
  if (!t->q || !t->k || !t->v || !t->o || !t->lse) return S2_ERR_NULL;
  if (need_bwd && (!t->d_o || !t->dq || !t->dk || !t->dv)) return S2_ERR_NULL;
  if (!(scale > 0.f) || !std::isfinite(scale)) return S2_ERR_BAD_PARAM;
  if (t->batch < 1 || t->heads < 1 || t->seqlen < 1) return S2_ERR_SHAPE;
  if (t->head_dim != 64 && t->head_dim != 128) return S2_ERR_SHAPE;
  if ((int64_t)t->batch * t->heads * t->seqlen > (int64_t)1 << 40) return S2_ERR_SHAPE;
  const int64_t strides[6] = {t->q_stride_b, t->q_stride_h, t->q_stride_t,
                              t->kv_stride_b, t->kv_stride_h, t->kv_stride_t};
  for (int64_t s : strides)
    if (s < 0 || (s & 7) != 0) return S2_ERR_ALIGN;
  if (t->q_stride_t < t->head_dim || t->kv_stride_t < t->head_dim) return S2_ERR_ALIGN;
  // the kernels address the 16 rows of a piece with unsigned 32-bit byte offsets
  if (t->q_stride_t > (1 << 24) || t->kv_stride_t > (1 << 24)) return S2_ERR_SHAPE;
  const void* ptrs[9] = {t->q, t->k, t->v, t->o, t->lse, t->d_o, t->dq, t->dk, t->dv};
  for (int i = 0; i < (need_bwd ? 9 : 5); ++i)
    if (!aligned16(ptrs[i])) return S2_ERR_ALIGN;
  return S2_OK;
}

s2::AttnParams make_params(const s2_tensors* t, float scale) {
  s2::AttnParams p{};
  p.q = static_cast<const uint16_t*>(t->q);
  p.k = static_cast<const uint16_t*>(t->k);
  p.v = static_cast<const uint16_t*>(t->v);
  p.o = static_cast<uint16_t*>(t->o);
  p.lse = t->lse;
  p.d_o = static_cast<const uint16_t*>(t->d_o);
  p.dq = static_cast<uint16_t*>(t->dq);
  p.dk = static_cast<uint16_t*>(t->dk);
  p.dv = static_cast<uint16_t*>(t->dv);
  p.batch = t->batch;
  p.heads = t->heads;
  p.seqlen = t->seqlen;
  p.q_row0 = 0;
  p.q_rows = t->seqlen;
  p.head_dim = t->head_dim;
  p.q_sb = t->q_stride_b;
  p.q_sh = t->q_stride_h;
  p.q_st = t->q_stride_t;
  p.kv_sb = t->kv_stride_b;
  p.kv_sh = t->kv_stride_h;
  p.kv_st = t->kv_stride_t;
  p.scale = scale;
  p.scale_log2e = scale * 1.4426950408889634f;
  // The dK/dV kernel forms P as exp(s * (S - lse / s)).  s is the scale, but not below 2^-120, so that lse / s is finite; where it is not
  // the scale P is off by a factor of exp(S * (s - scale)), which is 1 to float32's precision for |S| up to 2^96.
  const float s = std::max(scale, 0x1p-120f);
  p.neg_inv_scale = -1.0f / s;
  p.p_scale_log2e = s * 1.4426950408889634f;
  return p;
}

// The layout's lists live on the device that was current when it was built.
bool layout_on_current_device(const s2_layout* L) {
  if (!L->on_device) return false;
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) {
    (void)hipGetLastError();
    return false;
  }
  return dev == L->device;
}

int check_layout_fits(const s2_layout* L, const s2_tensors* t) {
  if (!L) return S2_ERR_NULL;
  if (t->heads != L->p.num_heads) return S2_ERR_SHAPE;
  if ((int64_t)t->seqlen != (int64_t)L->p.num_blocks * L->p.block_size) return S2_ERR_SHAPE;
  return S2_OK;
}

}  // namespace

extern "C" {

namespace {
// Tile lists for the three passes, then the device copy when a GPU is visible.  Takes ownership
// of L: on failure it is deleted.
int finish_layout(s2_layout* L, int st, s2_layout** out) {
  std::vector<int32_t> last_row;
  if (st == S2_OK) {
    try {
      last_row.resize(L->col_ptr.size() - 1);
      for (size_t j = 0; j < last_row.size(); ++j) last_row[j] = L->col_ptr[j + 1] > L->col_ptr[j] ? L->row_idx[(size_t)L->col_ptr[j + 1] - 1] : -1;
      const int S = L->p.block_size;
      static_assert(s2::kFwdBM == s2::kBwdBM, "forward and dQ walk the same lists");
      s2::build_tiles(*L, s2::kBwdBM / S, false, L->q_tiles);
      s2::build_tiles(*L, s2::kBwdBN / S, true, L->kv_tiles);
      s2::build_splits(*L);
      s2::build_ds_units(*L);
    } catch (const std::bad_alloc&) {
      st = S2_ERR_OVERFLOW;
    }
  }
  if (st != S2_OK) {
    delete L;
    return st;
  }
  int ndev = 0;
  if (hipGetDeviceCount(&ndev) == hipSuccess && ndev > 0) {
    int dev = 0;
    bool ok = hip_ok(hipGetDevice(&dev)) && upload_tiles(L->q_tiles) && upload_tiles(L->kv_tiles) && upload(L->row_ptr, &L->d_row_ptr) &&
              upload(L->col_idx, &L->d_col_idx) && upload(last_row, &L->d_last_row) && upload(L->dq_units, &L->d_dq_units) &&
              upload(L->kv_split_codes, &L->d_kv_split_codes);
    if (!ok) {
      free_device_copies(L);
      delete L;
      return S2_ERR_HIP;
    }
    L->device = dev;
    L->on_device = true;
  } else {
    (void)hipGetLastError();  // no GPU: a host-only layout is still a valid result
  }
  *out = L;
  return S2_OK;
}
}  // namespace

int s2_layout_build(const s2_layout_params* params, s2_layout** out) {
  if (!params || !out) return S2_ERR_NULL;
  *out = nullptr;
  s2_layout* L = new (std::nothrow) s2_layout();
  if (!L) return S2_ERR_OVERFLOW;
  int st;
  try {
    st = s2::build_host(*params, *L);
  } catch (const std::bad_alloc&) {
    st = S2_ERR_OVERFLOW;
  }
  return finish_layout(L, st, out);
}

int s2_layout_from_csr(int32_t num_heads, int32_t num_blocks, int32_t block_size, const int32_t* row_ptr,
                       const int32_t* col_idx, s2_layout** out) {
  if (!row_ptr || !col_idx || !out) return S2_ERR_NULL;
  *out = nullptr;
  s2_layout* L = new (std::nothrow) s2_layout();
  if (!L) return S2_ERR_OVERFLOW;
  int st;
  try {
    st = s2::build_from_csr(num_heads, num_blocks, block_size, row_ptr, col_idx, *L);
  } catch (const std::bad_alloc&) {
    st = S2_ERR_OVERFLOW;
  }
  return finish_layout(L, st, out);
}

int s2_layout_destroy(s2_layout* layout) {
  if (!layout) return S2_ERR_NULL;
  if (layout->on_device) free_device_copies(layout);
  delete layout;
  return S2_OK;
}

int s2_layout_get(const s2_layout* L, s2_layout_view* out) {
  if (!L || !out) return S2_ERR_NULL;
  out->row_ptr = L->row_ptr.data();
  out->col_idx = L->col_idx.data();
  out->col_ptr = L->col_ptr.data();
  out->row_idx = L->row_idx.data();
  out->nnz = L->nnz;
  out->num_heads = L->p.num_heads;
  out->num_blocks = L->p.num_blocks;
  out->block_size = L->p.block_size;
  out->max_row_blocks = L->max_row_blocks;
  out->covers_all = L->covers_all;
  out->on_device = L->on_device ? 1 : 0;
  return S2_OK;
}

int s2_layout_get_tiles(const s2_layout* L, int which, s2_tile_view* out) {
  if (!L || !out) return S2_ERR_NULL;
  if (which != S2_TILES_FWD && which != S2_TILES_DQ && which != S2_TILES_DKDV) return S2_ERR_BAD_PARAM;
  const s2::TileList& t = which == S2_TILES_DKDV ? L->kv_tiles : L->q_tiles;
  out->ptr = t.ptr.data();
  out->ent = t.ent.data();
  out->order = t.order.data();
  out->members = t.members.data();
  out->tiles_per_head = t.tiles_per_head;
  out->group = t.group;
  out->blocks_per_unit = 1;
  return S2_OK;
}

int s2_layout_get_ds_units(const s2_layout* L, s2_ds_units_view* out) {
  if (!L || !out) return S2_ERR_NULL;
  out->dq_units = L->dq_units.data();
  out->count = (int64_t)L->dq_units.size();
  out->ds_units = L->ds_units;
  return S2_OK;
}

int s2_attn_fwd(const s2_layout* layout, const s2_tensors* t, float scale, void* stream) {
  if (!layout) return S2_ERR_NULL;
  int st = check_tensors(t, false, scale);
  if (st != S2_OK) return st;
  st = check_layout_fits(layout, t);
  if (st != S2_OK) return st;
  if (!layout_on_current_device(layout)) return S2_ERR_NO_DEVICE;
  s2::AttnParams p = make_params(t, scale);
  p.block_size = layout->p.block_size;
  set_tiles(p, layout);
  return hip_ok(s2::launch_fwd(p, false, static_cast<hipStream_t>(stream))) ? S2_OK : S2_ERR_HIP;
}

namespace {

size_t round256(size_t bytes) { return (bytes + 255) / 256 * 256; }

// The backward's workspace: the row statistics -delta = -rowsum(dO * O) and -lse / scale; then dS, where it is kept;
// then, for launches of so few tiles that the longest ones may be cut, a counter per key tile and the sums of the
// parts.  Without the last nothing is cut, without room for dS it is not kept, and neither depends on the other.
struct BwdWorkspace {
  size_t stats;      // bytes of either of the first two arrays
  size_t count;      // of the counters
  size_t sums;       // of the sums
  int64_t slots;     // parts that there is room for
  size_t required() const { return 2 * stats; }
  size_t cut() const { return count + sums; }
};
BwdWorkspace bwd_workspace(int32_t batch, int32_t heads, int32_t seqlen, int32_t head_dim) {
  BwdWorkspace w{};
  const int64_t rows = (int64_t)batch * heads * seqlen;
  w.stats = round256((size_t)rows * sizeof(float));
  const int64_t per_head = (seqlen + s2::kBwdBN - 1) / s2::kBwdBN, tiles = (int64_t)batch * heads * per_head;
  // From 4096 tiles on (eight rounds of the chip's 512 workgroup slots) the longest tile no longer decides.  (head_dim
  // is not checked here: the query has never done so, and no call takes one that is neither 64 nor 128.)
  if (tiles < 4096 && head_dim > 0) {
    w.count = round256((size_t)tiles * sizeof(int32_t));
    // no tile is longer than all of its head's rows, two 64-row steps to a tile, and no part shorter than four steps
    w.slots = std::min<int64_t>(768, tiles * std::min<int64_t>(8, (2 * per_head + 3) / 4));
    w.sums = (size_t)w.slots * s2::kBwdBN * head_dim * 2 * sizeof(float);
  }
  return w;
}

}  // namespace

size_t s2_attn_bwd_workspace_bytes(int32_t batch, int32_t heads, int32_t seqlen, int32_t head_dim) {
  if (batch < 1 || heads < 1 || seqlen < 1) return 0;
  const BwdWorkspace w = bwd_workspace(batch, heads, seqlen, head_dim);
  return w.required() + w.cut();
}

namespace {

// Whether and how to cut the longest key tiles.  A stripe column is attended by every later row, so a head
// has a few tiles of up to N / 64 steps among many short ones.  With enough (batch, head) pairs the long
// ones are hidden behind the rest; with few the launch is as long as its longest tile while most
// of the chip idles.  `even`: the steps a workgroup slot would walk if all were shared out evenly (a tile
// costs about five steps besides its own, an XCD holds 64 workgroups of head_dim 128 and the
// equivalent of 80 of 64).  Measured, forward + backward with the longest tile / even = 4.4 (8 heads
// x 4096): 202 -> 89 us; 2.3 (2 x 16 x 3904): 255 -> 183; 3.0 (16 x 16384): 969 -> 637; 1.5 (2 x 20 x 8192,
// blocks of 128): 677 -> 616; 1.2 (3 x 16 x 8192): 791 -> 764; 0.88 (4 x 16 x 8192): 999 uncut, 1026 cut.  The
// best length of a part was 6 to 8, 24, 64, 48 to 64 and 64 steps, that is about 3/4 of `even` plus 3: a
// part's own cost (its start, 64 KB per 128 keys and 64 features written and read again) against the evenness of the launch.
// Where all tiles start at once they should still do so when cut: 52 heads x 800 x 128 in blocks of 32, 49 workgroups for
// an XCD's 64 slots uncut and 84 cut, forward and backward 78 us uncut, 90 cut; 42 heads, 42 and 54, 66 and 54.  Where no
// cut leaves it so, a second round still costs less than a tile much longer than a part: with longest tile / best = 10 (8 heads x
// 8192 x 128, 64 workgroups and 88) 311 us uncut and 109 cut, 4.7 (16 x 4096 x 128) 191 and 112, 2.7 (4 x 8 x 2048 x 128) 123 and 89, 8.9 (8 x
// 10240 x 64) 262 and 119, but with 2.4 (3 x 8 x 2560 x 128) 172 and 168, or 141 and 152 in the launch that has the dQ tiles too, and with
// 1.9 (4 x 8 x 2048 x 128) 139 and 146 there.
// (batch, head) pairs that are left over from a multiple of eight are shared by the XCDs.  They count as a whole pair for whether to cut and
// what starts at once, as the parts of one tile lie on XCDs next to each other; for the best length three quarters of what they lack of one are added. And a
// cut whose parts all start at once is then no good where they are half as long again as the best length, or two thirds of it.  Backward, us,
// with pairs / 8, with that rounded up and so: 7 heads x 8192 x 128 122, 105 and 102, 4 x 23 x 768 79, 72 and 72, 2 x 8192 x 64 38, 56 and 35, 9 x 8192 x 64 84, 66 and 67, 3 x 4
// x 3072 x 128, blocks of 128, 72, 57 and 57.  Over 332 shapes with pairs left over each is this much behind the best of all cuts: 4.0, 3.5 and 2.6 %.
void choose_split(s2::AttnParams& p, const s2_layout* L, const BwdWorkspace& w, unsigned char* room) {
  const double slots = p.head_dim == 128 ? 64 : 80;
  const int T = p.kv_tiles.tiles_per_head;
  const int pairs = (p.batch * p.heads + 7) / 8;  // of an XCD
  const double even = (L->kv_head_steps + 5.0 * T) / slots;  // of each of them
  if (L->kv_max_steps <= 1.1 * pairs * even) return;
  const double best = 0.75 * (3 * pairs + p.batch * p.heads / 8.0) / 4 * even + 3;
  double off;  // how far from the best length the parts are of the cut that `closest` has found
  auto closest = [&](bool one_round) {
    const s2::SplitLevel* use = nullptr;
    off = 0;
    for (const s2::SplitLevel& lv : L->kv_levels) {
      if ((int64_t)p.batch * p.heads * lv.n_items > w.slots || 2 * lv.steps > L->kv_max_steps) continue;
      if (one_round && pairs * (T + lv.n_items - lv.n_long) > slots) continue;
      const double o = std::max(lv.steps / best, best / lv.steps);
      if (use && o >= off) continue;
      use = &lv;
      off = o;
    }
    return use;
  };
  const bool one_round = pairs * T <= slots;
  const s2::SplitLevel* use = closest(one_round);
  const double far = p.batch * p.heads % 8 ? 1.5 : HUGE_VAL;
  if (one_round && (!use || off > far) && L->kv_max_steps > 2.4 * best) use = closest(false);
  if (!use) return;
  p.split_codes = L->d_kv_split_codes + use->offset;
  p.split_items = use->n_items;
  p.split_long = use->n_long;
  p.split_count = reinterpret_cast<int32_t*>(room);
  p.split_sums = reinterpret_cast<float*>(room + w.count);
}

// The backward that keeps dS covers head_dim 128, mask blocks of 64 or 128 tokens (the layout then
// carries the unit table) and whole 128-row tiles.
bool keeps_ds(const s2_layout* L, int32_t seqlen, int32_t head_dim) {
  return L->ds_units > 0 && head_dim == 128 && seqlen % s2::kBwdBM == 0 &&
         (int64_t)seqlen == (int64_t)L->p.num_blocks * L->p.block_size;
}
}  // namespace

size_t s2_attn_bwd_layout_workspace_bytes(const s2_layout* layout, int32_t batch, int32_t heads, int32_t seqlen,
                                          int32_t head_dim) {
  const size_t small = s2_attn_bwd_workspace_bytes(batch, heads, seqlen, head_dim);
  if (!layout || small == 0 || heads != layout->p.num_heads || !keeps_ds(layout, seqlen, head_dim)) return small;
  return small + (size_t)batch * (size_t)layout->ds_units * 8192;
}

int s2_attn_bwd(const s2_layout* layout, const s2_tensors* t, float scale, void* workspace,
                size_t workspace_bytes, void* stream) {
  return s2_attn_bwd_stages(layout, t, scale, workspace, workspace_bytes, S2_BWD_ALL, stream);
}

int s2_attn_fwd_rows(const s2_layout* layout, const s2_tensors* t, int32_t q_row_start, int32_t q_rows,
                     float scale, void* stream) {
  if (!layout) return S2_ERR_NULL;
  int st = check_tensors(t, false, scale);
  if (st != S2_OK) return st;
  if (t->heads != layout->p.num_heads) return S2_ERR_SHAPE;
  if ((int64_t)t->seqlen > (int64_t)layout->p.num_blocks * layout->p.block_size) return S2_ERR_SHAPE;
  if (q_row_start < 0 || q_rows < s2::kFwdBM || q_row_start % s2::kFwdBM != 0 || q_rows % s2::kFwdBM != 0)
    return S2_ERR_SHAPE;
  if ((int64_t)q_row_start + q_rows > t->seqlen) return S2_ERR_SHAPE;
  if (!layout_on_current_device(layout)) return S2_ERR_NO_DEVICE;
  s2::AttnParams p = make_params(t, scale);
  p.q_row0 = q_row_start;
  p.q_rows = q_rows;
  p.block_size = layout->p.block_size;
  set_tiles(p, layout);
  return hip_ok(s2::launch_fwd(p, false, static_cast<hipStream_t>(stream))) ? S2_OK : S2_ERR_HIP;
}

int s2_attn_fwd_varlen(const s2_layout* layout, const s2_tensors* t, const int32_t* cu_seqlens,
                       int32_t num_seqs, int32_t max_seqlen, float scale, void* stream) {
  if (!layout || !cu_seqlens) return S2_ERR_NULL;
  int st = check_tensors(t, false, scale);
  if (st != S2_OK) return st;
  if (t->batch != 1 || t->heads != layout->p.num_heads) return S2_ERR_SHAPE;
  if (num_seqs < 1 || max_seqlen < 1) return S2_ERR_SHAPE;
  if ((int64_t)max_seqlen > (int64_t)layout->p.num_blocks * layout->p.block_size) return S2_ERR_SHAPE;
  if ((int64_t)num_seqs * t->heads > std::numeric_limits<int32_t>::max() / 2) return S2_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(cu_seqlens) & 3u) != 0) return S2_ERR_ALIGN;
  if (!layout_on_current_device(layout)) return S2_ERR_NO_DEVICE;
  s2::AttnParams p = make_params(t, scale);
  p.batch = num_seqs;
  p.q_rows = max_seqlen;
  p.cu_seqlens = cu_seqlens;
  p.block_size = layout->p.block_size;
  set_tiles(p, layout);
  // one grid slot per (sequence, head, 128-row tile of the longest length allowed)
  const int64_t slots = 8 * (((int64_t)num_seqs * t->heads + 7) / 8) * ((max_seqlen + s2::kFwdBM - 1) / s2::kFwdBM);
  if (slots > std::numeric_limits<int32_t>::max()) return S2_ERR_SHAPE;
  return hip_ok(s2::launch_fwd(p, false, static_cast<hipStream_t>(stream))) ? S2_OK : S2_ERR_HIP;
}

size_t s2_attn_bwd_varlen_workspace_bytes(int32_t heads, int32_t rows, int32_t head_dim) {
  (void)head_dim;
  if (heads < 1 || rows < 1) return 0;
  // the two row statistics per (head, row), plus one chunk of slack each: the dK/dV kernel fetches the
  // statistics of a whole 64-row chunk even where a sequence ends inside it
  const size_t floats = (size_t)heads * rows + 64;
  return 2 * (((floats * sizeof(float) + 255) / 256) * 256);
}

int s2_attn_bwd_varlen(const s2_layout* layout, const s2_tensors* t, const int32_t* cu_seqlens,
                       int32_t num_seqs, int32_t max_seqlen, float scale, void* workspace,
                       size_t workspace_bytes, void* stream) {
  if (!layout || !cu_seqlens) return S2_ERR_NULL;
  int st = check_tensors(t, true, scale);
  if (st != S2_OK) return st;
  if (t->batch != 1 || t->heads != layout->p.num_heads) return S2_ERR_SHAPE;
  if (num_seqs < 1 || max_seqlen < 1) return S2_ERR_SHAPE;
  if ((int64_t)max_seqlen > (int64_t)layout->p.num_blocks * layout->p.block_size) return S2_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(cu_seqlens) & 3u) != 0) return S2_ERR_ALIGN;
  const size_t need = s2_attn_bwd_varlen_workspace_bytes(t->heads, t->seqlen, t->head_dim);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 || workspace_bytes < need)
    return S2_ERR_WORKSPACE;
  if (!layout_on_current_device(layout)) return S2_ERR_NO_DEVICE;
  s2::AttnParams p = make_params(t, scale);
  p.batch = num_seqs;
  p.q_rows = max_seqlen;
  p.cu_seqlens = cu_seqlens;
  p.block_size = layout->p.block_size;
  set_tiles(p, layout);
  p.neg_delta = static_cast<float*>(workspace);
  p.neg_lse = p.neg_delta + need / 8;
  // one grid slot per (sequence, head, tile): query tiles of the longest length allowed, key tiles of the layout
  const int64_t pairs = 8 * (((int64_t)num_seqs * t->heads + 7) / 8);
  const int64_t slots = pairs * std::max<int64_t>((max_seqlen + s2::kBwdBM - 1) / s2::kBwdBM, layout->kv_tiles.tiles_per_head);
  if (slots > std::numeric_limits<int32_t>::max()) return S2_ERR_SHAPE;
  // (whole runs of key tiles can be a few more)
  if (s2::key_map(num_seqs * t->heads, layout->kv_tiles.tiles_per_head).grid() > std::numeric_limits<int32_t>::max()) return S2_ERR_SHAPE;
  return hip_ok(s2::launch_bwd(p, false, s2::kBwdAll, static_cast<hipStream_t>(stream))) ? S2_OK : S2_ERR_HIP;
}

int s2_attn_bwd_stages(const s2_layout* layout, const s2_tensors* t, float scale, void* workspace,
                       size_t workspace_bytes, int stages, void* stream) {
  if (!layout) return S2_ERR_NULL;
  if (stages < 1 || stages > S2_BWD_ALL) return S2_ERR_BAD_PARAM;
  int st = check_tensors(t, true, scale);
  if (st != S2_OK) return st;
  st = check_layout_fits(layout, t);
  if (st != S2_OK) return st;
  const BwdWorkspace w = bwd_workspace(t->batch, t->heads, t->seqlen, t->head_dim);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 || workspace_bytes < w.required())
    return S2_ERR_WORKSPACE;
  if (!layout_on_current_device(layout)) return S2_ERR_NO_DEVICE;
  s2::AttnParams p = make_params(t, scale);
  p.neg_delta = static_cast<float*>(workspace);
  p.neg_lse = p.neg_delta + w.stats / sizeof(float);
  p.block_size = layout->p.block_size;
  set_tiles(p, layout);
  unsigned char* const ws = static_cast<unsigned char*>(workspace);
  size_t used = w.required();
  // Room for dS selects the backward that computes nothing twice.  Where there is room for dS or for cutting
  // tiles but not for both, the workspace is of the size asked for cutting alone if that is the larger of the two.
  const size_t ds_bytes = (size_t)t->batch * (size_t)layout->ds_units * 8192;
  if (keeps_ds(layout, t->seqlen, t->head_dim) && workspace_bytes >= used + ds_bytes &&
      (workspace_bytes >= used + ds_bytes + w.cut() || workspace_bytes < used + w.cut() || ds_bytes > w.cut())) {
    p.ds_store = reinterpret_cast<uint16_t*>(ws + used);
    p.ds_units = layout->ds_units;
    p.dq_units = layout->d_dq_units;
    used += ds_bytes;
  }
  if (w.slots > 0 && workspace_bytes >= used + w.cut()) choose_split(p, layout, w, ws + used);
  return hip_ok(s2::launch_bwd(p, false, stages, static_cast<hipStream_t>(stream))) ? S2_OK : S2_ERR_HIP;
}

static int dense_params(const s2_tensors* t, s2::AttnParams& p) {
  if (t->seqlen % 128 != 0) return S2_ERR_SHAPE;
  p.block_size = s2::kChunk;
  p.q_tiles.tiles_per_head = t->seqlen / s2::kBwdBM;
  p.q_tiles.group = s2::kBwdBM / s2::kChunk;
  p.kv_tiles.tiles_per_head = t->seqlen / s2::kBwdBN;
  p.kv_tiles.group = s2::kBwdBN / s2::kChunk;
  return S2_OK;
}

int s2_dense_causal_fwd(const s2_tensors* t, float scale, void* stream) {
  int st = check_tensors(t, false, scale);
  if (st != S2_OK) return st;
  s2::AttnParams p = make_params(t, scale);
  st = dense_params(t, p);
  if (st != S2_OK) return st;
  return hip_ok(s2::launch_fwd(p, true, static_cast<hipStream_t>(stream))) ? S2_OK : S2_ERR_HIP;
}

int s2_dense_causal_bwd(const s2_tensors* t, float scale, void* workspace, size_t workspace_bytes,
                        void* stream) {
  int st = check_tensors(t, true, scale);
  if (st != S2_OK) return st;
  const BwdWorkspace w = bwd_workspace(t->batch, t->heads, t->seqlen, t->head_dim);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 || workspace_bytes < w.required())
    return S2_ERR_WORKSPACE;
  s2::AttnParams p = make_params(t, scale);
  st = dense_params(t, p);
  if (st != S2_OK) return st;
  p.neg_delta = static_cast<float*>(workspace);
  p.neg_lse = p.neg_delta + w.stats / sizeof(float);
  return hip_ok(s2::launch_bwd(p, true, s2::kBwdAll, static_cast<hipStream_t>(stream))) ? S2_OK : S2_ERR_HIP;
}

size_t s2_dense_causal_bwd_workspace_bytes(int32_t batch, int32_t heads, int32_t seqlen, int32_t head_dim) {
  if (batch < 1 || heads < 1 || seqlen < 1) return 0;
  return bwd_workspace(batch, heads, seqlen, head_dim).required();
}

int32_t s2_attn_decode_default_splits(int32_t nseq, int32_t heads, int32_t max_len) {
  if (nseq < 1 || heads < 1 || max_len < 1) return 1;
  // aim for a few workgroups per compute unit (256 CUs); never more splits than 1K-token pieces
  const int64_t pairs = (int64_t)nseq * heads;
  int64_t want = (4 * 256 + pairs - 1) / pairs;
  const int64_t cap = (max_len + 1023) / 1024;
  if (want > cap) want = cap;
  if (want < 1) want = 1;
  if (want > 64) want = 64;
  return (int32_t)want;
}

size_t s2_attn_decode_workspace_bytes(int32_t nseq, int32_t heads, int32_t head_dim, int32_t max_len,
                                      int32_t num_splits) {
  if (nseq < 1 || heads < 1 || head_dim < 1) return 0;
  if (num_splits <= 0) num_splits = s2_attn_decode_default_splits(nseq, heads, max_len);
  const size_t items = (size_t)nseq * heads * num_splits;
  return ((items * (head_dim + 2) * sizeof(float) + 255) / 256) * 256;
}

namespace {

bool good_block_size(int S) { return S == 16 || S == 32 || S == 64 || S == 128; }

// The pattern a decode call follows: the closed form of `lp`, or, when `layout` is given, the
// layout's own rows (then lp = &layout->p supplies S and the head count only).
int check_pattern(const s2_layout_params* lp, const s2_layout* layout, int heads, int64_t max_len) {
  if (!good_block_size(lp->block_size)) return S2_ERR_BAD_PARAM;
  if (heads != lp->num_heads) return S2_ERR_SHAPE;
  if (layout) {
    if (max_len > (int64_t)lp->num_blocks * lp->block_size) return S2_ERR_SHAPE;
    return layout_on_current_device(layout) ? S2_OK : S2_ERR_NO_DEVICE;
  }
  if (lp->dense != 0 && lp->dense != 1) return S2_ERR_BAD_PARAM;
  if (!lp->dense && (lp->local_blocks < 1 || lp->stride < 0 || lp->window_blocks < 0)) return S2_ERR_BAD_PARAM;
  if (lp->head_index_base < 0) return S2_ERR_BAD_PARAM;
  return S2_OK;
}

// Split count when the caller leaves it to the library; never more than the public default, which also
// sizes the workspace.  A trip of a workgroup's wavefronts, a unit each (64 tokens, or a block of 32), takes 1.5 to 2 us
// however few workgroups there are, the second launch that merges splits 2 to 3 us.  Three ranges:
//  - All of a call's workgroups are of eight wavefronts and fit the chip at once: one split is best up to three trips
//    (four at head_dim 64), then as many as still fit, down to one trip each: 32 pairs of 19 units 11.1 us in one
//    split, 11.5 in two; of 31 units 16.3 in one, 11.2 in four; 75 pairs of 34 units 14.2, 12.5 in three, 16.1 in four.
//    Where only one fits but leaves a third of the chip idle, three splits of four wavefronts share it better (160 pairs of 95
//    units 60.1 us in one, 55.4; of 47 units 29.8, 28.5; 192 pairs: 71.8, 78.6).  Long rows of many pairs are cut
//    into pieces of 24 units though not all fit: sequences of different lengths even out better, and equal ones lose
//    little.  From 384 units on where two fit (four in blocks of 32, whose units are half as large), from 512 where
//    one does: 96 pairs of 128 to 512 units x 128 179 us in two splits, 163 in eight, all of 384 203 and 206; 80 pairs of 256
//    to 1024 32-token units x 64 101 in three, 82 in twelve; 180 pairs of 128 to 512 x 128 370 in one, 350 in six.
//  - Above that (192 pairs, 256 in blocks of 16), up to 255 pairs: one split while rows are short, then pieces of a dozen units.  At
//    head_dim 128 from 256 units on (200 pairs of 64 to 256 units 204 us in one split, 179 in six, all of 384 411 and 414, but
//    all of 128 139 and 148), at 64 from 96 (all of 128 89 and 83, of 64 34 and 39), in blocks of 32 from 64 (of 64 x 128
//    47 in one, 39 in two; of 256 to 1024 x 64 470 in one, 176 in six).
//  - With more pairs the cache's bytes count, and splits must be worth their partials: a dozen units each at least (512
//    pairs, 19 units: 33.5 us in one split, 37.0 in two).
int choose_splits(const s2_layout_params* lp, const s2_layout* layout, int nseq, int heads, int head_dim, int max_len,
                  size_t workspace_bytes) {
  const int splits = s2_attn_decode_default_splits(nseq, heads, max_len);
  const int S = lp->block_size;
  const int64_t blocks = layout ? layout->max_row_blocks : s2::row_blocks(*lp, 0, (max_len - 1) / S, nullptr, 0);
  const int64_t units64 = blocks * S / 64;                // 64 tokens each
  const int64_t units = S == 32 ? blocks : units64;       // as the kernel counts them, in the longest row
  const int64_t pairs = (int64_t)nseq * heads;
  int64_t cap;
  const int64_t fit = s2::kDecodeWideGroups / pairs;  // splits of eight wavefronts that fit
  const int64_t few = S == 16 ? 256 : 192;                // the first range's pairs
  if (pairs >= 256 && pairs > few) {
    cap = units64 / 12;
  } else if (pairs > few) {
    cap = units >= (S == 32 ? 64 : head_dim == 64 ? 96 : 256) ? units / 12 : 1;
  } else if (units <= (head_dim == 128 ? 24 : 32)) {
    cap = 1;
  } else if (fit <= (S == 32 ? 4 : 2) && units >= (fit == 1 && S != 32 ? 512 : 384)) {
    cap = units / 24;
  } else {
    cap = std::min<int64_t>((units + 7) / 8, fit);
    if (cap == 1 && S != 16 && 3 * pairs <= 512) cap = 3;
  }
  int n = (int)std::max<int64_t>(1, std::min<int64_t>(splits, cap));
  // a workspace that holds the partials of a split to every 768 tokens is enough
  while (n > 1 && 12 * (int64_t)n > units64 && s2_attn_decode_workspace_bytes(nseq, heads, head_dim, max_len, n) > workspace_bytes) --n;
  return n;
}

extern "C++" template <class PARAMS>
void set_pattern(PARAMS& p, const s2_layout_params* lp, const s2_layout* layout) {
  p.block_size = lp->block_size;
  p.local_blocks = lp->local_blocks;
  p.stride = lp->stride;
  p.window_blocks = lp->window_blocks;
  p.dense = lp->dense;
  p.head_index_base = lp->head_index_base;
  if (layout) {
    p.row_ptr = layout->d_row_ptr;
    p.col_idx = layout->d_col_idx;
    p.num_blocks = lp->num_blocks;
  }
}

// Where the arrays of a plan lie in its workspace: the new tokens of 256 sequences each come first.
struct PlanWorkspace {
  size_t seq, pair, group, state, bytes;
};
PlanWorkspace plan_workspace(const s2::KvPlanParams& p) {
  PlanWorkspace w;
  auto after = [](size_t at, size_t bytes) { return (at + bytes + 255) / 256 * 256; };
  w.seq = after(0, ((size_t)p.nseq + 255) / 256 * sizeof(int64_t));
  w.pair = after(w.seq, (size_t)p.nseq * 4 * sizeof(int32_t));
  w.group = after(w.pair, (size_t)p.pairs * 2 * sizeof(int32_t));
  w.state = after(w.group, (size_t)p.groups * 2 * sizeof(int32_t));
  w.bytes = after(w.state, 2 * sizeof(int32_t));
  return w;
}

int decode_contiguous(const s2_layout_params* lp, const s2_layout* layout, const s2_decode_args* a, float scale,
                      void* workspace, size_t workspace_bytes, void* stream) {
  if (!a->q || !a->k_cache || !a->v_cache || !a->seq_lens || !a->o) return S2_ERR_NULL;
  if (!(scale > 0.f) || !std::isfinite(scale)) return S2_ERR_BAD_PARAM;
  if (a->nseq < 1 || a->heads < 1 || a->max_len < 1) return S2_ERR_SHAPE;
  if (a->head_dim != 64 && a->head_dim != 128) return S2_ERR_SHAPE;
  int st = check_pattern(lp, layout, a->heads, a->max_len);
  if (st != S2_OK) return st;
  if (a->num_splits < 0 || a->num_splits > 64) return S2_ERR_BAD_PARAM;
  const int64_t strides[3] = {a->kv_stride_seq, a->kv_stride_head, a->kv_stride_tok};
  for (int64_t s : strides)
    if (s < 0 || (s & 7) != 0) return S2_ERR_ALIGN;
  if (a->kv_stride_tok < a->head_dim) return S2_ERR_ALIGN;
  if (!aligned16(a->q) || !aligned16(a->k_cache) || !aligned16(a->v_cache) || !aligned16(a->o) ||
      (reinterpret_cast<uintptr_t>(a->seq_lens) & 3u) != 0)
    return S2_ERR_ALIGN;
  const int splits = a->num_splits > 0 ? a->num_splits : choose_splits(lp, layout, a->nseq, a->heads, a->head_dim, a->max_len, workspace_bytes);
  const size_t need = s2_attn_decode_workspace_bytes(a->nseq, a->heads, a->head_dim, a->max_len, splits);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 || workspace_bytes < need)
    return S2_ERR_WORKSPACE;

  s2::DecodeParams p{};
  p.q = static_cast<const uint16_t*>(a->q);
  p.k_cache = static_cast<const uint16_t*>(a->k_cache);
  p.v_cache = static_cast<const uint16_t*>(a->v_cache);
  p.seq_lens = a->seq_lens;
  p.o = static_cast<uint16_t*>(a->o);
  p.lse = a->lse;
  const size_t items = (size_t)a->nseq * a->heads * splits;
  p.part_acc = static_cast<float*>(workspace);
  p.part_ml = p.part_acc + items * a->head_dim;
  p.nseq = a->nseq;
  p.heads = a->heads;
  p.head_dim = a->head_dim;
  p.max_len = a->max_len;
  p.num_splits = splits;
  p.q_ss = (int64_t)a->heads * a->head_dim;
  p.q_sh = a->head_dim;
  p.kv_ss = a->kv_stride_seq;
  p.kv_sh = a->kv_stride_head;
  p.kv_st = a->kv_stride_tok;
  p.scale = scale;
  p.scale_log2e = scale * 1.4426950408889634f;
  set_pattern(p, lp, layout);
  return hip_ok(s2::launch_decode(p, static_cast<hipStream_t>(stream))) ? S2_OK : S2_ERR_HIP;
}

// (q and o: element (b, h, d) at b * q_ss + h * q_sh + d)
int decode_paged(const s2_layout_params* lp, const s2_layout* layout, const s2_paged_decode_args* a, int64_t q_ss, int64_t q_sh, float scale,
                 void* workspace, size_t workspace_bytes, void* stream) {
  if (!a->q || !a->k_pages || !a->v_pages || !a->block_table || !a->seq_lens || !a->o) return S2_ERR_NULL;
  if (!(scale > 0.f) || !std::isfinite(scale)) return S2_ERR_BAD_PARAM;
  if (!good_block_size(lp->block_size)) return S2_ERR_BAD_PARAM;
  if (a->nseq < 1 || a->heads < 1 || a->max_blocks < 1 || a->num_pages < 1) return S2_ERR_SHAPE;
  if ((int64_t)a->max_blocks * lp->block_size > std::numeric_limits<int32_t>::max()) return S2_ERR_SHAPE;
  if (a->head_dim != 64 && a->head_dim != 128) return S2_ERR_SHAPE;
  const int max_len = a->max_blocks * lp->block_size;
  int st = check_pattern(lp, layout, a->heads, max_len);
  if (st != S2_OK) return st;
  if (a->num_splits < 0 || a->num_splits > 64) return S2_ERR_BAD_PARAM;
  if (a->page_stride < 0 || (a->page_stride & 7) != 0 || a->tok_stride < 0 || (a->tok_stride & 7) != 0)
    return S2_ERR_ALIGN;
  if (a->tok_stride < a->head_dim) return S2_ERR_ALIGN;
  if (!aligned16(a->q) || !aligned16(a->k_pages) || !aligned16(a->v_pages) || !aligned16(a->o) ||
      (reinterpret_cast<uintptr_t>(a->seq_lens) & 3u) != 0 ||
      (reinterpret_cast<uintptr_t>(a->block_table) & 3u) != 0 ||
      (reinterpret_cast<uintptr_t>(a->missing) & 3u) != 0)
    return S2_ERR_ALIGN;
  const int splits = a->num_splits > 0 ? a->num_splits : choose_splits(lp, layout, a->nseq, a->heads, a->head_dim, max_len, workspace_bytes);
  const size_t need = s2_attn_decode_workspace_bytes(a->nseq, a->heads, a->head_dim, max_len, splits);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 || workspace_bytes < need)
    return S2_ERR_WORKSPACE;

  s2::DecodeParams p{};
  p.q = static_cast<const uint16_t*>(a->q);
  p.k_cache = static_cast<const uint16_t*>(a->k_pages);
  p.v_cache = static_cast<const uint16_t*>(a->v_pages);
  p.seq_lens = a->seq_lens;
  p.o = static_cast<uint16_t*>(a->o);
  p.lse = a->lse;
  const size_t items = (size_t)a->nseq * a->heads * splits;
  p.part_acc = static_cast<float*>(workspace);
  p.part_ml = p.part_acc + items * a->head_dim;
  p.nseq = a->nseq;
  p.heads = a->heads;
  p.head_dim = a->head_dim;
  p.max_len = max_len;
  p.num_splits = splits;
  p.q_ss = q_ss;
  p.q_sh = q_sh;
  p.kv_ss = a->page_stride;
  p.kv_sh = 0;
  p.kv_st = a->tok_stride;
  p.scale = scale;
  p.scale_log2e = scale * 1.4426950408889634f;
  set_pattern(p, lp, layout);
  p.block_table = a->block_table;
  p.missing = a->missing;
  p.max_blocks = a->max_blocks;
  p.num_pages = a->num_pages;
  return hip_ok(s2::launch_decode(p, static_cast<hipStream_t>(stream))) ? S2_OK : S2_ERR_HIP;
}

// A paged cache of any format, with strides in bytes.
int check_cache(const s2_paged_cache* c, s2::CacheRef& r) {
  if (!c->k_pages || !c->v_pages || !c->block_table) return S2_ERR_NULL;
  if (c->format != S2_KV_BF16 && c->format != S2_KV_MXFP8 && c->format != S2_KV_MXFP4) return S2_ERR_BAD_PARAM;
  if (!good_block_size(c->block_size)) return S2_ERR_BAD_PARAM;
  if (c->format != S2_KV_BF16 && (!c->k_scales || !c->v_scales)) return S2_ERR_NULL;
  if (c->nseq < 1 || c->heads < 1 || c->max_blocks < 1 || c->num_pages < 1) return S2_ERR_SHAPE;
  if (c->head_dim != 64 && c->head_dim != 128) return S2_ERR_SHAPE;
  if ((int64_t)c->nseq * c->heads > std::numeric_limits<int32_t>::max() / 64) return S2_ERR_SHAPE;
  // (positions of a tree's nodes go up to 64 beyond the last)
  if ((int64_t)c->max_blocks * c->block_size > std::numeric_limits<int32_t>::max() - 64) return S2_ERR_SHAPE;
  const int64_t element = c->format == S2_KV_BF16 ? 2 : 1;
  const int64_t row = c->format == S2_KV_BF16 ? 2 * c->head_dim : c->format == S2_KV_MXFP8 ? c->head_dim : c->head_dim / 2;
  if (!aligned16(c->k_pages) || !aligned16(c->v_pages) || (reinterpret_cast<uintptr_t>(c->block_table) & 3u) != 0) return S2_ERR_ALIGN;
  if (c->page_stride < 0 || c->page_stride % (16 / element) != 0 || c->tok_stride < 0 || c->tok_stride % (16 / element) != 0) return S2_ERR_ALIGN;
  if (c->tok_stride * element < row) return S2_ERR_ALIGN;
  // the kernels address a page's rows with 32-bit byte offsets
  constexpr int64_t kPage = (int64_t)1 << 30;
  if (c->tok_stride > kPage / element / c->block_size || c->page_stride > ((int64_t)1 << 56)) return S2_ERR_SHAPE;
  r = s2::CacheRef{};
  if (c->format != S2_KV_BF16) {
    const int64_t scales = c->head_dim / 32;
    if ((reinterpret_cast<uintptr_t>(c->k_scales) & 3u) != 0 || (reinterpret_cast<uintptr_t>(c->v_scales) & 3u) != 0) return S2_ERR_ALIGN;
    if (c->scale_page_stride < 0 || c->scale_page_stride % scales != 0 || c->scale_tok_stride < scales || c->scale_tok_stride % scales != 0)
      return S2_ERR_ALIGN;
    if (c->scale_tok_stride > kPage / c->block_size || c->scale_page_stride > ((int64_t)1 << 56)) return S2_ERR_SHAPE;
    r.ks = static_cast<uint8_t*>(c->k_scales);
    r.vs = static_cast<uint8_t*>(c->v_scales);
    r.scale_page = c->scale_page_stride;
    r.scale_tok = (int)c->scale_tok_stride;
  }
  r.k = static_cast<uint8_t*>(c->k_pages);
  r.v = static_cast<uint8_t*>(c->v_pages);
  r.table = c->block_table;
  r.page = c->page_stride * element;
  r.tok = (int)(c->tok_stride * element);
  r.format = c->format;
  r.heads = c->heads;
  r.head_dim = c->head_dim;
  r.max_blocks = c->max_blocks;
  r.num_pages = c->num_pages;
  r.block_shift = 31 - __builtin_clz((unsigned)c->block_size);
  return S2_OK;
}

// What s2_kv_append_paged and s2_kv_read_paged have in common, and the launch.
int cache_rows(s2::KvRowsParams& p, const s2_paged_cache* c, const void* k, const void* v, void* stream) {
  if (!p.cu || !p.start) return S2_ERR_NULL;
  if (p.num_rows < 0 || p.max_rows < 0) return S2_ERR_SHAPE;
  if (p.num_rows > 0 && (!k || !v)) return S2_ERR_NULL;
  if (!aligned16(k) || !aligned16(v) || (reinterpret_cast<uintptr_t>(p.cu) & 3u) != 0 || (reinterpret_cast<uintptr_t>(p.start) & 3u) != 0)
    return S2_ERR_ALIGN;
  if (p.stride_row < 0 || (p.stride_row & 7) != 0 || p.stride_head < 0 || (p.stride_head & 7) != 0) return S2_ERR_ALIGN;
  if (p.stride_row > (int64_t)1 << 40 || p.stride_head > (int64_t)1 << 40) return S2_ERR_SHAPE;
  p.nseq = c->nseq;
  p.bound = p.rows ? p.num_items : p.num_rows;
  // (items beyond the last row or index are none that is moved; they are counted, in 32 bits)
  if (!p.skipped) p.max_rows = std::min(p.max_rows, p.bound);
  if (p.skipped && p.max_rows > std::numeric_limits<int32_t>::max() / ((int64_t)c->nseq * c->heads)) return S2_ERR_SHAPE;
  if (p.max_rows == 0) return S2_OK;
  if (s2::kv_rows_groups(p) > s2::kMostGroups) return S2_ERR_SHAPE;
  return hip_ok(s2::launch_kv_rows(p, static_cast<hipStream_t>(stream))) ? S2_OK : S2_ERR_HIP;
}

// The most splits that the library takes for a call over a cache of any format.
int most_cache_splits(int64_t pairs, int64_t max_len) {
  return (int)std::max<int64_t>(1, std::min<int64_t>({64, (1024 + pairs - 1) / pairs, (max_len + 127) / 128}));
}

// The splits of a call over a cache when the caller leaves them to the library.
// A decode step over 8 or 4 bits: as many workgroups of eight wavefronts as there are compute units, while each wavefront but one in four has a unit of 64
// tokens (e4m3, D = 128, us: 8 heads of 47 units in 4 splits 13.2, 8 10.0, 16 9.0; 32 in 4 13.6, 8 11.2, 16 11.5; of 19 units in 4 10.1, 8 8.7, 16 10.3;
// 64 of 31 to 46 units in 2 20.0, 4 15.3, 8 15.7), and else four workgroups of four to a compute unit where that leaves 24 units to each (512
// of up to 46 units in one split 62.6, in two 65.6).
// Trees of up to 32 nodes: a workgroup to a compute unit, and three units to it (it takes two at a time; bf16, D = 128, 8 nodes, us: 32 pairs of 47 units in 4
// splits 19.7, 8 16.3, 12 18.7, 16 16.5; e4m3: 8 of 47 in 6 13.5, 16 11.1, 32 11.4; 16 nodes, 256 of 46 in one 39.6, in two 41.7).  From 129 to 255 pairs that is
// one split, which long rows over 8 bits would rather have in more: in 1, 2 and 3, 8 nodes, 160 pairs of 46 units bf16 50, 54, 48, e4m3 36, 32, 29; of 21 units 27, 31, 27
// and 19, 20, 20; 224 of 46 58, 59, 63 and 38, 37, 38.
// Larger ones, whose workgroups take a unit at a time between two barriers: two to a compute unit, and two units to each (64 nodes, bf16: 32 pairs of
// 47 units in 4 31.6, 8 23.1, 16 22.8, 24 26.2; 40 nodes, e2m1: 4 of 47 in 12 15.1, 24 12.6, 32 13.5; 33 nodes, D = 64: 91 of 9 in 2 19.7, 6 16.6, 8 17.9).
int choose_cache_splits(const s2_layout_params* lp, const s2_layout* layout, int nodes, int nseq, int heads, int max_len) {
  const int S = lp->block_size;
  const int64_t blocks = layout ? layout->max_row_blocks : s2::row_blocks(*lp, 0, (max_len - 1) / S, nullptr, 0);
  const int64_t units = (blocks * S + 63) / 64, pairs = (int64_t)nseq * heads;
  const int64_t want = nodes > 32  ? std::min<int64_t>((512 + pairs - 1) / pairs, units / 2)
                       : nodes > 0 ? std::min<int64_t>(256 / pairs, units / 3)
                                   : std::max(std::min<int64_t>(s2::kCacheWideGroups / pairs, units / 2), std::min<int64_t>(1024 / pairs, units / 24));
  return (int)std::max<int64_t>(1, std::min<int64_t>(want, most_cache_splits(pairs, max_len)));
}

// A tree, or (without parents) a decode step over 8 or 4 bits.
int attend_cache(const s2_layout_params* lp, const s2_layout* layout, const s2_paged_cache* c, s2::CacheAttnParams& p, float scale,
                 int num_splits, void* workspace, size_t workspace_bytes, void* stream) {
  if (!p.q || !p.seq_lens || !p.o) return S2_ERR_NULL;
  if (!(scale > 0.f) || !std::isfinite(scale)) return S2_ERR_BAD_PARAM;
  int st = check_cache(c, p.c);
  if (st != S2_OK) return st;
  if (lp->block_size != c->block_size) return S2_ERR_SHAPE;
  const int max_len = c->max_blocks * c->block_size;
  st = check_pattern(lp, layout, c->heads, max_len);
  if (st != S2_OK) return st;
  if (num_splits < 0 || num_splits > 64) return S2_ERR_BAD_PARAM;
  for (int64_t s : {p.q_ss, p.q_sh, p.q_sn, p.kv_ss, p.kv_sh, p.kv_sn}) {
    if (s < 0 || (s & 7) != 0) return S2_ERR_ALIGN;
    if (s > (int64_t)1 << 40) return S2_ERR_SHAPE;
  }
  if (!aligned16(p.q) || !aligned16(p.k_draft) || !aligned16(p.v_draft) || !aligned16(p.o) || (reinterpret_cast<uintptr_t>(p.seq_lens) & 3u) != 0 ||
      (reinterpret_cast<uintptr_t>(p.parents) & 3u) != 0 || (reinterpret_cast<uintptr_t>(p.lse) & 3u) != 0 ||
      (reinterpret_cast<uintptr_t>(p.missing) & 3u) != 0)
    return S2_ERR_ALIGN;
  int splits = num_splits > 0 ? num_splits : choose_cache_splits(lp, layout, p.parents ? p.nodes : 0, c->nseq, c->heads, max_len);
  const int64_t pairs = (int64_t)c->nseq * c->heads;
  if (pairs * splits > s2::kMostGroups || (pairs * p.nodes + 3) / 4 > s2::kMostGroups) return S2_ERR_SHAPE;
  auto bytes = [&](int n) { return s2_attn_tree_workspace_bytes(c->nseq, c->heads, p.nodes, c->head_dim, max_len, n); };
  // (a smaller workspace is for fewer splits, where the caller has not asked for a number)
  while (num_splits == 0 && splits > 1 && bytes(splits) > workspace_bytes) --splits;
  const size_t need = bytes(splits);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 || workspace_bytes < need) return S2_ERR_WORKSPACE;
  p.part_acc = static_cast<float*>(workspace);
  p.part_ml = p.part_acc + (size_t)c->nseq * c->heads * p.nodes * splits * c->head_dim;
  p.nseq = c->nseq;
  p.heads = c->heads;
  p.max_len = max_len;
  p.num_splits = splits;
  p.scale = scale;
  p.scale_log2e = scale * 1.4426950408889634f;
  set_pattern(p, lp, layout);
  return hip_ok(s2::launch_cache_attn(p, static_cast<hipStream_t>(stream))) ? S2_OK : S2_ERR_HIP;
}

int decode_cache(const s2_layout_params* lp, const s2_layout* layout, const s2_paged_cache* c, const s2_cache_decode_args* a, float scale,
                 void* workspace, size_t workspace_bytes, void* stream) {
  if (c->format == S2_KV_BF16) {
    if (c->block_size != lp->block_size) return S2_ERR_SHAPE;
    if ((int64_t)c->nseq * c->heads > std::numeric_limits<int32_t>::max() / 64) return S2_ERR_SHAPE;
    const int64_t ss = c->nseq == 1 ? 0 : a->q_stride_seq, sh = c->heads == 1 ? 0 : a->q_stride_head;  // (of one there is no next)
    if (ss < 0 || (ss & 7) != 0 || sh < 0 || (sh & 7) != 0 || (reinterpret_cast<uintptr_t>(a->lse) & 3u) != 0) return S2_ERR_ALIGN;
    if (ss > (int64_t)1 << 40 || sh > (int64_t)1 << 40) return S2_ERR_SHAPE;
    s2_paged_decode_args d{};
    d.q = a->q;
    d.k_pages = c->k_pages;
    d.v_pages = c->v_pages;
    d.block_table = c->block_table;
    d.seq_lens = a->seq_lens;
    d.o = a->o;
    d.lse = a->lse;
    d.missing = a->missing;
    d.nseq = c->nseq;
    d.heads = c->heads;
    d.head_dim = c->head_dim;
    d.max_blocks = c->max_blocks;
    d.num_pages = c->num_pages;
    d.num_splits = a->num_splits;
    d.page_stride = c->page_stride;
    d.tok_stride = c->tok_stride;
    int st = decode_paged(lp, layout, &d, ss, sh, scale, workspace, workspace_bytes, stream);
    if (st == S2_ERR_WORKSPACE && a->num_splits == 0) {
      // (a smaller workspace is for fewer splits, as below)
      auto bytes = [&](int n) { return s2_attn_decode_workspace_bytes(c->nseq, c->heads, c->head_dim, c->max_blocks * c->block_size, n); };
      d.num_splits = s2_attn_decode_default_splits(c->nseq, c->heads, c->max_blocks * c->block_size);
      while (d.num_splits > 1 && bytes(d.num_splits) > workspace_bytes) --d.num_splits;
      st = decode_paged(lp, layout, &d, ss, sh, scale, workspace, workspace_bytes, stream);
    }
    return st;
  }
  s2::CacheAttnParams p{};
  p.q = static_cast<const uint16_t*>(a->q);
  p.seq_lens = a->seq_lens;
  p.o = static_cast<uint16_t*>(a->o);
  p.lse = a->lse;
  p.missing = a->missing;
  p.nodes = 1;
  p.q_ss = a->q_stride_seq;
  p.q_sh = a->q_stride_head;
  return attend_cache(lp, layout, c, p, scale, a->num_splits, workspace, workspace_bytes, stream);
}

int tree_cache(const s2_layout_params* lp, const s2_layout* layout, const s2_paged_cache* c, const s2_tree_args* a, float scale,
               void* workspace, size_t workspace_bytes, void* stream) {
  if (!a->k || !a->v || !a->parents) return S2_ERR_NULL;
  if (a->nodes < 1 || a->nodes > 64) return S2_ERR_SHAPE;
  s2::CacheAttnParams p{};
  p.q = static_cast<const uint16_t*>(a->q);
  p.k_draft = static_cast<const uint16_t*>(a->k);
  p.v_draft = static_cast<const uint16_t*>(a->v);
  p.parents = a->parents;
  p.seq_lens = a->seq_lens;
  p.o = static_cast<uint16_t*>(a->o);
  p.lse = a->lse;
  p.missing = a->missing;
  p.nodes = a->nodes;
  p.q_ss = a->q_stride_seq;
  p.q_sh = a->q_stride_head;
  p.q_sn = a->q_stride_node;
  p.kv_ss = a->kv_stride_seq;
  p.kv_sh = a->kv_stride_head;
  p.kv_sn = a->kv_stride_node;
  return attend_cache(lp, layout, c, p, scale, a->num_splits, workspace, workspace_bytes, stream);
}

// Rows of a tensor: n of them, `stride` elements apart, for each of its dimensions but the last.
struct Steps {
  int64_t n, stride;
};
// Whether so many steps of each stride (fewer than n, either way; strides in descending order, none 0) lead to less than `row` elements from -offset.
bool steps_meet(const Steps* s, int count, int64_t row, __int128 offset) {
  if (count == 0) return offset > -row && offset < row;
  __int128 reach = row - 1;
  for (int i = 1; i < count; ++i) reach += (__int128)(s[i].n - 1) * s[i].stride;
  // (what is further away the other strides cannot make up for)
  auto floor_of = [&](__int128 x) { return x < 0 ? -((-x + s[0].stride - 1) / s[0].stride) : x / s[0].stride; };
  const __int128 lo = std::max<__int128>(-floor_of(reach + offset), 1 - s[0].n), hi = std::min<__int128>(floor_of(reach - offset), s[0].n - 1);
  for (__int128 k = lo; k <= hi; ++k)
    if (steps_meet(s + 1, count - 1, row, offset + k * s[0].stride)) return true;
  return false;
}
// Whether two rows of `row` elements share one, as those of a broadcast dimension do: of what is written none may (it would hold what came last).
bool rows_overlap(int64_t row, std::initializer_list<Steps> dims) {
  Steps s[3];
  int count = 0;
  for (const Steps& d : dims)
    if (d.n > 1) s[count++] = d;
  std::sort(s, s + count, [](const Steps& a, const Steps& b) { return a.stride > b.stride; });
  // each stride beyond all that the smaller ones reach: as nearly all tensors lie
  __int128 extent = row;
  int i = count - 1;
  for (; i >= 0 && s[i].stride >= extent; --i) extent += (__int128)(s[i].n - 1) * s[i].stride;
  if (i < 0) return false;
  if (s[count - 1].stride < row) return true;
  for (; i >= 0; --i) {  // (two rows whose first difference is k steps of stride i)
    __int128 reach = row - 1;
    for (int j = i + 1; j < count; ++j) reach += (__int128)(s[j].n - 1) * s[j].stride;
    for (__int128 k = 1; k < s[i].n && k * s[i].stride <= reach; ++k)
      if (steps_meet(s + i + 1, count - i - 1, row, k * s[i].stride)) return true;
  }
  return false;
}

// The most splits that the library takes for a chunk: units of 64 tokens go two to a split, and the workgroups of the tiles that sequences fill a workgroup to a
// compute unit, or two of the kernel for 33 to 64 rows, whose wavefronts wait for each other.  bf16, head_dim 128, 44 units for a query, us by splits:
//   256 rows, 32 heads (64 tiles)    1: 73  2: 49  4: 36  6: 39  8: 38  16: 52      4 x 256 rows, 32 heads (256)   1: 76  2: 79  4: 89
//   16 rows, 32 heads                1: 30  4: 17  8: 13.9  12: 15.1  16: 15.3      48 rows, 32 heads              1: 74  8: 21.4  16: 21.0  24: 21.7
//   4 x 48 rows, 32 heads            1: 74  2: 48  4: 37  6: 36  8: 41              and 12 units, 16 rows, 8 heads 1: 12.6  4: 11.8  6: 10.7  12: 11.2
int most_chunk_splits(const s2::CacheChunkParams& p, int64_t max_len) {
  const int64_t rows = (int64_t)1 << p.tile_shift, fill = p.max_new > 32 && p.max_new <= s2::kChunkFew ? 512 : 256;
  const int64_t groups = p.heads * std::min((p.max_new + rows - 1) / rows * p.nseq, p.num_rows / rows + p.nseq);
  return (int)std::max<int64_t>(1, std::min<int64_t>({64, (fill + groups / 2) / groups, (max_len + 127) / 128}));
}

// (the fields that decide the launch's size)
s2::CacheChunkParams chunk_sizes(int nseq, int heads, int max_new, int num_rows) {
  s2::CacheChunkParams p{};
  p.nseq = nseq;
  p.heads = heads;
  p.num_rows = num_rows;
  p.max_new = std::min(max_new, num_rows);
  return p;
}

int chunk_cache(const s2_layout_params* lp, const s2_layout* layout, const s2_paged_cache* c, const s2_chunk_args* a, float scale, void* workspace,
                size_t workspace_bytes, void* stream) {
  if (!a->cu_new || !a->start) return S2_ERR_NULL;
  if (!(scale > 0.f) || !std::isfinite(scale)) return S2_ERR_BAD_PARAM;
  s2::CacheRef cache;
  int st = check_cache(c, cache);
  if (st != S2_OK) return st;
  if (lp->block_size != c->block_size) return S2_ERR_SHAPE;
  const int max_len = c->max_blocks * c->block_size;
  st = check_pattern(lp, layout, c->heads, max_len);
  if (st != S2_OK) return st;
  if (a->num_splits < 0 || a->num_splits > 64) return S2_ERR_BAD_PARAM;
  if (a->num_rows < 0 || a->max_new < 0) return S2_ERR_SHAPE;
  if (a->num_rows > 0 && (!a->q || !a->o)) return S2_ERR_NULL;
  for (int64_t s : {a->q_stride_row, a->q_stride_head}) {
    if (s < 0 || (s & 7) != 0) return S2_ERR_ALIGN;
    if (s > (int64_t)1 << 40) return S2_ERR_SHAPE;
  }
  if (!aligned16(a->q) || !aligned16(a->o)) return S2_ERR_ALIGN;
  for (const void* x : {(const void*)a->cu_new, (const void*)a->start, (const void*)a->lse, (const void*)a->missing})
    if ((reinterpret_cast<uintptr_t>(x) & 3u) != 0) return S2_ERR_ALIGN;
  s2::CacheChunkParams p = chunk_sizes(c->nseq, c->heads, a->max_new, a->num_rows);
  if (p.max_new == 0) return S2_OK;
  if (rows_overlap(c->head_dim, {{a->num_rows, a->q_stride_row}, {c->heads, a->q_stride_head}})) return S2_ERR_SHAPE;
  const int64_t groups = s2::chunk_tiles(p) * c->heads;
  if (groups > s2::kMostGroups) return S2_ERR_SHAPE;
  const int64_t blocks = layout ? layout->max_row_blocks : s2::row_blocks(*lp, 0, (max_len - 1) / c->block_size, nullptr, 0);
  const int64_t units = (blocks * c->block_size + 63) / 64;
  int splits = a->num_splits > 0 ? a->num_splits : (int)std::max<int64_t>(1, std::min<int64_t>(most_chunk_splits(p, max_len), (units + 1) / 2));
  auto bytes = [&](int n) { return n == 1 ? 0 : s2_attn_chunk_workspace_bytes(c->nseq, c->heads, a->max_new, a->num_rows, c->head_dim, max_len, n); };
  // (a smaller workspace is for fewer splits, where the caller has not asked for a number)
  while (a->num_splits == 0 && splits > 1 && (!workspace || bytes(splits) > workspace_bytes)) --splits;
  if (splits > 1 && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 || workspace_bytes < bytes(splits))) return S2_ERR_WORKSPACE;
  const int64_t rows = (int64_t)c->nseq * c->heads * p.max_new;
  if (groups * splits > s2::kMostGroups || (splits > 1 && (rows + 3) / 4 > s2::kMostGroups)) return S2_ERR_SHAPE;
  p.c = cache;
  p.q = static_cast<const uint16_t*>(a->q);
  p.cu = a->cu_new;
  p.start = a->start;
  p.o = static_cast<uint16_t*>(a->o);
  p.lse = a->lse;
  p.missing = a->missing;
  p.part_acc = static_cast<float*>(workspace);
  p.part_ml = splits > 1 ? p.part_acc + (size_t)rows * splits * c->head_dim : nullptr;
  p.max_len = max_len;
  p.num_splits = splits;
  p.q_sr = a->q_stride_row;
  p.q_sh = a->q_stride_head;
  p.scale = scale;
  p.scale_log2e = scale * 1.4426950408889634f;
  set_pattern(p, lp, layout);
  return hip_ok(s2::launch_cache_chunk(p, static_cast<hipStream_t>(stream))) ? S2_OK : S2_ERR_HIP;
}

int kv_plan(const s2_layout_params* lp, const s2_layout* layout, const s2_kv_plan_args* a, void* workspace, size_t workspace_bytes, void* stream) {
  if (!a->block_table || !a->lens || !a->new_lens || !a->free_pages || !a->free_state || !a->new_table || !a->new_free_pages || !a->new_free_state)
    return S2_ERR_NULL;
  if (!good_block_size(lp->block_size)) return S2_ERR_BAD_PARAM;
  if (a->nseq < 1 || a->heads < 1 || a->max_blocks < 1 || a->num_pages < 1) return S2_ERR_SHAPE;
  if (a->positions && a->num_rows < 0) return S2_ERR_SHAPE;
  const int64_t pairs = (int64_t)a->nseq * a->heads, max_len = (int64_t)a->max_blocks * lp->block_size;
  if (pairs > std::numeric_limits<int32_t>::max() / 64 || max_len > std::numeric_limits<int32_t>::max() - 64) return S2_ERR_SHAPE;
  const int st = check_pattern(lp, layout, a->heads, max_len);
  if (st != S2_OK) return st;
  for (const void* x : {(const void*)a->block_table, (const void*)a->lens, (const void*)a->new_lens, (const void*)a->query_from, (const void*)a->free_pages,
                        (const void*)a->free_state, (const void*)a->new_table, (const void*)a->new_free_pages, (const void*)a->new_free_state,
                        (const void*)a->cu_new, (const void*)a->positions, (const void*)a->seq_lens, (const void*)a->short_of})
    if ((reinterpret_cast<uintptr_t>(x) & 3u) != 0) return S2_ERR_ALIGN;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 || workspace_bytes < s2_kv_plan_workspace_bytes(a->nseq, a->heads))
    return S2_ERR_WORKSPACE;
  s2::KvPlanParams p{};
  p.table = a->block_table;
  p.lens = a->lens;
  p.new_lens = a->new_lens;
  p.query_from = a->query_from;
  p.ring = a->free_pages;
  p.free_state = a->free_state;
  p.new_table = a->new_table;
  p.new_ring = a->new_free_pages;
  p.new_state = a->new_free_state;
  p.cu_new = a->cu_new;
  p.positions = a->positions;
  p.seq_lens = a->seq_lens;
  p.short_of = a->short_of;
  p.pairs = pairs;
  p.nseq = a->nseq;
  p.heads = a->heads;
  p.max_blocks = a->max_blocks;
  p.max_len = (int)max_len;
  p.num_pages = a->num_pages;
  p.num_rows = a->num_rows;
  p.block_shift = 31 - __builtin_clz((unsigned)lp->block_size);
  p.apart = a->new_table != a->block_table;
  set_pattern(p, lp, layout);
  if (layout) p.last_row = layout->d_last_row;
  s2::plan_groups(p);
  if (p.groups + (int64_t)a->nseq + a->num_pages / s2::kRingEach + 1 > s2::kMostGroups) return S2_ERR_SHAPE;
  const PlanWorkspace w = plan_workspace(p);
  char* const at = static_cast<char*>(workspace);
  p.ws_fresh = reinterpret_cast<int64_t*>(at);
  p.ws_seq = reinterpret_cast<int32_t*>(at + w.seq);
  p.ws_pair = reinterpret_cast<int32_t*>(at + w.pair);
  p.ws_group = reinterpret_cast<int32_t*>(at + w.group);
  p.ws_state = reinterpret_cast<int32_t*>(at + w.state);
  return hip_ok(s2::launch_kv_plan(p, static_cast<hipStream_t>(stream))) ? S2_OK : S2_ERR_HIP;
}

// What s2_qk_norm_rope_fwd and _bwd have in common.
int qk_rope(const s2_qk_norm_rope_args* a, bool bwd, s2::QkRopeParams& p) {
  if (!a->q && !a->k) return S2_ERR_NULL;
  const void* const x[2] = {a->q, a->k};
  void* const out[2] = {bwd ? a->dq : a->q_out, bwd ? a->dk : a->k_out};
  const void* const g[2] = {a->d_q_out, a->d_k_out};
  const float* const weight[2] = {a->q_weight, a->k_weight};
  float* const d_weight[2] = {a->dq_weight, a->dk_weight};
  for (int i = 0; i < 2; ++i)
    if (x[i] && (!out[i] || (bwd && (!g[i] || (weight[i] && !d_weight[i]))))) return S2_ERR_NULL;
  if (a->rotary_dim > 0 && !a->inv_freq) return S2_ERR_NULL;
  if (!(a->eps >= 0.f) || !std::isfinite(a->eps) || (a->interleaved != 0 && a->interleaved != 1)) return S2_ERR_BAD_PARAM;
  if (a->batch < 1 || a->heads < 1 || a->seqlen < 0) return S2_ERR_SHAPE;
  if (a->head_dim != 64 && a->head_dim != 128) return S2_ERR_SHAPE;
  if (a->rotary_dim < 0 || a->rotary_dim > a->head_dim || a->rotary_dim % 16 != 0) return S2_ERR_SHAPE;
  const int64_t rows = (int64_t)a->batch * a->seqlen;
  if (rows > s2::kMostGroups || rows * a->heads > std::numeric_limits<int32_t>::max()) return S2_ERR_SHAPE;
  for (int64_t s : {a->in_stride_b, a->in_stride_h, a->in_stride_t, a->out_stride_b, a->out_stride_h, a->out_stride_t}) {
    if (s < 0 || (s & 7) != 0) return S2_ERR_ALIGN;
    if (s > (int64_t)1 << 40) return S2_ERR_SHAPE;
  }
  if (rows > 0 && (bwd ? rows_overlap(a->head_dim, {{a->batch, a->in_stride_b}, {a->heads, a->in_stride_h}, {a->seqlen, a->in_stride_t}})
                       : rows_overlap(a->head_dim, {{a->batch, a->out_stride_b}, {a->heads, a->out_stride_h}, {a->seqlen, a->out_stride_t}})))
    return S2_ERR_SHAPE;
  const bool alike = (a->batch == 1 || a->in_stride_b == a->out_stride_b) && (a->heads == 1 || a->in_stride_h == a->out_stride_h) &&
                     (a->seqlen <= 1 || a->in_stride_t == a->out_stride_t);
  // (queries and keys go through at the same time)
  if (x[0] && x[1] && rows > 0) {
    if (out[0] == out[1] || (bwd && weight[0] && weight[1] && d_weight[0] == d_weight[1])) return S2_ERR_SHAPE;
    for (int i = 0; i < 2; ++i)
      if (out[i] == x[1 - i] || (bwd && out[i] == g[1 - i])) return S2_ERR_SHAPE;
  }
  for (int i = 0; i < 2; ++i) {
    if (!x[i]) continue;
    for (const void* y : {x[i], (const void*)out[i], bwd ? g[i] : nullptr, (const void*)weight[i]})
      if (!aligned16(y)) return S2_ERR_ALIGN;
    if (bwd && (reinterpret_cast<uintptr_t>(d_weight[i]) & 3u) != 0) return S2_ERR_ALIGN;
    // (in place a row goes where it came from)
    if (!alike && rows > 0 && out[i] == (bwd ? g[i] : x[i])) return S2_ERR_SHAPE;
    p.x[i] = static_cast<const uint16_t*>(x[i]);
    p.y[i] = static_cast<uint16_t*>(out[i]);
    p.g[i] = static_cast<const uint16_t*>(g[i]);
    p.weight[i] = weight[i];
    p.d_weight[i] = d_weight[i];
  }
  if ((reinterpret_cast<uintptr_t>(a->inv_freq) & 3u) != 0 || (reinterpret_cast<uintptr_t>(a->positions) & 3u) != 0) return S2_ERR_ALIGN;
  p.inv_freq = a->inv_freq;
  p.positions = a->positions;
  p.batch = a->batch;
  p.heads = a->heads;
  p.seqlen = a->seqlen;
  p.head_dim = a->head_dim;
  p.rotary_dim = a->rotary_dim;
  p.interleaved = a->interleaved;
  p.eps = a->eps;
  p.x_sb = a->in_stride_b;
  p.x_sh = a->in_stride_h;
  p.x_st = a->in_stride_t;
  p.y_sb = a->out_stride_b;
  p.y_sh = a->out_stride_h;
  p.y_st = a->out_stride_t;
  p.rows = (int)rows;
  return S2_OK;
}

}  // namespace

int s2_attn_chunk_paged(const s2_layout_params* lp, const s2_paged_cache* c, const s2_chunk_args* a, float scale, void* workspace,
                        size_t workspace_bytes, void* stream) {
  if (!lp || !c || !a) return S2_ERR_NULL;
  return chunk_cache(lp, nullptr, c, a, scale, workspace, workspace_bytes, stream);
}

int s2_attn_chunk_paged_layout(const s2_layout* layout, const s2_paged_cache* c, const s2_chunk_args* a, float scale, void* workspace,
                               size_t workspace_bytes, void* stream) {
  if (!layout || !c || !a) return S2_ERR_NULL;
  return chunk_cache(&layout->p, layout, c, a, scale, workspace, workspace_bytes, stream);
}

size_t s2_attn_chunk_workspace_bytes(int32_t nseq, int32_t heads, int32_t max_new, int32_t num_rows, int32_t head_dim, int32_t max_len, int32_t num_splits) {
  if (nseq < 1 || heads < 1 || max_new < 1 || num_rows < 1 || head_dim < 1) return 0;
  s2::CacheChunkParams p = chunk_sizes(nseq, heads, max_new, num_rows);
  if (num_splits <= 0) {
    s2::chunk_tiles(p);
    num_splits = most_chunk_splits(p, max_len);
  }
  if (num_splits == 1) return 0;
  const size_t items = (size_t)nseq * heads * p.max_new * num_splits;
  return ((items * (head_dim + 2) * sizeof(float) + 255) / 256) * 256;
}

int s2_kv_plan_paged(const s2_layout_params* lp, const s2_kv_plan_args* a, void* workspace, size_t workspace_bytes, void* stream) {
  if (!lp || !a) return S2_ERR_NULL;
  return kv_plan(lp, nullptr, a, workspace, workspace_bytes, stream);
}

int s2_kv_plan_paged_layout(const s2_layout* layout, const s2_kv_plan_args* a, void* workspace, size_t workspace_bytes, void* stream) {
  if (!layout || !a) return S2_ERR_NULL;
  return kv_plan(&layout->p, layout, a, workspace, workspace_bytes, stream);
}

size_t s2_kv_plan_workspace_bytes(int32_t nseq, int32_t heads) {
  if (nseq < 1 || heads < 1) return 0;
  s2::KvPlanParams p{};
  p.nseq = nseq;
  p.pairs = (int64_t)nseq * heads;
  s2::plan_groups(p);
  return plan_workspace(p).bytes;
}

int s2_qk_norm_rope_fwd(const s2_qk_norm_rope_args* a, void* stream) {
  if (!a) return S2_ERR_NULL;
  s2::QkRopeParams p{};
  const int st = qk_rope(a, false, p);
  if (st != S2_OK || p.rows == 0) return st;
  if (s2::qk_rope_groups(p) > s2::kMostGroups) return S2_ERR_SHAPE;
  return hip_ok(s2::launch_qk_rope(p, static_cast<hipStream_t>(stream))) ? S2_OK : S2_ERR_HIP;
}

int s2_qk_norm_rope_bwd(const s2_qk_norm_rope_args* a, void* workspace, size_t workspace_bytes, void* stream) {
  if (!a) return S2_ERR_NULL;
  s2::QkRopeParams p{};
  const int st = qk_rope(a, true, p);
  if (st != S2_OK) return st;
  if ((a->q && a->q_weight) || (a->k && a->k_weight)) {
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 ||
        workspace_bytes < s2_qk_norm_rope_bwd_workspace_bytes(a->batch, a->heads, a->seqlen, a->head_dim))
      return S2_ERR_WORKSPACE;
    p.part = static_cast<float*>(workspace);
  }
  if (p.rows == 0 && !p.part) return S2_OK;
  return hip_ok(s2::launch_qk_rope_bwd(p, static_cast<hipStream_t>(stream))) ? S2_OK : S2_ERR_HIP;
}

size_t s2_qk_norm_rope_bwd_workspace_bytes(int32_t batch, int32_t heads, int32_t seqlen, int32_t head_dim) {
  if (batch < 1 || heads < 1 || seqlen < 0 || (head_dim != 64 && head_dim != 128)) return 0;
  const int64_t rows = std::min<int64_t>((int64_t)batch * seqlen, s2::kMostGroups);
  return ((size_t)std::max(1, s2::qk_rope_parts((int)rows, heads, head_dim)) * 2 * head_dim * sizeof(float) + 255) / 256 * 256;
}

int s2_kv_append_paged(const s2_paged_cache* c, const s2_kv_append_args* a, void* stream) {
  if (!c || !a) return S2_ERR_NULL;
  s2::KvRowsParams p{};
  const int st = check_cache(c, p.c);
  if (st != S2_OK) return st;
  if ((reinterpret_cast<uintptr_t>(a->rows) & 3u) != 0 || (reinterpret_cast<uintptr_t>(a->skipped) & 3u) != 0) return S2_ERR_ALIGN;
  if (a->rows && a->num_items < 0) return S2_ERR_SHAPE;
  p.k = static_cast<const uint16_t*>(a->k);
  p.v = static_cast<const uint16_t*>(a->v);
  p.cu = a->cu_new;
  p.start = a->start;
  p.rows = a->rows;
  p.skipped = a->skipped;
  p.num_rows = a->num_rows;
  p.num_items = a->num_items;
  p.max_rows = a->max_new;
  p.stride_row = a->stride_row;
  p.stride_head = a->stride_head;
  return cache_rows(p, c, a->k, a->v, stream);
}

int s2_kv_read_paged(const s2_paged_cache* c, const s2_kv_read_args* a, void* stream) {
  if (!c || !a) return S2_ERR_NULL;
  s2::KvRowsParams p{};
  const int st = check_cache(c, p.c);
  if (st != S2_OK) return st;
  p.k_out = static_cast<uint16_t*>(a->k);
  p.v_out = static_cast<uint16_t*>(a->v);
  p.cu = a->cu_rows;
  p.start = a->start;
  p.num_rows = a->num_rows;
  p.max_rows = a->num_rows > 0 ? a->max_rows : std::min(a->max_rows, 0);  // (without rows there is no output to tell the two launches apart by)
  p.stride_row = a->stride_row;
  p.stride_head = a->stride_head;
  return cache_rows(p, c, a->k, a->v, stream);
}

int s2_attn_decode_paged_cache(const s2_layout_params* lp, const s2_paged_cache* c, const s2_cache_decode_args* a, float scale,
                               void* workspace, size_t workspace_bytes, void* stream) {
  if (!lp || !c || !a) return S2_ERR_NULL;
  return decode_cache(lp, nullptr, c, a, scale, workspace, workspace_bytes, stream);
}

int s2_attn_decode_paged_cache_layout(const s2_layout* layout, const s2_paged_cache* c, const s2_cache_decode_args* a, float scale,
                                      void* workspace, size_t workspace_bytes, void* stream) {
  if (!layout || !c || !a) return S2_ERR_NULL;
  return decode_cache(&layout->p, layout, c, a, scale, workspace, workspace_bytes, stream);
}

int s2_attn_tree_paged(const s2_layout_params* lp, const s2_paged_cache* c, const s2_tree_args* a, float scale, void* workspace,
                       size_t workspace_bytes, void* stream) {
  if (!lp || !c || !a) return S2_ERR_NULL;
  return tree_cache(lp, nullptr, c, a, scale, workspace, workspace_bytes, stream);
}

int s2_attn_tree_paged_layout(const s2_layout* layout, const s2_paged_cache* c, const s2_tree_args* a, float scale, void* workspace,
                              size_t workspace_bytes, void* stream) {
  if (!layout || !c || !a) return S2_ERR_NULL;
  return tree_cache(&layout->p, layout, c, a, scale, workspace, workspace_bytes, stream);
}

size_t s2_attn_tree_workspace_bytes(int32_t nseq, int32_t heads, int32_t nodes, int32_t head_dim, int32_t max_len, int32_t num_splits) {
  if (nseq < 1 || heads < 1 || nodes < 1 || head_dim < 1) return 0;
  if (num_splits <= 0) num_splits = most_cache_splits((int64_t)nseq * heads, max_len);
  const size_t items = (size_t)nseq * heads * nodes * num_splits;
  return ((items * (head_dim + 2) * sizeof(float) + 255) / 256) * 256;
}

int s2_attn_decode(const s2_layout_params* lp, const s2_decode_args* a, float scale, void* workspace,
                   size_t workspace_bytes, void* stream) {
  if (!lp || !a) return S2_ERR_NULL;
  return decode_contiguous(lp, nullptr, a, scale, workspace, workspace_bytes, stream);
}

int s2_attn_decode_static(const s2_layout_params* lp, const s2_decode_args* a, float scale, void* stream) {
  if (!lp || !a) return S2_ERR_NULL;
  // the size check comes first and needs no device: shapes whose partials do not fit are refused
  if (a->nseq < 1 || a->heads < 1 || a->max_len < 1) return S2_ERR_SHAPE;
  if (a->head_dim != 64 && a->head_dim != 128) return S2_ERR_SHAPE;
  if (a->num_splits < 0 || a->num_splits > 64) return S2_ERR_BAD_PARAM;
  // num_splits == 0: the call may pick fewer splits than this bound, never more
  const size_t need = s2_attn_decode_workspace_bytes(a->nseq, a->heads, a->head_dim, a->max_len, a->num_splits);
  if (need > kStaticScratchBytes) return S2_ERR_WORKSPACE;
  int ndev = 0;
  if (hipGetDeviceCount(&ndev) != hipSuccess || ndev < 1) {
    (void)hipGetLastError();
    return S2_ERR_NO_DEVICE;
  }
  void* ptr = scratch_on_current_device();
  if (!ptr) return S2_ERR_HIP;
  return decode_contiguous(lp, nullptr, a, scale, ptr, kStaticScratchBytes, stream);
}

int s2_attn_decode_paged(const s2_layout_params* lp, const s2_paged_decode_args* a, float scale,
                         void* workspace, size_t workspace_bytes, void* stream) {
  if (!lp || !a) return S2_ERR_NULL;
  return decode_paged(lp, nullptr, a, (int64_t)a->heads * a->head_dim, a->head_dim, scale, workspace, workspace_bytes, stream);
}

int s2_attn_decode_layout(const s2_layout* layout, const s2_decode_args* a, float scale, void* workspace,
                          size_t workspace_bytes, void* stream) {
  if (!layout || !a) return S2_ERR_NULL;
  return decode_contiguous(&layout->p, layout, a, scale, workspace, workspace_bytes, stream);
}

int s2_attn_decode_paged_layout(const s2_layout* layout, const s2_paged_decode_args* a, float scale,
                                void* workspace, size_t workspace_bytes, void* stream) {
  if (!layout || !a) return S2_ERR_NULL;
  return decode_paged(&layout->p, layout, a, (int64_t)a->heads * a->head_dim, a->head_dim, scale, workspace, workspace_bytes, stream);
}

int s2_layout_resident_blocks(const s2_layout* L, int32_t head, int32_t length, int32_t* blocks,
                              int32_t capacity, int32_t* count) {
  if (!L || !count) return S2_ERR_NULL;
  if (capacity < 0 || (capacity > 0 && !blocks)) return S2_ERR_NULL;
  const int B = L->p.num_blocks, S = L->p.block_size;
  if (head < 0 || head >= L->p.num_heads || length < 1 || (int64_t)length > (int64_t)B * S)
    return S2_ERR_BAD_PARAM;
  // A block among 0..i (i = row of the newest token) stays while row i or any later row keeps it:
  // walk each such column's list of attending rows (ascending) and look at its last entry.
  const int i = (length - 1) / S;
  int64_t n = 0;
  for (int j = 0; j <= i; ++j) {
    const int32_t lo = L->col_ptr[(size_t)head * B + j], hi = L->col_ptr[(size_t)head * B + j + 1];
    if (hi > lo && L->row_idx[hi - 1] >= i) {
      if (n < capacity) blocks[n] = j;
      ++n;
    }
  }
  *count = (int32_t)n;
  return n > capacity ? S2_ERR_OVERFLOW : S2_OK;
}

int s2_kv_resident_blocks(const s2_layout_params* lp, int32_t head, int32_t length, int32_t* blocks,
                          int32_t capacity, int32_t* count) {
  if (!lp || !count) return S2_ERR_NULL;
  if (capacity < 0 || (capacity > 0 && !blocks)) return S2_ERR_NULL;
  if (!good_block_size(lp->block_size)) return S2_ERR_BAD_PARAM;
  if (lp->dense != 0 && lp->dense != 1) return S2_ERR_BAD_PARAM;
  if (!lp->dense && (lp->local_blocks < 1 || lp->stride < 0 || lp->window_blocks < 0)) return S2_ERR_BAD_PARAM;
  if (lp->head_index_base < 0 || lp->num_heads < 1) return S2_ERR_BAD_PARAM;
  if (head < 0 || head >= lp->num_heads || length < 1) return S2_ERR_BAD_PARAM;
  // Every block a later row keeps among blocks 0..i is also kept by row i = (length-1) div S
  // (the mask only loses columns as the row index grows: a local block drops out of the window,
  // a stripe block stays until the optional window passes it), so the answer is row i itself.
  const int i = (length - 1) / lp->block_size;
  const int64_t n = s2::row_blocks(*lp, head, i, blocks, capacity);
  *count = (int32_t)n;
  return n > capacity ? S2_ERR_OVERFLOW : S2_OK;
}

const char* s2_status_string(int status) {
  switch (status) {
    case S2_OK: return "ok";
    case S2_ERR_NULL: return "a required pointer is NULL";
    case S2_ERR_BAD_PARAM: return "parameter out of range";
    case S2_ERR_SHAPE: return "tensor shape does not fit";
    case S2_ERR_ALIGN: return "pointer or stride not aligned";
    case S2_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
    case S2_ERR_HIP: return "HIP runtime error";
    case S2_ERR_NO_DEVICE: return "layout has no device copy";
    case S2_ERR_OVERFLOW: return "size overflow or out of memory";
    default: return "unknown status";
  }
}

int s2_last_hip_error(void) { return g_last_hip_error; }
int s2_version(void) { return 100; }

}  // extern "C"
