// Paged latent cache: launch arguments, the plan that the attention kernels work by, and the device
// code that finds a token's sequence, position and pool row.
//
// The lengths and block table are in device memory, so that a captured graph serves batches of
// changing lengths; the host knows the tensors' sizes only. Whatever those arrays hold, no access
// leaves the tensors: offsets are clamped to the call's token rows, lengths to the table's width, and
// a table entry outside the pool is a hole.
#pragma once
#include "vmla_device.h"

namespace vmla {

// Positions, mask blocks and windows are clamped to this, so that their sums stay within 64 bits.
constexpr int64_t kPagedFar = int64_t(1) << 60;

struct PagedGeo {
  const int32_t* cu;         // [n_seqs + 1] first token row of each sequence
  const int32_t* kv_len;     // [n_seqs] cached tokens, the new ones (the last of them) included
  const int64_t* first_pos;  // [n_seqs] absolute position of cached token 0, or nullptr (all 0)
  const int32_t* table;      // [n_seqs][max_pages] page ids
  int32_t n_seqs, n_tokens, page_tokens, max_pages, n_pages;
  int32_t max_kv;            // max_pages * page_tokens (< 2^31, validated on the host)
  uint32_t page_mul;         // j / page_tokens = (j * page_mul) >> (31 + page_shift) for j < 2^31
  int32_t page_shift;
  int64_t mask_block;        // block-causal mask: tokens per block, 0 = none
  int64_t window;            // sliding window in tokens, 0 = all
  int32_t grid_h, grid_w;
};

// The division's factor: with s = ceil(log2 d) and m = ceil(2^(31+s) / d), m d exceeds 2^(31+s) by
// less than d <= 2^s, so j m / 2^(31+s) exceeds j / d by less than j / (2^31 d) < 1 / d.
__host__ inline void set_page_division(PagedGeo& g) {
  int s = 0;
  while ((int64_t(1) << s) < g.page_tokens) ++s;
  g.page_shift = s;
  g.page_mul = (uint32_t)(((uint64_t(1) << (31 + s)) + g.page_tokens - 1) / g.page_tokens);
}

__host__ __device__ inline int32_t page_of(const PagedGeo& g, int32_t j) {
  return (int32_t)(((uint64_t)(uint32_t)j * g.page_mul) >> (31 + g.page_shift));
}

// Sequence s: its token rows [lo, hi) of the call and its cached tokens.
struct PagedSeq {
  int32_t lo, hi, kv;
  int64_t first;
};

// Element i of an array that no kernel of the call writes; with UNIFORM (i the same in all lanes) by a
// scalar load, which does not wait for the vector loads in flight.
template <bool UNIFORM, class T>
__device__ __forceinline__ T paged_read(const T* p, int64_t i) {
  if constexpr (UNIFORM) {
    typedef const __attribute__((address_space(4))) T* scalar_ptr;
    return *(scalar_ptr)(uintptr_t)(p + i);
  } else {
    return p[i];
  }
}

template <bool UNIFORM = false>
__device__ __forceinline__ PagedSeq paged_seq(const PagedGeo& g, int s) {
  PagedSeq q;
  q.lo = min(max(paged_read<UNIFORM>(g.cu, s), 0), g.n_tokens);
  q.hi = min(max(paged_read<UNIFORM>(g.cu, s + 1), q.lo), g.n_tokens);
  q.kv = min(max(paged_read<UNIFORM>(g.kv_len, s), 0), g.max_kv);
  const int64_t f = g.first_pos ? paged_read<UNIFORM>(g.first_pos, s) : 0;
  q.first = f < 0 ? 0 : f < kPagedFar ? f : kPagedFar;
  return q;
}

// The sequence of token row t (cu[s] <= t < cu[s + 1]), or -1 behind the last one.
__device__ __forceinline__ int paged_seq_of(const PagedGeo& g, int t) {
  int lo = 0, hi = g.n_seqs;  // the first s with cu[s + 1] > t
  while (lo < hi) {
    const int m = (lo + hi) >> 1;
    if (g.cu[m + 1] > t) hi = m;
    else lo = m + 1;
  }
  return lo < g.n_seqs && t >= g.cu[lo] ? lo : -1;
}

// The pool row of cached token j, -1 for a hole (j outside the sequence, or its page outside the pool).
__device__ __forceinline__ int32_t paged_row(const PagedGeo& g, int s, int32_t kv, int32_t j) {
  if (j < 0 || j >= kv) return -1;
  const int32_t p = page_of(g, j);
  const int32_t page = g.table[(int64_t)s * g.max_pages + p];
  return page < 0 || page >= g.n_pages ? -1 : page * g.page_tokens + (j - p * g.page_tokens);
}

// (f, y, x) of an absolute position.
__device__ __forceinline__ void paged_pos(const PagedGeo& g, int64_t pos, int64_t& f, int& y, int& x) {
  const int64_t p = pos < 0 ? 0 : pos;
  const int64_t hw = (int64_t)g.grid_h * g.grid_w;
  f = floor_div(p, hw);
  const int r = (int)(p - f * hw);
  y = r / g.grid_w;
  x = r - y * g.grid_w;
}

// The cached tokens [b, e) that the query at cached index i sees (i < 0: a row before the cached
// tokens): keys below the end of the query's mask block and, with a window, at most that many below it.
__device__ __forceinline__ void paged_seen(const PagedGeo& g, const PagedSeq& q, int32_t i, int32_t& b,
                                           int32_t& e) {
  int64_t end = q.kv;
  if (g.mask_block > 0) {
    const int64_t p = q.first + i;  // floor division: rows before position 0 count down
    int64_t blk = p / g.mask_block;
    if (p - blk * g.mask_block < 0) --blk;
    end = (blk + 1) * g.mask_block - q.first;
  }
  const int64_t beg = g.window > 0 ? end - g.window : 0;
  e = (int32_t)(end < 0 ? 0 : end > q.kv ? q.kv : end);
  b = (int32_t)(beg < 0 ? 0 : beg > e ? e : beg);
}

// The running maximum starts at the lowest finite value, not at -inf: a row that has seen nothing yet
// (and one that never will) then keeps all its exponentials at exp2(-inf) = 0, with no inf - inf.
constexpr float kLowest = -3.402823466e38f;
constexpr float kMasked = -__builtin_huge_valf();
constexpr float kLazyMaxStep = 8.0f;  // the running max is raised when exceeded by more (log2 units)

// bf16 values with infinities and NaN replaced by zero. In a tile that is masked for some row, a key's
// probability may be 0 while its latent is not finite, and 0 * NaN would reach the rows that do not see
// it; a row that does see it has a NaN score, since the latent is part of the key.
__device__ __forceinline__ bf16x8 finite_or_zero(bf16x8 v) {
  u32x4 u = as_u32x4(v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = (u[i] & 0x7f80u) == 0x7f80u ? 0u : u[i] & 0xffffu;
    const uint32_t hi = (u[i] & 0x7f800000u) == 0x7f800000u ? 0u : u[i] & 0xffff0000u;
    u[i] = lo | hi;
  }
  return as_bf16x8(u);
}

// The plan of one attention call, in the workspace: written by paged_plan_kernel, read by the
// attention and the output kernels of the same call.
//   Row blocks: the (token, head) rows of a sequence in blocks of R, sequences in order. A block's keys
//   are the tiles that some of its rows see: `n_units` units of `unit` keys from `key0` (a block that
//   sees nothing keeps one unit: it still writes its rows).
//   Work: the units of all blocks in order, split evenly over G workgroups; workgroup w takes
//   [w U / G, (w + 1) U / G). Consecutive units of one block are a segment. A block inside one workgroup
//   is written as its latents; of a split one each workgroup leaves a partial result, in slot 2 w + 1
//   for the block's first segment and 2 w for a later one (a workgroup has at most one of each). A
//   workgroup takes its segments last to first: all ranges are equally long, the last segment starts at
//   a block's first key and the first ends at a block's last, so that the workgroups walk the keys of a
//   sequence at about the same place at the same time and find tiles in their XCD's L2.
struct PagedBlock {
  int32_t seq, row0, key0, n_units;
};
struct PagedWork {
  int32_t block, end, n_units, pad;  // last row block, the end in its units, units of the workgroup
};
struct PagedPlan {
  int64_t* head;        // [2]: units U, workgroups G in use
  int32_t* seq_block;   // [n_seqs + 1] first row block of each sequence
  PagedBlock* block;    // [max_blocks]
  int64_t* first_unit;  // [max_blocks + 1]
  PagedWork* work;      // [n_wg]
};

struct PagedWriteArgs : WriteArgs {
  PagedGeo pg;
};

struct PagedAttendArgs : AttendArgs {
  PagedGeo pg;
  PagedPlan plan;
  float* o_lat;        // workspace: [n_tokens * H][d_c] fp32, rows of unsplit blocks
  uint16_t* zero_row;  // workspace: a row of zeros, staged in a hole's place
  int32_t max_blocks;  // row blocks the plan holds
  int32_t rows, unit;  // rows per block, keys per unit
};

constexpr int kPagedMaxSeqs = 4096;

hipError_t launch_paged_cache_write(const PagedWriteArgs& a, hipStream_t s);
hipError_t launch_paged_absorb(const PagedAttendArgs& a, hipStream_t s);
hipError_t launch_paged_plan(const PagedAttendArgs& a, hipStream_t s);
hipError_t launch_paged_attend(const PagedAttendArgs& a, hipStream_t s);
hipError_t launch_paged_out(const PagedAttendArgs& a, hipStream_t s);

// Rows per block and keys per unit of the attention kernel for sequences of at most max_rows rows.
void paged_attend_shape(int d_c, int d_rope, int64_t max_rows, int32_t* rows, int32_t* unit);
// The kernel of many rows per block (k_paged_wide.hip): its block, 0 where it is not built, and launch.
int paged_wide_rows(int d_c, int d_rope);
hipError_t launch_paged_attend_wide(const PagedAttendArgs& a, hipStream_t s);

constexpr int kCopyPairs = 440;  // page pairs per launch: they travel in the kernel's arguments
struct PagesCopyArgs {
  uint16_t* pool[2];        // c_kv, k_r: [n_layers][n_pages][page bytes]
  int64_t layer_bytes[2], page_bytes[2];
  int32_t n_layers, n_pairs;
  int32_t src[kCopyPairs], dst[kCopyPairs];
};
hipError_t launch_pages_copy(const PagesCopyArgs& a, hipStream_t s);

}  // namespace vmla
