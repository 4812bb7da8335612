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

// Element i of an array that no workgroup of the same launch writes (the scalar cache, which earlier launches'
// writes do reach, would not see its); with UNIFORM (i the same in all lanes) by a scalar load, which does not
// wait for the vector loads in flight.
template <bool UNIFORM, class T>
__device__ __forceinline__ T paged_read(const T* p, int64_t i) {
  if constexpr (UNIFORM && !std::is_integral<T>::value) {
    typedef uint32_t words __attribute__((ext_vector_type(sizeof(T) / 4)));
    typedef const __attribute__((address_space(4))) words* scalar_ptr;
    return __builtin_bit_cast(T, *(scalar_ptr)(uintptr_t)(p + i));
  } else if constexpr (UNIFORM) {
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

// The sequence of token row t (cu[s] <= t < cu[s + 1]), or -1 behind the last one, for a row per lane (all
// lanes of the wave take part): the ends of 64 groups of sequences come from one load, a lane each, and
// the rest of the search, for more than 64 sequences, from memory.
__device__ __forceinline__ int paged_seq_of_lanes(const PagedGeo& g, int t) {
  const int lane = threadIdx.x & 63, stride = (g.n_seqs + 63) >> 6;
  const int end = g.cu[min((lane + 1) * stride, g.n_seqs)];  // end of the lane's group of sequences
  int c = 0;  // groups that end at or before row t
#pragma unroll
  for (int d = 32; d > 0; d >>= 1)
    if (__shfl(end, c + d - 1) <= t) c += d;
  if (__shfl(end, c) <= t) ++c;
  int lo = min(c * stride, g.n_seqs), hi = min(lo + stride, g.n_seqs);
  if (stride == 1) {
    hi = lo;
  } else {
    while (lo < hi) {
      const int m = (lo + hi) >> 1;
      if (g.cu[m + 1] > t) hi = m;
      else lo = m + 1;
    }
  }
  return lo < g.n_seqs && t >= g.cu[lo] ? lo : -1;
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

// What the query at cached index i sees (i < 0: a row before the cached tokens), not clamped to the
// cached tokens: keys below the end of the query's mask block and, with a window, at most that many below
// it. to_next: tokens to the next mask block.
__device__ __forceinline__ void paged_seen(const PagedGeo& g, const PagedSeq& q, int32_t i, int64_t& beg,
                                           int64_t& end, int64_t& to_next) {
  end = q.kv;
  to_next = kPagedFar;
  if (g.mask_block > 0) {
    const int64_t p = q.first + i;  // floor division: rows before position 0 count down
    int64_t blk = p / g.mask_block;
    if (p - blk * g.mask_block < 0) --blk;
    to_next = (blk + 1) * g.mask_block - p;
    end = i + to_next;
  }
  beg = g.window > 0 ? end - g.window : -kPagedFar;
}

// D(16x16) += A(16x32) B(32x16). Lane l holds A[l%16][8(l/16) .. +8], B[8(l/16) .. +8][l%16];
// accumulator element i of lane l is D[4(l/16) + i][l%16].
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// A constant of these bits, put into its register where it is used: out of the loops, where the compiler moves
// constants that no instruction can hold, it would keep a register that is not there.
template <uint32_t BITS>
__device__ __forceinline__ uint32_t bits_here() {
  uint32_t v;
  asm volatile("v_mov_b32 %0, %1" : "=v"(v) : "n"(BITS));
  return v;
}

// Direct global-to-LDS load of 16 B per lane (see lds_dma16) from a scalar base and a lane offset in bytes.
// The base has to be settled (no VALU instruction may write it in the five wait states before): callers
// compute it with scalar arithmetic.
__device__ __forceinline__ void lds_dma16_row(const void* base, uint32_t off, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(off), "s"(base), "s"(lds_base)
               : "memory", "m0");
}

// The running maximum starts at the lowest finite value, not at -inf: a row that has seen nothing yet
// (and one that never will) then keeps all its exponentials at exp2(-inf) = 0, with no inf - inf.
constexpr float kLowest = -3.402823466e38f;
constexpr float kMasked = -__builtin_huge_valf();
constexpr float kLazyMaxStep = 8.0f;  // the running max is raised when exceeded by more (log2 units)

// The second query term's part of a score, made finite: of an infinite key it is an infinity too, whose sign may
// be the opposite of the first term's, which alone is the score then.
__device__ __forceinline__ float second_part(float v, float most) { return __builtin_amdgcn_fmed3f(v, kLowest, most); }
__device__ __forceinline__ float most_here() { return __uint_as_float(bits_here<0x7f7fffffu>()); }

// Of 32 keys, those of the bit set `keys` in [b, e).
__device__ __forceinline__ uint32_t seen_keys(uint32_t keys, int b, int e) {
  const int lo = min(max(b, 0), 32), hi = min(max(e, 0), 32);
  return keys & (uint32_t)(((uint64_t)1 << hi) - ((uint64_t)1 << min(lo, hi)));
}

// The lane, computed where it is used: kept over the main loop it would cost a register that is not there.
__device__ __forceinline__ int lane_here() {
  uint32_t zero = 0;
  asm volatile("" : "+s"(zero));
  return (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, zero));
}

typedef __attribute__((address_space(3))) uint32_t lds_u32;

// bf16 values with infinities and NaN replaced by zero. In a tile that is masked for some row, a key's
// probability may be 0 while its latent is not finite, and 0 * NaN would reach the rows that do not see
// it. The rows that do see it get a NaN sum instead: 0 * inf or inf - inf, whatever the sign of the score.
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
// Whether some of them are (an exponent of all ones carries into the sign's place).
__device__ __forceinline__ bool not_finite(u32x4 u) {
  const uint32_t e = 0x7f807f80u, one = 0x00800080u;
  return (((u[0] & e) + one | (u[1] & e) + one | (u[2] & e) + one | (u[3] & e) + one) & 0x80008000u) != 0;
}
#define kNotANumber __uint_as_float(0xffffffffu)  // (an inline constant of the instructions, which 0x7fc00000 is not)

// Of a tile's 32 keys those whose latents are not all finite; chunk_at(key, c): where 8 of them are. For waves
// that clear the latents in registers, called where some score is minus infinity, as it is with such a latent
// if it is not NaN or plus infinity (which make the sum NaN by themselves). An infinite k^R makes such scores
// too, with finite latents: a key of no weight.
template <int CHUNKS, class At>
__device__ __forceinline__ uint32_t not_finite_keys(At chunk_at) {
  const int lane = lane_here();
  uint64_t bad = 0;
#pragma unroll 1
  for (int c = 0; c < CHUNKS; c += 2) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(chunk_at(lane & 31, c + (lane >> 5)));
    bad |= __builtin_amdgcn_ballot_w64(not_finite(v));
  }
  return (uint32_t)bad | (uint32_t)(bad >> 32);
}

// For workgroups that clear them in LDS: 8 values, a lane, made finite in place. The bits key() of those that
// were not are added to `word`.
template <class Key>
__device__ __forceinline__ void clear_not_finite(uint16_t* p, uint32_t* word, Key key) {
  u32x4* const at = reinterpret_cast<u32x4*>(p);
  const u32x4 v = *at;
  const bool bad = not_finite(v);
  if (__builtin_amdgcn_ballot_w64(bad) == 0) return;
  *at = as_u32x4(finite_or_zero(as_bf16x8(v)));
  // (of an atomic OR the compiler makes a loop over the lanes)
  asm volatile("ds_or_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : : "v"(lds_addr(word)), "v"(bad ? key() : 0u) : "memory");
}
// Behind it, by all waves: the cleared latents visible, and the keys. `word` was 0 and is left so; the callers
// have a barrier between two rounds.
__device__ __forceinline__ uint32_t cleared_keys(uint32_t* word) {
  __syncthreads();
  uint32_t at = lds_addr(word);
  asm volatile("" : "+v"(at));  // (see bits_here)
  volatile lds_u32* const here = (volatile lds_u32*)(at);
  const uint32_t keys = __builtin_amdgcn_readfirstlane(*here);
  if (keys != 0) {
    __syncthreads();  // every wave has read it
    if (threadIdx.x == 0) *here = 0;
  }
  return keys;
}

// The plan of one attention call, in the workspace: written beside the absorbed queries (paged_plan),
// read by the attention and the output kernels of the same call.
//   Row blocks: the (token, head) rows of a sequence in blocks of R, sequences in order. A block's keys
//   are the units of `unit` keys from `key0` that some of its rows see (a block that sees nothing keeps
//   one: it still writes its rows).
//   Work: every block counts as its units and `cost` more, which stand for what a workgroup spends on
//   entering and leaving a block. The blocks in order are split evenly over G workgroups by these counts:
//   workgroup w takes counts [w U / G, (w + 1) U / G), and of a block the units behind its first `cost`
//   counts. A block inside one workgroup is written as its latents; of a split one each workgroup leaves
//   a partial result, in slot 2 w + 1 for the block's first unit and 2 w for a later start (a workgroup
//   has at most one of each). A workgroup takes its blocks last to first: all ranges are about equally
//   long, the last block's part starts at its first key and the first block's ends at its last, so that
//   the workgroups walk the keys of a sequence at about the same place at the same time and find tiles
//   in their XCD's L2.
struct PagedBlock {
  int32_t seq, row0, key0, n_units;  // sequence, first row in it, first key (a multiple of 32), units
  int32_t lo, n_rows, kv;            // the sequence's first token row, its rows, its cached tokens
  int32_t head0;                     // head of the first row
  int32_t all_b, all_e;              // the keys [all_b, all_e) that all rows of the block see
  int32_t to_next;                   // tokens from the first row's to the next mask block (saturated)
  int32_t pad;
  int64_t beg0, end0;                // the first row's keys, not clamped to the cached tokens
};
static_assert(sizeof(PagedBlock) == 64, "one scalar load");

// The keys [b, e) that row r of the block (counted from its first row) sees. A block's rows are at most
// 256 tokens, so that only mask blocks below that length are crossed more than once. Without a branch that
// lanes take differently: where such a branch rejoined in a kernel that fills the register file, the
// compiler moved another value for the lanes in it only.
__device__ __forceinline__ void paged_row_sees(const PagedGeo& g, const PagedBlock& p, int H, int r,
                                               int32_t& b, int32_t& e) {
  const int d = (p.head0 + r) / H - p.to_next;  // tokens past the first boundary
  const int more = g.mask_block <= 256 ? max(d, 0) / max((int)g.mask_block, 1) : 0;
  const int64_t off = (d >= 0 ? 1 + more : 0) * g.mask_block;
  const int64_t end = p.end0 + off, beg = p.beg0 + off;
  e = (int32_t)(end < 0 ? 0 : end > p.kv ? p.kv : end);
  b = (int32_t)(beg < 0 ? 0 : beg > e ? e : beg);
}

struct PagedWork {
  int32_t block, end, n, last_ns;  // last row block, the end in its counts, counts of the workgroup; the
                                   // workgroups that share the last block
};
// Where a row's latents are, written by the workgroup that has its block's first unit (the absorb kernel
// clears it): ns workgroups share its block, w0 the first of them, row its place in the block; ns 1: its
// row of o_lat; ns 0: the row belongs to no sequence.
struct alignas(8) PagedRow {  // (one store: rows that bad offsets give to two blocks have either's record)
  int32_t w0;
  uint16_t ns, row;
};

struct PagedPlan {
  int64_t* first;         // [max_blocks] first count of each block
  PagedBlock* block;      // [max_blocks]
  PagedWork* work;        // [n_wg]
  PagedBlock* work_block; // [n_wg] the record of work[].block
  PagedRow* row;          // [n_tokens * H]
};

struct PagedWriteArgs : WriteArgs {
  PagedGeo pg;
};

struct PagedAttendArgs : AttendArgs {
  PagedGeo pg;
  PagedPlan plan;
  uint16_t* q_lo;      // workspace: q_cat's second bf16 term, q_cat - bf16(q_cat), for the few-row kernel, or nullptr
  uint8_t* q_low;      // workspace: the same in 8 bits (low_bits_of), for the kernels of many rows, or nullptr
  float* o_lat;        // workspace: [n_tokens * H][d_c] fp32, rows of unsplit blocks
  int32_t max_blocks;  // row blocks the plan holds
  int32_t rows, unit;  // rows per block, keys per unit
  int32_t cost;        // counts of a block beyond its units
};

// The kernels of many rows multiply the second term of q_cat where one alone would be off by more than about the
// output's own rounding: where a block has a row longer than kOneTerm (against keys of unit RMS: the standard
// deviation of its scores, in exponents of 2) and, of whatever scale queries and keys are, where the scores of some
// row are further apart than kSpread in the first tile of a workgroup's part of a block, or in a later one that
// raises a running maximum, as those of larger keys do: then it takes its part again from the start. Of 256 rows
// one is found in the first tile if their deviation is 3 or more; at 1.4, of a plain softmax over unit vectors,
// none in 10^6 tiles is.
constexpr float kOneTerm = 2.3f, kSpread = 10.f;

// sum + the squares of 8 values.
__device__ __forceinline__ float add_squares(bf16x8 v, float sum) {
  const u32x4 u = as_u32x4(v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = u[i];
    const bf16x2 h = __builtin_bit_cast(bf16x2, w);
    sum = __builtin_amdgcn_fdot2_f32_bf16(h, h, sum, false);
  }
  return sum;
}

// The second bf16 term of four values of q_cat (their first has been, or is, rounded from them). The few-row
// kernel reads it as it is. For the kernels of many rows, which seldom do, the absorption writes half the bytes: the
// 8 bits of the value that follow its first term's, as the signed distance from it in steps of the float's bit
// pattern (of 2^-8 of the first term's last place).
__device__ __forceinline__ bf16x4 second_term_of(f32x4 v) {
  return to_bf16x4(v - __builtin_convertvector(to_bf16x4(v), f32x4));
}
__device__ __forceinline__ uint32_t low_bits(float v, uint32_t first) {  // in bits 8 .. 15
  return (uint32_t)min((int)(__float_as_uint(v) - (first << 16)), 0x7fff);
}
__device__ __forceinline__ uint32_t low_bits_of(f32x4 v) {
  const u32x2 h = __builtin_bit_cast(u32x2, to_bf16x4(v));
  const uint32_t l01 = __builtin_amdgcn_perm(low_bits(v[1], h[0] >> 16), low_bits(v[0], h[0] & 0xffffu), 0x0c0c0501u);
  const uint32_t l23 = __builtin_amdgcn_perm(low_bits(v[3], h[1] >> 16), low_bits(v[2], h[1] & 0xffffu), 0x0c0c0501u);
  return l01 | l23 << 16;
}
// The second term from the first and those bits (exact: it has at most 8).
__device__ __forceinline__ bf16x8 second_term(bf16x8 first, u32x2 low) {
  const u32x4 h = as_u32x4(first);
  f32x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t hi = i & 1 ? h[i >> 1] & 0xffff0000u : h[i >> 1] << 16;
    const int32_t lo = (int32_t)(low[i >> 2] << (24 - 8 * (i & 3))) >> 24;
    v[i] = __uint_as_float(hi + ((uint32_t)lo << 8)) - __uint_as_float(hi);
  }
  return to_bf16x8(v);
}
__device__ __forceinline__ void paged_q_lo(const PagedAttendArgs& a, int64_t at, f32x4 v) {
  if (a.q_lo) *reinterpret_cast<bf16x4*>(a.q_lo + at) = second_term_of(v);
  if (a.q_low) *reinterpret_cast<uint32_t*>(a.q_low + at) = low_bits_of(v);
}
// Both terms of a pair.
__device__ __forceinline__ void paged_q_pair(const PagedAttendArgs& a, int64_t at, float u, float v) {
  const uint16_t hu = to_bf16_bits(u), hv = to_bf16_bits(v);
  *reinterpret_cast<uint32_t*>(a.qcat + at) = (uint32_t)hu | (uint32_t)hv << 16;
  if (a.q_lo)
    *reinterpret_cast<uint32_t*>(a.q_lo + at) = (uint32_t)to_bf16_bits(u - bf16_bits_to_f32(hu)) |
                                                (uint32_t)to_bf16_bits(v - bf16_bits_to_f32(hv)) << 16;
  if (a.q_low)
    *reinterpret_cast<uint16_t*>(a.q_low + at) =
        (uint16_t)__builtin_amdgcn_perm(low_bits(v, hv), low_bits(u, hu), 0x0c0c0501u);
}

constexpr int kPagedMaxSeqs = 4096;

hipError_t launch_paged_cache_write(const PagedWriteArgs& a, hipStream_t s);
hipError_t launch_paged_absorb(const PagedAttendArgs& a, hipStream_t s);
hipError_t launch_paged_absorb_tiles(const PagedAttendArgs& a, hipStream_t s);  // (k_attend.hip)
hipError_t launch_paged_attend(const PagedAttendArgs& a, hipStream_t s);
hipError_t launch_paged_out(const PagedAttendArgs& a, hipStream_t s);

// Rows per block and keys per unit of the attention kernel for sequences of at most max_rows rows.
void paged_attend_shape(int d_c, int d_rope, int64_t max_rows, int32_t* rows, int32_t* unit, int32_t* cost);
// The kernels of many rows per block (k_paged_wide.hip, for d_c = 512 k_paged_wide512.hip): rows, and launch.
int paged_wide_rows(int d_c, int d_rope);
hipError_t launch_paged_attend_wide(const PagedAttendArgs& a, hipStream_t s);
hipError_t launch_paged_attend_wide512(const PagedAttendArgs& a, hipStream_t s);

constexpr int kCopyPairs = 440;  // page pairs per launch: they travel in the kernel's arguments
struct PagesCopyArgs {
  uint16_t* pool[2];        // c_kv, k_r: [n_layers][n_pages][page bytes]
  int64_t layer_bytes[2], page_bytes[2];
  int32_t n_layers, n_pairs;
  int32_t src[kCopyPairs], dst[kCopyPairs];
};
hipError_t launch_pages_copy(const PagesCopyArgs& a, hipStream_t s);

}  // namespace vmla
