// Latent attention of new tokens over a paged cache (Section "Inference-Time Reparameterization", with
// a sequence's cached tokens in pages instead of a ring).
//
//   paged_plan     row blocks, their key ranges and the even split of the work (vmla_paged.h)
//   q_absorb       as for the ring (k_attend.hip), each token at its sequence's position
//   paged_attend   S^T = [c_kv | k_r] q_cat^T, masked, online softmax in base 2, O_lat^T += c_kv^T P^T
//   paged_out      merges the partial results of split row blocks, divides by the sum, applies W_UV_h
//
// Rows are (token, head) pairs, head-minor: every head of a token reads the same latents, so a block of
// rows shares each staged tile.
#include <type_traits>

#include "vmla_device.h"
#include "vmla_paged.h"

namespace vmla {
namespace {

// D(16x16) += A(16x32) B(32x16). Lane l holds A[l%16][8(l/16) .. +8], B[8(l/16) .. +8][l%16];
// accumulator element i of lane l is D[4(l/16) + i][l%16].
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Direct global-to-LDS load of 4 B per lane: lane l's word lands at lds_base + 4 l (see lds_dma16).
__device__ __forceinline__ void lds_dma4(const int32_t* gptr, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off"
               :
               : "v"(gptr), "s"(lds_base)
               : "memory", "m0");
}

// ---- plan -----------------------------------------------------------------------------------
// One workgroup. Sequences, then row blocks, are scanned 1,024 at a time.
constexpr int kPlanThreads = 1024;

// Exclusive prefix sums of v over the workgroup's threads; total: the sum.
__device__ __forceinline__ int64_t plan_scan(int64_t v, int64_t& total) {
  __shared__ int64_t wave_sum[kPlanThreads / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t x = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();  // the previous scan's sums are read
  if (lane == 63) wave_sum[wave] = x;
  __syncthreads();
  int64_t base = 0;
  total = 0;
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) base += wave_sum[w];
    total += wave_sum[w];
  }
  return base + x - v;
}

__global__ __launch_bounds__(kPlanThreads) void paged_plan_kernel(const PagedAttendArgs a) {
  __shared__ int32_t first_block[kPagedMaxSeqs + 1];
  const PagedGeo& g = a.pg;
  const int tid = threadIdx.x, H = a.n_heads, R = a.rows;
  int64_t blocks = 0;
  for (int s0 = 0; s0 < g.n_seqs; s0 += kPlanThreads) {
    const int s = s0 + tid;
    int64_t n = 0, total;
    if (s < g.n_seqs) {
      const PagedSeq q = paged_seq(g, s);
      n = ((int64_t)(q.hi - q.lo) * H + R - 1) / R;
    }
    const int64_t at = blocks + plan_scan(n, total);
    // offsets that go down could ask for more blocks than the call's rows make: those are left out
    if (s < g.n_seqs) first_block[s] = (int32_t)min(at, (int64_t)a.max_blocks);
    blocks += total;
  }
  blocks = min(blocks, (int64_t)a.max_blocks);
  if (tid == 0) first_block[g.n_seqs] = (int32_t)blocks;
  __syncthreads();
  for (int s = tid; s <= g.n_seqs; s += kPlanThreads) a.plan.seq_block[s] = first_block[s];
  int64_t units = 0;
  for (int r0 = 0; r0 < blocks; r0 += kPlanThreads) {
    const int r = r0 + tid;
    int64_t n = 0, total;
    if (r < blocks) {
      int lo = 0, hi = g.n_seqs - 1;  // the last s with first_block[s] <= r
      while (lo < hi) {
        const int m = (lo + hi + 1) >> 1;
        if (first_block[m] <= r) lo = m;
        else hi = m - 1;
      }
      const PagedSeq q = paged_seq(g, lo);
      const int row0 = (r - first_block[lo]) * R, n_rows = (q.hi - q.lo) * H;
      const int base = q.kv - (q.hi - q.lo);  // cached index of the sequence's first new token
      int32_t b, e, b1, e1;
      paged_seen(g, q, base + row0 / H, b, e);
      paged_seen(g, q, base + (min(row0 + R, n_rows) - 1) / H, b1, e1);
      PagedBlock p;
      p.seq = lo;
      p.row0 = row0;
      p.key0 = b & ~31;
      p.n_units = max(1, (int)(((int64_t)e1 - p.key0 + a.unit - 1) / a.unit));
      a.plan.block[r] = p;
      n = p.n_units;
    }
    const int64_t at = units + plan_scan(n, total);
    if (r < blocks) a.plan.first_unit[r] = at;
    units += total;
  }
  if (tid == 0) {
    a.plan.first_unit[blocks] = units;
    a.plan.head[0] = units;
    a.plan.head[1] = min(units, (int64_t)a.n_wg);
  }
  __syncthreads();
  const int64_t G = min(units, (int64_t)a.n_wg);
  for (int w = tid; w < a.n_wg; w += kPlanThreads) {
    PagedWork k{};
    if (w < G) {
      const int64_t u = floor_div((int64_t)w * units, G), u1 = floor_div((int64_t)(w + 1) * units, G);
      int lo = 0, hi = (int)blocks - 1;  // the last block with first_unit < u1
      while (lo < hi) {
        const int m = (lo + hi + 1) >> 1;
        if (a.plan.first_unit[m] < u1) lo = m;
        else hi = m - 1;
      }
      k.block = lo;
      k.end = (int32_t)(u1 - a.plan.first_unit[lo]);
      k.n_units = (int32_t)(u1 - u);
    }
    a.plan.work[w] = k;
  }
  // the row that is staged in place of a hole
  for (int i = tid; i < a.dqk_pad; i += kPlanThreads) a.zero_row[i] = 0;
}

// ---- attention of few rows -------------------------------------------------------------------
// A workgroup's units are NW tiles of 32 keys, one per wave: each wave streams its own tiles through
// two LDS buffers with direct global-to-LDS loads, tile t + 1 in flight while tile t is used, and keeps
// its own running maximum, sum and latents of all rows; the waves never wait for each other until the
// segment's end, where their results are merged through LDS.
constexpr int few_waves(int dc) { return dc <= 256 ? 4 : 2; }

template <int DC, int DR, int QB>
struct FewCfg {
  static constexpr int DQKP = (DC + DR + 31) / 32 * 32;  // [c_kv | k_r | pad], whole 32-wide k-steps
  static constexpr int KS = DQKP / 32;
  static constexpr int DV = DC / 16;                     // 16-column blocks of the latent
  static constexpr int CPR = DQKP / 8;                   // 16-byte chunks per tile row
  static constexpr int TILE = 32 * DQKP;                 // elements
  static constexpr int NDMA = 32 * CPR / 64;             // 1 KB loads per tile
  static constexpr int NW = few_waves(DC);
  static constexpr int ROWS = 16 * QB;
  static constexpr int UNIT = 32 * NW;
  static constexpr int RS = DC + 4;                      // row stride of the merged latents (floats)
  // Chunk position of logical chunk c in row r. CPR is 4 or 12 mod 16, so the rows r .. r + 3 of one
  // chunk fall on different groups of four 4-bank groups; the XOR separates the rows 4 apart, by bit 1
  // first, since the transpose reads take two adjacent chunks of rows 4 j .. 4 j + 3 and the next four.
  __device__ static constexpr int swz(int r) {
    const int q = (r >> 2) & 3;
    return ((q & 1) << 1) | (q >> 1);
  }
  static_assert(CPR % 16 == 4 || CPR % 16 == 12, "bank spread of the tile rows");
  static_assert(DC % 16 == 0 && 16 * CPR % 64 == 0 && NDMA + 1 < 64, "tile shape");
  static_assert(ROWS * RS * 4 <= 2 * TILE * 2, "a wave's results fit its tile buffers");
};

template <int DC, int DR, int QB>
__global__ __launch_bounds__(64 * few_waves(DC)) void paged_attend_few_kernel(const PagedAttendArgs a) {
  using C = FewCfg<DC, DR, QB>;
  constexpr int NW = C::NW;
  __shared__ __attribute__((aligned(16))) uint16_t tiles[NW][2][C::TILE];
  __shared__ int32_t ids[NW][2][64];
  __shared__ float red_m[NW][C::ROWS], red_l[NW][C::ROWS];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int gq = lane >> 4, l16 = lane & 15;
  const PagedGeo& g = a.pg;
  const int H = a.n_heads;
  const PagedWork wk = a.plan.work[blockIdx.x];
  int left = __builtin_amdgcn_readfirstlane(wk.n_units);
  int blk = __builtin_amdgcn_readfirstlane(wk.block), end = __builtin_amdgcn_readfirstlane(wk.end);

  // Load j of a tile fills the chunk slots 64 j .. 64 j + 63: of this lane's chunk, in bits 0..15 the
  // offset in its row's c_kv, or (bit 31) k_r (the pad reads k_r again, against zeros in q_cat), in bits
  // 16..19 the row modulo 16. Half a tile is a whole number of loads, and the other half repeats it.
  uint32_t d_at[C::NDMA / 2];
#pragma unroll
  for (int j = 0; j < C::NDMA / 2; ++j) {
    const int slot = j * 64 + lane, r = slot / C::CPR, c = (slot % C::CPR) ^ C::swz(r);
    d_at[j] = (uint32_t)r << 16 | (c < DC / 8 ? c * 8 : 0x80000000u | (c < (DC + DR) / 8 ? c * 8 - DC : 0));
  }

  while (left > 0) {
    const PagedBlock pb = a.plan.block[blk];
    const int seq = __builtin_amdgcn_readfirstlane(pb.seq), row0 = __builtin_amdgcn_readfirstlane(pb.row0);
    const int n_units = __builtin_amdgcn_readfirstlane(pb.n_units);
    if (end == 0) end = n_units;  // a segment before the workgroup's last ends with its block
    const int take = min(left, end), u0 = end - take;
    const int key0 = __builtin_amdgcn_readfirstlane(pb.key0) + u0 * C::UNIT + wave * 32;  // this wave's first
    const PagedSeq q = paged_seq<true>(g, seq);
    const int n_rows = (q.hi - q.lo) * H, base = q.kv - (q.hi - q.lo);
    const int32_t* table = g.table + (int64_t)seq * g.max_pages;

    // this lane's rows and what they see
    bf16x8 qv[QB][C::KS];
    int see_b[QB], see_e[QB];
    int b_max = 0, e_min = 0x7fffffff;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const int r = row0 + 16 * qb + l16;
      see_b[qb] = 0;
      see_e[qb] = 0x7fffffff;
      if (r < n_rows) {
        paged_seen(g, q, base + r / H, see_b[qb], see_e[qb]);
        b_max = max(b_max, see_b[qb]);
        e_min = min(e_min, see_e[qb]);
      }
      const uint16_t* src = a.qcat + ((int64_t)q.lo * H + (r < n_rows ? r : row0)) * a.dqk_pad;
#pragma unroll
      for (int ks = 0; ks < C::KS; ++ks) {
        const int c = ks * 32 + 8 * gq;
        u32x4 v = {0, 0, 0, 0};
        if (r < n_rows && c < a.dqk_pad) v = ldg16(src + c);
        qv[qb][ks] = as_bf16x8(v);
      }
    }
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) {
      b_max = max(b_max, __shfl_xor(b_max, d));
      e_min = min(e_min, __shfl_xor(e_min, d));
    }
    b_max = __builtin_amdgcn_readfirstlane(b_max);
    e_min = __builtin_amdgcn_readfirstlane(e_min);

    f32x4 o[QB][C::DV];
    float m_run[QB], l_run[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      m_run[qb] = kLowest;
      l_run[qb] = 0.f;
#pragma unroll
      for (int d = 0; d < C::DV; ++d) o[qb][d] = f32x4{};
    }

    // page ids of tile t's keys, one per lane, into slot t & 1 (a key outside the sequence reads the
    // nearest entry of the table, and is no row below)
    auto load_ids = [&](int t) {
      const int key = min(max(key0 + t * C::UNIT + (lane & 31), 0), g.max_kv - 1);
      lds_dma4(table + page_of(g, key), __builtin_amdgcn_readfirstlane(lds_addr(&ids[wave][t & 1][0])));
    };
    auto row_of = [&](int t) {  // this lane's key's pool row, -1: none
      const int key = key0 + t * C::UNIT + (lane & 31);
      const int32_t page = *(volatile int32_t*)&ids[wave][t & 1][lane];
      if (key >= q.kv || page < 0 || page >= g.n_pages) return -1;
      return page * g.page_tokens + key - page_of(g, key) * g.page_tokens;
    };
    auto load_tile = [&](int t, int row) {
      const uint32_t lds = lds_addr(&tiles[wave][t & 1][0]);
#pragma unroll
      for (int j = 0; j < C::NDMA; ++j) {
        const uint32_t at = d_at[j % (C::NDMA / 2)];
        const int32_t r = __shfl(row, (int)(at >> 16 & 15) + (j < C::NDMA / 2 ? 0 : 16));
        const bool kr = (int32_t)at < 0;
        const uint16_t* p = kr ? a.k_r : a.c_kv;
        p += (int64_t)r * (kr ? DR : DC) + (at & 0xffffu);
        lds_dma16(r < 0 ? a.zero_row : p, __builtin_amdgcn_readfirstlane(lds + 1024u * j));
      }
    };

    // the tile rows' K operand of step ks (lane: row l16 + 16 kb, chunk 4 ks + gq) and the transpose
    // reads' rows 4 gq + .. (lane: row 4 gq + l16 / 4 (+ 16), columns 4 (l16 % 4) + 16 d)
    const int k_sw = C::swz(l16), v_sw = C::swz(4 * gq);
    const int v_row = 4 * gq + (l16 >> 2), v_col = l16 & 3;

    load_ids(0);
    wait_vmcnt<0>();
    int row = row_of(0);
    load_ids(1);
    load_tile(0, row);
    for (int t = 0; t < take; ++t) {
      const uint32_t there = (uint32_t)__builtin_amdgcn_ballot_w64(row >= 0);  // keys of tile t that exist
      if (t + 1 < take) {
        wait_vmcnt<C::NDMA>();  // the ids of tile t + 1
        row = row_of(t + 1);
        load_ids(t + 2);
        load_tile(t + 1, row);
        wait_vmcnt<C::NDMA + 1>();  // tile t
      } else {
        wait_vmcnt<0>();
      }
      if (there == 0) continue;
      const int k0 = key0 + t * C::UNIT;
      const uint16_t* tile = tiles[wave][t & 1];
      const bool masked = there != 0xffffffffu || k0 < b_max || k0 + 32 > e_min;

      f32x4 s[QB][2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) s[qb][kb] = f32x4{};
#pragma unroll
        for (int ks = 0; ks < C::KS; ++ks) {
          const bf16x8 k = as_bf16x8(*reinterpret_cast<const u32x4*>(
              &tile[(16 * kb + l16) * C::DQKP + ((4 * ks + gq) ^ k_sw) * 8]));
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) s[qb][kb] = mfma16(k, qv[qb][ks], s[qb][kb]);
        }
      }
      if (masked) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int k = 16 * kb + 4 * gq + i;
              const bool seen = (there >> k & 1) && k0 + k >= see_b[qb] && k0 + k < see_e[qb];
              s[qb][kb][i] = seen ? s[qb][kb][i] : kMasked;
            }
      }
      float own[QB];
      bool grow = false;
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        own[qb] = kMasked;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) own[qb] = fmaxf(own[qb], s[qb][kb][i]);
        grow |= own[qb] > m_run[qb] + kLazyMaxStep;
      }
      if (__builtin_amdgcn_ballot_w64(grow) != 0) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          float m = fmaxf(own[qb], __shfl_xor(own[qb], 16));
          m = fmaxf(m_run[qb], fmaxf(m, __shfl_xor(m, 32)));
          const float alpha = fast_exp2(m_run[qb] - m);
          m_run[qb] = m;
          l_run[qb] *= alpha;
#pragma unroll
          for (int d = 0; d < C::DV; ++d) o[qb][d] *= alpha;
        }
      }
      bf16x8 p[QB];
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        // the sum is taken over the bf16-rounded probabilities, the values that the product uses
        bf16x2 h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x2 e = {fast_exp2(s[qb][i >> 1][2 * (i & 1)] - m_run[qb]),
                           fast_exp2(s[qb][i >> 1][2 * (i & 1) + 1] - m_run[qb])};
          h[i] = __builtin_convertvector(e, bf16x2);
          l_run[qb] = __builtin_amdgcn_fdot2_f32_bf16(h[i], kOnesBf16x2, l_run[qb], false);
        }
        p[qb] = as_bf16x8(u32x4{__builtin_bit_cast(uint32_t, h[0]), __builtin_bit_cast(uint32_t, h[1]),
                                __builtin_bit_cast(uint32_t, h[2]), __builtin_bit_cast(uint32_t, h[3])});
      }
      // keys 4 gq + 0 .. 3 and 16 + 4 gq + 0 .. 3 in k-order, for both operands
      const uint16_t* v0 = tile + v_row * C::DQKP + (v_col & 1) * 4;
#pragma unroll
      for (int d = 0; d < C::DV; ++d) {
        const int ch = ((2 * d + (v_col >> 1)) ^ v_sw) * 8;
        const i16x4 lo = lds_read_tr(v0 + ch), hi = lds_read_tr(v0 + 16 * C::DQKP + ch);
        bf16x8 v = join_bf16x8(lo, hi);
        if (masked) v = finite_or_zero(v);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) o[qb][d] = mfma16(v, p[qb], o[qb][d]);
      }
    }

    // ---- the waves' results, merged in wave order ----
    float* res = reinterpret_cast<float*>(&tiles[wave][0][0]);  // [ROWS][RS]: this wave's own buffers
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      float l = l_run[qb];
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      if (gq == 0) {
        red_m[wave][16 * qb + l16] = m_run[qb];
        red_l[wave][16 * qb + l16] = l;
      }
#pragma unroll
      for (int d = 0; d < C::DV; ++d)
        *reinterpret_cast<f32x4*>(&res[(16 * qb + l16) * C::RS + 16 * d + 4 * gq]) = o[qb][d];
    }
    __syncthreads();
    const bool whole = take == n_units;
    const int64_t slot = 2 * (int64_t)blockIdx.x + (u0 == 0);
    for (int i = threadIdx.x; i < C::ROWS * (DC / 4); i += NW * 64) {
      const int r = i / (DC / 4), c = i % (DC / 4) * 4;
      if (row0 + r >= n_rows) break;
      float m = kLowest, l = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) m = fmaxf(m, red_m[w][r]);
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float f = fast_exp2(red_m[w][r] - m);
        l += f * red_l[w][r];
        v += f * *reinterpret_cast<const f32x4*>(
                     reinterpret_cast<const float*>(&tiles[w][0][0]) + r * C::RS + c);
      }
      if (whole) {
        v *= l == 0.f ? 0.f : 1.f / l;  // a row that sees nothing: zeros
        *reinterpret_cast<f32x4*>(a.o_lat + ((int64_t)q.lo * H + row0 + r) * DC + c) = v;
      } else {
        *reinterpret_cast<f32x4*>(a.o_part + (slot * C::ROWS + r) * DC + c) = v;
        if (c == 0) {
          a.ml_part[(slot * C::ROWS + r) * 2] = m;
          a.ml_part[(slot * C::ROWS + r) * 2 + 1] = l;
        }
      }
    }
    __syncthreads();  // the buffers are free for the next segment
    left -= take;
    end = 0;
    --blk;
  }
}

// ---- merge and value up-projection -------------------------------------------------------------
// grid (ceil(n_tokens / TG), H), 256 threads: the latents of TG tokens of one head, merged where their
// row block was split, then out^T[v][token] = W_UV_h[v][:] . o_lat[token][:]. The latents go into the
// product as two bf16 terms (16 bits of fraction): one alone adds a rounding as large as the output's
// own, 2^-8 of the value, for a product that costs next to nothing here.
template <int DC, int TG>
__global__ __launch_bounds__(256) void paged_out_kernel(const PagedAttendArgs a) {
  constexpr int LS = (DC > 32 ? DC : 32) + 8;  // LDS row stride (elements)
  constexpr int KS = (DC + 31) / 32;
  constexpr int C4 = DC / 4;                   // 16-byte chunks of a partial row
  constexpr int SL = 256 / C4 < 16 ? 256 / C4 : 16;  // splits read side by side
  __shared__ __attribute__((aligned(16))) uint16_t lat[2][TG][LS];  // o_lat's first and second term
  __shared__ f32x4 part[SL][C4];
  __shared__ float part_m[SL], part_l[SL];
  __shared__ int32_t tok_row[TG], tok_w0[TG], tok_ns[TG];  // (ns 0: no token of a sequence)
  const PagedGeo& g = a.pg;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int gq = lane >> 4, l16 = lane & 15;
  const int H = a.n_heads, h = blockIdx.y, t0 = blockIdx.x * TG;

  if (tid < TG) {
    const int t = t0 + tid, s = t < g.n_tokens ? paged_seq_of(g, t) : -1;
    const int r = s >= 0 ? (t - max(g.cu[s], 0)) * H + h : 0;
    const int blk = s >= 0 ? a.plan.seq_block[s] + r / a.rows : 0;
    const bool known = s >= 0 && blk < a.plan.seq_block[g.n_seqs];  // (else offsets that go down)
    tok_ns[tid] = 0;
    if (known) {
      const int64_t U = a.plan.head[0], G = a.plan.head[1];
      const int w0 = (int)floor_div((a.plan.first_unit[blk] + 1) * G - 1, U);
      tok_row[tid] = r % a.rows;
      tok_w0[tid] = w0;
      tok_ns[tid] = (int)floor_div(a.plan.first_unit[blk + 1] * G - 1, U) - w0 + 1;
    }
  }
  if constexpr (DC < 32) {
    for (int i = tid; i < 2 * TG * LS; i += 256) (&lat[0][0][0])[i] = 0;
  }
  __syncthreads();
  auto put = [&](int t, int c4, f32x4 v) {  // chunk c4 of token t's latents
    const bf16x4 hi = to_bf16x4(v);
    const f32x4 rest = v - __builtin_convertvector(hi, f32x4);
    *reinterpret_cast<bf16x4*>(&lat[0][t][c4 * 4]) = hi;
    *reinterpret_cast<bf16x4*>(&lat[1][t][c4 * 4]) = to_bf16x4(rest);
  };

  // tokens of unsplit blocks: every load issued before the first is used
  constexpr int PER = (TG * C4 + 255) / 256;
  f32x4 whole[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = tid + 256 * i, t = e / C4;
    if (e < TG * C4 && tok_ns[t] == 1)
      whole[i] = *reinterpret_cast<const f32x4*>(a.o_lat + ((int64_t)(t0 + t) * H + h) * DC + e % C4 * 4);
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = tid + 256 * i, t = e / C4;
    if (e < TG * C4 && tok_ns[t] == 1) put(t, e % C4, whole[i]);
  }
  for (int t = 0; t < TG; ++t) {
    const int ns = tok_ns[t], w0 = tok_w0[t];
    if (ns <= 1) continue;
    const int slice = tid / C4, c = tid % C4;
    float m = kLowest, l = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (slice < SL) {
      for (int k = slice; k < ns; k += SL) {
        const int64_t row = (2 * (int64_t)(w0 + k) + (k == 0)) * a.rows + tok_row[t];
        const f32x2 ml = *reinterpret_cast<const f32x2*>(a.ml_part + row * 2);
        const f32x4 x = *reinterpret_cast<const f32x4*>(a.o_part + row * DC + c * 4);
        const float m1 = fmaxf(m, ml[0]), f0 = fast_exp2(m - m1), f1 = fast_exp2(ml[0] - m1);
        l = l * f0 + ml[1] * f1;
        v = v * f0 + x * f1;
        m = m1;
      }
      part[slice][c] = v;
      if (c == 0) {
        part_m[slice] = m;
        part_l[slice] = l;
      }
    }
    __syncthreads();
    if (tid < C4) {
      m = kLowest;
      l = 0.f;
      v = f32x4{0.f, 0.f, 0.f, 0.f};
      for (int k = 0; k < SL; ++k) m = fmaxf(m, part_m[k]);
      for (int k = 0; k < SL; ++k) {
        const float f = fast_exp2(part_m[k] - m);
        l += part_l[k] * f;
        v += part[k][tid] * f;
      }
      v *= l == 0.f ? 0.f : 1.f / l;  // a row that sees nothing: zeros
      put(t, tid, v);
    }
    __syncthreads();
  }
  __syncthreads();

  const int t = min(l16, TG - 1);
  bf16x8 b[2][KS];
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      b[k][ks] = as_bf16x8(*reinterpret_cast<const u32x4*>(&lat[k][t][ks * 32 + 8 * gq]));
  for (int vb = wave; vb < a.d_v / 16; vb += 4) {
    const uint16_t* w = a.w_uv + ((int64_t)h * a.d_v + vb * 16 + l16) * DC;
    f32x4 acc = {};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      u32x4 x = {0, 0, 0, 0};
      if (ks * 32 + 8 * gq < DC) x = ldg16(w + ks * 32 + 8 * gq);
      acc = mfma16(as_bf16x8(x), b[0][ks], acc);
      acc = mfma16(as_bf16x8(x), b[1][ks], acc);
    }
    if (l16 < TG && tok_ns[t] > 0)
      *reinterpret_cast<bf16x4*>(a.out + ((int64_t)(t0 + t) * H + h) * a.d_v + vb * 16 + 4 * gq) = to_bf16x4(acc);
  }
}

#define VMLA_PAGED_SHAPES(X) X(16, 8) X(64, 32) X(128, 32) X(192, 32) X(256, 32) X(512, 32)

}  // namespace

void paged_attend_shape(int d_c, int d_rope, int64_t max_rows, int32_t* rows, int32_t* unit) {
  const int wide = paged_wide_rows(d_c, d_rope);
  if (wide > 0 && max_rows > 32) {
    *rows = wide;
    *unit = 32;
    return;
  }
  *rows = max_rows <= 16 ? 16 : 32;
  *unit = 32 * few_waves(d_c);
}

hipError_t launch_paged_plan(const PagedAttendArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(paged_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_paged_attend(const PagedAttendArgs& a, hipStream_t s) {
  if (a.rows > 32) return launch_paged_attend_wide(a, s);
#define X(DC, DR)                                                                                     \
  if (a.d_c == DC && a.d_rope == DR) {                                                                \
    if (a.rows == 16)                                                                                 \
      hipLaunchKernelGGL((paged_attend_few_kernel<DC, DR, 1>), dim3(a.n_wg),                          \
                         dim3(64 * few_waves(DC)), 0, s, a);                                          \
    else                                                                                              \
      hipLaunchKernelGGL((paged_attend_few_kernel<DC, DR, 2>), dim3(a.n_wg),                          \
                         dim3(64 * few_waves(DC)), 0, s, a);                                          \
    return hipGetLastError();                                                                         \
  }
  VMLA_PAGED_SHAPES(X)
#undef X
  return hipErrorInvalidValue;
}

hipError_t launch_paged_out(const PagedAttendArgs& a, hipStream_t s) {
#define X(DC, DR)                                                                                     \
  if (a.d_c == DC && a.d_rope == DR) {                                                                \
    if (a.pg.n_tokens <= 128)                                                                         \
      hipLaunchKernelGGL((paged_out_kernel<DC, 1>), dim3(a.pg.n_tokens, a.n_heads), dim3(256), 0, s, a); \
    else                                                                                              \
      hipLaunchKernelGGL((paged_out_kernel<DC, 16>), dim3((a.pg.n_tokens + 15) / 16, a.n_heads),      \
                         dim3(256), 0, s, a);                                                         \
    return hipGetLastError();                                                                         \
  }
  VMLA_PAGED_SHAPES(X)
#undef X
  return hipErrorInvalidValue;
}

}  // namespace vmla
