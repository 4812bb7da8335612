// Latent attention of new tokens over a paged cache (Section "Inference-Time Reparameterization", with
// a sequence's cached tokens in pages instead of a ring).
//
//   q_absorb       as for the ring (k_attend.hip), each token at its sequence's position; and, by one
//                  workgroup, the plan: row blocks, their key ranges and the even split of the work
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

typedef __attribute__((address_space(3))) int32_t lds_i32;

// Direct global-to-LDS load of 4 B per lane: lane l's word lands at lds_base + 4 l (see lds_dma16).
__device__ __forceinline__ void lds_dma4(const int32_t* gptr, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off"
               :
               : "v"(gptr), "s"(lds_base)
               : "memory", "m0");
}

// Waits until at most N vector-memory operations of the wave are outstanding; later LDS reads stay behind.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
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
  // Tile layout. d_c = 512: c_kv rows of 1 KB, so that a load is one row from a scalar base, then the k_r
  // rows. Otherwise rows [c_kv | k_r | pad].
  static constexpr bool SPLIT = DC == 512;
  static constexpr int STRIDE = SPLIT ? DC : DQKP;
  // The absorbed queries' two bf16 terms (see the scores). They are in LDS where with the accumulators they
  // would fill the registers: both, or at d_c = 512, where the tiles leave no room for more, the first.
  static constexpr bool QLDS = QB * (2 * KS + DV) * 4 > 190;
  static constexpr bool LO_REG = !QLDS || SPLIT;
  // Chunk position of logical chunk c in row r. CPR is 4 or 12 mod 16, so the rows r .. r + 3 of one
  // chunk fall on different groups of four 4-bank groups; the XOR separates the rows 4 apart, by bit 1
  // first, since the transpose reads take two adjacent chunks of rows 4 j .. 4 j + 3 and the next four.
  __device__ static constexpr int swz(int r) {
    const int q = (r >> 2) & 3;
    return ((q & 1) << 1) | (q >> 1);
  }
  // SPLIT: rows of 64 chunks start on the same banks, so the XOR separates all 16 rows, and the rows
  // 0 .. 7 and 8 .. 15 of the transpose reads by pairs of chunks.
  __device__ static constexpr int swz16(int r) { return ((r << 1) & 15) | ((r >> 3) & 1); }
  static_assert(CPR % 16 == 4 || CPR % 16 == 12, "bank spread of the tile rows");
  static_assert(DC % 16 == 0 && 16 * CPR % 64 == 0 && NDMA + 1 < 64, "tile shape");
  static_assert(ROWS * RS * 4 <= 2 * TILE * 2, "a wave's results fit its tile buffers");
};

template <int DC, int DR, int QB>
__global__ __launch_bounds__(64 * few_waves(DC)) void paged_attend_few_kernel(const PagedAttendArgs a) {
  using C = FewCfg<DC, DR, QB>;
  constexpr int NW = C::NW;
  __shared__ __attribute__((aligned(16))) uint16_t tiles[NW][2][C::TILE];
  __shared__ __attribute__((aligned(16))) uint16_t qs[C::QLDS ? (C::LO_REG ? 1 : 2) * C::ROWS * C::DQKP : 8];
  __shared__ int32_t ids[NW][2][64];
  __shared__ float red_m[NW][C::ROWS], red_l[NW][C::ROWS];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int gq = lane >> 4, l16 = lane & 15;
  const PagedGeo& g = a.pg;
  const int H = a.n_heads;
  const PagedWork wk = paged_read<true>(a.plan.work, blockIdx.x);
  int left = wk.n, blk = wk.block, end = wk.end;

  // Load j of a tile fills the chunk slots 64 j .. 64 j + 63: of this lane's chunk, in bits 0..15 the
  // offset in its row's c_kv, or (bit 31) k_r, or (bit 30) the pad of q_cat's first row, which is zero as the
  // pad has to be (an infinity there, times the zero in q_cat, would be NaN); in bits 16..19 the row modulo
  // 16. Half a tile is a whole number of loads, and the other half repeats it.
  // (SPLIT: of the two loads of k_r, from load 32 on.)
  constexpr int NAT = C::SPLIT ? 1 : C::NDMA / 2;
  uint32_t d_at[NAT];
  if constexpr (C::SPLIT) {
    const int r = lane >> 2;
    d_at[0] = 0x80000000u | (uint32_t)r << 16 | (((lane & 3) ^ C::swz(r)) * 8);
  } else {
#pragma unroll
    for (int j = 0; j < NAT; ++j) {
      const int slot = j * 64 + lane, r = slot / C::CPR, c = (slot % C::CPR) ^ C::swz(r);
      d_at[j] = (uint32_t)r << 16 | (c < DC / 8 ? c * 8 : c < (DC + DR) / 8 ? 0x80000000u | (c * 8 - DC) : 0x40000000u);
    }
  }

  while (left > 0) {
    const bool last = blk == wk.block;  // (whose record the plan has copied: one load less in line)
    const PagedBlock pb = last ? paged_read<true>(a.plan.work_block, blockIdx.x) : paged_read<true>(a.plan.block, blk);
    if (end < 0) end = pb.n_units + a.cost;  // a block before the workgroup's last is taken to its end
    const int len = min(left, end), u1 = end - a.cost, u0 = max(u1 - len, 0), take = u1 - u0;
    left -= len;
    end = -1;
    --blk;
    if (take <= 0) continue;
    const int key0 = pb.key0 + u0 * C::UNIT + wave * 32;  // this wave's first
    const int row0 = pb.row0, n_rows = pb.n_rows;
    const int32_t* table = g.table + (int64_t)pb.seq * g.max_pages;

    // page ids of tile t's keys, one per lane, into slot t & 1 (a key outside the sequence reads the
    // nearest entry of the table, and is no row below)
    auto load_ids = [&](int t) {
      const int key = min(key0 + t * C::UNIT + (lane & 31), g.max_kv - 1);
      lds_dma4(table + page_of(g, key), __builtin_amdgcn_readfirstlane(lds_addr(&ids[wave][t & 1][0])));
    };
    load_ids(0);
    load_ids(1);

    // this lane's rows and what they see
    bf16x8 qv[C::QLDS ? 1 : QB][C::KS], qlo[C::LO_REG ? QB : 1][C::KS];
    int see_b[QB], see_e[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const int r = row0 + 16 * qb + l16;
      paged_row_sees(g, pb, H, min(16 * qb + l16, n_rows - 1 - row0), see_b[qb], see_e[qb]);  // (past the end: as the last)
      auto own_row = [&](const uint16_t* q, bf16x8 (&v)[C::KS]) {
        const uint16_t* src = q + ((int64_t)pb.lo * H + (r < n_rows ? r : row0)) * C::DQKP + 8 * gq;
#pragma unroll
        for (int ks = 0; ks < C::KS; ++ks) {
          u32x4 x = ldg16(src + ks * 32);
          if (r >= n_rows) x = u32x4{0, 0, 0, 0};
          v[ks] = as_bf16x8(x);
        }
      };
      if constexpr (!C::QLDS) own_row(a.qcat, qv[qb]);
      if constexpr (C::LO_REG) own_row(a.q_lo, qlo[qb]);
    }
    if constexpr (C::QLDS) {  // laid out as the tile's rows, so that the reads are as free of conflicts
      for (int i = threadIdx.x; i < (C::LO_REG ? 1 : 2) * C::ROWS * C::CPR; i += NW * 64) {
        const int rr = i / C::CPR, c = i % C::CPR, r = rr % C::ROWS;
        u32x4 v = ldg16((rr < C::ROWS ? a.qcat : a.q_lo) +
                        ((int64_t)pb.lo * H + row0 + (row0 + r < n_rows ? r : 0)) * C::DQKP + c * 8);
        if (row0 + r >= n_rows) v = u32x4{0, 0, 0, 0};
        *reinterpret_cast<u32x4*>(&qs[rr * C::DQKP + (c ^ C::swz(r)) * 8]) = v;
      }
      __syncthreads();
    }

    f32x4 o[QB][C::DV];
    float m_run[QB], l_run[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      m_run[qb] = kLowest;
      l_run[qb] = 0.f;
#pragma unroll
      for (int d = 0; d < C::DV; ++d) o[qb][d] = f32x4{};
    }

    auto row_of = [&](int t) {  // this lane's key's pool row, -1: none
      const int key = key0 + t * C::UNIT + (lane & 31);
      // (through an LDS pointer: a generic one would wait for every load in flight)
      const int32_t page = *(const volatile lds_i32*)(&ids[wave][t & 1][lane]);
      const int row = page * g.page_tokens + key - page_of(g, key) * g.page_tokens;
      return key < pb.kv && (uint32_t)page < (uint32_t)g.n_pages ? row : -1;
    };
    auto load_tile = [&](int t, int row) {
      const int at_row = max(row, 0);  // in a missing key's place, the pool's first row: masked, made finite
      const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_addr(&tiles[wave][t & 1][0]));
      if constexpr (C::SPLIT) {
        int ln = lane;
        asm volatile("" : "+v"(ln));  // the 16 offsets are recomputed: kept across the loop they would spill
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          const uint32_t r = __builtin_amdgcn_readlane(at_row, j);
          lds_dma16_row(a.c_kv + (uint64_t)r * DC, (ln ^ C::swz16(j)) * 16, lds + 1024u * j);
        }
      }
#pragma unroll
      for (int j = C::SPLIT ? 32 : 0; j < C::NDMA; ++j) {
        const int half = C::SPLIT ? j - 32 : j / NAT;
        uint32_t at = d_at[j % NAT];
        // recomputed from one register a load: kept across the loop, the addresses' parts would fill the file
        if constexpr (DC == 256) asm volatile("" : "+v"(at));
        const uint32_t r = __shfl(at_row, (int)(at >> 16 & 15) + 16 * half);
        const bool kr = (int32_t)at < 0;
        const uint16_t* p = (kr ? a.k_r : a.c_kv) + (at & 0xffffu);
        p += (uint64_t)r * (uint32_t)(kr ? DR : DC);
        if constexpr (C::DQKP > DC + DR) p = at & 0x40000000u ? a.qcat + DC + DR : p;
        lds_dma16(p, lds + 1024u * j);
      }
    };

    // The K operand of step ks (lane: row l16 + 16 kb, chunk 4 ks + gq) and the transpose reads' rows (lane:
    // row 4 gq + l16 / 4 (+ 16), columns 4 (l16 % 4) + 16 d). The XORs stay below 4 (SPLIT: 16) chunks, so
    // that a few bases and immediate offsets reach every step.
    const int v_row = 4 * gq + (l16 >> 2), v_ch = (l16 >> 1) & 1;
    constexpr int NKB = C::SPLIT ? 5 : 1, NVB = C::SPLIT ? 8 : 2;
    int k_base[NKB], v_base[NVB];
    if constexpr (C::SPLIT) {
#pragma unroll
      for (int i = 0; i < 4; ++i) k_base[i] = l16 * DC + (((4 * i + gq) ^ C::swz16(l16)) << 3);
      k_base[4] = 32 * DC + l16 * DR + ((gq ^ C::swz(l16)) << 3);
#pragma unroll
      for (int i = 0; i < 8; ++i) v_base[i] = v_row * DC + (((2 * i + v_ch) ^ C::swz16(v_row)) << 3) + (l16 & 1) * 4;
    } else {
      k_base[0] = l16 * C::DQKP + ((gq ^ C::swz(l16)) << 3);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        v_base[i] = v_row * C::DQKP + (((2 * i + v_ch) ^ C::swz(v_row)) << 3) + (l16 & 1) * 4;
    }
    auto k_at = [&](int kb, int ks) {
      if constexpr (C::SPLIT)
        return ks < DC / 32 ? k_base[ks & 3] + kb * 16 * DC + (ks >> 2) * 128 : k_base[4] + kb * 16 * DR;
      else return k_base[0] + kb * 16 * C::DQKP + ks * 32;
    };
    auto v_at = [&](int d) {
      if constexpr (C::SPLIT) return v_base[d & 7] + (d >> 3) * 128;
      else return v_base[d & 1] + (d >> 1) * 32;
    };
    auto q_at = [&](int term, int qb, int ks) {
      if constexpr (C::QLDS)
        return as_bf16x8(*reinterpret_cast<const u32x4*>(
            &qs[(term * C::ROWS + 16 * qb + l16) * C::DQKP + ((gq ^ C::swz(l16)) << 3) + ks * 32]));
      else return qv[qb][ks];
    };

    auto use_tile = [&](int t, uint32_t there) {
      const int k0 = key0 + t * C::UNIT;
      const uint16_t* tile = tiles[wave][t & 1];
      const bool masked = there != 0xffffffffu || k0 < pb.all_b || k0 + 32 > pb.all_e;

      // Both terms of the absorbed queries: one alone is off by up to 2^-8 of each component, which moves a
      // score of size |s| by about 2^-9.5 |s| and weighs most where the softmax is peaked (scores of standard
      // deviation 4: outputs off by 0.0044 in the 2-norm with one term, 0.0018 with two). These matrix steps
      // pass under the loads of the keys, which bound this kernel. The second term's sum is kept apart: of an
      // infinite k^R the two may be infinities of opposite signs, and the first alone is the score.
      f32x4 s[QB][2], s_lo[QB][2];
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) s[qb][0] = s[qb][1] = s_lo[qb][0] = s_lo[qb][1] = f32x4{};
#pragma unroll
      for (int ks = 0; ks < C::KS; ++ks) {
        const bf16x8 k0v = as_bf16x8(*reinterpret_cast<const u32x4*>(&tile[k_at(0, ks)]));
        const bf16x8 k1v = as_bf16x8(*reinterpret_cast<const u32x4*>(&tile[k_at(1, ks)]));
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          const bf16x8 qk = q_at(0, qb, ks);
          s[qb][0] = mfma16(k0v, qk, s[qb][0]);
          s[qb][1] = mfma16(k1v, qk, s[qb][1]);
          bf16x8 ql;
          if constexpr (C::LO_REG) ql = qlo[qb][ks];
          else ql = q_at(1, qb, ks);
          s_lo[qb][0] = mfma16(k0v, ql, s_lo[qb][0]);
          s_lo[qb][1] = mfma16(k1v, ql, s_lo[qb][1]);
        }
      }
      const float most = most_here();
#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int i = 0; i < 8; ++i) s[qb][i >> 2][i & 3] += second_part(s_lo[qb][i >> 2][i & 3], most);
      if (masked) {
        float least = s[0][0][0];
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
#pragma unroll
          for (int i = 0; i < 8; ++i) least = fminf(least, s[qb][i >> 2][i & 3]);
        uint32_t bad = 0;
        if (__builtin_amdgcn_ballot_w64(least == kMasked) != 0)
          bad = not_finite_keys<DC / 8>([&](int r, int c) {
            return tile + r * C::STRIDE + (c ^ (C::SPLIT ? C::swz16(r) : C::swz(r))) * 8;
          });
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          const uint32_t sees = seen_keys(there, see_b[qb] - k0, see_e[qb] - k0), seen = sees >> (4 * gq);
          l_run[qb] = sees & bad ? kNotANumber : l_run[qb];
#pragma unroll
          for (int i = 0; i < 8; ++i)
            s[qb][i >> 2][i & 3] = seen >> (16 * (i >> 2) + (i & 3)) & 1 ? s[qb][i >> 2][i & 3] : kMasked;
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
      auto pv = [&](auto clear) {
#pragma unroll
        for (int d = 0; d < C::DV; ++d) {
          const uint16_t* v0 = tile + v_at(d);
          const i16x4 lo = lds_read_tr(v0), hi = lds_read_tr(v0 + 16 * C::STRIDE);
          bf16x8 v = join_bf16x8(lo, hi);
          if constexpr (decltype(clear)::value) v = finite_or_zero(v);
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) o[qb][d] = mfma16(v, p[qb], o[qb][d]);
        }
      };
      if (masked) pv(std::true_type{});
      else pv(std::false_type{});
    };

    wait_loads<0>();
    int row = row_of(0), row_n = row_of(1);
    load_tile(0, row);
    load_ids(2);
    if (take > 1) load_tile(1, row_n);
    // outstanding at the top of iteration t: the loads of tile t, the ids of tile t + 2, the loads of t + 1
    for (int t = 0; t < take; ++t) {
      const uint32_t there = (uint32_t)__builtin_amdgcn_ballot_w64(row >= 0);  // keys of tile t that exist
      if (t + 1 < take) wait_loads<C::NDMA + 1>();
      else wait_loads<0>();
      if (there != 0) use_tile(t, there);
      row = row_n;
      if (t + 2 < take) {
        wait_loads<C::NDMA>();  // the ids of tile t + 2
        row_n = row_of(t + 2);
        load_ids(t + 3);
        load_tile(t + 2, row_n);  // into tile t's buffer: its values are in registers
      }
    }

    // ---- the waves' results, merged in wave order ----
    float* res = reinterpret_cast<float*>(&tiles[wave][0][0]);  // [ROWS][RS]: this wave's own buffers
    const bool whole = take == pb.n_units;
    const int64_t slot = 2 * (int64_t)blockIdx.x + (u0 == 0);
    if (u0 == 0 && (int)threadIdx.x < C::ROWS && row0 + (int)threadIdx.x < n_rows)
      a.plan.row[(int64_t)pb.lo * H + row0 + threadIdx.x] =
          PagedRow{(int32_t)blockIdx.x, (uint16_t)(last ? wk.last_ns : 1), (uint16_t)threadIdx.x};
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
        v += f * *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(&tiles[w][0][0]) + r * C::RS + c);
      }
      if (whole) {
        v *= l == 0.f ? 0.f : 1.f / l;  // a row that sees nothing: zeros
        *reinterpret_cast<f32x4*>(a.o_lat + ((int64_t)pb.lo * H + row0 + r) * DC + c) = v;
      } else {
        *reinterpret_cast<f32x4*>(a.o_part + (slot * C::ROWS + r) * DC + c) = v;
        if (c == 0) {
          a.ml_part[(slot * C::ROWS + r) * 2] = m;
          a.ml_part[(slot * C::ROWS + r) * 2 + 1] = l;
        }
      }
    }
    __syncthreads();  // the buffers are free for the next block
  }
}

// ---- merge and value up-projection -------------------------------------------------------------
// out[token, h] = W_UV_h o_lat[token, h], o_lat merged where its row block was split. The latents go into
// the product as two bf16 terms (16 bits of fraction): one alone adds a rounding as large as the output's
// own, 2^-8 of the value, for a product that costs next to nothing here.
__device__ __forceinline__ void two_terms(f32x8 v, bf16x8& hi, bf16x8& lo) {
  hi = to_bf16x8(v);
  lo = to_bf16x8(v - __builtin_convertvector(hi, f32x8));
}
// Partial row of split k of a row (its first partial has the first key: slot 2 w + 1).
__device__ __forceinline__ int64_t paged_part_row(const PagedAttendArgs& a, const PagedRow& r, int k) {
  return (2 * (int64_t)(r.w0 + k) + (k == 0)) * a.rows + r.row;
}

// Few tokens (single-token steps, whose rows are split the most): a workgroup per row.
// Slices of the workgroup merge the splits side by side, each with its own running maximum; a wave then
// takes 16 of the d_v outputs at a time, whose weights are on their way meanwhile.
template <int DC>
__global__ __launch_bounds__(256) void paged_out_row_kernel(const PagedAttendArgs a) {
  constexpr int LS = (DC > 32 ? DC : 32);
  constexpr int KS = (DC + 31) / 32;
  constexpr int C4 = DC / 4;                           // 16-byte chunks of a partial row
  constexpr int SL = 256 / C4 < 16 ? 256 / C4 : 16;    // slices
  constexpr int AHEAD = DC > 256 ? 1 : 2;
  __shared__ __attribute__((aligned(16))) uint16_t lat[2][LS];  // o_lat's first and second term
  __shared__ f32x4 part[SL][C4];
  __shared__ float part_m[SL], part_l[SL];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int gq = lane >> 4, l16 = lane & 15;
  const int64_t row = blockIdx.x;
  const int h = (int)(blockIdx.x % (unsigned)a.n_heads);
  const PagedRow at = paged_read<true>(a.plan.row, row);

  const int n_vb = a.d_v / 16;
  auto weight = [&](int vb, int ks) {
    u32x4 x = {0, 0, 0, 0};
    if (ks * 32 + 8 * gq < DC)
      x = ldg16(a.w_uv + ((int64_t)h * a.d_v + vb * 16 + l16) * DC + ks * 32 + 8 * gq);
    return as_bf16x8(x);
  };
  bf16x8 wv[AHEAD][KS];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) wv[i][ks] = weight(min(wave * AHEAD + i, n_vb - 1), ks);
  if (at.ns == 0) return;  // a row of no sequence

  auto put = [&](int c4, f32x4 v) {
    const bf16x4 hi = to_bf16x4(v);
    *reinterpret_cast<bf16x4*>(&lat[0][c4 * 4]) = hi;
    *reinterpret_cast<bf16x4*>(&lat[1][c4 * 4]) = to_bf16x4(v - __builtin_convertvector(hi, f32x4));
  };
  if constexpr (DC < 32) {
    if (tid < 32) lat[0][tid] = lat[1][tid] = 0;
    __syncthreads();
  }
  if (at.ns == 1) {
    if (tid < C4) put(tid, *reinterpret_cast<const f32x4*>(a.o_lat + row * DC + tid * 4));
  } else {
    const int slice = tid / C4, c = tid % C4;
    if (slice < SL) {
      float m = kLowest, l = 0.f;
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
      for (int k = slice; k < at.ns; k += 4 * SL) {
        f32x2 ml[4];
        f32x4 x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int64_t pr = paged_part_row(a, at, k + j * SL < at.ns ? k + j * SL : k);  // (past the last: not used)
          ml[j] = *reinterpret_cast<const f32x2*>(a.ml_part + pr * 2);
          x[j] = *reinterpret_cast<const f32x4*>(a.o_part + pr * DC + c * 4);
        }
        float m1 = m;
#pragma unroll
        for (int j = 0; j < 4; ++j) m1 = fmaxf(m1, ml[j][0]);
        const float f = fast_exp2(m - m1);
        l *= f;
        v *= f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (k + j * SL < at.ns) {
            const float fj = fast_exp2(ml[j][0] - m1);
            l += fj * ml[j][1];
            v += fj * x[j];
          }
        }
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
      float m = kLowest, l = 0.f;
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
      for (int k = 0; k < SL; ++k) m = fmaxf(m, part_m[k]);
      for (int k = 0; k < SL; ++k) {
        const float f = fast_exp2(part_m[k] - m);
        l += part_l[k] * f;
        v += part[k][tid] * f;
      }
      put(tid, v * (l == 0.f ? 0.f : 1.f / l));  // (a row that sees nothing: zeros)
    }
  }
  __syncthreads();
  for (int vb = wave * AHEAD; vb < n_vb; vb += 4 * AHEAD) {
    if (vb != wave * AHEAD) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) wv[i][ks] = weight(min(vb + i, n_vb - 1), ks);
    }
    f32x4 acc[AHEAD] = {};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const bf16x8 b = as_bf16x8(*reinterpret_cast<const u32x4*>(&lat[k][ks * 32 + 8 * gq]));
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) acc[i] = mfma16(wv[i][ks], b, acc[i]);
      }
    if (l16 == 0) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        if (vb + i < n_vb)
          *reinterpret_cast<bf16x4*>(a.out + row * a.d_v + (vb + i) * 16 + 4 * gq) = to_bf16x4(acc[i]);
    }
  }
}

// More tokens: 4 waves x 16 tokens of one head per workgroup. A lane holds 8 of every 32 latents of its
// token, loaded as the B operand needs them (whole lines: four lanes a token) and merged over the splits
// in registers; W_UV_h passes through LDS, 64 rows at a time, and is read by all waves. Two blocks of 16
// tokens per wave halve the reads of W_UV_h, and the workgroups that fit a compute unit: 8,190 tokens x 12
// heads 41 us against 34, 2,808 tokens with two to three splits a row 30 against 24.
template <int DC>
__global__ __launch_bounds__(256, DC <= 192 ? 4 : DC <= 256 ? 3 : 2) void paged_out_tiles_kernel(const PagedAttendArgs a) {
  constexpr int KS = (DC + 31) / 32;
  constexpr int LS = KS * 32 + 8;               // LDS row stride (elements): rows 16 bytes apart in banks
  constexpr int VR = 64, CPR = KS * 4;          // W rows per pass, 16-byte chunks per row
  constexpr int PER = VR * CPR / 256;           // W chunks per thread and pass
  constexpr int YS = KS > 6 ? 4 : KS;           // k-steps of a further split in flight
  __shared__ __attribute__((aligned(16))) uint16_t wl[VR * LS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int gq = lane >> 4, l16 = lane & 15;
  const int H = a.n_heads, n = a.pg.n_tokens;
  const int h = (int)(blockIdx.x % (unsigned)H);
  const int t = ((int)(blockIdx.x / (unsigned)H) * 4 + wave) * 16 + l16;

  u32x4 wv[PER];
  auto load_w = [&](int v0) {  // (rows past d_v repeat the last; d_c = 16: the second half of a k-step is zero)
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = tid + 256 * i, r = min(v0 + e / CPR, a.d_v - 1), c = e % CPR;
      wv[i] = c * 8 < DC ? ldg16(a.w_uv + ((int64_t)h * a.d_v + r) * DC + c * 8) : u32x4{0, 0, 0, 0};
    }
  };
  load_w(0);

  const int64_t row = (int64_t)min(t, n - 1) * H + h;
  const PagedRow at = a.plan.row[row];
  const int ns = t < n ? at.ns : 0;
  f32x8 x[KS];
  auto load = [&](const float* p, int k0, auto& v) {  // the lane's latents of the k-steps from k0 on
#pragma unroll
    for (int ks = 0; ks < (int)(sizeof(v) / sizeof(v[0])); ++ks) {
      const int c = (k0 + ks) * 32 + 8 * gq;
      f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
      if (DC % 32 == 0 || c < DC) {
        lo = *reinterpret_cast<const f32x4*>(p + c);
        hi = *reinterpret_cast<const f32x4*>(p + c + 4);
      }
      v[ks] = f32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    }
  };
  load(ns <= 1 ? a.o_lat + row * DC : a.o_part + paged_part_row(a, at, 0) * DC, 0, x);
  if (ns > 1) {
    auto ml_of = [&](int k) { return *reinterpret_cast<const f32x2*>(a.ml_part + paged_part_row(a, at, k) * 2); };
    float m = kLowest, l = 0.f;
    for (int k = 0; k < ns; ++k) m = fmaxf(m, ml_of(k)[0]);
    for (int k = 0; k < ns; ++k) {
      const f32x2 ml = ml_of(k);
      l += fast_exp2(ml[0] - m) * ml[1];
    }
    const float il = l == 0.f ? 0.f : 1.f / l;  // (a row that sees nothing: zeros)
    const float f0 = fast_exp2(ml_of(0)[0] - m) * il;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) x[ks] *= f0;
    for (int k = 1; k < ns; ++k) {
      const float* p = a.o_part + paged_part_row(a, at, k) * DC;
      const float f = fast_exp2(ml_of(k)[0] - m) * il;
#pragma unroll
      for (int k0 = 0; k0 < KS; k0 += YS) {
        f32x8 y[YS];
        load(p, k0, y);
#pragma unroll
        for (int ks = 0; ks < YS; ++ks) x[k0 + ks] += f * y[ks];
      }
    }
  }
  bf16x8 o[2][KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) two_terms(x[ks], o[0][ks], o[1][ks]);

  for (int v0 = 0; v0 < a.d_v; v0 += VR) {
    if (v0 > 0) __syncthreads();  // the previous rows are used
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = tid + 256 * i;
      *reinterpret_cast<u32x4*>(&wl[e / CPR * LS + e % CPR * 8]) = wv[i];
    }
    __syncthreads();
    if (v0 + VR < a.d_v) load_w(v0 + VR);
#pragma unroll 1
    for (int vb = 0; vb < VR / 16 && v0 + vb * 16 < a.d_v; ++vb) {
      f32x4 acc = {};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8 w = as_bf16x8(*reinterpret_cast<const u32x4*>(&wl[(vb * 16 + l16) * LS + ks * 32 + 8 * gq]));
        acc = mfma16(w, o[0][ks], acc);
        acc = mfma16(w, o[1][ks], acc);
      }
      if (ns > 0) *reinterpret_cast<bf16x4*>(a.out + row * a.d_v + v0 + vb * 16 + 4 * gq) = to_bf16x4(acc);
    }
  }
}

#define VMLA_PAGED_SHAPES(X) X(16, 8) X(64, 32) X(128, 32) X(192, 32) X(256, 32) X(512, 32)

}  // namespace

namespace {
// 16-row blocks per workgroup of the few-row kernel, at most: beyond, the wide kernel is as fast or faster. us,
// few / wide, d_c = 192: 24 rows x 8 sequences of 16,000 keys 22.1 / 20.6, of 32,760 32.6 / 32.3, x 32 of 2,000 to
// 32,760 52.4 / 62.1; 48 rows x 8 of 3,000 to 16,000 22.6 / 19.0, to 32,760 31.9 / 23.7. At d_c = 256 and 512 two
// blocks' accumulators and queries do not fit.
constexpr int few_most(int dc) { return dc <= 192 ? 2 : 1; }
}  // namespace

void paged_attend_shape(int d_c, int d_rope, int64_t max_rows, int32_t* rows, int32_t* unit, int32_t* cost) {
  const int most = 16 * few_most(d_c);
  if (max_rows > most) {
    *rows = paged_wide_rows(d_c, d_rope);
    *unit = 32;
    *cost = 8;
    return;
  }
  *rows = max_rows <= 16 ? 16 : most;
  *unit = 32 * few_waves(d_c);
  *cost = 3;
}

hipError_t launch_paged_attend(const PagedAttendArgs& a, hipStream_t s) {
  if (a.unit == 32) return launch_paged_attend_wide(a, s);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(a.n_wg), dim3(64 * few_waves(a.d_c)), 0, s, a);
    return hipGetLastError();
  };
#define X(DC, DR)                                                                                     \
  if (a.d_c == DC && a.d_rope == DR) {                                                                \
    if (a.rows == 16) return go(paged_attend_few_kernel<DC, DR, 1>);                                  \
    return go(paged_attend_few_kernel<DC, DR, few_most(DC)>);                                         \
  }
  VMLA_PAGED_SHAPES(X)
#undef X
  return hipErrorInvalidValue;
}

// The output kernel by row costs about 3 us and 1 us per 150 rows, whatever the splits; the one by tiles 9 us,
// 1 us per 1,500 rows and 2.3 us per split, which it merges one after the other (d_c = 192). us, row / tiles:
// 384 rows x 8 splits 6.2 / 12, 1,536 x 8 14.0 / 31, 1,536 x 32 16.8 / 81, 3,600 x 17 28.9 / 58,
// 1,440 x 2 12.6 / 12, 33,696 x 2 198 / 24. Splits are estimated from the row blocks that the tensors' sizes allow.
hipError_t launch_paged_out(const PagedAttendArgs& a, hipStream_t s) {
  const int n = a.pg.n_tokens;
  const int64_t rows = (int64_t)n * a.n_heads, blocks = rows / a.rows + 1;
  const bool by_row = rows <= 1000 + 400 * (a.n_wg / blocks);
#define X(DC, DR)                                                                                        \
  if (a.d_c == DC && a.d_rope == DR) {                                                                   \
    if (by_row)                                                                                          \
      hipLaunchKernelGGL(paged_out_row_kernel<DC>, dim3((unsigned)rows), dim3(256), 0, s, a);            \
    else                                                                                                 \
      hipLaunchKernelGGL(paged_out_tiles_kernel<DC>, dim3((unsigned)(((int64_t)n + 63) / 64 * a.n_heads)), \
                         dim3(256), 0, s, a);                                                            \
    return hipGetLastError();                                                                            \
  }
  VMLA_PAGED_SHAPES(X)
#undef X
  return hipErrorInvalidValue;
}

}  // namespace vmla
