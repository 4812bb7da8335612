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

// D(16x16) += A(16x32) B(32x16). Lane l holds A[l%16][8(l/16) .. +8], B[8(l/16) .. +8][l%16];
// accumulator element i of lane l is D[4(l/16) + i][l%16].
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

typedef __attribute__((address_space(3))) int32_t lds_i32;

// Direct global-to-LDS load of 4 B per lane: lane l's word lands at lds_base + 4 l (see lds_dma16).
__device__ __forceinline__ void lds_dma4(const int32_t* gptr, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off"
               :
               : "v"(gptr), "s"(lds_base)
               : "memory", "m0");
}

// The same of 16 B from a scalar base and a lane offset in bytes. The base has to be settled (no VALU
// instruction may write it in the five wait states before): callers compute it with scalar arithmetic.
__device__ __forceinline__ void lds_dma16_row(const void* base, uint32_t off, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(off), "s"(base), "s"(lds_base)
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
  static constexpr int QP = QB % 2 ? 1 : 2;              // 16-row blocks merged at a time
  static constexpr int UNIT = 32 * NW;
  static constexpr int RS = DC + 4;                      // row stride of the merged latents (floats)
  // Tile layout. d_c = 512: c_kv rows of 1 KB, so that a load is one row from a scalar base, then the k_r
  // rows. Otherwise rows [c_kv | k_r | pad].
  static constexpr bool SPLIT = DC == 512;
  static constexpr int STRIDE = SPLIT ? DC : DQKP;
  // The queries are in LDS where with the accumulators they would fill the registers.
  static constexpr bool QLDS = QB * (KS + DV) * 4 > 190;
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
  static_assert(16 * QP * RS * 4 <= 2 * TILE * 2, "a wave's results fit its tile buffers");
};

template <int DC, int DR, int QB>
__global__ __launch_bounds__(64 * few_waves(DC)) void paged_attend_few_kernel(const PagedAttendArgs a) {
  using C = FewCfg<DC, DR, QB>;
  constexpr int NW = C::NW;
  __shared__ __attribute__((aligned(16))) uint16_t tiles[NW][2][C::TILE];
  __shared__ __attribute__((aligned(16))) uint16_t qs[C::QLDS ? C::ROWS * C::DQKP : 8];
  __shared__ int32_t ids[NW][2][64];
  __shared__ float red_m[NW][16 * C::QP], red_l[NW][16 * C::QP];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int gq = lane >> 4, l16 = lane & 15;
  const PagedGeo& g = a.pg;
  const int H = a.n_heads;
  const PagedWork wk = paged_read<true>(a.plan.work, blockIdx.x);
  int left = wk.n, blk = wk.block, end = wk.end;

  // Load j of a tile fills the chunk slots 64 j .. 64 j + 63: of this lane's chunk, in bits 0..15 the
  // offset in its row's c_kv, or (bit 31) k_r (the pad reads k_r again, against zeros in q_cat), in bits
  // 16..19 the row modulo 16. Half a tile is a whole number of loads, and the other half repeats it.
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
      d_at[j] = (uint32_t)r << 16 | (c < DC / 8 ? c * 8 : 0x80000000u | (c < (DC + DR) / 8 ? c * 8 - DC : 0));
    }
  }

  while (left > 0) {
    const PagedBlock pb = paged_read<true>(a.plan.block, blk);
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

    // this lane's rows and what they see
    bf16x8 qv[C::QLDS ? 1 : QB][C::KS];
    int see_b[QB], see_e[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const int r = row0 + 16 * qb + l16;
      see_b[qb] = 0;
      see_e[qb] = 0x7fffffff;
      if (r < n_rows) paged_row_sees(g, pb, H, 16 * qb + l16, see_b[qb], see_e[qb]);
      if constexpr (!C::QLDS) {
        const uint16_t* src = a.qcat + ((int64_t)pb.lo * H + (r < n_rows ? r : row0)) * C::DQKP + 8 * gq;
#pragma unroll
        for (int ks = 0; ks < C::KS; ++ks) {
          u32x4 v = ldg16(src + ks * 32);
          if (r >= n_rows) v = u32x4{0, 0, 0, 0};
          qv[qb][ks] = as_bf16x8(v);
        }
      }
    }
    if constexpr (C::QLDS) {  // laid out as the tile's rows, so that the reads are as free of conflicts
      for (int i = threadIdx.x; i < C::ROWS * C::CPR; i += NW * 64) {
        const int r = i / C::CPR, c = i % C::CPR;
        u32x4 v = ldg16(a.qcat + ((int64_t)pb.lo * H + row0 + (row0 + r < n_rows ? r : 0)) * C::DQKP + c * 8);
        if (row0 + r >= n_rows) v = u32x4{0, 0, 0, 0};
        *reinterpret_cast<u32x4*>(&qs[r * C::DQKP + (c ^ C::swz(r)) * 8]) = v;
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
      if (key >= pb.kv || page < 0 || page >= g.n_pages) return -1;
      return page * g.page_tokens + key - page_of(g, key) * g.page_tokens;
    };
    auto load_tile = [&](int t, int row) {
      const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_addr(&tiles[wave][t & 1][0]));
      if constexpr (C::SPLIT) {
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          const int32_t r = __builtin_amdgcn_readlane(row, j);
          lds_dma16_row(r < 0 ? a.zero_row : a.c_kv + (int64_t)r * DC, (lane ^ C::swz16(j)) * 16, lds + 1024u * j);
        }
      }
#pragma unroll
      for (int j = C::SPLIT ? 32 : 0; j < C::NDMA; ++j) {
        const int half = C::SPLIT ? j - 32 : j / NAT;
        uint32_t at = d_at[j % NAT];
        // recomputed from one register a load: kept across the loop, the addresses' parts would fill the file
        if constexpr (QB * DC >= 256) asm volatile("" : "+v"(at));
        const int32_t r = __shfl(row, (int)(at >> 16 & 15) + 16 * half);
        const bool kr = (int32_t)at < 0;
        const uint16_t* p = kr ? a.k_r : a.c_kv;
        p += (int64_t)r * (kr ? DR : DC) + (at & 0xffffu);
        lds_dma16(r < 0 ? a.zero_row : p, lds + 1024u * j);
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
    auto q_at = [&](int qb, int ks) {
      if constexpr (C::QLDS)
        return as_bf16x8(*reinterpret_cast<const u32x4*>(
            &qs[(16 * qb + l16) * C::DQKP + ((gq ^ C::swz(l16)) << 3) + ks * 32]));
      else return qv[qb][ks];
    };

    wait_loads<0>();
    int row = row_of(0);
    load_ids(1);
    load_tile(0, row);
    for (int t = 0; t < take; ++t) {
      const uint32_t there = (uint32_t)__builtin_amdgcn_ballot_w64(row >= 0);  // keys of tile t that exist
      if (t + 1 < take) {
        wait_loads<C::NDMA>();  // the ids of tile t + 1
        row = row_of(t + 1);
        load_ids(t + 2);
        load_tile(t + 1, row);
        wait_loads<C::NDMA + 1>();  // tile t
      } else {
        wait_loads<0>();
      }
      if (there == 0) continue;
      const int k0 = key0 + t * C::UNIT;
      const uint16_t* tile = tiles[wave][t & 1];
      const bool masked = there != 0xffffffffu || k0 < pb.all_b || k0 + 32 > pb.all_e;

      f32x4 s[QB][2];
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) s[qb][0] = s[qb][1] = f32x4{};
#pragma unroll
      for (int ks = 0; ks < C::KS; ++ks) {
        const bf16x8 k0v = as_bf16x8(*reinterpret_cast<const u32x4*>(&tile[k_at(0, ks)]));
        const bf16x8 k1v = as_bf16x8(*reinterpret_cast<const u32x4*>(&tile[k_at(1, ks)]));
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          const bf16x8 qk = q_at(qb, ks);
          s[qb][0] = mfma16(k0v, qk, s[qb][0]);
          s[qb][1] = mfma16(k1v, qk, s[qb][1]);
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
    }

    // ---- the waves' results, merged in wave order, 16 QP rows at a time ----
    float* res = reinterpret_cast<float*>(&tiles[wave][0][0]);  // [16 QP][RS]: this wave's own buffers
    const bool whole = take == pb.n_units;
    const int64_t slot = 2 * (int64_t)blockIdx.x + (u0 == 0);
#pragma unroll
    for (int q0 = 0; q0 < QB; q0 += C::QP) {
#pragma unroll
      for (int qp = 0; qp < C::QP; ++qp) {
        const int qb = q0 + qp;
        float l = l_run[qb];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (gq == 0) {
          red_m[wave][16 * qp + l16] = m_run[qb];
          red_l[wave][16 * qp + l16] = l;
        }
#pragma unroll
        for (int d = 0; d < C::DV; ++d)
          *reinterpret_cast<f32x4*>(&res[(16 * qp + l16) * C::RS + 16 * d + 4 * gq]) = o[qb][d];
      }
      __syncthreads();
      for (int i = threadIdx.x; i < 16 * C::QP * (DC / 4); i += NW * 64) {
        const int rr = i / (DC / 4), r = 16 * q0 + rr, c = i % (DC / 4) * 4;
        if (row0 + r >= n_rows) break;
        float m = kLowest, l = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) m = fmaxf(m, red_m[w][rr]);
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          const float f = fast_exp2(red_m[w][rr] - m);
          l += f * red_l[w][rr];
          v += f * *reinterpret_cast<const f32x4*>(
                       reinterpret_cast<const float*>(&tiles[w][0][0]) + rr * C::RS + c);
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
      __syncthreads();  // the buffers are free for the next rows or segment
    }
  }
}

// ---- merge and value up-projection -------------------------------------------------------------
// grid (ceil(n_tokens / TG), H), 256 threads: the latents of TG tokens of one head, merged where their
// row block was split, then out^T[v][token] = W_UV_h[v][:] . o_lat[token][:]. The latents go into the
// product as two bf16 terms (16 bits of fraction): one alone adds a rounding as large as the output's
// own, 2^-8 of the value, for a product that costs next to nothing here.
// TG = 1 (few tokens: single-token steps, whose rows are split the most): the splits are read by slices
// of the workgroup side by side, each with its own running maximum. More tokens: the coefficient of
// every (token, split) goes into a table, and a thread sums its chunks, four in flight per split.
constexpr int kOutSplits = 8;  // splits the table holds; tokens of more are merged one split after the other

template <int DC, int TG>
__global__ __launch_bounds__(256, DC <= 256 ? 3 : 2) void paged_out_kernel(const PagedAttendArgs a) {
  constexpr int LS = (DC > 32 ? DC : 32) + 8;  // LDS row stride (elements)
  constexpr int KS = (DC + 31) / 32;
  constexpr int C4 = DC / 4;                   // 16-byte chunks of a partial row
  constexpr int SL = TG > 1 ? 1 : 256 / C4 < 16 ? 256 / C4 : 16;  // slices of splits
  constexpr int NB = (TG + 15) / 16;           // blocks of 16 tokens
  __shared__ __attribute__((aligned(16))) uint16_t lat[2][TG][LS];  // o_lat's first and second term
  __shared__ f32x4 part[SL][C4];
  __shared__ float part_m[SL], part_l[SL];
  __shared__ float coef[TG > 1 ? TG : 1][kOutSplits];
  __shared__ int32_t tok_row[TG], tok_w0[TG], tok_ns[TG], most_s;  // (ns 0: no token of a sequence)
  const PagedGeo& g = a.pg;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int gq = lane >> 4, l16 = lane & 15;
  const int H = a.n_heads, h = blockIdx.y, t0 = blockIdx.x * TG;

  // the weights of the wave's first output blocks, on their way while the latents are merged
  const int n_vb = a.d_v / 16;
  auto weight = [&](int vb, int ks) {
    u32x4 x = {0, 0, 0, 0};
    if (ks * 32 + 8 * gq < DC) x = ldg16(a.w_uv + ((int64_t)h * a.d_v + vb * 16 + l16) * DC + ks * 32 + 8 * gq);
    return as_bf16x8(x);
  };
  constexpr int AHEAD = DC > 256 ? 1 : 2;
  bf16x8 wv[AHEAD][KS];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) wv[i][ks] = weight(min(wave * AHEAD + i, n_vb - 1), ks);

  // partial row of split k of a token (its first partial has the first key: slot 2 w + 1)
  auto part_row = [&](int w0, int k, int row) { return (2 * (int64_t)(w0 + k) + (k == 0)) * a.rows + row; };
  if (wave == 0) {
    const int t = t0 + min(lane, TG - 1);
    const int s0 = paged_seq_of_lanes(g, t), s = t < g.n_tokens ? s0 : -1;
    const int r = s >= 0 ? (t - max(g.cu[s], 0)) * H + h : 0;
    const int blk = s >= 0 ? a.plan.seq_block[s] + r / a.rows : 0;
    const bool known = s >= 0 && blk < a.plan.seq_block[g.n_seqs];  // (else offsets that go down)
    int ns = 0, w0 = 0;
    if (known) {
      const int64_t U = a.plan.head[0], G = a.plan.head[1];
      w0 = (int)floor_div((a.plan.first[blk] + a.cost + 1) * G - 1, U);
      ns = (int)floor_div(a.plan.first[blk + 1] * G - 1, U) - w0 + 1;
    }
    int most = ns;
    if constexpr (TG > 1) {
      const int row = r % a.rows;
      if (ns > 1 && ns <= kOutSplits) {
        f32x2 ml[kOutSplits];
#pragma unroll
        for (int k = 0; k < kOutSplits; ++k)
          ml[k] = *reinterpret_cast<const f32x2*>(a.ml_part + part_row(w0, min(k, ns - 1), row) * 2);
        float m = kLowest, l = 0.f;
#pragma unroll
        for (int k = 0; k < kOutSplits; ++k) m = fmaxf(m, ml[k][0]);
#pragma unroll
        for (int k = 0; k < kOutSplits; ++k) l += k < ns ? fast_exp2(ml[k][0] - m) * ml[k][1] : 0.f;
        const float il = l == 0.f ? 0.f : 1.f / l;  // (a row that sees nothing: zeros)
        if (lane < TG)
#pragma unroll
          for (int k = 0; k < kOutSplits; ++k) coef[lane][k] = k < ns ? fast_exp2(ml[k][0] - m) * il : 0.f;
      } else if (lane < TG) {
#pragma unroll
        for (int k = 0; k < kOutSplits; ++k) coef[lane][k] = k == 0 ? 1.f : 0.f;
      }
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) most = max(most, __shfl_xor(most, d));
    }
    if (lane < TG) {
      tok_ns[lane] = ns;
      tok_row[lane] = r % a.rows;
      tok_w0[lane] = w0;
    }
    if (lane == 0) most_s = most;
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
  // the online merge of chunk c of token t's partial results k0, k0 + SL, ..
  auto merge = [&](int t, int c, int k0, float& m, float& l, f32x4& v) {
    const int ns = tok_ns[t], w0 = tok_w0[t];
    m = kLowest;
    l = 0.f;
    v = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int k = k0; k < ns; k += 4 * SL) {
      f32x2 ml[4];
      f32x4 x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int kk = k + j * SL < ns ? k + j * SL : k;  // (past the last: read again, weighed by zero)
        const int64_t row = part_row(w0, kk, tok_row[t]);
        ml[j] = *reinterpret_cast<const f32x2*>(a.ml_part + row * 2);
        x[j] = *reinterpret_cast<const f32x4*>(a.o_part + row * DC + c * 4);
      }
      float m1 = m;
#pragma unroll
      for (int j = 0; j < 4; ++j) m1 = fmaxf(m1, ml[j][0]);
      const float f = fast_exp2(m - m1);
      l *= f;
      v *= f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (k + j * SL < ns) {
          const float fj = fast_exp2(ml[j][0] - m1);
          l += fj * ml[j][1];
          v += fj * x[j];
        }
      }
      m = m1;
    }
  };
  const int most = most_s;
  if constexpr (TG == 1) {
    if (most == 0) return;
    if (most == 1) {
      if (tid < C4) put(0, tid, *reinterpret_cast<const f32x4*>(a.o_lat + ((int64_t)t0 * H + h) * DC + tid * 4));
    } else {
      const int slice = tid / C4, c = tid % C4;
      if (slice < SL) {
        float m, l;
        f32x4 v;
        merge(0, c, slice, m, l, v);
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
        put(0, tid, v * (l == 0.f ? 0.f : 1.f / l));
      }
    }
  } else {
    // chunk e = (token, 4 columns); a token of no sequence reads row 0 and is not stored
    constexpr int N = (TG * C4 + 255) / 256, IN = N < 4 ? N : 4;
    auto source = [&](int e, int k) {
      const int t = min(e / C4, TG - 1), ns = tok_ns[t];
      const float* p = ns <= 1 ? a.o_lat + ((int64_t)(ns == 0 ? 0 : t0 + t) * H + h) * DC
                               : a.o_part + part_row(tok_w0[t], min(k, ns - 1), tok_row[t]) * DC;
      return reinterpret_cast<const f32x4*>(p + e % C4 * 4);
    };
#pragma unroll 1
    for (int i0 = 0; i0 < N; i0 += IN) {
      f32x4 v[IN];
#pragma unroll
      for (int i = 0; i < IN; ++i) v[i] = *source(tid + 256 * (i0 + i), 0);
      if (most > 1) {
#pragma unroll
        for (int i = 0; i < IN; ++i) v[i] *= coef[min((tid + 256 * (i0 + i)) / C4, TG - 1)][0];
        for (int k = 1; k < min(most, kOutSplits); ++k) {
          f32x4 x[IN];
#pragma unroll
          for (int i = 0; i < IN; ++i) x[i] = *source(tid + 256 * (i0 + i), k);
#pragma unroll
          for (int i = 0; i < IN; ++i) {
            const float f = coef[min((tid + 256 * (i0 + i)) / C4, TG - 1)][k];
            if (f != 0.f) v[i] += f * x[i];
          }
        }
      }
#pragma unroll
      for (int i = 0; i < IN; ++i) {
        const int e = tid + 256 * (i0 + i), t = e / C4;
        if (e >= TG * C4) continue;
        if (tok_ns[t] > kOutSplits) {
          float m, l;
          merge(t, e % C4, 0, m, l, v[i]);
          v[i] *= l == 0.f ? 0.f : 1.f / l;
        }
        put(t, e % C4, v[i]);
      }
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
#pragma unroll 1
    for (int nb = 0; nb < NB; ++nb) {
      const int t = min(16 * nb + l16, TG - 1);
      f32x4 acc[AHEAD] = {};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const bf16x8 b = as_bf16x8(*reinterpret_cast<const u32x4*>(&lat[k][t][ks * 32 + 8 * gq]));
#pragma unroll
          for (int i = 0; i < AHEAD; ++i) acc[i] = mfma16(wv[i][ks], b, acc[i]);
        }
      if (16 * nb + l16 < TG && tok_ns[t] > 0) {
        uint16_t* dst = a.out + ((int64_t)(t0 + t) * H + h) * a.d_v + vb * 16 + 4 * gq;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
          if (vb + i < n_vb) *reinterpret_cast<bf16x4*>(dst + i * 16) = to_bf16x4(acc[i]);
      }
    }
  }
}

#define VMLA_PAGED_SHAPES(X) X(16, 8) X(64, 32) X(128, 32) X(192, 32) X(256, 32) X(512, 32)

}  // namespace

namespace {
// 16-row blocks per workgroup of the few-row kernel: the most whose accumulators leave the registers room
constexpr int few_most(int dc) { return dc <= 128 ? 4 : dc <= 192 ? 3 : 1; }
}  // namespace

void paged_attend_shape(int d_c, int d_rope, int64_t max_rows, int32_t* rows, int32_t* unit, int32_t* cost) {
  const int wide = paged_wide_rows(d_c, d_rope), most = 16 * few_most(d_c);
  if (wide > 0 && max_rows > most) {
    *rows = wide;
    *unit = 32;
    *cost = 8;
    return;
  }
  *rows = max_rows <= 16 || most == 16 ? 16 : max_rows <= 32 ? 32 : most;
  *unit = 32 * few_waves(d_c);
  *cost = 1;
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
    if (a.rows == 32) return go(paged_attend_few_kernel<DC, DR, (few_most(DC) > 1 ? 2 : 1)>);         \
    return go(paged_attend_few_kernel<DC, DR, few_most(DC)>);                                         \
  }
  VMLA_PAGED_SHAPES(X)
#undef X
  return hipErrorInvalidValue;
}

hipError_t launch_paged_out(const PagedAttendArgs& a, hipStream_t s) {
  const int n = a.pg.n_tokens;
  auto go = [&](auto kernel, int tg) {
    hipLaunchKernelGGL(kernel, dim3((n + tg - 1) / tg, a.n_heads), dim3(256), 0, s, a);
    return hipGetLastError();
  };
#define X(DC, DR)                                                       \
  if (a.d_c == DC && a.d_rope == DR) {                                  \
    if (n <= 128) return go(paged_out_kernel<DC, 1>, 1);                \
    if (n <= 1024 || DC > 256) return go(paged_out_kernel<DC, 16>, 16); \
    return go(paged_out_kernel<DC, (DC > 256 ? 16 : 64)>, 64);            \
  }
  VMLA_PAGED_SHAPES(X)
#undef X
  return hipErrorInvalidValue;
}

}  // namespace vmla
