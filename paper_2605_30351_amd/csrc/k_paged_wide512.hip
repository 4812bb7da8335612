// Paged attention at d_c = 512 for more than 16 rows per sequence.
//
// 64 rows x 512 fp32 latents are 128 registers a lane of four waves, a wave per SIMD. A workgroup takes 64
// rows and its waves split each step two ways (16x16x32 MFMA throughout):
//   scores  wave w: rows 32 (w / 2) .. +31 against keys 16 (w % 2) .. +15 of the tile, so that each K row
//           is read from LDS by two waves, not four;
//   PV      wave w: all 64 rows, columns 128 w .. +127, so that each V column is read once. The
//           probabilities pass between the waves through LDS.
// Three tile buffers: step t takes the scores and probabilities of tile t + 1, PV of tile t and the loads
// of tile t + 2, with one barrier. Probabilities are taken under the running maximum of before, which they
// may exceed by up to 2^8; a tile that exceeds it by more (seen by any wave) makes all waves, after the
// barrier, agree on the new maxima, take the probabilities again and rescale.
// Per tile and workgroup: 66 MFMAs a wave (1,056 cycles) over 68 KB of K and 32 KB of V reads (780 cycles at
// 128 bytes a cycle).
//
// Queries are one bf16 term (outputs off by 0.0026 in the 2-norm at scores of standard deviation 1) while that is
// enough, by the rule of kOneTerm and kSpread. A workgroup's part of a block that needs the second (one alone:
// 0.0042 at 4, two 0.0018) takes its 64 rows in two passes of 32, whose second terms fit LDS beside the tiles: a
// wave then has 16 rows for the scores, and 50 MFMAs a tile and pass.
#include <type_traits>

#include "vmla_paged.h"

namespace vmla {
namespace {

constexpr int kDC = 512, kDR = 32, kRows = 64, kWaves = 4;
constexpr int kKS = (kDC + kDR) / 32;               // 32-wide k-steps
constexpr int kTile = 32 * (kDC + kDR);             // elements: c_kv rows of 1 KB, then k_r rows of 64 bytes
constexpr int kPS = 40;                             // row stride of the probabilities (elements)

// Chunk position of chunk c in row r: c_kv rows start on the same banks, so the XOR separates all 16 rows
// of an operand read and the pairs of chunks of a transpose read; k_r rows by fours.
__device__ constexpr int swz16(int r) { return ((r << 1) & 15) | ((r >> 3) & 1); }
__device__ constexpr int swz4(int r) { return (((r >> 2) & 1) << 1) | ((r >> 3) & 1); }

__global__ __launch_bounds__(64 * kWaves, 1) void paged_attend_wide512_kernel(const PagedAttendArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t tile[3][kTile];
  __shared__ __attribute__((aligned(16))) uint16_t probs[2][kRows * kPS];
  __shared__ float tile_max[2][kRows];  // per key half
  __shared__ float factor[kRows], sums[2][kRows];
  __shared__ __attribute__((aligned(16))) uint16_t q_lo[2][kKS][64 * 8];  // second terms, by row group and lane
  __shared__ int grown[3];
  __shared__ int two_terms;     // the segment is to be taken with two terms: by its rows, or its first tile's scores
  __shared__ int far[2];        // its later scores are far apart (segments in turn)
  __shared__ uint32_t cleared;  // keys of the tile in work, between settle()'s barriers

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rg = wave >> 1, kh = wave & 1;  // score rows of half rg and keys 16 kh ..
  const PagedGeo& pg = a.pg;
  const int H = a.n_heads;
  const PagedWork wk = paged_read<true>(a.plan.work, blockIdx.x);
  int left = wk.n, blk = wk.block, end = wk.end;
  if (threadIdx.x == 0) cleared = 0;

  // (see k_paged_wide.hip: a part whose later scores were too far apart for one term is taken again)
  bool again = false, one_term = false;
  int left0 = 0, blk0 = 0, end0 = 0, turn = 0;
  for (;;) {
    __syncthreads();  // the previous block's tiles and sums are no longer read
    again = one_term && __builtin_amdgcn_readfirstlane(far[turn]) != 0;
    if (again) {
      left = left0;
      blk = blk0;
      end = end0;
    }
    one_term = false;
    if (left <= 0) break;
    left0 = left;
    blk0 = blk;
    end0 = end;
    const bool last = blk == wk.block;
    const PagedBlock pb = last ? paged_read<true>(a.plan.work_block, blockIdx.x) : paged_read<true>(a.plan.block, blk);
    if (end < 0) end = pb.n_units + a.cost;  // a block before the workgroup's last is taken to its end
    const int len = min(left, end), u1 = end - a.cost, u0 = max(u1 - len, 0), n_tiles = u1 - u0;
    left -= len;
    end = -1;
    --blk;
    if (n_tiles <= 0) continue;
    const int row0 = pb.row0, n_rows = pb.n_rows, key0 = pb.key0 + u0 * 32;
    const int32_t* table = pg.table + (int64_t)pb.seq * pg.max_pages;
    turn ^= 1;
    if (threadIdx.x == 0) two_terms = far[turn] = 0;

    // One pass over the segment's keys: of all 64 rows with one term, or with both of the rows from 32 sub on. False,
    // with nothing done, if the rows or the first tile's scores ask for both.
    auto pass = [&](auto with_both, int sub) __attribute__((always_inline)) -> bool {
      constexpr bool BOTH = decltype(with_both)::value;
      constexpr int RB = BOTH ? 1 : 2;  // 16-row blocks a wave has for the scores
      // (from the lane computed here: kept for both kinds of pass, the bases would fill the register file)
      const int lane = lane_here(), gq = lane >> 4, l16 = lane & 15, l32 = lane & 31;
      // K operand of k-step ks: row 16 kh + l16, chunk 4 ks + gq; V^T: rows 4 gq + l16 / 4 (+ 16), columns
      // 128 wave + 16 d + 4 (l16 % 4); a few bases reach every step with immediate offsets
      int k_base[5], v_base[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) k_base[i] = (16 * kh + l16) * kDC + (((4 * i + gq) ^ swz16(l16)) << 3);
      k_base[4] = 32 * kDC + (16 * kh + l16) * kDR + ((gq ^ swz4(l16)) << 3);
      const int v_row = 4 * gq + (l16 >> 2), v_ch = (l16 >> 1) & 1;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        v_base[i] = v_row * kDC + 128 * wave + (((2 * i + v_ch) ^ swz16(v_row)) << 3) + (l16 & 1) * 4;

      auto load_id = [&](int t) { return table[page_of(pg, min(key0 + t * 32 + l32, pg.max_kv - 1))]; };
      const int key_end = min(key0 + n_tiles * 32, pb.kv);
      auto row_of = [&](int t, int32_t page) {  // this lane's key's pool row, -1: none, or past the segment
        const int key = key0 + t * 32 + l32;
        const int row = page * pg.page_tokens + key - page_of(pg, key) * pg.page_tokens;
        return key < key_end && (uint32_t)page < (uint32_t)pg.n_pages ? row : -1;
      };
      // wave w loads the c_kv rows 8 w .. +7, each from a scalar base, and waves 0 and 1 sixteen k_r rows each
      auto load_row = [&](int row, uint16_t* buf, int j) {
        const uint32_t r = __builtin_amdgcn_readlane(max(row, 0), 8 * wave + j);  // (a missing key: the first row)
        const int sw = 8 * (wave & 1) + j;                                          // (the row modulo 16)
        int ln = lane;
        asm volatile("" : "+v"(ln));  // the offset is recomputed: eight of them kept across the loop would spill
        lds_dma16_row(a.c_kv + (uint64_t)r * kDC, (ln ^ (((sw << 1) & 15) | (sw >> 3))) * 16,
                      __builtin_amdgcn_readfirstlane(lds_addr(buf)) + 1024u * (8 * wave + j));
      };
      auto load_k_r = [&](int row, uint16_t* buf) {
        const int rr = lane >> 2;
        const uint32_t r = __shfl(max(row, 0), 16 * (wave & 1) + rr);
        if (wave < 2)
          lds_dma16(a.k_r + (uint64_t)r * kDR + ((lane & 3) ^ swz4(rr)) * 8,
                    __builtin_amdgcn_readfirstlane(lds_addr(buf)) + 1024u * (32 + wave));
      };
      auto load_tile = [&](int row, uint16_t* buf) {
#pragma unroll
        for (int j = 0; j < 8; ++j) load_row(row, buf, j);
        load_k_r(row, buf);
      };
      auto exist = [](int row) { return (uint32_t)__builtin_amdgcn_ballot_w64(row >= 0); };

      const int own = 16 * RB * rg + l16;  // this lane's first row in the pass
      const int32_t id0 = load_id(0), id1 = load_id(1);
      int32_t id = load_id(2);
      int row = row_of(0, id0);
      uint32_t there = exist(row), there_n;
      load_tile(row, tile[0]);
      row = row_of(1, id1);
      there_n = exist(row);
      load_tile(row, tile[1]);

      bf16x8 q[RB][kKS];
      int see_b[RB], see_e[RB];
      float q2 = 0.f;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const int rr = 32 * sub + own + 16 * rb, r = row0 + rr;
        const int64_t at = ((int64_t)pb.lo * H + (r < n_rows ? r : row0)) * (kDC + kDR) + 8 * gq;
        float len = 0.f;
#pragma unroll
        for (int ks = 0; ks < kKS; ++ks) {
          u32x4 v = ldg16(a.qcat + at + ks * 32);
          if (r >= n_rows) v = u32x4{0, 0, 0, 0};
          q[rb][ks] = as_bf16x8(v);
        }
        if constexpr (BOTH) {  // (the two waves of a row group share its second terms)
#pragma unroll
          for (int ks = 0; ks < kKS; ++ks) {
            if ((ks & 1) != kh) continue;
            const u32x2 low = *reinterpret_cast<const u32x2*>(a.q_low + at + ks * 32);
            *reinterpret_cast<bf16x8*>(&q_lo[rg][ks][lane * 8]) =
                second_term(q[rb][ks], r < n_rows ? low : u32x2{0, 0});
          }
        } else {
#pragma unroll
          for (int ks = 0; ks < kKS; ++ks) len = add_squares(q[rb][ks], len);
          len += __shfl_xor(len, 16);
          q2 = fmaxf(q2, half_swap_sum(len));
        }
        paged_row_sees(pg, pb, H, min(rr, n_rows - 1 - row0), see_b[rb], see_e[rb]);  // (past the end: as the last)
      }
      f32x4 o[2 * RB][8];  // rows 16 rb .. of the pass, columns 128 wave + 16 d ..
      float m_run[RB], l_run[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        m_run[rb] = kLowest;
        l_run[rb] = 0.f;
      }
#pragma unroll
      for (int rb = 0; rb < 2 * RB; ++rb)
#pragma unroll
        for (int d = 0; d < 8; ++d) o[rb][d] = f32x4{};

      // the latents of tile t in buf, made finite if a key is missing or some row of the block does not see one
      // A row that sees a latent that was not finite gets a NaN sum.
      auto settle = [&](int t, uint32_t keys, uint16_t* buf) {
        const int k0 = key0 + t * 32;
        if (keys == 0xffffffffu && k0 >= pb.all_b && k0 + 32 <= pb.all_e) return;
        for (int i = threadIdx.x; i < 32 * kDC / 8; i += 64 * kWaves)
          clear_not_finite(buf + i * 8, &cleared, [&] { return 1u << (i / (kDC / 8)); });
        const uint32_t bad = cleared_keys(&cleared);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          l_run[rb] = seen_keys(keys, see_b[rb] - k0, see_e[rb] - k0) & bad ? kNotANumber : l_run[rb];
      };
      // S^T of this wave's rows and keys: two chains of matrix steps per row block, so that few wait for the
      // last, K read three steps ahead, and between(ks) after each step: the loads of a later tile go out there
      auto scores = [&](const uint16_t* buf, f32x4 (&s)[RB], auto between) {
        f32x4 odd[RB];
        [[maybe_unused]] f32x4 lo = {};
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) s[rb] = odd[rb] = f32x4{};
        bf16x8 k[4];
        auto read = [&](int ks) {
          const int at = ks < kDC / 32 ? k_base[ks & 3] + (ks >> 2) * 128 : k_base[4];
          k[ks & 3] = as_bf16x8(*reinterpret_cast<const u32x4*>(&buf[at]));
        };
#pragma unroll
        for (int ks = 0; ks < 3; ++ks) read(ks);
#pragma unroll
        for (int ks = 0; ks < kKS; ++ks) {
          if (ks + 3 < kKS) read(ks + 3);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) {
            if (ks & 1) odd[rb] = mfma16(k[ks & 3], q[rb][ks], odd[rb]);
            else s[rb] = mfma16(k[ks & 3], q[rb][ks], s[rb]);
          }
          if constexpr (BOTH)
            lo = mfma16(k[ks & 3], as_bf16x8(*reinterpret_cast<const u32x4*>(&q_lo[rg][ks][lane * 8])), lo);
          between(ks);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) s[rb] += odd[rb];
        if constexpr (BOTH) {
          const float most = most_here();
#pragma unroll
          for (int i = 0; i < 4; ++i) s[0][i] += second_part(lo[i], most);
        }
      };
      auto mask = [&](int t, uint32_t keys, f32x4 (&s)[RB]) {
        const int k0 = key0 + t * 32;
        if (keys != 0xffffffffu || k0 < pb.all_b || k0 + 32 > pb.all_e) {
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) {
            const uint32_t seen = seen_keys(keys, see_b[rb] - k0, see_e[rb] - k0) >> (16 * kh + 4 * gq);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[rb][i] = seen >> i & 1 ? s[rb][i] : kMasked;
          }
        }
      };
      // the probabilities of tile t's keys of this wave under m_run, into LDS, and their sums
      auto probabilities = [&](int t, const f32x4 (&s)[RB], float (&l)[RB]) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          const f32x2 e0 = {fast_exp2(s[rb][0] - m_run[rb]), fast_exp2(s[rb][1] - m_run[rb])};
          const f32x2 e1 = {fast_exp2(s[rb][2] - m_run[rb]), fast_exp2(s[rb][3] - m_run[rb])};
          const bf16x2 h0 = __builtin_convertvector(e0, bf16x2), h1 = __builtin_convertvector(e1, bf16x2);
          l[rb] = __builtin_amdgcn_fdot2_f32_bf16(h0, kOnesBf16x2, 0.f, false);
          l[rb] = __builtin_amdgcn_fdot2_f32_bf16(h1, kOnesBf16x2, l[rb], false);
          *reinterpret_cast<u32x2*>(&probs[t & 1][(own + 16 * rb) * kPS + 8 * gq + 4 * kh]) =
              u32x2{__builtin_bit_cast(uint32_t, h0), __builtin_bit_cast(uint32_t, h1)};
        }
      };
      auto max_of = [](const f32x4& v) { return fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])); };
      // whether some row's scores (masked) are further apart than kSpread: of four differences a lane, of keys 8 apart,
      // two, so that a single key that stands out does not count
      auto apart = [&](const f32x4 (&s)[RB]) {
        bool is = false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          f32x4 d;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t bits = __float_as_uint(s[rb][i]);
            const auto pair = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
            const float v = fabsf(__uint_as_float(pair[0]) - __uint_as_float(pair[1]));
            d[i] = v < -kMasked ? v : 0.f;  // (a hidden key's is infinite, or NaN)
          }
          is |= fminf(fmaxf(d[0], d[1]), fmaxf(d[2], d[3])) > kSpread;
        }
        return __builtin_amdgcn_ballot_w64(is) != 0;
      };
      // whether some score of tile t exceeds its row's m_run by more than kLazyMaxStep
      auto watch = [&](int t, const f32x4 (&s)[RB]) {
        bool grow = false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) grow |= max_of(s[rb]) > m_run[rb] + kLazyMaxStep;
        if (__builtin_amdgcn_ballot_w64(grow) != 0 && lane == 0) grown[t % 3] = 1;
      };
      // after a barrier: agree on tile t's maxima where some wave saw growth; the probabilities are taken again
      auto agree = [&](int t, const f32x4 (&s)[RB], float (&l)[RB]) {
        if (grown[t % 3] == 0) return;
        if (!BOTH && t > 0 && apart(s)) far[turn] = 1;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          float m = max_of(s[rb]);
          m = fmaxf(m, __shfl_xor(m, 16));
          m = fmaxf(m, __shfl_xor(m, 32));
          if (gq == 0) tile_max[kh][own + 16 * rb] = m;
        }
        __syncthreads();
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          const int r = own + 16 * rb;
          const float m = fmaxf(m_run[rb], fmaxf(tile_max[0][r], tile_max[1][r]));
          const float f = fast_exp2(m_run[rb] - m);
          m_run[rb] = m;
          l_run[rb] *= f;
          if (kh == 0 && gq == 0) factor[r] = f;
        }
        probabilities(t, s, l);
        __syncthreads();
#pragma unroll
        for (int rb = 0; rb < 2 * RB; ++rb) {
          const float f = factor[16 * rb + l16];
#pragma unroll
          for (int d = 0; d < 8; ++d) o[rb][d] *= f;
        }
      };

      f32x4 s[RB];
      float l_new[RB];
      if (threadIdx.x < 3) grown[threadIdx.x] = 0;
      wait_vmcnt<0>();
      __syncthreads();
      scores(tile[0], s, [](int) {});
      mask(0, there, s);
      if (!BOTH && (__builtin_amdgcn_ballot_w64(q2 > kOneTerm * kOneTerm) != 0 || apart(s))) two_terms = 1;
      watch(0, s);
      probabilities(0, s, l_new);
      __syncthreads();
      if (!BOTH && __builtin_amdgcn_readfirstlane(two_terms) != 0) return false;
      settle(0, there, tile[0]);
      agree(0, s, l_new);
      for (int t = 0; t < n_tiles; ++t) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) l_run[rb] += l_new[rb];
        const uint16_t* cur = tile[t % 3];
        uint16_t* nxt = tile[(t + 1) % 3];
        if (threadIdx.x == 0) grown[(t + 2) % 3] = 0;  // last read before the previous barrier
        uint16_t* stg = tile[(t + 2) % 3];
        row = row_of(t + 2, id);
        scores(nxt, s, [&](int ks) {
          if (ks >= 1 && ks <= 8) load_row(row, stg, ks - 1);
          if (ks == 9) load_k_r(row, stg);
          if (ks == 10) id = load_id(t + 3);
        });
        bf16x8 p[2 * RB];
#pragma unroll
        for (int rb = 0; rb < 2 * RB; ++rb)
          p[rb] = as_bf16x8(*reinterpret_cast<const u32x4*>(&probs[t & 1][(16 * rb + l16) * kPS + 8 * gq]));
        bf16x8 v[3];
        auto vread = [&](int d) {
          v[d % 3] = join_bf16x8(lds_read_tr(cur + v_base[d]), lds_read_tr(cur + v_base[d] + 16 * kDC));
        };
        vread(0);
        vread(1);
#pragma unroll
        for (int d = 0; d < 8; ++d) {
          if (d + 2 < 8) vread(d + 2);
#pragma unroll
          for (int rb = 0; rb < 2 * RB; ++rb) o[rb][d] = mfma16(v[d % 3], p[rb], o[rb][d]);
        }
        const uint32_t keys = there_n;
        mask(t + 1, keys, s);
        watch(t + 1, s);
        probabilities(t + 1, s, l_new);
        there_n = exist(row);
        wait_vmcnt<0>();  // this wave's part of tile t + 2 is in LDS
        __syncthreads();
        settle(t + 1, keys, nxt);
        agree(t + 1, s, l_new);
      }

      // ---- a whole block's latents, or this segment's partial result ----
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        float l = l_run[rb];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (gq == 0) sums[kh][own + 16 * rb] = l;
      }
      __syncthreads();
      const bool whole = n_tiles == pb.n_units;
      const int64_t slot_row = (2 * (int64_t)blockIdx.x + (u0 == 0)) * kRows;
#pragma unroll
      for (int rb = 0; rb < 2 * RB; ++rb) {
        const int lr = 16 * rb + l16, rr = 32 * sub + lr, r = row0 + rr;
        if (r >= n_rows) continue;
        const float l = sums[0][lr] + sums[1][lr];
        const float f = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;  // (a row that sees nothing: zeros)
        float* dst = (whole ? a.o_lat + ((int64_t)pb.lo * H + r) * kDC : a.o_part + (slot_row + rr) * kDC) + 128 * wave;
#pragma unroll
        for (int d = 0; d < 8; ++d) *reinterpret_cast<f32x4*>(dst + 16 * d + 4 * gq) = o[rb][d] * f;
      }
      if (kh == 0 && gq == 0) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          const int lr = own + 16 * rb, rr = 32 * sub + lr, r = row0 + rr;
          if (r >= n_rows) continue;
          if (u0 == 0)
            a.plan.row[(int64_t)pb.lo * H + r] =
                PagedRow{(int32_t)blockIdx.x, (uint16_t)(last ? wk.last_ns : 1), (uint16_t)rr};
          if (!whole) {
            a.ml_part[(slot_row + rr) * 2] = m_run[rb];
            a.ml_part[(slot_row + rr) * 2 + 1] = sums[0][lr] + sums[1][lr];
          }
        }
      }
      return true;
    };

    one_term = !again && pass(std::false_type{}, 0);
    if (!one_term) {
      for (int sub = 0; sub < 2 && row0 + 32 * sub < n_rows; ++sub) {
        __syncthreads();  // the previous pass's tiles and sums are no longer read
        pass(std::true_type{}, sub);
      }
    }
  }
}

}  // namespace

hipError_t launch_paged_attend_wide512(const PagedAttendArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(paged_attend_wide512_kernel, dim3(a.n_wg), dim3(64 * kWaves), 0, s, a);
  return hipGetLastError();
}

}  // namespace vmla
