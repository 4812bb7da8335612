// Paged attention of many rows per sequence (chunks and prompts): the pipeline of latent_attend
// (k_attend.hip) over pages and under a mask.
//
// NW waves x 32 rows share each staged tile of 32 keys [c_kv | k_r | pad]. Three tile buffers: iteration
// t computes the scores of tile t + 1 while the exponentials of tile t run on the VALU, accumulates
// PV of tile t, and stages tile t + 2 with direct global-to-LDS loads. Every wave looks up the pages of
// the 32 keys itself, a lane a key, one tile before it stages it, so that the lookup's latency passes
// under a whole iteration; the rows of its own loads come from the other lanes.
// S^T = MFMA(A = K tile rows from LDS, B = q_cat rows in registers), so that a lane holds one row's
// scores of 16 keys and its mask is two comparisons with what that row sees, taken only in tiles that
// cross a row's limits, a hole or the sequence's end. In tiles that cross the limits of the block's rows
// the workgroup also clears infinities and NaN from the latents between the tile's scores and its PV: a
// key hidden from a row has probability 0 there, and 0 * NaN would reach it. The same holds for missing
// keys (holes, keys past the end), in whose place the pool's first row is staged.
//
// Queries are multiplied as one bf16 term (14 of the 26 matrix steps of a tile at d_c = 192) while scores are small:
// the rounding moves a score by about 2^-9.5 of its size, and so the output by 0.0016 in the 2-norm at scores of
// standard deviation 1, beside 0.0017 of the output's own rounding, and in proportion beyond. A workgroup's part
// of a block that needs it (kOneTerm, kSpread) is multiplied with both terms, the second from LDS before the first:
// a tile takes about 1.5 times as long. Looking for it costs 1% at most: it is done in the first tile and where a
// running maximum is raised (a look at every tile cost 4 to 10%).
#include <type_traits>

#include "vmla_paged.h"

namespace vmla {
namespace {

template <int DC, int DR, int NW>
struct WideCfg {
  static constexpr int DQKP = (DC + DR + 15) / 16 * 16;
  static constexpr int KS = DQKP / 16;
  static constexpr int DVB = (DC + 31) / 32;
  static constexpr int CPR = DQKP / 8;          // 16-byte chunks per tile row
  static constexpr int TILE = 32 * DQKP;        // elements
  static constexpr int NDMA = 32 * CPR / 64;    // 1 KB loads per tile
  static constexpr int PER_WAVE = (NDMA + NW - 1) / NW;
  static constexpr int ROWS = 32 * NW;
  // Eight accumulator blocks (d_c = 256, one wave per SIMD) live in accumulation registers: they are
  // rescaled (rarely) through LDS, since a VALU use would move all of them in every step.
  static constexpr bool RESC_LDS = DVB >= 8;
  // chunk position of chunk c in row r: the 16-row operand reads and the 4-row transpose reads hit 16
  // distinct 4-bank groups
  __device__ static constexpr int pos(int r, int c) { return (c & ~3) | ((c ^ (r >> 2)) & 3); }
  __device__ static constexpr int at(int r, int c) { return r * DQKP + pos(r, c >> 3) * 8 + (c & 7); }
  static_assert(DQKP % 32 == 0 && 32 * CPR % 64 == 0 && DVB * 32 <= DQKP, "tile shape");
};

template <int DC, int DR, int NW>
__global__ __launch_bounds__(NW * 64, 1) void paged_attend_wide_kernel(const PagedAttendArgs a) {
  using C = WideCfg<DC, DR, NW>;
  __shared__ __attribute__((aligned(16))) uint16_t tile[3][C::TILE];
  __shared__ __attribute__((aligned(16))) uint16_t q_lo[NW][C::KS][64 * 8];  // each wave's second term, by lane
  __shared__ uint32_t cleared;  // keys of the tile in work, between settle()'s barriers
  __shared__ int two_terms;     // the segment is to be taken with two terms: by its rows, or its first tile's scores
  __shared__ int far[2];        // its later scores are far apart (segments in turn)
  __shared__ __attribute__((aligned(16))) float resc[C::RESC_LDS ? NW : 1][C::RESC_LDS ? 64 * 16 : 4];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 5, l32 = lane & 31;
  const PagedGeo& pg = a.pg;
  const int H = a.n_heads;
  const PagedWork wk = paged_read<true>(a.plan.work, blockIdx.x);
  int left = wk.n, blk = wk.block, end = wk.end;
  if (threadIdx.x == 0) cleared = 0;

  // this wave's loads j = wave + NW i of a tile: where this lane's chunk is in pool row 0 of c_kv, or of k_r, or
  // (the pad, which has to be zero: times the zero in q_cat an infinity would be NaN) in the pad of q_cat's
  // first row; the tile row, and the bytes of a pool row
  const uint16_t* d_src[C::PER_WAVE];
  int d_row[C::PER_WAVE];
  bool d_kr[C::PER_WAVE], d_pad[C::PER_WAVE];
#pragma unroll
  for (int i = 0; i < C::PER_WAVE; ++i) {
    const int j = wave + NW * i, slot = (j < C::NDMA ? j : 0) * 64 + lane;
    const int r = slot / C::CPR, c = C::pos(r, slot % C::CPR);
    d_row[i] = r;
    d_kr[i] = c >= DC / 8;
    d_pad[i] = c >= (DC + DR) / 8;  // (never at most widths)
    d_src[i] = c < DC / 8 ? a.c_kv + c * 8 : d_pad[i] ? a.qcat + DC + DR : a.k_r + (c * 8 - DC);
  }
  // K operand of step ks: row l32, chunk 2 ks + g; V^T transpose reads: rows 4 g + tr_row (+ 8), columns
  // tr_col (+ 32 d, + 16 rows per half)
  const int hk = (l32 >> 2) & 3;
  const int koff_e = l32 * C::DQKP + ((g ^ hk) << 3);
  const int koff_o = l32 * C::DQKP + (((2 + g) ^ hk) << 3) - 16;
  const int tr_row = (lane & 15) >> 2, tr_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  const int vofs_lo = C::at(4 * g + tr_row, tr_col), vofs_hi = C::at(4 * g + tr_row + 8, tr_col);

  // A part whose later scores were too far apart for one term is taken again, with two: the waves agree on that at
  // the barrier that the next part begins with, so that its results, wrong then, are written without a wait.
  bool again = false, one_term = false;
  int left0 = 0, blk0 = 0, end0 = 0, turn = 0;
  for (;;) {
    __syncthreads();  // the previous segment's tiles are no longer read
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
    const bool last = blk == wk.block;  // (whose record the plan has copied: one load less in line)
    const PagedBlock pb = last ? paged_read<true>(a.plan.work_block, blockIdx.x) : paged_read<true>(a.plan.block, blk);
    if (end < 0) end = pb.n_units + a.cost;  // a block before the workgroup's last is taken to its end
    const int len = min(left, end), u1 = end - a.cost, u0 = max(u1 - len, 0), n_tiles = u1 - u0;
    left -= len;
    end = -1;
    --blk;
    if (n_tiles <= 0) continue;
    const int row0 = pb.row0 + wave * 32, n_rows = pb.n_rows;
    const int key0 = pb.key0 + u0 * 32;
    const int32_t* table = pg.table + (int64_t)pb.seq * pg.max_pages;
    turn ^= 1;
    if (threadIdx.x == 0) two_terms = far[turn] = 0;

    // page ids of tile t's keys, one per lane (a key outside the sequence reads the nearest entry)
    auto load_id = [&](int t) { return table[page_of(pg, min(key0 + t * 32 + l32, pg.max_kv - 1))]; };
    const int key_end = min(key0 + n_tiles * 32, pb.kv);
    auto row_of = [&](int t, int32_t page) {  // this lane's key's pool row, -1: none, or past the segment
      const int key = key0 + t * 32 + l32;
      const int row = page * pg.page_tokens + key - page_of(pg, key) * pg.page_tokens;
      return key < key_end && (uint32_t)page < (uint32_t)pg.n_pages ? row : -1;
    };
    uint32_t from[C::PER_WAVE];  // the pool rows of this lane's chunks (a missing key stages the first row)
    auto rows_for = [&](int row) {
#pragma unroll
      for (int i = 0; i < C::PER_WAVE; ++i) {
        from[i] = __shfl(max(row, 0), d_row[i]);
        if constexpr (C::DQKP > DC + DR) from[i] = d_pad[i] ? 0 : from[i];
      }
    };
    auto load_part = [&](int i, uint16_t* buf) {
      const int j = wave + NW * i;
      if (C::NDMA % NW == 0 || j < C::NDMA)
        lds_dma16(d_src[i] + (uint64_t)from[i] * (uint32_t)(d_kr[i] ? DR : DC),
                  __builtin_amdgcn_readfirstlane(lds_addr(buf) + 1024u * j));
    };
    auto load_tile = [&](int row, uint16_t* buf) {
      rows_for(row);
#pragma unroll
      for (int i = 0; i < C::PER_WAVE; ++i) load_part(i, buf);
    };
    auto exist = [](int row) { return (uint32_t)__builtin_amdgcn_ballot_w64(row >= 0); };

    const int32_t id0 = load_id(0), id1 = load_id(1);
    int32_t id = load_id(2);
    int row = row_of(0, id0);
    uint32_t there = exist(row), there_n;  // keys of the tile whose scores are computed next, and after
    load_tile(row, tile[0]);
    row = row_of(1, id1);
    there_n = exist(row);
    load_tile(row, tile[1]);

    // queries, B-operand layout: lane holds row l32, dims 16 ks + 8 g .. +8; and what that row sees
    bf16x8 q[C::KS];
    int see_b, see_e;
    const int r_own = row0 + l32;
    const bool live = r_own < n_rows;
    {
      const uint16_t* src = a.qcat + ((int64_t)pb.lo * H + (live ? r_own : 0)) * C::DQKP + 8 * g;
#pragma unroll
      for (int ks = 0; ks < C::KS; ++ks) {
        u32x4 v = ldg16(src + ks * 16);
        if (!live) v = u32x4{0, 0, 0, 0};
        q[ks] = as_bf16x8(v);
      }
      paged_row_sees(pg, pb, H, min(wave * 32 + l32, n_rows - 1 - pb.row0), see_b, see_e);  // (past the end: as the last)
    }
    // rows are in token order: the limits of the wave's first and last row hold for all
    const int b_max = __builtin_amdgcn_readlane(see_b, max(min(n_rows - 1 - row0, 31), 0));
    const int e_min = __builtin_amdgcn_readfirstlane(see_e);
    f32x16 o[C::DVB];
    float m_run = kLowest, l_run = 0.f, spoiled = 0.f, own_max;
#pragma unroll
    for (int d = 0; d < C::DVB; ++d) o[d] = f32x16{};

    // the latents of tile t in buf, made finite if some row of the block does not see one of its keys
    // (called by all waves, after every wave has used the tile's K and before any uses its V)
    // A row that sees a latent that was not finite is spoiled: its sum becomes NaN.
    auto settle = [&](int t, uint32_t keys, uint16_t* buf) {
      const int k0 = key0 + t * 32;
      if (keys == 0xffffffffu && k0 >= pb.all_b && k0 + 32 <= pb.all_e) return;
      for (int i0 = wave * 64; i0 < 32 * C::CPR; i0 += NW * 64) {
        const int i = i0 + lane_here();
        clear_not_finite(buf + i * 8, &cleared, [&] {
          const int r = i / C::CPR;
          return C::pos(r, i % C::CPR) < DC / 8 ? 1u << r : 0u;
        });
      }
      if (seen_keys(keys, see_b - k0, see_e - k0) & cleared_keys(&cleared)) spoiled = kNotANumber;
    };

    auto mask = [&](f32x16& s, uint32_t keys, int t) {
      const int k0 = key0 + t * 32;
      if (keys == 0xffffffffu && k0 >= b_max && k0 + 32 <= e_min) return;
      const uint32_t seen = seen_keys(keys, see_b - k0, see_e - k0) >> (4 * g);
      const float masked = __uint_as_float(bits_here<0xff800000u>());  // kMasked
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = seen >> (8 * (r >> 2) + (r & 3)) & 1 ? s[r] : masked;
    };
    // Whether some row's scores (masked) are further apart than kSpread. Of four differences a lane, of keys 1, 8, 10
    // and 16 apart, two have to be, so that a single key that stands out does not count.
    auto apart = [&](const f32x16& s) {
      f32x4 d = {fabsf(s[0] - s[1]), fabsf(s[2] - s[6]), fabsf(s[4] - s[12]), fabsf(s[9] - s[15])};
#pragma unroll
      for (int i = 0; i < 4; ++i) d[i] = d[i] < -kMasked ? d[i] : 0.f;  // (a hidden key's is infinite, or NaN)
      return __builtin_amdgcn_ballot_w64(fminf(fmaxf(d[0], d[1]), fmaxf(d[2], d[3])) > kSpread) != 0;
    };
    auto max_of = [&](const f32x16& v) {  // a tree of three-input maxima
      const float a0 = fmaxf(fmaxf(v[0], v[1]), v[2]), a1 = fmaxf(fmaxf(v[3], v[4]), v[5]);
      const float a2 = fmaxf(fmaxf(v[6], v[7]), v[8]), a3 = fmaxf(fmaxf(v[9], v[10]), v[11]);
      const float a4 = fmaxf(fmaxf(v[12], v[13]), v[14]);
      return fmaxf(fmaxf(fmaxf(a0, a1), a2), fmaxf(fmaxf(a3, a4), v[15]));
    };
    // each lane sees half of its row's keys; growth on either half sends the wave through the rare path
    auto raise_max = [&](const f32x16& s, auto both) {
      if (__builtin_amdgcn_ballot_w64(own_max > m_run + kLazyMaxStep) == 0) return;
      if (!decltype(both)::value && apart(s)) far[turn] = 1;
      const float m_new = fmaxf(m_run, half_swap_max(own_max));
      const float alpha = fast_exp2(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int d = 0; d < C::DVB; ++d) {
        if constexpr (C::RESC_LDS) {
          f32x16* slot = reinterpret_cast<f32x16*>(&resc[wave][lane * 16]);
          *slot = o[d];
          asm volatile("" ::: "memory");
          f32x16 tmp = *slot;
          tmp *= alpha;
          *slot = tmp;
          asm volatile("" ::: "memory");
          o[d] = *slot;
        } else {
          o[d] *= alpha;
        }
      }
    };

    float q2 = 0.f;  // the squared length of this lane's query
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) q2 = add_squares(q[ks], q2);
    const bool long_row = __builtin_amdgcn_ballot_w64(half_swap_sum(q2) > kOneTerm * kOneTerm) != 0;
    auto fetch_lo = [&]() {
      const int ln = lane_here(), r = row0 + (ln & 31);
      const uint8_t* src = a.q_low + ((int64_t)pb.lo * H + (r < n_rows ? r : 0)) * C::DQKP + 8 * (ln >> 5);
#pragma unroll
      for (int ks = 0; ks < C::KS; ++ks) {
        u32x2 v = *reinterpret_cast<const u32x2*>(src + ks * 16);
        if (r >= n_rows) v = u32x2{0, 0};
        *reinterpret_cast<bf16x8*>(&q_lo[wave][ks][ln * 8]) = second_term(q[ks], v);
      }
    };
    auto add_low = [&](const uint16_t* buf, f32x16& s) __attribute__((always_inline)) {
      const uint16_t* own = &q_lo[wave][0][lane_here() * 8];
#pragma unroll
      for (int ks = 0; ks < C::KS; ++ks) {
        s = mfma32(as_bf16x8(*reinterpret_cast<const u32x4*>(&buf[((ks & 1) ? koff_o : koff_e) + ks * 16])),
                   as_bf16x8(*reinterpret_cast<const u32x4*>(own + ks * 512)), s);
        if (ks & 1) __builtin_amdgcn_sched_barrier(0);  // (all reads at once would not fit the registers)
      }
      const float most = most_here();
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = second_part(s[r], most);
    };

    // One step: scores of tile t + 1 (QK), the exponentials of tile t (SM) and O += V^T P^T of tile t (PV)
    // as one fenced stream of slots, K reads two slots and V reads one slot ahead (see k_attend.hip).
    auto step = [&](int t, const f32x16& s_cur, f32x16& s_nxt, const uint16_t* cur, uint16_t* nxt,
                    uint16_t* stg, auto two_terms) __attribute__((always_inline)) {
      // the loads of tile t + 2 go out between the first matrix steps, so that these wait neither for the
      // exchange of its rows nor for the addresses
      row = row_of(t + 2, id);
      rows_for(row);
      constexpr int NS = C::KS, NPV = 2 * C::DVB;
      constexpr int NSLOT = NS > NPV + 2 ? NS : NPV + 2;
      constexpr int NSM = NS < 4 ? NS : 4;
      static_assert(C::PER_WAVE + 1 < NSLOT, "slots for the loads");
      auto kread = [&](int ks) {
        return as_bf16x8(*reinterpret_cast<const u32x4*>(&nxt[((ks & 1) ? koff_o : koff_e) + ks * 16]));
      };
      const lds_u16 *vlo = as_lds(cur) + vofs_lo, *vhi = as_lds(cur) + vofs_hi;
      auto vread = [&](int j) {
        const int kk = j / C::DVB, d = j % C::DVB;
        return join_bf16x8(lds_read_tr(vlo + kk * 16 * C::DQKP + d * 32),
                           lds_read_tr(vhi + kk * 16 * C::DQKP + d * 32));
      };
      uint32_t pk[8];
      auto sm_pair = [&](int p) {  // the sum is taken over the rounded probabilities, as PV uses them
        const f32x2 e = {fast_exp2(s_cur[2 * p] - m_run), fast_exp2(s_cur[2 * p + 1] - m_run)};
        const bf16x2 h = __builtin_convertvector(e, bf16x2);
        l_run = __builtin_amdgcn_fdot2_f32_bf16(h, kOnesBf16x2, l_run, false);
        pk[p] = __builtin_bit_cast(uint32_t, h);
      };
      f32x16 acc = {};
      if constexpr (decltype(two_terms)::value) add_low(nxt, acc);
      bf16x8 kq[3], vq[2];
      kq[0] = kread(0);
      if (NS > 1) kq[1] = kread(1);
#pragma unroll
      for (int ks = 0; ks < NSLOT; ++ks) {
        if (ks + 2 < NS) kq[(ks + 2) % 3] = kread(ks + 2);
        const int j = ks - 2;
        if (j + 1 >= 0 && j + 1 < NPV) vq[(j + 1) & 1] = vread(j + 1);
        __builtin_amdgcn_sched_barrier(0);
        if (ks == 0) __builtin_amdgcn_s_setprio(1);
        if (ks == NSLOT / 2) __builtin_amdgcn_s_setprio(0);
        if (ks < NS) acc = mfma32(kq[ks % 3], q[ks], acc);
        if (ks >= 1 && ks - 1 < C::PER_WAVE) load_part(ks - 1, stg);
        if (ks == C::PER_WAVE + 1) id = load_id(t + 3);
        if (ks < NSM) {
#pragma unroll
          for (int p = ks * 8 / NSM; p < (ks + 1) * 8 / NSM; ++p) sm_pair(p);
        }
        if (j >= 0 && j < NPV) {
          const int kk = j / C::DVB, d = j % C::DVB;
          const bf16x8 pb = as_bf16x8(kk == 0 ? u32x4{pk[0], pk[1], pk[2], pk[3]} : u32x4{pk[4], pk[5], pk[6], pk[7]});
          o[d] = mfma32(vq[j & 1], pb, o[d]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      s_nxt = acc;
      const uint32_t keys = there_n;  // of tile t + 1
      there_n = exist(row);
      wait_vmcnt<0>();  // this wave's part of tile t + 2 is in LDS
      __syncthreads();
      settle(t + 1, keys, nxt);
      mask(s_nxt, keys, t + 1);
      own_max = max_of(s_nxt);
      raise_max(s_nxt, two_terms);
    };

    wait_vmcnt<0>();
    __syncthreads();
    if (row0 >= n_rows) {  // no rows: this wave only loads
      __syncthreads();
      settle(0, there, tile[0]);
      one_term = !again && __builtin_amdgcn_readfirstlane(two_terms) == 0;
      int fill = 2;
      for (int t = 0; t < n_tiles; ++t) {
        row = row_of(t + 2, id);
        id = load_id(t + 3);
        load_tile(row, tile[fill]);
        fill = fill == 2 ? 0 : fill + 1;
        const uint32_t keys = there_n;
        there_n = exist(row);
        wait_vmcnt<0>();
        __syncthreads();
        settle(t + 1, keys, tile[(t + 1) % 3]);
      }
    } else {
      f32x16 s_a = {}, s_b;
#pragma unroll
      for (int ks = 0; ks < C::KS; ++ks)
        s_a = mfma32(as_bf16x8(*reinterpret_cast<const u32x4*>(&tile[0][((ks & 1) ? koff_o : koff_e) + ks * 16])),
                     q[ks], s_a);
      mask(s_a, there, 0);
      if (long_row || apart(s_a)) two_terms = 1;
      __syncthreads();  // every wave has used tile 0's K
      settle(0, there, tile[0]);
      one_term = !again && __builtin_amdgcn_readfirstlane(two_terms) == 0;
      if (!one_term) {  // (K is as it was, but for what makes a row NaN)
        fetch_lo();
        s_b = f32x16{};
        add_low(tile[0], s_b);
        s_a += s_b;
      }
      own_max = max_of(s_a);
      m_run = fmaxf(kLowest, half_swap_max(own_max));  // nothing to rescale yet
      auto steps = [&](auto both) __attribute__((always_inline)) {
        uint16_t *pc = tile[0], *pn = tile[1], *ps = tile[2];  // tile t lives in buffer t mod 3
        int t = 0;
        for (; t + 1 < n_tiles; t += 2) {
          step(t, s_a, s_b, pc, pn, ps, both);
          step(t + 1, s_b, s_a, pn, ps, pc, both);
          uint16_t* tmp = pc;
          pc = ps;
          ps = pn;
          pn = tmp;
        }
        if (t < n_tiles) step(t, s_a, s_b, pc, pn, ps, both);
      };
      if (one_term) steps(std::false_type{});
      else steps(std::true_type{});

      // ---- a whole block's latents, or this segment's partial result ----
      const float l = half_swap_sum(l_run + spoiled);
      if (r_own < n_rows) {
        const bool whole = n_tiles == pb.n_units;
        const int64_t prow = (2 * (int64_t)blockIdx.x + (u0 == 0)) * C::ROWS + wave * 32 + l32;
        const float f = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;  // (a row that sees nothing: zeros)
        float* dst = whole ? a.o_lat + ((int64_t)pb.lo * H + r_own) * DC : a.o_part + prow * DC;
#pragma unroll
        for (int d = 0; d < C::DVB; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int c = d * 32 + 8 * i + 4 * g;
            if (c < DC)
              *reinterpret_cast<f32x4*>(dst + c) =
                  f32x4{o[d][4 * i] * f, o[d][4 * i + 1] * f, o[d][4 * i + 2] * f, o[d][4 * i + 3] * f};
          }
        if (u0 == 0 && g == 0)
          a.plan.row[(int64_t)pb.lo * H + r_own] =
              PagedRow{(int32_t)blockIdx.x, (uint16_t)(last ? wk.last_ns : 1), (uint16_t)(wave * 32 + l32)};
        if (!whole && g == 0) {
          a.ml_part[prow * 2] = m_run;
          a.ml_part[prow * 2 + 1] = l;
        }
      }
    }
  }
}

// Waves per workgroup: eight (two per SIMD) while their accumulators fit; the tiny shape's are the tests'
constexpr int wide_waves(int dc) { return dc == 16 || dc == 256 ? 4 : 8; }

#define VMLA_PAGED_WIDE_SHAPES(X) X(16, 8) X(64, 32) X(128, 32) X(192, 32) X(256, 32)

}  // namespace

int paged_wide_rows(int d_c, int d_rope) {
#define X(DC, DR) if (d_c == DC && d_rope == DR) return 32 * wide_waves(DC);
  VMLA_PAGED_WIDE_SHAPES(X)
#undef X
  return 64;  // d_c = 512
}

hipError_t launch_paged_attend_wide(const PagedAttendArgs& a, hipStream_t s) {
#define X(DC, DR)                                                                                       \
  if (a.d_c == DC && a.d_rope == DR) {                                                                  \
    hipLaunchKernelGGL((paged_attend_wide_kernel<DC, DR, wide_waves(DC)>), dim3(a.n_wg),                \
                       dim3(64 * wide_waves(DC)), 0, s, a);                                             \
    return hipGetLastError();                                                                           \
  }
  VMLA_PAGED_WIDE_SHAPES(X)
#undef X
  if (a.d_c == 512 && a.d_rope == 32) return launch_paged_attend_wide512(a, s);
  return hipErrorInvalidValue;
}

}  // namespace vmla
