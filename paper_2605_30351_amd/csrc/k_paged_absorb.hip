// Query absorption of a paged attention call of few tokens, and the choice of the kernel that absorbs.
//
// q_cat[token, h] = [W_UK_h^T q_nope | RoPE(q_R)] * scale * log2 e. The matrix kernel (k_attend.hip) takes
// 128 tokens of a head per workgroup: with a few tokens only H workgroups run, each through a chain of
// staging, matrix steps and a staged store, 7 us at d_c = 192 and 14 us at 512. Here a workgroup takes up
// to kFewTokens tokens of one head, and its threads share W_UK_h's rows: thread (row group, 8 columns)
// has all its rows in flight at once and multiplies them on the VALU, and the row groups are summed
// through LDS. The last wave meanwhile finds the tokens' positions and rotates their positional queries.
#include "vmla_paged.h"
#include "vmla_paged_plan.h"

namespace vmla {
namespace {

constexpr int kFewTokens = 4;
// Calls of up to this many tokens take this kernel. d_c = 192, 12 heads, us here / matrix kernel: 68 tokens
// 7.5 / 11.0, 132 tokens 8.6 / 13.2, 244 tokens 10.4 / 13.2; d_c = 512, 132 tokens 13.0 / 29.3.
constexpr int kFewCalls = 256;
constexpr int kFewMaxNope = 128;

template <int DC, int DR>
__global__ __launch_bounds__(256) void paged_absorb_few_kernel(const PagedAttendArgs a) {
  constexpr int DQKP = (DC + DR + 15) / 16 * 16;
  constexpr int C8 = DC / 8, RG = 256 / C8;               // column chunks, row groups
  constexpr int PER = (kFewMaxNope + RG - 1) / RG;        // rows per thread
  constexpr int AT_ONCE = PER < 16 ? PER : 16;
  constexpr int TT = kFewTokens;
  __shared__ float qn[TT][kFewMaxNope];
  __shared__ __attribute__((aligned(16))) float red[RG][TT][DC + 4];
  static_assert(sizeof(red) >= kPlanLds, "the plan's arrays");
  if (blockIdx.x == 0) {
    if (blockIdx.y == 0) paged_plan(a, red);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int H = a.n_heads, h = blockIdx.y, dn = a.d_nope, t0 = ((int)blockIdx.x - 1) * TT;
  const int nt = min(a.pg.n_tokens - t0, TT);
  const int c8 = tid % C8, rg = tid / C8;
  const uint16_t* w = a.w_uk + (int64_t)h * dn * DC + c8 * 8;

  u32x4 wv[AT_ONCE];
#pragma unroll
  for (int i = 0; i < AT_ONCE; ++i) wv[i] = ldg16(w + (int64_t)min(rg + RG * i, dn - 1) * DC);
  for (int i = tid; i < TT * dn; i += 256) {
    const int t = i / dn, k = i - t * dn;
    qn[t][k] = t < nt ? bf16_bits_to_f32(a.q_nope[((int64_t)(t0 + t) * H + h) * dn + k]) : 0.f;
  }
  if (wave == 3) {  // positions and the RoPE part: lane = (token, pair)
    constexpr int NP = DR / 2;
    const int t = lane >> 4, pr = lane & 15;
    static_assert(NP <= 16 && TT <= 4, "a pair per lane");
    const int tok = min(t0 + t, a.pg.n_tokens - 1);
    const int s = paged_seq_of_lanes(a.pg, tok);
    const int64_t row = (int64_t)tok * H + h;
    TokenPos pos{};
    if (s >= 0) {
      const PagedSeq q = paged_seq(a.pg, s);
      paged_pos(a.pg, q.first + q.kv - (q.hi - tok), pos.f, pos.y, pos.x);
    }
    if (t < nt && pr < NP) {
      const uint32_t raw = *reinterpret_cast<const uint32_t*>(a.q_r + row * DR + 2 * pr);
      float u = bf16_bits_to_f32((uint16_t)(raw & 0xffff)), v = bf16_bits_to_f32((uint16_t)(raw >> 16));
      rope_rotate(a.rope, pr, pos, u, v);
      paged_q_pair(a, row * DQKP + DC + 2 * pr, u * a.qscale, v * a.qscale);
      if (pr == 0) {
        a.plan.row[row] = PagedRow{};
        for (int c = DC + DR; c < DQKP; c += 2) paged_q_pair(a, row * DQKP + c, 0.f, 0.f);
      }
    }
  }
  __syncthreads();
  float acc[TT][8];
#pragma unroll
  for (int t = 0; t < TT; ++t)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[t][e] = 0.f;
#pragma unroll
  for (int i0 = 0; i0 < PER; i0 += AT_ONCE) {
    if (i0 > 0) {
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) wv[i] = ldg16(w + (int64_t)min(rg + RG * (i0 + i), dn - 1) * DC);
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int k = rg + RG * (i0 + i);
      if (k < dn) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[2 * e] = __uint_as_float(wv[i][e] << 16);
          x[2 * e + 1] = __uint_as_float(wv[i][e] & 0xffff0000u);
        }
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[t][e] += qn[t][k] * x[e];
      }
    }
  }
  if (rg < RG) {
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        *reinterpret_cast<f32x4*>(&red[rg][t][c8 * 8 + 4 * e]) =
            f32x4{acc[t][4 * e], acc[t][4 * e + 1], acc[t][4 * e + 2], acc[t][4 * e + 3]};
  }
  __syncthreads();
  for (int i = tid; i < nt * (DC / 4); i += 256) {
    const int t = i / (DC / 4), c = i % (DC / 4) * 4;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int g = 0; g < RG; ++g) v += *reinterpret_cast<const f32x4*>(&red[g][t][c]);
    const int64_t at = ((int64_t)(t0 + t) * H + h) * DQKP + c;
    *reinterpret_cast<bf16x4*>(a.qcat + at) = to_bf16x4(v * a.qscale);
    paged_q_lo(a, at, v * a.qscale);
  }
}

}  // namespace

hipError_t launch_paged_absorb(const PagedAttendArgs& a, hipStream_t s) {
  if (a.pg.n_tokens > kFewCalls) return launch_paged_absorb_tiles(a, s);
  const dim3 grid((a.pg.n_tokens + kFewTokens - 1) / kFewTokens + 1, a.n_heads);
#define X(DC, DR)                                                                        \
  if (a.d_c == DC && a.d_rope == DR) {                                                   \
    hipLaunchKernelGGL((paged_absorb_few_kernel<DC, DR>), grid, dim3(256), 0, s, a);     \
    return hipGetLastError();                                                            \
  }
  X(16, 8) X(64, 32) X(128, 32) X(192, 32) X(256, 32) X(512, 32)
#undef X
  return hipErrorInvalidValue;
}

}  // namespace vmla
