// The plan of a paged attention call (vmla_paged.h says what it holds).
#pragma once
#include "vmla_paged.h"

namespace vmla {

// By one workgroup of 256 threads, beside the workgroups that absorb the queries: its chain of loads and
// scans, 6 to 8 us, then passes under theirs (a launch of its own took that long and stood in line).
constexpr int kPlanThreads = 256;
constexpr int kPlanNear = 512;  // blocks whose first counts are searched in LDS

// Exclusive prefix sums of v over the workgroup's threads; total: the sum.
__device__ __forceinline__ int64_t plan_scan(int64_t v, int64_t& total, int64_t* wave_sum) {
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

// lds: kPlanLds bytes, the other workgroups' staging area (an array of its own would cost all of them).
constexpr int kPlanLds = kPlanNear * 8 + kPlanThreads / 64 * 8 + (kPagedMaxSeqs + 2) * 4;

__device__ __forceinline__ void paged_plan(const PagedAttendArgs& a, void* lds) {
  int64_t* const first_near = reinterpret_cast<int64_t*>(lds);
  int64_t* const wave_sum = first_near + kPlanNear;
  int32_t* const first_block = reinterpret_cast<int32_t*>(wave_sum + kPlanThreads / 64);
  const PagedGeo& g = a.pg;
  const int tid = (int)threadIdx.x, H = a.n_heads, R = a.rows;
  int64_t blocks = 0;
  for (int s0 = 0; s0 < g.n_seqs; s0 += kPlanThreads) {
    const int s = s0 + tid;
    int64_t n = 0, total;
    if (s < g.n_seqs) {
      const PagedSeq q = paged_seq(g, s);
      n = ((int64_t)(q.hi - q.lo) * H + R - 1) / R;
    }
    const int64_t at = blocks + plan_scan(n, total, wave_sum);
    // offsets that go down could ask for more blocks than the call's rows make: those are left out
    if (s < g.n_seqs) first_block[s] = (int32_t)min(at, (int64_t)a.max_blocks);
    blocks += total;
  }
  blocks = min(blocks, (int64_t)a.max_blocks);
  if (tid == 0) first_block[g.n_seqs] = (int32_t)blocks;
  __syncthreads();
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
      const int i0 = q.kv - (q.hi - q.lo) + row0 / H;  // cached index of the first row's token
      PagedBlock p{};
      p.seq = lo;
      p.row0 = row0;
      p.lo = q.lo;
      p.n_rows = n_rows;
      p.kv = q.kv;
      p.head0 = row0 % H;
      int64_t to_next;
      paged_seen(g, q, i0, p.beg0, p.end0, to_next);
      p.to_next = (int32_t)min(to_next, (int64_t)1 << 30);
      int32_t b, e, b1, e1;
      paged_row_sees(g, p, H, 0, b, e);
      paged_row_sees(g, p, H, min(R, n_rows - row0) - 1, b1, e1);
      p.all_b = b1;
      p.all_e = e;
      p.key0 = b & ~31;
      p.n_units = max(1, (int)(((int64_t)e1 - p.key0 + a.unit - 1) / a.unit));
      a.plan.block[r] = p;
      n = p.n_units + a.cost;
    }
    const int64_t at = units + plan_scan(n, total, wave_sum);
    if (r < blocks) {
      a.plan.first[r] = at;
      if (r < kPlanNear) first_near[r] = at;
    }
    units += total;
  }
  __syncthreads();
  const int64_t G = min(units, (int64_t)a.n_wg);
  auto first_of = [&](int b) { return b < kPlanNear ? first_near[b] : a.plan.first[b]; };
  for (int w = tid; w < a.n_wg; w += kPlanThreads) {
    PagedWork k{};
    if (w < G) {
      const int64_t u = floor_div((int64_t)w * units, G), u1 = floor_div((int64_t)(w + 1) * units, G);
      int lo = 0, hi = (int)blocks - 1;  // the last block with first < u1
      while (lo < hi) {
        const int m = (lo + hi + 1) >> 1;
        if (first_of(m) < u1) lo = m;
        else hi = m - 1;
      }
      k.block = lo;
      const int64_t at = first_of(lo);
      const PagedBlock p = a.plan.block[lo];
      k.end = (int32_t)(u1 - at);
      k.n = (int32_t)(u1 - u);
      k.last_ns = attend_owner(at + a.cost + p.n_units - 1, units, (int)G) -
                  attend_owner(at + a.cost, units, (int)G) + 1;
      a.plan.work_block[w] = p;
    }
    a.plan.work[w] = k;
  }
}

}  // namespace vmla
