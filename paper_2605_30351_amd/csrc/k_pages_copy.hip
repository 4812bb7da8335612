// Copies of whole pages inside a paged cache, in every layer (forked and compacted sequences).
//
// The pairs travel in the kernel's arguments: the host has checked them, no list has to live in device
// memory, and a captured graph holds its own. One workgroup copies one stretch of one page of one layer
// with 16-byte loads and stores.
#include "vmla_device.h"
#include "vmla_paged.h"

namespace vmla {
namespace {

constexpr int kCopyThreads = 256, kCopyUnroll = 4;
constexpr int kCopyBytes = kCopyThreads * kCopyUnroll * 16;  // per workgroup

// grid: (stretches of a page of c_kv then of k_r, pairs, layers)
__global__ __launch_bounds__(kCopyThreads) void pages_copy_kernel(const PagesCopyArgs a) {
  const int n0 = (int)((a.page_bytes[0] + kCopyBytes - 1) / kCopyBytes);
  const int k = (int)blockIdx.x >= n0;
  const int64_t off = (int64_t)((int)blockIdx.x - (k ? n0 : 0)) * kCopyBytes + threadIdx.x * 16;
  const int64_t bytes = a.page_bytes[k];
  char* layer = reinterpret_cast<char*>(a.pool[k]) + blockIdx.z * a.layer_bytes[k];
  const char* src = layer + a.src[blockIdx.y] * bytes;
  char* dst = layer + a.dst[blockIdx.y] * bytes;
  u32x4 v[kCopyUnroll];
#pragma unroll
  for (int i = 0; i < kCopyUnroll; ++i) {
    const int64_t at = off + i * kCopyThreads * 16;
    if (at < bytes) v[i] = *reinterpret_cast<const u32x4*>(src + at);
  }
#pragma unroll
  for (int i = 0; i < kCopyUnroll; ++i) {
    const int64_t at = off + i * kCopyThreads * 16;
    if (at < bytes) *reinterpret_cast<u32x4*>(dst + at) = v[i];
  }
}

}  // namespace

hipError_t launch_pages_copy(const PagesCopyArgs& a, hipStream_t s) {
  int64_t n = 0;
  for (int k = 0; k < 2; ++k) n += (a.page_bytes[k] + kCopyBytes - 1) / kCopyBytes;
  hipLaunchKernelGGL(pages_copy_kernel, dim3((unsigned)n, a.n_pairs, a.n_layers), dim3(kCopyThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace vmla
