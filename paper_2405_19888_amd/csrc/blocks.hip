// Copy of cache blocks: pool[dst[i]] = pool[src[i]] for every pool of a call (keys, values and
// scales of all layers), in a launch for every kCopyPools of them.
//
// Bound by memory: each byte is read and written once.  A workgroup copies 16 KiB of one block of
// one pool, 16 bytes a lane and four loads in flight; a block smaller than that (scales) takes one
// workgroup.
#include "cache8_args.h"

namespace parrot {

constexpr int kCopyChunk = 16384;        // bytes of a workgroup

__global__ __launch_bounds__(256) void k_copy_blocks(CopyArgs a, int chunks) {
  const int chunk = blockIdx.x % chunks, rest = blockIdx.x / chunks;
  const int i = rest % a.n, p = rest / a.n;
  const unsigned bytes = a.bytes[p];
  const unsigned at = (unsigned)chunk * kCopyChunk;
  if (at >= bytes) return;
  const int from = ld_uniform(a.src + i), to = ld_uniform(a.dst + i);
  if (from < 0 || to < 0 || from >= a.blocks || to >= a.blocks || from == to) return;
  const char* s = (const char*)a.base[p] + (size_t)from * bytes + at;
  char* d = (char*)a.base[p] + (size_t)to * bytes + at;
  const unsigned n = min((unsigned)kCopyChunk, bytes - at);
  if (bytes % 16 == 0) {
    u32x4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const unsigned o = (k * 256 + threadIdx.x) * 16;
      if (o < n) v[k] = ld16(s + o);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const unsigned o = (k * 256 + threadIdx.x) * 16;
      if (o < n) *reinterpret_cast<u32x4*>(d + o) = v[k];
    }
  } else {
    for (unsigned o = threadIdx.x * 2; o < n; o += 512)
      *reinterpret_cast<unsigned short*>(d + o) = *reinterpret_cast<const unsigned short*>(s + o);
  }
}

hipError_t launch_copy_blocks(const CopyArgs& a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  if (a.n < 1 || a.pools < 1 || a.pools > kCopyPools || a.blocks < 1) return hipErrorInvalidValue;
  unsigned most = 0;
  for (int p = 0; p < a.pools; ++p) most = a.bytes[p] > most ? a.bytes[p] : most;
  const long chunks = ((long)most + kCopyChunk - 1) / kCopyChunk;
  if (chunks * a.n * a.pools * 256 > 0xffffffffL) return hipErrorInvalidValue;
  hipExtLaunchKernelGGL(k_copy_blocks, dim3((unsigned)(chunks * a.n * a.pools)), dim3(256), 0, s, e0, e1, 0, a, (int)chunks);
  return hipGetLastError();
}

}  // namespace parrot
