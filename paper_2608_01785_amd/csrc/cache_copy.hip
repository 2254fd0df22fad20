// Copies within a key/value cache: the first positions of one slot to another, in
// every layer.
//
// The first n positions of a head, n rounded up to whole value tiles, are one
// contiguous run in the keys and one in the values, 2 n dh bytes each: a copy is
// 2 heads layers runs between two slots.  A block moves a segment of a run, every
// thread two 16-byte words, both loaded before the first is stored.  The runs'
// segments are numbered without gaps, however long each copy is.  Memory bounds it, at
// two bytes moved for each copied: 120 slots of 4 MB take 158 us (6.4 TB/s read and
// written, some of it from the last-level cache; 480 slots 782, 5.2), 16 copies of 33 to
// 512 positions in 16 layers 103 (5.5; 127 in a grid over the longest copy, half of whose
// blocks have nothing to do), 64 positions in 4 layers 3.2.
// Segments of 16 KB take a tenth more where runs are short, of 32 KB half as much again.
#include "decoding_kernels.h"
#include "hs_device.h"

namespace hs {
namespace {

constexpr int kCopyThreads = 256;
constexpr int kCopyWords = kCopySegment / (kCopyThreads * 16);  // of a thread

__global__ __launch_bounds__(kCopyThreads) void cache_copy_kernel(CacheCopyArgs a) {
  // x: (head, segment); y: (layer, keys or values).
  const int head = blockIdx.x / uint32_t(a.segments), at_segment = blockIdx.x % uint32_t(a.segments);
  // The last copy that starts at or before the segment.
  int which = -1;
#pragma unroll
  for (int i0 = 0; i0 < kCopyList; i0 += 64) {
    const int i = i0 + int(threadIdx.x & 63);
    if (i0 < a.n_copies) which += __popcll(__ballot(i < a.n_copies && a.copies[min(i, a.n_copies - 1)].first <= at_segment));
  }
  const CacheCopyArgs::Copy c = a.copies[__builtin_amdgcn_readfirstlane(which)];
  const int64_t first = int64_t(at_segment - c.first) * kCopySegment, bytes = int64_t(c.tiles) * 64 * a.dh;
  uint16_t* base = (blockIdx.y & 1) ? a.v[blockIdx.y >> 1] : a.k[blockIdx.y >> 1];
  uint8_t* p = reinterpret_cast<uint8_t*>(base) + head * a.head_bytes + first;
  const int64_t slot = a.head_bytes * a.heads;
  const uint8_t* src = p + c.src * slot;
  uint8_t* dst = p + c.dst * slot;
  const int left = int(min(bytes - first, int64_t(kCopySegment)));
  u32x4 w[kCopyWords];
#pragma unroll
  for (int i = 0; i < kCopyWords; ++i) {
    const int at = (i * kCopyThreads + int(threadIdx.x)) * 16;
    if (at < left) w[i] = *reinterpret_cast<const u32x4*>(src + at);
  }
#pragma unroll
  for (int i = 0; i < kCopyWords; ++i) {
    const int at = (i * kCopyThreads + int(threadIdx.x)) * 16;
    if (at < left) *reinterpret_cast<u32x4*>(dst + at) = w[i];
  }
}

}  // namespace

hipError_t launch_cache_copy(const CacheCopyArgs& a, int, hipStream_t s) {
  if (a.n_copies < 1) return hipSuccess;
  hipLaunchKernelGGL(cache_copy_kernel, dim3(uint32_t(a.segments) * a.heads, 2 * a.layers), dim3(kCopyThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace hs
