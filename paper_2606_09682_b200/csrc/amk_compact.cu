// amk_kv_compact: kept rows of KV caches moved together, in place, in every plane.
#include <cuda_runtime.h>

#include "amk_op_util.h"

namespace {

constexpr int kThreads = 256;
constexpr int kVec = 4;   // 16-byte pieces a thread carries from one batch of rows to the next

// One block per (plane, cache).  The rows go in batches, in ascending order: a batch is read into registers, the
// whole block has read it (barrier), then it is written.  keep is strictly ascending from keep[0] >= base, so
// keep[i] >= base + i: a batch is written at or below its own first source, never onto the source of a later batch.
__global__ void __launch_bounds__(kThreads) kv_compact_kernel(uint4* kv, int64_t cache_pieces, int n_planes,
                                                              int64_t max_seq, int row_pieces, const int* base_of,
                                                              const int* keep_of, int64_t max_keep,
                                                              const int* count_of) {
  const int plane = blockIdx.x % n_planes, cache = blockIdx.x / n_planes;
  const int base = base_of[cache], n = count_of[cache];
  const int* keep = keep_of + (int64_t)cache * max_keep;
  bool bad = n < 0 || n > max_keep || base < 0;
  if (!bad)
    for (int i = threadIdx.x; i < n; i += kThreads)
      bad |= keep[i] >= max_seq || keep[i] < (i ? keep[i - 1] + 1 : base);
  if (__syncthreads_or(bad)) return;
  uint4* p = kv + cache * cache_pieces + plane * (max_seq * row_pieces);
  const int64_t pieces = (int64_t)n * row_pieces;
  for (int64_t at = 0; at < pieces; at += kThreads * kVec) {
    uint4 r[kVec];
#pragma unroll
    for (int j = 0; j < kVec; j++) {
      const int64_t e = at + j * kThreads + threadIdx.x;
      if (e < pieces) r[j] = p[(int64_t)keep[e / row_pieces] * row_pieces + e % row_pieces];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kVec; j++) {
      const int64_t e = at + j * kThreads + threadIdx.x;
      if (e < pieces) p[(int64_t)base * row_pieces + e] = r[j];
    }
  }
}

}  // namespace

extern "C" amk_status amk_kv_compact(void* kv, int64_t n_caches, int64_t cache_stride, int64_t n_planes,
                                     int64_t max_seq, int64_t row_bytes, const int32_t* base, const int32_t* keep,
                                     int64_t max_keep, const int32_t* count, char* msg, size_t msg_bytes,
                                     void* cuda_stream) {
  const amk::Reason fail(msg, msg_bytes, "amk_kv_compact");
  if (n_caches < 0 || n_planes < 1 || max_seq < 1 || max_keep < 0 || max_keep > max_seq || max_seq > 0x7fffffff ||
      n_planes > 0x7fffffff)
    return fail(AMK_ERR_INVALID_ARG, "%lld caches of %lld planes of %lld rows, %lld kept at most",
                (long long)n_caches, (long long)n_planes, (long long)max_seq, (long long)max_keep);
  if (row_bytes < 16 || row_bytes > 1024 || row_bytes % 16)
    return fail(AMK_ERR_INVALID_ARG, "row_bytes %lld: a multiple of 16 up to 1024", (long long)row_bytes);
  if (n_caches == 0 || max_keep == 0) return AMK_OK;
  if (n_caches > 0x7fffffff / n_planes) return fail(AMK_ERR_INVALID_ARG, "more than 2^31 - 1 planes");
  if (!kv || !base || !keep || !count) return fail(AMK_ERR_INVALID_ARG, "NULL pointer");
  if (!amk::aligned(kv, 16) || !amk::aligned(base, 4) || !amk::aligned(keep, 4) || !amk::aligned(count, 4))
    return fail(AMK_ERR_INVALID_ARG, "kv must be 16-byte aligned, base, keep and count 4-byte aligned");
  if (n_caches > 1 && (cache_stride % 16 || cache_stride / row_bytes / n_planes < max_seq))
    return fail(AMK_ERR_INVALID_ARG, "cache_stride %lld: a multiple of 16, no less than one cache",
                (long long)cache_stride);
  kv_compact_kernel<<<(int)(n_caches * n_planes), kThreads, 0, (cudaStream_t)cuda_stream>>>(
      (uint4*)kv, cache_stride / 16, (int)n_planes, max_seq, (int)(row_bytes / 16), base, keep, max_keep, count);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? AMK_OK : fail(AMK_ERR_CUDA, "launch failed: %s", cudaGetErrorString(e));
}
