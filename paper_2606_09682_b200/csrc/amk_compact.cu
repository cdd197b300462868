// amk_kv_compact: kept rows of KV caches moved together, in place, in every plane.
#include <cuda_runtime.h>

#include "amk_op_util.h"
#include "amk_ptx.cuh"

namespace {

// One block per (cache, plane).  The rows go in batches, in ascending order: a batch is read into registers, the whole
// block has read it (barrier), then it is written.  keep is strictly ascending from keep[0] >= base, so
// keep[i] >= base + i: a batch is written at or below its own first source, never onto the source of a later batch.
// Bound: HBM for long lists (each row once in, once out): what counts is the bytes a block has under way, VEC 16-byte
// pieces a thread.  Short lists are one batch of few threads.
template <int THREADS, int VEC>
__global__ void __launch_bounds__(THREADS) kv_compact_kernel(uint4* kv, int64_t cache_pieces, int n_planes,
                                                             int64_t max_seq, int row_pieces, const int* base_of,
                                                             const int* keep_of, int64_t max_keep, const int* count_of) {
  const int plane = blockIdx.x % n_planes, cache = blockIdx.x / n_planes;
  amk::wait_for_grid_before();
  const int base = base_of[cache], n = count_of[cache];
  const int* keep = keep_of + (int64_t)cache * max_keep;
  bool bad = n < 0 || n > max_keep || base < 0;
  if (!bad)
    for (int i = threadIdx.x; i < n; i += THREADS)
      bad |= keep[i] >= max_seq || keep[i] < (i ? keep[i - 1] + 1 : base);
  if (__syncthreads_or(bad)) return;
  const int rows = THREADS / row_pieces;             // rows a pass; threads behind the last whole row have none
  const int r0 = (int)threadIdx.x < rows * row_pieces ? threadIdx.x / row_pieces : n;
  uint4* p = kv + cache * cache_pieces + plane * (max_seq * row_pieces) + threadIdx.x % row_pieces;
  for (int at = 0; at < n; at += rows * VEC) {
    uint4 r[VEC];
#pragma unroll
    for (int j = 0; j < VEC; j++)
      if (r0 < n - at - j * rows) r[j] = p[(int64_t)keep[at + r0 + j * rows] * row_pieces];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < VEC; j++)
      if (r0 < n - at - j * rows) p[(int64_t)(base + at + r0 + j * rows) * row_pieces] = r[j];
  }
}

}  // namespace

extern "C" amk_status amk_kv_compact(void* kv, int64_t n_caches, int64_t cache_stride, int64_t n_planes,
                                     int64_t max_seq, int64_t row_bytes, const int32_t* base, const int32_t* keep,
                                     int64_t max_keep, const int32_t* count, char* msg, size_t msg_bytes,
                                     void* cuda_stream) {
  const amk::Reason fail(msg, msg_bytes, "amk_kv_compact");
  if (n_caches < 0 || n_planes < 1 || max_seq < 1 || max_keep < 0 || max_keep > max_seq || max_seq > 0x7fff0000 ||
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
  const int64_t blocks = n_caches * n_planes;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  // (26 rows of 256 bytes in 512 planes: 3.1 us the small way; 5000 rows of 128 bytes in 352 planes, 422 MB: 256 threads x 4
  // pieces 86 us, 512 x 8 84 us, 1024 x 4 78 us, 1024 x 8 73 us = 5.8 TB/s)
  const bool few = max_keep * row_bytes <= 65536;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;            // the kernel waits for the one before it itself
  at.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(few ? 256 : 1024);
  cfg.stream = st;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, few ? kv_compact_kernel<256, 4> : kv_compact_kernel<1024, 8>, (uint4*)kv,
                                           cache_stride / 16, (int)n_planes, max_seq, (int)(row_bytes / 16), base, keep, max_keep,
                                           count);
  return e == cudaSuccess ? AMK_OK : fail(AMK_ERR_CUDA, "launch failed: %s", cudaGetErrorString(e));
}
