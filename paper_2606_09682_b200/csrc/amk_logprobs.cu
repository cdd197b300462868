// amk_token_logprobs: log probabilities of given tokens, row entropies and top alternatives.
#include <cuda_runtime.h>
#include <math_constants.h>

#include "amk_op_util.h"
#include "amk_ptx.cuh"

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float load(const float* x, int64_t i) { return x[i]; }
__device__ __forceinline__ float load(const unsigned short* x, int64_t i) { return __uint_as_float((unsigned)x[i] << 16); }

struct Args {
  int64_t vocab, stride;
  const int* tokens;
  int top;
  float *lp, *ent;
  int* top_id;
  float* top_lp;
};

template <class T>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(const T* logits, Args a) {
  __shared__ float red[3][kThreads / 32];
  __shared__ unsigned long long best[kThreads / 32];
  const int64_t r = blockIdx.x;
  const T* x = logits + r * a.stride;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float m = -CUDART_INF_F;
  bool nan = false;
  for (int64_t i = threadIdx.x; i < a.vocab; i += kThreads) {
    const float v = load(x, i);
    nan |= v != v;
    m = fmaxf(m, v);
  }
  nan = __syncthreads_or(nan);
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
  if (lane == 0) red[0][warp] = m;
  __syncthreads();
  for (int w = 0; w < kThreads / 32; w++) m = fmaxf(m, red[0][w]);
  float s = 0, t = 0;
  for (int64_t i = threadIdx.x; i < a.vocab; i += kThreads) {
    const float d = load(x, i) - m;
    const float e = expf(d);
    s += e;
    if (e > 0) t += e * d;
  }
  for (int o = 16; o; o >>= 1) {
    s += __shfl_xor_sync(~0u, s, o);
    t += __shfl_xor_sync(~0u, t, o);
  }
  if (lane == 0) red[1][warp] = s, red[2][warp] = t;
  __syncthreads();
  s = t = 0;
  for (int w = 0; w < kThreads / 32; w++) s += red[1][w], t += red[2][w];
  const float bad = nan || !(fabsf(m) < CUDART_INF_F) ? CUDART_NAN_F : 0.f;
  const float ls = logf(s) + bad;
  if (threadIdx.x == 0) {
    const int tok = a.tokens[r];
    if (a.lp) a.lp[r] = tok < 0 || tok >= a.vocab ? CUDART_NAN_F : load(x, tok) - m - ls;
    if (a.ent) a.ent[r] = ls - t / s;
  }
  // the k-th alternative: the largest key {value, lowest index first} below the one before
  unsigned long long prev = ~0ull;
  for (int k = 0; k < a.top; k++) {
    unsigned long long b = 0;
    for (int64_t i = threadIdx.x; i < a.vocab; i += kThreads) {
      const float v = load(x, i);
      if (v != v) continue;
      const unsigned u = __float_as_uint(v == 0.f ? 0.f : v);
      const unsigned long long key =
          (unsigned long long)((u >> 31) ? ~u : u | 0x80000000u) << 32 | (0xffffffffu - (unsigned)i);
      if (key < prev && key > b) b = key;
    }
    for (int o = 16; o; o >>= 1) {
      const unsigned long long ob = __shfl_xor_sync(~0u, b, o);
      b = ob > b ? ob : b;
    }
    __syncthreads();
    if (lane == 0) best[warp] = b;
    __syncthreads();
    for (int w = 0; w < kThreads / 32; w++) b = best[w] > b ? best[w] : b;
    if (threadIdx.x == 0) {
      const int id = (int)(0xffffffffu - (unsigned)b);
      a.top_id[r * a.top + k] = b ? id : -1;
      a.top_lp[r * a.top + k] = b ? load(x, id) - m - ls : CUDART_NAN_F;
    }
    prev = b;
  }
}

}  // namespace

extern "C" amk_status amk_token_logprobs(const void* logits, uint32_t dtype, int64_t rows, int64_t vocab,
                                         int64_t row_stride, const int32_t* tokens, uint32_t top_k, float* logprob,
                                         float* entropy, int32_t* top_tokens, float* top_logprobs, char* msg,
                                         size_t msg_bytes, void* cuda_stream) {
  const amk::Reason fail(msg, msg_bytes, "amk_token_logprobs");
  if (dtype > 1) return fail(AMK_ERR_UNSUPPORTED, "dtype %u: 0 (float) or 1 (bf16)", dtype);
  if (top_k > AMK_LOGPROBS_MAX_TOP)
    return fail(AMK_ERR_UNSUPPORTED, "top_k = %u exceeds AMK_LOGPROBS_MAX_TOP = %d", top_k, AMK_LOGPROBS_MAX_TOP);
  if (rows < 0 || rows > 0x7fffffff || vocab < 1 || vocab > 0x7fffffff)
    return fail(AMK_ERR_INVALID_ARG, "%lld rows of %lld logits", (long long)rows, (long long)vocab);
  if (rows == 0) return AMK_OK;
  if (rows > 1 && row_stride < vocab)
    return fail(AMK_ERR_INVALID_ARG, "row_stride %lld is less than a row", (long long)row_stride);
  if (!logits || !tokens || (top_k && (!top_tokens || !top_logprobs)))
    return fail(AMK_ERR_INVALID_ARG, "NULL pointer");
  if (!amk::aligned(logits, dtype ? 2 : 4) || !amk::aligned(tokens, 4) || !amk::aligned(logprob, 4) ||
      !amk::aligned(entropy, 4) || !amk::aligned(top_tokens, 4) || !amk::aligned(top_logprobs, 4))
    return fail(AMK_ERR_INVALID_ARG, "pointers must be aligned to their elements");
  const Args a{vocab, row_stride, tokens, (int)top_k, logprob, entropy, top_tokens, top_logprobs};
  if (dtype)
    logprobs_kernel<<<(int)rows, kThreads, 0, (cudaStream_t)cuda_stream>>>((const unsigned short*)logits, a);
  else
    logprobs_kernel<<<(int)rows, kThreads, 0, (cudaStream_t)cuda_stream>>>((const float*)logits, a);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? AMK_OK : fail(AMK_ERR_CUDA, "launch failed: %s", cudaGetErrorString(e));
}
