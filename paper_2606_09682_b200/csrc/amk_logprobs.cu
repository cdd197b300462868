// amk_token_logprobs: log probabilities of given tokens, row entropies and top alternatives, in one pass over the logits.
//
// Mathematics.  With the running maximum r, R = r log2 e rounded and y = x log2 e - R, a thread sums s = sum 2^y and
// t = sum 2^y y over its share of the row; when R rises by d, s' = 2^-d s and t' = 2^-d (t - d s).  Shares are joined the
// same way: log probability of x = (x - r) - ln s + ln 2 (r log2 e - R), entropy = ln s - ln 2 t / s.  (Far from zero R is not
// rounded: below.)
//
// Alternatives.  Sorting is kept out of the pass: a thread keeps only the maximum of its share.  The k-th largest of
// those maxima is a lower bound of the k-th largest logit, so the alternatives lie in the shares whose maximum reaches
// it -- about k of the 256 -- and only those are read again (from L2), into sorted lists of 32 keys, one lane each, that
// are merged pairwise: {value, lowest index first} as one 64-bit key.
//
// Bound: HBM (the logits once).  A row is one block's, or with few rows a cluster's of up to four, whose parts meet
// in distributed shared memory: one launch, no scratch.
#include <cuda_runtime.h>
#include <math_constants.h>

#include "amk_op_util.h"
#include "amk_ptx.cuh"

namespace {

using namespace amk;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kUnroll = 4;                    // 16-byte pieces that a thread takes at a time
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr unsigned kAll = 0xffffffffu;

struct Args {
  int64_t vocab, stride;
  const int* tokens;
  int top;
  float *lp, *ent;
  int* top_id;
  float* top_lp;
};

__device__ __forceinline__ float load(const float* x, int64_t i) { return x[i]; }
__device__ __forceinline__ float load(const unsigned short* x, int64_t i) { return __uint_as_float((unsigned)x[i] << 16); }
// the elements of a 16-byte piece
__device__ __forceinline__ void widen(float (&v)[4], const uint4& u) {
  v[0] = __uint_as_float(u.x), v[1] = __uint_as_float(u.y), v[2] = __uint_as_float(u.z), v[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ void widen(float (&v)[8], const uint4& u) {
  v[0] = amk::bf16_lo(u.x), v[1] = amk::bf16_hi(u.x), v[2] = amk::bf16_lo(u.y), v[3] = amk::bf16_hi(u.y);
  v[4] = amk::bf16_lo(u.z), v[5] = amk::bf16_hi(u.z), v[6] = amk::bf16_lo(u.w), v[7] = amk::bf16_hi(u.w);
}
__device__ __forceinline__ float max_nan(float a, float b) {   // NaN if one of them is
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
// {value, lowest index first}, larger is better; NaN and "none" are 0
__device__ __forceinline__ unsigned long long key_of(float v, unsigned i) {
  if (v != v) return 0;
  const unsigned u = __float_as_uint(v == 0.f ? 0.f : v);
  return (unsigned long long)((u >> 31) ? ~u : u | 0x80000000u) << 32 | (0xffffffffu - i);
}
__device__ __forceinline__ float key_value(unsigned long long k) {
  const unsigned u = (unsigned)(k >> 32);
  return __uint_as_float((u >> 31) ? u & 0x7fffffffu : ~u);
}

__device__ __forceinline__ float min3(float a, float b, float c) {
  float d;
  asm("min.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// A share's sums, for a reference r: the largest x so far, or -kFar.  While |r| is below kFar, y = x log2 e - R with R the rounded
// r log2 e is one fused multiply-add; what the rounding of R leaves, eps(r), is in every y alike and taken out of the
// logarithm at the end.  It is half an ulp of R at most: 2^-4 at kFar, but 439 at 1e10, more than an exponential can
// take, so from kFar on y = (x - r) log2 e and eps is 0 (at -kFar the two are the same).
// Logits below -kFar are masks, and no more than a few tokens of a row may be without one: nothing is raised for them, they
// are 2^-kFar there.  A block whose part holds nothing else takes its sums again.  (600 rows of 128256, all but 1 in 1000 at -1e9, top 5:
// fp32 55 us, bf16 43 us; with every thread's own far reference 80 and 70 us.)
constexpr float kFar = 1048576.f, kHuge = 1.0e30f, kLowest = -3.402823466e38f;
__device__ __forceinline__ float ref(float r) { return r * kLog2e; }               // of an r below kFar
__device__ __forceinline__ float eps(float r) { return fabsf(r) < kFar ? fmaf(r, kLog2e, -ref(r)) : 0.f; }
struct Sums {
  float r, s, t;                                             // reference, sum of 2^y, sum of 2^y y
  __device__ __forceinline__ void raise(float to) {            // a finite reference, not below the old one
    // by how much the reference rises; (2^-1000 is 0 here; keeps 0 * d from being NaN)
    const float d = fminf(fmaf(to - r, kLog2e, eps(r) - eps(to)), 1000.f);
    const float f = exp2_fast(-d);
    t = f * (t - d * s);
    s *= f;
    r = to;
  }
  __device__ __forceinline__ void join(float r2, float s2, float t2) {
    Sums o{r2, s2, t2};
    if (o.r > r) raise(o.r);
    else o.raise(r);
    s += o.s, t += o.t;
  }
  __device__ __forceinline__ void see(float mx) {              // (infinity and NaN spoil the row's results anyway)
    if (mx > r && mx < CUDART_INF_F) raise(mx);
  }
  __device__ __forceinline__ void add(float x) {               // any x: -infinity and the lowest value are 0, not 0 * infinity
    const float y = fmaxf(fmaf(x - r, kLog2e, eps(r)), -200.f);
    const float e = exp2_fast(y);
    s += e;
    t = fmaf(e, y, t);
  }
};

// ---- lists of 32, one lane each, descending ---------------------------------------------------------------------
template <class K>
__device__ __forceinline__ K shfl_xor(K v, int o) { return __shfl_xor_sync(kAll, v, o); }
template <class K>
__device__ __forceinline__ K sort32(K v, int lane) {           // bitonic
#pragma unroll
  for (int size = 2; size <= 32; size *= 2)
#pragma unroll
    for (int o = size / 2; o; o /= 2) {
      const K w = shfl_xor(v, o);
      const bool first = !(lane & o), desc = !(lane & size) || size == 32;
      v = (first == desc) ? (v > w ? v : w) : (v < w ? v : w);
    }
  return v;
}
// the 32 best of two descending lists: b comes reversed, so that the maxima form a bitonic run
template <class K>
__device__ __forceinline__ K merge32(K a, K b_reversed, int lane) {
  K v = a > b_reversed ? a : b_reversed;
#pragma unroll
  for (int o = 16; o; o /= 2) {
    const K w = shfl_xor(v, o);
    v = !(lane & o) ? (v > w ? v : w) : (v < w ? v : w);
  }
  return v;
}
// every warp's list merged; the result is in warp 0.  `buf`: kWarps lists.
template <class K>
__device__ __forceinline__ K merge_warps(K v, K (*buf)[32], int warp, int lane) {
#pragma unroll
  for (int n = kWarps / 2; n; n /= 2) {
    if (warp >= n && warp < 2 * n) buf[warp][lane] = v;
    __syncthreads();
    if (warp < n) v = merge32(v, buf[warp + n][31 - lane], lane);
  }
  return v;
}

// C blocks a row.  Blocks on an SM: 5 for fp32, 3 for bf16, whose 32 values at a time need the registers.  (Without alternatives /
// with 5 / with 20 of them: 2001 bf16 rows of 128256, 5 blocks 187 / 201 / 228 us, 4 122 / 139 / 164 us, 3 94 / 111 / 132 us; 600
// fp32 rows, 3 blocks 59 / 69 / 84 us, 4 64 / 74 / 92 us, 5 50 / 57 / 72 us.)  Of a block's part, thread f has the 16-byte pieces
// f, f + 256, ...; the first block's threads also one element each in front of the first piece, the last block's one behind
// the last.
template <class T>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 4 ? 5 : 3) logprobs_kernel(const T* __restrict__ logits, const Args a, int C) {
  constexpr int kVec = 16 / sizeof(T);
  __shared__ unsigned long long lists[kWarps][32];
  __shared__ float part[4];                          // this block's reference, sums, NaN flag
  __shared__ float red[4][kWarps];
  __shared__ unsigned flagged[kWarps];
  __shared__ float bound;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const unsigned rank = C > 1 ? cluster_rank() : 0;
  amk::wait_for_grid_before();
  const int64_t row = C > 1 ? blockIdx.x / C : blockIdx.x;
  const T* x = logits + row * a.stride;
  const int vocab = (int)a.vocab;
  const int head = min(vocab, (int)((16 - ((uintptr_t)x & 15)) % 16 / sizeof(T)));
  const int pieces = (vocab - head) / kVec, tail = vocab - head - pieces * kVec;
  const int per = (pieces + C - 1) / C, p0 = min(pieces, (int)rank * per), n = min(pieces, p0 + per) - p0;
  const uint4* v4 = (const uint4*)(x + head) + p0;
  const int base = head + p0 * kVec;                 // index of the part's first element

  Sums sum{-kFar, 0.f, 0.f};
  float top = -CUDART_INF_F;                         // NaN if there was one
  auto single = [&](int i) {
    const float v = load(x, i);
    top = max_nan(top, v);
    sum.see(v);
    sum.add(v);
  };
  if (rank == 0 && (int)threadIdx.x < head) single(threadIdx.x);
  int at = threadIdx.x;                              // kUnroll pieces at a time, the next ones on their way
  {
    uint4 u[kUnroll];
    bool more = at + (kUnroll - 1) * kThreads < n;
    if (more) {
#pragma unroll
      for (int j = 0; j < kUnroll; j++) u[j] = __ldg(v4 + at + j * kThreads);
    }
    uint64_t s2 = pair(sum.s, 0.f), t2 = pair(sum.t, 0.f);
    while (more) {
      at += kUnroll * kThreads;
      more = at + (kUnroll - 1) * kThreads < n;
      uint4 next[kUnroll];
      if (more) {
#pragma unroll
        for (int j = 0; j < kUnroll; j++) next[j] = __ldg(v4 + at + j * kThreads);
      }
      float mx = -CUDART_INF_F, mn = CUDART_INF_F;
#pragma unroll
      for (int j = 0; j < kUnroll; j++) {
        float v[kVec];
        widen(v, u[j]);
#pragma unroll
        for (int k = 0; k < kVec; k += 2) mx = max3_nan(mx, v[k], v[k + 1]), mn = min3(mn, v[k], v[k + 1]);
      }
      top = max_nan(top, mx);
      // (masked: values so low that 0 times y could be 0 times infinity, or a reference that wants the other y)
      const bool rises = mx > sum.r, masked = mn < -kHuge || (rises && mx >= kFar) || sum.r >= kFar;
      if (rises || masked) {
        float a0, a1;
        unpair(a0, a1, s2);
        sum.s = a0 + a1;
        unpair(a0, a1, t2);
        sum.t = a0 + a1;
        sum.see(mx);
        if (masked) {
#pragma unroll 1
          for (int j = 0; j < kUnroll; j++) {
            float v[kVec];
            widen(v, j == 0 ? u[0] : j == 1 ? u[1] : j == 2 ? u[2] : u[3]);
#pragma unroll
            for (int k = 0; k < kVec; k++) sum.add(v[k]);
          }
        }
        s2 = pair(sum.s, 0.f), t2 = pair(sum.t, 0.f);
      }
      if (!masked) {
        const uint64_t l2 = pair(kLog2e, kLog2e), r2 = pair(-ref(sum.r), -ref(sum.r));
#pragma unroll
        for (int j = 0; j < kUnroll; j++) {
          float v[kVec];
          widen(v, u[j]);
#pragma unroll
          for (int k = 0; k < kVec; k += 2) {
            const uint64_t y = fma2(pair(v[k], v[k + 1]), l2, r2);
            float y0, y1;
            unpair(y0, y1, y);
            const uint64_t e = pair(exp2_fast(y0), exp2_fast(y1));
            s2 = add2(s2, e);
            t2 = fma2(e, y, t2);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < kUnroll; j++) u[j] = next[j];
    }
    float a0, a1;
    unpair(a0, a1, s2);
    sum.s = a0 + a1;
    unpair(a0, a1, t2);
    sum.t = a0 + a1;
  }
  for (; at < n; at += kThreads) {
    float v[kVec];
    widen(v, __ldg(v4 + at));
    float mx = v[0];
#pragma unroll
    for (int k = 1; k < kVec; k++) mx = max_nan(mx, v[k]);
    top = max_nan(top, mx);
    sum.see(mx);
#pragma unroll
    for (int k = 0; k < kVec; k++) sum.add(v[k]);
  }
  if (rank == (unsigned)C - 1 && (int)threadIdx.x < tail) single(head + pieces * kVec + threadIdx.x);
  const bool share_nan = top != top;

  // the block's sums
  const bool nan = __any_sync(kAll, share_nan) != 0;
  float r = sum.r, m = share_nan ? CUDART_INF_F : top;   // (m: whether the maximum is infinite; a NaN spoils the row as well)
#pragma unroll
  for (int o = 16; o; o /= 2) r = fmaxf(r, shfl_xor(r, o)), m = fmaxf(m, shfl_xor(m, o));
  sum.raise(r);
#pragma unroll
  for (int o = 16; o; o /= 2) sum.s += shfl_xor(sum.s, o), sum.t += shfl_xor(sum.t, o);
  if (lane == 0) red[0][warp] = r, red[1][warp] = sum.s, red[2][warp] = sum.t, red[3][warp] = nan ? CUDART_INF_F : m;

  // the block's alternatives, in warp 0
  unsigned long long best = 0;
  if (a.top) {
    const unsigned mine = share_nan ? 0 : (unsigned)(key_of(top, 0) >> 32);   // a share with NaN bounds nothing
    const unsigned sorted = sort32(mine, lane);
    const unsigned all = merge_warps(sorted, (unsigned (*)[32])lists, warp, lane);
    const unsigned kth = __shfl_sync(kAll, all, a.top - 1);
    if (threadIdx.x == 0) bound = __uint_as_float(kth);
    __syncthreads();
    const unsigned low = __float_as_uint(bound);
    const float lowest = low ? key_value((unsigned long long)low << 32) : -CUDART_INF_F;
    const unsigned f = __ballot_sync(kAll, share_nan || (mine && mine >= low));
    if (lane == 0) flagged[warp] = f;
    __syncthreads();
    // flagged shares go round the warps; a warp reads one share at a time, a piece for each lane
    unsigned long long kth_key = 0;
    auto take = [&](unsigned long long k) {          // this lane's candidate joins the warp's list
      unsigned w = __ballot_sync(kAll, k > kth_key);
      if (!w) return;
      if (__popc(w) > 4) {
        best = merge32(best, __shfl_sync(kAll, sort32(k, lane), 31 - lane), lane);
      } else {
        for (; w; w &= w - 1) {
          const unsigned long long c = __shfl_sync(kAll, k, __ffs(w) - 1), up = __shfl_up_sync(kAll, best, 1);
          if (c > best) best = lane && c > up ? up : c;
        }
      }
      kth_key = __shfl_sync(kAll, best, a.top - 1);
    };
    int turn = 0;
    for (int w = 0; w < kWarps; w++) {
      for (unsigned g = flagged[w]; g; g &= g - 1, turn++) {
        if (turn % kWarps != warp) continue;
        const int share = w * 32 + __ffs(g) - 1;
        if (rank == 0 && share < head) take(lane == 0 ? key_of(load(x, share), share) : 0);
        if (rank == (unsigned)C - 1 && share < tail) {
          const int i = head + pieces * kVec + share;
          take(lane == 0 ? key_of(load(x, i), i) : 0);
        }
        for (int i0 = share; i0 < n; i0 += 32 * kThreads) {
          const int i = i0 + lane * kThreads;
          float v[kVec];
          float mx = CUDART_NAN_F;
          if (i < n) {
            widen(v, __ldg(v4 + i));
#pragma unroll
            for (int k = 0; k < kVec; k++) mx = fmaxf(mx, v[k]);
          }
          if (!__any_sync(kAll, mx >= lowest)) continue;
#pragma unroll
          for (int k = 0; k < kVec; k++) take(mx >= lowest && v[k] >= lowest ? key_of(v[k], base + i * kVec + k) : 0);
        }
      }
    }
    __syncthreads();
    best = merge_warps(best, lists, warp, lane);
  }
  __syncthreads();
  float most = red[3][0];                            // the block's maximum
#pragma unroll
  for (int w = 1; w < kWarps; w++) most = fmaxf(most, red[3][w]);
  if (most < -kFar) {                                // nothing but masks: the sums again, for that reference
    Sums own{fmaxf(most, kLowest), 0.f, 0.f};        // (all of -infinity: sums of 0, below any other part's reference)
    const int again = most > -CUDART_INF_F ? n : 0;
    if (rank == 0 && (int)threadIdx.x < head) own.add(load(x, threadIdx.x));
#pragma unroll 1
    for (int i = threadIdx.x; i < again; i += kThreads) {
      float v[kVec];
      widen(v, __ldg(v4 + i));
#pragma unroll
      for (int k = 0; k < kVec; k++) own.add(v[k]);
    }
    if (rank == (unsigned)C - 1 && (int)threadIdx.x < tail) own.add(load(x, head + pieces * kVec + threadIdx.x));
#pragma unroll
    for (int o = 16; o; o /= 2) own.s += shfl_xor(own.s, o), own.t += shfl_xor(own.t, o);
    __syncthreads();                                 // (red[3] has been read)
    if (lane == 0) red[0][warp] = own.r, red[1][warp] = own.s, red[2][warp] = own.t;
    __syncthreads();
  }
  if (warp == 0) {
    Sums b{lane < kWarps ? red[0][lane] : -kFar, lane < kWarps ? red[1][lane] : 0.f, lane < kWarps ? red[2][lane] : 0.f};
    float mm = lane < kWarps ? red[3][lane] : -CUDART_INF_F;
#pragma unroll
    for (int o = kWarps / 2; o; o /= 2) {
      b.join(shfl_xor(b.r, o), shfl_xor(b.s, o), shfl_xor(b.t, o));
      mm = fmaxf(mm, shfl_xor(mm, o));
    }
    if (C > 1) {
      if (lane == 0) part[0] = b.r, part[1] = b.s, part[2] = b.t, part[3] = mm;
      lists[0][lane] = best;
    }
    sum = b;
    m = mm;
  }
  if (C > 1) {
    __syncthreads();
    cluster_sync();
    if (rank == 0 && warp == 0) {
      for (int c = 1; c < C; c++) {
        sum.join(remote_f32(&part[0], c), remote_f32(&part[1], c), remote_f32(&part[2], c));
        m = fmaxf(m, remote_f32(&part[3], c));
        if (a.top) best = merge32(best, remote_u64(&lists[0][31 - lane], c), lane);
      }
    }
    cluster_sync();                                  // the others' shared memory has been read
  }
  if (rank || warp) return;
  m = __shfl_sync(kAll, m, 0);
  const float s = __shfl_sync(kAll, sum.s, 0), t = __shfl_sync(kAll, sum.t, 0);
  const float r0 = __shfl_sync(kAll, sum.r, 0);
  // NaN without a finite maximum, or with a NaN
  const float ls = fabsf(m) < CUDART_INF_F ? logf(s) : CUDART_NAN_F, from_r = fmaf(-kLn2, eps(r0), ls);
  if (lane == 0) {
    const int tok = a.tokens[row];
    if (a.lp) a.lp[row] = tok < 0 || tok >= vocab ? CUDART_NAN_F : load(x, tok) - r0 - from_r;
    if (a.ent) a.ent[row] = fmaf(-kLn2, t / s, ls);
  }
  if (lane < a.top) {
    a.top_id[row * a.top + lane] = best ? (int)(0xffffffffu - (unsigned)best) : -1;
    a.top_lp[row * a.top + lane] = best ? key_value(best) - r0 - from_r : CUDART_NAN_F;
  }
}

template <class T>
cudaError_t launch(const void* logits, const Args& a, int64_t rows, int C, cudaStream_t st) {
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;         // the kernel waits for the one before it itself
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)C, at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(rows * C));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cfg.attrs = at;
  cfg.numAttrs = C > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, logprobs_kernel<T>, (const T*)logits, a, C);
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
  // Blocks a row: doubled until there are two for each SM, while a block keeps 2048 logits.  (fp32 logits, calls in a row, top 5 /
  // top 20, 1, 2, 4 and 8 blocks a row: one row of 32000 8.1 / 9.7, 8.0 / 9.6, 8.8 / 10.3, 10.6 / 12.2 us; 64 of 128256 25.4 / 29.0,
  // 17.7 / 20.2, 15.3 / 17.3, 17.1 / 19.5 us; 200 of 128256 31.8 / 37.2, 25.4 / 29.1, 35.9 / 40.5, 47.5 / 54.8 us.)
  int dev = 0, sms = 148, C = 1;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    (void)cudaGetLastError();
  while (C < 4 && rows * C < 2 * sms && vocab / (2 * C) >= 2048) C *= 2;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  const cudaError_t e = dtype ? launch<unsigned short>(logits, a, rows, C, st) : launch<float>(logits, a, rows, C, st);
  return e == cudaSuccess ? AMK_OK : fail(AMK_ERR_CUDA, "launch failed: %s", cudaGetErrorString(e));
}
