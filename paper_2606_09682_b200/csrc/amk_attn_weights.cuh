// The kernel of amk_attention_weights: what the queries of some tokens attend to, added up for each cached position.
#pragma once
#include "amk_attn.cuh"

namespace amk {

struct WeightsParams {
  const unsigned short* q;
  const void* k;
  const float* lse;
  const int* lens;
  const float* before;
  float* out;
  int64_t q_seq, q_row, q_head, k_seq, k_head, k_row, b_seq, b_head, o_seq, o_head;
  int n_seqs, nq, nkv, rep, rows, slots;
  float scale, decay;
};

// One thread for a cached position, which it holds in registers; the queries go by in shared memory.
template <int HD, bool FP8>
__global__ void __launch_bounds__(kTile) weights_kernel(const WeightsParams p) {
  constexpr int kQueries = 8;
  __shared__ float qs[kQueries][HD];
  __shared__ float ls[kQueries];
  const int seq = blockIdx.z, head = blockIdx.y, key = blockIdx.x * kTile + threadIdx.x;
  wait_for_grid_before();
  const int len = p.lens[seq];
  float* out = p.out + seq * p.o_seq + head * p.o_head;
  if (len < 0 || len > p.slots - p.rows) {
    if (key < p.slots) out[key] = CUDART_NAN_F;
    return;
  }
  const int keys = len + p.rows;
  float kf[HD];
  if (key < keys) {
    const int64_t at = seq * p.k_seq + head * p.k_head + key * p.k_row;
#pragma unroll
    for (int e = 0; e < HD; e++) {
      if (FP8) {
        unsigned w[2];
        widen_e4m3(w, ((const unsigned char*)p.k)[at + e]);
        float hi;
        unpack_f16(kf[e], hi, w[0]);
      } else {
        kf[e] = __uint_as_float((unsigned)((const unsigned short*)p.k)[at + e] << 16);
      }
    }
  }
  float sum = 0.f;
  const int all = p.rows * p.rep, first = max(0, (int)(blockIdx.x * kTile) - len) * p.rep;
  for (int r0 = first; r0 < all; r0 += kQueries) {
    const int n = min(kQueries, all - r0);
    __syncthreads();
    for (int i = threadIdx.x; i < n * HD; i += kTile) {
      const int r = r0 + i / HD, tok = r / p.rep, h = head * p.rep + r - tok * p.rep;
      qs[i / HD][i % HD] = __uint_as_float((unsigned)p.q[seq * p.q_seq + tok * p.q_row + h * p.q_head + i % HD] << 16);
    }
    if ((int)threadIdx.x < n) {
      const int r = r0 + threadIdx.x, tok = r / p.rep;
      ls[threadIdx.x] = p.lse[((int64_t)seq * p.rows + tok) * p.nq + head * p.rep + r - tok * p.rep];
    }
    __syncthreads();
    for (int i = 0; i < n; i++) {
      if (key > len + (r0 + i) / p.rep || key >= keys || fabsf(ls[i]) == CUDART_INF_F) continue;
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < HD; e++) s = fmaf(qs[i][e], kf[e], s);
      sum += exp2f(fmaf(s, p.scale * kLog2e, -ls[i] * kLog2e));
    }
  }
  if (key >= p.slots) return;
  if (key >= keys) sum = 0.f;
  if (key < len && p.before && p.decay != 0.f) sum = fmaf(p.decay, p.before[seq * p.b_seq + head * p.b_head + key], sum);
  out[key] = sum;
}

}  // namespace amk
