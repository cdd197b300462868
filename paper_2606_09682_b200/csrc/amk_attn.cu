// amk_prompt_attention and amk_tree_attention: argument checks and launches.
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <math.h>
#include <math_constants.h>

#include "amk_op_util.h"
#include "amk_ptx.cuh"

namespace {

using amk::Reason;

struct Params {
  const unsigned char *q, *k, *v;
  __nv_bfloat16* out;
  float* lse;
  const int* lens;                 // prompt: cu_seqlens; tree: cache_len
  const unsigned long long* mask;
  int64_t q_seq, q_row, q_head, k_seq, k_row, k_head, v_seq, v_row, v_head, o_seq, o_row, o_head;
  int n_seqs, nq, rep, rows, slots;   // rows: prompt: all tokens; tree: drafted tokens of a sequence
  float scale;
};

template <bool FP8>
__device__ __forceinline__ float element(const unsigned char* p, int64_t i) {
  if (FP8) {
    __nv_fp8_e4m3 e;
    e.__x = p[i];
    return (float)e;
  }
  return __uint_as_float((unsigned)((const unsigned short*)p)[i] << 16);
}

// One warp per (token, head): 32 keys at a time, one per lane.
template <int HD, bool TREE, bool FP8>
__global__ void __launch_bounds__(128) attn_kernel(const Params p) {
  __shared__ float qs[4][HD];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t w = (int64_t)blockIdx.x * 4 + warp;
  const int h = (int)(w % p.nq), g = h / p.rep;
  const int64_t row = w / p.nq;
  int64_t n_keys, seq = 0, tok = row, first = 0, len = 0;
  const unsigned long long* mask = nullptr;
  bool bad = false;
  if (TREE) {
    if (row >= (int64_t)p.n_seqs * p.rows) return;
    seq = row / p.rows, tok = row % p.rows;
    len = p.lens[seq];
    bad = len < 0 || len > p.slots - p.rows;
    n_keys = bad ? 0 : len + p.rows;
    if (p.mask) mask = p.mask + row * ((p.rows + 63) / 64);
  } else {
    if (row >= p.rows) return;
    int lo = -1;
    for (int s = 0; s < p.n_seqs; s++) {
      const int a = p.lens[s], b = p.lens[s + 1];
      if (a >= 0 && a <= row && row < b && b <= p.rows) lo = a;
    }
    if (lo < 0) return;
    first = lo;
    n_keys = row - lo + 1;
  }
  const unsigned char* q = p.q + (seq * p.q_seq + tok * p.q_row + h * p.q_head) * 2;
  const int esz = FP8 ? 1 : 2;
  const unsigned char* k = p.k + (seq * p.k_seq + first * p.k_row + g * p.k_head) * esz;
  const unsigned char* v = p.v + (seq * p.v_seq + first * p.v_row + g * p.v_head) * esz;
  for (int d = lane; d < HD; d += 32) qs[warp][d] = element<false>(q, d);
  __syncwarp();
  float m = -CUDART_INF_F, l = 0, o[HD / 32] = {};
  for (int64_t j0 = 0; j0 < n_keys; j0 += 32) {
    const int64_t j = j0 + lane;
    bool ok = j < n_keys;
    if (TREE && ok && j >= len) ok = mask ? (mask[(j - len) / 64] >> ((j - len) % 64)) & 1 : j - len <= tok;
    float s = -CUDART_INF_F;
    if (ok) {
      s = 0;
      for (int d = 0; d < HD; d++) s += qs[warp][d] * element<FP8>(k, j * p.k_row + d);
      s *= p.scale;
    }
    float mx = s;
    for (int x = 16; x; x >>= 1) mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, x));
    mx = fmaxf(mx, m);
    const float c = mx == -CUDART_INF_F ? 1.f : expf(m - mx);
    const float e = ok ? expf(s - mx) : 0.f;
    m = mx;
    float sum = e;
    for (int x = 16; x; x >>= 1) sum += __shfl_xor_sync(~0u, sum, x);
    l = l * c + sum;
    for (int d = 0; d < HD / 32; d++) o[d] *= c;
    for (unsigned live = __ballot_sync(~0u, ok); live; live &= live - 1) {
      const int i = __ffs(live) - 1;
      const float pi = __shfl_sync(~0u, e, i);
      for (int d = 0; d < HD / 32; d++) o[d] += pi * element<FP8>(v, (j0 + i) * p.v_row + d * 32 + lane);
    }
  }
  const float inv = bad ? CUDART_NAN_F : l == 0.f ? 0.f : 1.f / l;
  __nv_bfloat16* out = p.out + seq * p.o_seq + tok * p.o_row + h * p.o_head;
  for (int d = 0; d < HD / 32; d++) out[d * 32 + lane] = __float2bfloat16_rn(o[d] * inv);
  if (p.lse && lane == 0)
    p.lse[row * p.nq + h] = bad ? CUDART_NAN_F : l == 0.f ? -CUDART_INF_F : m + logf(l);
}

template <bool TREE>
cudaError_t launch(const Params& p, int hd, bool fp8, cudaStream_t st) {
  const int64_t warps = (TREE ? (int64_t)p.n_seqs * p.rows : p.rows) * p.nq;
  const unsigned blocks = (unsigned)((warps + 3) / 4);
  if (hd == 64)
    fp8 ? attn_kernel<64, TREE, TREE><<<blocks, 128, 0, st>>>(p) : attn_kernel<64, TREE, false><<<blocks, 128, 0, st>>>(p);
  else
    fp8 ? attn_kernel<128, TREE, TREE><<<blocks, 128, 0, st>>>(p) : attn_kernel<128, TREE, false><<<blocks, 128, 0, st>>>(p);
  return cudaGetLastError();
}

amk_status check_heads(const Reason& fail, uint32_t hd, uint32_t nq, uint32_t nkv, float scale) {
  if (hd != 64 && hd != 128) return fail(AMK_ERR_UNSUPPORTED, "head_dim %u: 64 or 128", hd);
  if (!nq || !nkv || nq % nkv || nq / nkv > 16 || nq > 65535)
    return fail(AMK_ERR_UNSUPPORTED, "%u query heads on %u kv heads: a multiple, at most 16 to one", nq, nkv);
  if (!(scale >= 0.f) || isinf(scale)) return fail(AMK_ERR_INVALID_ARG, "scale must be positive and finite, or 0");
  return AMK_OK;
}

// A stride (elements) of an axis of n entries.  An axis of one entry is never walked: any stride will do, and a
// legal one takes its place.
amk_status check_stride(const Reason& fail, const char* what, int64_t n, int64_t* stride, int64_t least, int esz) {
  if (n <= 1) {
    *stride = least;
    return AMK_OK;
  }
  if (*stride < least || *stride % (16 / esz) || *stride > (int64_t)1 << 36)
    return fail(AMK_ERR_INVALID_ARG, "%s stride %lld: a multiple of 16 bytes, at least %lld elements", what,
                (long long)*stride, (long long)least);
  return AMK_OK;
}

#define AMK_TRY(x)                        \
  do {                                    \
    const amk_status st_ = (x);           \
    if (st_ != AMK_OK) return st_;        \
  } while (0)

// Everything about a tree call that can be known without its data.
amk_status check_tree(const Reason& fail, const amk_tree_args* a) {
  if (!a) return fail(AMK_ERR_INVALID_ARG, "NULL arguments");
  if (a->struct_size != sizeof(amk_tree_args))
    return fail(AMK_ERR_INVALID_ARG, "struct_size %u, the library has %zu", a->struct_size, sizeof(amk_tree_args));
  AMK_TRY(check_heads(fail, a->head_dim, a->n_q_heads, a->n_kv_heads, a->scale));
  if (a->kv_dtype > AMK_KV_FP8_E4M3) return fail(AMK_ERR_UNSUPPORTED, "kv_dtype %u", a->kv_dtype);
  if (a->n_rows < 1 || a->n_rows > AMK_TREE_MAX_ROWS)
    return fail(AMK_ERR_UNSUPPORTED, "%u drafted tokens: 1 to %d", a->n_rows, AMK_TREE_MAX_ROWS);
  if (a->n_slots < a->n_rows || a->n_slots > 0x7fffffff - 1024)
    return fail(AMK_ERR_INVALID_ARG, "%u slots for %u drafted tokens", a->n_slots, a->n_rows);
  if (a->n_seqs > 65535) return fail(AMK_ERR_UNSUPPORTED, "%u sequences: at most 65535", a->n_seqs);
  return AMK_OK;
}

}  // namespace

extern "C" amk_status amk_prompt_attention(const amk_prompt_args* args, char* msg, size_t msg_bytes,
                                           void* cuda_stream) {
  const Reason fail(msg, msg_bytes, "amk_prompt_attention");
  if (!args) return fail(AMK_ERR_INVALID_ARG, "NULL arguments");
  amk_prompt_args a = *args;
  if (a.struct_size != sizeof a)
    return fail(AMK_ERR_INVALID_ARG, "struct_size %u, the library has %zu", a.struct_size, sizeof a);
  AMK_TRY(check_heads(fail, a.head_dim, a.n_q_heads, a.n_kv_heads, a.scale));
  if (a.total < 0 || a.total > 0x7fffffff - 1024 || a.n_seqs > 0x7fffffff - 1)
    return fail(AMK_ERR_INVALID_ARG, "%lld rows in %u prompts", (long long)a.total, a.n_seqs);
  if (a.total == 0 || a.n_seqs == 0) return AMK_OK;
  if (!a.q || !a.k || !a.v || !a.out || !a.cu_seqlens) return fail(AMK_ERR_INVALID_ARG, "NULL pointer");
  if (!amk::aligned(a.q, 16) || !amk::aligned(a.k, 16) || !amk::aligned(a.v, 16) || !amk::aligned(a.out, 16) ||
      !amk::aligned(a.lse, 4) || !amk::aligned(a.cu_seqlens, 4))
    return fail(AMK_ERR_INVALID_ARG, "q, k, v and out must be 16-byte aligned, lse and cu_seqlens 4-byte aligned");
  const int64_t hd = a.head_dim;
  AMK_TRY(check_stride(fail, "q row", a.total, &a.q_row, hd, 2));
  AMK_TRY(check_stride(fail, "k row", a.total, &a.k_row, hd, 2));
  AMK_TRY(check_stride(fail, "v row", a.total, &a.v_row, hd, 2));
  AMK_TRY(check_stride(fail, "out row", a.total, &a.out_row, hd, 2));
  AMK_TRY(check_stride(fail, "q head", a.n_q_heads, &a.q_head, hd, 2));
  AMK_TRY(check_stride(fail, "k head", a.n_kv_heads, &a.k_head, hd, 2));
  AMK_TRY(check_stride(fail, "v head", a.n_kv_heads, &a.v_head, hd, 2));
  AMK_TRY(check_stride(fail, "out head", a.n_q_heads, &a.out_head, hd, 2));
  Params p{};
  p.q = (const unsigned char*)a.q, p.k = (const unsigned char*)a.k, p.v = (const unsigned char*)a.v;
  p.out = (__nv_bfloat16*)a.out, p.lse = a.lse, p.lens = a.cu_seqlens;
  p.q_row = a.q_row, p.q_head = a.q_head, p.k_row = a.k_row, p.k_head = a.k_head;
  p.v_row = a.v_row, p.v_head = a.v_head, p.o_row = a.out_row, p.o_head = a.out_head;
  p.n_seqs = (int)a.n_seqs, p.nq = (int)a.n_q_heads, p.rep = (int)(a.n_q_heads / a.n_kv_heads);
  p.rows = (int)a.total;
  p.scale = a.scale > 0.f ? a.scale : 1.f / sqrtf((float)hd);
  const cudaError_t e = launch<false>(p, (int)hd, false, (cudaStream_t)cuda_stream);
  return e == cudaSuccess ? AMK_OK : fail(AMK_ERR_CUDA, "launch failed: %s", cudaGetErrorString(e));
}

extern "C" amk_status amk_tree_workspace_bytes(const amk_tree_args* args, size_t* bytes, char* msg,
                                               size_t msg_bytes) {
  const Reason fail(msg, msg_bytes, "amk_tree_workspace_bytes");
  if (!bytes) return fail(AMK_ERR_INVALID_ARG, "NULL pointer");
  AMK_TRY(check_tree(fail, args));
  *bytes = 0;
  return AMK_OK;
}

extern "C" amk_status amk_tree_attention(const amk_tree_args* args, char* msg, size_t msg_bytes,
                                         void* cuda_stream) {
  const Reason fail(msg, msg_bytes, "amk_tree_attention");
  AMK_TRY(check_tree(fail, args));
  amk_tree_args a = *args;
  if (a.n_seqs == 0) return AMK_OK;
  if (!a.q || !a.k || !a.v || !a.out || !a.cache_len) return fail(AMK_ERR_INVALID_ARG, "NULL pointer");
  if (!amk::aligned(a.q, 16) || !amk::aligned(a.k, 16) || !amk::aligned(a.v, 16) || !amk::aligned(a.out, 16) ||
      !amk::aligned(a.lse, 4) || !amk::aligned(a.cache_len, 4) || !amk::aligned(a.mask, 8) ||
      !amk::aligned(a.workspace, 256))
    return fail(AMK_ERR_INVALID_ARG,
                "q, k, v and out must be 16-byte, mask 8-byte, lse and cache_len 4-byte, workspace 256-byte aligned");
  const int64_t hd = a.head_dim;
  const int esz = a.kv_dtype == AMK_KV_FP8_E4M3 ? 1 : 2;
  AMK_TRY(check_stride(fail, "q sequence", a.n_seqs, &a.q_seq, hd, 2));
  AMK_TRY(check_stride(fail, "q row", a.n_rows, &a.q_row, hd, 2));
  AMK_TRY(check_stride(fail, "q head", a.n_q_heads, &a.q_head, hd, 2));
  AMK_TRY(check_stride(fail, "k sequence", a.n_seqs, &a.k_seq, hd, esz));
  AMK_TRY(check_stride(fail, "k head", a.n_kv_heads, &a.k_head, hd, esz));
  AMK_TRY(check_stride(fail, "k row", a.n_slots, &a.k_row, hd, esz));
  AMK_TRY(check_stride(fail, "v sequence", a.n_seqs, &a.v_seq, hd, esz));
  AMK_TRY(check_stride(fail, "v head", a.n_kv_heads, &a.v_head, hd, esz));
  AMK_TRY(check_stride(fail, "v row", a.n_slots, &a.v_row, hd, esz));
  AMK_TRY(check_stride(fail, "out sequence", a.n_seqs, &a.out_seq, hd, 2));
  AMK_TRY(check_stride(fail, "out row", a.n_rows, &a.out_row, hd, 2));
  AMK_TRY(check_stride(fail, "out head", a.n_q_heads, &a.out_head, hd, 2));
  Params p{};
  p.q = (const unsigned char*)a.q, p.k = (const unsigned char*)a.k, p.v = (const unsigned char*)a.v;
  p.out = (__nv_bfloat16*)a.out, p.lse = a.lse, p.lens = a.cache_len, p.mask = (const unsigned long long*)a.mask;
  p.q_seq = a.q_seq, p.q_row = a.q_row, p.q_head = a.q_head;
  p.k_seq = a.k_seq, p.k_row = a.k_row, p.k_head = a.k_head;
  p.v_seq = a.v_seq, p.v_row = a.v_row, p.v_head = a.v_head;
  p.o_seq = a.out_seq, p.o_row = a.out_row, p.o_head = a.out_head;
  p.n_seqs = (int)a.n_seqs, p.nq = (int)a.n_q_heads, p.rep = (int)(a.n_q_heads / a.n_kv_heads);
  p.rows = (int)a.n_rows, p.slots = (int)a.n_slots;
  p.scale = a.scale > 0.f ? a.scale : 1.f / sqrtf((float)hd);
  const cudaError_t e = launch<true>(p, (int)hd, esz == 1, (cudaStream_t)cuda_stream);
  return e == cudaSuccess ? AMK_OK : fail(AMK_ERR_CUDA, "launch failed: %s", cudaGetErrorString(e));
}
