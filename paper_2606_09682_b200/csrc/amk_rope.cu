// amk_norm_rope_append: heads normed, rotated and stored, one pass over new rows of q, k and v.
//
// Mathematics.  A lane holds eight elements i .. i+7 of a head and the eight i + hd/2 .. that they are rotated with, so that
// only the norm's sum crosses lanes.  The angle of pair i at position n is n theta^(-2i/hd); in turns, n f_i with
// f_i = theta^(-2i/hd) / 2 pi, it is made in 64 bits, its whole turns taken off, and only then rounded to fp32: off by 2^-26 of
// a turn, and near position 2^31 by 2^-24 more (theta >= 1).  The eight angles of a lane are those of every head of its token.
//
// Bound: HBM, each element once in and once out.  A warp takes the heads of one token, or, with few tokens, a share of them, and
// goes on to further tokens.  Heads come by asynchronous copies, seven steps ahead, into places of shared memory that each lane
// writes and reads alone: loads into registers cost the registers that keep enough bytes under way (8111 tokens of 32 + 8 + 8
// heads of 128, normed, 202 MB: 49.5 us with four steps in registers and scalar arithmetic, 40.5 with packed arithmetic and the
// weights in the rotation's factors, 37.8 with copies, 38.3 with the norms beyond fp32, 5.3 TB/s; without norms 35.3; a copy of as
// many bytes 31.7; into an 8-bit cache 38.6, 183 MB).
#include <cuda_bf16.h>
#include <math.h>

#include "amk.h"
#include "amk_op_launch.h"
#include "amk_op_util.h"
#include "amk_ptx.cuh"

namespace {

using amk::Reason;

struct RopeParams {
  const unsigned short *q, *k, *v;
  const uint4 *q_weight, *k_weight;
  const int* positions;
  const int64_t* slots;
  unsigned short *q_out, *k_out;
  void *k_cache, *v_cache;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, qo_row, qo_head, ko_row, ko_head;
  int64_t kc_seq, kc_head, kc_row, vc_seq, vc_head, vc_row;
  int64_t rows, all_slots;
  int nq, nkv;
  unsigned slots_of;               // rows of a cache
  int split;                       // warps that share a token
  float eps;
  double turns[64];                // f_i
};

// kAhead: places for steps on their way, one of them the step at hand (8 / 10 / 12 of them with 5 / 5 / 4 blocks an SM: 38.1 / 39.2 /
// 39.7 us; six blocks have too few registers: 56)
constexpr int kThreads = 128, kBlocks = 5, kAhead = 8;

__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {
  unsigned r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ unsigned pack_e4m3(float a, float b, float c, float d) {
  unsigned r;
  asm("{ .reg .b16 l, h; cvt.rn.satfinite.e4m3x2.f32 l, %2, %1; cvt.rn.satfinite.e4m3x2.f32 h, %4, %3; mov.b32 %0, {l, h}; }"
      : "=r"(r)
      : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
__device__ __forceinline__ void widen(float (&x)[8], const uint4& u) {
  const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; i++) x[2 * i] = amk::bf16_lo(w[i]), x[2 * i + 1] = amk::bf16_hi(w[i]);
}
__device__ __forceinline__ uint4 narrow(const float (&x)[8]) {
  return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}
// eight elements of a cache row from element i on
template <bool FP8>
__device__ __forceinline__ void store(void* cache, int64_t at, const float (&x)[8]) {
  if (FP8)
    *(uint2*)((unsigned char*)cache + at) = make_uint2(pack_e4m3(x[0], x[1], x[2], x[3]), pack_e4m3(x[4], x[5], x[6], x[7]));
  else
    *(uint4*)((unsigned short*)cache + at) = narrow(x);
}

// What a head's elements are multiplied with: z[i] = f (x lo_x[i] - y lo_y[i]), z[i + hd/2] = f (y hi_y[i] + x hi_x[i]) for x, y the
// elements i and i + hd/2 and f the norm's factor; two at a time.
struct Turn {
  uint64_t lo_x[4], lo_y[4], hi_y[4], hi_x[4];
  // from the cosines and sines and the weights (null: 1)
  __device__ __forceinline__ void set(const float (&c)[8], const float (&s)[8], const uint4* weight, int l, int half) {
    float a[8], b[8];
#pragma unroll
    for (int j = 0; j < 8; j++) a[j] = b[j] = 1.f;
    if (weight) widen(a, __ldg(weight + l)), widen(b, __ldg(weight + half + l));
#pragma unroll
    for (int j = 0; j < 4; j++) {
      lo_x[j] = amk::pair(c[2 * j] * a[2 * j], c[2 * j + 1] * a[2 * j + 1]);
      lo_y[j] = amk::pair(-s[2 * j] * b[2 * j], -s[2 * j + 1] * b[2 * j + 1]);
      hi_y[j] = amk::pair(c[2 * j] * b[2 * j], c[2 * j + 1] * b[2 * j + 1]);
      hi_x[j] = amk::pair(s[2 * j] * a[2 * j], s[2 * j + 1] * a[2 * j + 1]);
    }
  }
};
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ void widen2(uint64_t (&x)[4], const uint4& u) {
  const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; i++) x[i] = amk::pair(amk::bf16_lo(w[i]), amk::bf16_hi(w[i]));
}

__device__ __forceinline__ void copy_async(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(amk::smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 2) : "memory"); }

template <int HD, bool FP8>
__global__ void __launch_bounds__(kThreads, kBlocks) rope_kernel(const __grid_constant__ RopeParams p) {
  constexpr int kLanes = HD / 16, kGroups = 32 / kLanes, kOwn = 8 / kGroups;   // lanes of a head, heads of a step, angles a lane makes
  // what is on its way: every lane brings its own elements and reads them itself
  __shared__ uint4 held[kThreads / 32][kAhead][2][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane % kLanes, g = lane / kLanes, e = 8 * l;
  const int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + warp;
  const int64_t first = p.split == 1 ? w : w / p.split, next = (int64_t)gridDim.x * (kThreads / 32) / p.split;   // (split > 1: one row each)
  const int part = (int)(w - first * p.split);
  amk::wait_for_grid_before();
  // The steps of a token, kGroups heads each, queries, keys and values, in turn for the warps that share it.
  const int q_steps = (p.nq + kGroups - 1) / kGroups, k_steps = (p.nkv + kGroups - 1) / kGroups;
  const int steps = q_steps + (p.k_cache ? 2 : 1) * k_steps;
  int64_t asked_row = first;
  int asked = part, put = 0;                           // the next step to ask for, and where it goes
  const auto ask = [&]() {
    if (asked_row < p.rows) {
      const int kind = asked < q_steps ? 0 : asked < q_steps + k_steps ? 1 : 2;
      const int h = (asked - (kind == 0 ? 0 : kind == 1 ? q_steps : q_steps + k_steps)) * kGroups + g;
      if (h < (kind == 0 ? p.nq : p.nkv)) {
        const unsigned short* x = (kind == 0   ? p.q + asked_row * p.q_row + h * p.q_head
                                   : kind == 1 ? p.k + asked_row * p.k_row + h * p.k_head
                                               : p.v + asked_row * p.v_row + h * p.v_head) + e;
        copy_async(&held[warp][put][0][lane], x), copy_async(&held[warp][put][1][lane], x + HD / 2);
      }
      asked += p.split;
      if (asked >= steps) asked = part, asked_row += next;
    }
    copies_end();
    put = put + 1 == kAhead ? 0 : put + 1;
  };
  if (part >= steps) return;
#pragma unroll 1
  for (int i = 0; i < kAhead - 1; i++) ask();
  int get = 0;
#pragma unroll 1
  for (int64_t row = first; row < p.rows; row += next) {
    float c[8], s[8];
    {
      const double n = (double)p.positions[row];
      float cc[kOwn], ss[kOwn];
#pragma unroll
      for (int j = 0; j < kOwn; j++) {
        double t = n * p.turns[8 * l + g * kOwn + j];
        t -= rint(t);
        sincospif(2.f * (float)t, &ss[j], &cc[j]);
      }
#pragma unroll
      for (int j = 0; j < 8; j++) {
        c[j] = __shfl_sync(~0u, cc[j % kOwn], j / kOwn * kLanes + l);
        s[j] = __shfl_sync(~0u, ss[j % kOwn], j / kOwn * kLanes + l);
      }
    }
    int64_t kc = -1, vc = 0;                             // the token's row in the caches
    if (p.k_cache) {
      const int64_t slot = p.slots[row];
      if (slot >= 0 && slot < p.all_slots) {
        const int64_t seq = p.all_slots <= 0xffffffffll ? (unsigned)slot / p.slots_of : slot / p.slots_of;
        const int64_t at = slot - seq * p.slots_of;
        kc = seq * p.kc_seq + at * p.kc_row + e, vc = seq * p.vc_seq + at * p.vc_row + e;
      }
    }
    Turn turn;
    int step = part;
#pragma unroll 1
    for (int kind = 0; kind < 3; kind++) {               // queries, keys, values
      const int before = kind == 0 ? 0 : kind == 1 ? q_steps : q_steps + k_steps, end = kind == 0 ? q_steps : kind == 1 ? before + k_steps : steps;
      if (step >= end) continue;
      const int heads = kind == 0 ? p.nq : p.nkv;
      const uint4* weight = kind == 0 ? p.q_weight : p.k_weight;
      if (kind < 2) turn.set(c, s, weight, l, HD / 16);
      unsigned short* out = kind == 0 ? p.q_out + row * p.qo_row + e : kind == 1 && p.k_out ? p.k_out + row * p.ko_row + e : nullptr;
      const int64_t out_head = kind == 0 ? p.qo_head : p.ko_head;
      void* cache = kind == 0 || kc < 0 ? nullptr : kind == 1 ? p.k_cache : p.v_cache;
      const int64_t cache_at = kind == 1 ? kc : vc, cache_head = kind == 1 ? p.kc_head : p.vc_head;
#pragma unroll 1
      for (; step < end; step += p.split) {
        copies_wait();
        const int h = (step - before) * kGroups + g;
        uint4 lo = held[warp][get][0][lane], hi = held[warp][get][1][lane];
        get = get + 1 == kAhead ? 0 : get + 1;
        ask();                                           // (into the place of the step before this one)
        if (kind == 2) {
          if (h < heads && cache) {
            const int64_t at = cache_at + h * cache_head;
            if (FP8) {
              float x[8], y[8];
              widen(x, lo), widen(y, hi);
              store<FP8>(cache, at, x), store<FP8>(cache, at + HD / 2, y);
            } else {                                     // (the bits as they are)
              *(uint4*)((unsigned short*)cache + at) = lo, *(uint4*)((unsigned short*)cache + at + HD / 2) = hi;
            }
          }
          continue;
        }
        uint64_t x[4], y[4];
        widen2(x, lo), widen2(y, hi);
        if (weight) {
          uint64_t sums = mul2(x[0], x[0]), more = mul2(y[0], y[0]);
#pragma unroll
          for (int j = 1; j < 4; j++) sums = amk::fma2(x[j], x[j], sums), more = amk::fma2(y[j], y[j], more);
          float a, sum;
          amk::unpair(a, sum, amk::add2(sums, more));
          sum += a;
#pragma unroll
          for (int o = kLanes / 2; o; o /= 2) sum += __shfl_xor_sync(~0u, sum, o);
          const float mean = fmaf(sum, 1.f / HD, p.eps);
          float f = rsqrtf(mean);
          // Squares beyond fp32: once more, times 2^96 or 2^-70 (bf16's range is fp32's).  Of a head whose mean square is 2^128 or more an
          // element keeps its eight bits if it is 2^-71 at least, and smaller ones come out below bf16's least number, 2^-133, before the weight.
          if (!(mean > 1e-30f && mean < INFINITY)) {
            const float by = mean <= 1e-30f ? 0x1p96f : 0x1p-70f;
            const uint64_t by2 = amk::pair(by, by);
            sums = more = 0;
#pragma unroll
            for (int j = 0; j < 4; j++) x[j] = mul2(x[j], by2), y[j] = mul2(y[j], by2), sums = amk::fma2(x[j], x[j], sums), more = amk::fma2(y[j], y[j], more);
            amk::unpair(a, sum, amk::add2(sums, more));
            sum += a;
#pragma unroll
            for (int o = kLanes / 2; o; o /= 2) sum += __shfl_xor_sync(((1u << kLanes) - 1) << (lane & ~(kLanes - 1)), sum, o);
            f = rsqrtf(fmaf(sum, 1.f / HD, p.eps * by * by));
          }
          const uint64_t f2 = amk::pair(f, f);
#pragma unroll
          for (int j = 0; j < 4; j++) x[j] = mul2(x[j], f2), y[j] = mul2(y[j], f2);
        }
        if (h >= heads) continue;
        float z[8], t[8];
#pragma unroll
        for (int j = 0; j < 4; j++) {
          amk::unpair(z[2 * j], z[2 * j + 1], amk::fma2(x[j], turn.lo_x[j], mul2(y[j], turn.lo_y[j])));
          amk::unpair(t[2 * j], t[2 * j + 1], amk::fma2(y[j], turn.hi_y[j], mul2(x[j], turn.hi_x[j])));
        }
        if (out) {
          unsigned short* to = out + h * out_head;
          *(uint4*)to = narrow(z), *(uint4*)(to + HD / 2) = narrow(t);
        }
        if (cache) {
          const int64_t at = cache_at + h * cache_head;
          store<FP8>(cache, at, z), store<FP8>(cache, at + HD / 2, t);
        }
      }
    }
  }
}

// A stride (elements) of an axis of n entries, as the attentions': any will do for one entry.
amk_status check_stride(const Reason& fail, const char* what, int64_t n, int64_t* stride, int64_t least, int esz) {
  if (n <= 1) {
    *stride = least;
    return AMK_OK;
  }
  if (*stride < least || *stride % (16 / esz) || *stride > (int64_t)1 << 36)
    return fail(AMK_ERR_INVALID_ARG, "%s stride %lld: a multiple of 16 bytes, at least %lld elements", what, (long long)*stride,
                (long long)least);
  return AMK_OK;
}

}  // namespace

extern "C" amk_status amk_norm_rope_append(const amk_rope_args* args, char* msg, size_t msg_bytes, void* cuda_stream) {
  const Reason fail(msg, msg_bytes, "amk_norm_rope_append");
  if (!args) return fail(AMK_ERR_INVALID_ARG, "NULL arguments");
  amk_rope_args a = *args;
  if (a.struct_size != sizeof a)
    return fail(AMK_ERR_INVALID_ARG, "struct_size %u, the library has %zu", a.struct_size, sizeof a);
  if (a.reserved) return fail(AMK_ERR_INVALID_ARG, "reserved is %u, not 0", a.reserved);
  if (a.head_dim != 64 && a.head_dim != 128) return fail(AMK_ERR_UNSUPPORTED, "head_dim %u: 64 or 128", a.head_dim);
  if (!a.n_q_heads || !a.n_kv_heads || a.n_q_heads > 4096 || a.n_kv_heads > 4096)
    return fail(AMK_ERR_UNSUPPORTED, "%u query heads and %u kv heads: 1 to 4096", a.n_q_heads, a.n_kv_heads);
  if (a.kv_dtype > AMK_KV_FP8_E4M3) return fail(AMK_ERR_UNSUPPORTED, "kv_dtype %u", a.kv_dtype);
  if (!(a.eps >= 0.f) || isinf(a.eps)) return fail(AMK_ERR_INVALID_ARG, "eps must be at least 0 and finite");
  if (!(a.theta > 0.f) || isinf(a.theta)) return fail(AMK_ERR_INVALID_ARG, "theta must be positive and finite");
  if (a.rows < 0 || a.rows > 0x7fffffff - 1024) return fail(AMK_ERR_INVALID_ARG, "%lld rows", (long long)a.rows);
  const bool cached = a.k_cache != nullptr;
  if (cached != (a.v_cache != nullptr)) return fail(AMK_ERR_INVALID_ARG, "k_cache and v_cache: both or neither");
  if (cached && (!a.n_seqs || !a.n_slots || a.n_slots > 0x7fffffff))
    return fail(AMK_ERR_INVALID_ARG, "%u caches of %u rows", a.n_seqs, a.n_slots);
  if (a.rows == 0) return AMK_OK;
  if (!a.q || !a.k || !a.positions || !a.q_out || (cached && (!a.v || !a.slots))) return fail(AMK_ERR_INVALID_ARG, "NULL pointer");
  const void* vec[] = {a.q, a.k, a.v, a.q_weight, a.k_weight, a.q_out, a.k_out, a.k_cache, a.v_cache};
  for (const void* p : vec)
    if (!amk::aligned(p, 16)) return fail(AMK_ERR_INVALID_ARG, "q, k, v, weights, outputs and caches must be 16-byte aligned");
  if (!amk::aligned(a.positions, 4) || !amk::aligned(a.slots, 8))
    return fail(AMK_ERR_INVALID_ARG, "positions must be 4-byte, slots 8-byte aligned");
  const int64_t hd = a.head_dim, nq = a.n_q_heads, nkv = a.n_kv_heads;
  const int esz = a.kv_dtype == AMK_KV_FP8_E4M3 ? 1 : 2;
  struct { const char* what; int64_t n, *stride; int esz; bool used; } strides[] = {
      {"q row", a.rows, &a.q_row, 2, true}, {"q head", nq, &a.q_head, 2, true},
      {"k row", a.rows, &a.k_row, 2, true}, {"k head", nkv, &a.k_head, 2, true},
      {"v row", a.rows, &a.v_row, 2, cached}, {"v head", nkv, &a.v_head, 2, cached},
      {"q_out row", a.rows, &a.qo_row, 2, true}, {"q_out head", nq, &a.qo_head, 2, true},
      {"k_out row", a.rows, &a.ko_row, 2, a.k_out != nullptr}, {"k_out head", nkv, &a.ko_head, 2, a.k_out != nullptr},
      {"k_cache sequence", a.n_seqs, &a.kc_seq, esz, cached}, {"k_cache head", nkv, &a.kc_head, esz, cached},
      {"k_cache row", a.n_slots, &a.kc_row, esz, cached}, {"v_cache sequence", a.n_seqs, &a.vc_seq, esz, cached},
      {"v_cache head", nkv, &a.vc_head, esz, cached}, {"v_cache row", a.n_slots, &a.vc_row, esz, cached}};
  for (const auto& s : strides)
    if (s.used) {
      const amk_status st = check_stride(fail, s.what, s.n, s.stride, hd, s.esz);
      if (st != AMK_OK) return st;
    }
  if ((a.q_out == a.q && (a.qo_row != a.q_row || a.qo_head != a.q_head)) || (a.k_out == a.k && (a.ko_row != a.k_row || a.ko_head != a.k_head)))
    return fail(AMK_ERR_INVALID_ARG, "q_out is q or k_out is k, but at other strides");
  RopeParams p{};
  p.q = (const unsigned short*)a.q, p.k = (const unsigned short*)a.k, p.v = (const unsigned short*)a.v;
  p.q_weight = (const uint4*)a.q_weight, p.k_weight = (const uint4*)a.k_weight;
  p.positions = a.positions, p.slots = a.slots;
  p.q_out = (unsigned short*)a.q_out, p.k_out = (unsigned short*)a.k_out, p.k_cache = a.k_cache, p.v_cache = a.v_cache;
  p.q_row = a.q_row, p.q_head = a.q_head, p.k_row = a.k_row, p.k_head = a.k_head, p.v_row = a.v_row, p.v_head = a.v_head;
  p.qo_row = a.qo_row, p.qo_head = a.qo_head, p.ko_row = a.ko_row, p.ko_head = a.ko_head;
  p.kc_seq = a.kc_seq, p.kc_head = a.kc_head, p.kc_row = a.kc_row, p.vc_seq = a.vc_seq, p.vc_head = a.vc_head, p.vc_row = a.vc_row;
  p.rows = a.rows, p.all_slots = cached ? (int64_t)a.n_seqs * a.n_slots : 0, p.slots_of = a.n_slots;
  p.nq = (int)nq, p.nkv = (int)nkv;
  p.eps = a.eps;
  const long double step = powl((long double)a.theta, -2.0L / hd);
  long double f = 0.15915494309189533576888376337251436L;               // 1 / 2 pi
  for (int i = 0; i < hd / 2; i++, f *= step) p.turns[i] = (double)f;
  // a token's heads over several warps until there are 32 warps for each SM
  const int64_t group = 512 / hd, kv_steps = (nkv + group - 1) / group;
  const int64_t steps = (nq + group - 1) / group + kv_steps * (cached ? 2 : 1), want = (32ll * amk::multiprocessors() + a.rows - 1) / a.rows;
  p.split = (int)(steps < want ? steps : want);
  // what is resident at once; a warp goes on to further rows
  const int64_t most = kBlocks * (int64_t)amk::multiprocessors(), need = (a.rows * p.split + kThreads / 32 - 1) / (kThreads / 32);
  const int64_t blocks = p.split > 1 || need < most ? need : most;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  const auto kernel = hd == 64 ? (esz == 1 ? rope_kernel<64, true> : rope_kernel<64, false>)
                               : (esz == 1 ? rope_kernel<128, true> : rope_kernel<128, false>);
  const cudaError_t e = amk::launch_early(kernel, dim3((unsigned)blocks), kThreads, 0, 1, st, p);
  return e == cudaSuccess ? AMK_OK : fail(AMK_ERR_CUDA, "launch failed: %s", cudaGetErrorString(e));
}
