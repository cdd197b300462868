// amk_verify_draft: drafted tokens accepted or rejected against the target's probabilities, and the next token drawn.
//
// Mathematics.  With e(t) = exp((x(t) - m) / T) for a row's logits x and maximum m, the weights of the walk's state are
//   v_0 = e,  v_{k+1} = max(v_k / S_k - q, 0),  S_k = sum of v_k
// after k rejected children (guesses: v_k is e without the rejected tokens), r = v_k / S_k.  A child is accepted if
// u q < v_k / S_k; the token drawn is the first whose running sum of v_k is more than u[0] S_k.
//
// Which rows the walk reaches is known only as it goes, and each needs its S_0.  So a first kernel takes the maximum and the sum of
// every row in 32 bits, all rows at once at the memory's rate, and a second one, a cluster of blocks for each sequence, walks
// on those numbers alone (a cluster that takes its rows' sums itself, in one launch: guesses for one sequence of 6 rows of 128256 15.3
// us, so 11.9; for eight of them 28.8 and 22.5): a decision nearer than their error (kNear) is taken again with the sum in 64 bits.  Only a row where
// a child is rejected or a token drawn is read again (from L2), in 64 bits throughout: the border between two tokens of a
// vocabulary of 10^5 lies within the error of 32 bits in one draw of a hundred.
//
// Bound: HBM in the first kernel (each row once: 24.6 MB in about 8 us); in the second latency.  Of one sequence of 6 rows of 128256 both
// take 6.5 us with a greedy answer; a draw adds 3.7 (a pass over the row, the sums' exchange, the search), an accepted child 1, a
// rejected guess 1 (the draw's pass is over what they leave), the first child that is rejected with its probabilities 5.1 and each
// further one 2.5 (a pass, for the state's sum, and its exchange).  Of eight sequences all but the first kernel take twice as long:
// their 128 blocks in clusters of 16 behave as two waves (four sequences of the measured chains 14.1 us, eight 26.9, nine 32, sixteen
// 39).  From 75 sequences on each has one block, which keeps 8192 tokens and makes the weights of the others anew in every pass: 80
// sequences 243 us.  (6 sequences of 26 rows, 16 bits: 30 us.  With verdicts, states and sums made anew at each step and clusters of
// 8, the chains of eight 34 us and these 69.)
#include <cuda_runtime.h>
#include <math_constants.h>

#include <atomic>

#include "amk.h"
#include "amk_op_launch.h"
#include "amk_op_util.h"
#include "amk_ptx.cuh"

namespace {

using namespace amk;

constexpr int kThreads = 512, kWarps = kThreads / 32;    // the walk's
constexpr int kStatThreads = 256, kStatWarps = kStatThreads / 32, kLoads = 4;   // the first kernel's: 16 KB of logits a block
constexpr float kLog2e = 1.4426950408889634f;
// A row's sum in 32 bits.  An exponent y = (x - m) log2 e / T is rounded four times (the difference, log2 e, the quotient, the product):
// off by 2^-22.3 |y|, its power by 2^-22.8 |y| of itself; weighed by the powers, |y| is at most the logarithm of the vocabulary, 31:
// 2^-17.8.  Two powers a term: 2^-21 together.  A thread adds 32 terms, and then come eight steps of a tree: 40 2^-24; parts are added
// up in 64 bits, however many they are.  In all less than 2^-17 (of 10^5 tokens 2^-17.4).
constexpr double kNear = 1.0 / 65536;

struct Stat {
  float m, s;                                          // a row's (or a part's) maximum, and sum of exp((x - m) / T)
  int first;                                           // temperature 0: the first index of the maximum
  int pad;
};

struct VerifyParams {
  const void* logits;
  const float* draft;
  const int *tokens, *parents;
  const float *u, *temperature;
  const int* cache_len;
  int *count, *keep, *token;
  Stat* stats;                                         // [n_seqs * rows][parts]
  int64_t l_seq, l_row, d_seq, d_row;
  int rows, vocab, parts, cluster;
};

__device__ __forceinline__ float load(const float* x, int64_t i) { return __ldg(x + i); }
__device__ __forceinline__ float load(const unsigned short* x, int64_t i) { return __uint_as_float((unsigned)__ldg(x + i) << 16); }
template <class T>
__device__ __forceinline__ float element(const uint4& u, int k) {
  const unsigned w = sizeof(T) == 4 ? (&u.x)[k] : (&u.x)[k / 2];
  return sizeof(T) == 4 ? __uint_as_float(w) : k & 1 ? bf16_hi(w) : bf16_lo(w);
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

// ---- the rows' maxima and sums ----------------------------------------------------------------------------------
// A block has 16 KB of a row, counted from the 16-byte boundary at or in front of its first logit, and holds them in registers.
template <class T>
__global__ void __launch_bounds__(kStatThreads, 8) stats_kernel(const VerifyParams p) {
  constexpr int kVec = 16 / sizeof(T), kPart = kStatThreads * kLoads * kVec;
  __shared__ float red[kStatWarps];
  __shared__ int red_i[kStatWarps];
  const int64_t r = blockIdx.x / p.parts;
  const int part = (int)(blockIdx.x - r * p.parts);
  const int64_t s = r / p.rows, i = r - s * p.rows;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const T* x = (const T*)p.logits + s * p.l_seq + i * p.l_row;
  const int skew = (int)((uintptr_t)x / sizeof(T) % kVec);
  const uint4* x4 = (const uint4*)(x - skew);
  const int begin = part * kPart + (int)threadIdx.x * kVec - skew;         // this thread's first place, as an index of the row
  wait_for_grid_before();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const float t = p.temperature ? p.temperature[s] : 1.f;
  uint4 v[kLoads];
  float m = -CUDART_INF_F;
  const unsigned nothing = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;     // -infinity
#pragma unroll
  for (int j = 0; j < kLoads; j++) {
    const int at = begin + j * kStatThreads * kVec;
    v[j] = make_uint4(nothing, nothing, nothing, nothing);
    if (at >= 0 && at + kVec <= p.vocab) {
      v[j] = __ldg(x4 + (at + skew) / kVec);
    } else if (at > -kVec && at < p.vocab) {
#pragma unroll
      for (int k = 0; k < kVec; k++)
        if (at + k >= 0 && at + k < p.vocab) {
          if (sizeof(T) == 4) {
            (&v[j].x)[k] = __float_as_uint(load(x, at + k));
          } else {
            const unsigned w = __float_as_uint(load(x, at + k)) >> 16;
            (&v[j].x)[k / 2] = k & 1 ? ((&v[j].x)[k / 2] & 0xffffu) | w << 16 : ((&v[j].x)[k / 2] & 0xffff0000u) | w;
          }
        }
    }
  }
#pragma unroll
  for (int j = 0; j < kLoads; j++)
#pragma unroll
    for (int k = 0; k < kVec; k += 2) m = max3_nan(m, element<T>(v[j], k), element<T>(v[j], k + 1));
#pragma unroll
  for (int o = 16; o; o /= 2) m = max_nan(m, __shfl_xor_sync(~0u, m, o));
  if (lane == 0) red[warp] = m;
  __syncthreads();
  m = red[lane & (kStatWarps - 1)];
#pragma unroll
  for (int o = kStatWarps / 2; o; o /= 2) m = max_nan(m, __shfl_xor_sync(~0u, m, o));
  m = __shfl_sync(~0u, m, 0);
  float sum = 0.f;
  int first = 0x7fffffff;
  if (t > 0.f) {
    if (m > -CUDART_INF_F) {
      const float f = fminf(kLog2e / t, 3e38f);        // (a difference of 0 stays 0)
#pragma unroll
      for (int j = 0; j < kLoads; j++)
#pragma unroll
        for (int k = 0; k < kVec; k++) sum += exp2_fast((element<T>(v[j], k) - m) * f);
    }
  } else {
#pragma unroll
    for (int j = kLoads - 1; j >= 0; j--)
#pragma unroll
      for (int k = kVec - 1; k >= 0; k--)
        if (element<T>(v[j], k) == m) first = begin + j * kStatThreads * kVec + k;
  }
#pragma unroll
  for (int o = 16; o; o /= 2) {
    sum += __shfl_xor_sync(~0u, sum, o);
    first = min(first, __shfl_xor_sync(~0u, first, o));
  }
  __syncthreads();
  if (lane == 0) red[warp] = sum, red_i[warp] = first;
  __syncthreads();
  if (warp == 0) {
    sum = lane < kStatWarps ? red[lane] : 0.f, first = lane < kStatWarps ? red_i[lane] : 0x7fffffff;
#pragma unroll
    for (int o = kStatWarps / 2; o; o /= 2) {
      sum += __shfl_xor_sync(~0u, sum, o);
      first = min(first, __shfl_xor_sync(~0u, first, o));
    }
    if (lane == 0) p.stats[blockIdx.x] = Stat{m, sum, first, 0};
  }
}

// ---- the walk ---------------------------------------------------------------------------------------------------
__device__ __forceinline__ void st_remote(const void* mine, unsigned rank, double x) {
  asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(remote(mine, rank)), "d"(x) : "memory");
}

constexpr int kMaxRows = AMK_TREE_MAX_ROWS, kMaxCluster = 16;
enum { kReject, kAccept, kClose };
constexpr int kHeld = 16;                              // weights of a row that a thread keeps in registers

struct Walk {
  int parent[kMaxRows], token[kMaxRows];
  float x[kMaxRows], q[kMaxRows];                      // the token's logit and drafted probability in its parent's rows
  double e[kMaxRows], uq[kMaxRows];                    // its e there, and the number times the probability
  int verdict[kMaxRows];                               // as a first child: accepted, rejected, or not to be said in 32 bits
  float m[kMaxRows], s[kMaxRows];                      // the rows' statistics
  int first[kMaxRows];
  double inv[kMaxRows];                                // 1 / S_0 .. 1 / S_{k-1}
  int out[kMaxRows];                                   // guesses: the rejected tokens
  double run[kWarps];                                  // sums of the warps' runs of this block's share of the row
  double block[2][kMaxCluster];                        // the blocks' sums, of the last pass and the one before it
  double roots[32];                                    // 2^(j / 32)
  int over[kWarps], positive[kWarps];                  // in the search: the first place past the number, the last with a weight
};

// e^y for y <= 0, off by less than 2^-43 of itself: y = (n + f) ln 2 / 32 with |f| <= 1/2, 2^(n / 32) from the table and an exponent,
// the rest by its Taylor series (r^6 / 720 < 2^-48; r is off by 2^-53 |y|).  Below e^-700: 0.
__device__ __forceinline__ double exp_below(double y, const double* roots) {
  const double magic = 6755399441055744.0;             // 1.5 * 2^52: leaves the integer in the low word
  const double t = fma(y, 46.166241308446828384, magic);
  const int n = __double2loint(t);
  const double r = fma(t - magic, -0.021660849392498290195, y);
  double v = fma(r, 1.0 / 120, 1.0 / 24);
  v = fma(v, r, 1.0 / 6), v = fma(v, r, 0.5), v = fma(v, r, 1.0), v = fma(v, r, 1.0);
  const double w = roots[n & 31];
  v *= __hiloint2double(__double2hiint(w) + (int)((unsigned)(n >> 5) << 20), __double2loint(w));
  return y < -700.0 ? 0.0 : v;
}

// From the weights of one state to those of the next one, in place; token i + 32 j's is v[j].
template <int N>
__device__ __forceinline__ void reject(double (&v)[N], const float (&q)[N], const Walk& w, bool drafted, int j0, int i) {
  if (drafted) {
    const double inv = w.inv[j0];
#pragma unroll
    for (int j = 0; j < N; j++) {
      const double x = fma(v[j], inv, -(double)q[j]);
      v[j] = __double2hiint(x) < 0 ? 0.0 : x;
    }
  } else {
    const int out = w.out[j0];
#pragma unroll
    for (int j = 0; j < N; j++)
      if (i + 32 * j == out) v[j] = 0.0;
  }
}

__device__ __forceinline__ double shfl_xor(double x, int o) { return __shfl_xor_sync(~0u, x, o); }

template <class T>
__global__ void __launch_bounds__(kThreads, 1) walk_kernel(const VerifyParams p) {
  extern __shared__ __align__(16) unsigned char smem[];
  Walk& w = *(Walk*)smem;
  const int rank = p.cluster == 1 ? 0 : (int)cluster_rank();
  const int64_t seq = blockIdx.x / p.cluster;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const T* logits = (const T*)p.logits + seq * p.l_seq;
  const float* draft = p.draft ? p.draft + seq * p.d_seq : nullptr;
  if (threadIdx.x < 32) w.roots[threadIdx.x] = exp2(threadIdx.x / 32.0);
  wait_for_grid_before();
  const float t = p.temperature ? p.temperature[seq] : 1.f;
  const int* tokens = p.tokens + seq * p.rows;
  const int* parents = p.parents ? p.parents + seq * p.rows : nullptr;
  for (int i = threadIdx.x; i < p.rows; i += kThreads) {
    int parent = parents && i ? parents[i] : i - 1;
    const int tok = i ? tokens[i] : -1;
    const float u = p.u[seq * p.rows + i];
    if (parent >= i || tok < 0 || tok >= p.vocab) parent = -1;
    w.parent[i] = parent, w.token[i] = tok;
    if (parent >= 0) {
      w.x[i] = load(logits + parent * p.l_row, tok);
      w.q[i] = draft ? __ldg(draft + parent * p.d_row + tok) : 1.f;
      w.uq[i] = (double)u * (double)w.q[i];
    }
  }
  // the rows' parts, a lane each
  const float f = fminf(kLog2e / t, 3e38f);
  for (int i = warp; i < p.rows; i += kWarps) {
    const Stat* st = p.stats + (seq * p.rows + i) * p.parts;
    Stat a{-CUDART_INF_F, 0.f, 0x7fffffff, 0};
    if (lane < p.parts) a = st[lane];
    float m = a.m;
    for (int j = lane + 32; j < p.parts; j += 32) m = max_nan(m, st[j].m);
#pragma unroll
    for (int o = 16; o; o /= 2) m = max_nan(m, __shfl_xor_sync(~0u, m, o));
    double s = 0.0;
    int first = 0x7fffffff;
    for (int j = lane;;) {
      if (a.m > -CUDART_INF_F) s += (double)(a.s * exp2_fast((a.m - m) * f));
      if (a.m == m) first = min(first, a.first);
      if ((j += 32) >= p.parts) break;
      a = st[j];
    }
#pragma unroll
    for (int o = 16; o; o /= 2) s += __shfl_xor_sync(~0u, s, o);
    first = __reduce_min_sync(~0u, first);
    if (lane == 0) w.m[i] = m, w.s[i] = (float)s, w.first[i] = first;
  }
  if (p.cluster == 1) __syncthreads();
  else cluster_sync();                                 // (also: the other blocks have begun and can be written to)
  const bool greedy = t == 0.f, legal = t >= 0.f && t < CUDART_INF_F;
  const double inv_t = 1.0 / (double)t;
  const bool rough = t < 1e-37f || t > 1e30f;          // log2 e / t or x - m may be beyond fp32: the sums in 32 bits say nothing
  for (int i = threadIdx.x; i < p.rows; i += kThreads) {
    const int parent = w.parent[i];
    if (parent < 0) continue;
    const double uq = w.uq[i];
    if (greedy) {
      w.verdict[i] = w.token[i] == w.first[parent] && uq < 1.0 ? kAccept : kReject;
    } else {
      const double y = ((double)w.x[i] - (double)w.m[parent]) * inv_t, s = (double)w.s[parent];
      double e = exp_below(y, w.roots);
      if (e == 0.0) e = exp(y);
      w.e[i] = e;
      w.verdict[i] = !rough && fabs(uq * s - e) > kNear * e ? (uq * s < e ? kAccept : kReject) : kClose;
    }
  }
  __syncthreads();
  const int len = p.cache_len ? p.cache_len[seq] : 0;
  const bool tells = rank == 0 && threadIdx.x == 0;
  int* keep = p.keep + seq * p.rows;
  if (tells) keep[0] = len;

  // this block's share of a row, in runs for its warps
  const int share = (p.vocab + p.cluster - 1) / p.cluster, begin = min(rank * share, p.vocab), end = min(begin + share, p.vocab);
  const int run = (share + kWarps - 1) / kWarps, from = begin + warp * run, to = min(from + run, end);
  int at = 0, kept = 1, k = 0, parity = 0;
  bool summed = false;                                 // S_k is known in 64 bits, and the runs' sums are those of this state
  bool has_q = false;                                  // what this thread holds of the row: its drafted probabilities,
  int held_k = -1;                                     // ... and the weights of this state (-1: none)
  double held[kHeld];
  float held_q[kHeld];
  double total = 0.0;                                  // S_k
  double gone = 0.0;                                   // guesses: what the rejected tokens had of the 32-bit sum
  const T* x = logits;
  const float* q = draft;
  double m = 0.0;
  const auto e_of = [&](float xt) { return exp_below(((double)xt - m) * inv_t, w.roots); };
  const auto valid = [&](int node) { return legal && fabsf(w.m[node]) < CUDART_INF_F; };
  const auto enter = [&](int node) {
    at = node, k = 0, summed = has_q = false, held_k = -1, gone = 0.0;
    x = logits + node * p.l_row, m = (double)w.m[node];
    if (draft) q = draft + node * p.d_row;
  };
  // The sum of the state's weights over the row: the runs' and the blocks' sums stay in shared memory.  The whole cluster.
  // A thread keeps the first of its run; what is behind them (vocabularies beyond 8192 a block) is read again each time.
  const auto pass = [&](bool want_q) {
    const int i0 = from + lane;
    float xt[kHeld];
    const bool anew = held_k < 0 || held_k > k;
    if (anew) {
#pragma unroll
      for (int j = 0; j < kHeld; j++) xt[j] = i0 + 32 * j < to ? load(x, i0 + 32 * j) : -CUDART_INF_F;
    }
    if (want_q && !has_q) {
#pragma unroll
      for (int j = 0; j < kHeld; j++) held_q[j] = i0 + 32 * j < to ? __ldg(q + i0 + 32 * j) : 0.f;
      has_q = true;
    }
    if (anew) {
#pragma unroll
      for (int j = 0; j < kHeld; j++) held[j] = e_of(xt[j]);
      held_k = 0;
    }
#pragma unroll 1
    for (; held_k < k; held_k++) reject(held, held_q, w, draft, held_k, i0);
    double part[4] = {};
#pragma unroll
    for (int j = 0; j < kHeld; j++) part[j & 3] += held[j];
    constexpr int kAhead = 8;
#pragma unroll 1
    for (int i = i0 + 32 * kHeld; i < to; i += 32 * kAhead) {
      float a[kAhead], b[kAhead];
      double v[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; j++) {
        const bool in = i + 32 * j < to;
        a[j] = in ? load(x, i + 32 * j) : -CUDART_INF_F;
        b[j] = in && draft && k ? __ldg(q + i + 32 * j) : 0.f;
      }
#pragma unroll
      for (int j = 0; j < kAhead; j++) v[j] = e_of(a[j]);
#pragma unroll 1
      for (int n = 0; n < k; n++) reject(v, b, w, draft, n, i);
#pragma unroll
      for (int j = 0; j < kAhead; j++) part[j & 3] += v[j];
    }
    double sum = (part[0] + part[1]) + (part[2] + part[3]);
#pragma unroll
    for (int o = 16; o; o /= 2) sum += shfl_xor(sum, o);
    __syncthreads();                                   // (the last pass's sums have been read)
    if (lane == 0) w.run[warp] = sum;
    __syncthreads();
    parity ^= 1;
    if (warp == 0) {
      double all = lane < kWarps ? w.run[lane] : 0.0;
#pragma unroll
      for (int o = 16; o; o /= 2) all += shfl_xor(all, o);
      if (p.cluster == 1) w.block[parity][0] = all;
      else if (lane < p.cluster) st_remote(&w.block[parity][rank], lane, all);
    }
    if (p.cluster == 1) __syncthreads();
    else cluster_sync();
    double all = lane < p.cluster ? w.block[parity][lane] : 0.0;
#pragma unroll
    for (int o = 16; o; o /= 2) all += shfl_xor(all, o);
    return all;
  };
  // S_k for the state at hand; one without any weight is not one: the state before it stays
  const auto sum_up = [&](bool want_q) {
    while (!summed) {
      total = pass(want_q);
      if (total > 0.0 || k == 0) summed = true;
      else --k;
    }
  };
  enter(0);
  bool ok = valid(0);
  for (int i = 1; ok;) {
    // the next child
    for (; i < p.rows; i += 32) {
      const unsigned hit = __ballot_sync(~0u, i + lane < p.rows && w.parent[min(i + lane, p.rows - 1)] == at);
      if (hit) {
        i += __ffs(hit) - 1;
        break;
      }
    }
    if (i >= p.rows) break;
    const int c = i++;
    int verdict = w.verdict[c];
    if (!greedy && (k || summed)) {
      verdict = kClose;
      if (!draft && !summed && !rough) {               // a guess behind rejected ones: by what these leave of the 32-bit sum
        const double e = w.e[c], s32 = (double)w.s[at], s = s32 - gone;
        bool before = false;
        for (int j = 0; j < k; j++) before |= w.out[j] == w.token[c];
        if (before) verdict = kReject;
        else if (s > s32 / 1024 && fabs(w.uq[c] * s - e) * s > kNear * e * s32) verdict = w.uq[c] * s < e ? kAccept : kReject;
      }
    }
    if (verdict == kClose) {
      sum_up(draft && k);
      double v[1] = {w.e[c]};
      const float qt[1] = {w.q[c]};
      for (int n = 0; n < k; n++) reject(v, qt, w, draft, n, w.token[c]);
      verdict = w.uq[c] * total < v[0] ? kAccept : kReject;
    }
    const bool accept = verdict == kAccept;
    if (accept) {
      if (tells) keep[kept] = len + c;
      kept++;
      enter(c);
      ok = valid(c);
    } else if (!greedy) {
      if (draft) {
        sum_up(true);
        __syncthreads();
        if (threadIdx.x == 0) w.inv[k] = 1.0 / total;
      } else {
        bool before = false;
        for (int j = 0; j < k; j++) before |= w.out[j] == w.token[c];
        if (!before) gone += w.e[c];
        __syncthreads();
        if (threadIdx.x == 0) w.out[k] = w.token[c];
      }
      __syncthreads();
      ++k;
      summed = false;
    }
  }
  if (tells) p.count[seq] = kept;
  if (rank == 0)
    for (int i = kept + threadIdx.x; i < p.rows; i += kThreads) keep[i] = -1;
  if (!ok || greedy) {
    if (tells) p.token[seq] = ok ? w.first[at] : -1;
    return;
  }
  // the token: the block, the run and the place where the running sum passes the given number
  sum_up(draft && k);
  const double want = (double)p.u[seq * p.rows] * total;
  double before = 0.0;
  // the first of n sums with which the running sum passes the number, or the last with a weight; `before`: what is in front of it
  const auto find = [&](const double* sums, int n) {
    const double b = lane < n ? sums[lane] : 0.0;
    double c = b;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double y = __shfl_up_sync(~0u, c, o);
      if (lane >= o) c += y;
    }
    const unsigned over = __ballot_sync(~0u, b > 0.0 && before + c > want), some = __ballot_sync(~0u, b > 0.0);
    const int j = over ? __ffs(over) - 1 : some ? 31 - __clz(some) : 0;
    const double in_front = __shfl_sync(~0u, c, j ? j - 1 : 0);
    if (j) before += in_front;
    return j;
  };
  if (rank != find(w.block[parity], p.cluster)) return;
  const int mine = find(w.run, kWarps), first = begin + mine * run, behind = min(first + run, end);
  __syncthreads();
  // all warps over the one run, 512 places at a time
  int last_positive = -1;
  for (int i0 = first; i0 < behind; i0 += kThreads) {
    const int i = i0 + threadIdx.x;
    double v[1] = {i < behind ? e_of(load(x, i)) : 0.0};
    const float qt[1] = {i < behind && draft && k ? __ldg(q + i) : 0.f};
    for (int n = 0; n < k; n++) reject(v, qt, w, draft, n, i);
    double c = v[0];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double y = __shfl_up_sync(~0u, c, o);
      if (lane >= o) c += y;
    }
    __syncthreads();
    if (lane == 31) w.run[warp] = c;
    __syncthreads();
    double ahead = lane < kWarps ? w.run[lane] : 0.0;
#pragma unroll
    for (int o = 1; o < kWarps; o <<= 1) {
      const double y = __shfl_up_sync(~0u, ahead, o);
      if (lane >= o) ahead += y;
    }
    const double all = __shfl_sync(~0u, ahead, kWarps - 1);
    ahead = __shfl_sync(~0u, ahead, warp ? warp - 1 : 0);
    ahead = warp ? before + ahead : before;
    const unsigned over = __ballot_sync(~0u, v[0] > 0.0 && ahead + c > want), some = __ballot_sync(~0u, v[0] > 0.0);
    if (lane == 0) {
      w.over[warp] = over ? i0 + warp * 32 + __ffs(over) - 1 : -1;
      w.positive[warp] = some ? i0 + warp * 32 + 31 - __clz(some) : -1;
    }
    __syncthreads();
    int hit = -1;
    for (int j = 0; j < kWarps; j++) {
      if (hit < 0) hit = w.over[j];
      if (w.positive[j] >= 0) last_positive = w.positive[j];
    }
    if (hit >= 0) {
      if (threadIdx.x == 0) p.token[seq] = hit;
      return;
    }
    before += all;
  }
  if (threadIdx.x == 0) p.token[seq] = last_positive;
}

// ---- host -------------------------------------------------------------------------------------------------------
// The walk's shared memory and clusters of 16 blocks, allowed once on each device; *room: whether such a cluster can run at all.
template <class T>
cudaError_t allow(bool* room) {
  static std::atomic<unsigned long long> done{0}, large{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
  if (!(done.load(std::memory_order_acquire) & bit)) {
    e = cudaFuncSetAttribute(walk_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(Walk));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(walk_kernel<T>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = kMaxCluster, at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(kMaxCluster), cfg.blockDim = dim3(kThreads), cfg.dynamicSmemBytes = sizeof(Walk);
    cfg.attrs = &at, cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, walk_kernel<T>, &cfg) != cudaSuccess) (void)cudaGetLastError();
    else if (n > 0) large.fetch_or(bit, std::memory_order_release);
    done.fetch_or(bit, std::memory_order_release);
  }
  *room = large.load(std::memory_order_acquire) & bit;
  return cudaSuccess;
}

// parts of a row; its first logit may stand up to seven places behind the 16-byte boundary that they are counted from
int64_t parts_of(const amk_verify_args& a) {
  const int64_t part = kStatThreads * kLoads * (a.dtype ? 8 : 4);
  return (a.vocab + 7 + part - 1) / part;
}

// Everything about a call that can be known without its pointers.
amk_status check(const Reason& fail, const amk_verify_args* a) {
  if (!a) return fail(AMK_ERR_INVALID_ARG, "NULL arguments");
  if (a->struct_size != sizeof *a)
    return fail(AMK_ERR_INVALID_ARG, "struct_size %u, the library has %zu", a->struct_size, sizeof *a);
  if (a->dtype > 1) return fail(AMK_ERR_UNSUPPORTED, "dtype %u: 0 (float) or 1 (bf16)", a->dtype);
  if (a->n_rows < 1 || a->n_rows > AMK_TREE_MAX_ROWS)
    return fail(AMK_ERR_UNSUPPORTED, "%u rows: 1 to %d", a->n_rows, AMK_TREE_MAX_ROWS);
  if (a->vocab < 1 || a->vocab > 0x7fffffff - 65536) return fail(AMK_ERR_INVALID_ARG, "%lld logits a row", (long long)a->vocab);
  const int64_t parts = parts_of(*a);
  if ((int64_t)a->n_seqs > 0x7fffffff / 16 || (int64_t)a->n_seqs * a->n_rows > 0x7fffffff / parts)
    return fail(AMK_ERR_INVALID_ARG, "%u sequences of %u rows", a->n_seqs, a->n_rows);
  return AMK_OK;
}

}  // namespace

extern "C" amk_status amk_verify_workspace_bytes(const amk_verify_args* args, size_t* bytes, char* msg, size_t msg_bytes) {
  const Reason fail(msg, msg_bytes, "amk_verify_workspace_bytes");
  if (!bytes) return fail(AMK_ERR_INVALID_ARG, "NULL pointer");
  const amk_status st = check(fail, args);
  if (st != AMK_OK) return st;
  *bytes = sizeof(Stat) * (size_t)args->n_seqs * args->n_rows * (size_t)parts_of(*args);
  return AMK_OK;
}

extern "C" amk_status amk_verify_draft(const amk_verify_args* args, char* msg, size_t msg_bytes, void* cuda_stream) {
  const Reason fail(msg, msg_bytes, "amk_verify_draft");
  const amk_status ok = check(fail, args);
  if (ok != AMK_OK) return ok;
  const amk_verify_args& a = *args;
  if (a.n_seqs == 0) return AMK_OK;
  if (!a.logits || !a.tokens || !a.uniforms || !a.count || !a.keep || !a.token) return fail(AMK_ERR_INVALID_ARG, "NULL pointer");
  const void* words[] = {a.draft, a.tokens, a.parents, a.uniforms, a.temperature, a.cache_len, a.count, a.keep, a.token};
  for (const void* w : words)
    if (!aligned(w, 4)) return fail(AMK_ERR_INVALID_ARG, "pointers must be aligned to their elements");
  if (!aligned(a.logits, a.dtype ? 2 : 4) || !aligned(a.workspace, 256))
    return fail(AMK_ERR_INVALID_ARG, "logits must be aligned to their elements, the workspace to 256 bytes");
  const int64_t most = (int64_t)1 << 40;
  const bool seqs = a.n_seqs > 1, rows = a.n_rows > 1;
  if ((rows && (a.logits_row < a.vocab || a.logits_row > most)) || (seqs && (a.logits_seq < a.vocab || a.logits_seq > most)) ||
      (a.draft && ((rows && (a.draft_row < a.vocab || a.draft_row > most)) || (seqs && (a.draft_seq < a.vocab || a.draft_seq > most)))))
    return fail(AMK_ERR_INVALID_ARG, "strides must be at least the %lld logits of a row", (long long)a.vocab);
  const int64_t parts = parts_of(a);
  const size_t need = sizeof(Stat) * (size_t)a.n_seqs * a.n_rows * (size_t)parts;
  if (!a.workspace || a.workspace_bytes < need)
    return fail(AMK_ERR_INVALID_ARG, "workspace of %llu bytes, %zu are needed",
                (unsigned long long)(a.workspace ? a.workspace_bytes : 0), need);
  bool room = false;
  cudaError_t e = a.dtype ? allow<unsigned short>(&room) : allow<float>(&room);
  if (e != cudaSuccess) return fail(AMK_ERR_CUDA, "%s", cudaGetErrorString(e));
  VerifyParams p{};
  p.logits = a.logits, p.draft = a.draft, p.tokens = a.tokens, p.parents = a.parents, p.u = a.uniforms;
  p.temperature = a.temperature, p.cache_len = a.cache_len, p.count = a.count, p.keep = a.keep, p.token = a.token;
  p.stats = (Stat*)a.workspace;
  p.l_seq = seqs ? a.logits_seq : 0, p.l_row = rows ? a.logits_row : 0;
  p.d_seq = seqs ? a.draft_seq : 0, p.d_row = rows ? a.draft_row : 0;
  p.rows = (int)a.n_rows, p.vocab = (int)a.vocab, p.parts = (int)parts;
  const int sms = multiprocessors();
  p.cluster = 1;
  while (p.cluster < (room ? kMaxCluster : 8) && (int64_t)a.n_seqs * p.cluster * 2 <= sms && a.vocab / (2 * p.cluster) >= 1024) p.cluster *= 2;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  const unsigned stat_blocks = (unsigned)((int64_t)a.n_seqs * a.n_rows * parts), walk_blocks = a.n_seqs * (unsigned)p.cluster;
  e = launch_early(a.dtype ? stats_kernel<unsigned short> : stats_kernel<float>, dim3(stat_blocks), kStatThreads, 0, 1, st, p);
  if (e == cudaSuccess)
    e = launch_early(a.dtype ? walk_kernel<unsigned short> : walk_kernel<float>, dim3(walk_blocks), kThreads, sizeof(Walk),
                     (unsigned)p.cluster, st, p);
  return e == cudaSuccess ? AMK_OK : fail(AMK_ERR_CUDA, "launch failed: %s", cudaGetErrorString(e));
}
