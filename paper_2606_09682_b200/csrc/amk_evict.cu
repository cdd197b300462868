// amk_evict_select: which positions of a cache stay, by their scores.
//
// Each list is one block's.  The budget-th largest of its keys (the scores' bits in an order that integers have; positions that
// stay anyway hold the largest key) is found digit by digit from histograms of 11, 11 and 10 bits; then the positions whose key
// is larger stay, and of those with that very key the first ones.  Counts are integers: the result is the same every time.
//
// Bound: nothing alone.  While its blocks run an SM issues in 62 % of the cycles; of the 20 cycles from one instruction of a warp to
// its next, 4 wait for the scheduler, 3.5 at the barriers between the sweeps, 2 each for arithmetic, for shared memory and its
// atomics, and for memory; with few lists the barriers are what counts.  (256 lists of 8192: with a ballot for every 32 keys 25.2 us;
// sweeps over shared memory, four keys to a thread, 16.1; keys in registers, a run for each thread, 10.4, of equal scores 10.0.  128
// lists of 16384 9.6, 64 of 32768 18.8.)  Lists of more than 32768 slots are read again from L2 in the histograms, and chosen from in
// pieces, by one block: 24 lists of 100001 109 us.
#include <cuda_runtime.h>

#include <atomic>

#include "amk.h"
#include "amk_op_launch.h"
#include "amk_op_util.h"
#include "amk_ptx.cuh"

namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32, kBins = 2048;
constexpr int kSweep = 4 * kThreads;                   // keys of a sweep's round
constexpr int kPiece = 32768;                          // keys in shared memory at most, a multiple of kSweep

struct EvictParams {
  const float* scores;
  float* moved;
  const int* lens;
  int *keep, *count;
  int64_t seq, head, moved_seq, moved_head;
  int heads, slots, budget, first, recent;
};

// larger for larger scores; 0 for NaN, less than 2^32 - 1 for every number
__device__ __forceinline__ unsigned key_of(unsigned bits) {
  const float x = __uint_as_float(bits) + 0.f;         // (-0 becomes 0)
  const unsigned u = __float_as_uint(x);
  return x == x ? u ^ ((unsigned)((int)u >> 31) | 0x80000000u) : 0u;
}

// A list and what its block does whatever it holds.
struct List {
  const unsigned* in;
  unsigned* out;
  int* keep;
  int n;
};
// true: there is nothing to choose, and all is done
__device__ __forceinline__ bool begin_list(const EvictParams& p, List& a) {
  const int list = blockIdx.x, s = list / p.heads, h = list - s * p.heads;
  a.in = (const unsigned*)p.scores + s * p.seq + h * p.head;
  a.out = p.moved ? (unsigned*)p.moved + s * p.moved_seq + h * p.moved_head : nullptr;
  a.keep = p.keep + (int64_t)list * p.budget;
  a.n = p.lens[s];
  if (a.n < 0 || a.n > p.slots) {
    if (threadIdx.x == 0) p.count[list] = -1;
    for (int i = threadIdx.x; i < p.budget; i += kThreads) a.keep[i] = -1;
    if (a.out && a.out != a.in)
      for (int i = threadIdx.x; i < p.slots; i += kThreads) a.out[i] = a.in[i];
    return true;
  }
  const int count = min(a.n, p.budget);
  if (threadIdx.x == 0) p.count[list] = count;
  for (int i = count + threadIdx.x; i < p.budget; i += kThreads) a.keep[i] = -1;
  if (a.n > p.budget) return false;
  for (int i = threadIdx.x; i < a.n; i += kThreads) {
    a.keep[i] = i;
    if (a.out && a.out != a.in) a.out[i] = a.in[i];
  }
  if (a.out)
    for (int i = a.n + threadIdx.x; i < p.slots; i += kThreads) a.out[i] = 0;
  return true;
}

__device__ __forceinline__ int warp_scan(int x, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(~0u, x, o);
    if (lane >= o) x += y;
  }
  return x;
}

struct Shared {
  unsigned bins[kBins], digit[2], sums[kWarps];
};

// Keys above the border stay, and `equal` of those that have it.  each(f): calls f with every key of this thread.  bins are 0.
template <class Each>
__device__ __forceinline__ void find_border(Shared& h, unsigned& border, int& equal, const Each& each) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  border = 0;
#pragma unroll
  for (int pass = 0; pass < 3; pass++) {
    constexpr int kShift[3] = {21, 10, 0}, kWidth[3] = {11, 11, 10};
    __syncthreads();
    each([&](unsigned key) {
      if (pass == 0 || key >> (kShift[pass] + kWidth[pass]) == border) atomicAdd(&h.bins[key >> kShift[pass] & ((1u << kWidth[pass]) - 1)], 1u);
    });
    __syncthreads();
    // the digit: the largest one at or above which `equal` keys lie.  Two bins a thread, from the largest down.
    const int top = kBins - 1 - 2 * (int)threadIdx.x;
    uint2* pair = (uint2*)&h.bins[top - 1];
    const int a = (int)pair->y, b = (int)pair->x;
    *pair = make_uint2(0, 0);
    int sum = warp_scan(a + b, lane);
    if (lane == 31) h.sums[warp] = (unsigned)sum;
    __syncthreads();
    const int own = (int)h.sums[lane];                 // (32 warps, 32 lanes)
    sum += __reduce_add_sync(~0u, lane < warp ? own : 0);
    const int before = sum - a - b;
    if (before < equal && sum >= equal) {
      const bool first = before + a >= equal;
      h.digit[0] = (unsigned)(first ? top : top - 1), h.digit[1] = (unsigned)(first ? before : before + a);
    }
    __syncthreads();
    border = border << kWidth[pass] | h.digit[0];
    equal -= (int)h.digit[1];
  }
}

// Rows [base, base + rows) of the outputs, from the indices chosen behind `from`.  All scores of 1024 rows are read before one of
// them is written, and rows move down only: `out` may be `in`.
__device__ __forceinline__ void write_rows(const List& a, const unsigned short* chosen, int from, int base, int rows) {
  for (int i0 = 0; i0 < rows; i0 += kThreads) {
    const int i = i0 + threadIdx.x;
    int row = 0;
    unsigned bits = 0;
    if (i < rows) {
      row = from + chosen[i];
      if (a.out) bits = a.in[row];
    }
    if (a.out == a.in) __syncthreads();
    if (i < rows) {
      a.keep[base + i] = row;
      if (a.out) a.out[base + i] = bits;
    }
  }
}
__device__ __forceinline__ void clear_behind(const EvictParams& p, const List& a) {
  if (!a.out) return;
  if (a.out == a.in) __syncthreads();                  // (every row has been read)
  for (int i = p.budget + threadIdx.x; i < p.slots; i += kThreads) a.out[i] = 0;
}

// Counts of keys above the border stand in the upper half of a word, of those that have it in the lower half.
__device__ __forceinline__ unsigned packed(unsigned key, unsigned border) { return key > border ? 0x10000u : key == border ? 1u : 0u; }

// Up to 1024 E slots: a thread's keys, E in a row, in registers.
template <int E>
__global__ void __launch_bounds__(kThreads) evict_held_kernel(const EvictParams p) {
  extern __shared__ uint4 smem[];
  unsigned short* chosen = (unsigned short*)smem;
  __shared__ Shared h;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  List a;
  *(uint2*)&h.bins[2 * threadIdx.x] = make_uint2(0, 0);
  amk::wait_for_grid_before();
  if (begin_list(p, a)) return;
  const int i0 = threadIdx.x * E;
  unsigned key[E];                                     // 0 behind the end, which the order puts last
  if (((uintptr_t)a.in & 15) == 0 && i0 + E <= a.n) {
#pragma unroll
    for (int j = 0; j < E; j += 4) {
      const uint4 x = *(const uint4*)(a.in + i0 + j);
      key[j] = key_of(x.x), key[j + 1] = key_of(x.y), key[j + 2] = key_of(x.z), key[j + 3] = key_of(x.w);
    }
  } else {
#pragma unroll
    for (int j = 0; j < E; j++) key[j] = i0 + j < a.n ? key_of(a.in[i0 + j]) : 0u;
  }
  if (i0 < p.first || i0 + E > a.n - p.recent) {
#pragma unroll
    for (int j = 0; j < E; j++)
      if (i0 + j < a.n && (i0 + j < p.first || i0 + j >= a.n - p.recent)) key[j] = ~0u;
  }
  unsigned border;
  int equal = p.budget;
  find_border(h, border, equal, [&](auto f) {
#pragma unroll
    for (int j = 0; j < E; j++) f(key[j]);
  });
  unsigned own = 0;
#pragma unroll
  for (int j = 0; j < E; j++) own += packed(key[j], border);
  unsigned at = (unsigned)warp_scan((int)own, lane);
  if (lane == 31) h.sums[warp] = at;
  __syncthreads();
  const unsigned other = h.sums[lane];
  at += __reduce_add_sync(~0u, lane < warp ? other : 0) - own;
  if (own) {
    int more = (int)(at >> 16), ties = (int)(at & 0xffffu);
#pragma unroll
    for (int j = 0; j < E; j++) {
      const bool over = key[j] > border, even = key[j] == border;
      if (over || (even && ties < equal)) chosen[more + min(ties, equal)] = (unsigned short)(i0 + j);
      more += over, ties += even;
    }
  }
  __syncthreads();
  write_rows(a, chosen, 0, 0, p.budget);
  clear_behind(p, a);
}

// Any number of slots: the list is read again for each histogram, and then in pieces that lie in shared memory, a run of a piece for
// each warp.
__global__ void __launch_bounds__(kThreads) evict_kernel(const EvictParams p) {
  extern __shared__ uint4 smem[];
  unsigned* keys = (unsigned*)smem;                    // of a piece; 0 behind its end, which the order puts last
  unsigned short* chosen = (unsigned short*)(keys + kPiece);
  __shared__ Shared h;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  List a;
  *(uint2*)&h.bins[2 * threadIdx.x] = make_uint2(0, 0);
  amk::wait_for_grid_before();
  if (begin_list(p, a)) return;
  const auto key_at = [&](int i) { return i < p.first || i >= a.n - p.recent ? ~0u : key_of(a.in[i]); };
  unsigned border;
  int equal = p.budget;
  find_border(h, border, equal, [&](auto f) {
#pragma unroll 4
    for (int i = threadIdx.x; i < a.n; i += kThreads) f(key_at(i));
  });
  int above = 0, same = 0;                             // in the pieces in front
  for (int from = 0; from < a.n; from += kPiece) {
    const int m = min(kPiece, a.n - from), rounds = (m + kSweep - 1) / kSweep;
    __syncthreads();
#pragma unroll 4
    for (int i = threadIdx.x; i < rounds * kSweep; i += kThreads) keys[i] = i < m ? key_at(from + i) : 0;
    __syncthreads();
    const uint4* mine = smem + warp * rounds * 32 + lane;
    unsigned all = 0;
    for (int r = 0; r < rounds; r++) {
      const uint4 k = mine[r * 32];
      all += packed(k.x, border) + packed(k.y, border) + packed(k.z, border) + packed(k.w, border);
    }
    all = __reduce_add_sync(~0u, all);
    if (lane == 0) h.sums[warp] = all;
    __syncthreads();
    const unsigned own = h.sums[lane], total = __reduce_add_sync(~0u, own);
    unsigned run = __reduce_add_sync(~0u, lane < warp ? own : 0);
    const int base = above + min(same, equal);         // rows that stay in the pieces in front
    for (int r = 0; r < rounds; r++) {
      const uint4 k = mine[r * 32];
      const unsigned c[4] = {packed(k.x, border), packed(k.y, border), packed(k.z, border), packed(k.w, border)};
      const unsigned four = c[0] + c[1] + c[2] + c[3], scan = (unsigned)warp_scan((int)four, lane);
      unsigned at = run + scan - four;
      run += __shfl_sync(~0u, scan, 31);
      if (four) {
        const int i = ((warp * rounds + r) * 32 + lane) * 4;
#pragma unroll
        for (int j = 0; j < 4; j++) {
          const int ties = same + (int)(at & 0xffffu);
          if (c[j] > 1 || (c[j] && ties < equal)) chosen[above + (int)(at >> 16) + min(ties, equal) - base] = (unsigned short)(i + j);
          at += c[j];
        }
      }
    }
    above += (int)(total >> 16), same += (int)(total & 0xffffu);
    __syncthreads();
    write_rows(a, chosen, from, base, above + min(same, equal) - base);
  }
  clear_behind(p, a);
}

template <int E>
cudaError_t launch_held(const EvictParams& p, unsigned lists, cudaStream_t st) {
  return amk::launch_early(evict_held_kernel<E>, dim3(lists), kThreads, (size_t)2 * p.budget + 16, 1, st, p);
}

cudaError_t allow_smem() {
  static std::atomic<unsigned long long> done{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
  if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(evict_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPiece * 6);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(evict_held_kernel<32>, cudaFuncAttributeMaxDynamicSharedMemorySize, kPiece * 2 + 16);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
  return e;
}

}  // namespace

extern "C" amk_status amk_evict_select(const float* scores, int64_t n_seqs, int64_t n_heads, int64_t n_slots,
                                       int64_t scores_seq, int64_t scores_head, const int32_t* lens, int64_t budget,
                                       int64_t first, int64_t recent, int32_t* keep, int32_t* count, float* moved,
                                       int64_t moved_seq, int64_t moved_head, char* msg, size_t msg_bytes, void* cuda_stream) {
  const amk::Reason fail(msg, msg_bytes, "amk_evict_select");
  if (n_seqs < 0 || n_heads < 1 || n_slots < 1 || n_slots > 0x7fff0000 || n_seqs > 0x7fffffff / n_heads)
    return fail(AMK_ERR_INVALID_ARG, "%lld sequences of %lld heads and %lld slots", (long long)n_seqs, (long long)n_heads,
                (long long)n_slots);
  if (budget < 1 || budget > n_slots)
    return fail(AMK_ERR_INVALID_ARG, "budget %lld: 1 to the %lld slots", (long long)budget, (long long)n_slots);
  if (first < 0 || recent < 0 || first > budget || recent > budget - first)
    return fail(AMK_ERR_INVALID_ARG, "first %lld and recent %lld: at least 0, together no more than the budget of %lld",
                (long long)first, (long long)recent, (long long)budget);
  if (n_seqs == 0) return AMK_OK;
  if (!scores || !lens || !keep || !count) return fail(AMK_ERR_INVALID_ARG, "NULL pointer");
  if (!amk::aligned(scores, 4) || !amk::aligned(lens, 4) || !amk::aligned(keep, 4) || !amk::aligned(count, 4) ||
      !amk::aligned(moved, 4))
    return fail(AMK_ERR_INVALID_ARG, "pointers must be 4-byte aligned");
  if (n_heads == 1) scores_head = moved_head = n_slots;
  if (n_seqs == 1) scores_seq = moved_seq = n_slots;
  const int64_t most = (int64_t)1 << 36;
  if (scores_seq < n_slots || scores_head < n_slots || scores_seq > most || scores_head > most ||
      (moved && (moved_seq < n_slots || moved_head < n_slots || moved_seq > most || moved_head > most)))
    return fail(AMK_ERR_INVALID_ARG, "strides must be at least the %lld slots", (long long)n_slots);
  if (moved == scores && (moved_seq != scores_seq || moved_head != scores_head))
    return fail(AMK_ERR_INVALID_ARG, "moved is scores, but at other strides");
  const EvictParams p{scores, moved, lens, keep, count, scores_seq, scores_head, moved_seq, moved_head, (int)n_heads,
                      (int)n_slots, (int)budget, (int)first, (int)recent};
  const unsigned lists = (unsigned)(n_seqs * n_heads);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  cudaError_t e = allow_smem();
  if (e != cudaSuccess) return fail(AMK_ERR_CUDA, "%s", cudaGetErrorString(e));
  if (n_slots <= 4 * kThreads) e = launch_held<4>(p, lists, st);
  else if (n_slots <= 8 * kThreads) e = launch_held<8>(p, lists, st);
  else if (n_slots <= 16 * kThreads) e = launch_held<16>(p, lists, st);
  else if (n_slots <= 32 * kThreads) e = launch_held<32>(p, lists, st);
  else e = amk::launch_early(evict_kernel, dim3(lists), kThreads, (size_t)kPiece * 6, 1, st, p);
  return e == cudaSuccess ? AMK_OK : fail(AMK_ERR_CUDA, "launch failed: %s", cudaGetErrorString(e));
}
