// amk_evict_select: which positions of a cache stay, by their scores.
//
// Each list is one block's.  The budget-th largest of its keys (the scores' bits in an order that integers have; positions that
// stay anyway hold the largest key) is found digit by digit from histograms of 11, 11 and 10 bits; then the positions whose key
// is larger stay, and of those with that very key the first ones.  Counts are integers: the result is the same every time.
//
// Bound: latency, three histograms and their sums of a few thousand keys that lie in shared memory; lists longer than that are
// read again from L2 in the histograms, and chosen from in pieces.
#include <cuda_runtime.h>

#include <atomic>

#include "amk.h"
#include "amk_op_launch.h"
#include "amk_op_util.h"
#include "amk_ptx.cuh"

namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32, kBins = 2048;
constexpr int kPiece = 49152;                          // scores in shared memory at most

struct EvictParams {
  const float* scores;
  float* moved;
  const int* lens;
  int *keep, *count;
  int64_t seq, head, moved_seq, moved_head;
  int heads, slots, budget, first, recent, piece;      // piece: scores that the shared memory holds
};

// larger for larger scores; 0 for NaN, less than 2^32 - 1 for every number
__device__ __forceinline__ unsigned key_of(unsigned bits) {
  if ((bits & 0x7fffffffu) > 0x7f800000u) return 0;
  if (bits == 0x80000000u) bits = 0;
  return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

__global__ void __launch_bounds__(kThreads) evict_kernel(const EvictParams p) {
  extern __shared__ unsigned held[];
  __shared__ unsigned bins[kBins], digit[2];
  __shared__ int warp_a[kWarps], warp_b[kWarps];
  const int list = blockIdx.x, s = list / p.heads, h = list - s * p.heads;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const unsigned* in = (const unsigned*)p.scores + s * p.seq + h * p.head;
  unsigned* out = p.moved ? (unsigned*)p.moved + s * p.moved_seq + h * p.moved_head : nullptr;
  int* keep = p.keep + (int64_t)list * p.budget;
  amk::wait_for_grid_before();
  const int n = p.lens[s];
  if (n < 0 || n > p.slots) {
    if (threadIdx.x == 0) p.count[list] = -1;
    for (int i = threadIdx.x; i < p.budget; i += kThreads) keep[i] = -1;
    if (out && out != in)
      for (int i = threadIdx.x; i < p.slots; i += kThreads) out[i] = in[i];
    return;
  }
  const bool all = n <= p.budget, whole = n <= p.piece;
  unsigned border = 0;                                 // keys above it stay, and `equal` of those that have it
  int equal = n;
  if (!all) {
    if (whole) {
      for (int i = threadIdx.x; i < n; i += kThreads) held[i] = in[i];
    }
    int left = p.budget;
    unsigned above = 0;                                // the digits found so far
#pragma unroll 1
    for (int pass = 0; pass < 3; pass++) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 1024 : 2048;
      for (int i = threadIdx.x; i < kBins; i += kThreads) bins[i] = 0;
      __syncthreads();
      for (int i = threadIdx.x; i < n; i += kThreads) {
        const unsigned key = i < p.first || i >= n - p.recent ? ~0u : key_of(whole ? held[i] : in[i]);
        if (pass == 0 || key >> (pass == 1 ? 21 : 10) == above) atomicAdd(&bins[key >> shift & (width - 1)], 1u);
      }
      __syncthreads();
      // the digit: the largest one at or above which `left` keys lie.  Two bins a thread, from the largest down.
      const int top = kBins - 1 - 2 * (int)threadIdx.x;
      const int a = (int)bins[top], b = (int)bins[top - 1];
      int sum = a + b;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(~0u, sum, o);
        if (lane >= o) sum += x;
      }
      if (lane == 31) warp_a[warp] = sum;
      __syncthreads();
      const int own = warp_a[lane];                    // (32 warps, 32 lanes)
      sum += __reduce_add_sync(~0u, lane < warp ? own : 0);
      const int before = sum - a - b;
      if (before < left && before + a >= left) digit[0] = top, digit[1] = before;
      if (before + a < left && sum >= left) digit[0] = top - 1, digit[1] = before + a;
      __syncthreads();
      above = above << (pass == 2 ? 10 : 11) | digit[0];
      left -= (int)digit[1];
    }
    border = above;
    equal = left;
  }
  // which ones stay, piece by piece in ascending order; a warp has a run of a piece.  A piece is in shared memory before any of
  // its rows moves, and rows move down only: `moved` may be the scores themselves.
  int kept = 0, same = 0;                              // so far, among all keys / among those of the border
  const int per_piece = all ? n : p.piece;
  for (int from = 0; from < n && !all; from += per_piece) {
    const int m = min(per_piece, n - from), run = ((m + kWarps - 1) / kWarps + 31) & ~31;
    if (!whole) {
      __syncthreads();
      for (int i = threadIdx.x; i < m; i += kThreads) held[i] = in[from + i];
      __syncthreads();
    }
    const int begin = min(warp * run, m), end = min(begin + run, m);
    int more = 0, ties = 0;
    for (int i = begin + lane; i < end; i += 32) {
      const int at = from + i;
      const unsigned key = at < p.first || at >= n - p.recent ? ~0u : key_of(held[i]);
      more += key > border, ties += key == border;
    }
    more = __reduce_add_sync(~0u, more), ties = __reduce_add_sync(~0u, ties);
    __syncthreads();
    if (lane == 0) warp_a[warp] = more, warp_b[warp] = ties;
    __syncthreads();
    const int wa = warp_a[lane], wb = warp_b[lane];
    const int more_before = __reduce_add_sync(~0u, lane < warp ? wa : 0), all_more = __reduce_add_sync(~0u, wa);
    int tie = same + __reduce_add_sync(~0u, lane < warp ? wb : 0);
    const int all_ties = __reduce_add_sync(~0u, wb);
    // kept holds min(same, equal) ties
    int place = kept + more_before + min(tie, equal) - min(same, equal);
    for (int i0 = begin; i0 < end; i0 += 32) {
      const int i = i0 + lane, at = from + i;
      unsigned bits = 0, key = 0;
      if (i < end) {
        bits = held[i];
        key = at < p.first || at >= n - p.recent ? ~0u : key_of(bits);
      }
      const unsigned over = __ballot_sync(~0u, i < end && key > border), eq = __ballot_sync(~0u, i < end && key == border);
      const unsigned below = (1u << lane) - 1u;
      const bool stays = (over >> lane & 1) || ((eq >> lane & 1) && tie + __popc(eq & below) < equal);
      const unsigned in_all = __ballot_sync(~0u, stays);
      if (stays) {
        const int to = place + __popc(in_all & below);
        keep[to] = at;
        if (out) out[to] = bits;
      }
      place += __popc(in_all), tie += __popc(eq);
    }
    kept += all_more + min(same + all_ties, equal) - min(same, equal);
    same += all_ties;
  }
  const int count = all ? n : p.budget;
  if (all)
    for (int i = threadIdx.x; i < n; i += kThreads) {
      keep[i] = i;
      if (out && out != in) out[i] = in[i];
    }
  if (threadIdx.x == 0) p.count[list] = count;
  for (int i = count + threadIdx.x; i < p.budget; i += kThreads) keep[i] = -1;
  if (out) {
    __syncthreads();                                   // (in place: every piece has been read)
    for (int i = count + threadIdx.x; i < p.slots; i += kThreads) out[i] = 0;
  }
}

cudaError_t allow_smem() {
  static std::atomic<unsigned long long> done{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
  if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(evict_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPiece * 4);
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
  cudaError_t e = allow_smem();
  if (e != cudaSuccess) return fail(AMK_ERR_CUDA, "%s", cudaGetErrorString(e));
  const int piece = (int)(n_slots < kPiece ? n_slots : kPiece);
  const EvictParams p{scores, moved, lens, keep, count, scores_seq, scores_head, moved_seq, moved_head, (int)n_heads,
                      (int)n_slots, (int)budget, (int)first, (int)recent, piece};
  e = amk::launch_early(evict_kernel, dim3((unsigned)(n_seqs * n_heads)), kThreads, (size_t)piece * 4, 1,
                        (cudaStream_t)cuda_stream, p);
  return e == cudaSuccess ? AMK_OK : fail(AMK_ERR_CUDA, "launch failed: %s", cudaGetErrorString(e));
}
