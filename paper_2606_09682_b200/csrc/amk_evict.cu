// amk_evict_select: which positions of a cache stay, by their scores.
//
// Each list is one block's.  The budget-th largest of its keys (the scores' bits in an order that integers have; positions that
// stay anyway hold the largest key) is found digit by digit from histograms of 11, 11 and 10 bits; then the positions whose key
// is larger stay, and of those with that very key the first ones.  Counts are integers: the result is the same every time.
//
// Bound: the instructions of a few sweeps over keys that lie in shared memory, four to a thread at a time (a ballot for every 32 of
// them instead: 256 lists of 8192 25.2 us, so XXX), and with few lists the barriers between the sweeps.  Lists of more than
// 32768 scores are read again from L2 in the histograms, and chosen from in pieces.
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
  int heads, slots, budget, first, recent, piece;      // piece: scores that the shared memory holds
};

// larger for larger scores; 0 for NaN, less than 2^32 - 1 for every number
__device__ __forceinline__ unsigned key_of(unsigned bits) {
  if ((bits & 0x7fffffffu) > 0x7f800000u) return 0;
  if (bits == 0x80000000u) bits = 0;
  return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

__global__ void __launch_bounds__(kThreads) evict_kernel(const EvictParams p) {
  extern __shared__ uint4 smem[];
  unsigned* keys = (unsigned*)smem;                    // of a piece; 0 behind its end, which the order puts last
  unsigned short* chosen = (unsigned short*)(keys + p.piece);
  __shared__ unsigned bins[kBins], digit[2];
  __shared__ unsigned sums[kWarps];
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
  const int count = min(n, p.budget);
  if (threadIdx.x == 0) p.count[list] = count;
  for (int i = count + threadIdx.x; i < p.budget; i += kThreads) keep[i] = -1;
  if (n <= p.budget) {
    for (int i = threadIdx.x; i < n; i += kThreads) {
      keep[i] = i;
      if (out && out != in) out[i] = in[i];
    }
    if (out)
      for (int i = n + threadIdx.x; i < p.slots; i += kThreads) out[i] = 0;
    return;
  }
  const auto key_at = [&](int i) { return i < p.first || i >= n - p.recent ? ~0u : key_of(in[i]); };
  const auto bring = [&](int from) {                   // the keys of a piece; its rounds
    const int m = min(p.piece, n - from), rounds = (m + kSweep - 1) / kSweep;
#pragma unroll 4
    for (int i = threadIdx.x; i < rounds * kSweep; i += kThreads) keys[i] = i < m ? key_at(from + i) : 0;
    return rounds;
  };
  const bool whole = n <= p.piece;
  int rounds = 0;
  for (int i = threadIdx.x; i < kBins; i += kThreads) bins[i] = 0;
  if (whole) rounds = bring(0);
  // keys above the border stay, and `equal` of those that have it
  unsigned border = 0;
  int equal = p.budget;
#pragma unroll 1
  for (int pass = 0; pass < 3; pass++) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 1023 : 2047;
    const auto count_key = [&](unsigned key) {
      if (pass == 0 || key >> (pass == 1 ? 21 : 10) == border) atomicAdd(&bins[key >> shift & width], 1u);
    };
    __syncthreads();
    if (whole) {
      for (int r = 0; r < rounds; r++) {
        const uint4 k = smem[r * kThreads + threadIdx.x];
        count_key(k.x), count_key(k.y), count_key(k.z), count_key(k.w);
      }
    } else {
#pragma unroll 4
      for (int i = threadIdx.x; i < n; i += kThreads) count_key(key_at(i));
    }
    __syncthreads();
    // the digit: the largest one at or above which `equal` keys lie.  Two bins a thread, from the largest down.
    const int top = kBins - 1 - 2 * (int)threadIdx.x;
    const int a = (int)bins[top], b = (int)bins[top - 1];
    bins[top] = bins[top - 1] = 0;
    int sum = a + b;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(~0u, sum, o);
      if (lane >= o) sum += x;
    }
    if (lane == 31) sums[warp] = (unsigned)sum;
    __syncthreads();
    const int own = (int)sums[lane];                   // (32 warps, 32 lanes)
    sum += __reduce_add_sync(~0u, lane < warp ? own : 0);
    const int before = sum - a - b;
    if (before < equal && before + a >= equal) digit[0] = (unsigned)top, digit[1] = (unsigned)before;
    if (before + a < equal && sum >= equal) digit[0] = (unsigned)top - 1, digit[1] = (unsigned)(before + a);
    __syncthreads();
    border = border << (pass == 2 ? 10 : 11) | digit[0];
    equal -= (int)digit[1];
  }
  // Which ones stay, piece by piece in ascending order, a run of a piece for each warp.  Counts of keys above the border stand in
  // the upper half of a word, of those that have it in the lower half.  Rows move down only, and all scores of 1024 rows are read
  // before one of them is written: `moved` may be the scores themselves.
  int above = 0, same = 0;                             // in the pieces in front
  for (int from = 0; from < n; from += p.piece) {
    if (!whole) {
      __syncthreads();
      rounds = bring(from);
      __syncthreads();
    }
    const auto packed = [&](unsigned key) { return key > border ? 0x10000u : key == border ? 1u : 0u; };
    const uint4* mine = smem + warp * rounds * 32 + lane;
    unsigned all = 0;
    for (int r = 0; r < rounds; r++) {
      const uint4 k = mine[r * 32];
      all += packed(k.x) + packed(k.y) + packed(k.z) + packed(k.w);
    }
    all = __reduce_add_sync(~0u, all);
    __syncthreads();
    if (lane == 0) sums[warp] = all;
    __syncthreads();
    const unsigned own = sums[lane], total = __reduce_add_sync(~0u, own);
    unsigned run = __reduce_add_sync(~0u, lane < warp ? own : 0);
    const int base = above + min(same, equal);         // rows that stay in the pieces in front
    for (int r = 0; r < rounds; r++) {
      const uint4 k = mine[r * 32];
      const unsigned c[4] = {packed(k.x), packed(k.y), packed(k.z), packed(k.w)};
      const unsigned four = c[0] + c[1] + c[2] + c[3];
      unsigned scan = four;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned x = __shfl_up_sync(~0u, scan, o);
        if (lane >= o) scan += x;
      }
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
    const int rows = above + min(same, equal) - base;
    __syncthreads();
    for (int i0 = 0; i0 < rows; i0 += kThreads) {
      const int i = i0 + threadIdx.x;
      int row = 0;
      unsigned bits = 0;
      if (i < rows) {
        row = from + chosen[i];
        if (out) bits = in[row];
      }
      if (out == in) __syncthreads();
      if (i < rows) {
        keep[base + i] = row;
        if (out) out[base + i] = bits;
      }
    }
  }
  if (out) {
    if (out == in) __syncthreads();                    // (every row has been read)
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
  e = cudaFuncSetAttribute(evict_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPiece * 6);
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
  const int piece = n_slots < kPiece ? ((int)n_slots + kSweep - 1) / kSweep * kSweep : kPiece;
  const EvictParams p{scores, moved, lens, keep, count, scores_seq, scores_head, moved_seq, moved_head, (int)n_heads,
                      (int)n_slots, (int)budget, (int)first, (int)recent, piece};
  e = amk::launch_early(evict_kernel, dim3((unsigned)(n_seqs * n_heads)), kThreads, (size_t)piece * 6, 1,
                        (cudaStream_t)cuda_stream, p);
  return e == cudaSuccess ? AMK_OK : fail(AMK_ERR_CUDA, "launch failed: %s", cudaGetErrorString(e));
}
