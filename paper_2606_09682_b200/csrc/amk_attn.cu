// amk_prompt_attention, amk_tree_attention and amk_attention_weights: argument checks and launches.
#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>

#include <atomic>

#include "amk_attn.cuh"
#include "amk_attn_weights.cuh"
#include "amk_op_launch.h"
#include "amk_op_util.h"

namespace {

using amk::Reason;

using amk::AttnParams;

// cuTensorMapEncodeTiled of the driver that is loaded, or null
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
  static const EncodeTiled fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess) {
      (void)cudaGetLastError();
      f = nullptr;
    }
    return (EncodeTiled)f;
  }();
  return fn;
}

// A cache or a projection as {element, row, head, sequence}; boxes of 128 (box_rows) rows x 64 elements (bf16, swizzled for the
// tensor cores) or whole 8-bit rows.  Strides in elements; an axis of one entry has a legal stride already.
bool make_map(CUtensorMap* map, const void* base, bool fp8, int64_t hd, int64_t rows, int64_t heads, int64_t seqs,
              int64_t row, int64_t head, int64_t seq, int box_rows = amk::kTile) {
  const EncodeTiled encode = encode_tiled();
  if (!encode) return false;
  const cuuint64_t esz = fp8 ? 1 : 2;
  const cuuint64_t dims[4] = {(cuuint64_t)hd, (cuuint64_t)rows, (cuuint64_t)heads, (cuuint64_t)seqs};
  const cuuint64_t strides[3] = {(cuuint64_t)row * esz, (cuuint64_t)head * esz, (cuuint64_t)seq * esz};
  const cuuint32_t box[4] = {fp8 ? (cuuint32_t)hd : 64u, (cuuint32_t)box_rows, 1, 1}, steps[4] = {1, 1, 1, 1};
  return encode(map, fp8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base),
                dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                fp8 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The shared-memory limit of a kernel, raised once on each device.
template <int HD, bool TREE, bool FP8>
cudaError_t allow_smem() {
  static std::atomic<unsigned long long> done{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = dev < 64 ? 1ull << dev : 0;      // (0: set at every call)
  if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(amk::attn_kernel<HD, TREE, FP8>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           amk::AttnSmem<HD, FP8>::kBytes);
  if (e == cudaSuccess && TREE)
    e = cudaFuncSetAttribute(amk::attn_kernel<HD, TREE, FP8>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
  return e;
}

// Clusters of 2^i blocks of a tree kernel that the device can run at the same time, asked once on each device; 0: none, or it
// does not say.
template <int HD, bool FP8>
int cluster_room(int i) {
  static std::atomic<int> known[8][5];                 // plus one
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    (void)cudaGetLastError();
    return 0;
  }
  if (dev < 8 && known[dev][i].load(std::memory_order_acquire)) return known[dev][i].load(std::memory_order_acquire) - 1;
  int n = 0;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = 1u << i, at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(1u << i);
  cfg.blockDim = dim3(FP8 ? 768 : 640);
  cfg.dynamicSmemBytes = amk::AttnSmem<HD, FP8>::kBytes;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  if (allow_smem<HD, true, FP8>() != cudaSuccess ||
      cudaOccupancyMaxActiveClusters(&n, amk::attn_kernel<HD, true, FP8>, &cfg) != cudaSuccess) {
    (void)cudaGetLastError();
    n = 0;
  }
  if (dev < 8) known[dev][i].store(n + 1, std::memory_order_release);
  return n;
}

template <int HD, bool TREE, bool FP8>
cudaError_t launch_attn(const AttnParams& p, const CUtensorMap& k, const CUtensorMap& v, unsigned blocks,
                        cudaStream_t st) {
  const cudaError_t e = allow_smem<HD, TREE, FP8>();
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;         // the kernel waits for the one before it itself
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)p.cluster, at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(FP8 ? 768 : 640);
  cfg.dynamicSmemBytes = amk::AttnSmem<HD, FP8>::kBytes;
  cfg.stream = st;
  cfg.attrs = at;
  cfg.numAttrs = TREE && p.cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, amk::attn_kernel<HD, TREE, FP8>, p, k, v);
}

template <int HD>
cudaError_t launch_join(const AttnParams& p, unsigned blocks, cudaStream_t st) {
  // starts while the attention kernel runs and waits there for its end: the launch is off the path
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(p.rows * p.rep + 31) / 32 * (HD / 8), (unsigned)p.nkv, (unsigned)p.n_seqs);
  // a warp for each part that an item is expected in
  const int64_t items = (int64_t)p.nkv * p.row_tiles * p.n_seqs;
  cfg.blockDim = dim3(32 * (unsigned)(blocks >= 6 * items ? amk::kJoinWarps : blocks >= 3 * items ? 4 : 2));
  cfg.stream = st;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, amk::attn_join_kernel<HD>, p, (int)blocks);
}

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
    (void)cudaGetLastError();
    return 148;
  }
  return n;
}

// What amk_debug_operator_wait set.
std::atomic<unsigned> g_wait_cycles{amk::kWaitCycles};
std::atomic<unsigned> g_tiles{~0u};
template <class Params>
void set_limits(Params& p) {
  p.wait_cycles = g_wait_cycles.load(std::memory_order_relaxed);
  p.tiles = g_tiles.load(std::memory_order_relaxed);
}

// How a tree call is divided: rows of a block, blocks, scratch.  Runs of equal length for all blocks and a second kernel that
// joins the parts, or, in one launch and without scratch, for each item
//  - a cluster of blocks with two tiles each, where it has few rows: the parts meet in distributed shared memory, which is
//    slower than L2.  Clusters / runs, us a call in a graph: 4 items of 8 rows of 64, 17 tiles 10.6 / 12.0; 8 items of 16 rows of
//    128, 8 tiles 12.0 / 13.7, over the 8-bit cache 15.0 / 16.4; 3 items of 15 rows of 64, 4 tiles 10.4 / 11.7.  At the limit of
//    rows runs are not better yet (8 items of 32 rows of 128, 16 tiles 13.2 / 14.1), at 128 rows they are (8 items of 64, 4
//    tiles 12.5 / 12.3);
//  - one block, where its tiles (and three for its beginning and end) are no more than its share of the runs and six to ten
//    more, which is what the second kernel and the parts' way through memory cost.  One block / runs: 128 items of 128 rows of
//    128, 4 tiles 15.1 / 27.0, 12 tiles 30.1 / 42.3; 64 items of 128 rows of 64, 8 tiles 14.9 / 18.9; 32 items of 128 rows of 128,
//    4 tiles 14.6 / 18.6; over the 8-bit cache 128 items, 8 tiles 24.9 / 40.1; 32 items, 4 tiles 18.8 / 22.4.  Beyond the limit: 32
//    items, 6 tiles 16.4 / 18.8 (runs a little early), 9 tiles 18.8 / 20.0, 12 tiles 21.5 / 20.4, over the 8-bit cache 9 tiles
//    25.7 / 24.5; 8 items, 4 tiles 14.3 / 15.0, 6 tiles 16.1 / 15.0.  The lengths may be anything below the bound that is known
//    here, and the longest decides for single blocks, the sum for runs: no further than 12 tiles (128 full items of 16 tiles
//    would be 36.5 / 49.0).
struct TreePlan {
  int part_rows, row_tiles, cluster;
  unsigned blocks;
  size_t bytes;
};
constexpr int kMinTiles = 2;
TreePlan tree_plan(const amk_tree_args& a) {
  TreePlan t;
  const int64_t rows = (int64_t)a.n_rows * (a.n_q_heads / a.n_kv_heads);
  t.part_rows = rows <= amk::kTile ? amk::kTile : 2 * amk::kTile;
  t.row_tiles = (int)((rows + t.part_rows - 1) / t.part_rows);
  const int64_t most = a.n_slots - a.n_rows, len = a.max_len && a.max_len < most ? a.max_len : most;
  const int64_t tiles = (len + a.n_rows + amk::kTile - 1) / amk::kTile, items = (int64_t)a.n_kv_heads * t.row_tiles * a.n_seqs;
  const int sms = sm_count();
  t.cluster = 0;
  if (t.row_tiles == 1 && t.part_rows == amk::kTile && items <= sms) {
    int i = 0;
    while (i < 4 && tiles > kMinTiles << i) {
      const int more = a.head_dim == 64 ? a.kv_dtype ? cluster_room<64, true>(i + 1) : cluster_room<64, false>(i + 1)
                                        : a.kv_dtype ? cluster_room<128, true>(i + 1) : cluster_room<128, false>(i + 1);
      if (more < items) break;
      i++;
    }
    const bool meet = tiles <= kMinTiles << i && (i == 0 || rows * a.head_dim <= 2048);
    if (!meet) i = 0;
    if (meet || (tiles <= 12 && (tiles + 3) * (sms - items) <= (6 + items / 32) * sms)) {
      t.cluster = 1 << i;
      t.blocks = (unsigned)(items << i);
      t.bytes = 0;
      return t;
    }
  }
  const int64_t runs = ((tiles + amk::kUnitCost) * items + kMinTiles - 1) / kMinTiles;
  t.blocks = (unsigned)(runs < sms ? runs : sms);
  t.bytes = (size_t)2 * t.blocks * t.part_rows * (a.head_dim + 2) * 4;
  return t;
}

amk_status check_heads(const Reason& fail, uint32_t hd, uint32_t nq, uint32_t nkv, float scale) {
  if (hd != 64 && hd != 128) return fail(AMK_ERR_UNSUPPORTED, "head_dim %u: 64 or 128", hd);
  if (!nq || !nkv || nq % nkv || nq / nkv > 16 || nq > 4096)
    return fail(AMK_ERR_UNSUPPORTED, "%u query heads on %u kv heads: a multiple, at most 16 to one and 4096", nq, nkv);
  if (!(scale >= 0.f) || isinf(scale * amk::kLog2e))
    return fail(AMK_ERR_INVALID_ARG, "scale must be positive, or 0, and its product with log2 e finite");
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
  if ((a->n_slots / (double)amk::kTile + 2 + amk::kUnitCost) * a->n_kv_heads * a->n_seqs *
          (a->n_rows * 16.0 / amk::kTile + 1) > 0x7fffffff)
    return fail(AMK_ERR_UNSUPPORTED, "%u sequences of %u slots: more than 2^31 pieces of work", a->n_seqs, a->n_slots);
  return AMK_OK;
}

// Everything about a call of the weights that can be known without its data.
amk_status check_weights(const Reason& fail, const amk_attention_weights_args* a) {
  if (!a) return fail(AMK_ERR_INVALID_ARG, "NULL arguments");
  if (a->struct_size != sizeof *a)
    return fail(AMK_ERR_INVALID_ARG, "struct_size %u, the library has %zu", a->struct_size, sizeof *a);
  AMK_TRY(check_heads(fail, a->head_dim, a->n_q_heads, a->n_kv_heads, a->scale));
  if (a->kv_dtype > AMK_KV_FP8_E4M3) return fail(AMK_ERR_UNSUPPORTED, "kv_dtype %u", a->kv_dtype);
  if (!(fabsf(a->decay) < INFINITY)) return fail(AMK_ERR_INVALID_ARG, "decay must be finite");
  if (a->n_rows < 1 || a->n_slots < a->n_rows || a->n_slots > 0x7fffffff - 1024)
    return fail(AMK_ERR_INVALID_ARG, "%u slots for %u tokens", a->n_slots, a->n_rows);
  if (a->n_seqs > 65535) return fail(AMK_ERR_UNSUPPORTED, "%u sequences: at most 65535", a->n_seqs);
  // (tiles hold whole tokens: 64 rows at least)
  if ((a->n_slots / (double)amk::kTile + 2) * a->n_kv_heads * a->n_seqs * (a->n_rows * (a->n_q_heads / a->n_kv_heads) / 64.0 + 1) > 0x7fffffff)
    return fail(AMK_ERR_UNSUPPORTED, "%u sequences of %u tokens over %u slots: more than 2^31 pieces of work", a->n_seqs, a->n_rows,
                a->n_slots);
  return AMK_OK;
}

// How a call of the weights is divided: few rows (all of a kv head's in one tile) or many.
struct WeightsPlan {
  int q_stages, k_stages, raw_stages;   // tiles in shared memory
  int tokens, q_tiles, columns;    // tokens of a tile of query rows, tiles, rows of a tile up to a multiple of 32
  unsigned blocks;
  size_t bytes;                    // scratch: parts of units
};
WeightsPlan weights_plan(const amk_attention_weights_args& a) {
  WeightsPlan t;
  const int rep = (int)(a.n_q_heads / a.n_kv_heads), most = amk::kTile / rep;
  t.tokens = (int64_t)a.n_rows < most ? (int)a.n_rows : most;
  t.q_tiles = (int)((a.n_rows + t.tokens - 1) / t.tokens);
  t.columns = (t.tokens * rep + 31) / 32 * 32;
  const bool many = t.q_tiles > 1;
  const int twice = a.head_dim == 64 ? 2 : 1;
  if (a.kv_dtype == AMK_KV_FP8_E4M3) {
    t.k_stages = (many ? 1 : 2) * twice, t.q_stages = (many ? 3 : 2) * twice, t.raw_stages = (many ? 2 : 4) * twice;
  } else {
    t.k_stages = (many ? 2 : 4) * twice, t.q_stages = (many ? 3 : 2) * twice, t.raw_stages = 0;
  }
  const double span = (many ? amk::kManySpan : amk::kTile), steps = (a.n_slots / span + 1) * a.n_kv_heads * a.n_seqs * t.q_tiles;
  const int sms = sm_count();
  t.blocks = (unsigned)(steps < sms ? (steps < 1 ? 1 : steps) : sms);
  t.bytes = many ? (size_t)2 * t.blocks * (sizeof(int4) + amk::kManySpan * sizeof(float)) : 0;
  return t;
}

// The queries as {element, head of the group, kv head, token, sequence}; a box: 64 elements of all heads of a group and the
// tokens of a tile, which lie one behind the other as its rows.
bool make_query_map(CUtensorMap* map, const amk_attention_weights_args& a, int rep, int tokens) {
  const EncodeTiled encode = encode_tiled();
  if (!encode) return false;
  const cuuint64_t dims[5] = {a.head_dim, (cuuint64_t)rep, a.n_kv_heads, a.n_rows, a.n_seqs};
  const cuuint64_t strides[4] = {(cuuint64_t)a.q_head * 2, (cuuint64_t)a.q_head * rep * 2, (cuuint64_t)a.q_row * 2,
                                 (cuuint64_t)a.q_seq * 2};
  const cuuint32_t box[5] = {64, (cuuint32_t)rep, 1, (cuuint32_t)tokens, 1}, steps[5] = {1, 1, 1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(a.q), dims, strides, box, steps,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int HD, bool FP8>
cudaError_t launch_weights(const amk::WeightsParams& p, const CUtensorMap& q, const CUtensorMap& k, unsigned blocks, cudaStream_t st) {
  constexpr int kBytes = amk::WeightsSmem<HD, FP8, amk::kTile>::kBytes;             // (the same for both)
  static std::atomic<unsigned long long> done{0};      // devices on which the kernels' shared-memory limits are raised
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
  if (!(done.load(std::memory_order_acquire) & bit)) {
    e = cudaFuncSetAttribute(amk::weights_few_kernel<HD, FP8>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(amk::weights_many_kernel<HD, FP8>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (e != cudaSuccess) return e;
    done.fetch_or(bit, std::memory_order_release);
  }
  if (p.q_tiles > 1) return amk::launch_early(amk::weights_many_kernel<HD, FP8>, dim3(blocks), amk::kManyThreads, kBytes, 1, st, p, q, k);
  return amk::launch_early(amk::weights_few_kernel<HD, FP8>, dim3(blocks), amk::kFewThreads<FP8>, kBytes, 1, st, p, q, k);
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
  if (a.total < 0 || a.total > 0x7fffffff - 1024 || a.n_seqs > 0x7fffffff - 1024)
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
  AttnParams p{};
  p.q = (const unsigned short*)a.q, p.out = (__nv_bfloat16*)a.out, p.lse = a.lse, p.lens = a.cu_seqlens;
  p.q_row = a.q_row, p.q_head = a.q_head, p.o_row = a.out_row, p.o_head = a.out_head;
  p.n_seqs = (int)a.n_seqs, p.nq = (int)a.n_q_heads, p.nkv = (int)a.n_kv_heads, p.rep = p.nq / p.nkv;
  p.rep_inv = p.rep == 1 ? 0 : (unsigned)(((1ull << 32) + p.rep - 1) / p.rep);
  p.rows = (int)a.total;
  p.scale = a.scale > 0.f ? a.scale : 1.f / sqrtf((float)hd);
  set_limits(p);
  // blocks of 256 / rep tokens: every prompt may leave one that is not full
  const int64_t blocks = (a.total / (2 * amk::kTile / p.rep) + (a.total < a.n_seqs ? a.total : a.n_seqs)) * p.nkv;
  if (blocks > 0x7fffffff) return fail(AMK_ERR_UNSUPPORTED, "%lld blocks of queries", (long long)blocks);
  CUtensorMap mk, mv;
  if (!make_map(&mk, a.k, false, hd, a.total, p.nkv, 1, a.k_row, a.k_head, hd) ||
      !make_map(&mv, a.v, false, hd, a.total, p.nkv, 1, a.v_row, a.v_head, hd))
    return fail(AMK_ERR_CUDA, "cuTensorMapEncodeTiled failed or is missing");
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  const cudaError_t e = hd == 64 ? launch_attn<64, false, false>(p, mk, mv, (unsigned)blocks, st)
                                 : launch_attn<128, false, false>(p, mk, mv, (unsigned)blocks, st);
  return e == cudaSuccess ? AMK_OK : fail(AMK_ERR_CUDA, "launch failed: %s", cudaGetErrorString(e));
}

extern "C" amk_status amk_tree_workspace_bytes(const amk_tree_args* args, size_t* bytes, char* msg,
                                               size_t msg_bytes) {
  const Reason fail(msg, msg_bytes, "amk_tree_workspace_bytes");
  if (!bytes) return fail(AMK_ERR_INVALID_ARG, "NULL pointer");
  AMK_TRY(check_tree(fail, args));
  *bytes = tree_plan(*args).bytes;
  return AMK_OK;
}

extern "C" amk_status amk_operator_status(amk_status* st, char* msg, size_t msg_bytes, void* cuda_stream) {
  const Reason fail(msg, msg_bytes, "amk_operator_status");
  if (!st) return fail(AMK_ERR_INVALID_ARG, "NULL pointer");
  *st = AMK_OK;
  unsigned expired[2] = {0, 0};                        // how often, and how many were told of
  cudaError_t e = cudaStreamSynchronize((cudaStream_t)cuda_stream);
  if (e == cudaSuccess)
    e = cudaMemcpyFromSymbolAsync(expired, amk::g_attn_expired, 8, 0, cudaMemcpyDeviceToHost, (cudaStream_t)cuda_stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize((cudaStream_t)cuda_stream);
  if (e == cudaSuccess && expired[0] != expired[1]) {
    e = cudaMemcpyToSymbolAsync(amk::g_attn_expired, &expired[0], 4, 4, cudaMemcpyHostToDevice, (cudaStream_t)cuda_stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize((cudaStream_t)cuda_stream);
    *st = AMK_ERR_TIMEOUT;
  }
  return e == cudaSuccess ? AMK_OK : fail(AMK_ERR_CUDA, "%s", cudaGetErrorString(e));
}

extern "C" amk_status amk_debug_operator_wait(uint32_t cycles, uint32_t tiles) {
  if (cycles > amk::kWaitCycles) return AMK_ERR_INVALID_ARG;
  g_wait_cycles.store(cycles ? cycles : amk::kWaitCycles, std::memory_order_relaxed);
  g_tiles.store(tiles, std::memory_order_relaxed);
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
  const TreePlan t = tree_plan(a);
  if (t.bytes && (!a.workspace || a.workspace_bytes < t.bytes))
    return fail(AMK_ERR_INVALID_ARG, "workspace of %llu bytes, %zu are needed", (unsigned long long)(a.workspace ? a.workspace_bytes : 0),
                t.bytes);
  AttnParams p{};
  p.q = (const unsigned short*)a.q, p.out = (__nv_bfloat16*)a.out, p.lse = a.lse, p.lens = a.cache_len;
  p.mask = (const unsigned long long*)a.mask;
  p.part_o = (float*)a.workspace, p.part_lse = p.part_o + (size_t)2 * t.blocks * t.part_rows * a.head_dim;
  p.q_seq = a.q_seq, p.q_row = a.q_row, p.q_head = a.q_head;
  p.o_seq = a.out_seq, p.o_row = a.out_row, p.o_head = a.out_head;
  p.n_seqs = (int)a.n_seqs, p.nq = (int)a.n_q_heads, p.nkv = (int)a.n_kv_heads, p.rep = p.nq / p.nkv;
  p.rep_inv = p.rep == 1 ? 0 : (unsigned)(((1ull << 32) + p.rep - 1) / p.rep);
  p.rows = (int)a.n_rows, p.slots = (int)a.n_slots;
  p.part_rows = t.part_rows, p.row_tiles = t.row_tiles, p.min_tiles = kMinTiles, p.cluster = t.cluster;
  p.scale = a.scale > 0.f ? a.scale : 1.f / sqrtf((float)hd);
  set_limits(p);
  const bool fp8 = esz == 1;
  CUtensorMap mk, mv;
  if (!make_map(&mk, a.k, fp8, hd, a.n_slots, p.nkv, a.n_seqs, a.k_row, a.k_head, a.k_seq) ||
      !make_map(&mv, a.v, fp8, hd, a.n_slots, p.nkv, a.n_seqs, a.v_row, a.v_head, a.v_seq))
    return fail(AMK_ERR_CUDA, "cuTensorMapEncodeTiled failed or is missing");
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  cudaError_t e;
  if (hd == 64)
    e = fp8 ? launch_attn<64, true, true>(p, mk, mv, t.blocks, st) : launch_attn<64, true, false>(p, mk, mv, t.blocks, st);
  else
    e = fp8 ? launch_attn<128, true, true>(p, mk, mv, t.blocks, st) : launch_attn<128, true, false>(p, mk, mv, t.blocks, st);
  if (e == cudaSuccess && !t.cluster) e = hd == 64 ? launch_join<64>(p, t.blocks, st) : launch_join<128>(p, t.blocks, st);
  return e == cudaSuccess ? AMK_OK : fail(AMK_ERR_CUDA, "launch failed: %s", cudaGetErrorString(e));
}

extern "C" amk_status amk_attention_weights_workspace_bytes(const amk_attention_weights_args* args, size_t* bytes, char* msg,
                                                            size_t msg_bytes) {
  const Reason fail(msg, msg_bytes, "amk_attention_weights_workspace_bytes");
  if (!bytes) return fail(AMK_ERR_INVALID_ARG, "NULL pointer");
  AMK_TRY(check_weights(fail, args));
  *bytes = weights_plan(*args).bytes;
  return AMK_OK;
}

extern "C" amk_status amk_attention_weights(const amk_attention_weights_args* args, char* msg, size_t msg_bytes,
                                            void* cuda_stream) {
  const Reason fail(msg, msg_bytes, "amk_attention_weights");
  AMK_TRY(check_weights(fail, args));
  amk_attention_weights_args a = *args;
  if (a.n_seqs == 0) return AMK_OK;
  if (a.decay == 0.f) a.before = nullptr;
  if (!a.q || !a.k || !a.lse || !a.cache_len || !a.out) return fail(AMK_ERR_INVALID_ARG, "NULL pointer");
  if (!amk::aligned(a.q, 16) || !amk::aligned(a.k, 16) || !amk::aligned(a.lse, 4) || !amk::aligned(a.cache_len, 4) ||
      !amk::aligned(a.before, 4) || !amk::aligned(a.out, 4) || !amk::aligned(a.workspace, 256))
    return fail(AMK_ERR_INVALID_ARG, "q and k must be 16-byte, lse, cache_len, before and out 4-byte, workspace 256-byte aligned");
  const int64_t hd = a.head_dim;
  const int esz = a.kv_dtype == AMK_KV_FP8_E4M3 ? 1 : 2;
  AMK_TRY(check_stride(fail, "q sequence", a.n_seqs, &a.q_seq, hd, 2));
  AMK_TRY(check_stride(fail, "q row", a.n_rows, &a.q_row, hd, 2));
  AMK_TRY(check_stride(fail, "q head", a.n_q_heads, &a.q_head, hd, 2));
  AMK_TRY(check_stride(fail, "k sequence", a.n_seqs, &a.k_seq, hd, esz));
  AMK_TRY(check_stride(fail, "k head", a.n_kv_heads, &a.k_head, hd, esz));
  AMK_TRY(check_stride(fail, "k row", a.n_slots, &a.k_row, hd, esz));
  int64_t* sums[] = {&a.out_seq, &a.out_head, &a.before_seq, &a.before_head};
  for (int i = 0; i < (a.before ? 4 : 2); i++) {
    if ((i & 1 ? a.n_kv_heads : a.n_seqs) <= 1) *sums[i] = a.n_slots;
    if (*sums[i] < a.n_slots || *sums[i] > (int64_t)1 << 36)
      return fail(AMK_ERR_INVALID_ARG, "stride %lld of the sums: at least the %u slots", (long long)*sums[i], a.n_slots);
  }
  if (a.before == a.out && (a.before_seq != a.out_seq || a.before_head != a.out_head))
    return fail(AMK_ERR_INVALID_ARG, "out is before, but at other strides");
  const WeightsPlan t = weights_plan(a);
  if (t.bytes && (!a.workspace || a.workspace_bytes < t.bytes))
    return fail(AMK_ERR_INVALID_ARG, "workspace of %llu bytes, %zu are needed", (unsigned long long)(a.workspace ? a.workspace_bytes : 0),
                t.bytes);
  amk::WeightsParams p{};
  p.lse = a.lse, p.lens = a.cache_len, p.before = a.before, p.out = a.out;
  if (t.bytes) p.part_of = (int4*)a.workspace, p.part = (float*)(p.part_of + 2 * t.blocks);
  p.b_seq = a.before_seq, p.b_head = a.before_head, p.o_seq = a.out_seq, p.o_head = a.out_head;
  p.n_seqs = (int)a.n_seqs, p.nq = (int)a.n_q_heads, p.nkv = (int)a.n_kv_heads, p.rep = p.nq / p.nkv;
  p.rows = (int)a.n_rows, p.slots = (int)a.n_slots;
  p.tokens = t.tokens, p.q_tiles = t.q_tiles, p.columns = t.columns;
  p.rep_inv = p.rep == 1 ? 0 : (unsigned)(((1ull << 32) + p.rep - 1) / p.rep);
  p.q_stages = t.q_stages, p.k_stages = t.k_stages, p.raw_stages = t.raw_stages;
  p.scale = a.scale > 0.f ? a.scale : 1.f / sqrtf((float)hd), p.decay = a.decay;
  set_limits(p);
  CUtensorMap mq, mk;
  if (!make_query_map(&mq, a, p.rep, t.tokens) ||
      !make_map(&mk, a.k, esz == 1, hd, a.n_slots, p.nkv, a.n_seqs, a.k_row, a.k_head, a.k_seq, t.q_tiles > 1 ? amk::kManySpan : amk::kTile))
    return fail(AMK_ERR_CUDA, "cuTensorMapEncodeTiled failed or is missing");
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  cudaError_t e = hd == 64 ? (esz == 1 ? launch_weights<64, true>(p, mq, mk, t.blocks, st) : launch_weights<64, false>(p, mq, mk, t.blocks, st))
                           : (esz == 1 ? launch_weights<128, true>(p, mq, mk, t.blocks, st) : launch_weights<128, false>(p, mq, mk, t.blocks, st));
  if (e == cudaSuccess && t.bytes)
    e = amk::launch_early(amk::weights_join_kernel, dim3(t.blocks), amk::kManySpan, 0, 1, st, p, (int)t.blocks);
  return e == cudaSuccess ? AMK_OK : fail(AMK_ERR_CUDA, "launch failed: %s", cudaGetErrorString(e));
}
