// The kernels of amk_attention_weights: what the queries of some tokens attend to, added up for each cached position.
//
// Mathematics.  With the log-sum-exps known there is no maximum to find: w(j) = sum over the query rows (a row is a token and one
// of the query heads of a kv head) of 2^(S c - L), c = scale log2 e, L = lse log2 e.
//
// Few rows (128 or less for a kv head: a decoded token, a draft, the last tokens of a prompt): every K tile of 128 positions meets
// one tile of queries, and what counts is K's way from HBM.  weights_few_kernel takes S^T = K Q^T: a position is a lane of TMEM.
// (32 tokens, 32 heads of 128 on 8, four caches of 4097 to 8001 positions: 51 MB in 15.7 us, eleven tiles a block.  Blocks of 1 / 2 / 4 /
// 8 / 16 tiles from HBM take 6.6 / 7.6 / 9.5 / 13.2 / 19.8 us: 5.7 us for the launch, the division, the first tile and the last
// output, and 0.9 us a tile, 0.77 at the rate of a copy.  13 tokens over eight 8-bit caches: 45 MB in 22.7 us, the tiles' widening.)
//
// Many rows: what counts are the exponentials, 16 a cycle and SM, twice as long as the products.  weights_many_kernel takes
// S = Q K^T: a query row is a lane, whose L is a scalar, and a thread keeps the sums of 40 positions in registers over all
// query tiles of a unit; lanes are added up once, at its end.  (7001 tokens, 32 heads of 128 on 8, 784 M exponentials: 248 us, 74 % of
// their unit's rate; with the positions in the lanes there too, where every column's L is read from shared memory, 257 us.  A
// share of the exponentials as a polynomial on the fma pipe gained nothing in either: 250 / 260 / 271 us at none, an eighth and a
// quarter; the issue of instructions, 6.5 for each exponential, and the waits between them are what is left.  Over an 8-bit cache
// the same warps widen the tiles: 297 us.)
#pragma once
#include "amk_attn.cuh"
#include "amk_weights_units.h"

namespace amk {

static_assert(kFewSpan == kTile, "few rows: a unit is a tile");
struct WeightsParams : WeightsWork {
  const float* lse;
  const float* before;
  float* out;
  float* part;                     // many rows: [2 * gridDim][160]: sums of cut units
  int4* part_of;                   // [2 * gridDim]: {sequence, head, unit, whether the next block goes on}; sequence -1: none
  int64_t b_seq, b_head, o_seq, o_head;
  int nq, rep;
  int q_stages, k_stages, raw_stages;   // tiles in shared memory
  int columns;                     // few rows: rows of the tile, up to a multiple of 32
  unsigned rep_inv;                // ceil(2^32 / rep), 0 for rep = 1
  unsigned tiles;                  // K tiles that a block may ask for (a test's limit, else the largest number)
  unsigned wait_cycles;
  float scale, decay;
};

// One box of a five-dimensional tensor map, as tma_load_4d.
__device__ __forceinline__ void tma_load_5d(bool leader, void* dst, const CUtensorMap* map, int x, int y, int z, int w, int v,
                                            uint64_t* bar) {
  asm volatile(
      "{ .reg .pred q; setp.ne.u32 q, %8, 0;\n"
      "  @q cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2,%3,%4,%5,%6}], [%7]; }" ::"r"(
          smem_u32(dst)),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(v), "r"(smem_u32(bar)), "r"((unsigned)leader)
      : "memory");
}

// A tile of e4m3 codes to bf16 (both exact), laid out as the matrix instructions want it: chunks of 16 codes from `first` on, every
// `threads`-th.  Over f16, for which there is one instruction for two codes (128 x 128 codes, eight warps: 650 cycles; by shifts
// and a product with 2^120: 1130).  Half of a row's lanes store their second piece first: they lie in the same banks.
template <int HD, int ROWS, int BATCH>
__device__ __forceinline__ void widen_tile(unsigned char* dst, const unsigned char* src, int first, int threads) {
  constexpr int kChunks = HD / 16;                     // of a row
  for (int i0 = first; i0 < ROWS * kChunks; i0 += threads * BATCH) {
    uint4 v[BATCH];
#pragma unroll
    for (int b = 0; b < BATCH; b++)
      if (i0 + b * threads < ROWS * kChunks) v[b] = *(const uint4*)(src + (i0 + b * threads) * 16);
#pragma unroll
    for (int b = 0; b < BATCH; b++) {
      const int i = i0 + b * threads;
      if (i >= ROWS * kChunks) break;
      const unsigned c[4] = {v[b].x, v[b].y, v[b].z, v[b].w};
      unsigned w[8];
#pragma unroll
      for (int k = 0; k < 4; k++) {
        unsigned h[2];
        widen_e4m3(h, c[k]);
        float lo, hi;
        unpack_f16(lo, hi, h[0]);
        w[2 * k] = pack_bf16(lo, hi);
        unpack_f16(lo, hi, h[1]);
        w[2 * k + 1] = pack_bf16(lo, hi);
      }
      const int row = i / kChunks, cc = i % kChunks * 2, swap = cc >> 3 & 1;
      unsigned char* to = dst + (cc >> 3) * (ROWS * 128) + row * 128;
      const uint4 x = make_uint4(w[0], w[1], w[2], w[3]), y = make_uint4(w[4], w[5], w[6], w[7]);
      *(uint4*)(to + ((((cc & 7) + swap) ^ (row & 7)) << 4)) = swap ? y : x;
      *(uint4*)(to + ((((cc & 7) + 1 - swap) ^ (row & 7)) << 4)) = swap ? x : y;
    }
  }
}

// a position's sum, finished
__device__ __forceinline__ void weights_write(const WeightsParams& p, int seq, int head, int len, int key, float sum) {
  if (key >= p.slots) return;
  if (key >= len + p.rows) sum = 0.f;
  if (key < len && p.before) sum = fmaf(p.decay, p.before[seq * p.b_seq + head * p.b_head + key], sum);
  p.out[seq * p.o_seq + head * p.o_head + key] = sum;
}

// ---- runs -------------------------------------------------------------------------------------------------------
// Where this block's run begins, and its steps (one whole warp): {sequence, head, unit, step, steps, length of the sequence}
template <int SPAN>
__device__ __forceinline__ void find_run(const WeightsParams& p, int* start) {
  const int lane = threadIdx.x & 31;
  auto steps_of = [&](int s) { return s < p.n_seqs ? weights_steps<SPAN>(p, __ldg(p.lens + s)) * p.nkv : 0; };
  const int mine = steps_of(lane);
  int total = mine;
  for (int s = 32 + lane; s < p.n_seqs; s += 32) total += steps_of(s);
  total = warp_sum(total);
  const int per = (total + (int)gridDim.x - 1) / (int)gridDim.x;
  int at = (int)blockIdx.x * per, seq = 0, head = 0, unit = 0, step = 0, left = 0, len = 0;
  if ((int64_t)blockIdx.x * per < total) {
    left = min(per, total - at);
    for (int s0 = 0; s0 < p.n_seqs; s0 += 32) {
      const int own = s0 ? steps_of(s0 + lane) : mine;
      int n = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(~0u, n, o);
        if (lane >= o) n += x;
      }
      const unsigned hit = __ballot_sync(~0u, n > at);
      if (hit) {
        const int f = __ffs(hit) - 1;
        seq = s0 + f;
        int rel = at - __shfl_sync(~0u, n - own, f);
        const int of_head = __shfl_sync(~0u, own, f) / p.nkv;
        len = __ldg(p.lens + seq);
        head = rel / of_head, rel -= head * of_head;
        weights_place<SPAN>(p, len, rel, unit, step);
        break;
      }
      at -= __shfl_sync(~0u, n, 31);
    }
  }
  if (lane == 0) start[0] = seq, start[1] = head, start[2] = unit, start[3] = step, start[4] = left, start[5] = len;
}
// Slots behind the units, and sequences of an impossible length.
template <int SPAN>
__device__ __forceinline__ void fill_behind(const WeightsParams& p, int threads) {
  for (int r = blockIdx.x; r < p.n_seqs * p.nkv; r += gridDim.x) {
    const int s = r / p.nkv, units = weights_units<SPAN>(p, __ldg(p.lens + s));
    float* out = p.out + s * p.o_seq + (r - s * p.nkv) * p.o_head;
    for (int64_t i = (int64_t)units * SPAN + threadIdx.x; i < p.slots; i += threads) out[i] = units ? 0.f : CUDART_NAN_F;
  }
}

// ---- shared memory ----------------------------------------------------------------------------------------------
// 192 KB divided between Q tiles (128 rows), K tiles (SPAN rows) and, over the 8-bit cache, K tiles as they come.  With few rows the K
// tiles are what streams, else the Q tiles: a tile is on its way for 1.5 us, and the ring that streams has to hold what the
// others need meanwhile.
constexpr int kMaxStages = 10;
template <int HD, bool FP8, int SPAN>
struct WeightsSmem {
  static constexpr int kTileBytes = HD / 64 * kBox, kBoxK = 64 * SPAN * 2, kBytesK = HD / 64 * kBoxK;
  static constexpr int kRawBytes = FP8 ? HD * SPAN : 0;
  static constexpr int kHead = 192 * 1024, kHeadBytes = 16384;
  static constexpr int kBytes = kHead + kHeadBytes + 1024;         // + alignment of the dynamic buffer
  static_assert(kBytes <= 227 * 1024, "shared memory of one SM");
};
struct WeightsHead {
  uint64_t k_full[kMaxStages], k_empty[kMaxStages], raw_full[kMaxStages], raw_empty[kMaxStages], q_full[kMaxStages], q_empty[kMaxStages];
  uint64_t s_full[4], s_empty[4], fin;
  unsigned tmem;
  int dead;
  unsigned wait_cycles;
  int start[6];                        // where the block's run begins
  alignas(16) float less[12][kTile];   // few rows: [warp]: -lse log2 e of the rows; -infinity: adds nothing
  alignas(16) float sums[4][4][40];    // many rows: [warpgroup][warp]: sums of its 32 rows
};
static_assert(sizeof(WeightsHead) <= 16384, "head");
// a place in a ring of tiles and the parity of its round
struct RingAt {
  int at = 0;
  unsigned round = 0;
  __device__ __forceinline__ void next(int n) {
    if (++at == n) at = 0, round ^= 1;
  }
};

// What both kernels begin with.  widen_arrivals, s_arrivals: warps that arrive at a widened tile and at a free accumulator.
template <int HD, bool FP8>
__device__ __forceinline__ void weights_begin(const WeightsParams& p, WeightsHead& h, unsigned char* smem, int issuer_warp, int warp,
                                              int lane, int widen_arrivals, int s_arrivals, int threads) {
  if (warp == issuer_warp) {
    tmem_alloc(&h.tmem, 512);
    if (lane == 0) {
      for (int i = 0; i < p.k_stages; i++) mbar_init(&h.k_full[i], FP8 ? widen_arrivals : 1), mbar_init(&h.k_empty[i], 1);
      for (int i = 0; i < p.raw_stages; i++) mbar_init(&h.raw_full[i], 1), mbar_init(&h.raw_empty[i], widen_arrivals);
      for (int i = 0; i < p.q_stages; i++) mbar_init(&h.q_full[i], 1), mbar_init(&h.q_empty[i], 1);
      for (int i = 0; i < 4; i++) mbar_init(&h.s_full[i], 1), mbar_init(&h.s_empty[i], s_arrivals);
      mbar_init(&h.fin, 1);
      h.dead = 0, h.wait_cycles = p.wait_cycles;
      mbar_fence_init();
    }
  }
  // rows of a Q tile that no box fills
  const int filled = p.tokens * p.rep * 8;
  if (filled < kTile * 8) {
    for (int i = threadIdx.x; i < p.q_stages * HD / 64 * kBox / 16; i += threads)
      if (i % (kBox / 16) >= filled) ((uint4*)smem)[i] = make_uint4(0, 0, 0, 0);
    fence_async_smem();
  }
}
// The producer's K tile of SPAN positions from key0 on.
template <int HD, bool FP8, int SPAN>
__device__ __forceinline__ void ask_for_k(bool leader, const CUtensorMap* map, unsigned char* k_tiles, unsigned char* raw_tiles, int at,
                                          int key0, int head, int seq, uint64_t* full) {
  using L = WeightsSmem<HD, FP8, SPAN>;
  expect_tx(leader, full, FP8 ? L::kRawBytes : L::kBytesK);
  if (FP8) {
    tma_load_4d(leader, raw_tiles + at * L::kRawBytes, map, 0, key0, head, seq, full);
  } else {
#pragma unroll
    for (int x = 0; x < HD; x += 64) tma_load_4d(leader, k_tiles + at * L::kBytesK + x / 64 * L::kBoxK, map, x, key0, head, seq, full);
  }
}
template <int HD, bool FP8>
__device__ __forceinline__ void ask_for_q(bool leader, const WeightsParams& p, const CUtensorMap* map, unsigned char* smem, int at, int head,
                                          int tok0, int seq, uint64_t* full) {
  expect_tx(leader, full, (unsigned)(p.tokens * p.rep) * HD * 2);
#pragma unroll
  for (int x = 0; x < HD; x += 64) tma_load_5d(leader, smem + at * HD / 64 * kBox + x / 64 * kBox, map, x, 0, head, tok0, seq, full);
}
// The block's end, behind a barrier: if a wait ran out, copies and products in flight end (waits again, with a limit) before their
// memory is given back.
__device__ __noinline__ void weights_end(WeightsHead& h, int warp, int producer, uint64_t* k_full, unsigned k_asked, unsigned k_stages,
                                         unsigned q_asked, unsigned q_stages) {
  if (h.dead) {
    if (warp == producer) {
      const auto drain = [&](uint64_t* full, unsigned asked, unsigned stages) {
        for (unsigned i = asked > stages ? asked - stages : 0; i < asked; i++)
          for (int n = 0; n < 1 << 16 && !__all_sync(~0u, mbar_try_wait(&full[i % stages], i / stages & 1)); n++) {}
      };
      drain(k_full, k_asked, k_stages);
      drain(h.q_full, q_asked, q_stages);
    }
    if (warp == producer + 1) {
      mma_commit(elect_one(), &h.fin);
      for (int n = 0; n < 1 << 16 && !__all_sync(~0u, mbar_try_wait(&h.fin, 0)); n++) {}
    }
    __syncthreads();
  }
  if (warp == producer + 1) tmem_free(h.tmem, 512);
}

// ---- few rows ---------------------------------------------------------------------------------------------------
// The sum of a tile with values that are not finite, element by element: what is left out or hidden must not come in.
__device__ __noinline__ float weights_careful(unsigned ts, const float* less, int columns, int from, float c) {
  float sum = 0.f;
  for (int x = 0; x < columns; x += 32) {
    unsigned w[32];
    tmem_ld32(w, ts + x);
    tmem_wait_ld();
    tmem_pin(w);
#pragma unroll
    for (int k = 0; k < 32; k++) {
      const float l = less[x + k];
      if (x + k >= from && l != -CUDART_INF_F) sum += exp2_fast(fmaf(__uint_as_float(w[k]), c, l));
    }
  }
  return sum;
}
// What a thread adds up of 16 positions (lanes of TMEM) and 32 columns: it has two columns of every eight, of positions l / 4 (acc[0])
// and l / 4 + 8 (acc[1]).  So a column's `less` is read once for eight positions and not for each.  less: this lane's first.
// Positions see the columns from `from` on only, counted from this lane's first.
__device__ __forceinline__ void add_columns(uint64_t (&acc)[2], const unsigned (&w)[16], const float* less, uint64_t c2, bool hides, int from0,
                                            int from1) {
#pragma unroll
  for (int b = 0; b < 4; b++) {
    const float2 l = *(const float2*)(less + 8 * b);
#pragma unroll
    for (int g = 0; g < 2; g++) {
      float e0, e1;
      unpair(e0, e1, fma2(pair(__uint_as_float(w[4 * b + 2 * g]), __uint_as_float(w[4 * b + 2 * g + 1])), c2, pair(l.x, l.y)));
      e0 = exp2_fast(e0), e1 = exp2_fast(e1);
      if (hides) {
        const int from = g ? from1 : from0;
        if (8 * b < from) e0 = 0.f;
        if (8 * b + 1 < from) e1 = 0.f;
      }
      acc[g] = add2(acc[g], pair(e0, e1));
    }
  }
}

constexpr int kFewGroups = 3, kWideners = 8;           // warpgroups for the exponentials, warps that widen 8-bit tiles
template <bool FP8>
constexpr int kFewThreads = 32 * (4 * kFewGroups + 2 + (FP8 ? kWideners : 0));

// A producer warp brings K tiles, and Q once a head, by TMA, one warp issues the products into four accumulators in turn, three
// warpgroups take every third product each, so that the next one is there when they have done one.
template <int HD, bool FP8>
__global__ void __launch_bounds__(kFewThreads<FP8>, 1)
    weights_few_kernel(const WeightsParams p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k) {
  using L = WeightsSmem<HD, FP8, kTile>;
  constexpr int kProducer = 4 * kFewGroups, kIssuer = kProducer + 1;
  unsigned char* smem = attn_smem();
  WeightsHead& h = *(WeightsHead*)(smem + L::kHead);
  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  weights_begin<HD, FP8>(p, h, smem, kIssuer, warp, lane, kWideners, 4, kFewThreads<FP8>);
  if (warp == kProducer) prefetch_map(lane == 0, &map_q), prefetch_map(lane == 0, &map_k);
  wait_for_grid_before();
  if (warp == 0) find_run<kTile>(p, h.start);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const unsigned tmem = uniform(h.tmem);
  unsigned k_asked = 0, q_asked = 0;                   // the producer's
  unsigned char *k_tiles = smem + p.q_stages * L::kTileBytes, *raw_tiles = k_tiles + p.k_stages * L::kTileBytes;
  WeightsWalk<kTile> walk;
  walk.init(p, h.start);
  WeightsUnit u;
  if (warp < kProducer) {
    // ================================ exponentials and sums ============================================================
    const int wg = warp >> 2, id = (warp & 3) * 32 + (lane >> 2) + 8 * (lane & 3);       // id: this thread's position of a tile
    const unsigned lanes = tmem + ((unsigned)(warp & 3) * 32 << 16);
    const float c = p.scale * kLog2e;
    float* row = h.less[warp];
    const float* mine_of = row + 2 * (lane & 3);
    int l_seq = -1, l_head = -1;                       // whose rows `row` has
    for (int j = 0; walk.next(p, u); j++) {
      if (j % kFewGroups != wg) continue;
      const int key0 = u.at * kTile;
      if (u.seq != l_seq || u.head != l_head) {        // every warp brings the rows for itself
        l_seq = u.seq, l_head = u.head;
        const float* lse = p.lse + (int64_t)u.seq * p.rows * p.nq + u.head * p.rep;
        float l[4];
#pragma unroll
        for (int k = 0; k < 4; k++) {
          const int r = lane + 32 * k, t = p.rep_inv ? (int)__umulhi((unsigned)r, p.rep_inv) : r;
          l[k] = t < p.rows ? __ldg(lse + (int64_t)t * p.nq + r - t * p.rep) : CUDART_INF_F;
        }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 4; k++) row[lane + 32 * k] = fabsf(l[k]) == CUDART_INF_F ? -CUDART_INF_F : -l[k] * kLog2e;
        __syncwarp();
      }
      const bool hides = key0 + kTile - 1 > u.len;
      // the first column that this lane's first position sees, less its first column; a position further on sees rep less
      const int from = hides ? (min(max(key0 - u.len, -kTile), kTile) + (warp & 3) * 32 + (lane >> 2)) * p.rep - 2 * (lane & 3) : 0;
      const unsigned ts = lanes + (j & 3) * kTile;
      attn_wait(&h.s_full[j & 3], j >> 2 & 1, h);
      __syncwarp();
      tc_fence_after();
      const uint64_t c2 = pair(c, c);
      uint64_t acc[2][2] = {};                         // [16 positions][8 of them]
      // 16 positions are on their way while 16 are worked on
      unsigned w0[16], w1[16];
      tmem_ld_16x256b_x4(w0, ts);
#pragma unroll 1
      for (int x = 0; x < p.columns; x += 32) {
        tmem_wait_ld();
        tmem_pin(w0);
        tmem_ld_16x256b_x4(w1, ts + (16 << 16) + x);
        add_columns(acc[0], w0, mine_of + x, c2, hides, from - x, from - x + 8 * p.rep);
        tmem_wait_ld();
        tmem_pin(w1);
        if (x + 32 < p.columns) tmem_ld_16x256b_x4(w0, ts + x + 32);
        add_columns(acc[1], w1, mine_of + x, c2, hides, from - x + 16 * p.rep, from - x + 24 * p.rep);
      }
      float a[4];
#pragma unroll
      for (int k = 0; k < 4; k++) {
        float lo, hi;
        unpair(lo, hi, acc[k >> 1][k & 1]);
        a[k] = lo + hi;
        a[k] += __shfl_xor_sync(~0u, a[k], 1);
        a[k] += __shfl_xor_sync(~0u, a[k], 2);
      }
      // a position for each lane: l / 4 + 8 (l % 4)
      float sum = lane & 2 ? (lane & 1 ? a[3] : a[2]) : (lane & 1 ? a[1] : a[0]);
      if (__any_sync(~0u, !(sum < CUDART_INF_F))) {
        const float s = weights_careful(ts, row, p.columns, hides ? min(max(key0 + (warp & 3) * 32 + lane - u.len, 0), kTile) * p.rep : 0, c);
        sum = __shfl_sync(~0u, s, (lane >> 2) + 8 * (lane & 3));
      }
      tc_fence_before();
      warp_arrive(&h.s_empty[j & 3], lane);
      weights_write(p, u.seq, u.head, u.len, key0 + id, sum);
    }
    fill_behind<kTile>(p, 128 * kFewGroups);
  } else if (warp == kProducer) {
    // ================================ tiles ============================================================================
    const bool leader = elect_one();
    const int n_k = FP8 ? p.raw_stages : p.k_stages;   // the ring that K comes into
    int q_seq = -1, q_head = -1;
    RingAt k, q;
    bool on = true;
    while (walk.next(p, u)) {
      uint64_t *full = FP8 ? &h.raw_full[k.at] : &h.k_full[k.at], *empty = FP8 ? &h.raw_empty[k.at] : &h.k_empty[k.at];
      on = attn_wait(empty, k.round ^ 1, h) && on && k_asked < p.tiles;
      if (on) {
        ask_for_k<HD, FP8, kTile>(leader, &map_k, k_tiles, raw_tiles, k.at, u.at * kTile, u.head, u.seq, full);
        k_asked++;
      }
      k.next(n_k);
      if (u.seq == q_seq && u.head == q_head) continue;
      q_seq = u.seq, q_head = u.head;
      on = attn_wait(&h.q_empty[q.at], q.round ^ 1, h) && on;
      if (on) {
        ask_for_q<HD, FP8>(leader, p, &map_q, smem, q.at, u.head, 0, u.seq, &h.q_full[q.at]);
        q_asked++;
      }
      q.next(p.q_stages);
    }
  } else if (warp == kIssuer) {
    // ================================ the matrix products ==============================================================
    const bool leader = elect_one();
    const unsigned id_s = mma_idesc(kTile, 0, false, false) | (unsigned)(p.columns >> 3) << 17;
    const uint64_t q_desc = smem_desc(smem_u32(smem), 16, 1024), k_desc = smem_desc(smem_u32(k_tiles), 16, 1024);
    constexpr uint64_t kTileStep = L::kTileBytes >> 4;
    int q_seq = -1, q_head = -1, held = -1;            // held: the Q tile that is worked on
    RingAt k, q;
    bool on = true;
    for (int j = 0; uniform(walk.next(p, u)); j++) {
      if (uniform(u.seq != q_seq || u.head != q_head)) {
        q_seq = u.seq, q_head = u.head;
        if (on && held >= 0) mma_commit(leader, &h.q_empty[held]);
        held = uniform(q.at);
        on = attn_wait(&h.q_full[held], q.round, h) && on;
        q.next(p.q_stages);
      }
      on = attn_wait(&h.k_full[k.at], k.round, h) && on;
      const int at = uniform(j & 3);
      on = attn_wait(&h.s_empty[at], (j >> 2 & 1) ^ 1, h) && on;
      if (on) {
        tc_fence_after();
        const uint64_t ka = k_desc + uniform(k.at) * kTileStep, qa = q_desc + held * kTileStep;
#pragma unroll
        for (int e = 0; e < HD / 16; e++) {
          const int off = (e / 4 * kBox + e % 4 * 32) >> 4;
          mma_ss(leader, tmem + at * kTile, ka + off, qa + off, id_s, e > 0);
        }
        mma_commit(leader, &h.s_full[at]);
        mma_commit(leader, &h.k_empty[k.at]);
      }
      k.next(p.k_stages);
    }
  } else if (FP8) {
    // ================================ 8-bit tiles widened to bf16 ======================================================
    const int first = (warp - kIssuer - 1) % kWideners * 32 + lane;      // (below 256, which the compiler sees: a whole number of chunks)
    RingAt raw, k;
    while (walk.next(p, u)) {
      attn_wait(&h.raw_full[raw.at], raw.round, h);
      attn_wait(&h.k_empty[k.at], k.round ^ 1, h);
      widen_tile<HD, kTile, 4>(k_tiles + k.at * L::kTileBytes, raw_tiles + raw.at * L::kRawBytes, first, 32 * kWideners);
      fence_async_smem();
      warp_arrive(&h.k_full[k.at], lane);
      warp_arrive(&h.raw_empty[raw.at], lane);
      k.next(p.k_stages), raw.next(p.raw_stages);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  weights_end(h, warp, kProducer, FP8 ? h.raw_full : h.k_full, k_asked, FP8 ? p.raw_stages : p.k_stages, q_asked, p.q_stages);
}

// ---- many rows --------------------------------------------------------------------------------------------------
// N positions' sums over this lane's row: 2^(S c + less).  Hidden: positions from `end` on.
template <int FIRST, int N>
__device__ __forceinline__ void add_row(uint64_t (&acc)[20], const unsigned (&w)[N], uint64_t c2, uint64_t less2, bool hides, int end) {
#pragma unroll
  for (int k = 0; k < N / 2; k++) {
    float e0, e1;
    unpair(e0, e1, fma2(pair(__uint_as_float(w[2 * k]), __uint_as_float(w[2 * k + 1])), c2, less2));
    e0 = exp2_fast(e0), e1 = exp2_fast(e1);
    if (hides) e0 = FIRST + 2 * k < end ? e0 : 0.f, e1 = FIRST + 2 * k + 1 < end ? e1 : 0.f;
    acc[FIRST / 2 + k] = add2(acc[FIRST / 2 + k], pair(e0, e1));
  }
}

// Lanes that differ in bit O: each keeps one half of 2 N sums, and adds the other one's.
template <int O, int N, int ALL>
__device__ __forceinline__ void exchange(float (&v)[ALL], int lane) {
  const bool upper = lane & O;
#pragma unroll
  for (int i = 0; i < N; i++) {
    const float give = upper ? v[i] : v[i + N], take = upper ? v[i + N] : v[i];
    v[i] = take + __shfl_xor_sync(~0u, give, O);
  }
}

// A unit is 160 positions, 40 for each of four warpgroups, the products of the steps in three accumulators in turn: a warp waits for
// nobody but the issuer, which is two steps ahead.  (Two accumulators of 192 positions, three warpgroups: their release, the
// product and its arrival were as long as the exponentials, 250 us; four warpgroups of 64 positions have too few registers,
// 450 us.)  A unit that a run's border cuts leaves its parts in scratch and a second kernel adds them, in the order of the blocks.
constexpr int kManyThreads = 576, kManyBuffers = 3;
template <int HD, bool FP8>
__global__ void __launch_bounds__(kManyThreads, 1)
    weights_many_kernel(const WeightsParams p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k) {
  using L = WeightsSmem<HD, FP8, kManySpan>;
  constexpr int kProducer = 16, kIssuer = 17, kSpan = kManySpan, kEach = kSpan / 4;
  unsigned char* smem = attn_smem();
  WeightsHead& h = *(WeightsHead*)(smem + L::kHead);
  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  weights_begin<HD, FP8>(p, h, smem, kIssuer, warp, lane, kProducer, kProducer, kManyThreads);
  if (warp == kProducer) prefetch_map(lane == 0, &map_q), prefetch_map(lane == 0, &map_k);
  wait_for_grid_before();
  if (warp == 0) find_run<kSpan>(p, h.start);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const unsigned tmem = uniform(h.tmem);
  unsigned k_asked = 0, q_asked = 0;                   // the producer's
  unsigned char *k_tiles = smem + p.q_stages * L::kTileBytes, *raw_tiles = k_tiles + p.k_stages * L::kBytesK;
  WeightsWalk<kSpan> walk;
  walk.init(p, h.start);
  WeightsUnit u;
  if (warp < kProducer) {
    // ================================ exponentials and sums ============================================================
    const int wg = warp >> 2, r = (warp & 3) * 32 + lane;      // r: this thread's row of a Q tile
    const unsigned lanes = tmem + ((unsigned)(warp & 3) * 32 << 16) + wg * kEach;
    const int own_tok = p.rep_inv ? (int)__umulhi((unsigned)r, p.rep_inv) : r, own_head = r - own_tok * p.rep;
    const float c = p.scale * kLog2e;
    const uint64_t c2 = pair(c, c);
    RingAt raw, k, s;                                  // s: the accumulator

    bool cut0 = false, cut1 = false;
    while (walk.next(p, u)) {
      if (FP8) {                                       // widened by all
        attn_wait(&h.raw_full[raw.at], raw.round, h);
        attn_wait(&h.k_empty[k.at], k.round ^ 1, h);
        widen_tile<HD, kSpan, 2>(k_tiles + k.at * L::kBytesK, raw_tiles + raw.at * L::kRawBytes, threadIdx.x, 32 * kProducer);
        fence_async_smem();
        warp_arrive(&h.k_full[k.at], lane);
        warp_arrive(&h.raw_empty[raw.at], lane);
        k.next(p.k_stages), raw.next(p.raw_stages);
      }
      const int base = u.at * kSpan + wg * kEach;      // first position of this warpgroup
      const float* lse = p.lse + ((int64_t)u.seq * p.rows + own_tok) * p.nq + u.head * p.rep + own_head;
      const auto lse_of = [&](int tok0) {              // of this thread's row of the tile from token tok0 on
        return own_tok < p.tokens && tok0 + own_tok < p.rows ? __ldg(lse + (int64_t)tok0 * p.nq) : CUDART_INF_F;
      };
      int tok0 = (u.first + u.begin) * p.tokens;
      float l = lse_of(tok0), l1 = u.begin + 1 < u.end ? lse_of(tok0 + p.tokens) : 0.f;     // two steps ahead
      uint64_t acc[kEach / 2];                         // sums of 40 positions
#pragma unroll
      for (int i = 0; i < kEach / 2; i++) acc[i] = 0;
      // Some columns are on their way while others are worked on.
      unsigned w0[16], w1[16], w2[8];
      const auto have = [&](auto& w) {
        tmem_wait_ld();
        tmem_pin(w);
      };
#pragma unroll 1
      for (int i = u.begin; i < u.end; i++) {
        const bool out = fabsf(l) == CUDART_INF_F;     // (a row that adds nothing sees nothing)
        const int end = out ? 0 : u.len + tok0 + own_tok + 1 - base;
        const float less = out ? -CUDART_INF_F : -l * kLog2e;
        const uint64_t less2 = pair(less, less);
        const bool hides = __any_sync(~0u, end < kEach);
        tok0 += p.tokens;
        l = l1;
        if (i + 2 < u.end) l1 = lse_of(tok0 + p.tokens);
        attn_wait(&h.s_full[s.at], s.round, h);
        __syncwarp();
        tc_fence_after();
        const unsigned ts = lanes + s.at * kSpan;
        tmem_ld16(w0, ts);
        have(w0);
        tmem_ld16(w1, ts + 16);
        add_row<0>(acc, w0, c2, less2, hides, end);
        have(w1);
        tmem_ld8(w2, ts + 32);
        add_row<16>(acc, w1, c2, less2, hides, end);
        have(w2);
        tc_fence_before();
        warp_arrive(&h.s_empty[s.at], lane);
        s.next(kManyBuffers);
        add_row<32>(acc, w2, c2, less2, hides, end);
      }
      // The 32 rows of the warp: at each exchange a lane keeps half of its positions and gives away the others; then the four warps.
      float v[32], x[8];
#pragma unroll
      for (int i = 0; i < 16; i++) unpair(v[2 * i], v[2 * i + 1], acc[i]);
#pragma unroll
      for (int i = 0; i < 4; i++) unpair(x[2 * i], x[2 * i + 1], acc[16 + i]);
      exchange<16, 16>(v, lane), exchange<8, 8>(v, lane), exchange<4, 4>(v, lane), exchange<2, 2>(v, lane), exchange<1, 1>(v, lane);
      exchange<16, 4>(x, lane), exchange<8, 2>(x, lane), exchange<4, 1>(x, lane);
      x[0] += __shfl_xor_sync(~0u, x[0], 2);
      x[0] += __shfl_xor_sync(~0u, x[0], 1);
      float* sums = h.sums[wg][warp & 3];
      sums[lane] = v[0];                               // lane l has position l
      if (!(lane & 3)) sums[32 + (lane >> 2)] = x[0];
      named_barrier(1 + wg, 128);
      const bool whole = u.begin == 0 && u.end == u.all;
      const int id = threadIdx.x & 127;
      if (id < kEach) {
        const float sum = (h.sums[wg][0][id] + h.sums[wg][1][id]) + (h.sums[wg][2][id] + h.sums[wg][3][id]);
        if (whole) {
          weights_write(p, u.seq, u.head, u.len, base + id, sum);
        } else {
          const int rec = 2 * blockIdx.x + (u.begin == 0);
          p.part[(int64_t)rec * kSpan + wg * kEach + id] = sum;
          if (id == 0 && wg == 0) p.part_of[rec] = make_int4(u.seq, u.head, u.at, u.end < u.all);
        }
      }
      named_barrier(1 + wg, 128);                      // (the sums have been read)
      if (!whole) (u.begin == 0 ? cut1 : cut0) = true;
    }
    if (threadIdx.x == 0) {
      if (!cut0) p.part_of[2 * blockIdx.x] = make_int4(-1, 0, 0, 0);
      if (!cut1) p.part_of[2 * blockIdx.x + 1] = make_int4(-1, 0, 0, 0);
    }
    fill_behind<kSpan>(p, 32 * kProducer);
  } else if (warp == kProducer) {
    // ================================ tiles ============================================================================
    const bool leader = elect_one();
    const int n_k = FP8 ? p.raw_stages : p.k_stages;   // the ring that K comes into
    RingAt k, q;
    bool on = true;
    while (walk.next(p, u)) {
      uint64_t *full = FP8 ? &h.raw_full[k.at] : &h.k_full[k.at], *empty = FP8 ? &h.raw_empty[k.at] : &h.k_empty[k.at];
      on = attn_wait(empty, k.round ^ 1, h) && on && k_asked < p.tiles;
      if (on) {
        ask_for_k<HD, FP8, kSpan>(leader, &map_k, k_tiles, raw_tiles, k.at, u.at * kSpan, u.head, u.seq, full);
        k_asked++;
      }
      k.next(n_k);
      for (int i = u.begin; i < u.end; i++) {
        on = attn_wait(&h.q_empty[q.at], q.round ^ 1, h) && on;
        if (on) {
          ask_for_q<HD, FP8>(leader, p, &map_q, smem, q.at, u.head, (u.first + i) * p.tokens, u.seq, &h.q_full[q.at]);
          q_asked++;
        }
        q.next(p.q_stages);
      }
    }
  } else if (warp == kIssuer) {
    // ================================ the matrix products ==============================================================
    const bool leader = elect_one();
    constexpr unsigned kIdS = mma_idesc(kTile, kSpan, false, false);
    const uint64_t q_desc = smem_desc(smem_u32(smem), 16, 1024), k_desc = smem_desc(smem_u32(k_tiles), 16, 1024);
    RingAt k, q, s;                                    // s: the accumulator
    bool on = true;
    while (uniform(walk.next(p, u))) {
      on = attn_wait(&h.k_full[k.at], k.round, h) && on;
      const uint64_t ka = k_desc + uniform(k.at) * (uint64_t)(L::kBytesK >> 4);
      const int n = uniform(u.end - u.begin);
      for (int i = 0; i < n; i++) {
        on = attn_wait(&h.q_full[q.at], q.round, h) && on;
        const uint64_t qa = q_desc + uniform(q.at) * (uint64_t)(L::kTileBytes >> 4);
        const int at = uniform(s.at);
        on = attn_wait(&h.s_empty[at], s.round ^ 1, h) && on;
        if (on) {
          tc_fence_after();
#pragma unroll
          for (int e = 0; e < HD / 16; e++)
            mma_ss(leader, tmem + at * kSpan, qa + ((e / 4 * kBox + e % 4 * 32) >> 4), ka + ((e / 4 * L::kBoxK + e % 4 * 32) >> 4), kIdS, e > 0);
          mma_commit(leader, &h.s_full[at]);
          mma_commit(leader, &h.q_empty[q.at]);
        }
        q.next(p.q_stages), s.next(kManyBuffers);
      }
      if (on) mma_commit(leader, &h.k_empty[k.at]);
      k.next(p.k_stages);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  weights_end(h, warp, kProducer, FP8 ? h.raw_full : h.k_full, k_asked, FP8 ? p.raw_stages : p.k_stages, q_asked, p.q_stages);
}

// The parts of units that a border cut: one block for each block of the first kernel in whose run such a unit begins.
static __global__ void __launch_bounds__(kManySpan) weights_join_kernel(const WeightsParams p, int blocks) {
  constexpr int kSpan = kManySpan;                     // (as many threads)
  wait_for_grid_before();
  int at = 2 * blockIdx.x + 1;
  const int4 of = p.part_of[at];
  if (of.x < 0) return;
  float sum = p.part[(int64_t)at * kSpan + threadIdx.x];
  for (at++; at < 2 * blocks; at += 2) {
    sum += p.part[(int64_t)at * kSpan + threadIdx.x];
    if (!p.part_of[at].w) break;
  }
  weights_write(p, of.x, of.y, p.lens[of.x], of.z * kSpan + threadIdx.x, sum);
}

}  // namespace amk
