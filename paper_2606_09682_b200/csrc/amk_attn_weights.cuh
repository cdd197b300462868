// The kernel of amk_attention_weights: what the queries of some tokens attend to, added up for each cached position.
//
// Mathematics.  With the log-sum-exps known there is no maximum to find: w(j) = sum over the query rows (a row is a token and one
// of the query heads of a kv head) of 2^(S c - L), c = scale log2 e, L = lse log2 e.  The product is taken as S^T = K Q^T, so that a
// position is a lane of TMEM and its sum stays in one thread's register: no exchange between lanes.
//
// Work.  One block an SM.  A unit is a tile of 128 positions of a kv head, a step of it the product with one tile of query rows
// (as many whole tokens as fit into 128 rows); the steps of all units, in that order, are cut into equal runs, one for each
// block.  A unit that a run's border cuts leaves its parts in scratch and a second kernel adds them, in the order of the blocks.
// A producer warp brings K tiles (once a unit) and Q tiles (once a step, or once a head where one tile holds all rows) by
// TMA, one warp issues the products into four accumulators, four warpgroups take every fourth step each.
#pragma once
#include "amk_attn.cuh"

namespace amk {

struct WeightsParams {
  const float* lse;
  const int* lens;
  const float* before;
  float* out;
  float* part;                     // [2 * gridDim][128]: sums of cut units
  int4* part_of;                   // [2 * gridDim]: {sequence, head, tile, whether the next block goes on}; sequence -1: none
  int64_t b_seq, b_head, o_seq, o_head;
  int n_seqs, nq, nkv, rep, rows, slots;
  int tokens, q_tiles;             // tokens of a tile of query rows, tiles of all
  int columns;                     // rows of a tile, up to a multiple of 32
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
// Four e4m3 codes to four bf16, exactly: the seven bits without the sign, read as a bf16 four places lower, are 2^-120 times the
// code's value (also below the normal ones), for all but NaN.
__device__ __forceinline__ void widen_e4m3_bf16(unsigned* w, unsigned codes) {
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const unsigned a = __byte_perm(codes, 0, i ? 0x3424 : 0x1404), r = (a & 0x80008000u) | (a >> 4 & 0x07f007f0u);
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(w[i]) : "r"(r), "r"(0x7b807b80u), "r"(0x80008000u));
    if (((a & 0x7f007f00u) + 0x01000100u) & 0x80008000u) {
      if ((a & 0x7f00u) == 0x7f00u) w[i] |= 0x7fffu;
      if ((a & 0x7f000000u) == 0x7f000000u) w[i] |= 0x7fff0000u;
    }
  }
}

constexpr int kSumRing = 8;
template <int HD, bool FP8>
struct WeightsSmem {
  static constexpr int kTileBytes = HD / 64 * kBox;
  static constexpr int kStages = FP8 ? 2 : 3;                      // K tiles (bf16)
  static constexpr int kQStages = HD == 128 ? 3 : 4;
  static constexpr int kRawBytes = FP8 ? HD * kTile : 0, kRawStages = FP8 ? 2 : 0;
  static constexpr int kQ = 0;
  static constexpr int kRing = kQStages * kTileBytes;
  static constexpr int kRaw = kRing + kStages * kTileBytes;
  static constexpr int kHead = kRaw + kRawStages * kRawBytes;
  static constexpr int kBytes = kHead + 24576 + 1024;              // + alignment of the dynamic buffer
  static constexpr int kThreads = FP8 ? 704 : 576;
  static_assert(kBytes <= 227 * 1024, "shared memory of one SM");
};
struct WeightsHead {
  float sums[kSumRing][4][kTile];      // the warpgroups' shares of a unit
  float less[4][2][kTile];             // [warpgroup][step of it & 1]: -lse log2 e of the rows; -infinity: adds nothing
  uint64_t k_full[4], k_empty[4], raw_full[4], raw_empty[4], q_full[4], q_empty[4], s_full[4], s_empty[4], sums_full[kSumRing], fin;
  unsigned tmem;
  int dead;
  unsigned wait_cycles;
  int start[5];                        // where the block's run begins: sequence, head, tile, step; its steps
};
static_assert(sizeof(WeightsHead) <= 24576, "head");

// ---- units ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ int weights_tiles(const WeightsParams& p, int len) {         // 0: impossible length
  return len < 0 || len > p.slots - p.rows ? 0 : (len + p.rows + kTile - 1) / kTile;
}
// the first tile of query rows that sees a tile of positions
__device__ __forceinline__ int first_q_tile(const WeightsParams& p, int len, int tile) {
  return max(0, tile * kTile - len) / p.tokens;
}
__device__ __forceinline__ int weights_steps(const WeightsParams& p, int len) {         // of one head
  const int tiles = weights_tiles(p, len);
  if (p.q_tiles == 1 || !tiles) return tiles;
  const int full = min(tiles, len / kTile + 1);                    // tiles that all rows see
  int n = full * p.q_tiles;
  for (int j = full; j < tiles; j++) n += p.q_tiles - first_q_tile(p, len, j);
  return n;
}
struct WeightsUnit {
  int seq, head, len, tile;
  int first;                       // first tile of query rows of the unit
  int begin, end, all;             // steps of this block, steps of the unit
};
struct WeightsWalk {
  int left, seq, len, head, tile, tiles, step;
  __device__ __forceinline__ void init(const WeightsParams& p, const WeightsHead& h) {
    seq = h.start[0], head = h.start[1], tile = h.start[2], step = h.start[3], left = h.start[4];
    len = left ? __ldg(p.lens + seq) : 0;
    tiles = weights_tiles(p, len);
  }
  __device__ __forceinline__ bool next(const WeightsParams& p, WeightsUnit& u) {
    if (left <= 0) return false;
    while (tile >= tiles) {        // something is left: a unit follows
      tile = 0;
      if (tiles && head + 1 < p.nkv) {
        head++;
      } else {
        head = 0;
        len = __ldg(p.lens + ++seq);
        tiles = weights_tiles(p, len);
      }
    }
    u.seq = seq, u.head = head, u.len = len, u.tile = tile;
    u.first = first_q_tile(p, len, tile);
    u.all = p.q_tiles - u.first;
    u.begin = step, u.end = min(u.all, step + left);
    left -= u.end - u.begin;
    step = 0;
    tile++;
    return true;
  }
};

// a position's sum, finished
__device__ __forceinline__ void weights_write(const WeightsParams& p, int seq, int head, int len, int key, float sum) {
  if (key >= p.slots) return;
  if (key >= len + p.rows) sum = 0.f;
  if (key < len && p.before) sum = fmaf(p.decay, p.before[seq * p.b_seq + head * p.b_head + key], sum);
  p.out[seq * p.o_seq + head * p.o_head + key] = sum;
}

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

template <int HD, bool FP8>
__global__ void __launch_bounds__(FP8 ? 704 : 576, 1)
    weights_kernel(const WeightsParams p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k) {
  using L = WeightsSmem<HD, FP8>;
  constexpr int kProducer = 16, kIssuer = 17;
  unsigned char* smem = attn_smem();
  WeightsHead& h = *(WeightsHead*)(smem + L::kHead);
  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;

  if (warp == kIssuer) {
    tmem_alloc(&h.tmem, 512);
    if (lane == 0) {
      for (int i = 0; i < L::kStages; i++) mbar_init(&h.k_full[i], FP8 ? 4 : 1), mbar_init(&h.k_empty[i], 1);
      for (int i = 0; i < L::kRawStages; i++) mbar_init(&h.raw_full[i], 1), mbar_init(&h.raw_empty[i], 4);
      for (int i = 0; i < L::kQStages; i++) mbar_init(&h.q_full[i], 1), mbar_init(&h.q_empty[i], 1);
      for (int i = 0; i < 4; i++) mbar_init(&h.s_full[i], 1), mbar_init(&h.s_empty[i], 4);
      for (int i = 0; i < kSumRing; i++) mbar_init(&h.sums_full[i], 16);
      mbar_init(&h.fin, 1);
      h.dead = 0, h.wait_cycles = p.wait_cycles;
      mbar_fence_init();
    }
  }
  if (warp == kProducer) prefetch_map(lane == 0, &map_q), prefetch_map(lane == 0, &map_k);
  // rows of a Q tile that no box fills
  for (int i = threadIdx.x; i < L::kQStages * L::kTileBytes / 16; i += L::kThreads)
    if (i % (kBox / 16) >= p.tokens * p.rep * 8) ((uint4*)(smem + L::kQ))[i] = make_uint4(0, 0, 0, 0);
  fence_async_smem();
  wait_for_grid_before();
  if (warp == 0) {
    // which run is this block's
    auto steps_of = [&](int s) { return s < p.n_seqs ? weights_steps(p, __ldg(p.lens + s)) * p.nkv : 0; };
    const int mine = steps_of(lane);
    int total = mine;
    for (int s = 32 + lane; s < p.n_seqs; s += 32) total += steps_of(s);
    total = warp_sum(total);
    const int per = (total + (int)gridDim.x - 1) / (int)gridDim.x;
    int at = (int)blockIdx.x * per, seq = 0, head = 0, tile = 0, step = 0, left = 0;
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
          const int len = __ldg(p.lens + seq), of_head = __shfl_sync(~0u, own, f) / p.nkv;
          head = rel / of_head, rel -= head * of_head;
          const int tiles = weights_tiles(p, len), full = p.q_tiles == 1 ? tiles : min(tiles, len / kTile + 1);
          if (rel < full * p.q_tiles) {
            tile = rel / p.q_tiles, step = rel - tile * p.q_tiles;
          } else {
            rel -= full * p.q_tiles;
            for (tile = full;; tile++) {
              const int steps = p.q_tiles - first_q_tile(p, len, tile);
              if (rel < steps) break;
              rel -= steps;
            }
            step = rel;
          }
          break;
        }
        at -= __shfl_sync(~0u, n, 31);
      }
    }
    if (lane == 0) h.start[0] = seq, h.start[1] = head, h.start[2] = tile, h.start[3] = step, h.start[4] = left;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const unsigned tmem = uniform(h.tmem);
  unsigned k_asked = 0, q_asked = 0;                   // the producer's

  WeightsWalk walk;
  walk.init(p, h);
  WeightsUnit u;
  if (warp < 16) {
    // ================================ exponentials and sums ============================================================
    const int wg = warp >> 2, id = threadIdx.x & 127;
    const unsigned ts = tmem + ((unsigned)(warp & 3) * 32 << 16) + wg * kTile;
    const float c = p.scale * kLog2e;
    // slots behind the tiles, and sequences of an impossible length
    for (int r = blockIdx.x; r < p.n_seqs * p.nkv; r += gridDim.x) {
      const int s = r / p.nkv, len = __ldg(p.lens + s), tiles = weights_tiles(p, len);
      float* out = p.out + s * p.o_seq + (r - s * p.nkv) * p.o_head;
      for (int64_t i = (int64_t)tiles * kTile + threadIdx.x; i < p.slots; i += 512) out[i] = tiles ? 0.f : CUDART_NAN_F;
    }
    const int own_tok = id / p.rep, own_head = id - own_tok * p.rep;   // the query row of a tile whose lse this thread brings
    const bool own_row = own_tok < p.tokens;
    int g = 0, mine = 0, shared = 0;                   // steps in front of this unit, steps of this warpgroup, units of several steps
    bool cut0 = false, cut1 = false;
    while (walk.next(p, u)) {
      const int n = u.end - u.begin, key0 = u.tile * kTile, key = key0 + id;
      const float* lse = p.lse + (int64_t)u.seq * p.rows * p.nq + u.head * p.rep + own_head;
      const auto less_of = [&](int i) {                // of this thread's row of step i
        const int tok = (u.first + u.begin + i) * p.tokens + own_tok;
        float l = CUDART_INF_F;
        if (own_row && tok < p.rows) l = __ldg(lse + (int64_t)tok * p.nq);
        return fabsf(l) == CUDART_INF_F ? -CUDART_INF_F : -l * kLog2e;
      };
      float sum = 0.f;
      int i = (wg - g) & 3;
      float less = i < n ? less_of(i) : 0.f;
      for (; i < n; i += 4, mine++) {
        float* row = h.less[wg][mine & 1];
        row[id] = less;
        named_barrier(1 + wg, 128);
        const int tok0 = (u.first + u.begin + i) * p.tokens;
        const bool hides = key0 + kTile - 1 - u.len > tok0;
        const int from = hides ? min(max(key - u.len - tok0, 0), kTile) * p.rep : 0;    // first row that sees this position
        if (i + 4 < n) less = less_of(i + 4);
        attn_wait(&h.s_full[wg], mine & 1, h);
        __syncwarp();
        tc_fence_after();
        const uint64_t c2 = pair(c, c);
        uint64_t acc[2] = {0, 0};
#pragma unroll 1
        for (int x = 0; x < p.columns; x += 32) {
          unsigned w[32];
          tmem_ld32(w, ts + x);
          tmem_wait_ld();
          tmem_pin(w);
#pragma unroll
          for (int k = 0; k < 32; k += 4) {
            const float4 l = *(const float4*)(row + x + k);
            float e[4];
            unpair(e[0], e[1], fma2(pair(__uint_as_float(w[k]), __uint_as_float(w[k + 1])), c2, pair(l.x, l.y)));
            unpair(e[2], e[3], fma2(pair(__uint_as_float(w[k + 2]), __uint_as_float(w[k + 3])), c2, pair(l.z, l.w)));
#pragma unroll
            for (int j = 0; j < 4; j++) {
              e[j] = exp2_fast(e[j]);
              if (hides && x + k + j < from) e[j] = 0.f;
            }
            acc[0] = add2(acc[0], pair(e[0], e[1])), acc[1] = add2(acc[1], pair(e[2], e[3]));
          }
        }
        float a, b;
        unpair(a, b, add2(acc[0], acc[1]));
        a += b;
        if (__any_sync(~0u, !(a < CUDART_INF_F))) a = weights_careful(ts, row, p.columns, from, c);
        sum += a;
        tc_fence_before();
        warp_arrive(&h.s_empty[wg], lane);
      }
      const int last = (g + n - 1) & 3;                // the warpgroup that finishes the unit
      if (n > 1) {
        const int at = shared % kSumRing;
        if (wg != last && ((wg - g) & 3) < n) h.sums[at][wg][id] = sum;
        warp_arrive(&h.sums_full[at], lane);
        if (wg == last) {
          attn_wait(&h.sums_full[at], shared / kSumRing & 1, h);
          float all = 0.f;
#pragma unroll
          for (int j = 0; j < 4; j++)
            if (((j - g) & 3) < n) all += j == wg ? sum : h.sums[at][j][id];
          sum = all;
        }
        shared++;
      }
      const bool whole = u.begin == 0 && u.end == u.all;
      if (wg == last) {
        if (whole) {
          weights_write(p, u.seq, u.head, u.len, key, sum);
        } else {
          const int at = 2 * blockIdx.x + (u.begin == 0);
          p.part[(int64_t)at * kTile + id] = sum;
          if (id == 0) p.part_of[at] = make_int4(u.seq, u.head, u.tile, u.end < u.all);
        }
      }
      if (!whole) (u.begin == 0 ? cut1 : cut0) = true;
      g += n;
    }
    if (threadIdx.x == 0 && p.part) {
      if (!cut0) p.part_of[2 * blockIdx.x] = make_int4(-1, 0, 0, 0);
      if (!cut1) p.part_of[2 * blockIdx.x + 1] = make_int4(-1, 0, 0, 0);
    }
  } else if (warp == kProducer) {
    // ================================ tiles ============================================================================
    const bool leader = elect_one();
    const unsigned q_bytes = (unsigned)(p.tokens * p.rep) * HD * 2;
    int q_seq = -1, q_head = -1;
    bool on = true;
    while (walk.next(p, u)) {
      const int n = FP8 ? L::kRawStages : L::kStages, st = k_asked % n;
      uint64_t *full = FP8 ? &h.raw_full[st] : &h.k_full[st], *empty = FP8 ? &h.raw_empty[st] : &h.k_empty[st];
      on = on && attn_wait(empty, (k_asked / n & 1) ^ 1, h) && k_asked < p.tiles;
      if (on) {
        expect_tx(leader, full, FP8 ? L::kRawBytes : L::kTileBytes);
        if (FP8) {
          tma_load_4d(leader, smem + L::kRaw + st * L::kRawBytes, &map_k, 0, u.tile * kTile, u.head, u.seq, full);
        } else {
#pragma unroll
          for (int x = 0; x < HD; x += 64)
            tma_load_4d(leader, smem + L::kRing + st * L::kTileBytes + x / 64 * kBox, &map_k, x, u.tile * kTile, u.head, u.seq, full);
        }
        k_asked++;
      }
      for (int i = u.begin; i < u.end; i++) {
        if (p.q_tiles == 1 && u.seq == q_seq && u.head == q_head) continue;      // it is there already
        q_seq = u.seq, q_head = u.head;
        const int qs = q_asked % L::kQStages;
        on = on && attn_wait(&h.q_empty[qs], (q_asked / L::kQStages & 1) ^ 1, h);
        if (!on) continue;
        expect_tx(leader, &h.q_full[qs], q_bytes);
#pragma unroll
        for (int x = 0; x < HD; x += 64)
          tma_load_5d(leader, smem + L::kQ + qs * L::kTileBytes + x / 64 * kBox, &map_q, x, 0, u.head, (u.first + i) * p.tokens, u.seq,
                      &h.q_full[qs]);
        q_asked++;
      }
    }
  } else if (warp == kIssuer) {
    // ================================ the matrix products ==============================================================
    const bool leader = elect_one();
    const unsigned id_s = mma_idesc(kTile, 0, false, false) | (unsigned)(p.columns >> 3) << 17;
    const uint64_t q_desc = smem_desc(smem_u32(smem + L::kQ), 16, 1024), k_desc = smem_desc(smem_u32(smem + L::kRing), 16, 1024);
    constexpr uint64_t kTileStep = L::kTileBytes >> 4;
    int g = 0, k_at = 0, q_at = -1, q_seq = -1, q_head = -1;
    bool on = true;
    while (walk.next(p, u)) {
      const int ks = uniform(k_at % L::kStages);
      on = on && attn_wait(&h.k_full[ks], k_at / L::kStages & 1, h);
      for (int i = uniform(u.begin); i < uniform(u.end); i++, g++) {
        if (p.q_tiles > 1 || u.seq != q_seq || u.head != q_head) {
          q_seq = u.seq, q_head = u.head;
          if (on && q_at >= 0) mma_commit(leader, &h.q_empty[q_at % L::kQStages]);
          q_at++;
          on = on && attn_wait(&h.q_full[q_at % L::kQStages], q_at / L::kQStages & 1, h);
        }
        const int qs = uniform(q_at % L::kQStages), at = uniform(g & 3);
        on = on && attn_wait(&h.s_empty[at], (g >> 2 & 1) ^ 1, h);
        if (!on) continue;
        tc_fence_after();
        const uint64_t ka = k_desc + ks * kTileStep, qa = q_desc + qs * kTileStep;
#pragma unroll
        for (int k = 0; k < HD / 16; k++) {
          const int off = (k / 4 * kBox + k % 4 * 32) >> 4;
          mma_ss(leader, tmem + at * kTile, ka + off, qa + off, id_s, k > 0);
        }
        mma_commit(leader, &h.s_full[at]);
      }
      if (on) mma_commit(leader, &h.k_empty[ks]);
      k_at++;
    }
  } else if (FP8) {
    // ================================ 8-bit tiles widened to bf16: four warps ==========================================
    const int ct = (warp - 18) * 32 + lane;
    constexpr int kChunks = HD / 16;                   // 16-byte chunks of an 8-bit row, each two of a bf16 row
    constexpr int kRaws = FP8 ? L::kRawStages : 1;
    int pos = 0;
    while (walk.next(p, u)) {
      const int raw = pos % kRaws, st = pos % L::kStages;
      attn_wait(&h.raw_full[raw], pos / kRaws & 1, h);
      attn_wait(&h.k_empty[st], (pos / L::kStages & 1) ^ 1, h);
      const unsigned char* src = smem + L::kRaw + raw * L::kRawBytes;
      unsigned char* dst = smem + L::kRing + st * L::kTileBytes;
#pragma unroll 2
      for (int i = ct; i < kTile * kChunks; i += 128) {
        const int row = i / kChunks, cc = i % kChunks * 2;
        const uint4 v = *(const uint4*)(src + i * 16);
        unsigned w[8];
        widen_e4m3_bf16(w, v.x), widen_e4m3_bf16(w + 2, v.y), widen_e4m3_bf16(w + 4, v.z), widen_e4m3_bf16(w + 6, v.w);
        unsigned char* to = dst + cc / 8 * kBox + row * 128;
        *(uint4*)(to + (((cc & 7) ^ (row & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
        *(uint4*)(to + ((((cc & 7) + 1) ^ (row & 7)) << 4)) = make_uint4(w[4], w[5], w[6], w[7]);
      }
      fence_async_smem();
      warp_arrive(&h.k_full[st], lane);
      warp_arrive(&h.raw_empty[raw], lane);
      pos++;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (h.dead) {                                        // copies and products in flight end before their memory is given back
    constexpr unsigned kN = FP8 ? L::kRawStages : L::kStages;
    if (warp == kProducer) {
      uint64_t* full = FP8 ? h.raw_full : h.k_full;
      for (unsigned i = k_asked > kN ? k_asked - kN : 0; i < k_asked; i++)
        for (int n = 0; n < 1 << 16 && !__all_sync(~0u, mbar_try_wait(&full[i % kN], i / kN & 1)); n++) {}
      for (unsigned i = q_asked > L::kQStages ? q_asked - L::kQStages : 0; i < q_asked; i++)
        for (int n = 0; n < 1 << 16 && !__all_sync(~0u, mbar_try_wait(&h.q_full[i % L::kQStages], i / L::kQStages & 1)); n++) {}
    }
    if (warp == kIssuer) {
      mma_commit(elect_one(), &h.fin);
      for (int n = 0; n < 1 << 16 && !__all_sync(~0u, mbar_try_wait(&h.fin, 0)); n++) {}
    }
    __syncthreads();
  }
  if (warp == kIssuer) tmem_free(tmem, 512);
}

// The parts of units that a border cut: one block for each block of the first kernel in whose run such a unit begins.
static __global__ void __launch_bounds__(kTile) weights_join_kernel(const WeightsParams p, int blocks) {
  wait_for_grid_before();
  int at = 2 * blockIdx.x + 1;
  const int4 of = p.part_of[at];
  if (of.x < 0) return;
  float sum = p.part[(int64_t)at * kTile + threadIdx.x];
  for (at++; at < 2 * blocks; at += 2) {
    sum += p.part[(int64_t)at * kTile + threadIdx.x];
    if (!p.part_of[at].w) break;
  }
  weights_write(p, of.x, of.y, p.lens[of.x], of.z * kTile + threadIdx.x, sum);
}

}  // namespace amk
