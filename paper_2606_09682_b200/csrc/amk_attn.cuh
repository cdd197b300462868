// The attention kernel of amk_prompt_attention and amk_tree_attention, and the parameters they share.
//
// Mathematics.  For a block of query rows (a row is a query token and one of the query heads of a kv head: all heads
// of a group share the K/V tiles) and the key tiles it sees, one pass with a running maximum m and sum l:
//   S = Q K^T;  m' = max(m, rowmax S);  P = 2^((S - m') c), c = scale log2 e;  l = l 2^((m - m') c) + rowsum P;
//   O = O 2^((m - m') c) + P V;  at the end O / l.
// O is rescaled only when m rises by more than 8 / c (P then stays below 2^8, nothing is lost: P is a floating-point
// number and l and O share the reference).
#pragma once
#include <cuda_bf16.h>
#include <math_constants.h>

#include "amk_tc.cuh"

namespace amk {

struct AttnParams {
  const unsigned short* q;
  __nv_bfloat16* out;
  float* lse;
  const int* lens;                 // prompt: cu_seqlens; tree: cache_len
  const unsigned long long* mask;  // tree: or null
  float* part_o;                   // tree: [2 * gridDim][part_rows][HD]
  float* part_lse;                 // tree: [2 * gridDim][part_rows]
  int64_t q_seq, q_row, q_head, o_seq, o_row, o_head;
  int n_seqs, nq, nkv, rep;
  int rows;                        // prompt: all tokens; tree: drafted tokens of a sequence
  int slots;
  int part_rows;                   // tree: 128 (both warpgroups work on the same rows) or 256
  int row_tiles;                   // tree: blocks of part_rows rows per (sequence, kv head)
  int min_tiles;                   // tree: key tiles a block takes at least
  unsigned rep_inv;                // ceil(2^32 / rep), 0 for rep = 1
  float scale;
};

constexpr int kTile = 128;         // rows of a Q tile, keys of a K/V tile
// row / rep, exact for rows below 2^28
__device__ __forceinline__ int div_rep(const AttnParams& p, int row) {
  return p.rep_inv ? (int)__umulhi((unsigned)row, p.rep_inv) : row;
}
constexpr float kLog2e = 1.4426950408889634f;

// Set when a bounded wait of an attention kernel ran out; read and cleared by amk_operator_status.
static __device__ unsigned g_attn_expired;

__device__ __forceinline__ float exp2_fast(float x) {   // 2^x, relative error 2^-22; 2^-inf = 0
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {   // round to nearest even
  unsigned r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// two fp32 lanes in one instruction
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ void unpair(float& lo, float& hi, uint64_t a) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(a));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// acc + 0 * w for two bf16 at once: NaN from the first value on that is not finite
__device__ __forceinline__ unsigned zero_times(unsigned w, unsigned acc) {
  unsigned d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(w), "r"(0u), "r"(acc));
  return d;
}

// ---- what the blocks work on ------------------------------------------------------------------------------------
// One unit: a block of query rows of one (sequence, kv head) and a run of its key tiles.
struct Unit {
  int seq, head;
  int tok0, n_tok;        // first query token (within the sequence), tokens
  int row0, n_rows;       // tree: first row (token * rep + head) and rows of the unit; prompt: 0, n_tok * rep
  int key0;               // prompt: row of the sequence's first token; tree: 0
  int tile_begin, tile_end, item_tiles;
  int len;                // tree: context length
};

// Tree: the key tiles of all (sequence, kv head, row block) in that order, cut into equal runs, one for each block.
__device__ __forceinline__ int tree_tiles(const AttnParams& p, int len) {   // key tiles of one item; 0: bad length
  return len < 0 || len > p.slots - p.rows ? 0 : (len + p.rows + kTile - 1) / kTile;
}
// flat tiles of all sequences and tiles per block, the same in every block (one warp; result in every lane)
__device__ __forceinline__ int64_t tree_total(const AttnParams& p, int lane) {
  int64_t sum = 0;
  for (int b = lane; b < p.n_seqs; b += 32) sum += tree_tiles(p, p.lens[b]);
#pragma unroll
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
  return sum * p.nkv * p.row_tiles;
}
__device__ __forceinline__ int64_t tree_per_block(const AttnParams& p, int64_t total, int blocks) {
  const int64_t per = (total + blocks - 1) / blocks;
  return per < p.min_tiles ? p.min_tiles : per;
}

}  // namespace amk

namespace amk {

// ---- shared memory ----------------------------------------------------------------------------------------------
// Tiles of 64 elements x 128 rows of 128 bytes, swizzled by TMA's 128-byte pattern: the 16-byte chunk c of row r lies
// at r * 128 + ((c ^ (r & 7)) << 4).
constexpr int kBox = 64 * kTile * 2;
template <int HD, bool FP8>
struct AttnSmem {
  static constexpr int kTileBytes = HD / 64 * kBox;                // one bf16 tile of 128 rows
  static constexpr int kStages = FP8 ? (HD == 128 ? 3 : 6) : (HD == 128 ? 5 : 10);
  static constexpr int kRawBytes = FP8 ? HD * kTile : 0;           // one 8-bit tile
  static constexpr int kRawStages = FP8 ? (HD == 128 ? 4 : 8) : 0;
  static constexpr int kQ = 0;
  static constexpr int kRing = 2 * kTileBytes;
  static constexpr int kRaw = kRing + kStages * kTileBytes;
  static constexpr int kHead = kRaw + kRawStages * kRawBytes;      // AttnHead
  static constexpr int kBytes = kHead + 2048 + 1024;               // + alignment of the dynamic buffer
  static_assert(kBytes <= 227 * 1024, "shared memory of one SM");
};
struct AttnHead {
  uint64_t full[10], empty[10];        // ring of K and V tiles (bf16)
  uint64_t raw_full[8], raw_empty[8];  // ring of 8-bit tiles
  uint64_t q_full[2], s_full[2], p_full[2], o_done[2], fin;
  unsigned tmem;
  int dead;                            // a bounded wait ran out: nobody waits or issues any more
  int skip[2];                         // this step's P V was done by the warpgroup itself
  float m[kTile], l[kTile];            // second warpgroup's statistics (both on the same rows)
  int unit[8];
  int64_t walk[1];
};
static_assert(sizeof(AttnHead) <= 2048, "head");

constexpr long long kWaitCycles = 4000000000ll;
// Waits for the phase of the given parity, about two seconds at most (the SM's cycle counter: the global timer is read
// through a unit that all SMs share).
__device__ __forceinline__ void attn_wait(uint64_t* bar, unsigned parity, AttnHead& h) {
  if (mbar_try_wait(bar, parity)) return;
  const long long t0 = clock64();
  for (;;) {
    for (int i = 0; i < 32; i++)
      if (mbar_try_wait(bar, parity)) return;
    if (*(volatile int*)&h.dead) return;
    if (clock64() - t0 > kWaitCycles) {
      *(volatile int*)&h.dead = 1;
      atomicExch(&g_attn_expired, 1u);
      return;
    }
  }
}
__device__ __forceinline__ unsigned any_of_warpgroup(unsigned pred, int id) {
  unsigned r;
  asm volatile(
      "{ .reg .pred p, q; setp.ne.u32 p, %1, 0; bar.red.or.pred q, %2, 128, p; selp.u32 %0, 1, 0, q; }"
      : "=r"(r)
      : "r"(pred), "r"(id)
      : "memory");
  return r;
}

// ---- units ------------------------------------------------------------------------------------------------------
template <bool TREE>
struct Units;

template <>
struct Units<true> {
  int64_t left;                    // key tiles of this block's run that are still to come
  int seq, len, tiles, item, within, items;
  __device__ __forceinline__ void init(const AttnParams& p, const AttnHead& h) {
    left = h.walk[0];
    seq = h.unit[0], item = h.unit[1], within = h.unit[2], len = h.unit[3];
    tiles = tree_tiles(p, len);
    items = p.nkv * p.row_tiles;
  }
  __device__ __forceinline__ bool next(const AttnParams& p, const AttnHead&, Unit& u) {
    if (left <= 0) return false;
    while (item == items || tiles == 0) {   // something is left: a sequence with tiles follows
      item = 0;
      len = p.lens[++seq];
      tiles = tree_tiles(p, len);
    }
    const int run = left < tiles - within ? (int)left : tiles - within;
    u.seq = seq, u.head = p.row_tiles == 1 ? item : item / p.row_tiles, u.len = len;
    u.row0 = (item - u.head * p.row_tiles) * p.part_rows;
    u.n_rows = min(p.part_rows, p.rows * p.rep - u.row0);
    u.tok0 = 0, u.n_tok = p.rows, u.key0 = 0;
    u.tile_begin = within, u.tile_end = within + run, u.item_tiles = tiles;
    left -= run;
    within = 0;
    item++;
    return true;
  }
};

template <>
struct Units<false> {
  bool more;
  __device__ __forceinline__ void init(const AttnParams&, const AttnHead& h) { more = h.unit[0] >= 0; }
  __device__ __forceinline__ bool next(const AttnParams& p, const AttnHead& h, Unit& u) {
    if (!more) return false;
    more = false;
    u.seq = 0, u.head = h.unit[1], u.key0 = h.unit[2], u.tok0 = h.unit[3], u.n_tok = h.unit[4];
    u.row0 = 0, u.n_rows = u.n_tok * p.rep, u.len = 0;
    u.tile_begin = 0, u.tile_end = u.item_tiles = (u.tok0 + u.n_tok + kTile - 1) / kTile;
    return true;
  }
};

// Key tiles that row tile t of the unit works on; DUAL: every second one of the unit's.
template <bool TREE>
__device__ __forceinline__ int unit_steps(const AttnParams& p, const Unit& u, bool dual, int t) {
  const int n = u.tile_end - u.tile_begin;
  if (dual) return t ? n / 2 : (n + 1) / 2;
  const int first = t * kTile;
  if (u.n_rows <= first) return 0;
  if (TREE) return n;
  const int last = min(u.n_rows, first + kTile) - 1;
  return (u.tok0 + div_rep(p, last)) / kTile + 1;
}

// 32 bits of a drafted token's mask from drafted index idx on (idx may be negative: bits below 0 are 0)
__device__ __forceinline__ unsigned tree_bits32(const unsigned long long* w, int rows, int tok, int idx) {
  if (idx >= rows || idx <= -32) return 0;
  if (!w) {   // a chain: indices 0..tok
    const int n = tok + 1 - idx;   // bits below n
    unsigned r = n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
    if (idx < 0) r &= ~0u << -idx;
    return r;
  }
  unsigned long long v;
  if (idx < 0) {
    v = w[0] << -idx;
  } else {
    const int word = idx >> 6, off = idx & 63;
    v = w[word] >> off;
    if (off > 32 && (word + 1) * 64 < rows) v |= w[word + 1] << (64 - off);
  }
  const int left = rows - idx;      // bits from the last drafted token on are nobody's
  return left >= 32 ? (unsigned)v : (unsigned)v & ((1u << left) - 1u);
}

// O += P V of one tile for this warp's rows, key by key and only for the keys that a row sees: for tiles with values
// that are not finite behind a mask, where 0 * V would not be 0.
template <int HD>
__device__ __noinline__ void product_by_key(const float* pl, const uint4 see, const unsigned char* vt, unsigned to, bool more) {
  for (int x = 0; x < HD; x += 32) {
    unsigned o[32];
    tmem_ld32(o, to + x);
    tmem_wait_ld();
    tmem_pin(o);
    float a[32];
#pragma unroll
    for (int k = 0; k < 32; k++) a[k] = more ? __uint_as_float(o[k]) : 0.f;
    for (int k = 0; k < kTile; k++) {
      const unsigned w = k < 64 ? (k < 32 ? see.x : see.y) : (k < 96 ? see.z : see.w);
      if (!(w >> (k & 31) & 1)) continue;
#pragma unroll
      for (int ch = 0; ch < 4; ch++) {
        const int cc = x / 8 + ch;
        const uint4 v = *(const uint4*)(vt + cc / 8 * kBox + k * 128 + (((cc & 7) ^ (k & 7)) << 4));
        const unsigned vv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; e++) {
          a[ch * 8 + 2 * e] += pl[k] * bf16_lo(vv[e]);
          a[ch * 8 + 2 * e + 1] += pl[k] * bf16_hi(vv[e]);
        }
      }
    }
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 32; k++) o[k] = __float_as_uint(a[k]);
    tmem_st32(to + x, o);
  }
  tmem_wait_st();
}

// ---- the kernel -------------------------------------------------------------------------------------------------
template <int HD, bool TREE, bool FP8>
__global__ void __launch_bounds__(FP8 ? 512 : 384, 1)
    attn_kernel(const AttnParams p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using L = AttnSmem<HD, FP8>;
  constexpr int kProducer = FP8 ? 12 : 8, kIssuer = kProducer + 1;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  AttnHead& h = *(AttnHead*)(smem + L::kHead);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool dual = TREE && p.part_rows == kTile;

  if (warp == 0) {
    // which part of the work is this block's
    if (TREE) {
      const int64_t total = tree_total(p, lane);
      const int64_t per = tree_per_block(p, total, gridDim.x);
      const int64_t at = (int64_t)blockIdx.x * per, end = at + per < total ? at + per : total;
      int64_t before = 0;
      int seq = 0, item = 0, within = 0, len = 0;
      if (at < end) {
        const int64_t items = (int64_t)p.nkv * p.row_tiles;
        for (int b0 = 0;; b0 += 32) {
          int64_t n = b0 + lane < p.n_seqs ? tree_tiles(p, p.lens[b0 + lane]) * items : 0;
          const int64_t own = n;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const int64_t x = __shfl_up_sync(~0u, n, o);
            if (lane >= o) n += x;
          }
          const unsigned hit = __ballot_sync(~0u, before + n > at);
          if (hit) {
            const int f = __ffs(hit) - 1;
            seq = b0 + f;
            before += __shfl_sync(~0u, n - own, f);
            len = p.lens[seq];
            const int tiles = tree_tiles(p, len);
            const int64_t rel = at - before;
            item = (int)(rel / tiles), within = (int)(rel - (int64_t)item * tiles);
            break;
          }
          before += __shfl_sync(~0u, n, 31);
        }
      }
      if (lane == 0) h.walk[0] = end - at, h.unit[0] = seq, h.unit[1] = item, h.unit[2] = within, h.unit[3] = len;
    } else {
      // the blocks of all prompts in order; the last block of a long prompt has the most keys and goes first
      const int head = blockIdx.x % p.nkv, per = 2 * kTile / p.rep;
      int idx = (int)(gridDim.x / p.nkv) - 1 - blockIdx.x / p.nkv;
      int found = -1, tok0 = 0, n = 0, key0 = 0;
      for (int s0 = 0; s0 < p.n_seqs; s0 += 32) {
        int a = 0, b = 0;
        if (s0 + lane < p.n_seqs) a = p.lens[s0 + lane], b = p.lens[s0 + lane + 1];
        const bool ok = a >= 0 && a <= b && b <= p.rows;
        const int own = ok ? (b - a + per - 1) / per : 0;
        int sum = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int x = __shfl_up_sync(~0u, sum, o);
          if (lane >= o) sum += x;
        }
        const unsigned hit = __ballot_sync(~0u, sum > idx);
        if (hit) {
          const int f = __ffs(hit) - 1;
          const int blk = idx - __shfl_sync(~0u, sum - own, f);
          a = __shfl_sync(~0u, a, f), b = __shfl_sync(~0u, b, f);
          found = 0, key0 = a, tok0 = blk * per, n = min(per, b - a - tok0);
          break;
        }
        idx -= __shfl_sync(~0u, sum, 31);
      }
      if (lane == 0) h.unit[0] = found, h.unit[1] = head, h.unit[2] = key0, h.unit[3] = tok0, h.unit[4] = n;
    }
  }
  if (warp == kIssuer) {
    tmem_alloc(&h.tmem, 512);
    if (lane == 0) {
      for (int i = 0; i < L::kStages; i++) mbar_init(&h.full[i], FP8 ? 128 : 1), mbar_init(&h.empty[i], 1);
      for (int i = 0; i < L::kRawStages; i++) mbar_init(&h.raw_full[i], 1), mbar_init(&h.raw_empty[i], 128);
      for (int t = 0; t < 2; t++) {
        mbar_init(&h.q_full[t], 128), mbar_init(&h.s_full[t], 1);
        mbar_init(&h.p_full[t], 128), mbar_init(&h.o_done[t], 1);
      }
      mbar_init(&h.fin, 1);
      h.dead = 0;
      mbar_fence_init();
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const unsigned tmem = h.tmem;
  // TMEM columns: S0 (P0 over it), S1, O0, O1
  if (TREE) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  Units<TREE> units;
  units.init(p, h);
  Unit u;

  if (!FP8) {
    // 384 threads of 168 registers at launch: 256 x 208 + 128 x 88 = 64512, all of them
    if (warp < 8) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
  } else {
    // 512 threads of 128 registers at launch: 256 x 184 + 128 x 72 + 128 x 56 = 63488 of the 65536
    if (warp < 8) asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
    else if (warp < 12) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
  }

  if (warp < 8) {
    // ================================ softmax: one warpgroup for each row tile, one thread for each row ================
    const int t = warp >> 2, wt = threadIdx.x & 127;
    const unsigned lanes = (unsigned)(warp & 3) * 32 << 16;
    const unsigned ts = tmem + lanes + t * kTile, to = tmem + lanes + 2 * kTile + t * HD;
    unsigned char* qs = smem + L::kQ + t * L::kTileBytes;
    const float c = p.scale * kLog2e;
    unsigned s_phase = 0, o_phase = 0;
    int ring = 0;                                     // ring position of the unit's first tile
    while (units.next(p, h, u)) {
      const int steps = unit_steps<TREE>(p, u, dual, t);
      const int row_first = u.row0 + (dual ? 0 : t * kTile);                       // first row of this tile
      const int rows_here = dual ? u.n_rows : u.n_rows - t * kTile;                // may be <= 0
      if (steps) {
        // Q, 16 bytes at a time; rows that do not exist are zero
        constexpr int kChunks = HD / 8;
        const unsigned short* q = p.q + (int64_t)u.seq * p.q_seq + (int64_t)(u.key0 + u.tok0) * p.q_row +
                                  (int64_t)u.head * p.rep * p.q_head;
#pragma unroll
        for (int i0 = 0; i0 < kChunks; i0 += 8) {        // eight loads in flight before the first store
          uint4 v[8];
#pragma unroll
          for (int i = 0; i < 8; i++) {
            const int e = (i0 + i) * kTile + wt, r = e / kChunks, ch = e % kChunks;
            v[i] = make_uint4(0, 0, 0, 0);
            if (r < rows_here) {
              const int row = row_first + r, tok = div_rep(p, row), hh = row - tok * p.rep;
              v[i] = __ldg((const uint4*)(q + tok * p.q_row + hh * p.q_head + ch * 8));
            }
          }
#pragma unroll
          for (int i = 0; i < 8; i++) {
            const int e = (i0 + i) * kTile + wt, r = e / kChunks, ch = e % kChunks;
            *(uint4*)(qs + ch / 8 * kBox + r * 128 + (((ch & 7) ^ (r & 7)) << 4)) = v[i];
          }
        }
        fence_async_smem();
        mbar_arrive(&h.q_full[t]);
      }
      const int row = row_first + wt, tok = div_rep(p, row), hh = row - tok * p.rep;
      const bool valid = wt < rows_here;
      const bool live = (wt & ~31) < rows_here;        // this warp has rows; the others only keep step
      const unsigned long long* words = nullptr;
      if (TREE && p.mask && valid) words = p.mask + ((int64_t)u.seq * p.rows + tok) * ((p.rows + 63) / 64);
      const int key_end = TREE ? u.len + p.rows : u.tok0 + u.n_tok;    // keys nobody here sees: from it on
      // first key that a row of this tile may not see
      const int all_see = TREE ? u.len : u.tok0 + div_rep(p, row_first) + 1;
      float m = -CUDART_INF_F, l = 0.f;
      for (int i = 0; i < steps; i++) {
        const int rel = dual ? 2 * i + t : i;
        const int key = (u.tile_begin + rel) * kTile;
        attn_wait(&h.s_full[t], s_phase & 1, h);
        s_phase++;
        __syncwarp();
        tc_fence_after();
        unsigned sb[4][32];
        unsigned see[4] = {~0u, ~0u, ~0u, ~0u};
#define AMK_S(k) __uint_as_float(sb[(k) >> 5][(k) & 31])
        const bool masked = key + kTile > all_see;
        if (live) {
#pragma unroll
          for (int k = 0; k < 4; k++) tmem_ld32(sb[k], ts + 32 * k);
          tmem_wait_ld();
#pragma unroll
          for (int k = 0; k < 4; k++) tmem_pin(sb[k]);
          if (masked) {
#pragma unroll
            for (int w = 0; w < 4; w++) {
              const int first = key + 32 * w;
              if (TREE) {
                const int ctx = u.len - first;                  // context keys from `first` on
                if (ctx < 32)
                  see[w] = (ctx > 0 ? (1u << ctx) - 1u : 0u) |
                           tree_bits32(words, p.mask ? (words ? p.rows : 0) : p.rows, tok, -ctx);
              } else {
                const int n = u.tok0 + tok + 1 - first;
                see[w] = n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
              }
            }
#pragma unroll
            for (int k = 0; k < kTile; k++)
              if (!(see[k >> 5] >> (k & 31) & 1)) sb[k >> 5][k & 31] = 0xff800000u;   // -infinity
          }
          float mx[4];
#pragma unroll
          for (int k = 0; k < 4; k++) mx[k] = AMK_S(32 * k);
#pragma unroll
          for (int j = 1; j < 31; j += 2)
#pragma unroll
            for (int k = 0; k < 4; k++) mx[k] = max3(mx[k], AMK_S(32 * k + j), AMK_S(32 * k + j + 1));
#pragma unroll
          for (int k = 0; k < 4; k++) mx[k] = fmaxf(mx[k], AMK_S(32 * k + 31));
          mx[0] = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
          if (i == 0) {
            m = mx[0];
          } else {
            const bool need = mx[0] > m && (mx[0] - m) * c > 8.f;
            if (__any_sync(~0u, need)) {
              const float mn = fmaxf(m, mx[0]);
              const float f = m == mn ? 1.f : exp2_fast((m - mn) * c);
#pragma unroll
              for (int x = 0; x < HD; x += 32) {
                unsigned o[32];
                tmem_ld32(o, to + x);
                tmem_wait_ld();
                tmem_pin(o);
#pragma unroll
                for (int k = 0; k < 32; k++) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                tmem_st32(to + x, o);
              }
              l *= f;
              m = mn;
            }
          }
          const float mc = m == -CUDART_INF_F ? 0.f : -m * c;
          const uint64_t c2 = pair(c, c), mc2 = pair(mc, mc);
          uint64_t sum[2] = {0, 0};
#pragma unroll
          for (int k = 0; k < kTile; k += 2) {
            float e0, e1;
            unpair(e0, e1, fma2(pair(AMK_S(k), AMK_S(k + 1)), c2, mc2));
            e0 = exp2_fast(e0), e1 = exp2_fast(e1);
            sb[k >> 5][k & 31] = __float_as_uint(e0), sb[k >> 5][(k & 31) + 1] = __float_as_uint(e1);
            sum[k >> 1 & 1] = add2(sum[k >> 1 & 1], pair(e0, e1));
          }
          float s0, s1;
          unpair(s0, s1, add2(sum[0], sum[1]));
          l += s0 + s1;
#pragma unroll
          for (int x = 0; x < 2; x++) {
            unsigned r[32];
#pragma unroll
            for (int k = 0; k < 32; k++) r[k] = pack_bf16(AMK_S(x * 64 + 2 * k), AMK_S(x * 64 + 2 * k + 1));
            tmem_st32(ts + x * 32, r);
          }
        }
        unsigned slow = 0;
        if (masked) {
          // What a mask hides must not come through 0 * V either: V rows that no row of the block sees become zero; if
          // a row that some of them see is not finite, this tile's product is made here, key by key.
          const int pos = ring + 2 * rel + 1, st = pos % L::kStages;
          attn_wait(&h.full[st], pos / L::kStages & 1, h);
          unsigned char* vt = smem + L::kRing + st * L::kTileBytes;
          unsigned char* vr = vt + wt * 128;
          unsigned broken = 0;                         // becomes NaN (two bf16)
          if (key + wt >= key_end) {
#pragma unroll
            for (int ch = 0; ch < HD / 8; ch++) *(uint4*)(vr + ch / 8 * kBox + ((ch & 7) << 4)) = make_uint4(0, 0, 0, 0);
            fence_async_smem();
          } else {
#pragma unroll
            for (int ch = 0; ch < HD / 8; ch++) {
              const uint4 v = *(const uint4*)(vr + ch / 8 * kBox + (((ch & 7) ^ (wt & 7)) << 4));
              broken = zero_times(v.w, zero_times(v.z, zero_times(v.y, zero_times(v.x, broken))));
            }
          }
          slow = any_of_warpgroup((broken & 0x7fff7fffu) != 0, 1 + t);
          if (slow && live) {
            float pl[kTile];                           // (in local memory: the function walks it)
#pragma unroll
            for (int k = 0; k < kTile; k++) pl[k] = AMK_S(k);
            const uint4 sl = make_uint4(see[0], see[1], see[2], see[3]);
            product_by_key<HD>(pl, sl, vt, to, i > 0);
          }
        }
        tmem_wait_st();
        tc_fence_before();
        if (wt == 0) h.skip[t] = slow;
        mbar_arrive(&h.p_full[t]);
#undef AMK_S
      }
      ring += 2 * (u.tile_end - u.tile_begin);
      if (steps) {
        attn_wait(&h.o_done[t], o_phase & 1, h);
        o_phase++;
        __syncwarp();
        tc_fence_after();
      }

      // O / l, or this block's part of it
      float f0 = 1.f, f1 = 0.f;
      bool two = false;
      unsigned from0 = to, from1 = to;
      if (dual) {
        if (t == 1) {
          h.m[wt] = m, h.l[wt] = l;
          tc_fence_before();
        }
        named_barrier(3, 256);
        if (t == 0) {
          tc_fence_after();
          two = u.tile_end - u.tile_begin > 1;
          const float m1 = h.m[wt], l1 = h.l[wt];
          const float mn = fmaxf(m, m1);
          if (two && mn != -CUDART_INF_F) {
            f0 = m == mn ? 1.f : exp2_fast((m - mn) * c);
            f1 = m1 == mn ? 1.f : exp2_fast((m1 - mn) * c);
            l = l * f0 + l1 * f1;
            m = mn;
          }
          from1 = to + HD;
        }
      }
      if (steps && live && !(dual && t == 1)) {
        const bool whole = !TREE || (u.tile_begin == 0 && u.tile_end == u.item_tiles);
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const float lse2 = l == 0.f ? -CUDART_INF_F : m * c + log2f(l);
        const int64_t gtok = TREE ? (int64_t)u.seq * p.rows + tok : (int64_t)u.key0 + u.tok0 + tok;
        const int head = u.head * p.rep + hh;
        __nv_bfloat16* out = p.out + (TREE ? (int64_t)u.seq * p.o_seq + tok * p.o_row : gtok * p.o_row) + head * p.o_head;
        const int64_t slot = TREE ? ((int64_t)2 * blockIdx.x + (u.tile_begin == 0 ? 1 : 0)) * p.part_rows + wt + (dual ? 0 : t * kTile) : 0;
        float* part = TREE ? p.part_o + slot * HD : nullptr;
#pragma unroll
        for (int x = 0; x < HD; x += 32) {
          unsigned o[32];
          tmem_ld32(o, from0 + x);
          tmem_wait_ld();
          tmem_pin(o);
          float v[32];
#pragma unroll
          for (int k = 0; k < 32; k++) v[k] = __uint_as_float(o[k]) * f0;
          if (two) {
            tmem_ld32(o, from1 + x);
            tmem_wait_ld();
            tmem_pin(o);
#pragma unroll
            for (int k = 0; k < 32; k++) v[k] += __uint_as_float(o[k]) * f1;
          }
          if (valid) {
#pragma unroll
            for (int k = 0; k < 32; k++) v[k] = l == 0.f ? 0.f : v[k] * inv;
            if (whole) {
#pragma unroll
              for (int k = 0; k < 32; k += 8)
                *(uint4*)(out + x + k) = make_uint4(pack_bf16(v[k], v[k + 1]), pack_bf16(v[k + 2], v[k + 3]),
                                                    pack_bf16(v[k + 4], v[k + 5]), pack_bf16(v[k + 6], v[k + 7]));
            } else {
#pragma unroll
              for (int k = 0; k < 32; k += 4) *(float4*)(part + x + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
            }
          }
        }
        if (valid) {
          if (!whole) p.part_lse[slot] = lse2;
          else if (p.lse) p.lse[gtok * p.nq + head] = lse2 * 0.6931471805599453f;
        }
      }
      if (dual) {
        tc_fence_before();
        named_barrier(3, 256);       // the second warpgroup's O and statistics have been read
        tc_fence_after();
      }
    }
  } else if (warp == kProducer) {
    // ================================ K and V tiles into the ring ======================================================
    if (lane == 0) {
      constexpr int kN = FP8 ? L::kRawStages : L::kStages;
      uint64_t* full = FP8 ? h.raw_full : h.full;
      uint64_t* empty = FP8 ? h.raw_empty : h.empty;
      unsigned issued = 0;
      bool on = true;
      while (units.next(p, h, u)) {
        for (int j = u.tile_begin; j < u.tile_end; j++) {
          for (int kv = 0; kv < 2; kv++) {
            const int st = issued % kN;
            attn_wait(&empty[st], (issued / kN & 1) ^ 1, h);
            on = on && !*(volatile int*)&h.dead;
            if (!on) continue;
            const CUtensorMap* map = kv ? &map_v : &map_k;
            const int y = u.key0 + j * kTile;
            if (FP8) {
              mbar_expect_tx(&full[st], L::kRawBytes);
              tma_load_4d(smem + L::kRaw + st * L::kRawBytes, map, 0, y, u.head, u.seq, &full[st]);
            } else {
              unsigned char* dst = smem + L::kRing + st * L::kTileBytes;
              mbar_expect_tx(&full[st], L::kTileBytes);
              for (int x = 0; x < HD / 64; x++) tma_load_4d(dst + x * kBox, map, x * 64, y, u.head, u.seq, &full[st]);
            }
            issued++;
          }
        }
      }
      if (*(volatile int*)&h.dead) {   // copies in flight land before the block ends
        for (unsigned i = issued > kN ? issued - kN : 0; i < issued; i++)
          for (int n = 0; n < 1 << 16 && !mbar_try_wait(&full[i % kN], i / kN & 1); n++) {}
      }
    }
    __syncwarp();
  } else if (warp == kIssuer) {
    // ================================ the matrix products ==============================================================
    if (lane == 0) {
      constexpr unsigned kIdS = mma_idesc(kTile, kTile, false), kIdO = mma_idesc(kTile, HD, true);
      unsigned q_phase[2] = {0, 0}, p_phase[2] = {0, 0};
      int ring = 0;
      const unsigned q0 = smem_u32(smem + L::kQ), ring0 = smem_u32(smem + L::kRing);
      while (units.next(p, h, u)) {
        const int n0 = unit_steps<TREE>(p, u, dual, 0), n1 = unit_steps<TREE>(p, u, dual, 1);
        const int most = max(n0, n1);
        auto scores = [&](int t, int i) {
          const int pos = ring + 2 * (dual ? 2 * i + t : i), st = pos % L::kStages;
          attn_wait(&h.full[st], pos / L::kStages & 1, h);
          if (*(volatile int*)&h.dead) return;
          tc_fence_after();
          const unsigned qa = q0 + t * L::kTileBytes, ka = ring0 + st * L::kTileBytes;
#pragma unroll
          for (int k = 0; k < HD / 16; k++)
            mma_ss(tmem + t * kTile, smem_desc(qa + k / 4 * kBox + k % 4 * 32, 16, 1024),
                   smem_desc(ka + k / 4 * kBox + k % 4 * 32, 16, 1024), kIdS, k > 0);
          mma_commit(&h.s_full[t]);
          if (dual || t == 1 || i >= n1) mma_commit(&h.empty[st]);
        };
        for (int t = 0; t < 2; t++) {
          if (!(t ? n1 : n0)) continue;
          attn_wait(&h.q_full[t], q_phase[t]++ & 1, h);
          scores(t, 0);
        }
        for (int i = 0; i < most; i++) {
          for (int t = 0; t < 2; t++) {
            const int n = t ? n1 : n0;
            if (i >= n) continue;
            const int pos = ring + 2 * (dual ? 2 * i + t : i) + 1, st = pos % L::kStages;
            attn_wait(&h.p_full[t], p_phase[t]++ & 1, h);
            attn_wait(&h.full[st], pos / L::kStages & 1, h);
            if (!*(volatile int*)&h.dead) {
              tc_fence_after();
              if (!*(volatile int*)&h.skip[t]) {
                const unsigned va = ring0 + st * L::kTileBytes;
#pragma unroll
                for (int k = 0; k < kTile / 16; k++)
                  mma_ts(tmem + 2 * kTile + t * HD, tmem + t * kTile + k * 8, smem_desc(va + k * 2048, kBox, 1024), kIdO,
                         i > 0 || k > 0);
              }
              if (i + 1 == n) mma_commit(&h.o_done[t]);
              if (dual || t == 1 || i >= n1) mma_commit(&h.empty[st]);
            }
            if (i + 1 < n) scores(t, i + 1);
          }
        }
        ring += 2 * (u.tile_end - u.tile_begin);
      }
      if (*(volatile int*)&h.dead) {   // products in flight end before TMEM is given back
        mma_commit(&h.fin);
        for (int n = 0; n < 1 << 16 && !mbar_try_wait(&h.fin, 0); n++) {}
      }
    }
    __syncwarp();
  } else if (FP8 && warp >= 8 && warp < 12) {
    // ================================ 8-bit tiles widened to bf16 ======================================================
    const int wt = threadIdx.x & 127;
    constexpr int kChunks = HD / 16;                  // 16-byte chunks of an 8-bit row
    int pos = 0;
    while (units.next(p, h, u)) {
      for (int n = 2 * (u.tile_end - u.tile_begin); n; n--, pos++) {
        const int raw = pos % (FP8 ? L::kRawStages : 1), st = pos % L::kStages;
        attn_wait(&h.raw_full[raw], pos / (FP8 ? L::kRawStages : 1) & 1, h);
        attn_wait(&h.empty[st], (pos / L::kStages & 1) ^ 1, h);
        const unsigned char* src = smem + L::kRaw + raw * L::kRawBytes;
        unsigned char* dst = smem + L::kRing + st * L::kTileBytes;
#pragma unroll 4
        for (int i = 0; i < kChunks; i++) {
          const int e = i * kTile + wt, r = e / kChunks, ch = e % kChunks;
          const uint4 v = *(const uint4*)(src + e * 16);
          const unsigned vv[4] = {v.x, v.y, v.z, v.w};
          unsigned w[8];
#pragma unroll
          for (int k = 0; k < 8; k++) {
            unsigned half2;
            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(half2) : "h"((unsigned short)(vv[k >> 1] >> (k & 1) * 16)));
            float lo, hi;
            asm("{ .reg .b16 a, b; mov.b32 {a, b}, %2; cvt.f32.f16 %0, a; cvt.f32.f16 %1, b; }" : "=f"(lo), "=f"(hi) : "r"(half2));
            w[k] = pack_bf16(lo, hi);                 // exact: 4 significant bits, exponents of a half
          }
#pragma unroll
          for (int k = 0; k < 2; k++) {
            const int cc = 2 * ch + k;
            *(uint4*)(dst + cc / 8 * kBox + r * 128 + (((cc & 7) ^ (r & 7)) << 4)) =
                make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
          }
        }
        fence_async_smem();
        mbar_arrive(&h.full[st]);
        mbar_arrive(&h.raw_empty[raw]);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kIssuer) tmem_free(tmem, 512);
}

// ---- parts of one item joined (tree) ----------------------------------------------------------------------------
// One warp for each (row of an item); items whose tiles one block had are complete already, sequences of a bad length
// become NaN.  O = sum_i w_i O_i / sum_i w_i, w_i = 2^(lse_i - max): the parts carry O_i / l_i and log2 of their sums.
template <int HD>
__global__ void __launch_bounds__(256) attn_join_kernel(const AttnParams p, int blocks) {
  __shared__ int64_t sh[2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int head = blockIdx.y, seq = blockIdx.z;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tiles = tree_tiles(p, p.lens[seq]);
  if (warp == 0) {
    int64_t before = 0;
    for (int b = lane; b < seq; b += 32) before += tree_tiles(p, p.lens[b]);
#pragma unroll
    for (int o = 16; o; o >>= 1) before += __shfl_xor_sync(~0u, before, o);
    const int64_t total = tree_total(p, lane);
    if (lane == 0) sh[0] = before * p.nkv * p.row_tiles, sh[1] = tree_per_block(p, total, blocks);
  }
  __syncthreads();
  const int rows = p.rows * p.rep;
  const int row = blockIdx.x * 8 + warp;
  if (row >= rows) return;
  const int tok = div_rep(p, row), q_head = head * p.rep + row - tok * p.rep;
  __nv_bfloat16* out = p.out + (int64_t)seq * p.o_seq + tok * p.o_row + q_head * p.o_head;
  float* lse = p.lse ? p.lse + ((int64_t)seq * p.rows + tok) * p.nq + q_head : nullptr;
  constexpr int kEach = HD / 32;
  float v[kEach] = {};
  if (tiles == 0) {
#pragma unroll
    for (int k = 0; k < kEach; k++) v[k] = CUDART_NAN_F;
    if (lse && lane == 0) *lse = CUDART_NAN_F;
  } else {
    const int rt = row / p.part_rows;
    const int64_t first = sh[0] + ((int64_t)head * p.row_tiles + rt) * tiles, per = sh[1];
    const int c0 = (int)(first / per), c1 = (int)((first + tiles - 1) / per);
    if (c0 == c1) return;
    const int64_t local = row - rt * p.part_rows;
    auto slot = [&](int b) { return ((int64_t)2 * b + (b == c0 ? 1 : 0)) * p.part_rows + local; };
    float m = -CUDART_INF_F;
    bool nan = false;
    for (int b = c0 + lane; b <= c1; b += 32) {
      const float x = p.part_lse[slot(b)];
      nan |= x != x;
      m = fmaxf(m, x);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
    float sum = 0.f;
    for (int b = c0; b <= c1; b++) {
      const float w = m == -CUDART_INF_F ? 0.f : exp2f(p.part_lse[slot(b)] - m);
      sum += w;
      const float* o = p.part_o + slot(b) * HD + lane * kEach;
      float x[kEach];
      if (kEach == 4) *(float4*)x = *(const float4*)o;
      else *(float2*)x = *(const float2*)o;
#pragma unroll
      for (int k = 0; k < kEach; k++) v[k] += w * x[k];
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int k = 0; k < kEach; k++) v[k] *= inv;
    if (__any_sync(~0u, nan)) m = CUDART_NAN_F;
    if (lse && lane == 0) *lse = sum == 0.f ? (m == m ? -CUDART_INF_F : m) : (m + log2f(sum)) * 0.6931471805599453f;
  }
  if (kEach == 4) *(uint2*)(out + lane * 4) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[kEach - 2], v[kEach - 1]));
  else *(unsigned*)(out + lane * 2) = pack_bf16(v[0], v[1]);
}

}  // namespace amk
