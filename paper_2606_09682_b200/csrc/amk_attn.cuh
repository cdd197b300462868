// The attention kernel of amk_prompt_attention and amk_tree_attention, and the parameters they share.
//
// Mathematics.  For a block of query rows (a row is a query token and one of the query heads of a kv head: all heads
// of a group share the K/V tiles) and the key tiles it sees, one pass with a running maximum m and sum l:
//   S = Q K^T;  m' = max(m, rowmax S);  P = 2^((S - m') c), c = scale log2 e;  l = l 2^((m - m') c) + rowsum P;
//   O = O 2^((m - m') c) + P V;  at the end O / l.
// O is rescaled only when m rises by more than 8 / c (P then stays below 2^8, nothing is lost: P is a floating-point
// number and l and O share the reference).  Where P is f16 (below), 2^9 times as much is made of it.
//
// Work.  One block an SM: two row tiles of 128 rows share every K/V tile of 128 keys (prompts, large drafts), or, where a
// draft has 128 rows at most, take every second key tile each and are joined at the end.  A producer warp keeps a ring of
// tiles full by TMA, one warp issues the products (S and O in TMEM, P over S as the A operand of P V), four warpgroups
// make the softmax, so that one tile's exponentials run beside the other's products.  Prompts: units of 256 / rep tokens of
// a kv head, one for each block of the grid; a block that runs takes over the units of blocks that have not begun while its
// own last tiles are on their way (one unit a block: 468 us at 8192 tokens, 41 us for eight prompts of 1 to 1291 tokens; so:
// 445 and 35 us).  Trees: the key tiles of the whole batch in equal runs (below), parts joined by a second kernel.
//
// What bounds it.  Prompts: the chain scores -> softmax -> products of a tile, about 3500 cycles for 2054 cycles of products a
// pair of tiles (the exponentials alone are 2048): 8192 tokens, 32 heads of 128 on 8, 550 GFLOP in 445 us = 1.24 PFLOP/s for one
// launch; in a row of calls, under the power cap, 514 us = 1.07 PFLOP/s.
// head_dim 64 has half the products for the same exponentials.  Trees: HBM in long runs (32 sequences of 8000 positions,
// one token each: 1.05 GB in 178 us a call = 5.9 TB/s); a short call the 8 us that a cold block takes from its start to its first
// output, of which the tiles are the least.  The 8-bit cache: its tiles' way through shared memory (raw in, f16 out, read
// as operands).
// Registers are what this kernel is short of: a spilled one is fetched from L2 behind the stream of tiles (shared memory
// leaves no L1), and cost up to half the time where it stood in the steps.
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
  float* part_lse;                 // tree: [2 * gridDim][2][part_rows]: a row's maximum and its sum
  int64_t q_seq, q_row, q_head, o_seq, o_row, o_head;
  int n_seqs, nq, nkv, rep;
  int rows;                        // prompt: all tokens; tree: drafted tokens of a sequence
  int slots;
  int part_rows;                   // tree: 128 (both warpgroups work on the same rows) or 256
  int row_tiles;                   // tree: blocks of part_rows rows per (sequence, kv head)
  int min_tiles;                   // tree: key tiles a block takes at least
  int cluster;                     // tree: blocks of one item, which meet at the end; 0: runs and a second kernel
  unsigned rep_inv;                // ceil(2^32 / rep), 0 for rep = 1
  unsigned tiles;                  // K and V tiles that a block may ask for (a test's limit, else the largest number)
  unsigned wait_cycles;            // a wait runs out after so many
  float scale;
};

constexpr int kTile = 128;         // rows of a Q tile, keys of a K/V tile
// row / rep, exact for rows below 2^28
__device__ __forceinline__ int div_rep(const AttnParams& p, int row) {
  return p.rep_inv ? (int)__umulhi((unsigned)row, p.rep_inv) : row;
}
constexpr float kLog2e = 1.4426950408889634f;

// How often a bounded wait of an attention kernel ran out, and how many of these amk_operator_status has told of.  (Two numbers
// that only grow: one that is read and then cleared loses what happens in between on another stream.)
static __device__ unsigned g_attn_expired[2];

__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {   // round to nearest even
  unsigned r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// The same value in every lane, and the compiler knows it: addresses that follow from it stay in uniform registers,
// where the matrix instructions want them.
template <class T>
__device__ __forceinline__ T uniform(T x) {
  return (T)__shfl_sync(~0u, (int)x, 0);
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// Four e4m3 codes to four f16, exactly, NaN included.
__device__ __forceinline__ void widen_e4m3(unsigned* w, unsigned codes) {
  asm("{ .reg .b16 l, h; mov.b32 {l, h}, %2; cvt.rn.f16x2.e4m3x2 %0, l; cvt.rn.f16x2.e4m3x2 %1, h; }"
      : "=r"(w[0]), "=r"(w[1])
      : "r"(codes));
}
__device__ __forceinline__ unsigned pack_f16(float lo, float hi) {    // round to nearest even
  unsigned r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ void unpack_f16(float& lo, float& hi, unsigned w) {
  asm("{ .reg .b16 a, b; mov.b32 {a, b}, %2; cvt.f32.f16 %0, a; cvt.f32.f16 %1, b; }" : "=f"(lo), "=f"(hi) : "r"(w));
}
// Operands of the matrix instructions: bf16, or f16 over the 8-bit cache (see attn_kernel).
template <bool HALF>
__device__ __forceinline__ unsigned pack2(float lo, float hi) { return HALF ? pack_f16(lo, hi) : pack_bf16(lo, hi); }
template <bool HALF>
__device__ __forceinline__ void unpack2(float& lo, float& hi, unsigned w) {
  if (HALF) unpack_f16(lo, hi, w);
  else lo = bf16_lo(w), hi = bf16_hi(w);
}
// acc + 0 * w for two operands at once: NaN from the first value on that is not finite
template <bool HALF>
__device__ __forceinline__ unsigned zero_times(unsigned w, unsigned acc) {
  unsigned d;
  if (HALF) asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(w), "r"(0u), "r"(acc));
  else asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(w), "r"(0u), "r"(acc));
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

// Tree: the key tiles of all (sequence, kv head, row block) in that order, cut into equal runs, one for each block.  An
// item counts kUnitCost tiles more than it has, in front of its first: a block that begins another item reads another Q,
// fills the pipeline again and writes another output or part (2 / 3 / 4 / 5 / 6 / 7 / 9 / 12 tiles, us: eight ragged
// sequences of up to 8000 positions 65 / 50 / 49 / 45 / 45 / 45 / 45 / 46, over the 8-bit cache 76 / 58 / 55 / 52 / 52 / 52 /
// 54 / 55; sixty of up to 2000 there 110 / 99 / 90 / 88 / 89 / 88 / 92 / 99; one of 8099 20.7 / 20.5 / 20.3 / 20.5 / 20.5 / 20.7 /
// 20.6 / 19.8).
constexpr int kUnitCost = 6;
__device__ __forceinline__ int tree_tiles(const AttnParams& p, int len) {   // key tiles of one item; 0: bad length
  return len < 0 || len > p.slots - p.rows ? 0 : (len + p.rows + kTile - 1) / kTile;
}
__device__ __forceinline__ int tree_slots(int tiles) { return tiles ? tiles + kUnitCost : 0; }
// slots of a warp's 32 sequences from b0 on, this lane's
__device__ __forceinline__ int tree_slots_of(const AttnParams& p, int b) {
  return b < p.n_seqs ? tree_slots(tree_tiles(p, __ldg(p.lens + b))) * p.nkv * p.row_tiles : 0;
}
__device__ __forceinline__ int warp_sum(int x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
  return x;
}
// slots of one run, the same in every block; `first`: this lane's share of the first 32 sequences (one whole warp)
__device__ __forceinline__ int tree_run(const AttnParams& p, int first, int lane, int blocks) {
  int sum = first;
  for (int b = 32 + lane; b < p.n_seqs; b += 32) sum += tree_slots_of(p, b);
  return max((warp_sum(sum) + blocks - 1) / blocks, p.min_tiles);
}

}  // namespace amk

namespace amk {

// ---- shared memory ----------------------------------------------------------------------------------------------
// Tiles of 64 elements x 128 rows of 128 bytes, swizzled by TMA's 128-byte pattern: the 16-byte chunk c of row r lies
// at r * 128 + ((c ^ (r & 7)) << 4).
constexpr int kBox = 64 * kTile * 2;
constexpr int kHeadBytes = 8192;
constexpr int kUnitRing = 4;
template <int HD, bool FP8>
struct AttnSmem {
  static constexpr int kTileBytes = HD / 64 * kBox;                // one bf16 tile of 128 rows
  static constexpr int kStages = FP8 ? (HD == 128 ? 3 : 6) : (HD == 128 ? 4 : 8);
  static constexpr int kRawBytes = FP8 ? HD * kTile : 0;           // one 8-bit tile
  static constexpr int kRawStages = FP8 ? (HD == 128 ? 3 : 6) : 0;
  static constexpr int kQ = 0;
  static constexpr int kRing = 2 * kTileBytes;
  static constexpr int kRaw = kRing + kStages * kTileBytes;
  static constexpr int kHead = kRaw + kRawStages * kRawBytes;      // AttnHead
  static constexpr int kBytes = kHead + kHeadBytes + 1024;               // + alignment of the dynamic buffer
  static_assert(kBytes <= 227 * 1024, "shared memory of one SM");
};
struct AttnHead {
  uint64_t full[10], empty[10];        // ring of K and V tiles (bf16)
  uint64_t raw_full[8], raw_empty[8];  // ring of 8-bit tiles
  uint64_t q_full[2], s_full[2], p_full[2], o_done[2], fin;
  unsigned tmem;
  int dead;                            // a bounded wait ran out: nobody waits or issues any more
  unsigned wait_cycles;
  int skip[2];                         // this step's P V was done by the warpgroup itself
  float mx[2][2][kTile];               // [tile][half]: row maxima, and at the end row sums, of half the columns; last, in a
                                       // cluster, [0]: the part's maxima and sums
  float m[kTile], l[kTile];            // the second tile's statistics (both tiles of the same rows)
  int unit[8];                         // where the block's work begins; behind it what the producer had asked for at its end
  uint64_t unit_full[kUnitRing], unit_empty[kUnitRing], next_full;   // prompts: blocks of queries, taken one after the other
  int4 units[kUnitRing], now_of[2][2];                               // the producer's; the two last ones of each row tile
  uint4 next;                                                        // answer of the hardware's scheduler
  int walk[16][8];                     // each softmax warp's place in the walk and its unit: registers are short there
  Unit now[16];
  float row_c[2][kTile];               // 8-bit cache: scale * log2 e over the power of two that each row of Q was multiplied by
  unsigned long long word0[2][kTile];  // first word of each row's mask
};
static_assert(sizeof(AttnHead) <= kHeadBytes, "head");

constexpr unsigned kWaitCycles = 4000000000u;
// A whole warp waits for the phase of the given parity, about two seconds (kWaitCycles) at most (the SM's cycle counter: the global
// timer is read through a unit that all SMs share); false if that ran out.  The votes keep the warp's control flow
// uniform: behind a wait that each lane leaves by itself, the matrix instructions of one tile took ten times as long
// to issue (700 cycles instead of 70).
template <class Head>
__device__ __forceinline__ bool attn_wait(uint64_t* bar, unsigned parity, Head& h) {
  if (__all_sync(~0u, mbar_try_wait(bar, parity))) return true;
  const unsigned t0 = clock();
  for (;;) {
    for (int i = 0; i < 32; i++)
      if (__all_sync(~0u, mbar_try_wait(bar, parity))) return true;
    if (__any_sync(~0u, *(volatile int*)&h.dead)) return false;
    if (__any_sync(~0u, (unsigned)clock() - t0 > h.wait_cycles)) {
      *(volatile int*)&h.dead = 1;
      atomicAdd(&g_attn_expired[0], 1u);             // (of every lane: how many does not matter)
      return false;
    }
  }
}
// One arrival for the whole warp: 32 of them would queue up at the barrier's word.
__device__ __forceinline__ void warp_arrive(uint64_t* bar, int lane) {
  __syncwarp();
  if (lane == 0) mbar_arrive(bar);
}
// whether a predicate holds in any thread of a pair of warps
__device__ __forceinline__ bool any_of_pair(bool pred, int id) {
  unsigned r;
  asm volatile(
      "{ .reg .pred p, q; setp.ne.u32 p, %1, 0; bar.red.or.pred q, %2, 64, p; selp.u32 %0, 1, 0, q; }"
      : "=r"(r)
      : "r"((unsigned)pred), "r"(id)
      : "memory");
  return r != 0;
}
// barrier ids: 1..8 a pair of warps (the two halves of 32 rows), 9, 10 a tile, 11 both tiles
__device__ __forceinline__ unsigned any_of_tile(unsigned pred, int id) {
  unsigned r;
  asm volatile(
      "{ .reg .pred p, q; setp.ne.u32 p, %1, 0; bar.red.or.pred q, %2, 256, p; selp.u32 %0, 1, 0, q; }"
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
  int left;                        // slots of this block's run that are still to come
  int seq, len, tiles, item, within, items;
  __device__ __forceinline__ void init(const AttnParams& p, const AttnHead& h) {
    seq = h.unit[0], item = h.unit[1], within = h.unit[2], len = h.unit[3], left = h.unit[4];
    tiles = tree_tiles(p, len);
    items = p.nkv * p.row_tiles;
  }
  // the state in shared memory, one copy for a warp
  __device__ __forceinline__ void save(int* at, int lane) const {
    __syncwarp();
    if (lane == 0) at[0] = left, at[1] = seq, at[2] = len, at[3] = tiles, at[4] = item, at[5] = within;
    __syncwarp();
  }
  __device__ __forceinline__ void restore(const volatile int* at) {
    left = at[0], seq = at[1], len = at[2], tiles = at[3], item = at[4], within = at[5];
  }
  __device__ __forceinline__ bool next(const AttnParams& p, AttnHead&, Unit& u) {
    int first, last;
    do {
      if (left <= 0) return false;
      while (item == items || tiles == 0) {   // something is left: a sequence with tiles follows
        item = 0;
        len = __ldg(p.lens + ++seq);
        tiles = tree_tiles(p, len);
      }
      const int run = min(left, tiles + kUnitCost - within);
      first = max(within - kUnitCost, 0), last = within + run - kUnitCost;
      left -= run;
      within = 0;
      item++;
    } while (last <= first);                  // (only slots that stand for the beginning)
    u.seq = seq, u.head = p.row_tiles == 1 ? item - 1 : (item - 1) / p.row_tiles, u.len = len;
    u.row0 = (item - 1 - u.head * p.row_tiles) * p.part_rows;
    u.n_rows = min(p.part_rows, p.rows * p.rep - u.row0);
    u.tok0 = 0, u.n_tok = p.rows, u.key0 = 0;
    u.tile_begin = first, u.tile_end = last, u.item_tiles = tiles;
    return true;
  }
};

// Prompts: the block's own unit of queries, and then those of blocks that have not been launched yet, which the producer
// warp takes over from the hardware's scheduler one at a time, when it has asked for the last tile of the one before.  The
// others read them from a ring.
template <>
struct Units<false> {
  int n;                           // units taken so far
  __device__ __forceinline__ void init(const AttnParams&, const AttnHead&) { n = 0; }
  __device__ __forceinline__ static bool set(const AttnParams& p, const int4& x, Unit& u) {
    u.seq = 0, u.head = x.x, u.key0 = x.y, u.tok0 = x.z, u.n_tok = x.w;
    u.row0 = 0, u.n_rows = u.n_tok * p.rep, u.len = 0;
    u.tile_begin = 0, u.tile_end = u.item_tiles = (u.tok0 + u.n_tok + kTile - 1) / kTile;
    return x.x >= 0;
  }
  __device__ __forceinline__ int4 take(AttnHead& h, int lane) {
    const int at = n & (kUnitRing - 1);
    int4 x = make_int4(-1, 0, 0, 0);
    if (attn_wait(&h.unit_full[at], n / kUnitRing & 1, h)) x = *(const int4*)&h.units[at];
    n++;
    warp_arrive(&h.unit_empty[at], lane);
    return x;
  }
  // one warp
  __device__ __forceinline__ bool next(const AttnParams& p, AttnHead& h, Unit& u) { return set(p, take(h, threadIdx.x & 31), u); }
  // The eight warps of a row tile together: their barriers want all of them to see the same units, also after a wait that
  // ran out.  The barrier is also the one behind which the last unit's output has left the tile's shared memory.
  __device__ __forceinline__ bool next_of_tile(const AttnParams& p, AttnHead& h, Unit& u, int t, int warp, int lane, int id) {
    const int at = n & 1;
    if ((warp & 7) == 0) {
      const int4 x = take(h, lane);
      if (lane == 0) h.now_of[t][at] = x;
    } else {
      n++;
    }
    named_barrier(id, 256);
    return set(p, *(const int4*)&h.now_of[t][at], u);
  }
};

// Where the blocks of 256 / rep query tokens lie.  Those with the most keys come first, so that the short ones fill the
// end: all prompts' blocks by their place in the prompt, the last places first (with more than 32 prompts one prompt after
// the other, the last places first within each).  One whole warp; lane i has prompt s0 + i.
struct PromptBlocks {
  int s0, before;                  // first prompt of the 32 at hand, blocks of the prompts in front of them
  int a, b, own;                   // this lane's prompt and its blocks
  __device__ __forceinline__ void read(const AttnParams& p, int lane) {
    const int s = s0 + lane, per = 2 * kTile / p.rep;
    a = b = 0;
    if (s < p.n_seqs) a = __ldg(p.lens + s), b = __ldg(p.lens + s + 1);
    own = a >= 0 && a <= b && b <= p.rows ? (b - a + per - 1) / per : 0;
  }
  __device__ __forceinline__ void init(const AttnParams& p, int lane) {
    s0 = before = 0;
    read(p, lane);
  }
  // {head, first row of the prompt, first token, tokens} of a block of the grid; head -1: there is none
  __device__ __forceinline__ int4 find(const AttnParams& p, int block, int lane) {
    const int per = 2 * kTile / p.rep, head = block % p.nkv;
    int idx = block / p.nkv, f = -1, place = 0;
    if (p.n_seqs <= 32) {
      auto from = [&](int x) { return (int)__reduce_add_sync(~0u, max(own - x, 0)); };   // blocks from place x on
      if (from(0) > idx) {
        int low = 0, high = (int)__reduce_max_sync(~0u, own);              // the largest place with more than idx of them
        while (high - low > 1) {
          const int mid = (low + high) / 2;
          if (from(mid) > idx) low = mid;
          else high = mid;
        }
        unsigned here = __ballot_sync(~0u, own > low);
        for (int skip = idx - from(low + 1); skip; skip--) here &= here - 1;
        f = __ffs(here) - 1, place = low;
      }
    } else {
      if (idx < before) init(p, lane);
      for (;;) {
        int sum = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int x = __shfl_up_sync(~0u, sum, o);
          if (lane >= o) sum += x;
        }
        const unsigned hit = __ballot_sync(~0u, sum > idx - before);
        if (hit) {
          f = __ffs(hit) - 1;
          place = __shfl_sync(~0u, sum, f) - 1 - (idx - before);
          break;
        }
        if (p.n_seqs - s0 <= 32) break;
        before += __shfl_sync(~0u, sum, 31);
        s0 += 32;
        read(p, lane);
      }
    }
    if (f < 0) return make_int4(-1, 0, 0, 0);
    const int a_f = __shfl_sync(~0u, a, f), b_f = __shfl_sync(~0u, b, f);
    return make_int4(head, a_f, place * per, min(per, b_f - a_f - place * per));
  }
};

// Key tiles that row tile t of the unit works on; DUAL: every second one of the unit's.  A unit's key tiles are taken from the
// last one down: those that hide keys are then among the first, which wants the careful softmax anyway (prompts of
// 1 to 1291 tokens from the first one up 36.1 us, so 34.9 us; eight ragged sequences of up to 8000 positions with 32 tokens
// each 45.9 and 45.0 us; a single token over 1025 positions 9.2 and 9.5 us).
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

// the mask words of a drafted token (tokens behind the last: rows that nobody reads)
__device__ __forceinline__ int64_t mask_at(const AttnParams& p, int seq, int tok) {
  return ((int64_t)seq * p.rows + min(tok, p.rows - 1)) * ((p.rows + 63) / 64);
}
// 32 bits of a drafted token's mask from drafted index idx on (idx may be negative: bits below 0 are 0).  w0 is the
// mask's first word, w its words; without a mask (w null) a chain: indices 0..tok.
__device__ __forceinline__ unsigned tree_bits32(const unsigned long long* w, unsigned long long w0, int rows, int tok, int idx) {
  if (idx >= rows || idx <= -32) return 0;
  if (!w) {
    const int n = tok + 1 - idx;      // bits below n
    unsigned r = n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
    if (idx < 0) r &= ~0u << -idx;
    return r;
  }
  unsigned long long v;
  if (idx < 0) {
    v = w0 << -idx;
  } else {
    const int word = idx >> 6, off = idx & 63;
    v = (word ? w[word] : w0) >> off;
    if (off > 32 && (word + 1) * 64 < rows) v |= w[word + 1] << (64 - off);
  }
  const int left = rows - idx;        // bits from the last drafted token on are nobody's
  return left >= 32 ? (unsigned)v : (unsigned)v & ((1u << left) - 1u);
}

// O += P V of 64 keys for this warp's rows, key by key and only for the keys that a row sees: for tiles with values that
// are not finite behind a mask, where 0 * V would not be 0.  P in TMEM as the matrix unit would read it; vt: the tile, used
// from its row `key` on.
template <int HD, bool HALF>
__device__ __noinline__ void product_by_key(unsigned tp, unsigned see0, unsigned see1, const unsigned char* vt, int key,
                                            unsigned to, bool more) {
  float pl[64];                                        // (in local memory: walked by key)
  {
    unsigned r[32];
    tmem_ld32(r, tp);
    tmem_wait_ld();
    tmem_pin(r);
#pragma unroll
    for (int k = 0; k < 32; k++) unpack2<HALF>(pl[2 * k], pl[2 * k + 1], r[k]);
  }
  for (int x = 0; x < HD; x += 32) {
    unsigned o[32];
    tmem_ld32(o, to + x);
    tmem_wait_ld();
    tmem_pin(o);
    float a[32];
#pragma unroll
    for (int k = 0; k < 32; k++) a[k] = more ? __uint_as_float(o[k]) : 0.f;
    for (int k = 0; k < 64; k++) {
      if (!((k < 32 ? see0 : see1) >> (k & 31) & 1)) continue;
      const int r = key + k;
#pragma unroll
      for (int ch = 0; ch < 4; ch++) {
        const int cc = x / 8 + ch;
        const uint4 v = *(const uint4*)(vt + cc / 8 * kBox + r * 128 + (((cc & 7) ^ (r & 7)) << 4));
        const unsigned vv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; e++) {
          float v0, v1;
          unpack2<HALF>(v0, v1, vv[e]);
          a[ch * 8 + 2 * e] += pl[k] * v0;
          a[ch * 8 + 2 * e + 1] += pl[k] * v1;
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

// The block's dynamic shared memory, from a multiple of 1024 bytes on.
__device__ __forceinline__ unsigned char* attn_smem() {
  extern __shared__ unsigned char smem_raw[];
  return (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
}

// The block's end, all threads, behind a barrier: if a wait ran out, copies and products in flight end (waits again, with a limit)
// before their memory is given back.  A function of its own that finds everything by itself: whatever the kernel held in a
// register for this cost 4 % of a long prompt.
template <int HD, bool FP8>
__device__ __noinline__ void end_in_flight() {
  using L = AttnSmem<HD, FP8>;
  constexpr unsigned kN = FP8 ? L::kRawStages : L::kStages, kProducer = FP8 ? 20 : 16;
  AttnHead& h = *(AttnHead*)(attn_smem() + L::kHead);
  if (!h.dead) return;
  const unsigned warp = threadIdx.x >> 5;
  if (warp == kProducer) {
    uint64_t* full = FP8 ? h.raw_full : h.full;
    const unsigned issued = (unsigned)h.unit[5], asked = (unsigned)h.unit[6], told = (unsigned)h.unit[7];
    for (unsigned i = issued > kN ? issued - kN : 0; i < issued; i++)
      for (int n = 0; n < 1 << 16 && !__all_sync(~0u, mbar_try_wait(&full[i % kN], i / kN & 1)); n++) {}
    for (int n = 0; asked != told && n < 1 << 16 && !__all_sync(~0u, mbar_try_wait(&h.next_full, told & 1)); n++) {}
  }
  if (warp == kProducer + 1) {                         // the issuer
    mma_commit(elect_one(), &h.fin);
    for (int n = 0; n < 1 << 16 && !__all_sync(~0u, mbar_try_wait(&h.fin, 0)); n++) {}
  }
  __syncthreads();
}

// Over the 8-bit cache the matrix instructions work on f16: two e4m3 codes are two f16 by one conversion (to bf16 it takes
// three more), P has three bits more than in bf16, and a row of Q is exact in f16 after a power of two.  P is rounded to
// the operands' type (2^-8 of it in bf16), the sum l is not: the roundings of a row are independent and average out.
// f16 ends at 65504 and has its 11 bits down to 2^-14, the last one at 2^-24.  So that a key's share is not lost beside a far larger
// one whose V is small, P is 2^9 2^((S - m') c) there, l and O with it, and O is rescaled when m rises by more than 6 / c: the
// largest P of a row lies between 2^9 and 2^15, and P is off by 2^-11 of itself or 2^-34 of the largest.  (16 drafted tokens over
// eight caches of 64 to 8111 positions, 2^x up and a rise of 15 - x: x = 7 53.4, 9 53.5, 11 56.2 us; f16 without this 53.2.)
template <bool FP8>
struct Numerators {
  static constexpr float kRise = FP8 ? 6.f : 8.f, kUp = FP8 ? 9.f : 0.f;
};
// (S - m) c is made as S c - m c with the second product rounded, one instruction for two: that puts 2^-13 at most on an exponent
// while |m c| is below this, and any amount far beyond, where the difference is taken first.
constexpr float kFarScore = 4096.f;
// ---- the kernel -------------------------------------------------------------------------------------------------
template <int HD, bool TREE, bool FP8>
__global__ void __launch_bounds__(FP8 ? 768 : 640, 1)
    attn_kernel(const AttnParams p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using L = AttnSmem<HD, FP8>;
  constexpr int kProducer = FP8 ? 20 : 16, kIssuer = kProducer + 1;
  constexpr float kRise = Numerators<FP8>::kRise, kUp = Numerators<FP8>::kUp;
  unsigned char* smem = attn_smem();
  AttnHead& h = *(AttnHead*)(smem + L::kHead);
  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const bool dual = TREE && p.part_rows == kTile;

  // What touches no memory of the stream's comes first: the grid may begin while the one before it ends.
  if (warp == kIssuer) {
    tmem_alloc(&h.tmem, 512);
    if (lane == 0) {
      for (int i = 0; i < L::kStages; i++) mbar_init(&h.full[i], FP8 ? 6 : 1), mbar_init(&h.empty[i], 1);
      for (int i = 0; i < L::kRawStages; i++) mbar_init(&h.raw_full[i], 1), mbar_init(&h.raw_empty[i], 6);
      for (int t = 0; t < 2; t++) {
        mbar_init(&h.q_full[t], 8), mbar_init(&h.s_full[t], 1);
        mbar_init(&h.p_full[t], 8), mbar_init(&h.o_done[t], 1);
      }
      mbar_init(&h.fin, 1);
      h.dead = 0, h.wait_cycles = p.wait_cycles;
      mbar_fence_init();
    }
  }
  if (warp == kProducer) prefetch_map(lane == 0, &map_k), prefetch_map(lane == 0, &map_v);
  wait_for_grid_before();
  if (warp == 0) {
    // which part of the work is this block's
    if (TREE && p.cluster) {
      const int item = blockIdx.x / p.cluster, rank = blockIdx.x - item * p.cluster, seq = item / p.nkv;
      const int len = __ldg(p.lens + seq), tiles = tree_tiles(p, len), per = (tiles + p.cluster - 1) / p.cluster;
      const int begin = min(rank * per, tiles);
      if (lane == 0)
        h.unit[0] = seq, h.unit[1] = item - seq * p.nkv, h.unit[2] = kUnitCost + begin, h.unit[3] = len,
        h.unit[4] = min(per, tiles - begin);
    } else if (TREE) {
      const int mine = tree_slots_of(p, lane);
      const int per = tree_run(p, mine, lane, gridDim.x);
      int at = (int)blockIdx.x * per, seq = 0, item = 0, within = 0, len = 0, left = 0;
      for (int b0 = 0; b0 < p.n_seqs; b0 += 32) {
        const int own = b0 ? tree_slots_of(p, b0 + lane) : mine;
        int n = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int x = __shfl_up_sync(~0u, n, o);
          if (lane >= o) n += x;
        }
        const unsigned hit = __ballot_sync(~0u, n > at);
        if (hit && !left) {
          const int f = __ffs(hit) - 1;
          seq = b0 + f;
          len = __ldg(p.lens + seq);
          const int rel = at - __shfl_sync(~0u, n - own, f), slots = tree_slots(tree_tiles(p, len));
          item = rel / slots, within = rel - item * slots;
          left = per;                                 // or less: what the sequences from here on have
          at = 0;
          int rest = (b0 + lane > seq ? own : 0) + (lane == f ? own - rel : 0);
          for (int b = b0 + 32 + lane; rest < per && b < p.n_seqs; b += 32) rest += tree_slots_of(p, b);
          left = min(per, warp_sum(min(rest, per)));
          break;
        }
        at -= __shfl_sync(~0u, n, 31);
      }
      if (lane == 0) h.unit[0] = seq, h.unit[1] = item, h.unit[2] = within, h.unit[3] = len, h.unit[4] = left;
    }
  }
  PromptBlocks blocks;                                // (the producer's)
  int4 unit;
  if (!TREE && warp == kProducer) {
    if (lane == 0) {
      for (int i = 0; i < kUnitRing; i++) mbar_init(&h.unit_full[i], 1), mbar_init(&h.unit_empty[i], 3);
      mbar_init(&h.next_full, 1);
      mbar_fence_init();
    }
    blocks.init(p, lane);
    unit = blocks.find(p, blockIdx.x, lane);
    if (lane == 0 && unit.x >= 0) {                   // (else another block's comes first: below)
      h.units[0] = unit;
      mbar_arrive(&h.unit_full[0]);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const unsigned tmem = uniform(h.tmem);
  // TMEM columns: S0, S1, O0, O1; P of keys 0..63 over S columns 0..31, of keys 64..127 over 64..95
  if (TREE) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  Units<TREE> units;
  units.init(p, h);
  Unit u;

  if (!FP8) {
    // 640 threads of 96 registers at launch: 512 x 104 + 128 x 64 = 61440, all of them
    if (warp < 16) asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
  } else {
    // 768 threads of 80 registers at launch: 512 x 96 + 256 x 48 = 61440, all of them
    if (warp < 16) asm volatile("setmaxnreg.inc.sync.aligned.u32 96;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
  }

  if (warp < 16) {
    // ================================ softmax: two warpgroups for each row tile, half a row for each thread ============
    const int t = warp >> 3, half = warp >> 2 & 1, quarter = warp & 3, wr = quarter * 32 + lane, id = threadIdx.x & 255;
    const int pair_id = 1 + t * 4 + quarter, tile_id = 9 + t;
    const unsigned lanes = (unsigned)quarter * 32 << 16;
    const unsigned ts = tmem + lanes + t * kTile, to = tmem + lanes + 2 * kTile + t * HD;
    unsigned char* qs = smem + L::kQ + t * L::kTileBytes;
    float c = p.scale * kLog2e;
    unsigned s_phase = 0, o_phase = 0;
    int ring = 0;                                     // ring position of the unit's first tile
    bool again = false;
    if constexpr (TREE) units.save(h.walk[warp], lane);
    for (;;) {
      bool more;
      if constexpr (TREE) {
        units.restore(h.walk[warp]);
        more = units.next(p, h, u);
        units.save(h.walk[warp], lane);
      } else {
        more = units.next_of_tile(p, h, u, t, warp, lane, tile_id);
      }
      if (lane == 0) h.now[warp] = u;
      __syncwarp();
      if (!more) break;
      const int steps = unit_steps<TREE>(p, u, dual, t);
      const int row_first = u.row0 + (dual ? 0 : t * kTile);                       // first row of this tile
      const int rows_here = dual ? u.n_rows : u.n_rows - t * kTile;                // may be <= 0
      const unsigned short* q = p.q + (int64_t)u.seq * p.q_seq + (int64_t)(u.key0 + u.tok0) * p.q_row +
                                (int64_t)u.head * p.rep * p.q_head;
      const bool live = quarter * 32 < rows_here;      // this warp has rows; the others only keep step
      if (TREE && again && steps) named_barrier(tile_id, 256); // the last unit's output has left the tile's shared memory
      again = true;
      if (steps) {
        // Q, 16 bytes at a time, all loads in flight before the first store; rows that do not exist are zero
        constexpr int kChunks = HD / 8, kEach = kTile * kChunks / 256;
        uint4 v[kEach];
#pragma unroll
        for (int i = 0; i < kEach; i++) {
          const int e = i * 256 + id, r = e / kChunks, ch = e % kChunks;
          v[i] = make_uint4(0, 0, 0, 0);
          if (r < rows_here) {
            const int row = row_first + r, tok = div_rep(p, row), hh = row - tok * p.rep;
            v[i] = __ldg((const uint4*)(q + tok * p.q_row + hh * p.q_head + ch * 8));
          }
        }
        if (TREE && p.mask && half == 0)
          h.word0[t][wr] = __ldg(p.mask + mask_at(p, u.seq, div_rep(p, row_first + wr)));
        if (FP8) {
          // to f16, each row times the power of two that brings its largest value to 2^14..2^15: exact but for what is
          // 2^-30 of that.  A row's chunks lie in neighbouring lanes.
#pragma unroll
          for (int i = 0; i < kEach; i++) {
            unsigned w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
            unsigned top = 0;                         // largest magnitude, as bits
#pragma unroll
            for (int k = 0; k < 4; k++) top = max(top, max(w[k] & 0x7fffu, w[k] >> 16 & 0x7fffu));
#pragma unroll
            for (int o = kChunks / 2; o; o >>= 1) top = max(top, __shfl_xor_sync(~0u, top, o));
            const int power = top ? min(14 + 127 - (int)(top >> 7), 120) : 0;
            const float by = __uint_as_float((unsigned)(127 + power) << 23);
#pragma unroll
            for (int k = 0; k < 4; k++) w[k] = pack_f16(bf16_lo(w[k]) * by, bf16_hi(w[k]) * by);
            v[i] = make_uint4(w[0], w[1], w[2], w[3]);
            const int e = i * 256 + id;
            // (no less than the smallest normal number: 0 times the -infinity of a hidden key would be NaN, and scores
            // of 2^31 at most vanish either way)
            if (e % kChunks == 0)
              h.row_c[t][e / kChunks] = fmaxf(p.scale * kLog2e * __uint_as_float((unsigned)(127 - power) << 23), 1.17549435e-38f);
          }
        }
#pragma unroll
        for (int i = 0; i < kEach; i++) {
          const int e = i * 256 + id, r = e / kChunks, ch = e % kChunks;
          *(uint4*)(qs + ch / 8 * kBox + r * 128 + (((ch & 7) ^ (r & 7)) << 4)) = v[i];
        }
        fence_async_smem();
        tc_fence_before();                             // the last unit's S and O have been read
        warp_arrive(&h.q_full[t], lane);
      }
      if constexpr (TREE) {
        // the next unit's Q into L2: behind the stream of tiles a load from HBM takes microseconds
        Units<TREE> ahead = units;
        Unit n;
        if (ahead.next(p, h, n)) {
          const int r = id >> 1, first = n.row0 + (dual ? 0 : t * kTile);
          if (r < (dual ? n.n_rows : n.n_rows - t * kTile)) {
            const int row = first + r, tok = div_rep(p, row), hh = row - tok * p.rep;
            const unsigned short* a = p.q + (int64_t)n.seq * p.q_seq + (int64_t)n.head * p.rep * p.q_head + tok * p.q_row +
                                      hh * p.q_head + (id & 1) * (HD / 2);
            asm volatile("prefetch.global.L2 [%0];" ::"l"(a));
          }
        }
      }
      // the steps before this one have keys that a row of this tile may not see
      const int hiding = (dual ? u.tile_end : u.tile_begin + steps) - (TREE ? u.len : u.tok0 + div_rep(p, row_first) + 1) / kTile;
      const int mask_to = dual ? (hiding - t + 1) >> 1 : hiding;
      float m = -CUDART_INF_F, l = 0.f;
      // What the steps need of the unit they read from shared memory: a register spilled here would be fetched from behind
      // the stream of tiles.
      for (int i = 0; i < steps; i++) {
        const bool masked = i < mask_to;
        attn_wait(&h.s_full[t], s_phase & 1, h);
        s_phase++;
        __syncwarp();
        tc_fence_after();
        if (FP8 && i == 0) c = h.row_c[t][wr];
        unsigned see[2] = {~0u, ~0u};
        bool exact = i == 0 || masked;
        if (live && !exact) {
          // The running maximum seldom rises by more than P may grow: P is made with the old one in one
          // pass, and made again if it did.
          const float mc = m == -CUDART_INF_F ? kUp : fmaf(-m, c, kUp);
          const uint64_t c2 = pair(c, c), mc2 = pair(mc, mc);
          uint64_t sum[2] = {0, 0};
          unsigned r[32];
          float top = -CUDART_INF_F;
#pragma unroll
          for (int x = 0; x < 2; x++) {
            unsigned w[32];
            tmem_ld32(w, ts + half * 64 + x * 32);
            tmem_wait_ld();
            tmem_pin(w);
            float tops[2] = {-CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
            for (int k = 0; k < 32; k += 2) {
              const float a0 = __uint_as_float(w[k]), a1 = __uint_as_float(w[k + 1]);
              tops[k >> 1 & 1] = max3_nan(tops[k >> 1 & 1], a0, a1);
              const uint64_t z = fma2(pair(a0, a1), c2, mc2);
              float e0, e1;
              unpair(e0, e1, z);
              e0 = exp2_fast(e0), e1 = exp2_fast(e1);
              sum[k >> 1 & 1] = add2(sum[k >> 1 & 1], pair(e0, e1));
              r[x * 16 + k / 2] = pack2<FP8>(e0, e1);
            }
            top = max3_nan(top, tops[0], tops[1]);
          }
          // (a NaN among the scores, a first finite one, or a maximum far from zero takes the careful way too)
          exact = any_of_pair(!((top - m) * c <= kRise) || fabsf(mc) > kFarScore, pair_id);
          if (!exact) {
            tmem_st32(ts + half * 64, r);
            float s0, s1;
            unpair(s0, s1, add2(sum[0], sum[1]));
            l += s0 + s1;
          }
        }
        // The careful way: maximum first.  S is read from TMEM twice: that costs less than the registers that would keep
        // it, and spilled registers would travel behind the stream of tiles.
        if (live && exact) {
          if (masked) {
            const volatile Unit& v = h.now[warp];
            const int row = v.row0 + (dual ? 0 : t * kTile) + wr, tok = div_rep(p, row);
#pragma unroll
            for (int w = 0; w < 2; w++) {
              const int first = (dual ? v.tile_end - 1 - 2 * i - t : v.tile_begin + steps - 1 - i) * kTile + half * 64 + 32 * w;
              if (TREE) {
                const int ctx = v.len - first;                      // context keys from `first` on
                if (ctx < 32)
                  see[w] = (ctx > 0 ? (1u << ctx) - 1u : 0u) |
                           tree_bits32(p.mask ? p.mask + mask_at(p, v.seq, tok) : nullptr, h.word0[t][wr], p.rows, tok, -ctx);
              } else {
                const int n = v.tok0 + tok + 1 - first;
                see[w] = n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
              }
            }
          }
          float top = -CUDART_INF_F;
#pragma unroll (TREE ? 1 : 2)
          for (int x = 0; x < 2; x++) {                  // (rolled in short runs: this code is cold there)
            const unsigned sees = x ? see[1] : see[0];
            unsigned w[32];
            tmem_ld32(w, ts + half * 64 + x * 32);
            tmem_wait_ld();
            tmem_pin(w);
            if (masked) {
#pragma unroll
              for (int k = 0; k < 32; k++)
                if (!(sees >> k & 1)) w[k] = 0xff800000u;          // -infinity
            }
            float mx[4];
#pragma unroll
            for (int k = 0; k < 4; k++) mx[k] = fmaxf(__uint_as_float(w[8 * k]), __uint_as_float(w[8 * k + 1]));
#pragma unroll
            for (int j = 2; j < 8; j += 2)
#pragma unroll
              for (int k = 0; k < 4; k++) mx[k] = max3(mx[k], __uint_as_float(w[8 * k + j]), __uint_as_float(w[8 * k + j + 1]));
            top = max3(top, max3(mx[0], mx[1], mx[2]), mx[3]);
          }
          h.mx[t][half][wr] = top;
          named_barrier(pair_id, 64);
          top = fmaxf(top, h.mx[t][half ^ 1][wr]);
          if (i == 0) {
            m = top;
          } else {
            const bool need = top > m && (top - m) * c > kRise;
            if (__any_sync(~0u, need)) {              // the same in both halves
              const float mn = fmaxf(m, top);
              const float f = m == mn ? 1.f : exp2_fast((m - mn) * c);
#pragma unroll 1
              for (int x = half * (HD / 2); x < (half + 1) * (HD / 2); x += 32) {
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
          const float mc0 = m == -CUDART_INF_F ? kUp : fmaf(-m, c, kUp);
          const bool far = fabsf(mc0) > kFarScore;
          const float mc = far ? kUp : mc0, less = far ? -m : 0.f;
          const uint64_t c2 = pair(c, c), mc2 = pair(mc, mc), less2 = pair(less, less);
          uint64_t sum[2] = {0, 0};
#pragma unroll (TREE ? 1 : 2)
          for (int x = 0; x < 2; x++) {
            const unsigned sees = x ? see[1] : see[0];
            unsigned w[32], r[16];
            tmem_ld32(w, ts + half * 64 + x * 32);
            tmem_wait_ld();
            tmem_pin(w);
            if (masked) {
#pragma unroll
              for (int k = 0; k < 32; k++)
                if (!(sees >> k & 1)) w[k] = 0xff800000u;
            }
#pragma unroll
            for (int k = 0; k < 32; k += 2) {
              float e0, e1;
              unpair(e0, e1, fma2(add2(pair(__uint_as_float(w[k]), __uint_as_float(w[k + 1])), less2), c2, mc2));
              e0 = exp2_fast(e0), e1 = exp2_fast(e1);
              sum[k >> 1 & 1] = add2(sum[k >> 1 & 1], pair(e0, e1));
              r[k / 2] = pack2<FP8>(e0, e1);
            }
            tmem_st16(ts + half * 64 + x * 16, r);    // over S columns of its own that it has read
          }
          float s0, s1;
          unpair(s0, s1, add2(sum[0], sum[1]));
          l += s0 + s1;
        }
        unsigned slow = 0;
        if (masked) {
          // What a mask hides must not come through 0 * V either: V rows that no row of the block sees become zero; if
          // a row that some of them see is not finite, this tile's product is made here, key by key.
          const volatile Unit& u = h.now[warp];
          const int tile = dual ? u.tile_end - 1 - 2 * i - t : u.tile_begin + steps - 1 - i, key = tile * kTile;
          const int key_end = TREE ? u.len + p.rows : u.tok0 + u.n_tok;      // keys nobody here sees: from it on
          const int pos = ring + 2 * (u.tile_end - 1 - tile) + 1, st = pos % L::kStages;
          attn_wait(&h.full[st], pos / L::kStages & 1, h);
          unsigned char* vt = smem + L::kRing + st * L::kTileBytes;
          const int r = id & 127;
          unsigned broken = 0;                         // becomes NaN (two bf16)
#pragma unroll
          for (int j = 0; j < HD / 16; j++) {
            const int ch = (id >> 7) * (HD / 16) + j;
            uint4* at = (uint4*)(vt + ch / 8 * kBox + r * 128 + (((ch & 7) ^ (r & 7)) << 4));
            if (key + r >= key_end) {
              *at = make_uint4(0, 0, 0, 0);
            } else {
              const uint4 v = *at;
              broken = zero_times<FP8>(v.w, zero_times<FP8>(v.z, zero_times<FP8>(v.y, zero_times<FP8>(v.x, broken))));
            }
          }
          fence_async_smem();
          slow = any_of_tile((broken & 0x7fff7fffu) != 0, tile_id);
          if (slow && live) {
            tmem_wait_st();
            if (half == 0) product_by_key<HD, FP8>(ts, see[0], see[1], vt, 0, to, i > 0);
            tc_fence_before();
            named_barrier(pair_id, 64);
            tc_fence_after();
            if (half == 1) product_by_key<HD, FP8>(ts + 64, see[0], see[1], vt, 64, to, true);
          }
        }
        tmem_wait_st();
        tc_fence_before();
        if (masked && id == 0) h.skip[t] = slow;
        warp_arrive(&h.p_full[t], lane);
      }
      {
        const volatile Unit& v = h.now[warp];
        u.seq = v.seq, u.head = v.head, u.row0 = v.row0, u.n_rows = v.n_rows, u.key0 = v.key0, u.tok0 = v.tok0;
        u.tile_begin = v.tile_begin, u.tile_end = v.tile_end, u.item_tiles = v.item_tiles;
      }
      ring += 2 * (u.tile_end - u.tile_begin);
      if (steps) {
        attn_wait(&h.o_done[t], o_phase & 1, h);
        o_phase++;
        __syncwarp();
        tc_fence_after();
        if (live) {                                    // the row's sum: both halves'
          h.mx[t][half][wr] = l;
          named_barrier(pair_id, 64);
          l += h.mx[t][half ^ 1][wr];
          named_barrier(pair_id, 64);                  // (the next unit writes there)
        }
      }

      // O / l, or this block's part of it
      const int first_row = u.row0 + (dual ? 0 : t * kTile), n_here = dual ? u.n_rows : u.n_rows - t * kTile;
      const int row = first_row + wr, tok = div_rep(p, row), hh = row - tok * p.rep;
      const bool valid = wr < n_here;
      float f0 = 1.f, f1 = 0.f;
      bool two = false;
      if (dual) {
        if (t == 1) {
          if (half == 0) h.m[wr] = m, h.l[wr] = l;
          tc_fence_before();
        }
        named_barrier(11, 512);
        if (t == 0) {
          tc_fence_after();
          two = u.tile_end - u.tile_begin > 1;
          const float m1 = h.m[wr], l1 = h.l[wr];
          const float mn = fmaxf(m, m1);
          if (two && mn != -CUDART_INF_F) {
            f0 = m == mn ? 1.f : exp2_fast((m - mn) * c);
            f1 = m1 == mn ? 1.f : exp2_fast((m1 - mn) * c);
            l = l * f0 + l1 * f1;
            m = mn;
          }
        }
      }
      if (steps && live && !(dual && t == 1)) {
        const bool whole = !TREE || (u.tile_begin == 0 && u.tile_end == u.item_tiles);
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int64_t slot = TREE ? (int64_t)2 * blockIdx.x + (u.tile_begin == 0 ? 1 : 0) : 0;
        const int part_row = wr + (dual ? 0 : t * kTile);
        if (valid && half == 0) {                      // (before the output: two registers less are held there)
          // A part leaves its maximum, in units of q k, and its sum: their log2 as one number would lose the sum beside a
          // large maximum.
          const float part_m = FP8 ? m * (c / (p.scale * kLog2e)) : m, part_l = l * (FP8 ? 1.f / (1 << (int)kUp) : 1.f);
          if (TREE && !whole && p.cluster) {
            h.mx[0][0][wr] = part_m, h.mx[0][1][wr] = part_l;
          } else if (!whole) {
            float* part = p.part_lse + slot * 2 * p.part_rows + part_row;
            part[0] = part_m, part[p.part_rows] = part_l;
          } else if (p.lse) {
            const int64_t gtok = TREE ? (int64_t)u.seq * p.rows + tok : (int64_t)u.key0 + u.tok0 + tok;
            const float lse2 = l == 0.f ? -CUDART_INF_F : m * c + (log2f(l) - kUp);
            p.lse[gtok * p.nq + u.head * p.rep + hh] = lse2 * 0.6931471805599453f;
          }
        }
        __syncwarp();
#pragma unroll 1
        for (int x = half * (HD / 2); x < (half + 1) * (HD / 2); x += 16) {
          unsigned o[16], o1[16];
          float v[16];
          tmem_ld16(o, to + x);
          if (two) tmem_ld16(o1, to + HD + x);
          tmem_wait_ld();
          tmem_pin(o);
          if (two) tmem_pin(o1);
#pragma unroll
          for (int k = 0; k < 16; k++) {
            v[k] = __uint_as_float(o[k]) * f0;
            if (two) v[k] += __uint_as_float(o1[k]) * f1;
            v[k] = inv == 0.f ? 0.f : v[k] * inv;      // (nothing seen)
          }
          if (whole) {
            // over the tile's Q, 16-byte chunks permuted within a row so that neither side meets a bank twice
#pragma unroll
            for (int k = 0; k < 16; k += 8)
              *(uint4*)(qs + wr * (HD * 2) + (((x + k) / 8 ^ (wr & 7)) << 4)) =
                  make_uint4(pack_bf16(v[k], v[k + 1]), pack_bf16(v[k + 2], v[k + 3]), pack_bf16(v[k + 4], v[k + 5]),
                             pack_bf16(v[k + 6], v[k + 7]));
          } else if (TREE && p.cluster) {
            // over the ring, whose products are done: a row's 16-byte chunks permuted as above
#pragma unroll
            for (int k = 0; k < 16; k += 4)
              *(float4*)(smem + L::kRing + wr * (HD * 4) + (((x + k) / 4 ^ (wr & 7)) << 4)) =
                  make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
          } else if (valid) {
            // [slot][column / 4][row][4]: a warp's rows lie side by side
            float* part = p.part_o + ((slot * (HD / 4) + x / 4) * p.part_rows + part_row) * 4;
#pragma unroll
            for (int k = 0; k < 16; k += 4) *(float4*)(part + (int64_t)k * p.part_rows) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
          }
        }
        if (whole) {
          named_barrier(pair_id, 64);
          constexpr int kChunks = HD / 8;
          __nv_bfloat16* out = p.out + (int64_t)u.seq * p.o_seq + (int64_t)(u.key0 + u.tok0) * p.o_row +
                               (int64_t)u.head * p.rep * p.o_head;
#pragma unroll
          for (int i = 0; i < 32 * kChunks / 64; i++) {
            const int e = i * 64 + half * 32 + lane, r = quarter * 32 + e / kChunks, ch = e % kChunks;
            if (r < n_here) {
              const int row = first_row + r, tok = div_rep(p, row), hh = row - tok * p.rep;
              *(uint4*)(out + tok * p.o_row + hh * p.o_head + ch * 8) =
                  *(const uint4*)(qs + r * (HD * 2) + ((ch ^ (r & 7)) << 4));
            }
          }
        }
      }
      if (dual) {
        tc_fence_before();
        named_barrier(11, 512);      // the second tile's O and statistics have been read
        tc_fence_after();
      }
    }
  } else if (warp == kProducer) {
    // ================================ K and V tiles into the ring ======================================================
    constexpr int kN = FP8 ? L::kRawStages : L::kStages;
    uint64_t* full = FP8 ? h.raw_full : h.full;
    uint64_t* empty = FP8 ? h.raw_empty : h.empty;
    const bool leader = elect_one();
    unsigned issued = 0;
    bool on = true, gate = TREE;                      // (gate: within the first unit)
    unsigned taken = 1, asked = 0, told = 0;          // prompts: units put into the ring, questions to the scheduler, answers
    // The next block's unit.  The grid has as many blocks as the prompts can need: those that find no queries are taken over
    // as well, since one that is launched looks through all prompts first (20000 prompts of 10 tokens: 49 ms so, 2.5 ms now).
    auto next_unit = [&]() {
      int4 x = make_int4(-1, 0, 0, 0);
      while (on && x.x < 0) {
        expect_tx(leader, &h.next_full, 16);
        ask_for_block(leader, &h.next, &h.next_full);
        on = attn_wait(&h.next_full, asked++ & 1, h);
        if (!on) break;
        told++;
        const int block = uniform(block_of_answer(&h.next));
        fence_async_smem();                           // (read before the next answer is written there)
        if (block < 0) break;
        x = blocks.find(p, block, lane);
      }
      return x;
    };
    if (!TREE && unit.x < 0) {
      // This block's index stands for no queries.  In which order blocks are launched and taken over is not specified: what
      // the scheduler hands out instead is worked on like any unit, and the end is the answer that nothing is left.
      unit = next_unit();
      if (lane == 0) {
        h.units[0] = unit;
        mbar_arrive(&h.unit_full[0]);
      }
      __syncwarp();
    }
    for (;;) {
      if constexpr (TREE) {
        if (!uniform(units.next(p, h, u))) break;
      } else if (!Units<false>::set(p, unit, u)) {
        break;
      }
      const int tile_begin = uniform(u.tile_begin);
      for (int j = uniform(u.tile_end) - 1; j >= tile_begin; j--) {
        for (int kv = 0; kv < 2; kv++) {
          const int st = issued % kN;
          if (gate && issued == 2) {   // the first Q is not to queue behind the whole ring
            gate = false;
            for (int t = 0; t < 2; t++)
              if (unit_steps<TREE>(p, u, dual, t)) attn_wait(&h.q_full[t], 0, h);
          }
          on = on && issued != p.tiles && attn_wait(&empty[st], (issued / kN & 1) ^ 1, h);
          if (!on) continue;
          const CUtensorMap* map = kv ? &map_v : &map_k;
          const int y = uniform(u.key0) + j * kTile, z = uniform(u.head), w = uniform(u.seq);
          if (FP8) {
            expect_tx(leader, &full[st], L::kRawBytes);
            tma_load_4d(leader, smem + L::kRaw + st * L::kRawBytes, map, 0, y, z, w, &full[st]);
          } else {
            unsigned char* dst = smem + L::kRing + st * L::kTileBytes;
            expect_tx(leader, &full[st], L::kTileBytes);
#pragma unroll
            for (int x = 0; x < HD / 64; x++) tma_load_4d(leader, dst + x * kBox, map, x * 64, y, z, w, &full[st]);
          }
          issued++;
        }
      }
      gate = false;
      if constexpr (!TREE) {
        unit = next_unit();
        if (!on) break;
        const int at = taken & (kUnitRing - 1);
        if (!attn_wait(&h.unit_empty[at], (taken / kUnitRing & 1) ^ 1, h)) break;
        if (lane == 0) {
          h.units[at] = unit;
          mbar_arrive(&h.unit_full[at]);
        }
        __syncwarp();
        taken++;
        // its Q into L2
        const unsigned short* q = p.q + (int64_t)(unit.y + unit.z) * p.q_row + (int64_t)unit.x * p.rep * p.q_head;
        for (int r = lane; r < unit.w * p.rep; r += 32) {
          const int tok = div_rep(p, r);
          const unsigned short* row = q + tok * p.q_row + (r - tok * p.rep) * p.q_head;
          for (int x = 0; x < HD; x += 64) asm volatile("prefetch.global.L2 [%0];" ::"l"(row + x));
        }
      }
    }
    if (lane == 0) h.unit[5] = (int)issued, h.unit[6] = (int)asked, h.unit[7] = (int)told;
  } else if (warp == kIssuer) {
    // ================================ the matrix products ==============================================================
    // The whole warp walks the steps, so that addresses and phases stay warp-uniform; one lane issues.
    const bool leader = elect_one();
    constexpr unsigned kIdS = mma_idesc(kTile, kTile, false, FP8), kIdO = mma_idesc(kTile, HD, true, FP8);
    const uint64_t q_desc = smem_desc(smem_u32(smem + L::kQ), 16, 1024);
    const uint64_t k_desc = smem_desc(smem_u32(smem + L::kRing), 16, 1024);
    const uint64_t v_desc = smem_desc(smem_u32(smem + L::kRing), kBox, 1024);
    constexpr uint64_t kTileStep = L::kTileBytes >> 4;          // descriptors count in 16 bytes
    unsigned q_phase[2] = {0, 0}, p_phase[2] = {0, 0};
    int ring = 0;
    bool on = true;
    while (uniform(units.next(p, h, u))) {
      const int n0 = uniform(unit_steps<TREE>(p, u, dual, 0)), n1 = uniform(unit_steps<TREE>(p, u, dual, 1));
      const int most = max(n0, n1), tile_end = uniform(u.tile_end);
      const int skip[2] = {dual || !n0 ? 0 : most - n0, 0};     // the first key tiles that row tile 0 has no part in
      int all_see[2];                                           // first key that a row of tile t may not see
#pragma unroll
      for (int t = 0; t < 2; t++) all_see[t] = uniform(TREE ? u.len : u.tok0 + div_rep(p, u.row0 + t * kTile) + 1);
      auto scores = [&](int t, int i) {
        const int pos = ring + 2 * (dual ? 2 * i + t : i), st = pos % L::kStages;
        on = attn_wait(&h.full[st], pos / L::kStages & 1, h) && on;
        if (!on) return;
        tc_fence_after();
        const uint64_t qa = q_desc + t * kTileStep, ka = k_desc + st * kTileStep;
#pragma unroll
        for (int k = 0; k < HD / 16; k++) {
          const int off = (k / 4 * kBox + k % 4 * 32) >> 4;
          mma_ss(leader, tmem + t * kTile, qa + off, ka + off, kIdS, k > 0);
        }
        mma_commit(leader, &h.s_full[t]);
        if (dual || t == 1 || n1 == 0) mma_commit(leader, &h.empty[st]);
      };
      for (int i = -1; i < most; i++) {
#pragma unroll
        for (int t = 0; t < 2; t++) {
          const int end = (t ? n1 : n0) + skip[t], from = skip[t];
          if (i >= end || from == end) continue;
          if (i >= from) {
            const int rel = dual ? 2 * i + t : i, pos = ring + 2 * rel + 1, st = pos % L::kStages;
            const bool masked = (tile_end - rel) * kTile > all_see[t];
            on = attn_wait(&h.full[st], pos / L::kStages & 1, h) && on;
            on = attn_wait(&h.p_full[t], p_phase[t]++ & 1, h) && on;
            if (on) {
              tc_fence_after();
              if (!masked || !uniform(*(volatile int*)&h.skip[t])) {
                const uint64_t va = v_desc + st * kTileStep;
#pragma unroll
                for (int k = 0; k < kTile / 16; k++)
                  mma_ts(leader, tmem + 2 * kTile + t * HD, tmem + t * kTile + k / 4 * 64 + k % 4 * 8, va + k * 128, kIdO,
                         i > from || k > 0);
              }
              if (i + 1 == end) mma_commit(leader, &h.o_done[t]);
              if (dual || t == 1 || n1 == 0) mma_commit(leader, &h.empty[st]);
            }
          }
          if (i + 1 == from) on = attn_wait(&h.q_full[t], q_phase[t]++ & 1, h) && on;
          if (i + 1 >= from && i + 1 < end) scores(t, i + 1);
        }
      }
      ring += uniform(2 * (u.tile_end - u.tile_begin));
    }
  } else if (FP8) {
    // ================================ 8-bit tiles widened to f16: six warps ============================================
    const int ct = (warp < 20 ? warp - 16 : warp - 18) * 32 + lane;
    constexpr int kChunks = HD / 16, kAll = kChunks * kTile;   // 16-byte chunks of an 8-bit row, of a tile
    // where this thread's first chunk goes: two of an f16 row
    const int row0 = ct / kChunks, cc0 = ct % kChunks * 2;
    const int at0 = cc0 / 8 * kBox + row0 * 128 + (((cc0 & 7) ^ (row0 & 7)) << 4);
    const int at1 = cc0 / 8 * kBox + row0 * 128 + ((((cc0 & 7) + 1) ^ (row0 & 7)) << 4);
    int pos = 0;
    while (units.next(p, h, u)) {
      for (int n = 2 * (u.tile_end - u.tile_begin); n; n--, pos++) {
        const int raw = pos % (FP8 ? L::kRawStages : 1), st = pos % L::kStages;
        attn_wait(&h.raw_full[raw], pos / (FP8 ? L::kRawStages : 1) & 1, h);
        attn_wait(&h.empty[st], (pos / L::kStages & 1) ^ 1, h);
        const unsigned char* src = smem + L::kRaw + raw * L::kRawBytes;
        unsigned char* dst = smem + L::kRing + st * L::kTileBytes;
        // 192 chunks are a whole number of rows, a multiple of 8: only the row moves on from one to the next
#pragma unroll 2
        for (int i = 0; i < kAll - ct; i += 192) {
          const uint4 v = *(const uint4*)(src + (ct + i) * 16);
          unsigned w[8];
          widen_e4m3(w, v.x), widen_e4m3(w + 2, v.y), widen_e4m3(w + 4, v.z), widen_e4m3(w + 6, v.w);
          *(uint4*)(dst + at0 + i * (128 / kChunks)) = make_uint4(w[0], w[1], w[2], w[3]);
          *(uint4*)(dst + at1 + i * (128 / kChunks)) = make_uint4(w[4], w[5], w[6], w[7]);
        }
        fence_async_smem();
        warp_arrive(&h.full[st], lane);
        warp_arrive(&h.raw_empty[raw], lane);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  end_in_flight<HD, FP8>();
  if (warp == kIssuer) tmem_free(tmem, 512);
  if (TREE && p.cluster) {
    // the item's parts joined in the cluster: each block takes some of the rows and reads the others' parts of them
    if (p.cluster > 1) cluster_sync();
    if (warp < 16) {
      const int item = blockIdx.x / p.cluster, rank = blockIdx.x - item * p.cluster, seq = item / p.nkv;
      const int tiles = tree_tiles(p, h.unit[3]), per = (tiles + p.cluster - 1) / p.cluster;
      const int parts = tiles ? (tiles + per - 1) / per : 0;      // 1: complete already
      const int all = p.rows * p.rep, each = (all + p.cluster - 1) / p.cluster, last = min(all, (rank + 1) * each);
      constexpr int kChunks = HD / 4;
      if (parts != 1)
        for (int e = threadIdx.x + rank * each * kChunks; e < last * kChunks; e += 512) {
          const int row = e / kChunks, ch = e % kChunks;
          const unsigned char* o_at = smem + L::kRing + row * (HD * 4) + ((ch ^ (row & 7)) << 4);
          const float c = p.scale * kLog2e;
          float m = -CUDART_INF_F, sum = 0.f, v[4] = {};
          constexpr int kBatch = 4;                       // parts' loads under way
          for (int b0 = 0; b0 < parts; b0 += kBatch) {
            float x[kBatch], w[kBatch];
            float4 y[kBatch];
#pragma unroll
            for (int b = 0; b < kBatch; b++) {
              const int from = min(b0 + b, parts - 1);
              x[b] = remote_f32(&h.mx[0][0][row], from), w[b] = remote_f32(&h.mx[0][1][row], from), y[b] = remote_f32x4(o_at, from);
              if (b0 + b >= parts) x[b] = -CUDART_INF_F;
            }
            float mn = m;
#pragma unroll
            for (int b = 0; b < kBatch; b++) mn = fmaxf(mn, x[b]);
            const float f = m == mn ? 1.f : exp2f((m - mn) * c);
            m = mn;
            sum *= f;
#pragma unroll
            for (int k = 0; k < 4; k++) v[k] *= f;
#pragma unroll
            for (int b = 0; b < kBatch; b++) {
              w[b] = x[b] == -CUDART_INF_F ? 0.f : w[b] * exp2f((x[b] - m) * c);         // (nothing seen: 0)
              sum += w[b];
              v[0] += w[b] * y[b].x, v[1] += w[b] * y[b].y, v[2] += w[b] * y[b].z, v[3] += w[b] * y[b].w;
            }
          }
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
          for (int k = 0; k < 4; k++) v[k] = parts ? v[k] * inv : CUDART_NAN_F;
          const int tok = div_rep(p, row), head = (item - seq * p.nkv) * p.rep + row - tok * p.rep;
          *(uint2*)(p.out + (int64_t)seq * p.o_seq + tok * p.o_row + head * p.o_head + ch * 4) =
              make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
          if (p.lse && ch == 0)
            p.lse[((int64_t)seq * p.rows + tok) * p.nq + head] =
                !parts ? CUDART_NAN_F : sum == 0.f ? -CUDART_INF_F : (m * c + log2f(sum)) * 0.6931471805599453f;
        }
    }
    __syncwarp();
    if (p.cluster > 1) cluster_sync();                            // nobody leaves while its parts are read
  }
}

// ---- parts of one item joined (tree) ----------------------------------------------------------------------------
// Items whose tiles one block had are complete already; sequences of a bad length become NaN.
//   O = sum_i w_i O_i / sum_i w_i,  w_i = l_i 2^((m_i - max m) c): the parts carry O_i / l_i, m_i and l_i.
// A block takes 32 rows and 8 columns of one item, a lane one row; the warps share the parts out, so that one way to
// memory and back serves all of them, and meet in shared memory.
constexpr int kJoinWarps = 8;
template <int HD>
__global__ void __launch_bounds__(32 * kJoinWarps) attn_join_kernel(const AttnParams p, int blocks) {
  __shared__ int sh[2];
  __shared__ float some[kJoinWarps][10][32];          // each warp's columns, maximum and sum
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  constexpr int kSlices = HD / 8;
  const int head = blockIdx.y, seq = blockIdx.z, row0 = blockIdx.x / kSlices * 32, row = row0 + lane, col = blockIdx.x % kSlices * 8;
  const int tiles = tree_tiles(p, __ldg(p.lens + seq));
  if (warp == 0) {
    const int mine = tree_slots_of(p, lane);
    const int per = tree_run(p, mine, lane, blocks);
    int before = lane < seq ? mine : 0;
    for (int b = 32 + lane; b < seq; b += 32) before += tree_slots_of(p, b);
    before = warp_sum(before);
    if (lane == 0) sh[0] = before, sh[1] = per;
  }
  __syncthreads();
  const int rt = row0 / p.part_rows, local = row - rt * p.part_rows;
  const int first = sh[0] + (head * p.row_tiles + rt) * tree_slots(tiles) + kUnitCost, per = sh[1];
  const int c0 = first / per, parts = tiles ? (first + tiles - 1) / per - c0 + 1 : 0;
  // every thread waits for the attention kernel, also one that has nothing to do: what follows in the stream waits for
  // this grid alone
  wait_for_grid_before();
  if (parts == 1) return;                            // complete already
  const bool valid = row < p.rows * p.rep;
  const float c = p.scale * kLog2e;
  float m = -CUDART_INF_F, sum = 0.f, v[8] = {};
  if (valid) {
#pragma unroll 4
    for (int b = warp; b < parts; b += warps) {      // part b is slot 2 (c0 + b), the first one's the slot behind
      const int64_t slot = (int64_t)2 * (c0 + b) + (b == 0 ? 1 : 0);
      const float* at = p.part_lse + slot * 2 * p.part_rows + local;
      const float x = at[0], l = at[p.part_rows];
      const float* o = p.part_o + ((slot * (HD / 4) + col / 4) * p.part_rows + local) * 4;
      const float4 y = *(const float4*)o, z = *(const float4*)(o + (int64_t)4 * p.part_rows);
      const float mn = fmaxf(m, x);
      const float f = m == mn ? 1.f : exp2f((m - mn) * c), w = x == -CUDART_INF_F ? 0.f : l * exp2f((x - mn) * c);
      m = mn;
      sum = sum * f + w;
      v[0] = v[0] * f + w * y.x, v[1] = v[1] * f + w * y.y, v[2] = v[2] * f + w * y.z, v[3] = v[3] * f + w * y.w;
      v[4] = v[4] * f + w * z.x, v[5] = v[5] * f + w * z.y, v[6] = v[6] * f + w * z.z, v[7] = v[7] * f + w * z.w;
    }
  }
  some[warp][8][lane] = m, some[warp][9][lane] = sum;
#pragma unroll
  for (int k = 0; k < 8; k++) some[warp][k][lane] = v[k];
  __syncthreads();
  if (warp || !valid) return;
  for (int g = 1; g < warps; g++) {
    const float x = some[g][8][lane];
    const float mn = fmaxf(m, x);
    const float f = m == mn ? 1.f : exp2f((m - mn) * c), w = x == -CUDART_INF_F ? 0.f : exp2f((x - mn) * c);   // (nothing seen: 0)
    m = mn;
    sum = sum * f + w * some[g][9][lane];
#pragma unroll
    for (int k = 0; k < 8; k++) v[k] = v[k] * f + w * some[g][k][lane];
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int k = 0; k < 8; k++) v[k] = parts ? v[k] * inv : CUDART_NAN_F;
  const float lse = !parts ? CUDART_NAN_F : sum == 0.f ? -CUDART_INF_F : (m * c + log2f(sum)) * 0.6931471805599453f;
  const int tok = div_rep(p, row), q_head = head * p.rep + row - tok * p.rep;
  *(uint4*)(p.out + (int64_t)seq * p.o_seq + tok * p.o_row + q_head * p.o_head + col) =
      make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  if (p.lse && col == 0) p.lse[((int64_t)seq * p.rows + tok) * p.nq + q_head] = lse;
}

}  // namespace amk
