// How the work of amk_attention_weights is divided: integer arithmetic alone, for the kernels and for a check on the host.
//
// A unit is SPAN positions of a kv head, a step of it the product with one tile of query rows (as many whole tokens as fit into 128
// rows).  The steps of all units, sequence by sequence, head by head, are cut into equal runs, one for each block.  SPAN 128: few rows,
// one tile of them.
#pragma once
#ifndef AMK_HD
#if defined(__CUDACC__)
#define AMK_HD __host__ __device__ __forceinline__
#else
#define AMK_HD inline
#endif
#endif

namespace amk {

constexpr int kFewSpan = 128, kManySpan = 160;

struct WeightsWork {
  const int* lens;
  int n_seqs, nkv, rows, slots;
  int tokens, q_tiles;             // tokens of a tile of query rows, tiles of all
};
AMK_HD int weights_len(const WeightsWork& p, int seq) {
#if defined(__CUDA_ARCH__)
  return __ldg(p.lens + seq);
#else
  return p.lens[seq];
#endif
}

template <int SPAN>
AMK_HD int weights_units(const WeightsWork& p, int len) {              // of one head; 0: impossible length
  return len < 0 || len > p.slots - p.rows ? 0 : (len + p.rows + SPAN - 1) / SPAN;
}
// the first tile of query rows that sees a position of a unit
template <int SPAN>
AMK_HD int first_q_tile(const WeightsWork& p, int len, int unit) {
  const int behind = unit * SPAN - len;
  return SPAN == kFewSpan || behind <= 0 ? 0 : behind / p.tokens;
}
// units of one head whose every position all rows see (0 of 0: an impossible length may be any number)
template <int SPAN>
AMK_HD int full_units(const WeightsWork& p, int len, int units) {
  return SPAN == kFewSpan || units == 0 || units < len / SPAN + 1 ? units : len / SPAN + 1;
}
template <int SPAN>
AMK_HD int weights_steps(const WeightsWork& p, int len) {              // of one head
  const int units = weights_units<SPAN>(p, len), full = full_units<SPAN>(p, len, units);
  int n = full * p.q_tiles;
  for (int j = full; j < units; j++) n += p.q_tiles - first_q_tile<SPAN>(p, len, j);
  return n;
}
// the unit and its step that step `rel` of a head is
template <int SPAN>
AMK_HD void weights_place(const WeightsWork& p, int len, int rel, int& unit, int& step) {
  step = 0, unit = rel;
  if (SPAN == kFewSpan) return;
  const int full = full_units<SPAN>(p, len, weights_units<SPAN>(p, len));
  if (rel < full * p.q_tiles) {
    unit = rel / p.q_tiles, step = rel - unit * p.q_tiles;
    return;
  }
  rel -= full * p.q_tiles;
  for (unit = full;; unit++) {
    const int steps = p.q_tiles - first_q_tile<SPAN>(p, len, unit);
    if (rel < steps) break;
    rel -= steps;
  }
  step = rel;
}

struct WeightsUnit {
  int seq, head, len, at;          // at: which unit of the head
  int first;                       // first tile of query rows of the unit
  int begin, end, all;             // steps of this block, steps of the unit
};
// A block's run; start: {sequence, head, unit, step, steps, length of the sequence}
template <int SPAN>
struct WeightsWalk {
  int left, seq, len, head, at, units, step;
  AMK_HD void init(const WeightsWork& p, const int* start) {
    seq = start[0], head = start[1], at = start[2], step = start[3], left = start[4], len = start[5];
    units = weights_units<SPAN>(p, len);
  }
  AMK_HD bool next(const WeightsWork& p, WeightsUnit& u) {
    if (left <= 0) return false;
    while (at >= units) {          // something is left: a unit follows
      at = 0;
      if (units && head + 1 < p.nkv) {
        head++;
      } else {
        head = 0;
        len = weights_len(p, ++seq);
        units = weights_units<SPAN>(p, len);
      }
    }
    u.seq = seq, u.head = head, u.len = len, u.at = at;
    u.first = first_q_tile<SPAN>(p, len, at);
    u.all = SPAN == kFewSpan ? 1 : p.q_tiles - u.first;
    u.begin = step, u.end = u.all < step + left ? u.all : step + left;
    left -= u.end - u.begin;
    step = 0;
    at++;
    return true;
  }
};

}  // namespace amk
