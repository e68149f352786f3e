// How the attention over a paged cache (kv_attention.cu, kv_attention_tc.cu) divides a call among its
// CTAs, computed by each CTA from the batch's device arrays: no list is built on the host, so a call needs
// no copy, no synchronisation and can be captured in a graph while the lengths change.
//
// A unit is (sequence, key / value head, tile of its new tokens); its work is its key blocks.  The units lie
// one after another on a line, each as long as its cost (its blocks' and a constant for its ends), and the line is
// cut into G equal parts, one a CTA: equal work whatever the lengths are.  A unit that lies
// in several CTAs' ranges is computed in parts, which the CTA that finishes last joins in their order, so
// the result does not depend on which CTA that is.
#pragma once
#include "../../include/flglm_kernels.h"
#include "common.cuh"

struct KvBatchDev {
  const int32_t *cu, *lens, *table, *ctx;
  int S, T, table_stride, ps_log2, n_pages;
  int* status;
};

struct KvSeq {
  int q0, n, L, ctx;  // first row of the new tokens, their number, tokens in the cache, context length
};
// The arrays' values are brought into their ranges, so that no index leaves a buffer; a length outside is recorded.
FL_DEV KvSeq kv_seq(const KvBatchDev& b, int s) {
  KvSeq q;
  const int a = min(max(b.cu[s], 0), b.T), e = min(max(b.cu[s + 1], 0), b.T);
  const int64_t cap = (int64_t)b.table_stride << b.ps_log2;
  q.q0 = a;
  q.n = max(e - a, 0);
  const int len = b.lens[s];
  q.L = (int)min((int64_t)max(len, 0), cap);
  if (q.L != len) atomicOr(b.status, FL_KV_BAD_PAGE);
  q.ctx = b.ctx ? b.ctx[s] : 0;
  return q;
}
// Number of keys that new token i sees (they are the first ones): its own and those before it, the
// context's if it is shorter; none if the token lies before the cache's first one.
FL_DEV int kv_sees(const KvSeq& q, int i) { return max(0, min(q.L, max(q.L - q.n + i + 1, q.ctx))); }

// The page of block-table entry i of sequence s, or -1 (recorded) where the table holds no page of the cache.
FL_DEV int kv_page(const KvBatchDev& b, int s, int i) {
  const int p = __ldg(b.table + (int64_t)s * b.table_stride + i);
  if ((unsigned)p < (unsigned)b.n_pages) return p;
  atomicOr(b.status, FL_KV_BAD_PAGE);
  return -1;
}

// x / d in 32 bits where both fit (x >= 0, d > 0); the 64-bit division is a long way on this path.
FL_DEV int64_t kv_div(int64_t x, int64_t d) {
  return ((x | d) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)d) : x / d;
}

// Units of a sequence: U::units(q) tiles, U::cost(q, r) of tile r, for each of the kv heads.
template <class U>
struct KvWalk {
  int s, h, r;         // the current unit
  KvSeq q;
  int64_t start;       // its place on the line
  int units, cost;

  FL_DEV void set(const KvBatchDev& b, const U& u, int s_, int64_t seq_start, int64_t at, int kvh) {
    s = s_;
    q = kv_seq(b, s);
    units = u.units(q);
    int64_t head = 0;
    for (int i = 0; i < units; ++i) head += u.cost(q, i);
    h = (int)kv_div(at - seq_start, head);
    start = seq_start + h * head;
    r = 0;
    cost = u.cost(q, 0);
    while (r + 1 < units && start + cost <= at) {
      start += cost;
      cost = u.cost(q, ++r);
    }
  }
  FL_DEV bool next(const KvBatchDev& b, const U& u, int kvh) {  // false behind the last unit
    start += cost;
    if (++r == units) {
      r = 0;
      if (++h == kvh) {
        h = 0;
        do {
          if (++s >= b.S) return false;
          q = kv_seq(b, s);
        } while (q.n == 0);
        units = u.units(q);
      }
    }
    cost = u.cost(q, r);
    return true;
  }
};

// CTA i has [i q + min(i, r), (i + 1) q + min(i + 1, r)) with W = q G + r.
struct KvRange {
  int64_t lo, hi, q;
  int G, r;            // CTAs with work
  int s;               // sequence that holds lo, and where it starts
  int64_t seq_start;
  FL_DEV int cta_of(int64_t x) const {  // whose range holds x
    const int64_t longer = r * (q + 1);
    return (int)(x < longer ? kv_div(x, q + 1) : r + kv_div(x - longer, q));
  }
  FL_DEV int64_t lo_of(int i) const { return i * q + min(i, r); }
};

// CTA `cta`'s range, by a whole warp (each that needs it computes it: the arrays are short, a barrier is not).  At most
// `ctas` CTAs get work, and each that does at least about min_cost.
template <class U>
FL_DEV KvRange kv_plan(const KvBatchDev& b, const U& u, int kvh, int cta, int ctas, int min_cost) {
  const int lane = threadIdx.x & 31, per = (b.S + 31) / 32;
  const int s0 = lane * per, s1 = min(b.S, s0 + per);
  auto seq_cost = [&](int s) {
    const KvSeq q = kv_seq(b, s);
    int64_t c = 0;
    if (q.n > 0)
      for (int r = 0, n = u.units(q); r < n; ++r) c += u.cost(q, r);
    return c * kvh;
  };
  int64_t mine = 0, one = 0;
  for (int s = s0; s < s1; ++s) mine += one = seq_cost(s);
  int64_t incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t x = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += x;
  }
  const int64_t W = __shfl_sync(0xffffffffu, incl, 31);
  KvRange g;
  g.G = (int)max((int64_t)1, min((int64_t)ctas, kv_div(W, min_cost)));
  g.q = kv_div(W, g.G);
  g.r = (int)(W - g.q * g.G);
  g.lo = g.hi = 0;
  g.s = -1;
  g.seq_start = 0;
  if (W == 0 || cta >= g.G) return g;
  g.lo = g.lo_of(cta);
  g.hi = g.lo_of(cta + 1);
  int64_t at = incl - mine;
  const bool here = g.lo >= at && g.lo < incl;
  int s = s0;
  if (here && per > 1)
    for (one = seq_cost(s); g.lo >= at + one; one = seq_cost(++s)) at += one;
  const int from = __ffs(__ballot_sync(0xffffffffu, here)) - 1;
  g.s = __shfl_sync(0xffffffffu, s, from);
  g.seq_start = __shfl_sync(0xffffffffu, at, from);
  return g;
}

// Checks of a cache and a batch that the calls share (kv_cache.cu); fills *out but for ctx and status.
int fl_kv_check(const char* who, const fl_kv_cache* c, const fl_kv_batch* b, int n_heads, KvBatchDev* out);
