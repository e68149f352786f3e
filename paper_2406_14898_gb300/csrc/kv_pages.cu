// Sequences that share the pages of a cache: fork (continue, share, copy on write, extend, shorten, leave) and compact.
//
// A call is two launches, 6 to 7 us together where there is little to copy.  The plan is integer work on a few arrays:
// who has each page after the call, which are free, who gets which; it is bound by latency, loads one behind another and
// barriers.  One CTA does it with its counts in shared memory, or one cluster where the arrays are long, with its counts
// in global memory.  The second launch, over the whole GPU, writes the table and copies the pages' tokens in every
// cache.
#include "../../include/flglm_kernels.h"
#include "kv_plan.cuh"
#include "ptx.cuh"

namespace {

constexpr int PLAN_THREADS = 1024, MAX_PLAN_CTAS = 8;
constexpr int COPY_WARPS = 4, COPY_THREADS = 32 * COPY_WARPS, COPY_CTAS = 2;  // a CTA, CTAs of an SM
constexpr int STAGES = 3, BLOCK_BYTES = 8192;  // of a warp: blocks on their way through shared memory
constexpr int COPY_SMEM = COPY_WARPS * STAGES * BLOCK_BYTES;
constexpr int UNIT_BYTES = 16384;              // of a whole page that a warp copies at a time

struct PagesDev {
  const int32_t *lens, *table, *refs;
  int32_t *lens_to, *table_to, *refs_to;
  int S, n_pages, ps_log2, W;
};

// A workspace: what the plan tells the second launch, and the cluster's counts of each page, which are zero between calls.
struct Ws {
  int32_t* head;                      // copies, refused
  int32_t *delta, *writers, *lowest;  // zero between calls: holders more or less, sequences about to write, S - the first
  int4* rows;                         // of each sequence: parent, pages shared with it, place of its first new page, pages
  int32_t* first;                     // of each sequence: its first new page's place in `list`
  int32_t* list;                      // new pages in the order of their users (fork), free places (compact)
  int4* copies;                       // page, place of its new page in `list`, tokens
};
int64_t align4(int64_t n) { return (n + 3) & ~int64_t(3); }
int64_t ws_layout(int32_t* base, int64_t S, int64_t n_pages, Ws* w) {
  int64_t at = 0;
  auto take = [&](int64_t n) { int32_t* p = base + at; at += align4(n); return p; };
  w->delta = take(n_pages);
  w->writers = take(n_pages);
  w->lowest = take(n_pages);
  w->head = take(4);
  w->rows = (int4*)take(4 * S);
  w->first = take(S);
  w->list = take(n_pages);
  w->copies = (int4*)take(4 * (S > n_pages ? S : n_pages));
  return at;
}

FL_DEV int len_of(const PagesDev& a, int s, bool* bad = nullptr) {
  const int len = a.lens[s], L = (int)min((int64_t)max(len, 0), (int64_t)a.W << a.ps_log2);
  if (L != len && bad) *bad = true;
  return L;
}
FL_DEV int pages_of(const PagesDev& a, int L) { return (int)(((int64_t)L + (1 << a.ps_log2) - 1) >> a.ps_log2); }

// What a call makes of sequence s.
struct Row {
  int p, L, L2, held, want, had;  // parent (-1: none), tokens before and after, their pages; pages that s itself had
  int refuse, last;               // last: the partly filled page that it is about to write, -1: none
  bool bad;                       // a length or that page out of range
};
FL_DEV Row row_of(const PagesDev& a, const int32_t* parents, const int32_t* grow, int s) {
  Row r;
  const int own = len_of(a, s), more = grow ? grow[s] : 0;
  r.p = parents ? parents[s] : s;
  r.refuse = 0;
  r.bad = false;
  if (r.p < -1 || r.p >= a.S) {
    r.refuse = FL_KV_BAD_PARENT;
    r.p = -1;
  }
  r.L = r.p >= 0 ? len_of(a, r.p, &r.bad) : 0;
  const int64_t L2 = max((int64_t)0, (int64_t)r.L + more);
  if (L2 > ((int64_t)a.W << a.ps_log2)) r.refuse |= FL_KV_NO_ROOM;
  r.L2 = (int)min(L2, (int64_t)a.W << a.ps_log2);
  r.held = pages_of(a, r.L);
  r.want = pages_of(a, r.L2);
  r.had = pages_of(a, own);
  r.last = -1;
  if (r.L2 > r.L && (r.L & ((1 << a.ps_log2) - 1))) {
    const int q = a.table[(int64_t)r.p * a.W + r.held - 1];
    if ((unsigned)q < (unsigned)a.n_pages) r.last = q;
    else r.bad = true;
  }
  return r;
}

// Four numbers of CTA `rank` of the cluster, from the same place in its shared memory.
FL_DEV int4 ld_cluster_int4(const int4* p, uint32_t rank) {
  int4 v;
  asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(mapa_shared(smem_u32(p), rank))
               : "memory");
  return v;
}
FL_DEV int4 shfl_int4(int4 v, int lane) {
  return make_int4(__shfl_sync(0xffffffffu, v.x, lane), __shfl_sync(0xffffffffu, v.y, lane), __shfl_sync(0xffffffffu, v.z, lane),
                   __shfl_sync(0xffffffffu, v.w, lane));
}

// Exclusive prefix sums of x and y over the block's threads, and the block's sums.
struct Pair {
  uint64_t x;
  uint32_t y;
};
FL_DEV Pair block_scan(Pair v, Pair* sh, Pair* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const auto scan = [&](Pair& u) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint64_t x = __shfl_up_sync(0xffffffffu, u.x, d);
      const uint32_t y = __shfl_up_sync(0xffffffffu, u.y, d);
      if (lane >= d) u.x += x, u.y += y;
    }
  };
  Pair up = v;
  scan(up);
  if (lane == 31) sh[warp] = up;
  __syncthreads();
  Pair all = sh[lane];  // (PLAN_THREADS / 32 = 32 warps: every warp scans their sums)
  const Pair mine = sh[warp];
  scan(all);
  total->x = __shfl_sync(0xffffffffu, all.x, 31);
  total->y = __shfl_sync(0xffffffffu, all.y, 31);
  const Pair before{__shfl_sync(0xffffffffu, all.x, warp) - mine.x + up.x - v.x,
                    __shfl_sync(0xffffffffu, all.y, warp) - mine.y + up.y - v.y};
  __syncthreads();
  return before;
}

// Counts of each page: of the one CTA in shared memory, of a cluster in the workspace.  `have`: holders after the call, but for
// what new and copied pages change.
template <bool ONE>
struct Counts {
  const PagesDev& a;
  const Ws& w;
  int32_t *have, *writing, *lowest;
  FL_DEV Counts(const PagesDev& a_, const Ws& w_, int32_t* sh) : a(a_), w(w_) {
    have = ONE ? sh : w.delta;
    writing = ONE ? sh + a.n_pages : w.writers;
    lowest = ONE ? sh + 2 * a.n_pages : w.lowest;
    if (ONE) {
      for (int q = threadIdx.x; q < a.n_pages; q += PLAN_THREADS) {
        have[q] = a.refs[q];
        writing[q] = lowest[q] = 0;
      }
    }
  }
  FL_DEV int holders(int q) const { return ONE ? have[q] : a.refs[q] + __ldcg(have + q); }
  FL_DEV int writers(int q) const { return ONE ? writing[q] : __ldcg(writing + q); }
  FL_DEV int first_writer(int q) const { return a.S - (ONE ? lowest[q] : __ldcg(lowest + q)); }
  FL_DEV void clear(int q) const {
    if (!ONE) have[q] = writing[q] = lowest[q] = 0;
  }
};

template <bool ONE>
__global__ void __launch_bounds__(PLAN_THREADS) fork_plan_kernel(PagesDev a, const int32_t* parents, const int32_t* grow,
                                                                 Ws w, int* status) {
  pdl_wait();
  pdl_trigger();
  __shared__ Pair sh[32];
  __shared__ int4 sh_changed[PLAN_THREADS];  // sequence, parent, pages shared with it, pages that the sequence had
  __shared__ int sh_n, sh_longest, sh_refuse;
  __shared__ int4 sh_totals;  // of this CTA: pages wanted, copies, free pages, refused
  extern __shared__ int32_t sh_counts[];
  const int rank = ONE ? 0 : cluster_ctarank(), ctas = ONE ? 1 : cluster_nctarank(), tid = threadIdx.x, lane = tid & 31;
  const Counts<ONE> of(a, w, sh_counts);
  if (tid == 0) sh_n = sh_longest = sh_refuse = 0;
  __syncthreads();
  // Holders: old rows' pages lose one, new rows' gain one; where both are the same page nothing happens, which is
  // most of a beam search's rows.  1024 sequences at a time, the entries of those that change divided among all threads (or
  // such tiles among the CTAs, where there are enough).
  const int tiles = (a.S + PLAN_THREADS - 1) / PLAN_THREADS;
  const bool share = tiles < ctas;
  Row mine;  // of sequence tid, kept where there are no more than threads
  for (int tile = share ? 0 : rank; tile < tiles; tile += share ? 1 : ctas) {
    const int s = tile * PLAN_THREADS + tid;
    int keep = 0;
    bool changes = false;
    if (s < a.S) {
      mine = row_of(a, parents, grow, s);
      keep = min(mine.held, mine.want);
      changes = mine.p != s || keep != mine.had;
    }
    int place = 0;
    if (share) {  // in the sequences' order: the CTAs of a cluster divide one list
      Pair n;
      place = (int)block_scan(Pair{0, changes}, sh, &n).y;
      if (tid == 0) sh_n = (int)n.y;
    } else if (changes) {
      place = atomicAdd(&sh_n, 1);
    }
    if (changes) {
      atomicMax(&sh_longest, max(mine.had, keep));
      sh_changed[place] = make_int4(s, mine.p, keep, mine.had);
    }
    if (s < a.S) {
      if (mine.last >= 0 && (!share || rank == 0)) {
        atomicAdd(of.writing + mine.last, 1);
        atomicMax(of.lowest + mine.last, a.S - s);
      }
    }
    __syncthreads();
    const int longest = sh_longest, step = (share ? ctas : 1) * PLAN_THREADS;
    const int64_t all = (int64_t)sh_n * longest;
    constexpr int BATCH = 4;
    for (int64_t e0 = (share ? rank * PLAN_THREADS : 0) + tid; e0 < all; e0 += BATCH * step) {
      int x[BATCH], y[BATCH];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        x[k] = y[k] = -1;
        const int64_t e = e0 + (int64_t)k * step;
        if (e < all) {
          const int at = (int)kv_div(e, longest), i = (int)(e - (int64_t)at * longest);
          const int4 r = sh_changed[at];
          if (i < r.z && !(r.x == r.y && i < r.w)) x[k] = a.table[(int64_t)r.y * a.W + i];
          if (i < r.w && !(r.x == r.y && i < r.z)) y[k] = a.table[(int64_t)r.x * a.W + i];
        }
      }
#pragma unroll
      for (int k = 0; k < BATCH; ++k)
        if (x[k] != y[k]) {
          if ((unsigned)x[k] < (unsigned)a.n_pages) atomicAdd(of.have + x[k], 1);
          if ((unsigned)y[k] < (unsigned)a.n_pages) atomicSub(of.have + y[k], 1);
        }
    }
    __syncthreads();
    if (tid == 0) sh_n = sh_longest = 0;
    if (tiles > 1) __syncthreads();
  }
  if (!ONE) cluster_sync();
  // What each sequence wants, and what is free: this CTA's part of both, a warp's pages one after another.
  const bool kept = tiles <= 1;  // every CTA has every sequence's Row: the first one goes on with them
  const int per = kept ? a.S : (a.S + ctas - 1) / ctas, s0 = min(a.S, rank * per), s1 = min(a.S, s0 + per);
  const int wper = (a.n_pages + ctas * 32 - 1) / (ctas * 32), q0 = min(a.n_pages, (rank * 32 + (tid >> 5)) * wper),
            q1 = min(a.n_pages, q0 + wper);
  const auto row = [&](int s) { return kept ? mine : row_of(a, parents, grow, s); };
  const auto copied = [&](const Row& r, int s) {
    return r.last >= 0 && !(of.holders(r.last) == of.writers(r.last) && of.first_writer(r.last) == s);
  };
  Pair sum{0, 0}, total;  // pages wanted << 32 | copies; free pages
  for (int s = s0 + tid; s < s1; s += PLAN_THREADS) {
    const Row r = row(s);
    if (r.refuse) atomicOr(&sh_refuse, r.refuse);
    const int c = copied(r, s);
    sum.x += ((uint64_t)(max(0, r.want - r.held) + c) << 32) | c;
  }
  uint32_t nfree = 0;
  for (int q = q0; q < q1; q += 32) nfree += __popc(__ballot_sync(0xffffffffu, q + lane < q1 && of.holders(min(q + lane, a.n_pages - 1)) == 0));
  if (lane == 0) sum.y = nfree;
  const Pair before = block_scan(sum, sh, &total);  // (the free ones: of this warp's first lane)
  int64_t all_wanted = (int64_t)(total.x >> 32), all_free = total.y, wanted0 = 0, free0 = 0;
  int copies = (int)(uint32_t)total.x, copies0 = 0, refuse = sh_refuse;
  if (!ONE) {
    if (tid == 0) sh_totals = make_int4((int)all_wanted, copies, (int)all_free, refuse);
    cluster_sync();
    const int4 totals = ld_cluster_int4(&sh_totals, min(lane, ctas - 1));
    all_wanted = all_free = refuse = copies = 0;
    for (int c = 0; c < ctas; ++c) {
      const int4 t = shfl_int4(totals, c);
      if (c == rank) wanted0 = all_wanted, free0 = all_free, copies0 = copies;
      all_wanted += t.x;
      all_free += t.z;
      copies += t.y;
      refuse |= t.w;
    }
  }
  if (all_wanted > all_free) refuse |= FL_KV_NO_ROOM;
  if (rank == 0 && tid == 0) {
    if (refuse) atomicOr(status, refuse);
    w.head[0] = refuse ? 0 : copies;
    w.head[1] = refuse;
  }
  for (int base = s0; base < s1; base += PLAN_THREADS) {
    const int s = base + tid;
    Row r;
    int c = 0;
    Pair x{0, 0}, ahead = before;
    if (s < s1) {
      r = row(s);
      c = copied(r, s);
      x.x = ((uint64_t)(max(0, r.want - r.held) + c) << 32) | c;
    }
    total = Pair{0, 0};
    if (s1 - s0 > PLAN_THREADS) ahead = block_scan(x, sh, &total);  // (else the sums above are these)
    if (s < s1) {
      if (r.bad) atomicOr(status, FL_KV_BAD_PAGE);
      const int at = (int)(wanted0 + (int64_t)(ahead.x >> 32));
      w.first[s] = at;
      w.rows[s] = make_int4(r.p, min(r.held, r.want), r.held - c, r.want);
      a.lens_to[s] = refuse ? a.lens[s] : r.L2;
      if (c) w.copies[copies0 + (int)(uint32_t)ahead.x] = make_int4(r.last, at, r.L & ((1 << a.ps_log2) - 1), 0);
    }
    wanted0 += (int64_t)(total.x >> 32);
    copies0 += (int)(uint32_t)total.x;
  }
  int64_t at = free0 + __shfl_sync(0xffffffffu, before.y, 0);
  for (int q = q0; q < q1; q += 32) {
    const bool in = q + lane < q1;
    const int x = min(q + lane, a.n_pages - 1), have = of.holders(x), writers = of.writers(x);
    const unsigned m = __ballot_sync(0xffffffffu, in && have == 0);
    if (in) {
      const int64_t mine_at = at + __popc(m & ((1u << lane) - 1));
      const bool taken = have == 0 && mine_at < all_wanted;
      if (taken && !refuse) w.list[mine_at] = x;
      const int leave = writers == 0 ? 0 : have == writers ? writers - 1 : writers;
      a.refs_to[x] = refuse ? a.refs[x] : taken ? 1 : have - leave;
    }
    at += __popc(m);
  }
  if (!ONE) {
    cluster_sync();  // nobody looks at the counts any more
    for (int q = q0 + lane; q < q1; q += 32) of.clear(q);
  }
}

template <bool ONE>
__global__ void __launch_bounds__(PLAN_THREADS) compact_plan_kernel(PagesDev a, int32_t* moved, int32_t* used, Ws w) {
  pdl_wait();
  pdl_trigger();
  __shared__ Pair sh[32];
  __shared__ int4 sh_all, sh_stay;  // of this CTA
  const int rank = ONE ? 0 : cluster_ctarank(), ctas = ONE ? 1 : cluster_nctarank(), tid = threadIdx.x, lane = tid & 31;
  // a warp's pages one after another
  const int wper = (a.n_pages + ctas * 32 - 1) / (ctas * 32), q0 = min(a.n_pages, (rank * 32 + (tid >> 5)) * wper),
            q1 = min(a.n_pages, q0 + wper);
  const auto busy = [&](int q) { return __ballot_sync(0xffffffffu, q + lane < q1 && a.refs[min(q + lane, a.n_pages - 1)] > 0); };
  Pair total;
  uint32_t n = 0;
  for (int q = q0; q < q1; q += 32) n += __popc(busy(q));
  int before = (int)__shfl_sync(0xffffffffu, block_scan(Pair{0, lane == 0 ? n : 0}, sh, &total).y, 0), all = (int)total.y;
  if (!ONE) {
    if (tid == 0) sh_all = make_int4(all, 0, 0, 0);
    cluster_sync();
    const int of = ld_cluster_int4(&sh_all, min(lane, ctas - 1)).x;
    all = 0;
    for (int c = 0; c < ctas; ++c) {
      if (c == rank) before += all;
      all += __shfl_sync(0xffffffffu, of, c);
    }
  }
  // the pages in use among the first `all` stay
  n = 0;
  for (int q = q0; q < min(q1, all); q += 32) n += __popc(busy(q) & (all - q >= 32 ? ~0u : (1u << (all - q)) - 1));
  block_scan(Pair{0, lane == 0 ? n : 0}, sh, &total);
  int stay = (int)total.y;
  if (!ONE) {
    if (tid == 0) sh_stay = make_int4(stay, 0, 0, 0);
    cluster_sync();
    const int of = ld_cluster_int4(&sh_stay, min(lane, ctas - 1)).x;
    stay = 0;
    for (int c = 0; c < ctas; ++c) stay += __shfl_sync(0xffffffffu, of, c);
  }
  const int moves = all - stay;
  if (rank == 0 && tid == 0) {
    w.head[0] = moves;
    w.head[1] = 0;
    *used = all;
  }
  for (int q = q0; q < q1; q += 32) {
    const unsigned m = busy(q), bit = 1u << lane;
    const int x = q + lane, ahead = before + __popc(m & (bit - 1));
    if (x < q1) {
      if (x < all && !(m & bit)) __stcg(w.list + (x - ahead), x);
      if (x >= all && (m & bit)) __stcg(w.copies + (ahead - stay), make_int4(x, ahead - stay, 1 << a.ps_log2, 0));
    }
    before += __popc(m);
  }
  for (int s = rank * PLAN_THREADS + tid; s < a.S; s += ctas * PLAN_THREADS) a.lens_to[s] = a.lens[s];
  if (ONE) __syncthreads();
  else cluster_sync();
  for (int q = q0 + lane; q < q1; q += 32) {
    const int refs = a.refs[q];
    if (refs > 0 && q < all) {
      moved[q] = q;
      a.refs_to[q] = refs;
    } else if (refs <= 0) {
      moved[q] = -1;
      if (q >= all) a.refs_to[q] = 0;
    } else {
      a.refs_to[q] = 0;
    }
  }
  for (int i = rank * PLAN_THREADS + tid; i < moves; i += ctas * PLAN_THREADS) {
    const int src = __ldcg(&w.copies[i].x), dst = __ldcg(w.list + i);
    moved[src] = dst;
    a.refs_to[dst] = a.refs[src];
  }
}

struct Caches {
  char* at[2 * FL_KV_MAX_CACHES];  // keys and values of each
  int n, units;                    // arrays; units of a page
  int heads, row, by_token;        // bytes of a token's head; whether a token's heads lie next to each other
  int64_t page_stride, head_stride, token_stride;  // in bytes
};
FL_DEV int64_t shfl64(int64_t x, int lane) { return __shfl_sync(0xffffffffu, x, lane); }

// The copies, a warp a unit: from global memory into the warp's shared memory and from there to the new page, in
// blocks of 8 KB by bulk copies that one lane asks for, two loads ahead of a store.  What a page holds of its sequence is
// `runs` stretches of memory; each of its units has an equal part of their bytes, so that all are as long.
// HBM is the bound: 71 pages of 27 MB moved in 26 caches 616 us (6.3 TB/s read and written, with the plan), the copies of a beam
// search's 64 sequences 100 us (5.9 TB/s).  16-byte loads and stores by all threads took 661 and 118.
FL_DEV void copy_pages(const Caches& c, const Ws& w, int ps_log2, char* ring, uint64_t* full, int* status) {
  const int lane = threadIdx.x & 31, warps = gridDim.x * COPY_WARPS;
  const int64_t all = (int64_t)__ldcg(w.head) * c.n * c.units;
  int issued = 0, stored = 0;  // blocks
  bool ok = true;
  static_assert(STAGES == 3);
  int64_t to0 = 0, to1 = 0;  // of the blocks on their way, the first and the second
  int bytes0 = 0, bytes1 = 0;
  const auto store = [&] {  // the first block on its way
    const int st = stored % STAGES;
    ok = mbar_wait(full + st, stored / STAGES & 1);
    if (!ok) return;
    bulk_store((char*)to0, ring + st * BLOCK_BYTES, bytes0);
    bulk_commit();
    ++stored;
    to0 = to1, bytes0 = bytes1;
  };
  for (int64_t u0 = (int64_t)threadIdx.x / 32 * gridDim.x + blockIdx.x; u0 < all; u0 += 32ll * warps) {
    // 32 units at once, one a lane: where from, where to, how much
    const int64_t u = u0 + (int64_t)lane * warps;
    int64_t from = 0, to = 0;
    int begin = 0, end = 0, run = 1, inner = 1;  // the unit's part of the runs' bytes; bytes of a run, runs of an inner row of them
    if (u < all) {
      const int64_t x = kv_div(u, c.units), job_at = kv_div(x, c.n);
      const int part = (int)(u - x * c.units);
      const int4 job = __ldcg(w.copies + job_at);
      const int64_t base = (int64_t)c.at[x - job_at * c.n];
      from = base + job.x * c.page_stride;
      to = base + (int64_t)__ldcg(w.list + job.y) * c.page_stride;
      const int bytes = job.z * c.heads * c.row;
      if (c.by_token) {  // a token's heads lie next to each other, or a head's tokens do, or neither
        run = c.token_stride == (int64_t)c.heads * c.row ? bytes : c.heads * c.row;
      } else if (c.token_stride == c.row) {
        run = job.z == 1 << ps_log2 && c.head_stride == (int64_t)c.row << ps_log2 ? bytes : job.z * c.row;
      } else {
        run = c.row;
        inner = job.z;
      }
      begin = (int)((int64_t)bytes / 16 * part / c.units) * 16;
      end = (int)((int64_t)bytes / 16 * (part + 1) / c.units) * 16;
    }
    for (int l = 0; l < 32 && u0 + (int64_t)l * warps < all; ++l) {
      const int64_t f = shfl64(from, l), t = shfl64(to, l);
      const int b = __shfl_sync(0xffffffffu, begin, l), e = __shfl_sync(0xffffffffu, end, l), r = __shfl_sync(0xffffffffu, run, l),
                in = __shfl_sync(0xffffffffu, inner, l);
      if (lane == 0) {
        const int64_t outer = c.by_token ? c.token_stride : c.head_stride;
        int off = b % r, j = b / r % in;
        int64_t row = (int64_t)(b / r / in) * outer, col = j * c.token_stride;
        for (int at = b; at < e && ok;) {
          const int n = min(BLOCK_BYTES, min(r - off, e - at)), st = issued % STAGES;
          if (issued - stored == STAGES - 1) store();
          if (!ok) break;
          if (issued >= STAGES) bulk_wait_read<1>();  // the store before the last one is through with this stage
          (issued == stored ? to0 : to1) = t + row + col + off;
          (issued == stored ? bytes0 : bytes1) = n;
          mbar_arrive_expect_tx(full + st, n);
          bulk_load(ring + st * BLOCK_BYTES, (const char*)(f + row + col + off), n, full + st);
          ++issued;
          at += n;
          off += n;
          if (off == r) {
            off = 0;
            col += c.token_stride;
            if (++j == in) j = 0, col = 0, row += outer;
          }
        }
      }
    }
  }
  if (lane == 0) {
    while (ok && stored < issued) store();
    if (!ok) {
      atomicOr(status, FL_KV_TIMEOUT);
      for (int i = stored; i < issued; ++i) mbar_wait(full + i % STAGES, i / STAGES & 1);  // what is still on its way
    }
    bulk_wait_all();
  }
}

// The rows of the new table, in pieces of a block's threads each, from the last CTA on: the first ones begin with the copies.
template <class F>
FL_DEV void for_entries(const PagesDev& a, F f) {
  const int per = (a.W + COPY_THREADS - 1) / COPY_THREADS;
  for (int64_t u = gridDim.x - 1 - blockIdx.x; u < (int64_t)a.S * per; u += gridDim.x) {
    const int s = (int)kv_div(u, per), i = (int)(u - (int64_t)s * per) * COPY_THREADS + threadIdx.x;
    if (i < a.W) f(s, i);
  }
}

// Every warp's ring and barriers.
FL_DEV void copy_all(const Caches& c, const Ws& w, int ps_log2, int* status) {
  extern __shared__ __align__(128) char ring[];
  __shared__ uint64_t full[COPY_WARPS][STAGES];
  const int warp = threadIdx.x >> 5;
  if ((threadIdx.x & 31) == 0) {
    for (int i = 0; i < STAGES; ++i) mbar_init(&full[warp][i], 1);
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  __syncwarp();
  copy_pages(c, w, ps_log2, ring + warp * STAGES * BLOCK_BYTES, full[warp], status);
}

__global__ void __launch_bounds__(COPY_THREADS) fork_kernel(PagesDev a, Ws w, const __grid_constant__ Caches c, int* status) {
  pdl_wait();
  pdl_trigger();
  const bool refused = __ldcg(w.head + 1) != 0;
  for_entries(a, [&](int s, int i) {
    const int64_t e = (int64_t)s * a.W + i;
    const int4 r = __ldcg(w.rows + s);
    const int first = __ldcg(w.first + s);
    int page = -1;
    if (refused) {
      page = a.table[e];
    } else if (i >= r.z && i < r.w) {
      page = __ldcg(w.list + first + i - r.z);
    } else if (i < r.y) {
      page = a.table[(int64_t)r.x * a.W + i];
      if ((unsigned)page >= (unsigned)a.n_pages) atomicOr(status, FL_KV_BAD_PAGE);
    }
    a.table_to[e] = page;
  });
  copy_all(c, w, a.ps_log2, status);
}

__global__ void __launch_bounds__(COPY_THREADS) compact_kernel(PagesDev a, const int32_t* moved, Ws w,
                                                               const __grid_constant__ Caches c, int* status) {
  pdl_wait();
  pdl_trigger();
  for_entries(a, [&](int s, int i) {
    const int64_t e = (int64_t)s * a.W + i;
    int page = -1;
    bool bad = false;
    if (i < pages_of(a, len_of(a, s, &bad))) {
      const int x = a.table[e];
      if ((unsigned)x < (unsigned)a.n_pages) page = __ldcg(moved + x);
      bad |= page < 0;
    }
    if (bad) atomicOr(status, FL_KV_BAD_PAGE);
    a.table_to[e] = page;
  });
  copy_all(c, w, a.ps_log2, status);
}

int check_pages(const char* who, const fl_kv_pages* p, PagesDev* out) {
  if (!p || p->n_seqs < 0 || p->n_pages < 1 || p->table_stride < 1)
    return fl_internal_error(FL_ERR_INVALID_ARG, "%s: sizes", who);
  const int ps = p->page_size;
  if (ps < 16 || ps > 256 || (ps & (ps - 1)))
    return fl_internal_error(FL_ERR_UNSUPPORTED, "%s: page_size %d (a power of two, 16 to 256)", who, ps);
  int lg = 4;
  while ((1 << lg) < ps) ++lg;
  constexpr int64_t most = (1ll << 31) - 1024;
  if ((int64_t)p->n_seqs * p->table_stride > most || ((int64_t)p->table_stride << lg) > most || p->n_seqs > 1 << 20 ||
      p->n_pages > most)
    return fl_internal_error(FL_ERR_CAPACITY, "%s: more sequences, pages or tokens in a table row than are counted in 32 bits", who);
  *out = PagesDev{p->lens, p->table, p->refs, nullptr, nullptr, nullptr, p->n_seqs, p->n_pages, lg, p->table_stride};
  return FL_OK;
}

int check_call(const char* who, const fl_kv_cache* caches, int n, const fl_kv_pages* from, const fl_kv_pages* to,
               const void* ws, const int* status, PagesDev* a, Caches* c, Ws* w) {
  if (int rc = check_pages(who, from, a)) return rc;
  if (!to || to->n_seqs != from->n_seqs || to->n_pages != from->n_pages || to->page_size != from->page_size ||
      to->table_stride != from->table_stride)
    return fl_internal_error(FL_ERR_INVALID_ARG, "%s: `to` has other sizes than `from`", who);
  const int32_t* arrays[6] = {from->lens, from->table, from->refs, to->lens, to->table, to->refs};
  for (int i = 0; i < 6; ++i) {
    const bool needed = a->S > 0 || i % 3 == 2;
    if ((needed && !arrays[i]) || fl_misaligned(arrays[i], 4)) return fl_internal_error(FL_ERR_INVALID_ARG, "%s: arrays", who);
    for (int j = 0; j < i; ++j)
      if (needed && arrays[i] == arrays[j]) return fl_internal_error(FL_ERR_INVALID_ARG, "%s: two arrays are the same", who);
  }
  if (!caches || n < 1 || n > FL_KV_MAX_CACHES || !ws || fl_misaligned(ws, 16) || !status || fl_misaligned(status, 4))
    return fl_internal_error(FL_ERR_INVALID_ARG, "%s: args", who);
  for (int i = 0; i < n; ++i) {
    const fl_kv_cache &x = caches[i], &y = caches[0];
    KvBatchDev unused;
    const fl_kv_batch none{0, 0, 0, 1, nullptr, nullptr, nullptr};
    if (int rc = fl_kv_check(who, &x, &none, x.kv_heads, &unused)) return rc;
    if (x.n_pages != from->n_pages || x.page_size != from->page_size)
      return fl_internal_error(FL_ERR_INVALID_ARG, "%s: cache %d has other pages than the table", who, i);
    if (x.dtype != y.dtype || x.kv_heads != y.kv_heads || x.head_dim != y.head_dim || x.page_stride != y.page_stride ||
        x.head_stride != y.head_stride || x.token_stride != y.token_stride)
      return fl_internal_error(FL_ERR_INVALID_ARG, "%s: caches 0 and %d are not alike", who, i);
    c->at[2 * i] = (char*)x.k;
    c->at[2 * i + 1] = (char*)x.v;
  }
  c->n = 2 * n;
  c->heads = caches[0].kv_heads;
  c->row = caches[0].head_dim * 2;
  const int64_t page = (int64_t)c->heads * c->row << a->ps_log2;
  if (page >= 1ll << 31) return fl_internal_error(FL_ERR_CAPACITY, "%s: a page of %d heads", who, c->heads);
  c->units = (int)((page + UNIT_BYTES - 1) / UNIT_BYTES);
  c->page_stride = caches[0].page_stride * 2;
  c->head_stride = caches[0].head_stride * 2;
  c->token_stride = caches[0].token_stride * 2;
  c->by_token = c->token_stride != c->row && c->head_stride == c->row;
  a->lens_to = to->lens;
  a->table_to = to->table;
  a->refs_to = to->refs;
  ws_layout((int32_t*)const_cast<void*>(ws), a->S, a->n_pages, w);
  return FL_OK;
}

template <typename... KArgs, typename... Args>
cudaError_t launch_plan(void (*kern)(KArgs...), int ctas, int smem, cudaStream_t st, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // see pdl_wait
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(PLAN_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = ctas > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, static_cast<KArgs>(args)...);
}

// One CTA as long as what it goes through is short; tables of more entries take a cluster, whose barriers cost 5 us.  A whole call, one
// CTA / a cluster, us: beams that all change, 16 x 64 entries 7.8 / 13.4, 16 x 512 11.5 / 13.3, 16 x 1024 15.8 / 14.0, 16 x 4096 38.6 /
// 18.0, 64 x 1024 43.4 / 17.4; sequences that stay as they are, 192 x 71 8.5 / 11.1, 192 x 341 9.0 / 11.6, 64 x 1022 11.4 / 12.5, 1000 x 65
// 12.8 / 19.2.  The host does not know which of the two a call is: the bound is for the second kind, a server's calls.
bool small_plan(const PagesDev& a) { return a.n_pages <= 16384 && (int64_t)a.S * a.W <= 65536 && a.S <= PLAN_THREADS; }

}  // namespace

extern "C" size_t fl_k_kv_pages_workspace(const fl_kv_pages* pages) {
  PagesDev a;
  if (check_pages("kv pages workspace", pages, &a)) return 0;
  Ws w;
  return (size_t)ws_layout(nullptr, a.S, a.n_pages, &w) * 4;
}

extern "C" int fl_k_kv_fork(const fl_kv_cache* caches, int32_t n_caches, const fl_kv_pages* from, const fl_kv_pages* to,
                            const int32_t* parents, const int32_t* new_tokens, void* workspace, int* status, void* stream) {
  PagesDev a;
  Caches c;
  Ws w;
  if (int rc = check_call("kv fork", caches, n_caches, from, to, workspace, status, &a, &c, &w)) return rc;
  if (fl_misaligned(parents, 4) || fl_misaligned(new_tokens, 4)) return fl_internal_error(FL_ERR_INVALID_ARG, "kv fork: alignment");
  const cudaStream_t st = (cudaStream_t)stream;
  if (small_plan(a)) {
    FL_CUDA_TRY(fl_func_smem((const void*)fork_plan_kernel<true>, 3 * 16384 * 4));
    FL_CUDA_TRY(launch_plan(fork_plan_kernel<true>, 1, 12 * a.n_pages, st, a, parents, new_tokens, w, status));
  } else {
    FL_CUDA_TRY(launch_plan(fork_plan_kernel<false>, MAX_PLAN_CTAS, 0, st, a, parents, new_tokens, w, status));
  }
  FL_CUDA_TRY(fl_func_smem((const void*)fork_kernel, COPY_SMEM));
  FL_CUDA_TRY(fl_launch(fork_kernel, dim3(COPY_CTAS * fl_sm_count()), dim3(COPY_THREADS), COPY_SMEM, st, a, w, c, status));
  return FL_OK;
}

extern "C" int fl_k_kv_compact(const fl_kv_cache* caches, int32_t n_caches, const fl_kv_pages* from, const fl_kv_pages* to,
                               int32_t* moved, int32_t* used, void* workspace, int* status, void* stream) {
  PagesDev a;
  Caches c;
  Ws w;
  if (int rc = check_call("kv compact", caches, n_caches, from, to, workspace, status, &a, &c, &w)) return rc;
  if (!moved || !used || fl_misaligned(moved, 4) || fl_misaligned(used, 4))
    return fl_internal_error(FL_ERR_INVALID_ARG, "kv compact: args");
  const cudaStream_t st = (cudaStream_t)stream;
  if (a.n_pages <= 16384)
    FL_CUDA_TRY(launch_plan(compact_plan_kernel<true>, 1, 0, st, a, moved, used, w));
  else
    FL_CUDA_TRY(launch_plan(compact_plan_kernel<false>, MAX_PLAN_CTAS, 0, st, a, moved, used, w));
  FL_CUDA_TRY(fl_func_smem((const void*)compact_kernel, COPY_SMEM));
  FL_CUDA_TRY(fl_launch(compact_kernel, dim3(COPY_CTAS * fl_sm_count()), dim3(COPY_THREADS), COPY_SMEM, st, a, moved, w, c, status));
  return FL_OK;
}
