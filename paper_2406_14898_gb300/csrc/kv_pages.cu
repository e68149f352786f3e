// Sequences that share the pages of a cache: fork (continue, share, copy on write, extend, shorten, leave) and compact.
//
// A call is two launches.  The plan is integer work on a few arrays: who has each page after the call, which are free, who
// gets which.  One CTA does it, or one cluster where the arrays are long, with a barrier between its phases.  The second
// launch, over the whole GPU, writes the table and copies the pages' tokens in every cache.
#include "../../include/flglm_kernels.h"
#include "kv_plan.cuh"
#include "ptx.cuh"

namespace {

constexpr int PLAN_THREADS = 1024, MAX_PLAN_CTAS = 8;
constexpr int COPY_THREADS = 256;
constexpr int COPY_PIECES = 2048;  // 16-byte pieces of a unit of copying

struct PagesDev {
  const int32_t *lens, *table, *refs;
  int32_t *lens_to, *table_to, *refs_to;
  int S, n_pages, ps_log2, W;
};

// A workspace: what the plan tells the second launch, and counts of each page that are zero between calls.
struct Ws {
  int32_t* head;                        // copies, refused
  int4* totals;                         // of each CTA of the plan: pages wanted, copies, free pages, refused
  int32_t *delta, *writers, *lowest;    // zero between calls: holders more or less, sequences about to write, S - the first
  int32_t *wanted, *first;              // of each sequence: 2 pages wanted + copied, place of its first in `list`
  int32_t* list;                        // new pages in the order of their users (fork), free places (compact)
  int4* copies;                         // page, place of its new page in `list`, tokens
};
int64_t align4(int64_t n) { return (n + 3) & ~int64_t(3); }
int64_t ws_layout(int32_t* base, int64_t S, int64_t n_pages, Ws* w) {
  int64_t at = 0;
  auto take = [&](int64_t n) { int32_t* p = base + at; at += align4(n); return p; };
  w->delta = take(n_pages);
  w->writers = take(n_pages);
  w->lowest = take(n_pages);
  w->head = take(4);
  w->totals = (int4*)take(4 * MAX_PLAN_CTAS);
  w->wanted = take(S);
  w->first = take(S);
  w->list = take(n_pages);
  w->copies = (int4*)take(4 * (S > n_pages ? S : n_pages));
  return at;
}

// What a call makes of sequence s.
struct Row {
  int p, L, L2, held, want;  // parent (-1: none), tokens before and after, their pages
  int refuse;
};
FL_DEV int len_of(const PagesDev& a, int s, int* status) {
  const int64_t cap = (int64_t)a.W << a.ps_log2;
  const int len = __ldg(a.lens + s);
  const int L = (int)min((int64_t)max(len, 0), cap);
  if (L != len && status) atomicOr(status, FL_KV_BAD_PAGE);
  return L;
}
FL_DEV int pages_of(const PagesDev& a, int L) { return (int)(((int64_t)L + (1 << a.ps_log2) - 1) >> a.ps_log2); }
FL_DEV Row row_of(const PagesDev& a, const int32_t* parents, const int32_t* grow, int s, int* status) {
  Row r;
  r.p = parents ? __ldg(parents + s) : s;
  r.refuse = 0;
  if (r.p < -1 || r.p >= a.S) {
    r.refuse = FL_KV_BAD_PARENT;
    r.p = -1;
  }
  r.L = r.p >= 0 ? len_of(a, r.p, status) : 0;
  const int64_t L2 = max((int64_t)0, (int64_t)r.L + (grow ? __ldg(grow + s) : 0));
  if (L2 > ((int64_t)a.W << a.ps_log2)) r.refuse |= FL_KV_NO_ROOM;
  r.L2 = (int)min(L2, (int64_t)a.W << a.ps_log2);
  r.held = pages_of(a, r.L);
  r.want = pages_of(a, r.L2);
  return r;
}

FL_DEV uint32_t cluster_nctarank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}

// Exclusive prefix sum of x over the block's threads, and the block's sum.
template <class T>
FL_DEV T block_scan(T x, T* sh, T* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  T v = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const T y = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v += y;
  }
  if (lane == 31) sh[warp] = v;
  __syncthreads();
  if (warp == 0) {
    T w = lane < (int)(blockDim.x >> 5) ? sh[lane] : T(0), u = w;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const T y = __shfl_up_sync(0xffffffffu, u, d);
      if (lane >= d) u += y;
    }
    sh[lane] = u - w;
    if (lane == 31) sh[32] = u;
  }
  __syncthreads();
  const T before = sh[warp] + v - x;
  *total = sh[32];
  __syncthreads();
  return before;
}

__global__ void __launch_bounds__(PLAN_THREADS) fork_plan_kernel(PagesDev a, const int32_t* parents, const int32_t* grow,
                                                                 Ws w, int* status) {
  pdl_wait();
  pdl_trigger();
  __shared__ uint64_t sh[33];
  const int rank = cluster_ctarank(), ctas = cluster_nctarank(), tid = threadIdx.x, lane = tid & 31;
  const int ps = 1 << a.ps_log2;
  // Holders: old rows' pages lose one, new rows' gain one; where both are the same page nothing happens, which is
  // most of a beam search's rows.
  for (int s = rank * (PLAN_THREADS / 32) + (tid >> 5); s < a.S; s += ctas * (PLAN_THREADS / 32)) {
    const Row r = row_of(a, parents, grow, s, nullptr);
    const int had = pages_of(a, len_of(a, s, nullptr)), keep = min(r.held, r.want);
    const int32_t *mine = a.table + (int64_t)s * a.W, *theirs = a.table + (int64_t)max(r.p, 0) * a.W;
    for (int i = (r.p == s ? keep : 0) + lane; i < max(had, keep); i += 32) {
      const int x = i < keep ? __ldg(theirs + i) : -1, y = i < had ? __ldg(mine + i) : -1;
      if (x != y) {
        if ((unsigned)x < (unsigned)a.n_pages) atomicAdd(w.delta + x, 1);
        if ((unsigned)y < (unsigned)a.n_pages) atomicSub(w.delta + y, 1);
      }
    }
    if (lane == 0 && r.L2 > r.L && (r.L & (ps - 1))) {
      const int q = __ldg(theirs + r.held - 1);
      if ((unsigned)q < (unsigned)a.n_pages) {
        atomicAdd(w.writers + q, 1);
        atomicMax(w.lowest + q, a.S - s);
      }
    }
  }
  cluster_sync();
  // What each sequence wants, and what is free: this CTA's part of both.
  const int per = (a.S + ctas - 1) / ctas, s0 = min(a.S, rank * per), s1 = min(a.S, s0 + per);
  const int pper = (a.n_pages + ctas - 1) / ctas, q0 = min(a.n_pages, rank * pper), q1 = min(a.n_pages, q0 + pper);
  uint64_t sum = 0;  // pages wanted << 32 | copies
  int refuse = 0, nfree = 0;
  for (int s = s0 + tid; s < s1; s += PLAN_THREADS) {
    const Row r = row_of(a, parents, grow, s, status);
    refuse |= r.refuse;
    int copied = 0;
    if (r.L2 > r.L && (r.L & (ps - 1))) {
      const int q = __ldg(a.table + (int64_t)r.p * a.W + r.held - 1);
      if ((unsigned)q < (unsigned)a.n_pages)
        copied = !(__ldg(a.refs + q) + __ldcg(w.delta + q) == __ldcg(w.writers + q) && __ldcg(w.lowest + q) == a.S - s);
      else
        atomicOr(status, FL_KV_BAD_PAGE);
    }
    const int wanted = max(0, r.want - r.held) + copied;
    w.wanted[s] = 2 * wanted + copied;
    sum += ((uint64_t)wanted << 32) | copied;
  }
  for (int q = q0 + tid; q < q1; q += PLAN_THREADS) nfree += __ldg(a.refs + q) + __ldcg(w.delta + q) == 0;
  uint64_t total, total2;
  block_scan<uint64_t>(sum, sh, &total);
  block_scan<uint64_t>(nfree, sh, &total2);
  refuse = __syncthreads_or(refuse & FL_KV_NO_ROOM) ? FL_KV_NO_ROOM : 0;
  int bad = 0;
  for (int s = s0 + tid; s < s1; s += PLAN_THREADS)
    if (parents) {
      const int p = __ldg(parents + s);
      bad |= p < -1 || p >= a.S;
    }
  if (__syncthreads_or(bad)) refuse |= FL_KV_BAD_PARENT;
  if (tid == 0) __stcg(w.totals + rank, make_int4((int)(total >> 32), (int)(uint32_t)total, (int)total2, refuse));
  cluster_sync();
  int64_t all_wanted = 0, all_free = 0, wanted0 = 0, free0 = 0;
  int copies = 0, copies0 = 0;
  refuse = 0;
  for (int c = 0; c < ctas; ++c) {
    const int4 t = __ldcg(w.totals + c);
    if (c == rank) wanted0 = all_wanted, free0 = all_free, copies0 = copies;
    all_wanted += t.x;
    all_free += t.z;
    copies += t.y;
    refuse |= t.w;
  }
  if (all_wanted > all_free) refuse |= FL_KV_NO_ROOM;
  if (rank == 0 && tid == 0) {
    if (refuse) atomicOr(status, refuse);
    w.head[0] = refuse ? 0 : copies;
    w.head[1] = refuse;
  }
  for (int base = s0; base < s1; base += PLAN_THREADS) {
    const int s = base + tid;
    const int x = s < s1 ? w.wanted[s] : 0;
    const uint64_t before = block_scan<uint64_t>(((uint64_t)(x >> 1) << 32) | (x & 1), sh, &total);
    if (s < s1) {
      const Row r = row_of(a, parents, grow, s, nullptr);
      const int at = (int)(wanted0 + (int64_t)(before >> 32));
      w.first[s] = at;
      a.lens_to[s] = refuse ? __ldg(a.lens + s) : r.L2;
      if (x & 1)
        w.copies[copies0 + (int)(uint32_t)before] =
            make_int4(__ldg(a.table + (int64_t)r.p * a.W + r.held - 1), at, r.L & (ps - 1), 0);
    }
    wanted0 += (int64_t)(total >> 32);
    copies0 += (int)(uint32_t)total;
  }
  for (int base = q0; base < q1; base += PLAN_THREADS) {
    const int q = base + tid;
    int pre = -1, writers = 0;
    if (q < q1) {
      pre = __ldg(a.refs + q) + __ldcg(w.delta + q);
      writers = __ldcg(w.writers + q);
    }
    const uint64_t before = block_scan<uint64_t>(pre == 0, sh, &total);
    if (q < q1) {
      const int64_t at = free0 + (int64_t)before;
      const bool taken = pre == 0 && at < all_wanted;
      if (taken && !refuse) w.list[at] = q;
      const int leave = writers == 0 ? 0 : pre == writers ? writers - 1 : writers;
      a.refs_to[q] = refuse ? __ldg(a.refs + q) : taken ? 1 : pre - leave;
      w.delta[q] = w.writers[q] = w.lowest[q] = 0;
    }
    free0 += (int64_t)total;
  }
}

__global__ void __launch_bounds__(PLAN_THREADS) compact_plan_kernel(PagesDev a, int32_t* moved, int32_t* used, Ws w) {
  pdl_wait();
  pdl_trigger();
  __shared__ uint64_t sh[33];
  const int rank = cluster_ctarank(), ctas = cluster_nctarank(), tid = threadIdx.x;
  const int pper = (a.n_pages + ctas - 1) / ctas, q0 = min(a.n_pages, rank * pper), q1 = min(a.n_pages, q0 + pper);
  uint64_t total, n = 0;
  for (int q = q0 + tid; q < q1; q += PLAN_THREADS) n += __ldg(a.refs + q) > 0;
  block_scan<uint64_t>(n, sh, &total);
  if (tid == 0) __stcg(&w.totals[rank].x, (int)total);
  cluster_sync();
  int all = 0, before0 = 0;
  for (int c = 0; c < ctas; ++c) {
    if (c == rank) before0 = all;
    all += __ldcg(&w.totals[c].x);
  }
  // pages in use among the first `all`: those that stay
  const int edge = pper > 0 ? min(ctas - 1, all / pper) : 0;
  int stay = 0;
  for (int c = 0; c < edge; ++c) stay += __ldcg(&w.totals[c].x);
  n = 0;
  for (int q = edge * pper + tid; q < all; q += PLAN_THREADS) n += __ldg(a.refs + q) > 0;
  block_scan<uint64_t>(n, sh, &total);
  stay += (int)total;
  const int moves = all - stay;
  if (rank == 0 && tid == 0) {
    w.head[0] = moves;
    w.head[1] = 0;
    *used = all;
  }
  for (int base = q0; base < q1; base += PLAN_THREADS) {
    const int q = base + tid;
    const bool busy = q < q1 && __ldg(a.refs + q) > 0;
    const int before = before0 + (int)block_scan<uint64_t>(busy, sh, &total);
    if (q < q1) {
      if (q < all && !busy) w.list[q - before] = q;
      if (q >= all && busy) w.copies[before - stay] = make_int4(q, before - stay, 1 << a.ps_log2, 0);
    }
    before0 += (int)total;
  }
  for (int s = rank * PLAN_THREADS + tid; s < a.S; s += ctas * PLAN_THREADS) a.lens_to[s] = __ldg(a.lens + s);
  cluster_sync();
  for (int q = q0 + tid; q < q1; q += PLAN_THREADS) {
    const int refs = __ldg(a.refs + q);
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
    a.refs_to[dst] = __ldg(a.refs + src);
  }
}

struct Caches {
  uint4* at[2 * FL_KV_MAX_CACHES];  // keys and values of each
  int n, heads, row;                // arrays, heads, 16-byte pieces of a row
  int64_t page_stride, head_stride, token_stride;  // in pieces
};

FL_DEV void copy_pages(const Caches& c, const Ws& w, int ps_log2) {
  const int copies = __ldcg(w.head);
  const int row_log2 = 31 - __clz(c.row);
  const int units = (int)((((int64_t)c.heads * c.row << ps_log2) + COPY_PIECES - 1) / COPY_PIECES);  // of a whole page
  const bool heads_outer = c.head_stride >= c.token_stride;
  const int64_t all = (int64_t)copies * c.n * units;
  for (int64_t u = blockIdx.x; u < all; u += gridDim.x) {
    const int part = (int)(u % units);
    const int64_t x = u / units;
    const int4 job = __ldcg(w.copies + x / c.n);
    uint4* base = c.at[x % c.n];
    const int dst = __ldcg(w.list + job.y), pieces = job.z * c.heads * c.row;
    const uint4* from = base + job.x * c.page_stride;
    uint4* to = base + dst * c.page_stride;
    const int inner = heads_outer ? job.z : c.heads;
    uint4 v[COPY_PIECES / COPY_THREADS];
    int64_t off[COPY_PIECES / COPY_THREADS];
#pragma unroll
    for (int i = 0; i < COPY_PIECES / COPY_THREADS; ++i) {
      const int k = part * COPY_PIECES + i * COPY_THREADS + threadIdx.x;
      off[i] = -1;
      if (k < pieces) {
        const unsigned r = (unsigned)k >> row_log2, o = r / (unsigned)inner, j = r % (unsigned)inner;
        off[i] = (int64_t)o * (heads_outer ? c.head_stride : c.token_stride) +
                 (int64_t)j * (heads_outer ? c.token_stride : c.head_stride) + (k & (c.row - 1));
        v[i] = __ldcs(from + off[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < COPY_PIECES / COPY_THREADS; ++i)
      if (off[i] >= 0) to[off[i]] = v[i];
  }
}

// The rows of the new table, in pieces of a block's threads each.
template <class F>
FL_DEV void for_entries(const PagesDev& a, F f) {
  const int per = (a.W + COPY_THREADS - 1) / COPY_THREADS;
  for (int64_t u = blockIdx.x; u < (int64_t)a.S * per; u += gridDim.x) {
    const int s = (int)(u / per), i = (int)(u % per) * COPY_THREADS + threadIdx.x;
    if (i < a.W) f(s, i);
  }
}

__global__ void __launch_bounds__(COPY_THREADS) fork_kernel(PagesDev a, const int32_t* parents, const int32_t* grow, Ws w,
                                                            const __grid_constant__ Caches c, int* status) {
  pdl_wait();
  pdl_trigger();
  const bool refused = __ldcg(w.head + 1) != 0;
  for_entries(a, [&](int s, int i) {
    const int64_t e = (int64_t)s * a.W + i;
    if (refused) {
      a.table_to[e] = __ldg(a.table + e);
      return;
    }
    const Row r = row_of(a, parents, grow, s, nullptr);
    const int start = r.held - (__ldcg(w.wanted + s) & 1);
    int page = -1;
    if (i >= start && i < r.want) {
      page = __ldcg(w.list + __ldcg(w.first + s) + i - start);
    } else if (i < min(r.held, r.want)) {
      page = __ldg(a.table + (int64_t)r.p * a.W + i);
      if ((unsigned)page >= (unsigned)a.n_pages) atomicOr(status, FL_KV_BAD_PAGE);
    }
    a.table_to[e] = page;
  });
  copy_pages(c, w, a.ps_log2);
}

__global__ void __launch_bounds__(COPY_THREADS) compact_kernel(PagesDev a, const int32_t* moved, Ws w,
                                                               const __grid_constant__ Caches c, int* status) {
  pdl_wait();
  pdl_trigger();
  for_entries(a, [&](int s, int i) {
    const int64_t e = (int64_t)s * a.W + i;
    int page = -1;
    if (i < pages_of(a, len_of(a, s, status))) {
      const int x = __ldg(a.table + e);
      if ((unsigned)x < (unsigned)a.n_pages) page = __ldcg(moved + x);
      if (page < 0) atomicOr(status, FL_KV_BAD_PAGE);
    }
    a.table_to[e] = page;
  });
  copy_pages(c, w, a.ps_log2);
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
    c->at[2 * i] = (uint4*)x.k;
    c->at[2 * i + 1] = (uint4*)x.v;
  }
  c->n = 2 * n;
  c->heads = caches[0].kv_heads;
  c->row = caches[0].head_dim / 8;
  if (((int64_t)c->heads * c->row << a->ps_log2) >= 1ll << 31)
    return fl_internal_error(FL_ERR_CAPACITY, "%s: a page of %d heads", who, c->heads);
  c->page_stride = caches[0].page_stride / 8;
  c->head_stride = caches[0].head_stride / 8;
  c->token_stride = caches[0].token_stride / 8;
  a->lens_to = to->lens;
  a->table_to = to->table;
  a->refs_to = to->refs;
  ws_layout((int32_t*)const_cast<void*>(ws), a->S, a->n_pages, w);
  return FL_OK;
}

template <typename... KArgs, typename... Args>
cudaError_t launch_plan(void (*kern)(KArgs...), int ctas, cudaStream_t st, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // see pdl_wait
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(PLAN_THREADS);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, static_cast<KArgs>(args)...);
}

int plan_ctas(const PagesDev& a) { return (int64_t)a.S * a.W + a.n_pages > 16384 ? MAX_PLAN_CTAS : 1; }

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
  FL_CUDA_TRY(launch_plan(fork_plan_kernel, plan_ctas(a), st, a, parents, new_tokens, w, status));
  FL_CUDA_TRY(fl_launch(fork_kernel, dim3(4 * fl_sm_count()), dim3(COPY_THREADS), 0, st, a, parents, new_tokens, w, c, status));
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
  FL_CUDA_TRY(launch_plan(compact_plan_kernel, plan_ctas(a), st, a, moved, used, w));
  FL_CUDA_TRY(fl_launch(compact_kernel, dim3(4 * fl_sm_count()), dim3(COPY_THREADS), 0, st, a, moved, w, c, status));
  return FL_OK;
}
