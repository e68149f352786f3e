// Beam search: the next beams from every beam's logits, and the hypotheses' tokens from the back-pointers.
//
// Step.  With c(b, v) = score_b + x_bv - lse_b a search wants the best `beams` of beams x vocab candidates.  Within a
// beam c is ordered as x is, so each row needs only its largest logits and its log-sum-exp: one pass over the logits, which
// is the bound (HBM; for few rows the latency of a load, some barriers and the join).  A row is cut into slices, a CTA each,
// which goes through its slice in chunks, the next one's loads in flight.  Of the first chunk the B-th largest of 32 groups of
// threads' maxima bounds the B-th largest logit from below; of what comes later only what exceeds the bound is looked
// at, about B logits for each time that the slice doubles, and the bound is raised from those now and then.  The CTA of a
// search that comes last joins the slices' sums and lists.
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "../../include/flglm_kernels.h"
#include "kv_attention.cuh"
#include "ptx.cuh"

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32, GROUPS = 32, MAX_SLICES = 32;
constexpr int PIECES = 4, CHUNK_PIECES = PIECES * THREADS;  // 16-byte pieces of a thread and of a CTA in a chunk
constexpr int MAX_HITS = 512;
constexpr int MAX_SEARCHES = 16384, MAX_VOCAB = 1 << 19;
constexpr float LOG2E = 1.4426950408889634f;
static_assert(FL_BEAM_MAX <= GROUPS && GROUPS == 32 && FL_BEAM_MAX == 2 * WARPS);

struct Cand {  // a token and its logit
  float x;
  int v;
};
FL_DEV bool better(const Cand& a, const Cand& b) { return a.x > b.x || (a.x == b.x && a.v < b.v); }

struct StepArgs {
  fl_beam_search p;
  fl_beam_state from, to;
  const void* x;
  int64_t ld;
  int slices, per;  // slices of a row, 16-byte pieces of a slice
  int32_t *trace_tokens, *trace_parents, *tokens, *parents;
  unsigned* counters;
  float2* sums;  // [row][slice] (largest logit, sum of exp(x - it))
  Cand* lists;   // [row][slice][beam], best first; x = -inf: none
  int* status;
};

template <class T>
struct Piece;  // 16 bytes of logits
template <>
struct Piece<float> {
  static constexpr int N = 4;
  static constexpr uint32_t NONE = 0xff800000u;  // -inf
  FL_DEV static void get(const uint4& u, float (&f)[4]) {
    f[0] = __uint_as_float(u.x), f[1] = __uint_as_float(u.y), f[2] = __uint_as_float(u.z), f[3] = __uint_as_float(u.w);
  }
  FL_DEV static uint32_t max2(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }
  FL_DEV static float top(uint32_t a) { return __uint_as_float(a); }
  FL_DEV static uint4 without(const uint4& u, int e) {
    return make_uint4(e == 0 ? NONE : u.x, e == 1 ? NONE : u.y, e == 2 ? NONE : u.z, e == 3 ? NONE : u.w);
  }
};
template <class T, uint32_t INF2>
struct Piece16 {
  static constexpr int N = 8;
  static constexpr uint32_t NONE = INF2;
  FL_DEV static void get(const uint4& u, float (&f)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 y = KvIo<T>::unpack(w[i]);
      f[2 * i] = y.x, f[2 * i + 1] = y.y;
    }
  }
  FL_DEV static float top(uint32_t a) {
    const float2 y = KvIo<T>::unpack(a);
    return fmaxf(y.x, y.y);
  }
  FL_DEV static uint4 without(const uint4& u, int e) {
    const uint32_t m = e & 1 ? 0xffff0000u : 0xffffu, x = INF2 & m;
    return make_uint4(e >> 1 == 0 ? (u.x & ~m) | x : u.x, e >> 1 == 1 ? (u.y & ~m) | x : u.y, e >> 1 == 2 ? (u.z & ~m) | x : u.z,
                      e >> 1 == 3 ? (u.w & ~m) | x : u.w);
  }
};
template <>
struct Piece<__nv_bfloat16> : Piece16<__nv_bfloat16, 0xff80ff80u> {
  FL_DEV static uint32_t max2(uint32_t a, uint32_t b) {
    const __nv_bfloat162 y = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&y);
  }
};
template <>
struct Piece<__half> : Piece16<__half, 0xfc00fc00u> {
  FL_DEV static uint32_t max2(uint32_t a, uint32_t b) {
    const __half2 y = __hmax2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&y);
  }
};

// Whole numbers in the order of the floats (no NaN); 0 is below all of them.
FL_DEV uint32_t order32(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}
FL_DEV uint64_t order64(double x) {
  const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);
  return u >> 63 ? ~u : u | (1ull << 63);
}

// Two floats as one operand of the packed fp32 instructions.
FL_DEV uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
FL_DEV float2 unpack2(uint64_t x) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
  return r;
}
FL_DEV uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
FL_DEV uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// sum of exp(x - ref) over what a thread has seen.  x - ref is taken before the product with log2(e): rounding the product of x itself
// would be off by the same for every x near ref.
struct Sum {
  float ref = -INFINITY;
  uint64_t minus = 0, sum = 0;  // (-ref, -ref), or zeros where there is no ref yet; sums of every other element
  FL_DEV void add(float x, float y) {
    const float2 u = unpack2(mul2(add2(pack2(x, y), minus), pack2(LOG2E, LOG2E)));
    sum = add2(sum, pack2(exp2_hw(u.x), exp2_hw(u.y)));
  }
  FL_DEV float total() const { return unpack2(sum).x + unpack2(sum).y; }
  // room for x: sums of up to 2^19 exponentials of 16 and less are far from overflow
  FL_DEV void see(float x) {
    if (x > ref + 16.f) {
      const float f = ref == -INFINITY ? 1.f : exp2_hw((ref - x) * LOG2E);  // (1: nothing so far, or a NaN that stays)
      sum = mul2(sum, pack2(f, f));
      ref = x;
      minus = pack2(-x, -x);
    }
  }
};

struct Join {  // shared memory of the CTA that joins a search
  Cand lists[WARPS][MAX_SLICES * FL_BEAM_MAX];
  Cand best[FL_BEAM_MAX][FL_BEAM_MAX];
  uint64_t c[FL_BEAM_MAX][FL_BEAM_MAX];  // candidates of each beam, in order64; 0: none
  uint64_t few[FL_BEAM_MAX * FL_BEAM_MAX];
  int few_at[FL_BEAM_MAX * FL_BEAM_MAX], few_n;
  double live[FL_BEAM_MAX], ends[FL_BEAM_MAX], base[FL_BEAM_MAX], length;
  float m[FL_BEAM_MAX], end_x[FL_BEAM_MAX], pool[2 * FL_BEAM_MAX];
  int pool_step[2 * FL_BEAM_MAX], pool_beam[2 * FL_BEAM_MAX], end_rank[FL_BEAM_MAX];
  int token[FL_BEAM_MAX], parent[FL_BEAM_MAX];
};

// A search that stays as it is.
FL_DEV void rest(const StepArgs& a, int s) {
  const int B = a.p.beams, b = threadIdx.x;
  if (b == 0) {
    const int steps = a.from.steps[s], done = a.from.done[s];
    a.to.steps[s] = steps;
    a.to.done[s] = done;
  }
  if (b < B) {
    const int i = s * B + b;
    const float sc = a.from.scores[i], es = a.from.end_scores[i];
    const int et = a.from.end_steps[i], eb = a.from.end_beams[i];
    a.to.scores[i] = sc, a.to.end_scores[i] = es;
    a.to.end_steps[i] = et, a.to.end_beams[i] = eb;
    a.tokens[i] = max(a.p.eos, 0);
    a.parents[i] = -1;
  }
}

template <class T>
FL_DEV void join(const StepArgs& a, int s, int t, Join& j) {
  const int B = a.p.beams, P = a.slices, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == THREADS - 1) {
    j.length = pow((double)(t + 1), a.p.length_penalty);
    j.few_n = 0;
  }
  // each row's sum and best tokens, a warp a row
  for (int b = warp; b < B; b += WARPS) {
    const int row = s * B + b;
    const float score = a.from.scores[row];
    const bool reads = score > -INFINITY && score < INFINITY;
    float m = -INFINITY, sum = 0.f, e = -INFINITY;
    Cand* mine = j.lists[warp];
    if (reads) {
      const float2 part = lane < P ? __ldcg(a.sums + (int64_t)row * P + lane) : make_float2(-INFINITY, 0.f);
      for (int i = lane; i < P * B; i += 32) {
        const float2 y = __ldcg(reinterpret_cast<const float2*>(a.lists + (int64_t)row * P * B) + i);
        mine[i] = Cand{y.x, __float_as_int(y.y)};
      }
      if (a.p.eos >= 0) {
        float f[Piece<T>::N];
        Piece<T>::get(*reinterpret_cast<const uint4*>((const T*)a.x + (int64_t)row * a.ld + a.p.eos / Piece<T>::N * Piece<T>::N), f);
#pragma unroll
        for (int i = 0; i < Piece<T>::N; ++i) e = i == a.p.eos % Piece<T>::N ? f[i] : e;
      }
      m = part.x;
#pragma unroll
      for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
      sum = part.x == -INFINITY ? part.y : part.y * exp2_hw((part.x - m) * LOG2E);
      if (part.x == INFINITY) sum = NAN;
#pragma unroll
      for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    }
    const bool bad = score != score || score == INFINITY || sum != sum, live = reads && !bad && m > -INFINITY;
    if (bad && lane == 0) atomicOr(a.status, FL_BEAM_BAD_LOGITS);
    __syncwarp();
    int at = lane * B, k = 0;
    if (live) {
      const int stop = lane < P ? at + B : at;
      for (; k < B; ++k) {
        const Cand head = at < stop ? mine[at] : Cand{-INFINITY, 0};
        const uint32_t key = head.x > -INFINITY ? order32(head.x) : 0u, top = __reduce_max_sync(0xffffffffu, key);
        if (top == 0) break;
        const int v = __reduce_min_sync(0xffffffffu, key == top ? head.v : 0x7fffffff);
        if (key == top && head.v == v) {
          j.best[b][k] = head;
          ++at;
        }
      }
    }
    __syncwarp();
    if (lane >= k && lane < B) j.best[b][lane] = Cand{-INFINITY, 0};
    if (lane == 0) {
      // c = score + ((x - m) - log(sum)): exact for the smallest logits that a type has, too
      j.base[b] = live ? log((double)sum) : 0;
      j.m[b] = m;
      j.end_x[b] = live ? e : -INFINITY;
      j.token[b] = max(a.p.eos, 0);
      j.parent[b] = -1;
      j.live[b] = -INFINITY;
    }
  }
  __syncthreads();
  for (int i = tid; i < B * B + B; i += THREADS) {
    const int b = i < B * B ? i / B : i - B * B, k = i % B;
    const float x = i < B * B ? j.best[b][k].x : j.end_x[b];
    const double c = x > -INFINITY ? (double)a.from.scores[s * B + b] + (((double)x - j.m[b]) - j.base[b]) : -INFINITY;
    if (i < B * B) j.c[b][k] = x > -INFINITY ? order64(c) : 0;
    else j.ends[b] = c;
  }
  __syncthreads();
  // A row's last candidate bounds the search's last: only what reaches the best of those bounds is ranked, by counting who comes
  // before: by c, then the lower beam, then the order within the beam.
  uint64_t bound = 1;
  for (int b = 0; b < B; ++b) bound = max(bound, j.c[b][B - 1]);
  for (int i = tid; i < B * B; i += THREADS) {
    const uint64_t c = j.c[i / B][i % B];
    if (c >= bound) {
      const int n = atomicAdd(&j.few_n, 1);
      j.few[n] = c;
      j.few_at[n] = i;
    }
  }
  __syncthreads();
  const int n = j.few_n;
  for (int i = tid; i < n; i += THREADS) {
    const uint64_t c = j.few[i];
    const int at = j.few_at[i];
    int rank = 0;
    for (int o = 0; o < n; ++o) rank += j.few[o] > c || (j.few[o] == c && j.few_at[o] < at);
    if (rank < B) {
      const int b = at / B, k = at % B;
      const Cand y = j.best[b][k];
      j.token[rank] = y.v;
      j.parent[rank] = b;
      j.live[rank] = (double)a.from.scores[s * B + b] + (((double)y.x - j.m[b]) - j.base[b]);
    }
  }
  const int b = tid - (THREADS - 32);  // the hypotheses that end
  if (b >= 0 && b < B) {
    const double x = j.ends[b];
    const uint64_t c = x > -INFINITY ? order64(x) : 0;
    int rank = -1;
    if (c >= bound) {
      const Cand e{j.end_x[b], a.p.eos};
      rank = 0;
      for (int o = 0; o < n; ++o) {
        const int ob = j.few_at[o] / B;
        rank += ob == b ? better(j.best[ob][j.few_at[o] % B], e) : j.few[o] > c || (j.few[o] == c && ob < b);
      }
      for (int o = 0; o < B; ++o) {
        const uint64_t y = j.ends[o] > -INFINITY ? order64(j.ends[o]) : 0;
        rank += y > c || (y == c && o < b);
      }
      if (rank >= B) rank = -1;
    }
    j.end_rank[b] = rank;
  }
  __syncthreads();
  // the pool: what had ended, then what ends now in the order of its rank
  if (warp == 0) {
    const int pb = lane < FL_BEAM_MAX ? lane : lane - FL_BEAM_MAX;
    float x = -INFINITY;
    int step = 0, beam = 0, order = lane;
    if (pb < B) {
      if (lane < FL_BEAM_MAX) {
        x = a.from.end_scores[s * B + pb];
        step = a.from.end_steps[s * B + pb];
        beam = a.from.end_beams[s * B + pb];
      } else if (j.end_rank[pb] >= 0) {
        x = (float)(j.ends[pb] / j.length);
        step = t;
        beam = pb;
        order = FL_BEAM_MAX + j.end_rank[pb];
      }
    }
    if (!(x > -INFINITY)) x = -INFINITY, step = beam = 0;
    const uint64_t key = (uint64_t)order32(x) << 32 | (uint32_t)((63 - order) << 8 | (31 - lane));
    int rank = 0;
#pragma unroll 4
    for (int o = 0; o < 32; ++o) rank += __shfl_sync(0xffffffffu, key, o) > key;
    if (pb < B && rank < B) {  // (the places behind the pool's end are empty ones')
      j.pool[rank] = x;
      j.pool_step[rank] = step;
      j.pool_beam[rank] = beam;
    }
    __syncwarp();
    if (lane < B) {
      const int i = s * B + lane;
      const int64_t tr = ((int64_t)s * a.p.max_steps + t) * B + lane;
      a.to.scores[i] = (float)j.live[lane];
      a.to.end_scores[i] = j.pool[lane];
      a.to.end_steps[i] = j.pool_step[lane];
      a.to.end_beams[i] = j.pool_beam[lane];
      a.tokens[i] = a.trace_tokens[tr] = j.token[lane];
      a.trace_parents[tr] = j.parent[lane] < 0 ? lane : j.parent[lane];
      a.parents[i] = j.parent[lane] < 0 ? -1 : s * B + j.parent[lane];
    }
    if (lane == 0) {
      const float worst = j.pool[B - 1];
      const bool over = worst > -INFINITY && (a.p.early || worst >= (float)(j.live[0] / j.length));
      a.to.steps[s] = t + 1;
      a.to.done[s] = over || !(j.live[0] > -INFINITY);
    }
  }
}

template <class T>
__global__ void __launch_bounds__(THREADS, 3) beam_step_kernel(StepArgs a) {
  pdl_wait();
  pdl_trigger();
  using Io = Piece<T>;
  constexpr int N = Io::N;
  __shared__ float sh_group[GROUPS], sh_ref[WARPS], sh_sum[WARPS];
  __shared__ Cand sh_hits[2][MAX_HITS];
  __shared__ int sh_count[2], sh_last;
  extern __shared__ __align__(16) char sh_join[];
  const int B = a.p.beams, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int slice = blockIdx.x % (unsigned)a.slices, row = blockIdx.x / (unsigned)a.slices, s = row / B;
  const int all = (a.p.vocab + N - 1) / N, begin = slice * a.per, end = min(all, begin + a.per);
  const uint4* x = reinterpret_cast<const uint4*>((const T*)a.x + (int64_t)row * a.ld);
  uint4 cur[PIECES];
  auto load = [&](int first, uint4 (&u)[PIECES]) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int k = first + i * THREADS + tid;
      u[i] = k < end ? __ldcs(x + k) : make_uint4(Io::NONE, Io::NONE, Io::NONE, Io::NONE);
    }
  };
  load(begin, cur);  // before it is known whether the beam is live: one latency less
  const int t = a.from.steps[s];  // (no read-only loads of the state: `to` may be the same memory)
  const bool active = a.from.done[s] == 0 && t >= 0 && t < a.p.max_steps;
  const float score = a.from.scores[row];
  if (active && score > -INFINITY && score < INFINITY) {
    Sum z;
    float bound = -INFINITY;
    int side = 0, since = begin, kept = 0;  // the list in use; the first piece that came after it was ranked, what it had then
    if (tid == 0) sh_count[0] = 0;
    for (int first = begin, chunk = 0; first < end; first += CHUNK_PIECES, ++chunk) {
      uint4 next[PIECES];
      const bool last = first + CHUNK_PIECES >= end;
      if (!last) load(first + CHUNK_PIECES, next);
      // tokens behind the vocabulary; the eos, which is summed but no candidate to go on with
      const int lo = first * N, hi = (first + CHUNK_PIECES) * N;
      if (hi > a.p.vocab || (a.p.eos >= lo && a.p.eos < hi)) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
          const int v = (first + i * THREADS + tid) * N;
          if (a.p.eos >= v && a.p.eos < v + N) {
            float f[N], e = -INFINITY;
            Io::get(cur[i], f);
#pragma unroll
            for (int k = 0; k < N; ++k) e = k == a.p.eos - v ? f[k] : e;
            z.see(e);
            z.add(e, -INFINITY);
            cur[i] = Io::without(cur[i], a.p.eos - v);
          }
          if (v < a.p.vocab && v + N > a.p.vocab)
            for (int k = a.p.vocab - v; k < N; ++k) cur[i] = Io::without(cur[i], k);
        }
      }
      uint32_t most = Io::NONE;
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
        most = Io::max2(most, Io::max2(Io::max2(cur[i].x, cur[i].y), Io::max2(cur[i].z, cur[i].w)));
      const float top = Io::top(most);
      bool look = top > bound;
      if (chunk == 0) {
        float g = top;
#pragma unroll
        for (int d = 1; d < THREADS / GROUPS; d <<= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, d));
        if (tid % (THREADS / GROUPS) == 0) sh_group[tid / (THREADS / GROUPS)] = g;
        __syncthreads();
        // the B-th largest of the groups' maxima, and the largest
        g = sh_group[lane];
        int rank = 0;
#pragma unroll
        for (int o = 0; o < GROUPS; ++o) {
          const float y = sh_group[o];
          rank += y > g || (y == g && o < lane);
        }
        bound = __shfl_sync(0xffffffffu, g, __ffs(__ballot_sync(0xffffffffu, rank == B - 1)) - 1);
        z.see(__shfl_sync(0xffffffffu, g, __ffs(__ballot_sync(0xffffffffu, rank == 0)) - 1));
        look = top >= bound && top > -INFINITY;
      } else if (look) {
        z.see(top);
      }
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        float f[N];
        Io::get(cur[i], f);
#pragma unroll
        for (int k = 0; k < N; k += 2) z.add(f[k], f[k + 1]);
      }
      if (look) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
          float f[N];
          Io::get(cur[i], f);
#pragma unroll
          for (int k = 0; k < N; ++k)
            if (f[k] > bound || (chunk == 0 && f[k] == bound && f[k] > -INFINITY)) {
              const int n = atomicAdd(&sh_count[side], 1);
              if (n < MAX_HITS) sh_hits[side][n] = Cand{f[k], (first + i * THREADS + tid) * N + k};
            }
        }
      }
      if (last || chunk == 3 || chunk == 15) {
        // the best so far, ranked by counting, raise the bound
        __syncthreads();
        const int n = sh_count[side];
        Cand* to = sh_hits[side ^ 1];
        if (tid == 0) sh_count[side ^ 1] = min(n, B);
        if (n <= MAX_HITS) {
          for (int i = tid; i < n; i += THREADS) {
            const Cand mine = sh_hits[side][i];
            int r = 0;
            for (int o = 0; o < n; ++o) r += better(sh_hits[side][o], mine);
            if (r < B) to[r] = mine;
          }
        } else {
          // more than the list holds (logits that ascend, many equal ones): the best one behind the last found, B times
          Cand found{INFINITY, -1};
          for (int r = 0; r < B; ++r) {
            Cand mine{-INFINITY, 0x7fffffff};
            if (tid < kept && better(found, sh_hits[side][tid])) mine = sh_hits[side][tid];
            for (int k = since + tid; k < min(end, first + CHUNK_PIECES); k += THREADS) {
              float f[N];
              Io::get(x[k], f);
              for (int e = 0; e < N; ++e) {
                const Cand y{f[e], k * N + e};
                if (y.v < a.p.vocab && y.v != a.p.eos && better(found, y) && better(y, mine)) mine = y;
              }
            }
#pragma unroll
            for (int d = 16; d; d >>= 1) {
              const Cand o{__shfl_xor_sync(0xffffffffu, mine.x, d), __shfl_xor_sync(0xffffffffu, mine.v, d)};
              if (better(o, mine)) mine = o;
            }
            if (lane == 0) to[MAX_HITS - WARPS + warp] = mine;
            __syncthreads();
            for (int i = 0; i < WARPS; ++i)
              if (better(to[MAX_HITS - WARPS + i], mine)) mine = to[MAX_HITS - WARPS + i];
            __syncthreads();
            if (tid == 0) to[r] = mine;
            found = mine;
          }
        }
        __syncthreads();
        side ^= 1;
        since = first + CHUNK_PIECES;
        kept = min(n, B);
        if (n >= B) bound = to[B - 1].x;
        if (n > 0) z.see(to[0].x);
      }
      if (!last)
#pragma unroll
        for (int i = 0; i < PIECES; ++i) cur[i] = next[i];
    }
    // the slice's sum and list
    float ref = z.ref;
#pragma unroll
    for (int d = 16; d; d >>= 1) ref = fmaxf(ref, __shfl_xor_sync(0xffffffffu, ref, d));
    float sum = z.ref == -INFINITY ? z.total() : z.total() * exp2_hw((z.ref - ref) * LOG2E);
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (lane == 0) sh_ref[warp] = ref, sh_sum[warp] = sum;
    if (tid < B) a.lists[(int64_t)blockIdx.x * B + tid] = tid < sh_count[side] ? sh_hits[side][tid] : Cand{-INFINITY, 0};
    __syncthreads();
    if (tid == 0) {
      float m = sh_ref[0], q = 0.f;
      for (int i = 1; i < WARPS; ++i) m = fmaxf(m, sh_ref[i]);
      for (int i = 0; i < WARPS; ++i) q += sh_ref[i] == -INFINITY ? sh_sum[i] : sh_sum[i] * exp2_hw((sh_ref[i] - m) * LOG2E);
      a.sums[blockIdx.x] = make_float2(m, q);
    }
  }
  __syncthreads();
  if (tid == 0) sh_last = kv_part_done(a.counters + s, (unsigned)(B * a.slices));
  __syncthreads();
  if (!sh_last) return;
  if (active)
    join<T>(a, s, t, *reinterpret_cast<Join*>(sh_join));
  else
    rest(a, s);
}

int64_t part_bytes(const fl_beam_search* p, int slices) {
  return (int64_t)p->n_seqs * p->beams * slices * (sizeof(float2) + p->beams * sizeof(Cand));
}

const char* search_problem(const fl_beam_search* p, int* code) {
  *code = FL_ERR_INVALID_ARG;
  if (!p || p->n_seqs < 0 || p->beams < 1 || p->vocab < 1 || p->max_steps < 1 || p->eos < -1 || p->eos >= p->vocab ||
      (p->early != 0 && p->early != 1) || !std::isfinite(p->length_penalty))
    return "search";
  *code = FL_ERR_CAPACITY;
  if (p->beams > FL_BEAM_MAX) return "more than 16 beams";
  if (p->n_seqs > MAX_SEARCHES) return "more than 16384 searches";
  if (p->vocab > MAX_VOCAB) return "more than 2^19 tokens";
  if (p->max_steps > (1 << 24)) return "more than 2^24 steps";
  return nullptr;
}
bool state_ok(const fl_beam_state* s) {
  const void* at[6] = {s->scores, s->steps, s->done, s->end_scores, s->end_steps, s->end_beams};
  for (int i = 0; i < 6; ++i) {
    if (!at[i] || fl_misaligned(at[i], 4)) return false;
    for (int k = 0; k < i; ++k)
      if (at[i] == at[k]) return false;
  }
  return true;
}

// Slices of a row: enough for some CTAs per SM and wave, of a thread's piece at least.
template <class T>
int launch_step(StepArgs& a, cudaStream_t st) {
  constexpr int N = Piece<T>::N;
  const int pieces = (a.p.vocab + N - 1) / N;
  const int64_t rows = (int64_t)a.p.n_seqs * a.p.beams;
  const int64_t want = (16 * fl_sm_count() + rows - 1) / rows, most = (pieces + THREADS - 1) / THREADS;
  const int slices = (int)std::min<int64_t>(std::min<int64_t>(want, most), MAX_SLICES);
  a.per = (pieces + slices - 1) / slices;
  a.slices = (pieces + a.per - 1) / a.per;
  auto kern = beam_step_kernel<T>;
  FL_CUDA_TRY(fl_func_smem((const void*)kern, sizeof(Join)));
  FL_CUDA_TRY(fl_launch(kern, dim3((unsigned)(rows * a.slices)), dim3(THREADS), sizeof(Join), st, a));
  return FL_OK;
}

// ------------------------------------------------------------------------------- back-pointers
constexpr int TRACE_THREADS = 512, CHUNK = 32, BLOCK_STEPS = 2048;

struct TraceArgs {
  fl_beam_search p;
  fl_beam_state s;
  const int32_t *tokens, *parents;
  int n_best, pad;
  int32_t *out_tokens, *out_lens;
  float* out_scores;
  int* status;
};

// Beams after each step, from the last step to the first: b(t - 1) = parent[t][b(t)].  Following one pointer after
// another costs a load's latency a step; here each chunk of 32 steps becomes one map from the beams behind it to
// those before it, all chunks at once from shared memory, the hypotheses jump from chunk to chunk, and then all chunks
// are walked at once for the beams in between.
__global__ void __launch_bounds__(TRACE_THREADS) beam_trace_kernel(TraceArgs a) {
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) uint8_t sh[];
  const int B = a.p.beams, T = a.p.max_steps, n = a.n_best, s = blockIdx.x, tid = threadIdx.x;
  const int room = min(T, BLOCK_STEPS), chunks = (room + CHUNK - 1) / CHUNK;
  uint8_t* par = sh;                       // [step][beam]
  uint8_t* map = par + room * B;           // [chunk][beam]
  uint8_t* entry = map + chunks * B;       // [chunk][hypothesis]: its beam after the chunk's last step that it has
  uint8_t* chain = entry + chunks * n;     // [hypothesis][step]
  __shared__ int h_steps[FL_BEAM_MAX], h_ended[FL_BEAM_MAX], h_beam[FL_BEAM_MAX];
  if (tid < 32) {
    const int b = tid < FL_BEAM_MAX ? tid : tid - FL_BEAM_MAX;
    const int raw = a.s.steps[s], steps = min(max(raw, 0), T);
    bool bad = raw != steps;
    float x = -INFINITY;
    int before = 0, beam = 0;
    if (b < B) {
      if (tid < FL_BEAM_MAX) {
        x = a.s.end_scores[s * B + b];
        before = a.s.end_steps[s * B + b];
        beam = a.s.end_beams[s * B + b];
        if (x > -INFINITY) bad |= (unsigned)before >= (unsigned)T || (unsigned)beam >= (unsigned)B;
        if ((unsigned)before >= (unsigned)T) before = 0;
        if ((unsigned)beam >= (unsigned)B) beam = 0;
      } else if (a.s.done[s] == 0 && steps > 0) {
        x = (float)((double)a.s.scores[s * B + b] / pow((double)steps, a.p.length_penalty));
        before = steps;
        beam = b;
      }
    }
    if (!(x == x)) x = -INFINITY;
    if (bad) atomicOr(a.status, FL_BEAM_BAD_TRACE);
    int rank = 0;
    for (int o = 0; o < 32; ++o) {
      const float y = __shfl_sync(0xffffffffu, x, o);
      rank += y > x || (y == x && o < tid);
    }
    if (rank < n) {
      const bool some = x > -INFINITY;
      h_steps[rank] = some ? before : 0;
      h_ended[rank] = some && tid < FL_BEAM_MAX;
      h_beam[rank] = beam;
      a.out_scores[s * n + rank] = x;
      a.out_lens[s * n + rank] = some ? before + (tid < FL_BEAM_MAX) : 0;
    }
  }
  __syncthreads();
  for (int t1 = T; t1 > 0;) {
    const int t0 = (t1 - 1) / BLOCK_STEPS * BLOCK_STEPS, len = t1 - t0, nc = (len + CHUNK - 1) / CHUNK;
    const int64_t first = ((int64_t)s * T + t0) * B;
    int longest = 0;
    for (int h = 0; h < n; ++h) longest = max(longest, h_steps[h]);
    const int have = min(max(longest - t0, 0), len);  // steps that some hypothesis has
    for (int i = tid; i < have * B; i += TRACE_THREADS) {
      int p = __ldg(a.parents + first + i);
      if ((unsigned)p >= (unsigned)B) {
        atomicOr(a.status, FL_BEAM_BAD_TRACE);
        p = 0;
      }
      par[i] = (uint8_t)p;
    }
    __syncthreads();
    for (int i = tid; i < nc * B; i += TRACE_THREADS) {
      const int c = i / B, lo = c * CHUNK, hi = min(lo + CHUNK, have);
      int b = i % B;
      for (int t = hi - 1; t >= lo; --t) b = par[t * B + b];
      map[i] = (uint8_t)b;
    }
    __syncthreads();
    if (tid < n) {
      int b = h_beam[tid];
      const int mine = min(max(h_steps[tid] - t0, 0), len);  // its steps in this block
      for (int c = nc - 1; c >= 0; --c) {
        const int lo = c * CHUNK;
        entry[c * n + tid] = (uint8_t)b;
        if (mine <= lo) continue;
        if (mine >= min(lo + CHUNK, have))
          b = map[c * B + b];
        else
          for (int t = mine - 1; t >= lo; --t) b = par[t * B + b];
      }
      h_beam[tid] = b;
    }
    __syncthreads();
    for (int i = tid; i < nc * n; i += TRACE_THREADS) {
      const int c = i / n, h = i % n, lo = c * CHUNK;
      int b = entry[i];
      for (int t = min(lo + CHUNK, min(h_steps[h] - t0, len)) - 1; t >= lo; --t) {
        chain[h * room + t] = (uint8_t)b;
        b = par[t * B + b];
      }
    }
    __syncthreads();
    for (int h = 0; h < n; ++h) {
      int32_t* out = a.out_tokens + ((int64_t)s * n + h) * T + t0;
      const int mine = h_steps[h] - t0;
      for (int t = tid; t < len; t += TRACE_THREADS) {
        int v = a.pad;
        if (t < mine) v = __ldg(a.tokens + first + (int64_t)t * B + chain[h * room + t]);
        else if (t == mine && h_ended[h] && a.p.eos >= 0) v = a.p.eos;
        out[t] = v;
      }
    }
    __syncthreads();
    t1 = t0;
  }
}

}  // namespace

extern "C" size_t fl_k_beam_workspace(const fl_beam_search* search) {
  int code;
  if (const char* w = search_problem(search, &code)) {
    fl_internal_error(code, "beam workspace: %s", w);
    return 0;
  }
  return MAX_SEARCHES * sizeof(unsigned) + part_bytes(search, MAX_SLICES);
}

extern "C" int fl_k_beam_step(const fl_beam_search* search, const fl_beam_state* from, const fl_beam_state* to,
                              int32_t dtype, const void* logits, int64_t ld, int32_t* trace_tokens, int32_t* trace_parents,
                              int32_t* tokens, int32_t* parents, void* workspace, int* status, void* stream) {
  int code;
  if (const char* w = search_problem(search, &code)) return fl_internal_error(code, "beam step: %s", w);
  if (dtype != FL_DT_F32 && dtype != FL_DT_BF16 && dtype != FL_DT_F16)
    return fl_internal_error(FL_ERR_INVALID_ARG, "beam step: dtype %d", dtype);
  if (search->n_seqs == 0) return FL_OK;
  if (!from || !to || !state_ok(from) || !state_ok(to)) return fl_internal_error(FL_ERR_INVALID_ARG, "beam step: state");
  const void *f[6] = {from->scores, from->steps, from->done, from->end_scores, from->end_steps, from->end_beams};
  const void *t[6] = {to->scores, to->steps, to->done, to->end_scores, to->end_steps, to->end_beams};
  int same = 0;
  for (int i = 0; i < 6; ++i)
    for (int k = 0; k < 6; ++k)
      if (f[i] == t[k]) same += i == k ? 1 : 100;
  if (same != 0 && same != 6)
    return fl_internal_error(FL_ERR_INVALID_ARG, "beam step: `to` is neither `from` nor apart from it");
  if (!logits || !trace_tokens || !trace_parents || !tokens || !parents || !workspace || !status ||
      fl_misaligned(logits, 16) || fl_misaligned(trace_tokens, 4) || fl_misaligned(trace_parents, 4) ||
      fl_misaligned(tokens, 4) || fl_misaligned(parents, 4) || fl_misaligned(workspace, 16) || fl_misaligned(status, 4))
    return fl_internal_error(FL_ERR_INVALID_ARG, "beam step: args");
  if (ld < search->vocab || ld % (dtype == FL_DT_F32 ? 4 : 8))
    return fl_internal_error(FL_ERR_UNSUPPORTED, "beam step: row stride %lld (a multiple of 16 bytes, vocab or more)", (long long)ld);
  StepArgs a{*search, *from, *to, logits, ld, 0, 0, trace_tokens, trace_parents, tokens, parents, (unsigned*)workspace,
             nullptr, nullptr, status};
  a.sums = (float2*)((char*)workspace + MAX_SEARCHES * sizeof(unsigned));
  a.lists = (Cand*)(a.sums + (int64_t)search->n_seqs * search->beams * MAX_SLICES);
  const cudaStream_t st = (cudaStream_t)stream;
  return dtype == FL_DT_F32 ? launch_step<float>(a, st)
                            : dtype == FL_DT_F16 ? launch_step<__half>(a, st) : launch_step<__nv_bfloat16>(a, st);
}

extern "C" int fl_k_beam_trace(const fl_beam_search* search, const fl_beam_state* state, const int32_t* trace_tokens,
                               const int32_t* trace_parents, int32_t n_best, int32_t pad, int32_t* out_tokens,
                               int32_t* out_lens, float* out_scores, int* status, void* stream) {
  int code;
  if (const char* w = search_problem(search, &code)) return fl_internal_error(code, "beam trace: %s", w);
  if (n_best < 1 || n_best > search->beams) return fl_internal_error(FL_ERR_INVALID_ARG, "beam trace: n_best %d", n_best);
  if (search->n_seqs == 0) return FL_OK;
  if (!state || !state_ok(state) || !trace_tokens || !trace_parents || !out_tokens || !out_lens || !out_scores || !status ||
      fl_misaligned(trace_tokens, 4) || fl_misaligned(trace_parents, 4) || fl_misaligned(out_tokens, 4) ||
      fl_misaligned(out_lens, 4) || fl_misaligned(out_scores, 4) || fl_misaligned(status, 4))
    return fl_internal_error(FL_ERR_INVALID_ARG, "beam trace: args");
  const TraceArgs a{*search, *state, trace_tokens, trace_parents, n_best, pad, out_tokens, out_lens, out_scores, status};
  const int room = search->max_steps < BLOCK_STEPS ? search->max_steps : BLOCK_STEPS, chunks = (room + CHUNK - 1) / CHUNK;
  const int smem = (room + chunks) * (search->beams + n_best);
  // the limit of the largest call, once: a smaller one would lower it for a larger call made before
  FL_CUDA_TRY(fl_func_smem((const void*)beam_trace_kernel, (BLOCK_STEPS + BLOCK_STEPS / CHUNK) * 2 * FL_BEAM_MAX));
  FL_CUDA_TRY(fl_launch(beam_trace_kernel, dim3(search->n_seqs), dim3(TRACE_THREADS), smem, (cudaStream_t)stream, a));
  return FL_OK;
}
