// Beam search: the next beams from every beam's logits, and the hypotheses' tokens from the back-pointers.
//
// Step.  With c(b, v) = score_b + x_bv - lse_b a search wants the best `beams` of beams x vocab candidates.  Within a
// beam c is ordered as x is, so each row needs only its largest logits and its log-sum-exp: one pass over the logits, which
// is the bound (HBM; for few rows the latency of a load and two barriers).  A row is cut into slices, a CTA each, which
// keeps its slice in registers: the maximum of each of 32 groups of threads is taken, and the B-th largest of those bounds
// the slice's B-th largest logit from below, since B groups hold one that large each.  About B logits reach the
// bound; they are ranked by counting.  The CTA of a search that comes last joins the slices' sums and lists.
#include <cuda_fp16.h>

#include <cmath>

#include "../../include/flglm_kernels.h"
#include "kv_attention.cuh"
#include "ptx.cuh"

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32, GROUPS = 32, MAX_SLICES = 32, MAX_HITS = THREADS;
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
  FL_DEV static void get(const uint4& u, float* f) {
    f[0] = __uint_as_float(u.x), f[1] = __uint_as_float(u.y), f[2] = __uint_as_float(u.z), f[3] = __uint_as_float(u.w);
  }
};
template <class T>
struct Piece16 {
  static constexpr int N = 8;
  FL_DEV static void get(const uint4& u, float* f) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 y = KvIo<T>::unpack(w[i]);
      f[2 * i] = y.x, f[2 * i + 1] = y.y;
    }
  }
};
template <>
struct Piece<__nv_bfloat16> : Piece16<__nv_bfloat16> {};
template <>
struct Piece<__half> : Piece16<__half> {};

struct Join {  // shared memory of the CTA that joins a search
  Cand lists[WARPS][MAX_SLICES * FL_BEAM_MAX];
  Cand best[FL_BEAM_MAX][FL_BEAM_MAX];
  double c[FL_BEAM_MAX][FL_BEAM_MAX];  // -inf: no candidate
  double ends[FL_BEAM_MAX], live[FL_BEAM_MAX];
  float end_x[FL_BEAM_MAX], pool[2 * FL_BEAM_MAX];
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
  const int B = a.p.beams, P = a.slices, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // each row's sum and best tokens, a warp a row
  for (int b = warp; b < B; b += WARPS) {
    const int row = s * B + b;
    const float score = a.from.scores[row];
    double m = -INFINITY, sum = 0;
    const bool reads = score > -INFINITY && score < INFINITY;
    if (reads) {
      const float2 mine = lane < P ? __ldcg(a.sums + (int64_t)row * P + lane) : make_float2(-INFINITY, 0.f);
      float top = mine.x;
#pragma unroll
      for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      sum = mine.x == -INFINITY ? (double)mine.y : mine.y * exp((double)mine.x - top);
      if (mine.x == INFINITY) sum = NAN;
#pragma unroll
      for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      m = top;
    }
    // x - lse as (x - m) - log(sum): exact for the smallest logits that a type has, too
    const double part = log(sum);
    const bool bad = score != score || score == INFINITY || (reads && !(m + part < INFINITY));
    const bool live = reads && !bad && m > -INFINITY;
    if (bad && lane == 0) atomicOr(a.status, FL_BEAM_BAD_LOGITS);
    Cand* mine = j.lists[warp];
    __syncwarp();
    if (live)
      for (int i = lane; i < P * B; i += 32) {
        const float2 y = __ldcg(reinterpret_cast<const float2*>(a.lists + (int64_t)row * P * B) + i);
        mine[i] = Cand{y.x, __float_as_int(y.y)};
      }
    __syncwarp();
    int at = lane * B;
    for (int k = 0; k < B; ++k) {
      Cand head{-INFINITY, 0x7fffffff};
      if (live && lane < P && at < (lane + 1) * B) head = mine[at];
      Cand top = head;
#pragma unroll
      for (int d = 16; d; d >>= 1) {
        const Cand o{__shfl_xor_sync(0xffffffffu, top.x, d), __shfl_xor_sync(0xffffffffu, top.v, d)};
        if (better(o, top)) top = o;
      }
      if (head.x == top.x && head.v == top.v) ++at;
      if (lane == 0) {
        j.best[b][k] = top;
        j.c[b][k] = top.x > -INFINITY ? (double)score + (((double)top.x - m) - part) : -INFINITY;
      }
    }
    if (lane == 0) {
      float e = -INFINITY;
      if (live && a.p.eos >= 0) {
        uint4 u = *reinterpret_cast<const uint4*>((const T*)a.x + (int64_t)row * a.ld + a.p.eos / Piece<T>::N * Piece<T>::N);
        float f[Piece<T>::N];
        Piece<T>::get(u, f);
#pragma unroll
        for (int i = 0; i < Piece<T>::N; ++i) e = i == a.p.eos % Piece<T>::N ? f[i] : e;
      }
      j.end_x[b] = e;
      j.ends[b] = e > -INFINITY ? (double)score + (((double)e - m) - part) : -INFINITY;
      j.token[b] = max(a.p.eos, 0);
      j.parent[b] = -1;
      j.live[b] = -INFINITY;
    }
  }
  __syncthreads();
  // ranks by counting who comes before: by c, then the lower beam, then the order within the beam
  for (int i = threadIdx.x; i < B * B; i += THREADS) {
    const int b = i / B, k = i % B;
    const double c = j.c[b][k];
    int rank = k;
    for (int o = 0; o < B; ++o)
      if (o != b)
        for (int n = 0; n < B; ++n) rank += o < b ? j.c[o][n] >= c : j.c[o][n] > c;
    if (c > -INFINITY && rank < B) {
      j.token[rank] = j.best[b][k].v;
      j.parent[rank] = b;
      j.live[rank] = c;
    }
  }
  for (int b = warp; b < B; b += WARPS) {
    const double c = j.ends[b];
    const Cand e{j.end_x[b], a.p.eos};
    int rank = 0;
    if (c > -INFINITY) {
      for (int i = lane; i < B * B; i += 32) {
        const int o = i / B;
        const double x = j.c[o][i % B];
        rank += o == b ? better(j.best[o][i % B], e) : o < b ? x >= c : x > c;
      }
      if (lane < B && lane != b) rank += lane < b ? j.ends[lane] >= c && j.ends[lane] > -INFINITY : j.ends[lane] > c;
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) rank += __shfl_xor_sync(0xffffffffu, rank, d);
    if (lane == 0) j.end_rank[b] = c > -INFINITY && rank < B ? rank : -1;
  }
  __syncthreads();
  // the pool: what had ended, then what ends now in the order of its rank
  if (warp == 0) {
    const double length = pow((double)(t + 1), a.p.length_penalty);
    const int b = lane < FL_BEAM_MAX ? lane : lane - FL_BEAM_MAX;
    float x = -INFINITY;
    int step = 0, beam = 0, order = lane;
    if (b < B) {
      if (lane < FL_BEAM_MAX) {
        x = a.from.end_scores[s * B + b];
        step = a.from.end_steps[s * B + b];
        beam = a.from.end_beams[s * B + b];
      } else if (j.end_rank[b] >= 0) {
        x = (float)(j.ends[b] / length);
        step = t;
        beam = b;
        order = FL_BEAM_MAX + j.end_rank[b];
      }
    }
    if (!(x == x)) x = -INFINITY;
    int rank = 0;
    for (int o = 0; o < 32; ++o) {
      const float y = __shfl_sync(0xffffffffu, x, o);
      const int yo = __shfl_sync(0xffffffffu, order, o);
      rank += o != lane && (y > x || (y == x && (yo < order || (yo == order && o < lane))));
    }
    j.pool[lane] = -INFINITY;
    j.pool_step[lane] = j.pool_beam[lane] = 0;
    __syncwarp();
    if (x > -INFINITY && rank < FL_BEAM_MAX) {
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
      const bool over = worst > -INFINITY && (a.p.early || worst >= (float)(j.live[0] / length));
      a.to.steps[s] = t + 1;
      a.to.done[s] = over || !(j.live[0] > -INFINITY);
    }
  }
}

template <class T, int PIECES>
__global__ void __launch_bounds__(THREADS) beam_step_kernel(StepArgs a) {
  pdl_wait();
  pdl_trigger();
  constexpr int N = Piece<T>::N;
  __shared__ float sh_group[GROUPS];
  __shared__ float sh_sum[WARPS], sh_eos;
  __shared__ Cand sh_hits[MAX_HITS];
  __shared__ int sh_count, sh_last;
  extern __shared__ __align__(16) char sh_join[];
  const int B = a.p.beams, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int slice = blockIdx.x % (unsigned)a.slices, row = blockIdx.x / (unsigned)a.slices, s = row / B;
  const int t = a.from.steps[s];  // (no read-only loads of the state: `to` may be the same memory)
  const bool active = a.from.done[s] == 0 && t >= 0 && t < a.p.max_steps;
  const float score = a.from.scores[row];
  if (active && score > -INFINITY && score < INFINITY) {
    const int all = (a.p.vocab + N - 1) / N, begin = slice * a.per, end = min(all, begin + a.per);
    const T* x = (const T*)a.x + (int64_t)row * a.ld;
    uint4 raw[PIECES];
    float f[PIECES * N];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int k = begin + i * THREADS + tid;
      if (k < end) raw[i] = __ldcs(reinterpret_cast<const uint4*>(x) + k);
    }
    if (tid == 0) {
      sh_count = 0;
      sh_eos = -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int k = begin + i * THREADS + tid;
      Piece<T>::get(raw[i], f + i * N);
      if (k >= end)
#pragma unroll
        for (int e = 0; e < N; ++e) f[i * N + e] = -INFINITY;
    }
    // tokens behind the vocabulary, and the eos, which is no candidate to go on with
    if (end == all && all * N != a.p.vocab) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e)
          if ((begin + i * THREADS + tid) * N + e >= a.p.vocab) f[i * N + e] = -INFINITY;
    }
    __syncthreads();
    if (a.p.eos >= begin * N && a.p.eos < end * N) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e)
          if ((begin + i * THREADS + tid) * N + e == a.p.eos) {
            sh_eos = f[i * N + e];
            f[i * N + e] = -INFINITY;
          }
    }
    float top = f[0];
#pragma unroll
    for (int i = 1; i < PIECES * N; ++i) top = fmaxf(top, f[i]);
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
    const float bound = __shfl_sync(0xffffffffu, g, __ffs(__ballot_sync(0xffffffffu, rank == B - 1)) - 1);
    const float m = fmaxf(__shfl_sync(0xffffffffu, g, __ffs(__ballot_sync(0xffffffffu, rank == 0)) - 1), sh_eos);
    // x - m first: rounding the product of x itself would be off by the same for every x near m
    float sum = 0.f;
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < PIECES * N; ++i) sum += exp2_hw((f[i] - base) * LOG2E);
    if (tid == 0) sum += exp2_hw((sh_eos - base) * LOG2E);
    if (top >= bound && top > -INFINITY) {
#pragma unroll
      for (int i = 0; i < PIECES * N; ++i)
        if (f[i] >= bound && f[i] > -INFINITY) {
          const int n = atomicAdd(&sh_count, 1);
          if (n < MAX_HITS) sh_hits[n] = Cand{f[i], (begin + i / N * THREADS + tid) * N + i % N};
        }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (lane == 0) sh_sum[warp] = sum;
    __syncthreads();
    Cand* list = a.lists + (int64_t)blockIdx.x * B;
    const int hits = sh_count;
    if (tid == 0) {
      float z = 0.f;
      for (int i = 0; i < WARPS; ++i) z += sh_sum[i];
      a.sums[blockIdx.x] = make_float2(m, z);
    }
    if (hits <= MAX_HITS) {
      if (tid < hits) {
        const Cand mine = sh_hits[tid];
        int r = 0;
        for (int o = 0; o < hits; ++o) r += better(sh_hits[o], mine);
        if (r < B) list[r] = mine;
      }
      if (tid >= hits && tid < B) list[tid] = Cand{-INFINITY, 0};
    } else {
      // many equal logits: the best one behind the last found, B times
      __syncthreads();
      Cand last{INFINITY, -1};
      for (int r = 0; r < B; ++r) {
        Cand mine{-INFINITY, 0x7fffffff};
#pragma unroll
        for (int i = 0; i < PIECES * N; ++i) {
          const Cand y{f[i], (begin + i / N * THREADS + tid) * N + i % N};
          if (better(last, y) && better(y, mine)) mine = y;
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) {
          const Cand o{__shfl_xor_sync(0xffffffffu, mine.x, d), __shfl_xor_sync(0xffffffffu, mine.v, d)};
          if (better(o, mine)) mine = o;
        }
        if (lane == 0) sh_hits[warp] = mine;
        __syncthreads();
        for (int i = 0; i < WARPS; ++i)
          if (better(sh_hits[i], mine)) mine = sh_hits[i];
        __syncthreads();
        if (tid == 0) list[r] = mine;
        last = mine;
      }
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

template <class T, int PIECES>
int launch_step(const StepArgs& a, cudaStream_t st) {
  auto kern = beam_step_kernel<T, PIECES>;
  FL_CUDA_TRY(fl_func_smem((const void*)kern, sizeof(Join)));
  FL_CUDA_TRY(fl_launch(kern, dim3((unsigned)(a.p.n_seqs * a.p.beams * a.slices)), dim3(THREADS), sizeof(Join), st, a));
  return FL_OK;
}

// Slices of a row: as long as a CTA's registers hold (16 pieces of 4, 8 of 8 logits a thread), shorter where the GPU
// would not be full with those.
template <class T>
int launch_typed(StepArgs& a, cudaStream_t st) {
  constexpr int N = Piece<T>::N, MOST = 64 / N;
  const int pieces = (a.p.vocab + N - 1) / N;
  const int64_t rows = (int64_t)a.p.n_seqs * a.p.beams;
  int slices = (pieces + THREADS * MOST - 1) / (THREADS * MOST);
  while (slices < MAX_SLICES && rows * slices < 2 * fl_sm_count() && (slices + 1) * THREADS <= pieces) ++slices;
  a.slices = slices;
  a.per = (pieces + slices - 1) / slices;
  a.slices = (pieces + a.per - 1) / a.per;
  const int each = (a.per + THREADS - 1) / THREADS;
  if (each <= 1) return launch_step<T, 1>(a, st);
  if (each <= 2) return launch_step<T, 2>(a, st);
  if (each <= 4) return launch_step<T, 4>(a, st);
  if constexpr (MOST > 8)
    if (each > 8) return launch_step<T, 16>(a, st);
  return launch_step<T, 8>(a, st);
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
  return dtype == FL_DT_F32 ? launch_typed<float>(a, st)
                            : dtype == FL_DT_F16 ? launch_typed<__half>(a, st) : launch_typed<__nv_bfloat16>(a, st);
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
