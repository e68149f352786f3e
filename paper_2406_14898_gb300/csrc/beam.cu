// Beam search: the next beams from every beam's logits, and the hypotheses' tokens from the back-pointers.
//
// Step.  With c(b, v) = score_b + x_bv - lse_b a search wants the best `beams` of beams x vocab candidates.  Within a
// beam c is ordered as x is, so each row needs only its largest logits and its log-sum-exp: one pass over the logits.  A CTA goes
// through its part of a row in chunks, the next one's loads in flight.  Of the first chunk the B-th largest of 32 groups of
// threads' maxima bounds the B-th largest logit from below; of what comes later only what exceeds the bound is looked
// at, about B logits for each time that what has been seen doubles, which is when the bound is raised.  A second kernel, a
// CTA a search, joins the parts' sums and lists.  (With the join in the CTA that comes last, CTAs that joined came late
// for their next parts and so joined again: 64 x 16 rows of 130528 bf16 157 us, when two kernels took 92.)  Sums are kept for each
// chunk of a row, whose places do not depend on the cut (a part's sums as one: 64 x 16 rows of bf16 65.4 us for 68.1, but equal
// rows that were cut otherwise had sums that differed in their last bits).
//
// Many rows are bound by HBM and the instructions beside it: 1024 x 1 rows of 130528 fp32 93 us (5.7 TB/s), bf16 56.5 (4.7), 64 x 16
// rows of bf16 68 (3.9), of which the hits and lists take 8, the join 8.  Few rows are bound by latency: 1 x 4 rows of fp32 8.8
// us, of which the join takes 4.
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "../../include/flglm_kernels.h"
#include "kv_attention.cuh"
#include "ptx.cuh"

namespace {

constexpr int THREADS = 128, WARPS = THREADS / 32, GROUPS = 32, MAX_PARTS = 32;
constexpr int PIECES = 8, CHUNK_PIECES = PIECES * THREADS;  // 16-byte pieces of a thread and of a CTA in a chunk
constexpr int STAGES = 2, CTAS = 6;                          // chunks on their way or in use, CTAs of an SM
constexpr int MAX_HITS = 256, MAX_ROWS = 256;                // of a CTA
constexpr int MAX_SEARCHES = 16384, MAX_VOCAB = 1 << 19;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
static_assert(FL_BEAM_MAX <= GROUPS && GROUPS == 32);

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
  int crowded;  // more than a CTA per SM
  int row_chunks, usual_parts;  // of a row; parts that a row is cut into at most where all beams are live
  float penalty_hi, penalty_lo;
  int32_t *trace_tokens, *trace_parents, *tokens, *parents;
  float2* sums;  // [row][chunk] (its largest logit, sum of exp(x - it))
  Cand* lists;   // [row][part][beam], best first; x = -inf: none
  int32_t* parts;  // [row] parts that it was cut into
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
  FL_DEV static void word(uint32_t u, float (&f)[1]) { f[0] = __uint_as_float(u); }
  FL_DEV static uint32_t max4(const uint4& u) {
    float f[4], m;
    get(u, f);
    asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(f[0]), "f"(f[1]), "f"(f[2]));
    return __float_as_uint(fmaxf(m, f[3]));
  }
  FL_DEV static uint32_t max2(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }
  FL_DEV static float top(uint32_t a) { return __uint_as_float(a); }
  FL_DEV static float one(float x) { return x; }
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
  FL_DEV static void word(uint32_t u, float (&f)[2]) {
    const float2 y = KvIo<T>::unpack(u);
    f[0] = y.x, f[1] = y.y;
  }
  FL_DEV static float top(uint32_t a) {
    const float2 y = KvIo<T>::unpack(a);
    return fmaxf(y.x, y.y);
  }
  FL_DEV static float one(T x) { return (float)x; }
};
template <>
struct Piece<__nv_bfloat16> : Piece16<__nv_bfloat16, 0xff80ff80u> {
  FL_DEV static uint32_t max2(uint32_t a, uint32_t b) {
    const __nv_bfloat162 y = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&y);
  }
  FL_DEV static uint32_t max4(const uint4& u) { return max2(max2(u.x, u.y), max2(u.z, u.w)); }
};
template <>
struct Piece<__half> : Piece16<__half, 0xfc00fc00u> {
  FL_DEV static uint32_t max2(uint32_t a, uint32_t b) {
    const __half2 y = __hmax2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&y);
  }
  FL_DEV static uint32_t max4(const uint4& u) { return max2(max2(u.x, u.y), max2(u.z, u.w)); }
};

// Whole numbers in the order of the floats (no NaN); 0 is below all of them.
FL_DEV uint32_t order32(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// A number as the unevaluated sum of two floats, the first of which is the sum rounded (T. J. Dekker, A floating-point
// technique for extending the available precision, 1971): 48 bits, for the scores that are compared and the penalty, whose series
// are in one float from their small terms on.  (The
// double-precision units of this card run at a small fraction of these' rate.)
struct Two {
  float hi, lo;
};
FL_DEV Two two_sum(float a, float b) {
  const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
  return {s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t))};
}
FL_DEV Two two_prod(float a, float b) {
  const float p = __fmul_rn(a, b);
  return {p, __fmaf_rn(a, b, -p)};
}
FL_DEV Two add(Two x, float y) {
  const Two s = two_sum(x.hi, y);
  return two_sum(s.hi, __fadd_rn(s.lo, x.lo));
}
FL_DEV Two add(Two x, Two y) { return add(add(x, y.lo), y.hi); }
FL_DEV Two mul(Two x, Two y) {
  const Two p = two_prod(x.hi, y.hi);
  return two_sum(p.hi, __fmaf_rn(x.hi, y.lo, __fmaf_rn(x.lo, y.hi, p.lo)));
}
// In the order of the numbers; 0 is below all of them, and of an infinity.
FL_DEV float unorder32(uint32_t u) { return __uint_as_float(u >> 31 ? u & 0x7fffffffu : ~u); }
FL_DEV uint64_t order64(Two x) {
  return fabsf(x.hi) < INFINITY ? (uint64_t)order32(x.hi) << 32 | order32(x.lo) : 0;
}
constexpr float LN2_HI = 0.693147182464599609375f, LN2_LO = -1.904654299958e-9f;  // ln 2 in two floats
// ln x of a normal x, off by 2^-29 at most where |ln x| < 32: x = 2^e f, ln f = 2 (s + s^3 / 3 + s^5 / 5 + ...) with
// s = (f - 1) / (f + 1), |s| <= 0.172; s in two floats, the series from s^3 on in one.
FL_DEV Two log_two(float x) {
  int e = (int)(__float_as_uint(x) >> 23) - 127;
  float f = __uint_as_float((__float_as_uint(x) & 0x7fffffu) | 0x3f800000u);
  if (f > 1.41421356f) f *= 0.5f, ++e;
  const float n = f - 1.f;  // exact
  const Two d = two_sum(f, 1.f);
  const float q = n / d.hi, r = __fmaf_rn(-q, d.lo, __fmaf_rn(-q, d.hi, n)) / d.hi, z = q * q;
  const float tail = q * z * (0.666666667f + z * (0.4f + z * (0.285714286f + z * (0.222222222f + z * 0.181818182f))));
  Two y = add(two_prod((float)e, LN2_HI), __fmaf_rn((float)e, LN2_LO, 0.f));
  y = add(y, 2.f * q);
  return add(y, __fadd_rn(tail, 2.f * r));
}
// n^p, off by 2^-25 at most where it is a normal float: e^y with y = p ln n = k ln 2 + r, the series of e^r in one float
// behind its first two terms.
FL_DEV Two pow_two(float n, Two p) {
  const Two y = mul(log_two(n), p);
  if (!(fabsf(y.hi) < 80.f)) return {y.hi > 0 ? INFINITY : 0.f, 0.f};
  const float k = rintf(y.hi * LOG2E);
  const Two r = add(add(y, two_prod(-k, LN2_HI)), -k * LN2_LO);
  const float x = r.hi;
  const float tail = x * x * (0.5f + x * (0.166666667f + x * (0.0416666667f + x * (0.00833333333f + x * (0.00138888889f +
                     x * (0.000198412698f + x * 0.0000248015873f))))));
  const Two v = add(add(two_sum(1.f, x), r.lo), tail);
  const float scale = __uint_as_float((uint32_t)((int)k + 127) << 23);
  return {v.hi * scale, v.lo * scale};
}
// x / y rounded to a float, off by little more than half an ulp.
FL_DEV float div_two(Two x, Two y) {
  const float q = x.hi / y.hi;
  if (!(fabsf(q) < 1e37f && fabsf(q) > 1e-30f && y.hi < 1e37f && y.hi > 1e-30f)) return q;
  return __fadd_rn(q, __fadd_rn(__fmaf_rn(-q, y.hi, x.hi), __fmaf_rn(-q, y.lo, x.lo)) / y.hi);
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
FL_DEV uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// sum of exp(x - ref) over a thread's logits of a chunk, ref the largest of its warp's: so a chunk's sum depends on nothing but the
// chunk, wherever the rows are cut and whatever else is in the call, and rows of equal logits have equal sums.  The exponents are
// x log2(e) - c, c = ref log2(e) rounded, one fused operation each; what the rounding of c took (the same factor for all)
// is given back in the end.  Where ref is so large that this is no small factor, x - ref is taken first.
struct Sum {
  float ref;                // (0 where there is no number)
  uint64_t minus, sum = 0;  // (-c, -c); sums of every other element
  FL_DEV explicit Sum(float x) : ref(x == -INFINITY ? 0.f : x), minus(pack2(-ref * LOG2E, -ref * LOG2E)) {}
  FL_DEV bool far() const { return fabsf(ref) > 4096.f; }
  FL_DEV void add(float x, float y) {
    const float2 u = unpack2(fma2(pack2(x, y), pack2(LOG2E, LOG2E), minus));
    sum = add2(sum, pack2(exp2_hw(u.x), exp2_hw(u.y)));
  }
  FL_DEV void add_far(float x) { sum = add2(sum, pack2(exp2_hw((x - ref) * LOG2E), 0.f)); }
  // The warp's, from all of its lanes.
  FL_DEV float of_warp() const {
    const float2 u = unpack2(sum);
    float x = u.x + u.y;
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    const float e = far() ? 0.f : LN2 * fmaf(ref, LOG2E, unpack2(minus).x);  // 2^-12 at most: e^-e from its first terms
    return x * (1.f - e + 0.5f * e * e);
  }
};
// (a logit, sum of exp(x - it)): the same sum from a larger one, and two of them as one.
FL_DEV float scaled(float2 p, float m) {
  return p.x == -INFINITY ? p.y : p.x == INFINITY ? NAN : p.y * exp2_hw((p.x - m) * LOG2E);
}
FL_DEV float2 joined(float2 p, float2 q) {
  const float m = fmaxf(p.x, q.x);
  return make_float2(m, scaled(p, m) + scaled(q, m));
}

// A warp's 32 numbers in shared memory, each lane's own.
struct Lanes {
  float at[32];
  FL_DEV void operator=(float x) { at[threadIdx.x & 31] = x; }
};

// Shared memory of a search's join; behind it each warp's copy of a row's lists.
struct Join {
  Cand best[FL_BEAM_MAX][FL_BEAM_MAX];
  Two score[FL_BEAM_MAX][FL_BEAM_MAX];  // of each beam's candidates
  uint64_t key[FL_BEAM_MAX][FL_BEAM_MAX];  // their order64, descending; 0: none
  Two ends[FL_BEAM_MAX], length;           // of each beam's eos; steps^penalty
  int end_place[FL_BEAM_MAX];              // candidates of its beam ahead of it
  // the beams that go on (beam << 8 | place in its list); places of the eos that end; -1: none
  int next[FL_BEAM_MAX], end_rank[FL_BEAM_MAX];
  float pool[2 * FL_BEAM_MAX];
  int pool_step[2 * FL_BEAM_MAX], pool_beam[2 * FL_BEAM_MAX];
};

// 16 bytes of global memory to this thread's place in shared memory, in groups that the thread itself waits for.
FL_DEV void cp_async16(void* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}
FL_DEV void cp_async4(void* to, const void* from) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}
FL_DEV void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
FL_DEV void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

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

// One search's rows joined, a warp a row: of the parts' lists whichever one's best is the best of all comes next, B times; then each
// row's candidates are placed among all by searches in the other rows' lists.  Latency is the bound, 0.14 us a candidate of a row.
// (Rows merged as the parts are, by one warp: 0.18 us a candidate, 1 x 16 rows of bf16 16.6 us for 15.7, 64 x 16 66.8 for 65.5.  Lists
// merged two and two by exchanges between lanes: in registers 64 x 16 66.1, but 1 x 4 fp32 11.1 for 8.8, as so much code comes
// from L2; in shared memory, with less code, 68.2 and 12.5.)  What it reads is asked for at once, before it is known which of it counts.
template <class T>
__global__ void __launch_bounds__(32 * FL_BEAM_MAX) beam_join_kernel(StepArgs a) {
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) char sh_join[];
  Join& j = *reinterpret_cast<Join*>(sh_join);
  const int B = a.p.beams, threads = blockDim.x, s = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int t = a.from.steps[s];  // (no read-only loads of the state: `to` may be the same memory)
  const bool active = a.from.done[s] == 0 && t >= 0 && t < a.p.max_steps;
  float pool_score = -INFINITY;  // what had ended, for the first warp's work
  int pool_step = 0, pool_beam = 0;
  if (tid < B) {
    pool_score = a.from.end_scores[s * B + tid];
    pool_step = a.from.end_steps[s * B + tid];
    pool_beam = a.from.end_beams[s * B + tid];
  }
  if (warp < B) {
    const int b = warp, row = s * B + b;
    const float score = a.from.scores[row];
    const int said = a.parts[row];
    Cand* mine = reinterpret_cast<Cand*>(&j + 1) + warp * MAX_PARTS * B;
    const Cand* lists = a.lists + (int64_t)row * MAX_PARTS * B;
    const float2* sums = a.sums + (int64_t)row * a.row_chunks;
    float2 part = lane < a.row_chunks ? sums[lane] : make_float2(-INFINITY, 0.f);  // (of any content where the row is not used)
    const float e = a.p.eos >= 0 ? Piece<T>::one(((const T*)a.x)[(int64_t)row * a.ld + a.p.eos]) : -INFINITY;
    for (int i = lane; i < a.usual_parts * B; i += 32) mine[i] = lists[i];
    const bool reads = active && score > -INFINITY && score < INFINITY;
    const int P = reads ? said : 0;
    for (int i = a.usual_parts * B + lane; i < P * B; i += 32) mine[i] = lists[i];
    if (!reads) part = make_float2(-INFINITY, 0.f);
    for (int c = lane + 32; reads && c < a.row_chunks; c += 32) part = joined(part, sums[c]);
    float m = part.x;
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    float sum = scaled(part, m);
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    const bool bad = active && (score != score || score == INFINITY || (reads && sum != sum)), live = reads && !bad && m > -INFINITY;
    if (bad && lane == 0) atomicOr(a.status, FL_BEAM_BAD_LOGITS);
    __syncwarp();
    // lists merged: each lane has a slice's, its best one that is left and the next
    int at = lane * B, k = 0;
    const int stop = live && lane < P ? at + B : at;
    Cand head = at < stop ? mine[at] : Cand{-INFINITY, 0}, next = at + 1 < stop ? mine[at + 1] : Cand{-INFINITY, 0};
#pragma unroll 1
    for (; k < B; ++k) {
      const uint32_t key = head.x > -INFINITY ? order32(head.x) : 0u, top = __reduce_max_sync(0xffffffffu, key);
      if (top == 0) break;
      const unsigned who = __ballot_sync(0xffffffffu, key == top);
      bool won = key == top;
      if (who & (who - 1)) {  // (all lanes take part, whoever has won)
        const int v = __reduce_min_sync(0xffffffffu, won ? head.v : 0x7fffffff);
        won = won && head.v == v;
      }
      if (won) {
        j.best[b][k] = head;
        head = next;
        ++at;
        next = at + 1 < stop ? mine[at + 1] : Cand{-INFINITY, 0};
      }
    }
    __syncwarp();
    // c = score + ((x - m) - log(sum)): exact for the smallest logits that a type has, too
    const Two l = live ? log_two(sum) : Two{0.f, 0.f};
    const auto c_of = [&](float x) {
      return x > -INFINITY ? add(add(two_sum(x, -m), Two{-l.hi, -l.lo}), score) : Two{-INFINITY, 0.f};
    };
    const Cand one = lane < k ? j.best[b][lane] : Cand{-INFINITY, 0};
    const Two c = c_of(one.x);
    // a row's candidates stay in their order where their c differ by less than these numbers resolve
    uint64_t key = order64(c);
#pragma unroll
    for (int d = 1; d < FL_BEAM_MAX; d <<= 1) {
      const uint64_t y = __shfl_up_sync(0xffffffffu, key, d);
      if (lane >= d) key = min(key, y);
    }
    const Cand eos{live ? e : -INFINITY, a.p.eos};
    const Two end = c_of(eos.x);
    // (where the eos' c equals a candidate's, the order is that of the logits)
    const bool is_before = key > order64(end) || (key == order64(end) && better(one, eos));
    const int before = __popc(__ballot_sync(0xffffffffu, lane < B && key != 0 && is_before));
    if (lane < FL_BEAM_MAX) j.key[b][lane] = lane < B ? key : 0;
    if (lane < B) {
      j.best[b][lane] = one;
      j.score[b][lane] = c;
    }
    if (lane == 0) {
      j.ends[b] = end;
      j.end_place[b] = before;
      j.next[b] = j.end_rank[b] = -1;
    }
  }
  if (tid == threads - 1) j.length = pow_two((float)(t + 1), {a.penalty_hi, a.penalty_lo});
  __syncthreads();
  if (!active) {  // it stays as it is
    if (warp == 0) rest(a, s);
    return;
  }
  // The rows' lists joined: by c, then the lower beam, then that beam's order, in which its eos has its place.  A candidate's place is
  // how many are ahead of it in each list.  The first B go on; an eos among the first B of all ends a hypothesis.
  if (warp < B) {
    const int b = warp, k = lane % FL_BEAM_MAX;
    const auto ahead_in = [&](int q, uint64_t key) {  // of another beam's list
      const uint64_t least = key + (q > b);  // (key is not 0 and no infinity's: no overflow)
      int n = 0;
#pragma unroll
      for (int d = FL_BEAM_MAX / 2; d; d >>= 1) n += j.key[q][n + d - 1] >= least ? d : 0;
      return n + (j.key[q][n] >= least);
    };
    const uint64_t mine = j.key[b][k];
    int place = 0;
#pragma unroll 4
    for (int q = lane / FL_BEAM_MAX; q < B; q += 2) {
      const int n = ahead_in(q, mine);
      place += q == b ? k : n;
    }
    place += __shfl_xor_sync(0xffffffffu, place, FL_BEAM_MAX);
    if (mine != 0 && place < B && lane < FL_BEAM_MAX) j.next[place] = b << 8 | k;
    const uint64_t end = order64(j.ends[b]);
    if (end != 0) {
      int n = 0;
      if (lane < B) {
        const uint64_t other = order64(j.ends[lane]);
        n = lane == b ? j.end_place[b] : ahead_in(lane, end) + (other > end || (other == end && lane < b));
      }
      n = __reduce_add_sync(0xffffffffu, n);
      if (lane == 0 && n < B) j.end_rank[b] = n;
    }
  }
  __syncthreads();
  if (warp != 0) return;
  const int beam = lane % FL_BEAM_MAX, next = lane < B ? j.next[lane] : -1;
  const int end_rank = lane >= FL_BEAM_MAX && beam < B ? j.end_rank[beam] : -1;
  // the pool: what had ended, then what ends now in the order of its rank
  float x = pool_score;
  int step = pool_step, from_beam = pool_beam;
  if (!(x > -INFINITY)) x = -INFINITY, step = from_beam = 0;
  if (__any_sync(0xffffffffu, end_rank >= 0)) {
    if (end_rank >= 0) {
      x = div_two(j.ends[beam], j.length);
      step = t;
      from_beam = beam;
    }
    const int order = end_rank >= 0 ? FL_BEAM_MAX + end_rank : lane;
    const uint64_t place = (uint64_t)order32(x) << 32 | (uint32_t)((63 - order) << 8 | (31 - lane));
    int rank = 0;
#pragma unroll 8
    for (int o = 0; o < 32; ++o) rank += __shfl_sync(0xffffffffu, place, o) > place;
    j.pool[rank] = x;
    j.pool_step[rank] = step;
    j.pool_beam[rank] = from_beam;
    __syncwarp();
    x = j.pool[lane], step = j.pool_step[lane], from_beam = j.pool_beam[lane];
  }
  __syncwarp();
  const float worst = __shfl_sync(0xffffffffu, x, B - 1);
  if (lane < B) {
    const int i = s * B + lane, parent = next >> 8, token = next >= 0 ? j.best[parent][next & 255].v : max(a.p.eos, 0);
    const Two score = next >= 0 ? j.score[parent][next & 255] : Two{-INFINITY, 0.f};
    const int64_t tr = ((int64_t)s * a.p.max_steps + t) * B + lane;
    a.to.scores[i] = score.hi;
    a.to.end_scores[i] = x;
    a.to.end_steps[i] = step;
    a.to.end_beams[i] = from_beam;
    a.tokens[i] = a.trace_tokens[tr] = token;
    a.trace_parents[tr] = next < 0 ? lane : parent;
    a.parents[i] = next < 0 ? -1 : s * B + parent;
    if (lane == 0) {
      a.to.steps[s] = t + 1;
      a.to.done[s] = next < 0 || (worst > -INFINITY && (a.p.early || worst >= div_two(score, j.length)));
    }
  }
}

// The chunks of the live beams' rows lie one after another on a line, which is cut into equal pieces, one a CTA: a row's
// part is what lies in one CTA's piece.  A thread asks for its 16-byte pieces of a chunk a chunk ahead, into places of its own that
// nobody else waits for, and while a part ends the next one's first chunk is on its way.
template <class T>
__global__ void __launch_bounds__(THREADS, CTAS) beam_step_kernel(StepArgs a) {
  pdl_wait();
  // The join's CTAs may come while this kernel runs only where they find room beside it: else those that finish first would take
  // them all (1024 x 1 rows of bf16 62 us instead of 54).
  if (!a.crowded) pdl_trigger();
  using Io = Piece<T>;
  constexpr int N = Io::N;
  constexpr int RING = STAGES * CHUNK_PIECES * 16;
  static_assert(CTAS * (RING + MAX_HITS * sizeof(Cand) + MAX_ROWS * 4 + 2 * WARPS * sizeof(Lanes) + 4 * GROUPS * 4 + 128 + 1024) <= 228 * 1024,
                "so many CTAs fit an SM, which keeps 1 KB of each");
  __shared__ __align__(16) uint32_t sh_group[2][GROUPS], sh_key[2][GROUPS];
  __shared__ Lanes sh_ref[WARPS], sh_sum[WARPS];  // of a warp's part of up to 32 chunks
  __shared__ int sh_count, sh_few, sh_warp[WARPS];
  uint32_t* const sh_bits = reinterpret_cast<uint32_t*>(sh_sum);  // [THREADS], before there are sums
  static_assert(sizeof(sh_sum) == THREADS * sizeof(uint32_t));
  __shared__ int sh_rows[MAX_ROWS];
  __shared__ Cand sh_hits[MAX_HITS];
  extern __shared__ __align__(16) uint4 sh_ring[];  // [STAGES][CHUNK_PIECES]
  const int B = a.p.beams, rows = a.p.n_seqs * B, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int all = (a.p.vocab + N - 1) / N, L = a.row_chunks;
  // this CTA's chunks with n live rows: [c0, c1) of n L
  int c0, c1, ctas, n_live;
  const auto cut = [&](int n) {
    const int64_t chunks = (int64_t)n * L;
    n_live = n;
    ctas = (int)min((int64_t)gridDim.x, L <= MAX_PARTS ? chunks : (int64_t)(MAX_PARTS - 2) * n);  // no row in more than MAX_PARTS
    c0 = c1 = 0;
    if ((int)blockIdx.x >= ctas) return;
    const bool one = ctas == chunks;  // a chunk each
    c0 = one ? (int)blockIdx.x : (int)kv_div(blockIdx.x * chunks, ctas);
    c1 = one ? c0 + 1 : (int)kv_div((blockIdx.x + 1) * chunks, ctas);
  };
  // (no read-only loads of the state: `to` may be the same memory; no load behind another's outcome)
  const auto is_live = [&](int t, int done, float score) {
    return (done == 0) & (t >= 0) & (t < a.p.max_steps) & (score > -INFINITY) & (score < INFINITY);
  };
  // the first rows' states are asked for ahead of the logits
  constexpr int EARLY = 8;
  int early_t[EARLY], early_done[EARLY];
  float early_score[EARLY];
#pragma unroll
  for (int i = 0; i < EARLY; ++i) {
    const int row = tid + i * THREADS, s = row / B;
    if (i * THREADS >= rows) break;
    if (row < rows) early_t[i] = a.from.steps[s], early_done[i] = a.from.done[s], early_score[i] = a.from.scores[row];
  }
  // what is asked for next: a chunk of the line, its row, its first piece; the stage that it goes to
  int ask = 0, ask_first = 0, ask_stage = 0;
  const uint4* ask_x = nullptr;
  const auto ask_row = [&](int row) { ask_x = reinterpret_cast<const uint4*>((const T*)a.x + (int64_t)row * a.ld); };
  const auto ask_chunk = [&] {
    uint4* to = sh_ring + ask_stage * CHUNK_PIECES + tid;
    const uint4* from = ask_x + ask_first + tid;
    if (ask_first + CHUNK_PIECES <= all) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) cp_async16(to + i * THREADS, from + i * THREADS);
    } else {
#pragma unroll 1
      for (int k = ask_first + tid; k < all; k += THREADS, to += THREADS, from += THREADS) cp_async16(to, from);
    }
    ++ask;
    ask_first += CHUNK_PIECES;
    ask_stage = ask_stage + 1 == STAGES ? 0 : ask_stage + 1;
  };
  bool known = false;  // which rows are live; until then, and where all are, the k-th of them is row k
  int k0 = 0;
  const auto ask_more = [&] {  // one group each time, an empty one behind the last chunk
    if (ask < c1) {
      if (ask_first >= all) {
        ask_first = 0;
        ask_row(known ? sh_rows[ask / L - k0] : ask / L);
      }
      ask_chunk();
    }
    cp_async_commit();
  };
  const auto ask_first_ones = [&] {
    ask = c0;
    ask_first = c0 % L * CHUNK_PIECES;
    ask_stage = 0;
    ask_row(known ? sh_rows[0] : c0 / L);
    ask_more();
    ask_more();
  };
  // The first chunks as they are if all beams are live, before that is known.
  cut(rows);
  ask_first_ones();
  // which rows are live, a bit each, 32 x THREADS of them at a time; how many, and those of this CTA's piece
  const auto set_bits = [&](int row, bool x) {
    const uint32_t m = __ballot_sync(0xffffffffu, x);
    if (lane == 0) sh_bits[row / 32 % THREADS] = m;
  };
  const auto bits = [&](int base) {
    if (base == 0) {
#pragma unroll
      for (int i = 0; i < EARLY; ++i) {
        const int r = tid + i * THREADS;
        if (i * THREADS >= rows) break;
        set_bits(r, r < rows && is_live(early_t[i], early_done[i], early_score[i]));
      }
    }
#pragma unroll 4
    for (int r = base + (base == 0 ? EARLY * THREADS : 0) + tid; r < min(rows + 31 & ~31, base + 32 * THREADS); r += THREADS) {
      const int row = min(r, rows - 1), s = row / B;
      set_bits(r, r < rows && is_live(a.from.steps[s], a.from.done[s], a.from.scores[row]));
    }
    __syncthreads();
  };
  const int words = min(THREADS, (rows + 31) / 32);
  int total = 0, before = 0;  // live rows before this thread's 32
  const auto count = [&](int base) {
    const int n = base + 32 * tid < rows && tid < words ? __popc(sh_bits[tid]) : 0;
    before = n;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, before, d);
      if (lane >= d) before += y;
    }
    if (lane == 31) sh_warp[warp] = before;
    __syncthreads();
    before += total - n;
    for (int w = 0; w < WARPS; ++w) {
      if (w < warp) before += sh_warp[w];
      total += sh_warp[w];
    }
  };
  for (int base = 0; base < rows; base += 32 * THREADS) {
    if (base) __syncthreads();
    bits(base);
    count(base);
  }
  const bool guessed = total == rows;
  if (!guessed) cut(total);
  k0 = c0 / L;
  const int k1 = c0 < c1 ? (c1 - 1) / L : -1;  // its first and last live row are k0 and k1
  const bool again = rows > 32 * THREADS;                   // the bits and counts are those of the last rows only
  if (again) total = 0;
  for (int base = 0; base < rows; base += 32 * THREADS) {
    if (again) {
      __syncthreads();
      bits(base);
      count(base);
    }
    if (base + 32 * tid < rows && tid < words) {
      int k = before;
      for (uint32_t m = k <= k1 ? sh_bits[tid] : 0; m; m &= m - 1, ++k)
        if (k >= k0 && k <= k1) sh_rows[k - k0] = base + 32 * tid + __ffs(m) - 1;
    }
  }
  __syncthreads();
  if (c0 >= c1) {
    cp_async_wait<0>();
    return;
  }
  known = true;
  if (!guessed) {  // the first chunks came for nothing
    cp_async_wait<0>();
    ask_first_ones();
  }
  int stage = 0, raised = 0;
  static_assert(STAGES == 2 && PIECES * 4 == 32);
  for (int c = c0; c < c1;) {
    {
      const int k = c / L, row = sh_rows[k - k0], from = c - k * L, to = min(L, from + c1 - c);
      c += to - from;
      const int part_begin = from * CHUNK_PIECES, part_end = min(all, to * CHUNK_PIECES);
      // which part of its row: its CTA's distance from the one of the row's first chunk
      const int part = ctas == (int64_t)n_live * L ? from : blockIdx.x - (int)kv_div(((int64_t)k * L + 1) * ctas - 1, (int64_t)n_live * L);
      const int64_t at_part = (int64_t)row * MAX_PARTS + part;
      const int eos_piece = a.p.eos >= 0 && a.p.eos / N >= part_begin && a.p.eos / N < part_end ? a.p.eos / N : -1;
      float bound = -INFINITY, most = -INFINITY;  // of this thread
      bool settled = false;                       // the bound is that of all that has been seen
      if (tid == 0) sh_count = sh_few = 0;
      // the bound raised to the B-th largest of the groups' maxima, with a barrier; true where it is higher now
      const auto raise = [&] {
        float g = most;
#pragma unroll
        for (int d = 1; d < THREADS / GROUPS; d <<= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, d));
        uint32_t* keys = sh_key[raised & 1];
        if (tid % (THREADS / GROUPS) == 0) {
          const int i = tid / (THREADS / GROUPS);
          sh_group[raised & 1][i] = order32(g);
          keys[i] = (order32(g) & ~31u) | (31 - i);
        }
        __syncthreads();
        // (numbers that agree in all but their last bits count as equal, the lower group first: the B groups that are taken have
        // maxima of the bound and more whichever they are)
        const uint32_t key = keys[lane], ordered = sh_group[raised & 1][lane];
        ++raised;
        int rank = 0;
#pragma unroll
        for (int o = 0; o < GROUPS; o += 4) {
          const uint4 y = *reinterpret_cast<const uint4*>(keys + o);
          rank += (y.x > key) + (y.y > key) + (y.z > key) + (y.w > key);
        }
        const float b = unorder32(__reduce_min_sync(0xffffffffu, rank < B ? ordered : 0xffffffffu));
        const bool higher = b > bound;
        bound = b;
        settled = true;
        return higher;
      };
      // 32 chunks at a time, lane i of each warp with its part of the i-th one's sum
      for (int begin = part_begin; begin < part_end; begin += 32 * CHUNK_PIECES) {
        const int end = min(part_end, begin + 32 * CHUNK_PIECES);
        struct { float ref, sum; } z{-INFINITY, 0.f};
        for (int first = begin, chunk = 0; first < end; first += CHUNK_PIECES, ++chunk) {
          cp_async_wait<STAGES - 1>();
          uint4* places = sh_ring + stage * CHUNK_PIECES + tid;  // this thread's
          stage = stage + 1 == STAGES ? 0 : stage + 1;
          // nothing behind the slice's end and the vocabulary; the eos is summed, but no candidate to go on with
          if (first + CHUNK_PIECES >= end) {
#pragma unroll 1
            for (int i = 0; i < PIECES; ++i) {
              const int k = first + i * THREADS + tid;
              if (k >= end) places[i * THREADS] = make_uint4(Io::NONE, Io::NONE, Io::NONE, Io::NONE);
              else if ((k + 1) * N > a.p.vocab)
                for (int v = a.p.vocab - k * N; v < N; ++v) reinterpret_cast<T*>(places + i * THREADS)[v] = (T)-INFINITY;
            }
          }
          float apart = -INFINITY;
          if (eos_piece >= first && eos_piece < first + CHUNK_PIECES && (eos_piece - first) % THREADS == tid) {
            T* at = reinterpret_cast<T*>(places + (eos_piece - first - tid)) + a.p.eos % N;
            apart = Io::one(*at);
            *at = (T)-INFINITY;
          }
          uint4 cur[PIECES];
          uint32_t largest = Io::NONE;
#pragma unroll
          for (int i = 0; i < PIECES; ++i) cur[i] = places[i * THREADS];
#pragma unroll
          for (int i = 0; i < PIECES; ++i) largest = Io::max2(largest, Io::max4(cur[i]));
          const float top = Io::top(largest);
          most = fmaxf(most, top);
          bool equals = false;  // whether logits equal to the bound count: it is new, and fewer than B larger ones may have been seen
          const int seen = chunk + 1;
          settled = false;
          if ((seen & chunk) == 0) equals = raise() || chunk == 0;
          const bool look = top > -INFINITY && (equals ? top >= bound : top > bound);
          const float ref = unorder32(__reduce_max_sync(0xffffffffu, order32(fmaxf(top, apart))));
          Sum one(ref);
          if (!one.far()) {
            if (apart != -INFINITY) one.add(apart, -INFINITY);
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
              float f[N];
              Io::get(cur[i], f);
#pragma unroll
              for (int k = 0; k < N; k += 2) one.add(f[k], f[k + 1]);
            }
          } else {
            if (apart != -INFINITY) one.add_far(apart);
#pragma unroll 1
            for (int i = 0; i < PIECES * N; ++i) one.add_far(Io::one(reinterpret_cast<const T*>(places + i / N * THREADS)[i % N]));
          }
          const float total = one.of_warp();
          if (lane == chunk) z = {ref, total};
          // what exceeds the bound, a thread's logits at a time by its whole warp
          if (unsigned who = __ballot_sync(0xffffffffu, look)) {
            __syncwarp();  // (a thread's own copies are seen by the others)
            const uint4* its = places - lane + lane / 4 * THREADS;
            const int its_first = (first + lane / 4 * THREADS + tid - lane) * N + lane % 4 * (N / 4);
            for (; who; who &= who - 1) {
              const int l = __ffs(who) - 1;
              float f[N / 4];
              Io::word(reinterpret_cast<const uint32_t*>(its + l)[lane % 4], f);
#pragma unroll
              for (int k = 0; k < N / 4; ++k)
                if (f[k] > bound || (equals && f[k] == bound && f[k] > -INFINITY)) {
                  const int n = atomicAdd(&sh_count, 1);
                  if (n < MAX_HITS) sh_hits[n] = Cand{f[k], its_first + l * N + k};
                }
            }
            __syncwarp();  // the places have been read
          }
          ask_more();  // into the stage that has been read
        }
        const float ref = z.ref;
        const float sum = z.sum;
        sh_ref[warp] = ref;
        sh_sum[warp] = sum;
        // The part's list: of what has come together, what reaches the bound of the whole part, ranked by counting.
        const bool early = !settled;
        if (early) raise();
        else __syncthreads();
        int n = sh_count;
        if (end == part_end) {
          const uint4* x = reinterpret_cast<const uint4*>((const T*)a.x + (int64_t)row * a.ld);
          if (n > MAX_HITS) {
            // more than there was room for (logits that ascend): once more through the part, with that bound
            __syncthreads();
            if (tid == 0) sh_count = 0;
            __syncthreads();
            for (int k = part_begin + tid; k < part_end; k += THREADS) {
              float f[N];
              Io::get(x[k], f);
              for (int e = 0; e < N; ++e)
                if (f[e] >= bound && f[e] > -INFINITY && k * N + e < a.p.vocab && k * N + e != a.p.eos) {
                  const int at = atomicAdd(&sh_count, 1);
                  if (at < MAX_HITS) sh_hits[at] = Cand{f[e], k * N + e};
                }
            }
            __syncthreads();
            n = sh_count;
          } else if (early && n > 32) {
            static_assert(MAX_HITS == 2 * THREADS);
            const Cand h0 = sh_hits[tid], h1 = sh_hits[tid + THREADS];
            __syncthreads();
            if (tid < n && h0.x >= bound) sh_hits[atomicAdd(&sh_few, 1)] = h0;
            if (tid + THREADS < n && h1.x >= bound) sh_hits[atomicAdd(&sh_few, 1)] = h1;
            __syncthreads();
            n = sh_few;
          }
          Cand* list = a.lists + at_part * B;
          if (n <= MAX_HITS) {
            for (int i = tid; i < n; i += THREADS) {
              const Cand one = sh_hits[i];
              int r = 0;
              for (int o = 0; o < n; ++o) r += better(sh_hits[o], one);
              if (r < B) list[r] = one;
            }
            if (tid >= n && tid < B) list[tid] = Cand{-INFINITY, 0};
          } else {
            // many equal logits: the best one behind the last found, B times
            Cand found{INFINITY, -1};
            for (int r = 0; r < B; ++r) {
              Cand one{-INFINITY, 0x7fffffff};
              for (int k = part_begin + tid; k < part_end; k += THREADS) {
                float f[N];
                Io::get(x[k], f);
                for (int e = 0; e < N; ++e) {
                  const Cand y{f[e], k * N + e};
                  if (y.v < a.p.vocab && y.v != a.p.eos && better(found, y) && better(y, one)) one = y;
                }
              }
#pragma unroll
              for (int d = 16; d; d >>= 1) {
                const Cand o{__shfl_xor_sync(0xffffffffu, one.x, d), __shfl_xor_sync(0xffffffffu, one.v, d)};
                if (better(o, one)) one = o;
              }
              if (lane == 0) sh_hits[warp] = one;
              __syncthreads();
              for (int i = 0; i < WARPS; ++i)
                if (better(sh_hits[i], one)) one = sh_hits[i];
              __syncthreads();
              if (tid == 0) list[r] = one;
              found = one;
            }
          }
        }
        if (tid < (end - begin + CHUNK_PIECES - 1) / CHUNK_PIECES) {  // chunk tid's, the warps' in their order
          const int at = begin / CHUNK_PIECES + tid;
          float2 whole = make_float2(sh_ref[0].at[tid], sh_sum[0].at[tid]);
#pragma unroll
          for (int w = 1; w < WARPS; ++w) whole = joined(whole, make_float2(sh_ref[w].at[tid], sh_sum[w].at[tid]));
          a.sums[(int64_t)row * L + at] = whole;
          if (at == L - 1) a.parts[row] = part + 1;
        }
        __syncthreads();  // the hits' and the sums' places are free again
      }
    }
  }
  cp_async_wait<0>();  // (a first chunk that came for nothing)
  if (a.crowded) pdl_trigger();
}

// Chunks of a row of 16-byte pieces of N logits.
int chunks_of(int vocab, int N) { return ((vocab + N - 1) / N + CHUNK_PIECES - 1) / CHUNK_PIECES; }

int64_t part_bytes(const fl_beam_search* p) {  // (chunks of fp32 logits: the most)
  return (int64_t)p->n_seqs * p->beams * (chunks_of(p->vocab, 4) * sizeof(float2) + MAX_PARTS * p->beams * sizeof(Cand) + sizeof(int32_t)) + 16;
}

const char* search_problem(const fl_beam_search* p, int* code) {
  *code = FL_ERR_INVALID_ARG;
  if (!p || p->n_seqs < 0 || p->beams < 1 || p->vocab < 1 || p->max_steps < 1 || p->eos < -1 || p->eos >= p->vocab ||
      (p->early != 0 && p->early != 1))
    return "search";
  const double penalty = std::fabs(p->length_penalty);
  if (!(penalty <= 16 && penalty * std::log((double)p->max_steps) <= 80)) return "length_penalty";
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

template <class T>
int launch_step(StepArgs& a, cudaStream_t st) {
  constexpr int N = Piece<T>::N, ring = STAGES * CHUNK_PIECES * 16;
  const int rows = a.p.n_seqs * a.p.beams;
  a.row_chunks = chunks_of(a.p.vocab, N);
  // as many CTAs as run at once (more where one would have more rows than it keeps), and no more than chunks
  const int64_t slots = std::max(CTAS * fl_sm_count(), (rows + MAX_ROWS - 3) / (MAX_ROWS - 2));
  const int grid = (int)std::min<int64_t>(slots, (int64_t)rows * a.row_chunks);
  a.crowded = grid > fl_sm_count();
  a.usual_parts = std::min({MAX_PARTS, a.row_chunks, grid / rows + 2});
  auto kern = beam_step_kernel<T>;
  auto join = beam_join_kernel<T>;
  const auto join_smem = [](int beams) { return (int)sizeof(Join) + beams * MAX_PARTS * beams * (int)sizeof(Cand); };
  FL_CUDA_TRY(fl_func_smem((const void*)kern, ring));
  FL_CUDA_TRY(fl_func_smem((const void*)join, join_smem(FL_BEAM_MAX)));
  FL_CUDA_TRY(fl_launch(kern, dim3(grid), dim3(THREADS), ring, st, a));
  // four warps at least, and no more than it has work for (1024 x 1 rows of bf16 with one warp 60 us, with four 54, with sixteen 59)
  FL_CUDA_TRY(fl_launch(join, dim3(a.p.n_seqs), dim3(32 * std::max(4, a.p.beams)), join_smem(a.p.beams), st, a));
  return FL_OK;
}

// ------------------------------------------------------------------------------- back-pointers
constexpr int TRACE_THREADS = 256, CHUNK = 16, MAX_STEPS = 2048, MAX_TRACE_CTAS = 8;  // steps of a CTA, CTAs of a search

struct TraceArgs {
  fl_beam_search p;
  fl_beam_state s;
  const int32_t *tokens, *parents;
  int n_best, pad;
  float penalty_hi, penalty_lo;
  int block;  // steps of a CTA, CHUNK at least
  int32_t *out_tokens, *out_lens;
  float* out_scores;
  int* status;
};

FL_DEV uint32_t ld_cluster_u8(const void* p, uint32_t rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u8 %0, [%1];" : "=r"(v) : "r"(mapa_shared(smem_u32(p), rank)) : "memory");
  return v;
}

// Beams after each step, from the last step to the first: b(t - 1) = parent[t][b(t)].  Following one pointer after
// another costs a load's latency a step.  Here a cluster has a search and each of its CTAs some of the steps, of which each chunk
// of 16 becomes one map from the beams behind it to those before it, all at once from shared memory; those together give
// the CTA's map, the CTAs learn each other's, the hypotheses jump from CTA to CTA and from chunk to chunk, and then all
// chunks are walked at once for the beams in between.  Latency is the bound: 64 x 16 hypotheses of 2048 steps 16.7 us (a CTA a
// search 44), the best of 16 x 4 of 256 steps 6.2.  Eight CTAs fit an SM, a call's beside the last one's: with room for
// four 64 x 16 took 19.7.
__global__ void __launch_bounds__(TRACE_THREADS, 8) beam_trace_kernel(TraceArgs a) {
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) int32_t token[];  // [step][beam], a step's row from another bank than the next one's; then bytes
  const int B = a.p.beams, T = a.p.max_steps, n = a.n_best, block = a.block, line = block + 4, odd = B | 1, tid = threadIdx.x;
  const int rank = cluster_ctarank(), ctas = cluster_nctarank(), s = blockIdx.x / ctas;
  const int chunks = (block + CHUNK - 1) / CHUNK;
  uint8_t* par = reinterpret_cast<uint8_t*>(token + block * odd);  // [step][beam]
  uint8_t* map = par + block * B;       // [chunk][beam]
  uint8_t* entry = map + chunks * B;    // [chunk][hypothesis]: its beam after the chunk's last step that it has
  uint8_t* chain = entry + chunks * n;  // [hypothesis][step], a hypothesis's line from another bank than the next one's
  uint8_t* behind = chain + line * n;  // [chunk][beam]: the beam after the chunk's last step, by the beam behind the block
  __shared__ int h_steps[FL_BEAM_MAX], h_ended[FL_BEAM_MAX], h_beam[FL_BEAM_MAX], h_from[FL_BEAM_MAX], h_after[FL_BEAM_MAX];
  // beams before the block: by the beam behind it; of hypotheses that end in it
  __shared__ uint8_t of_block[FL_BEAM_MAX], of_part[FL_BEAM_MAX];
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
        x = div_two({a.s.scores[s * B + b], 0.f}, pow_two((float)steps, {a.penalty_hi, a.penalty_lo}));
        before = steps;
        beam = b;
      }
    }
    if (!(x == x)) x = -INFINITY;
    if (bad) atomicOr(a.status, FL_BEAM_BAD_TRACE);
    const uint64_t key = (uint64_t)order32(x) << 32 | (31 - tid);
    int place = 0;
#pragma unroll 8
    for (int o = 0; o < 32; ++o) place += __shfl_sync(0xffffffffu, key, o) > key;
    if (place < n) {
      const bool some = x > -INFINITY;
      h_steps[place] = some ? before : 0;
      h_ended[place] = some && tid < FL_BEAM_MAX;
      h_beam[place] = beam;
      if (rank == 0) {
        a.out_scores[s * n + place] = x;
        a.out_lens[s * n + place] = some ? before + (tid < FL_BEAM_MAX) : 0;
      }
    }
  }
  __syncthreads();
  int longest = 0;
  for (int h = 0; h < n; ++h) longest = max(longest, h_steps[h]);
  const int row = block * ctas;  // steps of the cluster at a time
  for (int base = (T - 1) / row * row; base >= 0; base -= row) {
    const int t0 = base + rank * block, len = max(0, min(block, T - t0)), nc = (len + CHUNK - 1) / CHUNK;
    const int have = min(max(longest - t0, 0), len);  // steps that some hypothesis has
    const int64_t first = ((int64_t)s * T + t0) * B;
    for (int i = tid; i < have * B; i += TRACE_THREADS) cp_async4(token + i / B * odd + i % B, a.tokens + first + i);
    cp_async_commit();
    for (int i = tid; i < have * B; i += 4 * TRACE_THREADS) {
      const int32_t* from = a.parents + first + i;
      int p[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) p[k] = i + k * TRACE_THREADS < have * B ? from[k * TRACE_THREADS] : 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if ((unsigned)p[k] >= (unsigned)B) {
          atomicOr(a.status, FL_BEAM_BAD_TRACE);
          p[k] = 0;
        }
        if (i + k * TRACE_THREADS < have * B) par[i + k * TRACE_THREADS] = (uint8_t)p[k];
      }
    }
    __syncthreads();
    for (int i = tid; i < nc * B; i += TRACE_THREADS) {
      const int c = i / B, lo = c * CHUNK;
      int b = i % B;
      for (int t = min(lo + CHUNK, have) - 1; t >= lo; --t) b = par[t * B + b];
      map[i] = (uint8_t)b;
    }
    __syncthreads();
    // The block from behind, chunk by chunk: for each beam that may be there, and for the hypotheses whose steps end in it.
    if (tid < B || (tid >= 32 && tid < 32 + n)) {
      const bool full = tid < B;
      const int i = full ? tid : tid - 32, mine = full ? have : min(max(h_steps[i] - t0, 0), len);
      uint8_t* told = full ? behind + i : entry + i;
      int b = full ? tid : h_beam[i];
      for (int c = nc - 1; c >= 0; --c) {
        const int lo = c * CHUNK;
        told[c * (full ? B : n)] = (uint8_t)b;
        if (mine >= min(lo + CHUNK, have))
          b = map[c * B + b];
        else
          for (int t = mine - 1; t >= lo; --t) b = par[t * B + b];
      }
      (full ? of_block : of_part)[i] = (uint8_t)b;
    }
    __syncthreads();
    if (ctas > 1) cluster_sync();
    if (tid < n) {  // the beam after the block's last step, if the hypothesis has that; the one before the row
      int b = h_beam[tid], after = b;
      for (int r = ctas - 1; r >= 0; --r) {
        if (r == rank) b = after;
        const int begin = base + r * block, end = min(begin + block, T), has = h_steps[tid];
        if (ctas == 1) break;
        if (has >= end && has > begin) after = (int)ld_cluster_u8(of_block + after, r);
        else if (has > begin) after = (int)ld_cluster_u8(of_part + tid, r);
      }
      if (ctas == 1) after = h_steps[tid] >= min(base + block, T) ? of_block[after] : of_part[tid];
      h_from[tid] = b;
      h_after[tid] = after;
    }
    if (ctas > 1) cluster_sync();  // (everybody has read the others' maps)
    else __syncthreads();
    if (tid < n) h_beam[tid] = h_after[tid];
    for (int i = tid; i < nc * n; i += TRACE_THREADS) {
      const int c = i / n, h = i % n, lo = c * CHUNK, has = min(h_steps[h] - t0, len);
      int beam = has == len ? behind[c * B + h_from[h]] : entry[i];
      for (int t = min(lo + CHUNK, has) - 1; t >= lo; --t) {
        chain[h * line + t] = (uint8_t)beam;
        beam = par[t * B + beam];
      }
    }
    cp_async_wait<0>();
    __syncthreads();
    // 32 steps of a hypothesis a warp
    const int pieces = (len + 31) / 32, lane = tid & 31;
#pragma unroll 4
    for (int i = tid >> 5; i < n * pieces; i += TRACE_THREADS / 32) {
      const int h = i / pieces, t = i % pieces * 32 + lane, has = h_steps[h] - t0;
      if (t >= len) continue;
      int v = a.pad;
      if (t < has) v = token[t * odd + chain[h * line + t]];
      else if (t == has && h_ended[h] && a.p.eos >= 0) v = a.p.eos;
      a.out_tokens[((int64_t)s * n + h) * T + t0 + t] = v;
    }
    __syncthreads();
  }
}

}  // namespace

extern "C" size_t fl_k_beam_workspace(const fl_beam_search* search) {
  int code;
  if (const char* w = search_problem(search, &code)) {
    fl_internal_error(code, "beam workspace: %s", w);
    return 0;
  }
  return part_bytes(search);
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
  const float penalty = (float)search->length_penalty;
  StepArgs a{*search, *from, *to, logits, ld, 0, 0, 0, penalty, (float)(search->length_penalty - penalty), trace_tokens, trace_parents,
             tokens, parents, nullptr, nullptr, nullptr, status};
  a.sums = (float2*)workspace;
  const int64_t rows = (int64_t)search->n_seqs * search->beams;
  a.lists = (Cand*)(a.sums + rows * chunks_of(search->vocab, 4));
  a.parts = (int32_t*)(a.lists + rows * MAX_PARTS * search->beams);
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
  const float penalty = (float)search->length_penalty;
  // CTAs of 64 steps, as many as a cluster has; longer ones where those are too few (the best of 16 x 4 beams of 256 steps with CTAs of
  // 256 6.7 us)
  constexpr int CTA_STEPS = 64;
  const int T = search->max_steps;
  int ctas = 1;
  while (ctas < MAX_TRACE_CTAS && T > ctas * CTA_STEPS) ctas *= 2;
  const int block = std::min(MAX_STEPS, std::max(CHUNK, (T + ctas - 1) / ctas)), chunks = (block + CHUNK - 1) / CHUNK;
  const TraceArgs a{*search,    *state, trace_tokens, trace_parents, n_best, pad, penalty, (float)(search->length_penalty - penalty), block,
                    out_tokens, out_lens, out_scores, status};
  // the limit of the largest call, once: a smaller one would lower it for a larger call made before
  constexpr int most = MAX_STEPS * 4 * (FL_BEAM_MAX + 1) + (MAX_STEPS * 2 + 4 + MAX_STEPS / CHUNK * 3) * FL_BEAM_MAX;
  FL_CUDA_TRY(fl_func_smem((const void*)beam_trace_kernel, most));
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // see pdl_wait
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3(search->n_seqs * ctas);
  cfg.blockDim = dim3(TRACE_THREADS);
  cfg.dynamicSmemBytes = block * (4 * (search->beams | 1) + search->beams) + (block + 4) * n_best + chunks * (2 * search->beams + n_best);
  cfg.stream = (cudaStream_t)stream;
  cfg.attrs = attr;
  cfg.numAttrs = ctas > 1 ? 2 : 1;
  FL_CUDA_TRY(cudaLaunchKernelEx(&cfg, beam_trace_kernel, a));
  return FL_OK;
}
