// Attention of few new tokens over the paged cache, and the entry point of all of it.
//
//   o = sum_u exp(s_u - m) v_u / sum_u exp(s_u - m),  s_u = scale q k_u,  m = max_u s_u
//
// over the keys u that a row sees, in one pass: a running maximum and sum per row (Milakov and
// Gimelshein 2018, "Online normalizer calculation for softmax"), and partial results over disjoint keys joined by
//   m = max m_i, l = sum l_i 2^(m_i - m), O = sum O_i 2^(m_i - m).
//
// A tile is 8 NR rows: (token, query head) pairs that read one key / value head.  What bounds a call with few rows
// is reading each key and value once, so nothing is staged: a warp reads 16 keys and 16 values straight from
// their page into the fragments of the warp-level tensor instruction (m16n8k16, the products are far from
// bounding anything: its pipe is busy 9% of the time), the next keys and values in flight while the last are used.  Both
// products are transposed, S^T = K Q^T and O^T = V^T P^T, so that the 8 rows are the narrow side.  The order of the dims
// inside a contraction and of the dims of O^T are free: they are chosen so that each lane reads 16
// consecutive bytes.
// One new token in each of 32 sequences of 64 to 4096 tokens, 32 key heads of 128: 984 MB read, each key and value once, in
// 147 to 149 us (6.6 TB/s); four sequences of 40001 to 65536, four key heads: 453 MB in 78 us (5.8 TB/s; the launch, plan and
// the join of each unit's parts are the rest).  A sequence of 300 takes 8.4 us, the latencies of the plan, the page table,
// the keys and the join one after another.
// P is rounded to 16 bits for its product, the sums take it unrounded: an error of half an ulp of the output's type per
// weight, independent of one another.
// Work is divided among the CTAs as kv_plan.cuh says.
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "../../include/flglm_kernels.h"
#include "common.cuh"
#include "kv_attention.cuh"
#include "kv_plan.cuh"

namespace {

constexpr int WARPS = 4, THREADS = 32 * WARPS;
constexpr int STEP = 16;              // keys a warp takes at a time (one page holds them)
constexpr int BK = WARPS * STEP;      // keys of a block
constexpr int JOIN = 8;               // parts read at a time when a unit is joined: when chosen, 453 MB in 80.3 us, one by one 82.9
constexpr int MIN_COST = 1;           // blocks that are worth a CTA: when chosen, one token over 5 MB in 9.6 us, 10.5 with 2, 14.8 with 4
constexpr float LOG2E_F = 1.4426950408889634f, LN2_F = 0.6931471805599453f;

template <class T>
FL_DEV void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <>
FL_DEV void mma16816<__nv_bfloat16>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
FL_DEV void mma16816<__half>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                             uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The transpose of an 8 x 8 matrix of 16-bit elements held two of a row per lane.
FL_DEV uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
FL_DEV uint32_t lows(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x5410); }
FL_DEV uint32_t highs(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x7632); }
FL_DEV uint4 ld_once(const void* p) {  // read once: not worth a line of L1
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

struct RowUnits {  // tiles of `tt` tokens, blocks of BK keys
  int tt;
  FL_DEV int units(const KvSeq& q) const { return (q.n + tt - 1) / tt; }
  FL_DEV int blocks(const KvSeq& q, int r) const { return (kv_sees(q, min(q.n, (r + 1) * tt) - 1) + BK - 1) / BK; }
  FL_DEV int cost(const KvSeq& q, int r) const { return blocks(q, r) + 1; }  // the ends cost about a block
};

// CTAs that an SM holds, as many as the registers allow without spilling: what they have in flight (16 KB each at head_dim
// 64, 32 at 128) hides the latency of the memory.  64 sequences of 2048 tokens, 8 key heads: at head_dim 128 up to 8 rows
// 88 us with 3 (984 MB of other sequences 150, with 2 178), up to 16 rows 107 with 2; at 64 up to 8 rows 49 with 4 (3: 56;
// 5, which spill, 48, but 27 for 23 on one long sequence), up to 16 rows 61 with 3 (2: 77).
constexpr int MAX_CTAS = 4;
constexpr int ctas_per_sm(int hd, int nr) { return (hd == 128 ? 3 : MAX_CTAS) - (nr - 1); }

template <class T, int HD, int NR>
__global__ void __launch_bounds__(THREADS, ctas_per_sm(HD, NR)) kv_attn_rows_kernel(KvAttnArgs a, int tt) {
  typedef KvIo<T> Io;
  constexpr int NJ = HD / 32;    // 16-byte pieces of a key that a lane reads
  constexpr int NH = HD / 64;    // ... of a value
  constexpr int ROWS = 8 * NR;
  constexpr int LANES = HD / 8;  // threads of a row when the warps' results are joined
  pdl_wait();  // the previous kernel on the stream has completed (see fl_launch)
  pdl_trigger();
  __shared__ int sh_last;
  __shared__ float sh_m[WARPS][ROWS], sh_l[WARPS][ROWS];
  extern __shared__ __align__(16) float sh_rows[];  // [WARPS][ROWS][HD + 4]
  auto sh_o = [&](int v, int row) { return sh_rows + (v * ROWS + row) * (HD + 4); };
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, c = lane & 3;
  const KvBatchDev& b = a.b;
  const RowUnits u{tt};
  const KvRange rg = kv_plan(b, u, a.kvh, blockIdx.x, gridDim.x, MIN_COST);
  if (rg.s < 0) return;
  const T* K = reinterpret_cast<const T*>(a.k);
  const T* V = reinterpret_cast<const T*>(a.v);
  float* part_o = a.parts;  // [cta][slot][ROWS][HD], then m and l [cta][slot][ROWS]
  float* part_ml = a.parts + (int64_t)gridDim.x * 2 * ROWS * HD;

  KvWalk<RowUnits> w;
  w.set(b, u, rg.s, rg.seq_start, rg.lo, a.kvh);
  do {
    const int nb = w.cost - 1;
    const int kb0 = (int)max((int64_t)0, rg.lo - w.start), kb1 = (int)min((int64_t)nb, rg.hi - w.start);
    if (kb0 >= kb1 && !(nb == 0 && w.start >= rg.lo && w.start < rg.hi)) continue;
    const int tok0 = w.r * tt, toks = min(tt, w.q.n - tok0), rows = toks * a.group;
    const int head0 = w.h * a.group;

    // this lane's part of the rows' queries (row g of each 8), and what each row that it holds scores of sees
    uint4 qf[NR][NJ];
    int sees[NR][2];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const int row = 8 * r + g;
      const T* qp = reinterpret_cast<const T*>(a.q) + (int64_t)(w.q.q0 + tok0 + row / a.group) * a.ldq +
                    (head0 + row % a.group) * HD + 8 * c;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
        qf[r][j] = row < rows ? *reinterpret_cast<const uint4*>(qp + 32 * j) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int sr = 8 * r + 2 * c + e;
        sees[r][e] = sr < rows ? kv_sees(w.q, tok0 + sr / a.group) : 0;
      }
    }
    const int first_sees = kv_sees(w.q, tok0), last_sees = kv_sees(w.q, tok0 + toks - 1);
    const int key_end = min(kb1 * BK, last_sees);

    float o[NR][NH][4][4], m[NR][2], l[NR][2];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      m[r][0] = m[r][1] = -INFINITY;
      l[r][0] = l[r][1] = 0.f;
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[r][h][t][e] = 0.f;
    }

    // one step of 16 keys: key g and 8 + g (all dims, 8 at c * 8 + 32 j), values 2c, 2c + 1, 8 + 2c, 8 + 2c + 1
    // (dims 8 g + 64 h)
    uint4 kf[2][NJ], vf[4][NH];
    auto base = [&](int key, int page) {
      return page * a.page_stride + w.h * a.head_stride + (key & ((1 << b.ps_log2) - 1)) * a.token_stride;
    };
    auto load_k = [&](int key, int page) {
      const T* p = K + base(key, page) + 8 * c;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const bool on = page >= 0 && key + 8 * i + g < key_end;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          kf[i][j] = on ? ld_once(p + (8 * i + g) * a.token_stride + 32 * j) : make_uint4(0, 0, 0, 0);
      }
    };
    auto load_v = [&](int key, int page) {
      const T* p = V + base(key, page) + 8 * g;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int k = (i >> 1) * 8 + 2 * c + (i & 1);
        const bool on = page >= 0 && key + k < key_end;
#pragma unroll
        for (int h = 0; h < NH; ++h) vf[i][h] = on ? ld_once(p + k * a.token_stride + 64 * h) : make_uint4(0, 0, 0, 0);
      }
    };
    auto page_of = [&](int key) { return key < key_end ? kv_page(b, w.s, key >> b.ps_log2) : -1; };

    int key = kb0 * BK + warp * STEP;
    int page = page_of(key), page_n = page_of(key + BK);
    load_k(key, page);
    load_v(key, page);
    for (; key < key_end; key += BK) {
      // S^T of the keys in place; then the next step's keys are asked for
      float s[NR][4];
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        s[r][0] = s[r][1] = s[r][2] = s[r][3] = 0.f;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          mma16816<T>(s[r], kf[0][j].x, kf[1][j].x, kf[0][j].y, kf[1][j].y, qf[r][j].x, qf[r][j].y);
          mma16816<T>(s[r], kf[0][j].z, kf[1][j].z, kf[0][j].w, kf[1][j].w, qf[r][j].z, qf[r][j].w);
        }
      }
      const int page_nn = page_of(key + 2 * BK);
      load_k(key + BK, page_n);
      // scaled scores (log2 units); keys past what a row sees become -inf (s[r][2 i + e]: key 8 i + g, row 2 c + e)
      bool grows = false;
#pragma unroll
      for (int r = 0; r < NR; ++r) {
#pragma unroll
        for (int x = 0; x < 4; ++x) s[r][x] *= a.scale_log2;
        if (key + STEP > first_sees) {
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if (key + 8 * (x >> 1) + g >= sees[r][x & 1]) s[r][x] = -INFINITY;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) grows |= fmaxf(s[r][e], s[r][2 + e]) > m[r][e] + 8.f;
      }
      // The reference that the exponents are taken from follows the row's maximum only when that has
      // grown by more than 2^8: p stays below 2^8, the sums lose nothing, and few steps rescale.
      if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
        for (int r = 0; r < NR; ++r) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float t = fmaxf(s[r][e], s[r][2 + e]);
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, x));
            t = fmaxf(t, m[r][e]);
            const float f = m[r][e] == -INFINITY ? 0.f : exp2_hw(m[r][e] - t);
            m[r][e] = t;
            l[r][e] *= f;
#pragma unroll
            for (int h = 0; h < NH; ++h)
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                o[r][h][x][e] *= f;
                o[r][h][x][2 + e] *= f;
              }
          }
        }
      }
      // P^T, rounded to the type of the tensor instruction; the sums take it unrounded
      uint32_t p[NR][2];
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        const float m0 = m[r][0] == -INFINITY ? 0.f : m[r][0], m1 = m[r][1] == -INFINITY ? 0.f : m[r][1];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float p0 = exp2_hw(s[r][2 * i] - m0), p1 = exp2_hw(s[r][2 * i + 1] - m1);
          l[r][0] += p0;
          l[r][1] += p1;
          p[r][i] = transpose8x8(Io::pack(p0, p1));
        }
      }
      // Rows that do not see a key have p = 0 for it, which only a finite value makes a term of zero: where
      // rows differ in what they see, infinities and NaN are looked for, and such a step goes key by key.
      bool odd = false;
      if (key + STEP > first_sees && first_sees < last_sees) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int h = 0; h < NH; ++h)
            odd |= !Io::finite(vf[i][h].x) || !Io::finite(vf[i][h].y) || !Io::finite(vf[i][h].z) || !Io::finite(vf[i][h].w);
        odd = __any_sync(0xffffffffu, odd);
      }
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        const uint32_t v0[4] = {vf[0][h].x, vf[0][h].y, vf[0][h].z, vf[0][h].w};
        const uint32_t v1[4] = {vf[1][h].x, vf[1][h].y, vf[1][h].z, vf[1][h].w};
        const uint32_t v2[4] = {vf[2][h].x, vf[2][h].y, vf[2][h].z, vf[2][h].w};
        const uint32_t v3[4] = {vf[3][h].x, vf[3][h].y, vf[3][h].z, vf[3][h].w};
#pragma unroll
        for (int t = 0; t < 4; ++t) {  // dims 8 g + 64 h + 2 t (rows g of the fragment) and + 1 (rows g + 8)
          const uint32_t a0 = lows(v0[t], v1[t]), a1 = highs(v0[t], v1[t]), a2 = lows(v2[t], v3[t]),
                         a3 = highs(v2[t], v3[t]);
          if (!odd) {
#pragma unroll
            for (int r = 0; r < NR; ++r) mma16816<T>(o[r][h][t], a0, a1, a2, a3, p[r][0], p[r][1]);
          } else {
#pragma unroll 1
            for (int i = 0; i < STEP; ++i) {
              const uint32_t at = (i & 7) >> 1 == c ? (i & 1 ? 0xffff0000u : 0xffffu) : 0u;  // key i's half, in its lanes
              const uint32_t lo = i < 8 ? at : 0u, hi = i < 8 ? 0u : at;
#pragma unroll
              for (int r = 0; r < NR; ++r) {
                float y[4] = {0.f, 0.f, 0.f, 0.f};
                mma16816<T>(y, a0 & lo, a1 & lo, a2 & hi, a3 & hi, p[r][0], p[r][1]);
#pragma unroll
                for (int x = 0; x < 4; ++x)
                  if (key + i < sees[r][x & 1]) o[r][h][t][x] += y[x];
              }
            }
          }
        }
      }
      load_v(key + BK, page_n);
      page_n = page_nn;
    }

    // the sums of a row over its keys (lanes of equal c hold the same rows)
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[r][e] += __shfl_xor_sync(0xffffffffu, l[r][e], x);
      }
    // ---- the warps' results joined
    __syncthreads();  // the last unit's have been read
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int row = 8 * r + 2 * c + e;
        if (g == 0) {
          sh_m[warp][row] = m[r][e];
          sh_l[warp][row] = l[r][e];
        }
#pragma unroll
        for (int h = 0; h < NH; ++h) {
          float* d = sh_o(warp, row) + 64 * h + 8 * g;
#pragma unroll
          for (int t = 0; t < 4; t += 2)
            *reinterpret_cast<float4*>(d + 2 * t) =
                make_float4(o[r][h][t][e], o[r][h][t][2 + e], o[r][h][t + 1][e], o[r][h][t + 1][2 + e]);
        }
      }
    __syncthreads();
    const bool whole = kb0 == 0 && kb1 == nb;
    const int d0 = 8 * (tid % LANES);
    auto finish = [&](int row, float mr, float lr, const float (&x)[8]) {
      const int64_t t = w.q.q0 + tok0 + row / a.group;
      const int h = head0 + row % a.group;
      const float inv = lr > 0.f ? 1.f / lr : lr == 0.f ? 0.f : lr;  // a sum that is NaN stays one
      T* dst = reinterpret_cast<T*>(a.o) + t * a.ldo + h * HD + d0;
      uint32_t y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = Io::pack(x[2 * i] * inv, x[2 * i + 1] * inv);
      *reinterpret_cast<uint4*>(dst) = make_uint4(y[0], y[1], y[2], y[3]);
      if (a.lse && d0 == 0) a.lse[(int64_t)h * b.T + t] = lr == 0.f ? -INFINITY : (mr + log2f(lr)) * LN2_F;
    };
    const int slot = 2 * blockIdx.x + (kb0 == 0);
#pragma unroll
    for (int r0 = 0; r0 < ROWS; r0 += THREADS / LANES) {
      const int row = r0 + tid / LANES;
      if (row >= rows) continue;
      float mr = -INFINITY, lr = 0.f, x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = 0.f;
#pragma unroll
      for (int v = 0; v < WARPS; ++v) mr = fmaxf(mr, sh_m[v][row]);
#pragma unroll
      for (int v = 0; v < WARPS; ++v) {  // no key in sight, or only NaN scores: sums of 0, or NaN, which a factor of 0 keeps
        const float f = sh_m[v][row] == -INFINITY ? 0.f : exp2_hw(sh_m[v][row] - mr);
        lr += sh_l[v][row] * f;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] += sh_o(v, row)[d0 + i] * f;
      }
      if (whole) {
        finish(row, mr, lr, x);
      } else {
        float* d = part_o + ((int64_t)slot * ROWS + row) * HD + d0;
        __stcg(reinterpret_cast<float4*>(d), make_float4(x[0], x[1], x[2], x[3]));
        __stcg(reinterpret_cast<float4*>(d) + 1, make_float4(x[4], x[5], x[6], x[7]));
        if (d0 == 0) __stcg(reinterpret_cast<float2*>(part_ml) + (int64_t)slot * ROWS + row, make_float2(mr, lr));
      }
    }
    if (whole) continue;
    // ---- a unit in parts: the CTA that is done last joins them in their order
    const int f0 = rg.cta_of(w.start), f1 = rg.cta_of(w.start + nb - 1);
    __syncthreads();
    if (tid == 0) sh_last = kv_part_done(a.counters + f0, f1 - f0 + 1);
    __syncthreads();
    if (!sh_last) continue;
#pragma unroll
    for (int r0 = 0; r0 < ROWS; r0 += THREADS / LANES) {
      const int row = r0 + tid / LANES;
      if (row >= rows) continue;
      float mr = -INFINITY, lr = 0.f, x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = 0.f;
      for (int fb = f0; fb <= f1; fb += JOIN) {  // some at a time: the reads wait together
        float2 ml[JOIN];
        float4 y[JOIN][2];
#pragma unroll
        for (int e = 0; e < JOIN; ++e) {
          const int f = min(fb + e, f1);
          const int64_t at = (int64_t)(2 * f + (f == f0)) * ROWS + row;
          ml[e] = __ldcg(reinterpret_cast<const float2*>(part_ml) + at);
          y[e][0] = __ldcg(reinterpret_cast<const float4*>(part_o + at * HD + d0));
          y[e][1] = __ldcg(reinterpret_cast<const float4*>(part_o + at * HD + d0) + 1);
          if (fb + e > f1) {
            ml[e] = make_float2(-INFINITY, 0.f);
            y[e][0] = y[e][1] = make_float4(0.f, 0.f, 0.f, 0.f);
          }
        }
#pragma unroll
        for (int e = 0; e < JOIN; ++e) {
          const float z[8] = {y[e][0].x, y[e][0].y, y[e][0].z, y[e][0].w, y[e][1].x, y[e][1].y, y[e][1].z, y[e][1].w};
          const float mn = fmaxf(mr, ml[e].x);
          const float fo = mr == -INFINITY ? 0.f : exp2_hw(mr - mn), fn = ml[e].x == -INFINITY ? 0.f : exp2_hw(ml[e].x - mn);
          mr = mn;
          lr = lr * fo + ml[e].y * fn;
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = x[i] * fo + z[i] * fn;
        }
      }
      finish(row, mr, lr, x);
    }
  } while (w.next(b, u, a.kvh) && w.start < rg.hi);
}

// Rows of a sequence and key head that the warp-level fragments hold in one tile.  More go to the tensor-core tiles of
// 128.  64 sequences of 2048 tokens, 8 key heads of 128, here and there: 8 rows 88 and 105 us, 16 rows 107 and 108; one
// such sequence 12.7 and 20.3, 17.9 and 21.3; 200 of 100 tokens 33 and 47, 48 and 50; at head_dim 64 61 and 92 with 16
// rows.  With 32 rows two tiles would read the keys twice: 257 and 107.
bool few_rows(int group, int max_new) { return (int64_t)group * max_new <= 16; }

template <class T, int HD, int NR>
int launch_rows(const KvAttnArgs& a, cudaStream_t st) {
  const int tt = 8 * NR / a.group, smem = WARPS * 8 * NR * (HD + 4) * (int)sizeof(float);
  FL_CUDA_TRY(fl_func_smem((const void*)kv_attn_rows_kernel<T, HD, NR>, smem));
  FL_CUDA_TRY(fl_launch(kv_attn_rows_kernel<T, HD, NR>, dim3(ctas_per_sm(HD, NR) * fl_sm_count()), dim3(THREADS), smem, st, a, tt));
  return FL_OK;
}
template <class T>
int dispatch_rows(int hd, int nr, const KvAttnArgs& a, cudaStream_t st) {
  if (hd == 128) return nr == 1 ? launch_rows<T, 128, 1>(a, st) : launch_rows<T, 128, 2>(a, st);
  return nr == 1 ? launch_rows<T, 64, 1>(a, st) : launch_rows<T, 64, 2>(a, st);
}

}  // namespace

extern "C" size_t fl_k_kv_attention_workspace(int32_t n_heads, const fl_kv_cache* cache, const fl_kv_batch* batch) {
  KvBatchDev bt;
  if (fl_kv_check("kv attention", cache, batch, n_heads, &bt)) return 0;
  const int group = n_heads / cache->kv_heads;
  if (group > 128) {
    fl_internal_error(FL_ERR_UNSUPPORTED, "kv attention: %d query heads per key head", group);
    return 0;
  }
  // enough for either kernel, so that it fits every batch of the cache
  const size_t rows = (size_t)MAX_CTAS * fl_sm_count() * 2 * 16 * (cache->head_dim + 2) * sizeof(float);
  return KV_COUNTERS * sizeof(unsigned) + std::max(rows, fl_kv_attention_tc_parts(cache->head_dim));
}

extern "C" int fl_k_kv_attention(const fl_kv_cache* cache, const fl_kv_batch* batch, int32_t n_heads, const void* q,
                                 int64_t ldq, float scale, const int32_t* context_lens, void* o, int64_t ldo,
                                 float* lse, void* workspace, int* status, void* stream) {
  KvAttnArgs a;
  if (int rc = fl_kv_check("kv attention", cache, batch, n_heads, &a.b)) return rc;
  if (!q || !o || !workspace || !status || !std::isfinite(scale) || fl_misaligned(q, 16) || fl_misaligned(o, 16) ||
      fl_misaligned(workspace, 16) || fl_misaligned(lse, 4) || fl_misaligned(status, 4) || fl_misaligned(context_lens, 4))
    return fl_internal_error(FL_ERR_INVALID_ARG, "kv attention: args");
  if (ldq % 8 || ldo % 8 || ldq < 0 || ldo < 0)
    return fl_internal_error(FL_ERR_UNSUPPORTED, "kv attention: ldq and ldo must be multiples of 8, not negative");
  a.group = n_heads / cache->kv_heads;
  if (a.group > 128) return fl_internal_error(FL_ERR_UNSUPPORTED, "kv attention: %d query heads per key head", a.group);
  if (batch->n_tokens == 0) return FL_OK;
  a.b.ctx = context_lens;
  a.q = q;
  a.k = cache->k;
  a.v = cache->v;
  a.o = o;
  a.ldq = ldq;
  a.ldo = ldo;
  a.page_stride = cache->page_stride;
  a.head_stride = cache->head_stride;
  a.token_stride = cache->token_stride;
  a.kvh = cache->kv_heads;
  a.lse = lse;
  a.scale_log2 = (scale == 0.f ? 1.f / sqrtf((float)cache->head_dim) : scale) * LOG2E_F;
  a.counters = (unsigned*)workspace;
  a.parts = (float*)((unsigned*)workspace + KV_COUNTERS);
  a.b.status = status;
  if (!few_rows(a.group, batch->max_new)) return fl_launch_kv_attention_tc(cache, a, n_heads, (cudaStream_t)stream);
  const int rows = batch->max_new * a.group;
  return (cache->dtype == FL_DT_F16 ? dispatch_rows<__half> : dispatch_rows<__nv_bfloat16>)(
      cache->head_dim, rows <= 8 && a.group <= 8 ? 1 : 2, a, (cudaStream_t)stream);
}
