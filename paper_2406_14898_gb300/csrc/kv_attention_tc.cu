// Attention of chunks of new tokens over the paged cache on the 5th-generation tensor cores.
//
// A tile is 128 rows, (token, query head) pairs of the query heads that share one key / value head, and key blocks of
// 128.  One CTA per SM runs two streams, each a tile's softmax over key blocks:
//   two tiles of a unit over the same blocks (each key block is read once for 256 rows), or
//   where a unit has one tile, that tile over the even and over the odd blocks, joined at the end.
//
//   warps 0-3, 4-7  softmax of stream 0 and 1: thread i owns row i (TMEM lane i): reads its 128 scores, takes
//                   p = 2^(s - m), writes p (16 bits) to TMEM; at the end O / l, or a part of it
//   warp 8          which units the CTA takes, told to the others a few ahead; TMA: K and V blocks page by page into a
//                   ring of stages, Q tiles
//   warps 9, 10     a stream each: S = Q K^T (both in shared memory), O += P V (P in TMEM, V as an MN-major operand)
//   warp 11         makes V blocks fit for weights of zero (see there) before anyone uses them
//
// TMEM: S of the streams at columns 0 and 128, O at 256.  P lies over its S at head_dim 128 (512 columns are
// taken), so the next S of a stream waits for its P V; at head_dim 64 it has columns of its own.
// A block of shared memory is [16 groups of 8 rows][head_dim / 64][8 rows][64 columns] in the 128-byte
// swizzle, so that one copy brings all columns of a page's rows.
// m follows a row's maximum only when that grew by more than 2^8, so O is seldom rescaled.  p is rounded to 16 bits, the type
// of the tensor instruction's operands; l sums it unrounded, in fp32 as O.
// Work is divided among the CTAs as kv_plan.cuh says.
//
// 2048 new tokens behind 27953, 32 query heads on 8: 0.97 TFLOP in 705 us (1.38 PFLOP/s; single calls 655, 1.48, before the
// card is at its power limit, the tensor pipe busy 62% of the time); 16 prompts of 72 to 979 tokens, 32 heads each with its
// own keys, 157 us (0.68 PFLOP/s); 8 chunks of 256 tokens after up to 2044, 70 us.  What bounds it is a stream's chain: scores, weights (two passes over 128 scores, an exponential each),
// products, about 3100 cycles a block of two streams where the products alone take 2048; a short unit adds its
// ends.  Short code counts: while a role waits its instructions leave the cache, so loops of 64 columns stay rolled, and
// what is rare is marked as unlikely to keep it out of their lines (776 to 767 us when that was done).
//
// Every wait is bounded.  A warp whose wait ran out records it and, in a role that issues, leaves; a softmax warp goes
// through the rest of its unit without waiting, and its warpgroup then leaves together.
#include <cuda.h>

#include <cmath>

#include "../../include/flglm_kernels.h"
#include "common.cuh"
#include "gemm_tc.cuh"
#include "kv_attention.cuh"
#include "ptx.cuh"

namespace {

constexpr int TB = 128;
constexpr int THREADS = 384, W_TMA = 8, W_MMA = 9, W_FIX = 11;
// Cost of a unit's ends (Q, the first scores, the output), in blocks of one tile: 16 prompts of 72 to 979 tokens in 157.5 us
// with 5, 159 with 4; before the streams took turns 162.5 with 4, 187 with 1, 165 with 8, and 8 chunks of 256 tokens 75.9, 84.7
// and 78.
constexpr int ENDS = 5;
constexpr int MIN_COST = 4;  // worth a CTA: when chosen, 12 small sequences in 26.9 us, with 10 in 29.2, with 1 as with 4
constexpr float LN2_F = 0.6931471805599453f;

template <int HD>
struct Cfg {
  static constexpr int NB = HD / 64;
  static constexpr int TILE = TB * HD * 2;
  // stages: what 227 KB hold beside two Q tiles (those prompts with 4 in 169.6 us), 8 at head_dim 64
  static constexpr int ST = HD == 128 ? 5 : 8;
  static constexpr int CTRL = 2048;
  static constexpr int SMEM = (2 + ST) * TILE + CTRL + 1024;
  static constexpr bool OWN_P = HD == 64;
};
static_assert(Cfg<128>::SMEM <= 227 * 1024 && Cfg<64>::SMEM <= 227 * 1024, "shared memory");

struct TcMaps {
  CUtensorMap q, k, v;
};
struct TcGeom {
  int tpt;               // tokens of a tile
  int box_rows;          // rows that one copy brings: a page's, 128 at most
  int by_head, per_page;  // coordinates of page p, head h: (0, p * per_page + h) or, heads side by side, (h * NB, p)
};

// 5-D tiled load of a page's rows.
FL_DEV void tma_load_5d(void* dst, const CUtensorMap* m, uint64_t* bar, int c2, int c3, int c4) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %3, %4, %5, %6}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(bar)), "r"(0), "r"(c2), "r"(c3), "r"(c4)
      : "memory");
}
FL_DEV void tma_load_3d(void* dst, const CUtensorMap* m, uint64_t* bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}
// A value that is the same in the whole warp, as one that the compiler knows to be: the tensor instructions take
// their operands from uniform registers, and moving them there one by one costs more than the product.
FL_DEV uint32_t uniform(uint32_t x) { return __shfl_sync(0xffffffffu, x, 0); }
FL_DEV void bar_sync(int id, int threads) { asm volatile("barrier.cta.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
FL_DEV bool bar_or(int id, int threads, bool x) {
  uint32_t y;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 q, %1, 0;\n\t"
      "barrier.cta.red.or.pred p, %2, %3, q;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(y)
      : "r"((uint32_t)x), "r"(id), "r"(threads)
      : "memory");
  return y != 0;
}

// Two fp32 operations an instruction.
FL_DEV float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\t"
      "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
FL_DEV float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\t"
      "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

template <class T>
constexpr uint32_t idesc(int N, bool b_mn) {  // fp16 operands: format 0 in place of bf16's 1
  return umma_idesc_bf16(TB, N, false, b_mn) & (sizeof(T) == 2 && KvIo<T>::is_half ? ~((1u << 7) | (1u << 10)) : ~0u);
}

struct TileUnits {
  int tpt;
  FL_DEV int units(const KvSeq& q) const { return (q.n + 2 * tpt - 1) / (2 * tpt); }
  FL_DEV bool two(const KvSeq& q, int r) const { return q.n - r * 2 * tpt > tpt; }
  FL_DEV int blocks(const KvSeq& q, int tok_end) const { return (kv_sees(q, min(q.n, tok_end) - 1) + TB - 1) / TB; }
  FL_DEV int cost(const KvSeq& q, int r) const {
    return (two(q, r) ? 2 : 1) * blocks(q, (r + 1) * 2 * tpt) + ENDS;
  }
};

// What a CTA does of a unit: key blocks [kb0, kb0 + n), of which stream s takes part in na[s].
struct Piece {
  int n, two, end, zero;        // end: no unit any more; zero: the streams (bits) whose rows see nothing at all
  int q0, h, toks[2];           // first row of Q, key / value head, tokens of each tile
  int kb0, kmax, nb[2], na[2];  // kmax: keys that some row sees; nb: blocks of the unit's tiles
  int vis, ctx, L;              // token i of the unit sees the first max(0, min(L, max(vis + i, ctx))) keys
  int f_lo, f_hi[2];            // CTAs that have parts of it
  FL_DEV int sees(int i) const { return max(0, min(L, max(vis + i, ctx))); }
  // Streams that compute their weights at the same time wait for their products at the same time, and some CTAs stay so to
  // the end, a fifth behind the others.  So in the blocks that both take part in, a stream's next scores are begun only when
  // the other one has found the maxima of the block before them: where the streams already alternate that has happened.
  // 2048 tokens behind 27953, single calls: 655 us, without turns 767; turns told before the maxima 721, behind the first
  // weights 900.
  FL_DEV int turns() const { return two ? na[0] : 0; }
};
constexpr int PIECES = 4;  // told ahead
FL_DEV Piece piece_of(const TileUnits& u, const KvWalk<TileUnits>& k, const KvRange& g) {
  Piece p;
  const int tok0 = k.r * 2 * u.tpt, left = k.q.n - tok0;
  p.end = 0;
  p.two = u.two(k.q, k.r);
  p.q0 = k.q.q0 + tok0;
  p.h = k.h;
  p.toks[0] = min(u.tpt, left);
  p.toks[1] = p.two ? min(u.tpt, left - u.tpt) : p.toks[0];
  p.vis = k.q.L - k.q.n + tok0 + 1;
  p.ctx = k.q.ctx;
  p.L = k.q.L;
  p.kmax = kv_sees(k.q, min(k.q.n, tok0 + 2 * u.tpt) - 1);
  p.nb[1] = (p.kmax + TB - 1) / TB;
  p.nb[0] = p.two ? u.blocks(k.q, tok0 + u.tpt) : p.nb[1];
  const int sh = p.two;  // a block of two tiles costs two
  p.kb0 = (int)max((int64_t)0, (g.lo - k.start + sh) >> sh);
  const int kb1 = (int)min((int64_t)p.nb[1], (g.hi - k.start + sh) >> sh);
  p.n = max(0, kb1 - p.kb0);
  p.na[0] = p.two ? min(p.n, max(0, p.nb[0] - p.kb0)) : (p.n + 1) / 2;
  p.na[1] = p.two ? p.n : p.n / 2;
  const bool first = k.start >= g.lo && k.start < g.hi;
  p.zero = first ? (p.nb[0] == 0 ? 1 : 0) | (p.two && p.nb[1] == 0 ? 2 : 0) : 0;
  p.f_lo = p.f_hi[0] = p.f_hi[1] = 0;
  if (p.n > 0 && p.n < p.nb[1]) {
    p.f_lo = g.cta_of(k.start);
    for (int s = 0; s < 2; ++s)
      if (p.nb[s] > 0) p.f_hi[s] = g.cta_of(k.start + ((int64_t)(p.nb[s] - 1) << sh));
  }
  return p;
}
// Place in the ring, from the piece's first stage on, of block t's values: keys of la blocks lie first, then each
// block's values and the keys la blocks further.
struct RingOrder {
  int n, la;
  FL_DEV int v(int t) const { return min(n, la) + t + min(t, max(n - la, 0)); }
};

// The rest of a wait whose first try ran out; one copy, the many places that wait keep short.
__device__ __noinline__ bool wait_longer(uint64_t* bar, uint32_t parity) { return mbar_wait_warp(bar, parity); }

// A row's scores scaled and rounded in place.  m is a rounded product: where it is huge, an unrounded product less m would
// be what it was rounded by, which is no exponent.
__device__ __noinline__ void round_scores(uint32_t t_s, float scale) {
  __syncwarp();
#pragma unroll 1
  for (int c = 0; c < TB; c += 32) {
    uint32_t r[32];
    tmem_ld32(t_s + c, r);
    tmem_ld_wait();
#pragma unroll
    for (int e = 0; e < 32; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * scale);
    tmem_st32(t_s + c, r);
  }
  tmem_st_wait();
}

// O += P V of one block without the tensor cores, for blocks whose values include infinities or NaN at keys that some
// row does not see: the row takes the keys that it sees.  P and O in TMEM, the block in shared memory.
template <class T, int HD>
__device__ __noinline__ void slow_pv(uint32_t t_p, uint32_t t_o, const uint8_t* sV, int sees, bool first) {
  constexpr int NB = HD / 64;
#pragma unroll 1
  for (int d = 0; d < HD; d += 16) {
    uint32_t o[16];
    tmem_ld16(t_o + d, o);
    tmem_ld_wait();
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = first ? 0.f : __uint_as_float(o[i]);
#pragma unroll 1
    for (int k0 = 0; k0 < TB; k0 += 32) {
      uint32_t p[16];
      __syncwarp();
      tmem_ld16(t_p + k0 / 2, p);
      tmem_ld_wait();
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        const int k = k0 + e;
        const float2 pp = KvIo<T>::unpack(p[e / 2]);
        const float pk = e & 1 ? pp.y : pp.x;
        const uint8_t* row = sV + (k >> 3) * NB * 1024 + (d >> 6) * 1024 + (k & 7) * 128;
        const int c = (d & 63) >> 3;
        if (k < sees) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint4 y = *reinterpret_cast<const uint4*>(row + (((c + h) ^ (k & 7)) << 4));
            const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 v = KvIo<T>::unpack(w[i]);
              x[8 * h + 2 * i] = fmaf(pk, v.x, x[8 * h + 2 * i]);
              x[8 * h + 2 * i + 1] = fmaf(pk, v.y, x[8 * h + 2 * i + 1]);
            }
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(x[i]);
    __syncwarp();
    tmem_st16(t_o + d, o);
  }
  tmem_st_wait();
}

template <class T, int HD>
__global__ void __launch_bounds__(THREADS, 1)
    kv_attn_tc_kernel(const __grid_constant__ TcMaps maps, const __grid_constant__ KvAttnArgs a, TcGeom geo) {
  typedef Cfg<HD> C;
  typedef KvIo<T> Io;
  constexpr int NB = C::NB, TILE = C::TILE, ST = C::ST;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = smem;
  uint8_t* sKV = smem + 2 * TILE;
  uint8_t* ctrl = sKV + ST * TILE;
  uint64_t* bars = reinterpret_cast<uint64_t*>(ctrl);
  enum {
    B_FULL = 0,              // a stage's copy has arrived
    B_READY = ST,            // and warp 11 has seen to it
    B_EMPTY = 2 * ST,        // both streams are done with it
    B_QF = 3 * ST, B_QE = B_QF + 2,
    B_S = B_QE + 2,          // scores of a stream
    B_PH = B_S + 2, B_P = B_PH + 2,  // the first half of its weights, all of them
    B_O = B_P + 2,           // its P V so far
    B_FREE = B_O + 2,        // its O has been read
    B_JOIN = B_FREE + 2,     // stream 1's part of a tile is ready for stream 0
    B_TURN = B_JOIN + 1,     // a stream knows a block's maxima (see turns)
    B_PIECE = B_TURN + 2, B_PDONE = B_PIECE + PIECES,
    B_END = B_PDONE + PIECES,
    BARS = B_END + 2
  };
  static_assert(BARS * 8 <= 528 && sizeof(Piece) * PIECES <= 384, "control block");
  volatile int* sh_flag = reinterpret_cast<volatile int*>(ctrl + 528);  // [0, 2) slow block, [2, 4) last part, [4] failed
  volatile int* sh_odd = sh_flag + 8;                                   // [stage] the block has infinities or NaN
  uint32_t* holder = reinterpret_cast<uint32_t*>(ctrl + 592);
  Piece* pieces = reinterpret_cast<Piece*>(ctrl + 640);
  float2* sh_ml = reinterpret_cast<float2*>(ctrl + 1024);               // stream 1's m and l when it is joined (1 KB)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const KvBatchDev& b = a.b;

  if (tid == 0) {
    for (int i = 0; i < BARS; ++i) {
      const bool four = (i >= B_PH && i < B_O) || (i >= B_FREE && i < B_PIECE);  // the softmax warps of a stream
      const bool both = (i >= B_EMPTY && i < B_QF) || (i >= B_QE && i < B_S);
      mbar_init(bars + i, four ? 4 : both ? 2 : i >= B_PDONE && i < B_END ? 11 : 1);
    }
    fence_mbar_init();
    for (int i = 0; i < 5; ++i) sh_flag[i] = 0;
    tma_prefetch_desc(&maps.q);
    tma_prefetch_desc(&maps.k);
    tma_prefetch_desc(&maps.v);
  }
  if (warp == W_MMA) {
    tmem_alloc(holder, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *holder;
  pdl_wait();  // the previous kernel on the stream has completed (see fl_launch)
  pdl_trigger();

  const TileUnits u{geo.tpt};
  bool ok = true;
  // by a whole warp; phase: the number of the barrier's phase waited for
  auto wait = [&](int i, uint32_t phase) {
    if (__all_sync(0xffffffffu, mbar_try_wait(smem_u32(bars + i), phase & 1))) return ok;
    if (ok && !wait_longer(bars + i, phase & 1)) {
      ok = false;
      sh_flag[4] = 1;
      atomicOr(b.status, FL_KV_TIMEOUT);
    }
    return ok;
  };
  uint32_t ring = 0, qi = 0;  // stages and Q tiles (a ring of two) used so far
  uint32_t np = 0;            // pieces so far
  auto piece_done = [&]() {   // the piece has been read
    __syncwarp();
    if (lane == 0) mbar_arrive(bars + B_PDONE + np % PIECES);
    ++np;
  };

  if (warp < 8) {
    const int s = warp >> 2, row = tid & 127;
    const uint32_t t_lane = tmem + (uint32_t((warp & 3) * 32) << 16);
    const uint32_t t_s = t_lane + s * TB, t_o = t_lane + 256 + s * HD, t_p = C::OWN_P ? t_lane + 384 + s * 64 : t_s;
    const int my_tok = row / a.group, my_head = row % a.group;  // inside the tile
    uint32_t ss = 0, pv = 0, uses = 0, joins = 0;
    bool slow_before = false;
    const float scale = fabsf(a.scale_log2);
    const uint32_t flip = a.scale_log2 < 0.f ? 0x80000000u : 0u;
    float4* part_o = reinterpret_cast<float4*>(a.parts);
    float2* part_ml = reinterpret_cast<float2*>(a.parts + (int64_t)gridDim.x * 4 * TB * HD);
    const bool o32 = ((reinterpret_cast<uintptr_t>(a.o) | (uintptr_t)(a.ldo * 2)) & 31) == 0;  // rows in whole sectors
    auto arrive = [&](int i) {  // behind this warp's accesses of TMEM
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bars + i);
    };
    while (true) {
      // the whole warpgroup goes on, or none of it
      if (bar_or(1 + s, 128, !wait(B_PIECE + np % PIECES, np / PIECES))) break;
      const Piece p = pieces[np % PIECES];
      piece_done();
      if (p.end) break;
      const RingOrder ro{p.n, p.two ? 1 : 2};
      const uint32_t base = ring;  // the piece's first stage
      ring += 2 * p.n;
      const int tok = p.two && s ? geo.tpt : 0, rows = (s ? p.toks[1] : p.toks[0]) * a.group;
      const bool valid = row < rows, on = (warp & 3) * 32 < rows;
      const int sees = valid ? p.sees(tok + my_tok) : 0, first_sees = p.sees(tok);
      const int turns = p.turns();
      const int nb = s ? p.nb[1] : p.nb[0], mine = s ? p.na[1] : p.na[0], f_hi = s ? p.f_hi[1] : p.f_hi[0];
      const int64_t t_row = p.q0 + tok + my_tok;
      const int head = p.h * a.group + my_head;
      if (mine == 0 && !((p.zero >> s) & 1)) continue;
      float m = -INFINITY, l = 0.f;
#pragma unroll 1
      for (int j = 0; j < mine; ++j) {
        const int t = p.two ? j : 2 * j + s, kb = (p.kb0 + t) * TB;
        const bool masks = !__all_sync(0xffffffffu, kb + TB <= sees) || a.scale_log2 < 0.f;
        const bool mixed = first_sees < min(kb + TB, p.kmax);
        wait(B_S + s, ss++);
        tc_fence_after();
        // a block where some row does not see a key that another does, and whose values are not all finite, is taken
        // without the tensor cores
        const uint32_t vi = base + ro.v(t), vst = vi % ST;
        bool slow = false;
        if (mixed) [[unlikely]] {
          wait(B_READY + vst, vi / ST);
          slow = sh_odd[vst] != 0;
        }
        if (slow != slow_before && row == 0) sh_flag[s] = slow;
        slow_before = slow;
        if (on) {
          if (masks) [[unlikely]] {  // keys not seen become -inf
#pragma unroll 1
            for (int c = 0; c < TB; c += 32) {
              uint32_t r[32];
              tmem_ld32(t_s + c, r);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 32; ++e) r[e] = kb + c + e >= sees ? 0xff800000u : r[e] ^ flip;
              tmem_st32(t_s + c, r);
            }
            tmem_st_wait();
          }
          // 64 columns at a time in loops that stay loops: the code is fetched once, and S is read twice at little cost
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
          for (int c = 0; c < TB; c += 64) {
            uint32_t r[64];
            tmem_ld32(t_s + c, *reinterpret_cast<uint32_t(*)[32]>(r));
            tmem_ld32(t_s + c + 32, *reinterpret_cast<uint32_t(*)[32]>(r + 32));
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 64; e += 8)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                mx[i] = fmaxf(fmaxf(mx[i], __uint_as_float(r[e + 2 * i])), __uint_as_float(r[e + 2 * i + 1]));
          }
          const float mt = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale;
          // below 2^24 the rounding of m is half a unit of the exponent at most, and the same for all of a row's keys
          const bool grows = mt > m + 8.f, huge = fabsf(mt) >= 0x1p24f && fabsf(mt) < INFINITY;
          float left = scale;  // what scores are still to be multiplied by
          if (j < turns) arrive(B_TURN + s);
          if (__any_sync(0xffffffffu, grows || huge)) [[unlikely]] {
            if (__any_sync(0xffffffffu, huge)) [[unlikely]] {
              round_scores(t_s, scale);
              left = 1.f;
            }
            const float mn = grows ? mt : m, f = m == -INFINITY ? 0.f : exp2_hw(m - mn);
            const float corr = grows ? f : 1.f;
            m = mn;
            l *= corr;
            if (j > 0) {
              wait(B_O + s, pv + j - 1);  // the products so far
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < HD; c += 32) {
                uint32_t o[32];
                tmem_ld32(t_o + c, o);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * corr);
                tmem_st32(t_o + c, o);
              }
            }
          }
          const float mref = m == -INFINITY ? 0.f : m;
          const float2 sc = make_float2(left, left), nm = make_float2(-mref, -mref);
          float2 lt[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll 1
          for (int c = 0; c < TB; c += 64) {
            uint32_t r[64];
            tmem_ld32(t_s + c, *reinterpret_cast<uint32_t(*)[32]>(r));
            tmem_ld32(t_s + c + 32, *reinterpret_cast<uint32_t(*)[32]>(r + 32));
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              const float2 x = fma2(make_float2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])), sc, nm);
              const float2 y = make_float2(exp2_hw(x.x), exp2_hw(x.y));
              lt[i & 1] = add2(lt[i & 1], y);
              r[i] = Io::pack(y.x, y.y);
            }
            tmem_st32(t_p + c / 2, *reinterpret_cast<uint32_t(*)[32]>(r));
            tmem_st_wait();
            if (c == 0 && !slow) arrive(B_PH + s);
          }
          lt[0] = add2(lt[0], lt[1]);
          l += lt[0].x + lt[0].y;
        } else {
          if (!slow) arrive(B_PH + s);
          if (j < turns) arrive(B_TURN + s);
        }
        if (slow) [[unlikely]] {
          if (j > 0) wait(B_O + s, pv + j - 1);
          else if (uses > 0) wait(B_FREE + s, uses - 1);
          tc_fence_after();
          __syncwarp();
          if (on) slow_pv<T, HD>(t_p, t_o, sKV + vst * TILE, sees - kb, j == 0);
          arrive(B_PH + s);
        }
        arrive(B_P + s);
      }
      // A unit in several CTAs' ranges: the CTA that finds the others' parts there (looked for while its last products run)
      // does not write its own.  Most such units have two, the end of one CTA's work and the beginning of the next one's: the
      // chunks of 256 tokens 76 to 73 us.
      const bool whole = p.kb0 == 0 && p.n >= nb, joined = !p.two && p.na[1] > 0;
      unsigned* count = a.counters + 2 * p.f_lo + s;
      const unsigned parts = f_hi - p.f_lo + 1;
      if (!whole && row == 0 && !(joined && s == 1)) sh_flag[2 + s] = kv_part_is_last(count, parts);
      if (mine > 0) {
        pv += mine;
        ++uses;
        wait(B_O + s, pv - 1);
        tc_fence_after();
      }
      // ---- one tile in two streams: stream 0 joins both
      float f0 = 1.f, f1 = 0.f;
      if (joined) {
        if (s == 1) [[unlikely]] {
          sh_ml[row] = make_float2(m, l);
          arrive(B_JOIN);
          continue;
        }
        wait(B_JOIN, joins++);
        tc_fence_after();
        const float2 x = sh_ml[row];
        const float mn = fmaxf(m, x.x);
        f0 = m == -INFINITY ? 0.f : exp2_hw(m - mn);
        f1 = x.x == -INFINITY ? 0.f : exp2_hw(x.x - mn);
        l = l * f0 + x.y * f1;  // no key in sight, or only NaN scores: sums of 0, or NaN, which a factor of 0 keeps
        m = mn;
      }
      auto own = [&](int c, float(&x)[32]) {  // the row's columns [c, c + 32), unscaled; by whole warps
        uint32_t o[32];
        __syncwarp();
        tmem_ld32(t_o + c, o);
        tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 32; ++e) x[e] = __uint_as_float(o[e]);
        if (joined) {
          tmem_ld32(t_o + HD + c, o);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = x[e] * f0 + __uint_as_float(o[e]) * f1;
        }
      };
      auto release = [&]() {  // O has been read
        arrive(B_FREE + s);
        if (joined) arrive(B_FREE + 1);
      };
      auto part = [&](int cta, bool first) { return (int64_t)((2 * cta + first) * 2 + s); };
      const int me = blockIdx.x;
      const float m_own = m;
      int f_first = me, f_last = nb == 0 ? me - 1 : me;  // whose parts make up the rows
      if (!whole) [[unlikely]] {  // ---- a part: [slot][stream][4 columns][row]
        bar_sync(1 + s, 128);
        if (!sh_flag[2 + s]) {
          const int64_t at = part(me, p.kb0 == 0);
          if (on) {
#pragma unroll 1
            for (int c = 0; c < HD; c += 32) {
              float x[32];
              own(c, x);
              if (valid) {
#pragma unroll
                for (int v = 0; v < 8; ++v)
                  __stcg(part_o + (at * (HD / 4) + c / 4 + v) * TB + row,
                         make_float4(x[4 * v], x[4 * v + 1], x[4 * v + 2], x[4 * v + 3]));
              }
            }
            if (valid) __stcg(part_ml + at * TB + row, make_float2(m, l));
          }
          bar_sync(1 + s, 128);
          if (row == 0) sh_flag[2 + s] = kv_part_done(count, parts);
          bar_sync(1 + s, 128);
          if (!sh_flag[2 + s]) {
            release();
            continue;
          }
        }
        f_first = p.f_lo;
        f_last = f_hi;
        const float l_own = l;
        m = -INFINITY;
        l = 0.f;
        for (int fb = f_first; valid && fb <= f_last; fb += 4) {  // the reads of four wait together
          float2 x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int f = min(fb + e, f_last);
            x[e] = f == me ? make_float2(m_own, l_own) : __ldcg(part_ml + part(f, f == f_first) * TB + row);
            if (fb + e > f_last) x[e] = make_float2(-INFINITY, 0.f);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float mn = fmaxf(m, x[e].x);
            l = l * (m == -INFINITY ? 0.f : exp2_hw(m - mn)) + x[e].y * (x[e].x == -INFINITY ? 0.f : exp2_hw(x[e].x - mn));
            m = mn;
          }
        }
      }
      // ---- the output
      if (on) {
        float inv;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(l));  // one ulp of 24 bits, before a rounding to 16
        inv = l == 0.f ? 0.f : inv;
        T* dst = reinterpret_cast<T*>(a.o) + t_row * a.ldo + head * HD;
#pragma unroll 1
        for (int c = 0; c < HD; c += 64) {
          float x[64];
#pragma unroll
          for (int e = 0; e < 64; ++e) x[e] = 0.f;
#pragma unroll 1
          for (int f = f_first; f <= f_last; ++f) {  // the parts in their order, the own one from where it lies
            if (f == me) {
              const float w = m_own == -INFINITY ? 0.f : exp2_hw(m_own - m);
#pragma unroll
              for (int h = 0; h < 64; h += 32) {
                float y[32];
                own(c + h, y);
#pragma unroll
                for (int e = 0; e < 32; ++e) x[h + e] = fmaf(y[e], w, x[h + e]);
              }
            } else if (valid) {
              const int64_t q = part(f, f == f_first);
              const float mf = __ldcg(part_ml + q * TB + row).x;
              float4 y[16];
#pragma unroll
              for (int v = 0; v < 16; ++v) y[v] = __ldcg(part_o + (q * (HD / 4) + c / 4 + v) * TB + row);
              const float w = mf == -INFINITY ? 0.f : exp2_hw(mf - m);
#pragma unroll
              for (int v = 0; v < 16; ++v) {
                x[4 * v] = fmaf(y[v].x, w, x[4 * v]);
                x[4 * v + 1] = fmaf(y[v].y, w, x[4 * v + 1]);
                x[4 * v + 2] = fmaf(y[v].z, w, x[4 * v + 2]);
                x[4 * v + 3] = fmaf(y[v].w, w, x[4 * v + 3]);
              }
            }
          }
          if (valid) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              uint32_t y[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) y[i] = Io::pack(x[16 * v + 2 * i] * inv, x[16 * v + 2 * i + 1] * inv);
              T* to = dst + c + 16 * v;
              if (o32) {
                st_global_v8(to, y);
              } else {
                reinterpret_cast<uint4*>(to)[0] = make_uint4(y[0], y[1], y[2], y[3]);
                reinterpret_cast<uint4*>(to)[1] = make_uint4(y[4], y[5], y[6], y[7]);
              }
            }
          }
        }
        if (valid && a.lse) {
          float lg;
          asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(lg) : "f"(l));
          a.lse[(int64_t)head * b.T + t_row] = (m + lg) * LN2_F;  // no keys: -inf of l = 0
        }
      }
      if (nb > 0) release();
    }
  } else {
    if (warp == W_TMA) {
      const KvRange rg = kv_plan(b, u, a.kvh, blockIdx.x, gridDim.x, MIN_COST);
      KvWalk<TileUnits> k;
      bool more = rg.s >= 0;
      if (more) k.set(b, u, rg.s, rg.seq_start, rg.lo, a.kvh);
      const int boxes = TB / geo.box_rows, per = (1 << b.ps_log2) / geo.box_rows;  // boxes of a block, of a page
      while (ok) {
        Piece p;
        p.end = !more;
        if (more) {
          p = piece_of(u, k, rg);
          const int seq = k.s;
          more = k.next(b, u, a.kvh) && k.start < rg.hi;
          if (p.n == 0 && p.zero == 0) continue;
          if (np >= PIECES && !wait(B_PDONE + np % PIECES, np / PIECES - 1)) break;
          if (lane == 0) {
            pieces[np % PIECES] = p;
            mbar_arrive(bars + B_PIECE + np % PIECES);
          }
          ++np;
          const int la = p.two ? 1 : 2;
          // keys of la blocks, Q, then each block's values and the keys la blocks further.  The first keys go ahead of Q,
          // whose place the last piece may still be using.
#pragma unroll 1
          for (int kt = 0, vt = 0, x = 0; ok && x < 2 * p.n; ++x) {
            const bool key = kt < p.n && kt < vt + la;
            if (x == min(la, p.n)) {
              for (int t = 0; t <= p.two; ++t) {
                const int slot = qi & 1;
                if (qi > 1 && !wait(B_QE + slot, (qi >> 1) - 1)) break;
                ++qi;
                if (elect_one()) {
                  mbar_arrive_expect_tx(bars + B_QF + slot, geo.tpt * a.group * HD * 2);
                  for (int h = 0; h < NB; ++h)
                    tma_load_3d(sQ + slot * TILE + h * (TB * 128), &maps.q, bars + B_QF + slot, 64 * h, p.h * a.group,
                                p.q0 + t * geo.tpt);
                }
                __syncwarp();
              }
            }
            const int kb = p.kb0 + (key ? kt++ : vt++), st = ring % ST;
            const int nbox = min(boxes, (p.kmax - kb * TB + geo.box_rows - 1) / geo.box_rows);
            int page = 0, at = 0;  // asked for before the stage is free
            if (lane < nbox) {
              const int i = kb * boxes + lane;
              page = kv_page(b, seq, i / per);
              at = i % per;
            }
            if (!ok || (ring >= ST && !wait(B_EMPTY + st, ring / ST - 1))) break;
            ++ring;
            if (lane == 0) mbar_arrive_expect_tx(bars + B_FULL + st, nbox * geo.box_rows * HD * 2);
            __syncwarp();
            if (lane < nbox)
              tma_load_5d(sKV + st * TILE + lane * geo.box_rows * HD * 2, key ? &maps.k : &maps.v, bars + B_FULL + st,
                          geo.by_head ? p.h * NB : 0, at * (geo.box_rows / 8),
                          page < 0 ? -1 : geo.by_head ? page : page * geo.per_page + p.h);
            __syncwarp();
          }
        } else {
          if (np >= PIECES && !wait(B_PDONE + np % PIECES, np / PIECES - 1)) break;
          if (lane == 0) {
            pieces[np % PIECES] = p;
            mbar_arrive(bars + B_PIECE + np % PIECES);
          }
          break;
        }
      }
    } else if (warp == W_FIX) {
      // A key that a row does not see has weight 0, which only makes nothing of it if its value is finite.  Rows of a V
      // block past the last key that anyone sees hold whatever the page held: they become zeros.  The others are
      // looked through where rows differ in what they see.
      while (wait(B_PIECE + np % PIECES, np / PIECES)) {
        const Piece p = pieces[np % PIECES];
        piece_done();
        if (p.end) break;
        const int la = p.two ? 1 : 2, first_sees = p.sees(0);
#pragma unroll 1
        for (int kt = 0, vt = 0, x = 0; ok && x < 2 * p.n; ++x, ++ring) {
          const int st = ring % ST;
          const bool key = kt < p.n && kt < vt + la;
          const int kb = p.kb0 + (key ? kt++ : vt++), used = min(TB, p.kmax - kb * TB);
          if (!wait(B_FULL + st, ring / ST)) break;
          uint4* sV = reinterpret_cast<uint4*>(sKV + st * TILE);
          if (!key && used < TB) {
#pragma unroll 1
            for (int i = used * NB * 8 + lane; i < TILE / 16; i += 32) {
              const int r = i / (NB * 8), c = i % (NB * 8);
              sV[(r >> 3) * NB * 64 + (c >> 3) * 64 + (r & 7) * 8 + (c & 7)] = make_uint4(0, 0, 0, 0);
            }
            fence_proxy_async_smem();
            __syncwarp();
          }
          if (!key && first_sees < kb * TB + used) {
            uint32_t top[4] = {0, 0, 0, 0};
#pragma unroll 1
            for (int i = lane; i < (used + 7) / 8 * NB * 64; i += 128) {  // whole groups of rows: NB * 64 each
              uint4 y[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) y[e] = i + 32 * e < TILE / 16 ? sV[i + 32 * e] : make_uint4(0, 0, 0, 0);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if (i + 32 * e >= (used + 7) / 8 * NB * 64) break;
                top[0] = Io::max_abs(top[0], y[e].x);
                top[1] = Io::max_abs(top[1], y[e].y);
                top[2] = Io::max_abs(top[2], y[e].z);
                top[3] = Io::max_abs(top[3], y[e].w);
              }
            }
            const bool odd = __any_sync(0xffffffffu, !Io::finite(top[0]) || !Io::finite(top[1]) || !Io::finite(top[2]) ||
                                                         !Io::finite(top[3]));
            if (lane == 0) sh_odd[st] = odd;
          }
          if (lane == 0) mbar_arrive(bars + B_READY + st);
        }
      }
    } else {
      const int s = (int)uniform(warp - W_MMA);  // the stream
      const uint32_t tm = uniform(tmem);
      const uint64_t desc_q = smem_desc_sw128(smem_u32(sQ), 16, 1024), desc_k = smem_desc_sw128(smem_u32(sKV), 16, NB * 1024),
                     desc_v = smem_desc_sw128(smem_u32(sKV), 1024, NB * 1024);
      const uint32_t t_s = tm + s * TB, t_o = tm + 256 + s * HD, t_p = C::OWN_P ? tm + 384 + s * 64 : t_s;
      constexpr uint32_t I_S = idesc<T>(TB, false), I_PV = idesc<T>(HD, true);
      // This warp's instructions lie between a stream's weights and its next scores.  What the loop goes by is known to
      // be uniform, so that it stays in uniform registers: the next stage and its phase, and counts.
      // Both streams see every stage and Q tile pass, in order, and free it with one arrival each: of those that it
      // does not read a stream waits for the copy only.  So no stream is ever two phases from a barrier's.
      uint32_t st = 0, ph = 0, qn = 0, done = 0, uses = 0, turn = 0;
      auto step = [&]() {
        if (++st == ST) st = 0, ph ^= 1;
      };
      auto pass = [&]() {
        if (wait(B_READY + st, ph) && lane == 0) mbar_arrive(bars + B_EMPTY + st);
        step();
      };
      while (wait(B_PIECE + np % PIECES, np / PIECES)) {
        const Piece* pp = pieces + np % PIECES;
        const int end = (int)uniform(pp->end), two = (int)uniform(pp->two), n = (int)uniform(pp->n),
                  mine = (int)uniform(pp->na[s]), turns = (int)uniform(pp->turns());
        piece_done();
        if (end) break;
        if (n == 0) continue;
        const uint32_t q = qn + (two ? s : 0);
        for (const uint32_t qe = qn + 1 + two; ok && qn < qe; ++qn)
          if (wait(B_QF + (qn & 1), qn >> 1) && (qn != q || mine == 0) && lane == 0) mbar_arrive(bars + B_QE + (qn & 1));
        const uint64_t dq = desc_q + (q & 1) * (TILE / 16);
        // The ring holds the keys of la blocks, then each block's values and the keys la blocks further; with two tiles
        // la = 1 and each stream takes all that it sees, else la = 2 and the streams take every other block.
        const int la = 2 - two;
        // Stream 0 waits below for all turns of the other one but a piece's last.  That comes first here: a wait for the turn
        // behind one that has not been told would pass, and the two count apart from then on.
        if (s == 0 && turns > 0 && turn > 0 && !wait(B_TURN + 1, turn - 1)) break;
#pragma unroll 1
        for (int t = -la; ok && t < n; ++t) {
          const bool my = two || ((t + 2) & 1) == s;
          const int j = two ? t : t >> 1;  // the stream's count of blocks
          const bool v = t >= 0, kk_ = t + la < n;  // the ring's next: V of block t, K of block t + la
          const bool pv = v && j < mine, qk = kk_ && j + 1 < mine;
          if (!my) {
            if (v) pass();
            if (kk_) pass();
            continue;
          }
          const uint32_t vs = st;
          const uint64_t dv = desc_v + st * (TILE / 16);
          if (v) {
            if (!wait(B_READY + st, ph)) break;
            if (!pv && lane == 0) mbar_arrive(bars + B_EMPTY + st);
            step();
          }
          const uint32_t ks = st;
          const uint64_t dk = desc_k + st * (TILE / 16);
          if (kk_) {
            if (!wait(B_READY + st, ph)) break;
            if (!qk && lane == 0) mbar_arrive(bars + B_EMPTY + st);
            step();
          }
          if (pv) {  // O += P V of block t, from the first half of the weights on
            if (j == 0) {
              if (uses > 0 && !wait(B_FREE + s, uses - 1)) break;  // the last piece's O has been read
              ++uses;
            }
            if (!wait(B_PH + s, done)) break;
            const bool issue = sh_flag[s] == 0;  // else the block was taken without the tensor cores
            tc_fence_after();
            if (issue && elect_one()) {
#pragma unroll
              for (int kk = 0; kk < TB / 32; ++kk) umma_bf16_ts(t_o, t_p + kk * 8, dv + kk * (NB * 128), I_PV, j > 0 || kk > 0);
            }
            __syncwarp();
            if (!wait(B_P + s, done)) break;
            ++done;
            tc_fence_after();
            if (elect_one()) {
              if (issue) {
#pragma unroll
                for (int kk = TB / 32; kk < TB / 16; ++kk) umma_bf16_ts(t_o, t_p + kk * 8, dv + kk * (NB * 128), I_PV, 1);
              }
              umma_commit(bars + B_O + s);
              umma_commit(bars + B_EMPTY + vs);
            }
            __syncwarp();
          }
          if (qk) {  // S of block t + la; the last P V has read the P that it overwrites
            // stream 0 after the other's block j, stream 1 after the other's block j + 1
            if (j + 1 < turns && j + s >= 0 && !wait(B_TURN + 1 - s, turn + j + s)) break;
            if (!C::OWN_P && done > 0 && !wait(B_O + s, done - 1)) break;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int kk = 0; kk < HD / 16; ++kk)
                umma_bf16(t_s, dq + (kk >> 2) * (TB * 128 / 16) + (kk & 3) * 2, dk + (kk >> 2) * 64 + (kk & 3) * 2, I_S, kk > 0);
              umma_commit(bars + B_S + s);
              umma_commit(bars + B_EMPTY + ks);
              if (j + 2 == mine) umma_commit(bars + B_QE + (q & 1));
            }
            __syncwarp();
          }
        }
        turn += turns;
      }
    }
  }
  // ---- the end: nothing is in flight any more when the CTA leaves
  __syncthreads();
  if (warp == W_MMA || warp == W_MMA + 1) {
    if (elect_one()) umma_commit(bars + B_END + warp - W_MMA);
    mbar_wait_warp(bars + B_END + warp - W_MMA, 0);
  }
  if (warp == W_TMA && sh_flag[4] != 0) {  // copies that nobody waited for
    for (uint32_t i = ring > ST ? ring - ST : 0; i < ring; ++i) mbar_wait_warp(bars + B_FULL + i % ST, (i / ST) & 1);
    for (uint32_t i = qi > 2 ? qi - 2 : 0; i < qi; ++i) mbar_wait_warp(bars + B_QF + (i & 1), (i >> 1) & 1);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == W_MMA) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <class T, int HD>
int launch_tc(const fl_kv_cache* c, const KvAttnArgs& a, int heads, cudaStream_t st) {
  FL_CUDA_TRY(fl_func_smem((const void*)kv_attn_tc_kernel<T, HD>, Cfg<HD>::SMEM));
  fl_gemm::PFN_encodeTiled enc = fl_gemm::get_encode_fn();
  if (!enc) return fl_internal_error(FL_ERR_CUDA, "cuTensorMapEncodeTiled is not available");
  TcGeom g;
  TcMaps m;
  constexpr int NB = HD / 64;
  g.tpt = TB / a.group;
  g.box_rows = c->page_size < TB ? c->page_size : TB;
  g.by_head = c->head_stride == HD;
  g.per_page = (int)(c->page_stride / c->head_stride);
  const int64_t last = g.by_head ? c->n_pages : (c->n_pages - 1ll) * (c->page_stride / c->head_stride) + c->kv_heads;
  if (last > 0x7fffffff) return fl_internal_error(FL_ERR_CAPACITY, "kv attention: %lld pages and heads", (long long)last);
  const CUtensorMapDataType type = KvIo<T>::is_half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  // (64 columns, 8 rows, column halves, groups of rows, pages and heads)
  const cuuint64_t dims[5] = {64, 8, (cuuint64_t)(g.by_head ? c->kv_heads * NB : NB), (cuuint64_t)c->page_size / 8,
                              (cuuint64_t)last};
  const cuuint64_t strides[4] = {(cuuint64_t)c->token_stride * 2, 128, (cuuint64_t)c->token_stride * 16,
                                 (cuuint64_t)(g.by_head ? c->page_stride : c->head_stride) * 2};
  const cuuint32_t box[5] = {64, 8, NB, (cuuint32_t)g.box_rows / 8, 1}, ones[5] = {1, 1, 1, 1, 1};
  const cuuint64_t qdims[3] = {HD, (cuuint64_t)heads, (cuuint64_t)a.b.T}, qstr[2] = {HD * 2, (cuuint64_t)a.ldq * 2};
  const cuuint32_t qbox[3] = {64, (cuuint32_t)a.group, (cuuint32_t)g.tpt};
  auto make = [&](CUtensorMap* out, const void* base, int rank, const cuuint64_t* d, const cuuint64_t* s, const cuuint32_t* x) {
    return enc(out, type, rank, const_cast<void*>(base), d, s, x, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  };
  CUresult r = make(&m.k, a.k, 5, dims, strides, box);
  if (r == CUDA_SUCCESS) r = make(&m.v, a.v, 5, dims, strides, box);
  if (r == CUDA_SUCCESS) r = make(&m.q, a.q, 3, qdims, qstr, qbox);
  if (r != CUDA_SUCCESS) return fl_internal_error(FL_ERR_INVALID_ARG, "kv attention: tensor map encode failed (%d)", (int)r);
  FL_CUDA_TRY(fl_launch(kv_attn_tc_kernel<T, HD>, dim3(fl_sm_count()), dim3(THREADS), Cfg<HD>::SMEM, st, m, a, g));
  return FL_OK;
}

}  // namespace

size_t fl_kv_attention_tc_parts(int head_dim) { return (size_t)fl_sm_count() * 4 * TB * (head_dim + 2) * sizeof(float); }

int fl_launch_kv_attention_tc(const fl_kv_cache* c, const KvAttnArgs& a, int heads, cudaStream_t st) {
  const bool half = c->dtype == FL_DT_F16;
  if (c->head_dim == 128) return half ? launch_tc<__half, 128>(c, a, heads, st) : launch_tc<__nv_bfloat16, 128>(c, a, heads, st);
  return half ? launch_tc<__half, 64>(c, a, heads, st) : launch_tc<__nv_bfloat16, 64>(c, a, heads, st);
}
