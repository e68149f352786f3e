// Attention of chunks of new tokens over the paged cache on the 5th-generation tensor cores.
//
// A tile is 128 rows, (token, query head) pairs of the query heads that share one key / value head, and key blocks of
// 128.  One CTA per SM runs two streams, each a tile's softmax over key blocks:
//   two tiles of a unit over the same blocks (each key block is read once for 256 rows), or
//   where a unit has one tile, that tile over the even and over the odd blocks, joined at the end.
// While one stream's scores are turned into weights the tensor cores work for the other.
//
//   warps 0-3, 4-7  softmax of stream 0 and 1: thread i owns row i (TMEM lane i): reads its 128 scores, takes
//                   p = 2^(s - m), writes p (16 bits) to TMEM; at the end O / l, or a part of it
//   warp 8          TMA: Q tiles, then K and V blocks page by page into a ring of stages
//   warp 9          S = Q K^T (both in shared memory) and O += P V (P in TMEM, V as an MN-major operand)
//
// TMEM: S of the streams at columns 0 and 128, O at 256.  P lies over its S at head_dim 128 (512 columns are
// taken), so the next S of a stream waits for its P V; at head_dim 64 it has columns of its own.
// A block of shared memory is [16 groups of 8 rows][head_dim / 64][8 rows][64 columns] in the 128-byte
// swizzle, so that one copy brings all columns of a page's rows.
// m follows a row's maximum only when that grew by more than 2^8, so O is seldom rescaled.
// Work is divided among the CTAs as kv_plan.cuh says.
//
// Every wait is bounded.  A warp whose wait ran out records it, issues nothing any more and goes through the rest of
// its steps without waiting, so that every barrier of the CTA is still reached by all.
#include <cuda.h>

#include <atomic>
#include <cmath>

#include "../../include/flglm_kernels.h"
#include "common.cuh"
#include "gemm_tc.cuh"
#include "kv_attention.cuh"
#include "ptx.cuh"

namespace {

constexpr int TB = 128;
constexpr int THREADS = 384, W_TMA = 8, W_MMA = 9;  // warps 10 and 11 complete the third warpgroup
// Registers a thread: at launch, and as the warpgroups then share them (the sum may not exceed the launch's:
// a request above it would wait forever; checked before the first launch)
constexpr int REGS_LAUNCH = 168, REGS_SOFTMAX = 208, REGS_REST = 80;
static_assert(2 * REGS_SOFTMAX + REGS_REST <= 3 * REGS_LAUNCH, "register split");
constexpr int ENDS = 2;      // cost of a unit's ends (Q, the first scores, the output), in blocks of one tile
constexpr int MIN_COST = 4;
constexpr float LN2_F = 0.6931471805599453f;

template <int HD>
struct Cfg {
  static constexpr int NB = HD / 64;
  static constexpr int TILE = TB * HD * 2;
  static constexpr int ST = HD == 128 ? 5 : 8;  // stages: what 227 KB hold beside two Q tiles; 8 at head_dim 64
  static constexpr int CTRL = 2048;
  static constexpr int SMEM = (2 + ST) * TILE + CTRL + 1024;
  static constexpr bool OWN_P = HD == 64;
};

struct TcMaps {
  CUtensorMap q, k, v;
};
struct TcGeom {
  int tpt;               // tokens of a tile
  int box_rows;          // rows that one copy brings: a page's, 128 at most
  int by_head, per_page; // coordinates of page p, head h: (0, p * per_page + h) or, heads side by side, (h * NB, p)
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

// What a CTA does of a unit: key blocks [kb0, kb0 + n), of which stream a takes part in na[a].
struct Piece {
  bool two, first;   // first: the unit begins in this CTA's range
  int tok0, kb0, n, nb[2], na[2], kmax, w;
};
FL_DEV Piece piece_of(const TileUnits& u, const KvWalk<TileUnits>& k, const KvRange& g) {
  Piece p;
  p.two = u.two(k.q, k.r);
  p.w = p.two ? 2 : 1;
  p.tok0 = k.r * 2 * u.tpt;
  p.kmax = kv_sees(k.q, min(k.q.n, p.tok0 + 2 * u.tpt) - 1);
  p.nb[1] = (p.kmax + TB - 1) / TB;
  p.nb[0] = p.two ? u.blocks(k.q, p.tok0 + u.tpt) : p.nb[1];
  p.first = k.start >= g.lo && k.start < g.hi;
  p.kb0 = (int)max((int64_t)0, (g.lo - k.start + p.w - 1) / p.w);
  const int kb1 = (int)min((int64_t)p.nb[1], (g.hi - k.start + p.w - 1) / p.w);
  p.n = max(0, kb1 - p.kb0);
  p.na[1] = p.n;
  p.na[0] = p.two ? min(p.n, max(0, p.nb[0] - p.kb0)) : p.n;
  if (!p.two) {
    p.na[0] = (p.n + 1) / 2;
    p.na[1] = p.n / 2;
  }
  return p;
}
// Place in the ring, from the piece's first stage on, of block t's values and keys: la blocks of keys, then
// each block's values and the keys la blocks further.
struct RingOrder {
  int n, la;
  FL_DEV int v(int t) const { return min(n, la) + t + min(t, max(n - la, 0)); }
  FL_DEV int k(int t) const { return t < la ? t : v(t - la) + 1; }
};

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
  enum { B_FULL = 0, B_EMPTY = ST, B_QF = 2 * ST, B_QE, B_S, B_P = B_S + 2, B_O = B_P + 2, B_FREE = B_O + 2, B_END = B_FREE + 2, BARS };
  static_assert(BARS * 8 <= 256, "control block");
  int64_t* sh_plan = reinterpret_cast<int64_t*>(ctrl + 256);                 // 15 of them
  volatile int* sh_flag = reinterpret_cast<volatile int*>(ctrl + 384);       // [0, 2) slow block, [2, 4) last part, [4] failed
  uint32_t* holder = reinterpret_cast<uint32_t*>(ctrl + 448);
  float2* sh_ml = reinterpret_cast<float2*>(ctrl + 512);                     // stream 1's rows, for joining (1 KB)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const KvBatchDev& b = a.b;

  if (tid == 0) {
    for (int i = 0; i < BARS; ++i) mbar_init(bars + i, (i >= B_P && i < B_P + 2) || (i >= B_FREE && i < B_FREE + 2) ? 4 : 1);
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
  const KvRange rg = kv_plan<THREADS>(b, u, a.kvh, blockIdx.x, gridDim.x, MIN_COST, sh_plan);
  const bool work = rg.s >= 0;

  bool ok = true;
  auto fail = [&]() {
    ok = false;
    sh_flag[4] = 1;
    atomicOr(a.status, FL_KV_TIMEOUT);
  };
  // by a whole warp; parity of the phase waited for
  auto wait = [&](int i, uint32_t phase) {
    if (ok && !mbar_wait_warp(bars + i, phase & 1)) fail();
  };
  uint32_t ring = 0;  // stages used before this piece

  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_SOFTMAX));
    if (work) {
      const int s = warp >> 2, row = tid & 127;
      const uint32_t t_lane = tmem + (uint32_t((warp & 3) * 32) << 16);
      const uint32_t t_s = t_lane + s * TB, t_o = t_lane + 256 + s * HD, t_p = C::OWN_P ? t_lane + 384 + s * 64 : t_s;
      uint32_t ss = 0, pv = 0, uses = 0;
      const float scale = fabsf(a.scale_log2);
      float4* part_o = reinterpret_cast<float4*>(a.parts);
      float2* part_ml = reinterpret_cast<float2*>(a.parts + (int64_t)gridDim.x * 4 * TB * HD);
      KvWalk<TileUnits> k;
      k.set(b, u, rg.s, rg.seq_start, rg.lo, a.kvh);
      do {
        const Piece p = piece_of(u, k, rg);
        const RingOrder ro{p.n, p.two ? 1 : 2};
        const uint32_t base = ring;  // the piece's first stage
        ring += 2 * p.n;
        const int tok = p.tok0 + (p.two && s ? geo.tpt : 0);
        const int rows = min(geo.tpt, k.q.n - tok) * a.group;
        const bool valid = row < rows, on = (warp & 3) * 32 < rows;
        const int mytok = tok + row / a.group;
        const int sees = valid ? kv_sees(k.q, mytok) : 0, first_sees = kv_sees(k.q, tok);
        // ---- the row's output, from o(c, x): its unscaled columns [c, c + 32)
        auto finish = [&](float m, float l, auto&& o) {
          const int h = k.h * a.group + row % a.group;
          const int64_t t = k.q.q0 + mytok;
          const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;  // a sum that is NaN stays one
          T* dst = reinterpret_cast<T*>(a.o) + t * a.ldo + h * HD;
#pragma unroll 1
          for (int c = 0; c < HD; c += 32) {
            float x[32];
            __syncwarp();
            o(c, x);
            if (valid) {
#pragma unroll
              for (int v = 0; v < 4; ++v) {
                uint32_t y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = Io::pack(x[8 * v + 2 * i] * inv, x[8 * v + 2 * i + 1] * inv);
                *reinterpret_cast<uint4*>(dst + c + 8 * v) = make_uint4(y[0], y[1], y[2], y[3]);
              }
            }
          }
          if (valid && a.lse) a.lse[(int64_t)h * b.T + t] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2_F;
        };
        if (p.nb[s] == 0) {  // rows that see nothing
          if (p.first && on && (p.two || s == 0))
            finish(-INFINITY, 0.f, [&](int, float(&x)[32]) {
#pragma unroll
              for (int i = 0; i < 32; ++i) x[i] = 0.f;
            });
          continue;
        }
        const int mine = p.na[s];
        if (mine == 0) continue;
        float m = -INFINITY, l = 0.f;
#pragma unroll 1
        for (int j = 0; j < mine; ++j) {
          const int t = p.two ? j : 2 * j + s, kb = (p.kb0 + t) * TB;
          wait(B_S + s, ss++);
          tc_fence_after();
          if (on) {
            uint32_t r[TB];
            tmem_ld32(t_s, *reinterpret_cast<uint32_t(*)[32]>(r));
            tmem_ld32(t_s + 32, *reinterpret_cast<uint32_t(*)[32]>(r + 32));
            tmem_ld32(t_s + 64, *reinterpret_cast<uint32_t(*)[32]>(r + 64));
            tmem_ld32(t_s + 96, *reinterpret_cast<uint32_t(*)[32]>(r + 96));
            tmem_ld_wait();
            if (a.scale_log2 < 0.f) {
#pragma unroll
              for (int e = 0; e < TB; ++e) r[e] ^= 0x80000000u;
            }
            if (!__all_sync(0xffffffffu, kb + TB <= sees)) {
#pragma unroll
              for (int e = 0; e < TB; ++e)
                if (kb + e >= sees) r[e] = 0xff800000u;
            }
            float mt = -INFINITY;
#pragma unroll
            for (int e = 0; e < TB; ++e) mt = fmaxf(mt, __uint_as_float(r[e]));
            mt *= scale;
            const bool grows = mt > m + 8.f;
            if (__any_sync(0xffffffffu, grows)) {
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
            float lt[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < TB / 2; ++c) {
              const float p0 = exp2_hw(fmaf(__uint_as_float(r[2 * c]), scale, -mref));
              const float p1 = exp2_hw(fmaf(__uint_as_float(r[2 * c + 1]), scale, -mref));
              lt[c & 1] += p0;
              lt[2 + (c & 1)] += p1;
              r[c] = Io::pack(p0, p1);
            }
            tmem_st32(t_p, *reinterpret_cast<uint32_t(*)[32]>(r));
            tmem_st32(t_p + 32, *reinterpret_cast<uint32_t(*)[32]>(r + 32));
            l += (lt[0] + lt[1]) + (lt[2] + lt[3]);
            tmem_st_wait();
          }
          // ---- values of keys that some row does not see have weight 0, which needs them finite: rows of the block
          // past the last key seen become zeros, the others are looked at where rows differ
          const int used = p.kmax - kb;  // keys of the block that some row of the unit sees
          const bool mixed = first_sees < min(kb + TB, p.kmax);
          bool slow = false;
          if (mixed || used < TB) {
            const uint32_t i = base + ro.v(t), st = i % ST;
            uint8_t* sV = sKV + st * TILE;
            wait(B_FULL + st, i / ST);
            bool odd = false;
            for (int x = row; x < TB * NB; x += 128) {  // row x / NB, 128 bytes of it
              const int kr = x / NB;
              uint4* at = reinterpret_cast<uint4*>(sV + (kr >> 3) * NB * 1024 + (x % NB) * 1024 + (kr & 7) * 128);
              if (kr >= used) {
#pragma unroll
                for (int v = 0; v < 8; ++v) at[v ^ (kr & 7)] = make_uint4(0, 0, 0, 0);
              } else if (mixed) {
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                  const uint4 y = at[v ^ (kr & 7)];
                  odd |= !Io::finite(y.x) || !Io::finite(y.y) || !Io::finite(y.z) || !Io::finite(y.w);
                }
              }
            }
            fence_proxy_async_smem();
            slow = mixed && bar_or(1 + s, 128, odd);
            if (slow) {
              if (j > 0) wait(B_O + s, pv + j - 1);
              else if (uses > 0) wait(B_FREE + s, uses - 1);
              tc_fence_after();
              __syncwarp();
              if (on) slow_pv<T, HD>(t_p, t_o, sV, sees - kb, j == 0);
            }
          }
          if (row == 0) sh_flag[s] = slow;
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bars + B_P + s);
        }
        pv += mine;
        ++uses;
        wait(B_O + s, pv - 1);
        tc_fence_after();
        // ---- one tile in two streams: stream 0 joins both
        const bool joined = !p.two && p.na[1] > 0;
        float f0 = 1.f, f1 = 0.f;
        if (joined) {
          if (s == 1) sh_ml[row] = make_float2(m, l);
          tc_fence_before();
          bar_sync(3, 256);
          tc_fence_after();
          if (s == 1) continue;
          const float2 x = sh_ml[row];
          const float mn = fmaxf(m, x.x);
          f0 = m == -INFINITY ? 0.f : exp2_hw(m - mn);
          f1 = x.x == -INFINITY ? 0.f : exp2_hw(x.x - mn);
          l = (f0 == 0.f ? 0.f : l * f0) + (f1 == 0.f ? 0.f : x.y * f1);
          m = mn;
        }
        auto own = [&](int c, float(&x)[32]) {  // by whole warps
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
            for (int e = 0; e < 32; ++e)
              x[e] = (f0 == 0.f ? 0.f : x[e] * f0) + (f1 == 0.f ? 0.f : __uint_as_float(o[e]) * f1);
          }
        };
        auto release = [&]() {  // O has been read
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(bars + B_FREE + s);
            if (joined) mbar_arrive(bars + B_FREE + 1);
          }
        };
        if (p.kb0 == 0 && p.n >= p.nb[s]) {
          if (on) finish(m, l, own);
          release();
          continue;
        }
        // ---- a part: [slot][stream][4 columns][row]
        auto part = [&](int cta, bool first) { return (int64_t)((2 * cta + first) * 2 + s); };
        const int64_t at = part(blockIdx.x, p.kb0 == 0);
        if (on) {
#pragma unroll 1
          for (int c = 0; c < HD; c += 32) {
            float x[32];
            own(c, x);
            if (valid) {
#pragma unroll
              for (int v = 0; v < 8; ++v)
                __stcg(part_o + (at * (HD / 4) + c / 4 + v) * TB + row, make_float4(x[4 * v], x[4 * v + 1], x[4 * v + 2], x[4 * v + 3]));
            }
          }
          if (valid) __stcg(part_ml + at * TB + row, make_float2(m, l));
        }
        release();
        const int f_lo = rg.cta_of(k.start), f_hi = rg.cta_of(k.start + (int64_t)p.w * (p.nb[s] - 1));
        __threadfence();
        bar_sync(1 + s, 128);
        if (row == 0) {
          sh_flag[2 + s] = atomicInc(a.counters + 2 * f_lo + s, f_hi - f_lo) == (unsigned)(f_hi - f_lo);
          __threadfence();
        }
        bar_sync(1 + s, 128);
        if (!sh_flag[2 + s]) continue;
        float ma = -INFINITY, la = 0.f;
        for (int f = f_lo; valid && f <= f_hi; ++f) ma = fmaxf(ma, __ldcg(part_ml + part(f, f == f_lo) * TB + row).x);
        for (int f = f_lo; valid && f <= f_hi; ++f) {
          const float2 x = __ldcg(part_ml + part(f, f == f_lo) * TB + row);
          if (x.x != -INFINITY) la += x.y * exp2_hw(x.x - ma);
        }
        if (on)
          finish(ma, la, [&](int c, float(&x)[32]) {
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] = 0.f;
            for (int f = f_lo; valid && f <= f_hi; ++f) {
              const int64_t q = part(f, f == f_lo);
              const float mf = __ldcg(part_ml + q * TB + row).x;
              if (mf == -INFINITY) continue;
              const float w = exp2_hw(mf - ma);
#pragma unroll
              for (int v = 0; v < 8; ++v) {
                const float4 y = __ldcg(part_o + (q * (HD / 4) + c / 4 + v) * TB + row);
                x[4 * v] = fmaf(y.x, w, x[4 * v]);
                x[4 * v + 1] = fmaf(y.y, w, x[4 * v + 1]);
                x[4 * v + 2] = fmaf(y.z, w, x[4 * v + 2]);
                x[4 * v + 3] = fmaf(y.w, w, x[4 * v + 3]);
              }
            }
          });
      } while (k.next(b, u, a.kvh) && k.start < rg.hi);
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_REST));
    if (work && warp == W_TMA) {
      KvWalk<TileUnits> k;
      k.set(b, u, rg.s, rg.seq_start, rg.lo, a.kvh);
      uint32_t pieces = 0;
      do {
        const Piece p = piece_of(u, k, rg);
        if (p.n == 0) continue;
        if (pieces > 0) wait(B_QE, pieces - 1);
        ++pieces;
        if (ok && elect_one()) {
          mbar_arrive_expect_tx(bars + B_QF, (p.two ? 2 : 1) * geo.tpt * a.group * HD * 2);
          for (int t = 0; t < (p.two ? 2 : 1); ++t)
            for (int h = 0; h < NB; ++h)
              tma_load_3d(sQ + t * TILE + h * (TB * 128), &maps.q, bars + B_QF, 64 * h, k.h * a.group,
                          k.q.q0 + p.tok0 + t * geo.tpt);
        }
        __syncwarp();
        const int boxes = TB / geo.box_rows, per = (1 << b.ps_log2) / geo.box_rows;  // boxes of a block, of a page
        auto load = [&](int t, bool v) {
          const int st = ring % ST;
          if (ring >= ST) wait(B_EMPTY + st, ring / ST - 1);
          ++ring;
          const int kb = p.kb0 + t;
          const int nbox = min(boxes, (p.kmax - kb * TB + geo.box_rows - 1) / geo.box_rows);
          int page = 0, part = 0;
          if (lane < nbox) {
            const int i = kb * boxes + lane;
            page = kv_page(b, k.s, i / per, a.status);
            part = i % per;
          }
          if (!ok) return;
          if (lane == 0) mbar_arrive_expect_tx(bars + B_FULL + st, nbox * geo.box_rows * HD * 2);
          __syncwarp();
          if (lane < nbox)
            tma_load_5d(sKV + st * TILE + lane * geo.box_rows * HD * 2, v ? &maps.v : &maps.k, bars + B_FULL + st,
                        geo.by_head ? k.h * NB : 0, part * (geo.box_rows / 8),
                        page < 0 ? -1 : geo.by_head ? page : page * geo.per_page + k.h);
          __syncwarp();
        };
        const int la = p.two ? 1 : 2;
        for (int t = 0; t < min(p.n, la); ++t) load(t, false);
        for (int t = 0; t < p.n; ++t) {
          load(t, true);
          if (t + la < p.n) load(t + la, false);
        }
      } while (k.next(b, u, a.kvh) && k.start < rg.hi);
    } else if (work && warp == W_MMA) {
      KvWalk<TileUnits> k;
      k.set(b, u, rg.s, rg.seq_start, rg.lo, a.kvh);
      uint32_t pieces = 0, ps[2] = {0, 0}, pv[2] = {0, 0}, uses[2] = {0, 0};
      constexpr uint32_t I_S = idesc<T>(TB, false), I_PV = idesc<T>(HD, true);
      do {
        const Piece p = piece_of(u, k, rg);
        if (p.n == 0) continue;
        const RingOrder ro{p.n, p.two ? 1 : 2};
        wait(B_QF, pieces++);
        int left = p.na[0] + p.na[1];
        auto qk = [&](int s, int t) {
          const uint32_t i = ring + ro.k(t), st = i % ST;
          wait(B_FULL + st, i / ST);
          if (!C::OWN_P && pv[s] > 0) wait(B_O + s, pv[s] - 1);  // its P V has read the P that S overwrites
          --left;
          tc_fence_after();
          if (ok && elect_one()) {
            const uint64_t dq = smem_desc_sw128(smem_u32(sQ + (p.two ? s * TILE : 0)), 16, 1024);
            const uint64_t dk = smem_desc_sw128(smem_u32(sKV + st * TILE), 16, NB * 1024);
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk)
              umma_bf16(tmem + s * TB, dq + (kk >> 2) * (TB * 128 / 16) + (kk & 3) * 2, dk + (kk >> 2) * 64 + (kk & 3) * 2,
                        I_S, kk > 0);
            umma_commit(bars + B_S + s);
            if (!p.two || s == 1) umma_commit(bars + B_EMPTY + st);
            if (left == 0) umma_commit(bars + B_QE);
          }
          __syncwarp();
        };
        auto pvs = [&](int s, int t, bool first) {
          wait(B_P + s, ps[s]++);
          const uint32_t i = ring + ro.v(t), st = i % ST;
          wait(B_FULL + st, i / ST);
          if (first) {
            if (uses[s] > 0) wait(B_FREE + s, uses[s] - 1);  // the last piece's O has been read
            ++uses[s];
          }
          ++pv[s];
          const bool slow = sh_flag[s] != 0;
          tc_fence_after();
          if (ok && elect_one()) {
            if (!slow) {
              const uint64_t dv = smem_desc_sw128(smem_u32(sKV + st * TILE), 1024, NB * 1024);
              const uint32_t tp = tmem + (C::OWN_P ? 384 + s * 64 : s * TB);
#pragma unroll
              for (int kk = 0; kk < TB / 16; ++kk)
                umma_bf16_ts(tmem + 256 + s * HD, tp + kk * 8, dv + kk * (NB * 128), I_PV, !first || kk > 0);
            }
            umma_commit(bars + B_O + s);
            if (!p.two || s == 1) umma_commit(bars + B_EMPTY + st);
          }
          __syncwarp();
        };
        if (p.two) {
          if (p.na[0] > 0) qk(0, 0);
          qk(1, 0);
          for (int t = 0; t < p.n; ++t)
            for (int s = t < p.na[0] ? 0 : 1; s < 2; ++s) {
              pvs(s, t, t == 0);
              if (t + 1 < p.na[s]) qk(s, t + 1);
            }
        } else {
          qk(0, 0);
          if (p.n > 1) qk(1, 1);
          for (int t = 0; t < p.n; ++t) {
            pvs(t & 1, t, t < 2);
            if (t + 2 < p.n) qk(t & 1, t + 2);
          }
        }
        ring += 2 * p.n;
      } while (k.next(b, u, a.kvh) && k.start < rg.hi);
    }
  }
  // ---- the end: nothing is in flight any more when the CTA leaves
  __syncthreads();
  if (warp == W_MMA) {
    if (elect_one()) umma_commit(bars + B_END);
    mbar_wait_warp(bars + B_END, 0);
  }
  if (warp == W_TMA && sh_flag[4] != 0)  // copies that nobody waited for
    for (uint32_t i = ring > ST ? ring - ST : 0; i < ring; ++i) mbar_wait_warp(bars + B_FULL + i % ST, (i / ST) & 1);
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
  static std::atomic<bool> split_ok{false};
  if (!split_ok.load(std::memory_order_relaxed)) {
    cudaFuncAttributes at;
    FL_CUDA_TRY(cudaFuncGetAttributes(&at, (const void*)kv_attn_tc_kernel<T, HD>));
    if (at.numRegs < REGS_LAUNCH)
      return fl_internal_error(FL_ERR_UNSUPPORTED, "kv attention: built with %d registers a thread", at.numRegs);
    split_ok.store(true, std::memory_order_relaxed);
  }
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
