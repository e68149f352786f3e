// Rotary positions and the write side of the paged key / value cache.
//
// A rotation turns pairs (a, b) of a head's dims by the position's angle: (a c - b s, a s + b c), its
// gradient by the transpose.  All three kernels here are bound by memory: each element is read and written
// once, 16 bytes a lane and access; the table's row (rotary_dim * 4 bytes, shared by every head of a token) comes
// from L1.  A thread takes 16 dims of one head, both halves of their pairs: enough to have in flight, and pairs never
// cross threads.  8192 rows of 64 heads in 46.6 us (5.8 TB/s), 10214 tokens appended in 88.7 (5.7 TB/s); few tokens
// take the launch and three dependent reads, 2.6 us.
#include <cuda_fp16.h>

#include <cmath>

#include "../../include/flglm_kernels.h"
#include "common.cuh"
#include "kv_plan.cuh"

namespace {

// Small blocks: as one ends another starts, so that some are always waiting for loads.  10214 tokens appended in 88.7
// us; 91, with 256 threads 98 and with 512 117, when this was chosen.
constexpr int BLOCK = 128;

// Eight consecutive elements as fp32, and back (one rounding).
template <class T>
struct Vec8;
template <>
struct Vec8<float> {
  float4 a, b;
  FL_DEV void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  FL_DEV void store(float* p) const {
    reinterpret_cast<float4*>(p)[0] = a;
    reinterpret_cast<float4*>(p)[1] = b;
  }
  FL_DEV void get(float (&f)[8]) const {
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
  }
  FL_DEV void set(const float (&f)[8]) {
    a = make_float4(f[0], f[1], f[2], f[3]);
    b = make_float4(f[4], f[5], f[6], f[7]);
  }
};
template <class T>
struct Vec8H {  // 16-bit types
  uint4 v;
  FL_DEV void load(const T* p) { v = *reinterpret_cast<const uint4*>(p); }
  FL_DEV void store(T* p) const { *reinterpret_cast<uint4*>(p) = v; }
};
template <>
struct Vec8<__nv_bfloat16> : Vec8H<__nv_bfloat16> {
  FL_DEV void get(float (&f)[8]) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 x = unpack_bf16x2(w[i]);
      f[2 * i] = x.x;
      f[2 * i + 1] = x.y;
    }
  }
  FL_DEV void set(const float (&f)[8]) {
    v = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
  }
};
template <>
struct Vec8<__half> : Vec8H<__half> {
  FL_DEV void get(float (&f)[8]) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 x = __half22float2(*reinterpret_cast<const __half2*>(w + i));
      f[2 * i] = x.x;
      f[2 * i + 1] = x.y;
    }
  }
  FL_DEV void set(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<__half2*>(w + i) = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
};

struct Rope {
  const int32_t *pos, *pos2;  // pos2: the second stream, or null
  const float* tab;
  int max_pos, rd;
  float sign;  // of the sines: -1 applies the transpose
  int interleaved;
};

// The 16 dims of a head that its thread i holds, eight at `a` and eight at `b`, which stream turns them (-1: copied), and
// the table entries of its pairs, four from pair `pa` and four from pair `pb` on.  The eights of a part's threads lie next
// to each other, so that every access of a row is of whole sectors.
struct Group {
  int a, b, stream, pa, pb;
};
FL_DEV Group group_of(const Rope& r, int i, int hd) {
  Group g;
  const int per = r.rd >> 4, second = r.pos2 ? per : 0;  // threads of each stream
  g.stream = i < per ? 0 : i < per + second ? 1 : -1;
  const int before = g.stream == 0 ? 0 : g.stream == 1 ? per : per + second;
  const int k = i - before, base = 16 * before, width = g.stream < 0 ? hd - base : r.rd;
  g.a = base + 8 * k;
  g.b = g.a + (width >> 1);
  g.pa = r.interleaved ? 4 * k : 8 * k;
  g.pb = r.interleaved ? (r.rd >> 2) + 4 * k : 8 * k + 4;
  return g;
}

// Turns the pairs of one group by position p; false (and zeros) where it is out of range.
template <class T>
FL_DEV bool turn(const Rope& r, const Group& g, int p, Vec8<T>& va, Vec8<T>& vb) {
  float a[8], b[8];
  if ((unsigned)p >= (unsigned)r.max_pos) {
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = 0.f;
    va.set(a);
    vb.set(a);
    return false;
  }
  const float* t = r.tab + (int64_t)p * r.rd;
  float c[8], s[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 x = __ldg(reinterpret_cast<const float4*>(t + 2 * (i < 2 ? g.pa : g.pb)) + (i & 1));
    c[2 * i] = x.x, s[2 * i] = r.sign * x.y, c[2 * i + 1] = x.z, s[2 * i + 1] = r.sign * x.w;
  }
  va.get(a);
  vb.get(b);
  if (r.interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = a[2 * i], y = a[2 * i + 1], z = b[2 * i], w = b[2 * i + 1];
      a[2 * i] = x * c[i] - y * s[i];
      a[2 * i + 1] = x * s[i] + y * c[i];
      b[2 * i] = z * c[4 + i] - w * s[4 + i];
      b[2 * i + 1] = z * s[4 + i] + w * c[4 + i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = a[i], y = b[i];
      a[i] = x * c[i] - y * s[i];
      b[i] = x * s[i] + y * c[i];
    }
  }
  va.set(a);
  vb.set(b);
  return true;
}

// A block's rows are (token, head) pairs in order; blockDim = (head_dim / 16) threads a row.
template <class T>
__global__ void __launch_bounds__(BLOCK) rotary_kernel(uint32_t rows, int heads, int per_row, const T* x, int64_t ldx,
                                                     int64_t hsx, T* y, int64_t ldy, int64_t hsy, Rope r,
                                                     int* __restrict__ status) {
  pdl_wait();  // the previous kernel on the stream has completed (see fl_launch)
  pdl_trigger();
  const uint32_t row = blockIdx.x * (blockDim.x / per_row) + threadIdx.x / per_row;
  if (row >= rows) return;
  const int i = threadIdx.x % per_row;
  const int64_t t = row / (uint32_t)heads;
  const int h = row % (uint32_t)heads;
  const Group g = group_of(r, i, 16 * per_row);
  const T* px = x + t * ldx + h * hsx;
  T* py = y + t * ldy + h * hsy;
  Vec8<T> a, b;
  a.load(px + g.a);
  b.load(px + g.b);
  if (g.stream >= 0 && !turn(r, g, __ldg((g.stream ? r.pos2 : r.pos) + t), a, b)) atomicOr(status, FL_KV_BAD_POSITION);
  a.store(py + g.a);
  b.store(py + g.b);
}

template <class T>
struct AppendArgs {
  const T *q, *k, *v;
  T *q_out, *ck, *cv;
  int64_t ldq, ldk, ldv, ldqo, page_stride, head_stride, token_stride;
  int heads, kvh;  // heads = 0: only the cache is written
};

// Rows: each token's query heads, key heads, value heads.
template <class T, int HD>
__global__ void __launch_bounds__(BLOCK) append_kernel(AppendArgs<T> p, KvBatchDev bt, Rope r, int* __restrict__ status) {
  pdl_wait();
  pdl_trigger();
  constexpr int PER = HD / 16;
  const uint32_t heads = p.heads + 2 * p.kvh, row = blockIdx.x * (BLOCK / PER) + threadIdx.x / PER;
  const int t = row / heads, j = row % heads;
  if (t >= bt.T) return;
  const int i = threadIdx.x % PER;
  const bool is_q = j < p.heads, is_v = j >= p.heads + p.kvh;
  const int h = is_q ? j : j - p.heads - (is_v ? p.kvh : 0);
  Group g = group_of(r, i, HD);
  if (is_v) g = Group{8 * i, HD / 2 + 8 * i, -1, 0, 0};
  const T* src = (is_q ? p.q + t * p.ldq : is_v ? p.v + t * p.ldv : p.k + t * p.ldk) + h * HD;
  Vec8<T> a, b;
  a.load(src + g.a);
  b.load(src + g.b);
  // the token's index in its sequence; queries need it only for a position
  int idx = -1, s = 0;
  if (!is_q || (g.stream == 0 && !r.pos)) {
    // one token a sequence is the usual call: try that first
    if (!(t < bt.S && __ldg(bt.cu + t) <= t && __ldg(bt.cu + t + 1) > t)) {
      int lo = 0, hi = bt.S;  // cu[lo] <= t < cu[hi] (assumed of the ends, checked below)
      while (hi - lo > 1) {
        const int mid = lo + ((hi - lo) >> 1);
        if (__ldg(bt.cu + mid) <= t) lo = mid; else hi = mid;
      }
      s = lo;
    } else {
      s = t;
    }
    const int end = __ldg(bt.cu + s + 1);
    if (__ldg(bt.cu + s) <= t && t < end) idx = __ldg(bt.lens + s) - (end - t);
  }
  if (g.stream >= 0) {
    const int pos = g.stream ? __ldg(r.pos2 + t) : r.pos ? __ldg(r.pos + t) : idx;
    if (!turn(r, g, pos, a, b)) atomicOr(status, FL_KV_BAD_POSITION);
  }
  T* dst;
  if (is_q) {
    dst = p.q_out + t * p.ldqo + h * HD;
  } else {
    const int e = idx >> bt.ps_log2;
    const int page = idx >= 0 && e < bt.table_stride ? kv_page(bt, s, e) : -1;
    if (page < 0) {
      atomicOr(status, FL_KV_BAD_PAGE);
      return;
    }
    dst = (is_v ? p.cv : p.ck) + page * p.page_stride + h * p.head_stride +
          (idx & ((1 << bt.ps_log2) - 1)) * p.token_stride;
  }
  a.store(dst + g.a);
  b.store(dst + g.b);
}

// fp64 angles: a table is made once per model.
__global__ void __launch_bounds__(256) rotary_table_kernel(int64_t n, int half, double base, int scaling, double factor,
                                                           double original, float2* __restrict__ tab) {
  pdl_wait();
  pdl_trigger();
  const int64_t x = blockIdx.x * 256ll + threadIdx.x;
  if (x >= n) return;
  const int64_t p = x / half;
  const int i = (int)(x % half);
  double f = pow(base, -(double)i / half), size = 1.0;
  if (scaling == FL_ROPE_SCALE_LINEAR) f /= factor;
  if (scaling == FL_ROPE_SCALE_NTK) f = pow(base * pow(factor, (double)half / (half - 1)), -(double)i / half);
  if (scaling == FL_ROPE_SCALE_BY_PARTS) {
    const double turns = original * f / 6.283185307179586476925286766559;
    const double keep = fmin(fmax((turns - 1.0) / 31.0, 0.0), 1.0);
    f = (1.0 - keep) * f / factor + keep * f;
    size = 0.1 * log(factor) + 1.0;
  }
  double s, c;
  sincos((double)p * f, &s, &c);
  tab[x] = make_float2((float)(size * c), (float)(size * s));
}

// Checks shared by the two calls that turn rows; null when they pass.
const char* rope_problem(int head_dim, int rd, int layout, const void* pos, const void* pos2, const void* tab,
                         int max_pos) {
  if (layout != FL_ROPE_HALF && layout != FL_ROPE_INTERLEAVED) return "layout";
  if (rd > 0 && (!tab || max_pos < 1)) return "no rotary table";
  if (fl_misaligned(tab, 16) || fl_misaligned(pos, 4) || fl_misaligned(pos2, 4)) return "alignment";
  return nullptr;
}
bool rope_supported(int head_dim, int rd, const void* pos2) {
  return rd >= 0 && rd % 16 == 0 && rd * (pos2 ? 2 : 1) <= head_dim && !(pos2 && rd == 0);
}

template <class T>
int launch_rotary(int T_, int heads, int hd, const void* x, int64_t ldx, int64_t hsx, void* y, int64_t ldy, int64_t hsy,
                  const Rope& r, int* status, cudaStream_t st) {
  const int per = hd / 16, block = per * (BLOCK / per);
  const int64_t rows = (int64_t)T_ * heads, each = BLOCK / per, grid = (rows + each - 1) / each;
  if (rows > 0x7fffffff) return fl_internal_error(FL_ERR_CAPACITY, "rotary: %lld rows", (long long)rows);
  FL_CUDA_TRY(fl_launch(rotary_kernel<T>, dim3((unsigned)grid), dim3(block), 0, st, (uint32_t)rows, heads, per, (const T*)x, ldx,
                        hsx, (T*)y, ldy, hsy, r, status));
  return FL_OK;
}

template <class T>
int launch_append(const fl_kv_cache* c, const KvBatchDev& bt, int heads, const void* q, int64_t ldq, const void* k,
                  int64_t ldk, const void* v, int64_t ldv, void* q_out, int64_t ldqo, const Rope& r, int* status,
                  cudaStream_t st) {
  AppendArgs<T> a{(const T*)q,    (const T*)k,    (const T*)v,    (T*)q_out, (T*)c->k, (T*)c->v, ldq, ldk, ldv, ldqo,
                  c->page_stride, c->head_stride, c->token_stride, q ? heads : 0, c->kv_heads};
  const int per = c->head_dim / 16;
  const int64_t rows = (int64_t)bt.T * (a.heads + 2 * a.kvh), each = BLOCK / per, grid = (rows + each - 1) / each;
  if (rows > 0x7fffffff) return fl_internal_error(FL_ERR_CAPACITY, "kv append: %lld rows", (long long)rows);
  if (c->head_dim == 128)
    FL_CUDA_TRY(fl_launch(append_kernel<T, 128>, dim3((unsigned)grid), dim3(BLOCK), 0, st, a, bt, r, status));
  else
    FL_CUDA_TRY(fl_launch(append_kernel<T, 64>, dim3((unsigned)grid), dim3(BLOCK), 0, st, a, bt, r, status));
  return FL_OK;
}

}  // namespace

int fl_kv_check(const char* who, const fl_kv_cache* c, const fl_kv_batch* b, int n_heads, KvBatchDev* out) {
  if (!c || !b || !c->k || !c->v || b->n_seqs < 0 || b->n_tokens < 0 || b->max_new < 0 || b->table_stride < 1 ||
      c->n_pages < 1 || c->kv_heads < 1 || n_heads < 1 || n_heads % c->kv_heads || (b->n_tokens > 0 && (b->n_seqs == 0 || b->max_new == 0)))
    return fl_internal_error(FL_ERR_INVALID_ARG, "%s: sizes", who);
  if (b->n_tokens > 0 && (!b->cu_new || !b->lens || !b->page_table))
    return fl_internal_error(FL_ERR_INVALID_ARG, "%s: null index array", who);
  if (c->dtype != FL_DT_BF16 && c->dtype != FL_DT_F16) return fl_internal_error(FL_ERR_UNSUPPORTED, "%s: dtype %d", who, c->dtype);
  if (c->head_dim != 64 && c->head_dim != 128)
    return fl_internal_error(FL_ERR_UNSUPPORTED, "%s: head_dim %d", who, c->head_dim);
  const int ps = c->page_size;
  if (ps < 16 || ps > 256 || (ps & (ps - 1)))
    return fl_internal_error(FL_ERR_UNSUPPORTED, "%s: page_size %d (a power of two, 16 to 256)", who, ps);
  if (c->head_stride < c->head_dim || c->token_stride < c->head_dim || c->page_stride < c->head_dim ||
      c->head_stride % 8 || c->token_stride % 8 || c->page_stride % c->head_stride)
    return fl_internal_error(FL_ERR_UNSUPPORTED, "%s: cache strides", who);
  if (fl_misaligned(c->k, 16) || fl_misaligned(c->v, 16) || fl_misaligned(b->cu_new, 4) || fl_misaligned(b->lens, 4) ||
      fl_misaligned(b->page_table, 4))
    return fl_internal_error(FL_ERR_INVALID_ARG, "%s: alignment", who);
  int lg = 4;
  while ((1 << lg) < ps) ++lg;
  // what the kernels count in 32 bits goes up to a few hundred past these: tokens of tiles and key blocks that end late
  constexpr int64_t most = (1ll << 31) - 1024;
  if (((int64_t)b->table_stride << lg) > most || b->n_tokens > most || b->n_seqs > most)
    return fl_internal_error(FL_ERR_CAPACITY, "%s: more than 2^31 - 1024 sequences, new tokens or tokens in a page table row", who);
  *out = KvBatchDev{b->cu_new, b->lens, b->page_table, nullptr, b->n_seqs, b->n_tokens, b->table_stride, lg, c->n_pages,
                    nullptr};
  return FL_OK;
}

extern "C" int fl_k_rotary_table(int32_t max_pos, int32_t rotary_dim, float base, int32_t scaling, float factor,
                                 int32_t original_max_pos, float* table, void* stream) {
  if (max_pos < 1 || rotary_dim < 2 || rotary_dim % 2 || !(base > 1.f) || !std::isfinite(base) || !table ||
      fl_misaligned(table, 16) || scaling < FL_ROPE_SCALE_NONE || scaling > FL_ROPE_SCALE_BY_PARTS)
    return fl_internal_error(FL_ERR_INVALID_ARG, "rotary table: args");
  if (scaling != FL_ROPE_SCALE_NONE && (!(factor >= 1.f) || !std::isfinite(factor)))
    return fl_internal_error(FL_ERR_INVALID_ARG, "rotary table: factor %g (1 or more)", factor);
  if ((scaling == FL_ROPE_SCALE_NTK && rotary_dim < 4) || (scaling == FL_ROPE_SCALE_BY_PARTS && original_max_pos < 1))
    return fl_internal_error(FL_ERR_INVALID_ARG, "rotary table: scaling");
  const int64_t n = (int64_t)max_pos * (rotary_dim / 2), grid = (n + 255) / 256;
  if (grid > 0x7fffffff) return fl_internal_error(FL_ERR_CAPACITY, "rotary table: %lld entries", (long long)n);
  FL_CUDA_TRY(fl_launch(rotary_table_kernel, dim3((unsigned)grid), dim3(256), 0, (cudaStream_t)stream, n,
                        rotary_dim / 2, (double)base, scaling, (double)factor, (double)original_max_pos,
                        (float2*)table));
  return FL_OK;
}

extern "C" int fl_k_rotary(int32_t T, int32_t n_heads, int32_t head_dim, int32_t rotary_dim, int32_t layout,
                           int32_t backward, int32_t dtype, const void* x, int64_t ldx, int64_t x_head_stride, void* y,
                           int64_t ldy, int64_t y_head_stride, const int32_t* positions, const int32_t* block_positions,
                           const float* rope_tab, int32_t max_pos, int* status, void* stream) {
  if (T < 0 || n_heads < 1 || !x || !y || !positions || !rope_tab || !status || (backward != 0 && backward != 1) ||
      fl_misaligned(x, 16) || fl_misaligned(y, 16) || fl_misaligned(status, 4))
    return fl_internal_error(FL_ERR_INVALID_ARG, "rotary: args");
  if (dtype != FL_DT_BF16 && dtype != FL_DT_F16 && dtype != FL_DT_F32)
    return fl_internal_error(FL_ERR_INVALID_ARG, "rotary: dtype %d", dtype);
  if (const char* w = rope_problem(head_dim, rotary_dim, layout, positions, block_positions, rope_tab, max_pos))
    return fl_internal_error(FL_ERR_INVALID_ARG, "rotary: %s", w);
  const int unit = dtype == FL_DT_F32 ? 4 : 8;
  if (head_dim < 16 || head_dim > 256 || head_dim % 16 || rotary_dim < 16 ||
      !rope_supported(head_dim, rotary_dim, block_positions))
    return fl_internal_error(FL_ERR_UNSUPPORTED, "rotary: head_dim %d, rotary_dim %d", head_dim, rotary_dim);
  if (ldx % unit || ldy % unit || x_head_stride % unit || y_head_stride % unit || ldx < 0 || ldy < 0 ||
      x_head_stride < 0 || y_head_stride < 0)
    return fl_internal_error(FL_ERR_UNSUPPORTED, "rotary: strides must be multiples of 16 bytes, not negative");
  if (T == 0) return FL_OK;
  const Rope r{positions, block_positions, rope_tab, max_pos, rotary_dim, backward ? -1.f : 1.f,
               layout == FL_ROPE_INTERLEAVED};
  const cudaStream_t st = (cudaStream_t)stream;
  if (dtype == FL_DT_F32)
    return launch_rotary<float>(T, n_heads, head_dim, x, ldx, x_head_stride, y, ldy, y_head_stride, r, status, st);
  if (dtype == FL_DT_F16)
    return launch_rotary<__half>(T, n_heads, head_dim, x, ldx, x_head_stride, y, ldy, y_head_stride, r, status, st);
  return launch_rotary<__nv_bfloat16>(T, n_heads, head_dim, x, ldx, x_head_stride, y, ldy, y_head_stride, r, status, st);
}

extern "C" int fl_k_kv_append(const fl_kv_cache* cache, const fl_kv_batch* batch, int32_t n_heads, const void* q,
                              int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, void* q_out,
                              int64_t ldqo, int32_t rotary_dim, int32_t layout, const int32_t* positions,
                              const int32_t* block_positions, const float* rope_tab, int32_t max_pos, int* status,
                              void* stream) {
  KvBatchDev bt;
  if (int rc = fl_kv_check("kv append", cache, batch, n_heads, &bt)) return rc;
  if (!k || !v || !status || (q && !q_out) || fl_misaligned(q, 16) || fl_misaligned(k, 16) || fl_misaligned(v, 16) ||
      fl_misaligned(q_out, 16) || fl_misaligned(status, 4))
    return fl_internal_error(FL_ERR_INVALID_ARG, "kv append: args");
  if (const char* w = rope_problem(cache->head_dim, rotary_dim, layout, positions, block_positions, rope_tab, max_pos))
    return fl_internal_error(FL_ERR_INVALID_ARG, "kv append: %s", w);
  if (!rope_supported(cache->head_dim, rotary_dim, block_positions))
    return fl_internal_error(FL_ERR_UNSUPPORTED, "kv append: rotary_dim %d", rotary_dim);
  if ((q && (ldq % 8 || ldqo % 8 || ldq < 0 || ldqo < 0)) || ldk % 8 || ldv % 8 || ldk < 0 || ldv < 0)
    return fl_internal_error(FL_ERR_UNSUPPORTED, "kv append: strides must be multiples of 8 elements, not negative");
  if (batch->n_tokens == 0) return FL_OK;
  bt.status = status;
  const Rope r{positions, block_positions, rope_tab, max_pos, rotary_dim, 1.f, layout == FL_ROPE_INTERLEAVED};
  return (cache->dtype == FL_DT_F16 ? launch_append<__half> : launch_append<__nv_bfloat16>)(
      cache, bt, n_heads, q, ldq, k, ldk, v, ldv, q_out, ldqo, r, status, (cudaStream_t)stream);
}
