// Layer norm of the chunk-aligned batch, each task with its own weights (mux_norm.h), forward and backward.
//
// All of it is bound by memory: about ten operations for the 4 (forward) or 6 bytes (backward) that a bf16 element moves.  A
// row is held in the registers of the lanes that own it from its first read to its last use, so that mean, squared
// deviations and the result (backward: both row sums and dX) take one pass over memory and the variance is summed from
// deviations, not as a difference of two large sums.  A wave owns a row (64 lanes, no barrier); wide rows belong to a workgroup.
// The gradients of the weights are sums down the columns: a lane keeps those of its columns in registers over the
// rows of its piece (part of a 64-row work item, so of one task), the waves of a workgroup are added in LDS, and a second launch
// adds the pieces of a task in their order (no atomics: results repeat bit for bit).
#include <algorithm>
#include <new>
#include <utility>

#include "mux_device_utils.h"
#include "mux_norm.h"

namespace mux {
namespace {

constexpr int kBatch = 32;      // tasks a launch (pointers as kernel arguments)

// VW consecutive elements of a row as they are stored
template <class S, int VW> struct Piece;
template <> struct Piece<bf16_t, 8> {
  uint4 r;
  __device__ __forceinline__ void load(const bf16_t* p) { r = *(const uint4*)p; }
  __device__ __forceinline__ void fill(bf16_t one) { const uint32_t v = one | (uint32_t)one << 16; r = uint4{v, v, v, v}; }
  __device__ __forceinline__ float get(int i) const {
    const uint32_t w = i < 2 ? r.x : i < 4 ? r.y : i < 6 ? r.z : r.w;
    return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
  }
  static __device__ __forceinline__ void store(bf16_t* p, const float* v) {
    *(uint4*)p = uint4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  }
};
template <> struct Piece<bf16_t, 1> {
  bf16_t r;
  __device__ __forceinline__ void load(const bf16_t* p) { r = *p; }
  __device__ __forceinline__ void fill(bf16_t one) { r = one; }
  __device__ __forceinline__ float get(int) const { return bf16_to_f32(r); }
  static __device__ __forceinline__ void store(bf16_t* p, const float* v) { *p = f32_to_bf16(v[0]); }
};
template <> struct Piece<float, 4> {
  float4 r;
  __device__ __forceinline__ void load(const float* p) { r = *(const float4*)p; }
  __device__ __forceinline__ void fill(float one) { r = float4{one, one, one, one}; }
  __device__ __forceinline__ float get(int i) const { return i == 0 ? r.x : i == 1 ? r.y : i == 2 ? r.z : r.w; }
  static __device__ __forceinline__ void store(float* p, const float* v) { *(float4*)p = float4{v[0], v[1], v[2], v[3]}; }
};
template <> struct Piece<float, 1> {
  float r;
  __device__ __forceinline__ void load(const float* p) { r = *p; }
  __device__ __forceinline__ void fill(float one) { r = one; }
  __device__ __forceinline__ float get(int) const { return r; }
  static __device__ __forceinline__ void store(float* p, const float* v) { *p = v[0]; }
};
template <class S> __device__ __forceinline__ S one_of();
template <> __device__ __forceinline__ bf16_t one_of<bf16_t>() { return 0x3F80; }
template <> __device__ __forceinline__ float one_of<float>() { return 1.f; }

struct NormParams {
  const int32_t* dtab;
  const void* gamma[kBatch];
  const void* beta[kBatch];
  int task_base;
  int item0;                // first 64-row work item of the launch
  int rows;                 // rows a piece: a power of two up to 64
  int N, T;
  float eps, inv_n;
  int64_t ldx, ldy;
  const void *X, *dY;
  void *Y, *dX;
  float *mean, *rstd;       // [T] each, null: not kept
  float* part;              // backward: [piece][2][N] partial sums of dgamma, dbeta, null: not wanted
};

// The rows of a workgroup: piece `blockIdx.x` of the launch, LPR lanes a row.
template <int LPR>
struct Rows {
  static constexpr int THREADS = LPR == 64 ? 256 : LPR, SUBS = THREADS / LPR;
  int task, row0, r0, r1;   // rows row0 + r0 .. row0 + r1 - 1, all of `task` (-1: of none)
  uint64_t valid;           // bit r: row0 + r is a token
  __device__ __forceinline__ Rows(const NormParams& p) {
    const int per = 64 / p.rows, item = p.item0 + (int)blockIdx.x / per;
    const ItemView it = load_item(p.dtab, 0, item);
    const uint32_t* bits = (const uint32_t*)(p.dtab + p.dtab[DH_OFF_ITEM_BITS]) + 2 * item;
    task = it.task;
    row0 = it.row0;
    r0 = (int)blockIdx.x % per * p.rows;
    r1 = min(r0 + p.rows, it.nrows);
    valid = task < 0 ? 0 : (uint64_t)bits[0] | (uint64_t)bits[1] << 32;
  }
  __device__ __forceinline__ bool any() const {      // a token among the piece's rows
    return r1 > r0 && (valid >> r0 & (~(uint64_t)0 >> (64 - (r1 - r0)))) != 0;
  }
};

// Sums over the LPR lanes of a row, the same value in every lane.  `slot` alternates between calls, so that one barrier a call is enough.
template <int LPR, int COUNT>
__device__ __forceinline__ void row_sum(float (&v)[COUNT], float (*lds)[COUNT][LPR / 64], int slot) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1)
#pragma unroll
    for (int k = 0; k < COUNT; ++k) v[k] += __shfl_xor(v[k], m);
  if constexpr (LPR > 64) {
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < COUNT; ++k) lds[slot][k][threadIdx.x >> 6] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < COUNT; ++k) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < LPR / 64; ++w) s += lds[slot][k][w];
      v[k] = s;
    }
  }
}

template <class S, int VW, int NV, int LPR>
__global__ __launch_bounds__(Rows<LPR>::THREADS) void k_norm_fwd(NormParams p) {
  typedef Piece<S, VW> P;
  __shared__ float lds[2][1][LPR / 64];
  const Rows<LPR> rows(p);
  const int sub = threadIdx.x / LPR, lane = threadIdx.x % LPR;
  const S* X = (const S*)p.X;
  S* Y = (S*)p.Y;
  P g[NV], b[NV];
  if (rows.task >= 0) {
    const S* gp = (const S*)p.gamma[rows.task - p.task_base];
    const S* bp = (const S*)p.beta[rows.task - p.task_base];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (lane + i * LPR) * VW;
      g[i].fill(one_of<S>());
      b[i].fill(0);
      if (gp && c < p.N) g[i].load(gp + c);
      if (bp && c < p.N) b[i].load(bp + c);
    }
  }
  for (int r = rows.r0 + sub; r < rows.r1; r += Rows<LPR>::SUBS) {
    const int row = rows.row0 + r;
    S* y = Y + (size_t)row * p.ldy;
    if (!(rows.valid >> r & 1)) {
      const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (lane + i * LPR) * VW;
        if (c < p.N) P::store(y + c, zero);
      }
      continue;
    }
    const S* x = X + (size_t)row * p.ldx;
    P v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (lane + i * LPR) * VW;
      v[i].fill(0);
      if (c < p.N) v[i].load(x + c);
    }
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < VW; ++e) s[0] += v[i].get(e);
    row_sum<LPR, 1>(s, lds, 0);
    const float mean = s[0] * p.inv_n;
    s[0] = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if ((lane + i * LPR) * VW >= p.N) continue;
#pragma unroll
      for (int e = 0; e < VW; ++e) {
        const float d = v[i].get(e) - mean;
        s[0] = fmaf(d, d, s[0]);
      }
    }
    row_sum<LPR, 1>(s, lds, 1);
    const float rstd = 1.f / sqrtf(s[0] * p.inv_n + p.eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (lane + i * LPR) * VW;
      if (c >= p.N) continue;
      float o[VW];
#pragma unroll
      for (int e = 0; e < VW; ++e) o[e] = fmaf((v[i].get(e) - mean) * rstd, g[i].get(e), b[i].get(e));
      P::store(y + c, o);
    }
    if (p.mean && lane == 0) { p.mean[row] = mean; p.rstd[row] = rstd; }
  }
}

template <class S, int VW, int NV, int LPR>
__global__ __launch_bounds__(Rows<LPR>::THREADS) void k_norm_bwd(NormParams p) {
  typedef Piece<S, VW> P;
  constexpr int SUBS = Rows<LPR>::SUBS;
  __shared__ float lds[2][2][LPR / 64];
  __shared__ float acc[SUBS > 1 ? 2 : 1][SUBS > 1 ? NV * VW * LPR : 1];
  const Rows<LPR> rows(p);
  const int sub = threadIdx.x / LPR, lane = threadIdx.x % LPR;
  const S *X = (const S*)p.X, *dY = (const S*)p.dY;
  S* dX = (S*)p.dX;
  P g[NV];
  float ag[NV][VW], ab[NV][VW];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    g[i].fill(one_of<S>());
#pragma unroll
    for (int e = 0; e < VW; ++e) ag[i][e] = ab[i][e] = 0.f;
  }
  if (rows.task >= 0) {
    const S* gp = (const S*)p.gamma[rows.task - p.task_base];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (lane + i * LPR) * VW;
      if (gp && c < p.N) g[i].load(gp + c);
    }
  }
  int slot = 0;
  for (int r = rows.r0 + sub; r < rows.r1; r += SUBS) {
    const int row = rows.row0 + r;
    S* dx = dX ? dX + (size_t)row * p.ldx : nullptr;
    if (!(rows.valid >> r & 1)) {
      if (!dx) continue;
      const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (lane + i * LPR) * VW;
        if (c < p.N) P::store(dx + c, zero);
      }
      continue;
    }
    const S *x = X + (size_t)row * p.ldx, *dy = dY + (size_t)row * p.ldy;
    P xv[NV], dv[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (lane + i * LPR) * VW;
      xv[i].fill(0);
      dv[i].fill(0);
      if (c < p.N) { xv[i].load(x + c); dv[i].load(dy + c); }
    }
    const float mean = p.mean[row], rstd = p.rstd[row];
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < VW; ++e) {
        const float xh = (xv[i].get(e) - mean) * rstd, d = dv[i].get(e), h = d * g[i].get(e);   // (d = 0 past the row)
        s[0] += h;
        s[1] = fmaf(h, xh, s[1]);
        ag[i][e] = fmaf(d, xh, ag[i][e]);
        ab[i][e] += d;
      }
    if (dx) {                                          // (uniform: every lane of the grid takes the same way)
      row_sum<LPR, 2>(s, lds, slot);
      slot ^= 1;
      const float m1 = s[0] * p.inv_n, m2 = s[1] * p.inv_n;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (lane + i * LPR) * VW;
        if (c >= p.N) continue;
        float o[VW];
#pragma unroll
        for (int e = 0; e < VW; ++e) {
          const float xh = (xv[i].get(e) - mean) * rstd, h = dv[i].get(e) * g[i].get(e);
          o[e] = rstd * (h - m1 - xh * m2);
        }
        P::store(dx + c, o);
      }
    }
  }
  if (!p.part || !rows.any()) return;                  // (uniform in the workgroup; k_norm_reduce skips the same pieces)
  float* part = p.part + ((size_t)p.item0 * (64 / p.rows) + blockIdx.x) * 2 * (size_t)p.N;
  if constexpr (SUBS > 1) {
    // the waves' sums one after the other, in a fixed order
    for (int w = SUBS - 1; w >= 0; --w) {
      if (sub == w) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int e = 0; e < VW; ++e) {
            const int at = (i * VW + e) * LPR + lane;
            if (w < SUBS - 1) { ag[i][e] += acc[0][at]; ab[i][e] += acc[1][at]; }
            if (w > 0) { acc[0][at] = ag[i][e]; acc[1][at] = ab[i][e]; }
          }
      }
      __syncthreads();
    }
    if (sub != 0) return;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (lane + i * LPR) * VW;
    if (c >= p.N) continue;
#pragma unroll
    for (int e = 0; e < VW; ++e) { part[c + e] = ag[i][e]; part[p.N + c + e] = ab[i][e]; }
  }
}

struct ReduceParams {
  const int32_t* dtab;
  float* dgamma[kBatch];
  float* dbeta[kBatch];
  int task_base, rows, N, accumulate;
  const float* part;
};

// The pieces of a task added up, in their order inside a wave, the waves in order.  grid = (64 columns each, the tasks of the launch, 2: dgamma, dbeta)
__global__ __launch_bounds__(1024) void k_norm_reduce(ReduceParams p) {
  __shared__ float lds[16][64];
  const int t = blockIdx.y, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int c = (int)blockIdx.x * 64 + lane;
  float* out = blockIdx.z ? p.dbeta[t] : p.dgamma[t];
  if (!out) return;
  float s = 0.f;
  if (p.part) {                                          // (null: a table without rows)
  const int32_t* ti = p.dtab + p.dtab[DH_NITEMS0 + 2] + 2 * (p.task_base + t);
  const int per = 64 / p.rows, begin = ti[0] * per, end = begin + ti[1] * per;
  const uint32_t* bits = (const uint32_t*)(p.dtab + p.dtab[DH_OFF_ITEM_BITS]);
  const uint64_t ones = ~(uint64_t)0 >> (64 - p.rows);
  for (int i = begin + wave; i < end; i += 16) {
    const uint32_t* w = bits + 2 * (i / per);
    const uint64_t valid = (uint64_t)w[0] | (uint64_t)w[1] << 32;
    if ((valid >> (i % per * p.rows) & ones) == 0) continue;       // no token: nothing was written
    if (c < p.N) s += p.part[((size_t)i * 2 + blockIdx.z) * (size_t)p.N + c];
  }
  }
  lds[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && c < p.N) {
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += lds[w][lane];
    out[c] = p.accumulate ? out[c] + s : s;
  }
}

mux_status check(const char* fn, const mux_norm_desc* d, const mux_segtab* st) {
  if (!d || !st) return fail(MUX_ERR_INVALID_ARG, std::string(fn) + ": null descriptor or table");
  if (d->dtype != MUX_DT_BF16 && d->dtype != MUX_DT_F32) return fail(MUX_ERR_INVALID_ARG, std::string(fn) + ": unknown dtype");
  if (d->width < 1) return fail(MUX_ERR_INVALID_ARG, std::string(fn) + ": width must be positive");
  if (!(d->eps > 0.f) || !(d->eps < INFINITY)) return fail(MUX_ERR_INVALID_ARG, std::string(fn) + ": eps must be positive and finite");
  if (d->width > MUX_NORM_MAX_WIDTH) return fail(MUX_ERR_UNSUPPORTED, std::string(fn) + ": width above MUX_NORM_MAX_WIDTH");
  if (d->ldx < d->width || d->ldy < d->width) return fail(MUX_ERR_SHAPE, std::string(fn) + ": a leading dimension is smaller than the width");
  if (d->n_tasks != st->n_tasks) return fail(MUX_ERR_SHAPE, std::string(fn) + ": descriptor and table disagree on the number of tasks");
  const int64_t ld = std::max(d->ldx, d->ldy);
  if (ld >= ((int64_t)1 << 40) || (int64_t)st->T * ld >= ((int64_t)1 << 40)) return fail(MUX_ERR_SHAPE, std::string(fn) + ": problem too large");
  return MUX_OK;
}

size_t esize(const mux_norm_desc* d) { return d->dtype == MUX_DT_F32 ? 4 : 2; }
size_t extent(const mux_norm_desc* d, const mux_segtab* st, int64_t ld) {       // bytes that T rows take
  return st->T > 0 ? ((size_t)(st->T - 1) * (size_t)ld + (size_t)d->width) * esize(d) : 0;
}

// Rows a workgroup takes, and so the number of partial sums.
int piece_rows(const mux_segtab* st) {
  int rows = 64;
  while (rows > 4 && (st->T + rows - 1) / rows < 2 * kComputeUnits) rows /= 2;
  return rows;
}

#define NORM_CASE(K, S, VW, NV, LPR) \
  else if (pieces <= NV * LPR) MUX_LAUNCH(name, (K<S, VW, NV, LPR>), grid, dim3(Rows<LPR>::THREADS), 0, stream, p)
#define NORM_LAUNCH(K, wave_most)                                                                                      \
  do {                                                                                                                 \
    const int pieces = vec ? d->width * (int)esize(d) / 16 : d->width;                                                 \
    if (d->dtype == MUX_DT_BF16 && vec) {                                                                              \
      if (false) {}                                                                                                    \
      NORM_CASE(K, bf16_t, 8, 1, 64); NORM_CASE(K, bf16_t, 8, 2, 64); NORM_CASE(K, bf16_t, 8, 4, 64);                  \
      NORM_CASE(K, bf16_t, 8, 5, 64); NORM_CASE(K, bf16_t, 8, 8, 64); NORM_CASE(K, bf16_t, 8, 10, 64);                 \
      NORM_CASE(K, bf16_t, 8, 4, 256); NORM_CASE(K, bf16_t, 8, 4, 1024);                                               \
    } else if (d->dtype == MUX_DT_BF16) {                                                                              \
      if (false) {}                                                                                                    \
      NORM_CASE(K, bf16_t, 1, 8, 64); NORM_CASE(K, bf16_t, 1, 8, 256); NORM_CASE(K, bf16_t, 1, 20, 256);               \
      NORM_CASE(K, bf16_t, 1, 32, 1024);                                                                               \
    } else if (vec) {                                                                                                  \
      if (false) {}                                                                                                    \
      NORM_CASE(K, float, 4, 2, 64); NORM_CASE(K, float, 4, 4, 64); NORM_CASE(K, float, 4, 10, 64);                    \
      NORM_CASE(K, float, 4, 16, 64); NORM_CASE(K, float, 4, 8, 256); NORM_CASE(K, float, 4, 8, 1024);                 \
    } else {                                                                                                           \
      if (false) {}                                                                                                    \
      NORM_CASE(K, float, 1, 8, 64); NORM_CASE(K, float, 1, 8, 256); NORM_CASE(K, float, 1, 20, 256);                  \
      NORM_CASE(K, float, 1, 32, 1024);                                                                                \
    }                                                                                                                  \
  } while (0)

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Launches over the tasks of the table, kBatch at a time, each over the work items of its tasks (the first also over those
// before them, the last over those behind).
template <bool BACKWARD>
void launch(const char* name, const mux_norm_desc* d, const mux_segtab* st, NormParams p, bool vec, hipStream_t stream) {
  p.rows = piece_rows(st);
  for (int base = 0; base < st->n_tasks; base += kBatch) {
    const int n = std::min(kBatch, st->n_tasks - base);
    p.task_base = base;
    for (int i = 0; i < n; ++i) {
      p.gamma[i] = d->gamma ? d->gamma[base + i] : nullptr;
      p.beta[i] = d->beta ? d->beta[base + i] : nullptr;
    }
    p.item0 = base == 0 ? 0 : st->task_item_begin[0][base];
    const int end = base + n == st->n_tasks ? (int)st->items[0].size() : st->task_item_begin[0][base + n];
    if (end <= p.item0) continue;
    const dim3 grid((unsigned)(end - p.item0) * (unsigned)(64 / p.rows));
    if constexpr (BACKWARD) NORM_LAUNCH(k_norm_bwd, 10);
    else NORM_LAUNCH(k_norm_fwd, 10);
  }
}

// Whether every row and weight can be moved in 16-byte pieces; false in `ok` where a pointer is not aligned to its element.
bool pieces16(const mux_norm_desc* d, std::initializer_list<const void*> ptrs, bool& ok) {
  const size_t e = esize(d);
  bool vec = d->width * e % 16 == 0 && d->ldx * (int64_t)e % 16 == 0 && d->ldy * (int64_t)e % 16 == 0;
  ok = true;
  auto look = [&](const void* q) {
    if ((uintptr_t)q % e) ok = false;
    if (!aligned16(q)) vec = false;
  };
  for (const void* q : ptrs) look(q);
  for (int t = 0; t < d->n_tasks; ++t) {
    if (d->gamma) look(d->gamma[t]);
    if (d->beta) look(d->beta[t]);
  }
  return vec;
}

// Whether the bytes [w, w + nw) that a call writes overlap the [r, r + nr) that it reads in another way than row by row in place
bool clash(const void* w, size_t nw, int64_t ldw, const void* r, size_t nr, int64_t ldr) {
  return overlap(w, nw, r, nr) && !(w == r && ldw == ldr);
}

mux_status last_hip(const char* fn) {
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(MUX_ERR_DEVICE, std::string(fn) + ": " + hipGetErrorString(e));
  return MUX_OK;
}

}  // namespace
}  // namespace mux

using namespace mux;

extern "C" size_t mux_norm_saved_bytes(const mux_norm_desc* desc, const mux_segtab* st) {
  if (!desc || !st) return 0;
  return align256((size_t)st->T * 2 * sizeof(float));
}

extern "C" size_t mux_norm_workspace_bytes(const mux_norm_desc* desc, const mux_segtab* st) {
  if (!desc || !st || desc->width < 1) return 0;
  return align256(st->items[0].size() * (size_t)(64 / piece_rows(st)) * 2 * (size_t)desc->width * sizeof(float));
}

extern "C" mux_status mux_norm_forward(const mux_norm_desc* desc, const mux_segtab* st, const void* dev_segtab, const void* X,
                                       void* Y, void* saved, void* hip_stream) {
  static const char* fn = "mux_norm_forward";
  if (mux_status s = check(fn, desc, st)) return s;
  if (st->T == 0) return MUX_OK;
  if (!dev_segtab || !X || !Y) return fail(MUX_ERR_INVALID_ARG, std::string(fn) + ": null device pointer");
  bool ok;
  const bool vec = pieces16(desc, {X, Y}, ok);
  if (!ok || (uintptr_t)saved % 4) return fail(MUX_ERR_UNSUPPORTED, std::string(fn) + ": a pointer is not aligned to its element");
  const size_t nx = extent(desc, st, desc->ldx), ny = extent(desc, st, desc->ldy), nw = (size_t)desc->width * esize(desc);
  const size_t ns = (size_t)st->T * 2 * sizeof(float);
  bool bad = clash(Y, ny, desc->ldy, X, nx, desc->ldx) || overlap(saved, ns, X, nx) || overlap(saved, ns, Y, ny);
  for (int t = 0; t < desc->n_tasks; ++t) {
    if (desc->gamma) bad = bad || overlap(Y, ny, desc->gamma[t], nw) || overlap(saved, ns, desc->gamma[t], nw);
    if (desc->beta) bad = bad || overlap(Y, ny, desc->beta[t], nw) || overlap(saved, ns, desc->beta[t], nw);
  }
  if (bad) return fail(MUX_ERR_INVALID_ARG, std::string(fn) + ": an output overlaps an input");
  NormParams p{};
  p.dtab = (const int32_t*)dev_segtab;
  p.N = desc->width; p.T = st->T;
  p.eps = desc->eps; p.inv_n = 1.f / (float)desc->width;
  p.ldx = desc->ldx; p.ldy = desc->ldy;
  p.X = X; p.Y = Y;
  p.mean = (float*)saved; p.rstd = saved ? (float*)saved + st->T : nullptr;
  launch<false>("norm_fwd", desc, st, p, vec, (hipStream_t)hip_stream);
  return last_hip(fn);
}

extern "C" mux_status mux_norm_backward(const mux_norm_desc* desc, const mux_segtab* st, const void* dev_segtab, const void* X,
                                        const void* dY, const void* saved, void* dX, void* const* dgamma, void* const* dbeta,
                                        int accumulate, void* ws, size_t ws_bytes, void* hip_stream) {
  static const char* fn = "mux_norm_backward";
  if (mux_status s = check(fn, desc, st)) return s;
  if (accumulate != 0 && accumulate != 1) return fail(MUX_ERR_INVALID_ARG, std::string(fn) + ": accumulate must be 0 or 1");
  if (st->T > 0 && (!dev_segtab || !X || !dY || !saved)) return fail(MUX_ERR_INVALID_ARG, std::string(fn) + ": null device pointer");
  const size_t nx = extent(desc, st, desc->ldx), ny = extent(desc, st, desc->ldy), nw = (size_t)desc->width * esize(desc);
  const size_t ng = (size_t)desc->width * sizeof(float), ns = (size_t)st->T * 2 * sizeof(float);
  std::vector<std::pair<uintptr_t, uintptr_t>> grads;    // the gradients' bytes
  bool aligned = (uintptr_t)saved % 4 == 0;
  try {
    grads.reserve((size_t)desc->n_tasks * 2);
    for (int t = 0; t < desc->n_tasks; ++t)
      for (void* const* list : {dgamma, dbeta})
        if (list && list[t]) {
          grads.push_back({(uintptr_t)list[t], (uintptr_t)list[t] + ng});
          aligned = aligned && (uintptr_t)list[t] % 4 == 0;
        }
    std::sort(grads.begin(), grads.end());
  } catch (const std::bad_alloc&) {
    return fail(MUX_ERR_HOST_NOMEM, std::string(fn) + ": out of host memory");
  }
  const bool wants = !grads.empty();
  if (!wants && (!dX || st->T == 0)) return MUX_OK;
  const size_t need = st->T > 0 && wants ? mux_norm_workspace_bytes(desc, st) : 0;
  if (need > 0 && !ws) return fail(MUX_ERR_INVALID_ARG, std::string(fn) + ": null workspace");
  if (ws_bytes < need) return fail(MUX_ERR_WORKSPACE, std::string(fn) + ": workspace too small");
  bool ok;
  const bool vec = pieces16(desc, {X, dY, dX}, ok);
  if (!ok || !aligned || (need > 0 && (uintptr_t)ws % 4))
    return fail(MUX_ERR_UNSUPPORTED, std::string(fn) + ": a pointer is not aligned to its element");
  bool bad = clash(dX, nx, desc->ldx, X, nx, desc->ldx) || clash(dX, nx, desc->ldx, dY, ny, desc->ldy) || overlap(dX, nx, saved, ns);
  for (size_t i = 0; i < grads.size(); ++i) {
    const void* q = (const void*)grads[i].first;
    bad = bad || (i > 0 && grads[i].first < grads[i - 1].second) || overlap(q, ng, X, nx) || overlap(q, ng, dY, ny) ||
          overlap(q, ng, dX, nx) || overlap(q, ng, saved, ns) || overlap(q, ng, ws, need);
  }
  for (int t = 0; t < desc->n_tasks; ++t)
    if (desc->gamma) bad = bad || overlap(dX, nx, desc->gamma[t], nw) || overlap(ws, need, desc->gamma[t], nw);
  for (const auto& r : {std::pair<const void*, size_t>(X, nx), {dY, ny}, {dX, nx}, {saved, ns}}) bad = bad || overlap(ws, need, r.first, r.second);
  if (bad) return fail(MUX_ERR_INVALID_ARG, std::string(fn) + ": an output overlaps an input or another output");
  hipStream_t stream = (hipStream_t)hip_stream;
  NormParams p{};
  p.dtab = (const int32_t*)dev_segtab;
  p.N = desc->width; p.T = st->T;
  p.eps = desc->eps; p.inv_n = 1.f / (float)desc->width;
  p.ldx = desc->ldx; p.ldy = desc->ldy;
  p.X = X; p.dY = dY; p.dX = dX;
  p.mean = (float*)saved; p.rstd = saved ? (float*)saved + st->T : nullptr;
  p.part = need > 0 ? (float*)ws : nullptr;
  if (st->T > 0) launch<true>("norm_bwd", desc, st, p, vec, stream);
  if (wants) {
    ReduceParams q{};
    q.dtab = (const int32_t*)dev_segtab;
    q.rows = piece_rows(st);
    q.N = desc->width;
    q.accumulate = accumulate;
    q.part = p.part;
    for (int base = 0; base < st->n_tasks; base += kBatch) {
      const int n = std::min(kBatch, st->n_tasks - base);
      q.task_base = base;
      for (int i = 0; i < n; ++i) {
        q.dgamma[i] = dgamma ? (float*)dgamma[base + i] : nullptr;
        q.dbeta[i] = dbeta ? (float*)dbeta[base + i] : nullptr;
      }
      MUX_LAUNCH("norm_reduce", k_norm_reduce, dim3((unsigned)(desc->width + 63) / 64, (unsigned)n, 2), dim3(1024), 0, stream, q);
    }
  }
  return last_hip(fn);
}
