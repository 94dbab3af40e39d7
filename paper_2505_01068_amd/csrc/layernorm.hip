// Layer normalisation of rows, forward and backward, as entry points of their own (include/imattn.h).
//
// Bound by HBM: the forward reads and writes a row once, the backward reads x and dy and writes dx once.  A row lives in the
// registers of LPR lanes (4 .. 64 of a wave, or a whole workgroup of 256 / 1024), NC chunks of 16 bytes each, so that mean,
// centred squares and the two sums of the gradient are taken over registers: two passes for the variance cost no traffic.
// 36864 rows of 1024 in bf16: forward 24 us (6.2 TB/s), backward 48 + 5 us (4.7 TB/s) -- a large copy reaches 4.8 TB/s from HBM, and a part of
// what is read was written just before; 48 rows of 32 in fp32: 2.2 us.
// The gradients of gain and bias: every thread keeps the sums of its own columns over the rows that it meets, the
// workgroup adds its threads' in a fixed order and writes one partial row; a second launch adds the partial rows.
#include <algorithm>

#include "entry.hpp"
#include "mfma_common.hpp"

namespace imattn {

template <class T> struct NormChunk { static constexpr int E = 16 / (int)sizeof(T); };

// The elements of a row that a lane holds, as they lie in memory; their conversion is a step of its own, so that loads can be under way across
// other work.  VEC (rows in whole, aligned 16-byte chunks): chunk lane + c LPR, elements side by side.  Otherwise element by element, neighbours in
// neighbouring lanes: element lane + (c E + e) LPR, so that odd widths are read and written in whole lines too.
template <class T, int LPR, int NC, bool VEC>
struct RowPart {
  static constexpr int E = NormChunk<T>::E;
  static __device__ __forceinline__ int at(int lane, int c, int e) { return VEC ? (lane + c * LPR) * E + e : lane + (c * E + e) * LPR; }
  u32x4 chunk[VEC ? NC : 1];
  T one[VEC ? 1 : NC * E];
  __device__ __forceinline__ void load(const T* p, bool is, int lane, int d) {   // what is missing is 0
    if constexpr (VEC) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        chunk[c] = u32x4{0u, 0u, 0u, 0u};
        if (is && at(lane, c, 0) < d) chunk[c] = *(const u32x4*)(p + at(lane, c, 0));
      }
    } else {
#pragma unroll
      for (int i = 0; i < NC * E; ++i) one[i] = T(0);
      if (is) {   // no branch between the loads: behind the end the last element again
#pragma unroll
        for (int i = 0; i < NC * E; ++i) one[i] = p[min(at(lane, 0, i), d - 1)];
      }
    }
  }
  __device__ __forceinline__ void get(int lane, int d, float (&v)[NC][E]) const {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if constexpr (!VEC) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[c][e] = at(lane, c, e) < d ? ldf(&one[c * E + e]) : 0.f;
      } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[c][e] = __uint_as_float(chunk[c][e]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[c][2 * e] = __uint_as_float(chunk[c][e] << 16);
          v[c][2 * e + 1] = __uint_as_float(chunk[c][e] & 0xffff0000u);
        }
      }
    }
  }
  static __device__ __forceinline__ void store(T* p, int lane, int d, const float (&v)[NC][E]) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if constexpr (!VEC) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (at(lane, c, e) < d) stf(p + at(lane, c, e), v[c][e]);
      } else if (at(lane, c, 0) < d) {
        u32x4 u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (sizeof(T) == 4) u[e] = __float_as_uint(v[c][e]);
          else u[e] = pack_bf16(v[c][2 * e], v[c][2 * e + 1]);
        }
        *(u32x4*)(p + at(lane, c, 0)) = u;
      }
    }
  }
};

// sum over the LPR lanes of a row; LPR > 64: over the workgroup, through `red` (one float a wave and call site)
template <int LPR>
__device__ __forceinline__ float row_sum(float v, float* red) {
#pragma unroll
  for (int o = (LPR < 64 ? LPR : 64) / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if constexpr (LPR > 64) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < LPR / 64; ++w) v += red[w];
  }
  return v;
}

struct NormArgs {
  long rows;
  int d, vec;                      // vec: every row, gamma and beta in whole, aligned 16-byte chunks
  const void *x, *gamma, *beta, *dy;
  long ldx, ldy, lddy, lddx;
  void *y, *dx;
  float *mean, *rstd, *partial, *dgamma, *dbeta;
  float eps, inv_d;
};

template <class T, int LPR, int NC, bool VEC>
__global__ __launch_bounds__(LPR > 256 ? LPR : 256) void norm_fwd_kernel(NormArgs a) {
  using Part = RowPart<T, LPR, NC, VEC>;
  constexpr int E = NormChunk<T>::E, WG = LPR > 256 ? LPR : 256, RPW = WG / LPR;
  __shared__ float red[2][2][WG / 64];
  touch_args<NormArgs>();
  const int lane = threadIdx.x % LPR;
  Part pg, pb;
  if (a.gamma) pg.load((const T*)a.gamma, true, lane, a.d);
  if (a.beta) pb.load((const T*)a.beta, true, lane, a.d);
  int turn = 0;   // the reduction buffers alternate, so that one barrier a sum suffices
  for (long row0 = (long)blockIdx.x * RPW; row0 < a.rows; row0 += (long)gridDim.x * RPW, turn ^= 1) {
    const long row = row0 + threadIdx.x / LPR;
    const bool mine = row < a.rows;
    Part part;
    float v[NC][E];
    part.load((const T*)a.x + row * a.ldx, mine, lane, a.d);
    part.get(lane, a.d, v);
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < E; ++e) s += v[c][e];
    const float mean = row_sum<LPR>(s, red[turn][0]) * a.inv_d;
    s = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v[c][e] -= mean;
        if (Part::at(lane, c, e) < a.d) s += v[c][e] * v[c][e];
      }
    const float rstd = 1.0f / sqrtf(row_sum<LPR>(s, red[turn][1]) * a.inv_d + a.eps);
    if (!mine) continue;
    if (a.mean && lane == 0) { a.mean[row] = mean; a.rstd[row] = rstd; }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < E; ++e) v[c][e] *= rstd;
    if (a.gamma) {
      float g[NC][E];
      pg.get(lane, a.d, g);
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < E; ++e) v[c][e] *= g[c][e];
    }
    if (a.beta) {
      float b[NC][E];
      pb.get(lane, a.d, b);
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < E; ++e) v[c][e] += b[c][e];
    }
    Part::store((T*)a.y + row * a.ldy, lane, a.d, v);
  }
}

template <class T, int LPR, int NC, bool VEC>
__global__ __launch_bounds__(LPR > 256 ? LPR : 256) void norm_bwd_kernel(NormArgs a) {
  using Part = RowPart<T, LPR, NC, VEC>;
  constexpr int E = NormChunk<T>::E, WG = LPR > 256 ? LPR : 256, RPW = WG / LPR;
  constexpr int COLS = LPR * NC * E;
  __shared__ float red[2][2][WG / 64];
  touch_args<NormArgs>();
  __shared__ float cols[LPR > 64 ? 1 : 2 * COLS];   // the workgroup's sums, where several waves share columns
  const int lane = threadIdx.x % LPR;
  float g[NC][E], dg[NC][E], db[NC][E];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int e = 0; e < E; ++e) { g[c][e] = 1.f; dg[c][e] = db[c][e] = 0.f; }
  if (a.gamma) {
    Part part;
    part.load((const T*)a.gamma, true, lane, a.d);
    part.get(lane, a.d, g);
  }
  int turn = 0;   // the reduction buffers alternate, so that one barrier a sum suffices
  // the next row's loads are under way while a row is worked on (36864 rows of 1024 in bf16: 69 -> 49 us)
  const long step = (long)gridDim.x * RPW;
  Part px, pdy;
  float next_mean = 0.f, next_rstd = 0.f;
  auto fetch = [&](long row) {
    const bool is = row < a.rows;
    next_mean = next_rstd = 0.f;
    if (is) { next_mean = a.mean[row]; next_rstd = a.rstd[row]; }
    px.load((const T*)a.x + row * a.ldx, is, lane, a.d);
    pdy.load((const T*)a.dy + row * a.lddy, is, lane, a.d);
  };
  fetch((long)blockIdx.x * RPW + threadIdx.x / LPR);
  for (long row0 = (long)blockIdx.x * RPW; row0 < a.rows; row0 += step, turn ^= 1) {
    const long row = row0 + threadIdx.x / LPR;
    const bool mine = row < a.rows;
    float xh[NC][E], w[NC][E];
    float s1 = 0.f, s2 = 0.f;
    const float mean = next_mean, rstd = next_rstd;
    px.get(lane, a.d, xh);
    pdy.get(lane, a.d, w);
    if (row0 + step < a.rows) fetch(row + step);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        xh[c][e] = Part::at(lane, c, e) < a.d ? (xh[c][e] - mean) * rstd : 0.f;   // (rows behind the last: mean = rstd = 0)
        dg[c][e] += w[c][e] * xh[c][e];
        db[c][e] += w[c][e];
        w[c][e] *= g[c][e];
        s1 += w[c][e];
        s2 += w[c][e] * xh[c][e];
      }
    if (!a.dx) continue;
    s1 = row_sum<LPR>(s1, red[turn][0]) * a.inv_d;
    s2 = row_sum<LPR>(s2, red[turn][1]) * a.inv_d;
    if (!mine) continue;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < E; ++e) w[c][e] = rstd * (w[c][e] - s1 - xh[c][e] * s2);
    Part::store((T*)a.dx + row * a.lddx, lane, a.d, w);
  }
  if (!a.partial && !a.dgamma && !a.dbeta) return;
  float* out_g = a.partial ? a.partial + (long)blockIdx.x * 2 * a.d : a.dgamma;
  float* out_b = a.partial ? out_g + a.d : a.dbeta;
  if constexpr (LPR > 64) {   // every thread has columns of its own
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int at = Part::at(lane, c, e);
        if (at < a.d && out_g) out_g[at] = dg[c][e];
        if (at < a.d && out_b) out_b[at] = db[c][e];
      }
  } else {
    // rows of a wave, then wave after wave; element (c, e) of lane l at (c E + e) LPR + l: neighbouring lanes in neighbouring banks
    for (int wv = 0; wv < WG / 64; ++wv) {
      if ((int)(threadIdx.x >> 6) == wv) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < E; ++e) {
            float p = dg[c][e], q = db[c][e];
#pragma unroll
            for (int o = 32; o >= LPR; o >>= 1) { p += __shfl_xor(p, o); q += __shfl_xor(q, o); }
            const int at = (c * E + e) * LPR + lane;
            if ((int)(threadIdx.x & 63) < LPR) {
              cols[at] = wv ? cols[at] + p : p;
              cols[COLS + at] = wv ? cols[COLS + at] + q : q;
            }
          }
      }
      __syncthreads();
    }
    for (int at = threadIdx.x; at < a.d; at += WG) {
      const int ce = VEC ? at / (E * LPR) * E + at % E : at / LPR, l = VEC ? at / E % LPR : at % LPR;
      if (out_g) out_g[at] = cols[ce * LPR + l];
      if (out_b) out_b[at] = cols[COLS + ce * LPR + l];
    }
  }
}

// Column sums of the partial rows [parts][2 d]: 32 columns a workgroup, its 32 rows of threads take every 32nd part and are
// added in their order.
__global__ __launch_bounds__(1024) void norm_reduce_kernel(const float* __restrict__ partial, int parts, int d, float* dgamma, float* dbeta) {
  __shared__ float sums[32][33];
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), r = threadIdx.x >> 5;
  float s = 0.f;
  if (col < 2 * d) {
#pragma unroll 8
    for (int p = r; p < parts; p += 32) s += partial[(long)p * 2 * d + col];
  }
  sums[r][threadIdx.x & 31] = s;
  __syncthreads();
  if (r == 0 && col < 2 * d) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += sums[i][threadIdx.x & 31];
    if (col < d) { if (dgamma) dgamma[col] = s; }
    else if (dbeta) dbeta[col - d] = s;
  }
}

// Lanes of a row: as few as hold it at one chunk a lane, up to a wave with four; then a workgroup.
static int norm_lanes(int d, int E) {
  const int chunks = (d + E - 1) / E;
  if (chunks > 1024) return 1024;
  if (chunks > 256) return 256;
  int l = 4;
  while (l < 64 && l < chunks) l *= 2;
  return l;
}
static long norm_row_blocks(long rows, int d, int E) {
  const int lpr = norm_lanes(d, E), rpw = lpr > 256 ? 1 : 256 / lpr;
  return (rows + rpw - 1) / rpw;
}
// Workgroups of the backward: 4 a CU walk over the rows, each one partial row of the gain's and the bias's gradient.
static int norm_bwd_grid(long rows, int d, int E) {
  return (int)std::min<long>(norm_row_blocks(rows, d, E), 4l * cu_count());
}

// The forward: a workgroup for every row or rows that fill it; where elements are loaded one by one (up to 64 loads a lane for gain and bias), 8 a CU walk
// over the rows and load these once (20000 rows of 1111 in bf16: 90 -> 42 us; whole chunks at 1024: 24 us, 6.3 TB/s).
static long norm_fwd_grid(const NormArgs& a, int E) {
  return std::min(norm_row_blocks(a.rows, a.d, E), a.vec ? 1l << 21 : 8l * cu_count());
}

template <class T>
static void norm_launch(const NormArgs& a, bool bwd, hipStream_t st) {
  constexpr int E = NormChunk<T>::E;
  const int lpr = norm_lanes(a.d, E), chunks = (a.d + E - 1) / E, nc = (chunks + lpr - 1) / lpr;
  const dim3 block(lpr > 256 ? lpr : 256), grid(bwd ? (unsigned)norm_bwd_grid(a.rows, a.d, E) : (unsigned)norm_fwd_grid(a, E));
#define NORM_GO(L, N)                                                                         \
  do {                                                                                        \
    if (bwd && a.vec) hipLaunchKernelGGL((norm_bwd_kernel<T, L, N, true>), grid, block, 0, st, a);   \
    else if (bwd) hipLaunchKernelGGL((norm_bwd_kernel<T, L, N, false>), grid, block, 0, st, a);      \
    else if (a.vec) hipLaunchKernelGGL((norm_fwd_kernel<T, L, N, true>), grid, block, 0, st, a);     \
    else hipLaunchKernelGGL((norm_fwd_kernel<T, L, N, false>), grid, block, 0, st, a);               \
  } while (0)
#define NORM_NC(L)                                                                            \
  do {                                                                                        \
    if (nc <= 2) NORM_GO(L, 2);                                                               \
    else NORM_GO(L, 4);                                                                       \
  } while (0)
  switch (lpr) {
    case 4: NORM_GO(4, 1); break;
    case 8: NORM_GO(8, 1); break;
    case 16: NORM_GO(16, 1); break;
    case 32: NORM_GO(32, 1); break;
    case 64: if (nc == 1) NORM_GO(64, 1); else NORM_NC(64); break;
    case 256: NORM_NC(256); break;
    default:   // (bf16 rows of IM_NORM_MAX_D have two chunks a lane)
      if constexpr (2 * 1024 * E < IM_NORM_MAX_D) NORM_NC(1024);
      else NORM_GO(1024, 2);
  }
#undef NORM_NC
#undef NORM_GO
}

static int norm_check(const char* what, int64_t rows, int32_t d, int32_t dtype) {
  if (dtype != IM_DTYPE_F32 && dtype != IM_DTYPE_BF16) return refuse(IM_ERR_INVALID, "%s: dtype must be IM_DTYPE_F32 or IM_DTYPE_BF16 (got %d)", what, dtype);
  if (rows < 0 || rows > (1ll << 31)) return refuse(IM_ERR_INVALID, "%s: rows must be in 0..2^31 (got %lld)", what, (long long)rows);
  if (d < 1) return refuse(IM_ERR_INVALID, "%s: d must be >= 1 (got %d)", what, d);
  if (d > IM_NORM_MAX_D) return refuse(IM_ERR_UNSUPPORTED, "%s: d must be <= %d (got %d)", what, IM_NORM_MAX_D, d);
  return IM_OK;
}
static int norm_rows_check(const char* what, const char* name, const void* p, int64_t ld, int64_t rows, int32_t d, size_t es) {
  if (rows == 0) return IM_OK;
  if (!p) return refuse(IM_ERR_INVALID, "%s: %s is NULL", what, name);
  if ((uintptr_t)p % es) return refuse(IM_ERR_INVALID, "%s: %s is not aligned to its elements", what, name);
  if (ld < d || ld > (1ll << 40)) return refuse(IM_ERR_INVALID, "%s: the row distance of %s must be at least d", what, name);
  return IM_OK;
}

}  // namespace imattn

using namespace imattn;

extern "C" {

int im_layernorm_sizes(int64_t rows, int32_t d, int32_t dtype, size_t* workspace_bytes) {
  if (int rc = norm_check("im_layernorm_sizes", rows, d, dtype)) return rc;
  if (!workspace_bytes) return refuse(IM_ERR_INVALID, "im_layernorm_sizes: workspace_bytes is NULL");
  const int grid = norm_bwd_grid(rows, d, dtype == IM_DTYPE_BF16 ? 8 : 4);
  *workspace_bytes = grid > 1 ? round256((size_t)grid * 2 * d * sizeof(float)) : 0;
  return IM_OK;
}

int im_layernorm_fwd(int64_t rows, int32_t d, int32_t dtype, const void* x, int64_t ldx, const void* gamma, const void* beta,
                     float eps, void* y, int64_t ldy, float* mean, float* rstd, void* hip_stream) {
  const char* what = "im_layernorm_fwd";
  if (int rc = norm_check(what, rows, d, dtype)) return rc;
  const size_t es = dtype == IM_DTYPE_BF16 ? 2 : 4;
  if (int rc = norm_rows_check(what, "x", x, ldx, rows, d, es)) return rc;
  if (int rc = norm_rows_check(what, "y", y, ldy, rows, d, es)) return rc;
  if (x == y && rows > 1 && ldx != ldy) return refuse(IM_ERR_INVALID, "%s: in place, the row distances of x and y must be the same", what);
  if (!(eps > 0.f) || eps > 3e38f) return refuse(IM_ERR_INVALID, "%s: eps must be finite and > 0", what);
  if (!mean != !rstd) return refuse(IM_ERR_INVALID, "%s: mean and rstd: both or neither", what);
  if (((uintptr_t)gamma | (uintptr_t)beta) % es) return refuse(IM_ERR_INVALID, "%s: gamma or beta is not aligned to its elements", what);
  if (((uintptr_t)mean | (uintptr_t)rstd) % 4) return refuse(IM_ERR_INVALID, "%s: mean or rstd is not aligned to its elements", what);
  if (rows == 0) return IM_OK;
  NormArgs a = {};
  a.rows = rows; a.d = d; a.x = x; a.ldx = ldx; a.gamma = gamma; a.beta = beta; a.y = y; a.ldy = ldy; a.mean = mean; a.rstd = rstd;
  a.eps = eps; a.inv_d = 1.0f / (float)d;
  a.vec = (((uintptr_t)x | (uintptr_t)y | (uintptr_t)gamma | (uintptr_t)beta) % 16 == 0) && d * es % 16 == 0 && ldx * es % 16 == 0 && ldy * es % 16 == 0;
  hipStream_t st = (hipStream_t)hip_stream;
  ProfScope ps(PF_MISC, st);
  if (dtype == IM_DTYPE_BF16) norm_launch<bf16_t>(a, false, st);
  else norm_launch<float>(a, false, st);
  return after_launch(what);
}

int im_layernorm_bwd(int64_t rows, int32_t d, int32_t dtype, const void* x, int64_t ldx, const void* gamma, const float* mean,
                     const float* rstd, const void* dy, int64_t lddy, void* dx, int64_t lddx, float* dgamma, float* dbeta,
                     void* workspace, size_t workspace_bytes, void* hip_stream) {
  const char* what = "im_layernorm_bwd";
  if (int rc = norm_check(what, rows, d, dtype)) return rc;
  const size_t es = dtype == IM_DTYPE_BF16 ? 2 : 4;
  if (int rc = norm_rows_check(what, "x", x, ldx, rows, d, es)) return rc;
  if (int rc = norm_rows_check(what, "dy", dy, lddy, rows, d, es)) return rc;
  if (!dx && !dgamma && !dbeta) return refuse(IM_ERR_INVALID, "%s: dx, dgamma and dbeta are all NULL", what);
  if (dx) if (int rc = norm_rows_check(what, "dx", dx, lddx, rows, d, es)) return rc;
  if (dx && dx == dy && rows > 1 && lddx != lddy) return refuse(IM_ERR_INVALID, "%s: in place, the row distances of dy and dx must be the same", what);
  if (rows > 0 && (!mean || !rstd)) return refuse(IM_ERR_INVALID, "%s: mean and rstd of the forward are needed", what);
  if ((uintptr_t)gamma % es) return refuse(IM_ERR_INVALID, "%s: gamma is not aligned to its elements", what);
  if (((uintptr_t)mean | (uintptr_t)rstd | (uintptr_t)dgamma | (uintptr_t)dbeta) % 4)
    return refuse(IM_ERR_INVALID, "%s: mean, rstd, dgamma or dbeta is not aligned to its elements", what);
  const int grid = norm_bwd_grid(rows, d, dtype == IM_DTYPE_BF16 ? 8 : 4);
  const bool sums = dgamma || dbeta;
  const size_t need = sums && grid > 1 ? round256((size_t)grid * 2 * d * sizeof(float)) : 0;
  if (need && (!workspace || workspace_bytes < need)) return refuse(IM_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", what, workspace_bytes, need);
  if (need && (uintptr_t)workspace % 16) return refuse(IM_ERR_INVALID, "%s: workspace must be 16-byte aligned", what);
  hipStream_t st = (hipStream_t)hip_stream;
  ProfScope ps(PF_MISC, st);
  if (rows == 0) {   // empty sums: no partial rows to read
    if (sums) hipLaunchKernelGGL(norm_reduce_kernel, dim3((2 * d + 31) / 32), dim3(1024), 0, st, (const float*)nullptr, 0, d, dgamma, dbeta);
    return after_launch(what);
  }
  NormArgs a = {};
  a.rows = rows; a.d = d; a.x = x; a.ldx = ldx; a.gamma = gamma; a.dy = dy; a.lddy = lddy; a.dx = dx; a.lddx = dx ? lddx : d;
  a.mean = (float*)mean; a.rstd = (float*)rstd; a.inv_d = 1.0f / (float)d;
  a.partial = need ? (float*)workspace : nullptr; a.dgamma = dgamma; a.dbeta = dbeta;
  a.vec = (((uintptr_t)x | (uintptr_t)dy | (uintptr_t)dx | (uintptr_t)gamma) % 16 == 0) && d * es % 16 == 0 && ldx * es % 16 == 0 && lddy * es % 16 == 0 &&
          a.lddx * es % 16 == 0;
  if (dtype == IM_DTYPE_BF16) norm_launch<bf16_t>(a, true, st);
  else norm_launch<float>(a, true, st);
  if (need) hipLaunchKernelGGL(norm_reduce_kernel, dim3((2 * d + 31) / 32), dim3(1024), 0, st, a.partial, grid, d, dgamma, dbeta);
  return after_launch(what);
}

}  // extern "C"
