// Layer normalisation of rows, forward and backward, as entry points of their own (include/imattn.h).
//
// Bound by HBM: the forward reads and writes a row once, the backward reads x and dy and writes dx once.  A row lives in the
// registers of LPR lanes (4 .. 64 of a wave, or a whole workgroup of 256 / 1024), NC chunks of 16 bytes each, so that mean,
// centred squares and the two sums of the gradient are taken over registers: two passes for the variance cost no traffic.
// The gradients of gain and bias: every thread keeps the sums of its own columns over the rows that it meets, the
// workgroup adds its threads' in a fixed order and writes one partial row; a second launch adds the partial rows.
#include <algorithm>

#include "entry.hpp"
#include "mfma_common.hpp"

namespace imattn {

template <class T> struct NormChunk { static constexpr int E = 16 / (int)sizeof(T); };

// E elements from p, of which the first n (<= E) exist; `whole`: p is 16-byte aligned and all exist
__device__ __forceinline__ void load_chunk(const float* p, int n, bool whole, float (&v)[4]) {
  if (whole) {
    const float4 u = *(const float4*)p;
    v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = e < n ? p[e] : 0.f;
}
__device__ __forceinline__ void load_chunk(const bf16_t* p, int n, bool whole, float (&v)[8]) {
  if (whole) {
    const u32x4 u = *(const u32x4*)p;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(u[e] << 16);
      v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e < n ? bf2f(p[e]) : 0.f;
}
__device__ __forceinline__ void store_chunk(float* p, int n, bool whole, const float (&v)[4]) {
  if (whole) { *(float4*)p = make_float4(v[0], v[1], v[2], v[3]); return; }
#pragma unroll
  for (int e = 0; e < 4; ++e) if (e < n) p[e] = v[e];
}
__device__ __forceinline__ void store_chunk(bf16_t* p, int n, bool whole, const float (&v)[8]) {
  if (whole) {
    u32x4 u;
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
    *(u32x4*)p = u;
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) if (e < n) p[e] = f2bf(v[e]);
}

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

template <class T, int LPR, int NC>
__global__ __launch_bounds__(LPR > 256 ? LPR : 256) void norm_fwd_kernel(NormArgs a) {
  constexpr int E = NormChunk<T>::E, WG = LPR > 256 ? LPR : 256, RPW = WG / LPR;
  __shared__ float red[2][2][WG / 64];
  const int lane = threadIdx.x % LPR;
  int turn = 0;   // the reduction buffers alternate, so that one barrier a sum suffices
  for (long row0 = (long)blockIdx.x * RPW; row0 < a.rows; row0 += (long)gridDim.x * RPW, turn ^= 1) {
    const long row = row0 + threadIdx.x / LPR;
    const bool mine = row < a.rows;
    const T* x = (const T*)a.x + (mine ? row : 0) * a.ldx;
    float v[NC][E];
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int at = (lane + c * LPR) * E, n = a.d - at;
#pragma unroll
      for (int e = 0; e < E; ++e) v[c][e] = 0.f;
      if (n > 0) load_chunk(x + at, n, a.vec, v[c]);
#pragma unroll
      for (int e = 0; e < E; ++e) s += v[c][e];
    }
    const float mean = row_sum<LPR>(s, red[turn][0]) * a.inv_d;
    s = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int n = a.d - (lane + c * LPR) * E;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v[c][e] -= mean;
        if (e < n) s += v[c][e] * v[c][e];
      }
    }
    const float rstd = 1.0f / sqrtf(row_sum<LPR>(s, red[turn][1]) * a.inv_d + a.eps);
    if (!mine) continue;
    if (a.mean && lane == 0) { a.mean[row] = mean; a.rstd[row] = rstd; }
    T* y = (T*)a.y + row * a.ldy;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int at = (lane + c * LPR) * E, n = a.d - at;
      if (n <= 0) continue;
      float g[E], b[E], o[E];
      if (a.gamma) load_chunk((const T*)a.gamma + at, n, a.vec, g);
      if (a.beta) load_chunk((const T*)a.beta + at, n, a.vec, b);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        o[e] = v[c][e] * rstd;
        if (a.gamma) o[e] *= g[e];
        if (a.beta) o[e] += b[e];
      }
      store_chunk(y + at, n, a.vec, o);
    }
  }
}

template <class T, int LPR, int NC>
__global__ __launch_bounds__(LPR > 256 ? LPR : 256) void norm_bwd_kernel(NormArgs a) {
  constexpr int E = NormChunk<T>::E, WG = LPR > 256 ? LPR : 256, RPW = WG / LPR;
  constexpr int COLS = LPR * NC * E;
  __shared__ float red[2][2][WG / 64];
  __shared__ float cols[LPR > 64 ? 1 : 2 * COLS];   // the workgroup's sums, where several waves share columns
  const int lane = threadIdx.x % LPR;
  float g[NC][E], dg[NC][E], db[NC][E];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int at = (lane + c * LPR) * E, n = a.d - at;
#pragma unroll
    for (int e = 0; e < E; ++e) { g[c][e] = 1.f; dg[c][e] = db[c][e] = 0.f; }
    if (a.gamma && n > 0) load_chunk((const T*)a.gamma + at, n, a.vec, g[c]);
  }
  int turn = 0;   // the reduction buffers alternate, so that one barrier a sum suffices
  for (long row0 = (long)blockIdx.x * RPW; row0 < a.rows; row0 += (long)gridDim.x * RPW, turn ^= 1) {
    const long row = row0 + threadIdx.x / LPR;
    const bool mine = row < a.rows;
    float xh[NC][E], w[NC][E];
    float s1 = 0.f, s2 = 0.f, mean = 0.f, rstd = 0.f;
    if (mine) { mean = a.mean[row]; rstd = a.rstd[row]; }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int at = (lane + c * LPR) * E, n = mine ? a.d - at : 0;
#pragma unroll
      for (int e = 0; e < E; ++e) xh[c][e] = w[c][e] = 0.f;
      if (n > 0) {
        load_chunk((const T*)a.x + row * a.ldx + at, n, a.vec, xh[c]);
        load_chunk((const T*)a.dy + row * a.lddy + at, n, a.vec, w[c]);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        xh[c][e] = e < n ? (xh[c][e] - mean) * rstd : 0.f;
        dg[c][e] += w[c][e] * xh[c][e];
        db[c][e] += w[c][e];
        w[c][e] *= g[c][e];
        s1 += w[c][e];
        s2 += w[c][e] * xh[c][e];
      }
    }
    if (!a.dx) continue;
    s1 = row_sum<LPR>(s1, red[turn][0]) * a.inv_d;
    s2 = row_sum<LPR>(s2, red[turn][1]) * a.inv_d;
    if (!mine) continue;
    T* dx = (T*)a.dx + row * a.lddx;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int at = (lane + c * LPR) * E, n = a.d - at;
      if (n <= 0) continue;
      float o[E];
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = rstd * (w[c][e] - s1 - xh[c][e] * s2);
      store_chunk(dx + at, n, a.vec, o);
    }
  }
  if (!a.partial && !a.dgamma && !a.dbeta) return;
  float* out_g = a.partial ? a.partial + (long)blockIdx.x * 2 * a.d : a.dgamma;
  float* out_b = a.partial ? out_g + a.d : a.dbeta;
  if constexpr (LPR > 64) {   // every thread has columns of its own
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int at = (lane + c * LPR) * E + e;
        if (at < a.d && out_g) out_g[at] = dg[c][e];
        if (at < a.d && out_b) out_b[at] = db[c][e];
      }
  } else {
    for (int wv = 0; wv < WG / 64; ++wv) {
      if ((int)(threadIdx.x >> 6) == wv) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < E; ++e) {
            float p = dg[c][e], q = db[c][e];
#pragma unroll
            for (int o = 32; o >= LPR; o >>= 1) { p += __shfl_xor(p, o); q += __shfl_xor(q, o); }
            const int at = (lane + c * LPR) * E + e;
            if ((int)(threadIdx.x & 63) < LPR) {
              cols[at] = wv ? cols[at] + p : p;
              cols[COLS + at] = wv ? cols[COLS + at] + q : q;
            }
          }
      }
      __syncthreads();
    }
    for (int at = threadIdx.x; at < a.d; at += WG) {
      if (out_g) out_g[at] = cols[at];
      if (out_b) out_b[at] = cols[COLS + at];
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

template <class T>
static void norm_launch(const NormArgs& a, bool bwd, hipStream_t st) {
  constexpr int E = NormChunk<T>::E;
  const int lpr = norm_lanes(a.d, E), chunks = (a.d + E - 1) / E, nc = (chunks + lpr - 1) / lpr;
  const dim3 block(lpr > 256 ? lpr : 256), grid(bwd ? (unsigned)norm_bwd_grid(a.rows, a.d, E) : (unsigned)std::min<long>(norm_row_blocks(a.rows, a.d, E), 1l << 21));
#define NORM_GO(L, N)                                                                         \
  do {                                                                                        \
    if (bwd) hipLaunchKernelGGL((norm_bwd_kernel<T, L, N>), grid, block, 0, st, a);           \
    else hipLaunchKernelGGL((norm_fwd_kernel<T, L, N>), grid, block, 0, st, a);               \
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
    default: NORM_NC(1024); break;
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
  if (!(eps > 0.f) || eps > 3e38f) return refuse(IM_ERR_INVALID, "%s: eps must be finite and > 0", what);
  if (!mean != !rstd) return refuse(IM_ERR_INVALID, "%s: mean and rstd: both or neither", what);
  if (((uintptr_t)gamma | (uintptr_t)beta) % es) return refuse(IM_ERR_INVALID, "%s: gamma or beta is not aligned to its elements", what);
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
  if (rows > 0 && (!mean || !rstd)) return refuse(IM_ERR_INVALID, "%s: mean and rstd of the forward are needed", what);
  if ((uintptr_t)gamma % es) return refuse(IM_ERR_INVALID, "%s: gamma is not aligned to its elements", what);
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
