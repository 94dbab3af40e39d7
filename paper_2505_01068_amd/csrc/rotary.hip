// Rotary positions with several axes, forward and backward (include/imattn.h).
//
// Bound by HBM: every element is read and written once.  A workgroup takes a few rows; its threads first form the cosine and
// sine of every (row, pair) once, in LDS, and then turn the pairs of all heads of queries and keys with them, 16 bytes at a
// time where the layout allows.  The angle is pos * inv_freq / (2 pi) in fp64 -- the product of two fp32 numbers
// is exact there -- of which only the fraction of a turn is kept, so that positions in the millions keep the accuracy of small ones.
// 8 x 4608 rows of 8 + 8 heads of 64 in bf16: 27 us for 151 MB that were just touched, 39 us when they come from HBM (a copy: 32); 16 rows: 4.9 us.
#include <algorithm>

#include "entry.hpp"
#include "mfma_common.hpp"

namespace imattn {

constexpr int ROT_THREADS = 256;

struct RotArgs {
  long rows_total;                 // batch * rows
  int rows, n_axes, end[IM_MAX_AXES];   // end[a]: pairs of axes 0..a
  int P, dh, qh, kh, inverse, rows_per_wg;
  int units_turn, units;           // units of a head: turned ones, then copied ones
  const float *pos, *inv_freq;
  long pos_batch;
  im_view_t q, qo, k, ko;
};

template <class T, int E>
struct Pack { float v[E]; };
template <class T, int E>
__device__ __forceinline__ Pack<T, E> rot_load(const T* p) {
  Pack<T, E> r;
  if constexpr (E == 1) r.v[0] = ldf(p);
  else {
    const u32x4 u = *(const u32x4*)p;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 4) r.v[e] = __uint_as_float(u[e]);
      else { r.v[2 * e] = __uint_as_float(u[e] << 16); r.v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u); }
    }
  }
  return r;
}
template <class T, int E>
__device__ __forceinline__ void rot_store(T* p, const Pack<T, E>& r) {
  if constexpr (E == 1) stf(p, r.v[0]);
  else {
    u32x4 u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 4) u[e] = __float_as_uint(r.v[e]);
      else u[e] = pack_bf16(r.v[2 * e], r.v[2 * e + 1]);
    }
    *(u32x4*)p = u;
  }
}

// fused operations written out: every layout's kernel gives the same bits
__device__ __forceinline__ void rot_turn(float x0, float x1, float2 w, float& y0, float& y1) {
  y0 = __builtin_fmaf(x0, w.x, -(x1 * w.y));
  y1 = __builtin_fmaf(x0, w.y, x1 * w.x);
}

// E elements a unit (1: any layout).  A turned unit is E pairs: two runs of E elements half the turned part apart, or
// (IL, neighbouring elements as pairs) one run of E elements, one pair for E = 1.
template <class T, int E, bool IL>
__global__ __launch_bounds__(ROT_THREADS) void rotary_kernel(RotArgs a) {
  extern __shared__ float2 turn[];   // [rows_per_wg][P]
  touch_args<RotArgs>();
  for (long row0 = (long)blockIdx.x * a.rows_per_wg; row0 < a.rows_total; row0 += (long)gridDim.x * a.rows_per_wg) {
    const int nrows = (int)(a.rows_total - row0 < a.rows_per_wg ? a.rows_total - row0 : a.rows_per_wg);
    const unsigned b0 = (unsigned)row0 / (unsigned)a.rows, t0 = (unsigned)row0 - b0 * (unsigned)a.rows;
    for (int i = threadIdx.x; i < nrows * a.P; i += ROT_THREADS) {
      unsigned r, p;
      udivmod((unsigned)i, (unsigned)a.P, r, p);
      unsigned b, t;
      udivmod(t0 + r, (unsigned)a.rows, b, t);
      b += b0;
      int axis = 0;
#pragma unroll
      for (int x = 0; x < IM_MAX_AXES - 1; ++x) axis += x + 1 < a.n_axes && (int)p >= a.end[x];
      constexpr double per_turn = 0.15915494309189533577;   // 1 / (2 pi)
      const double angle = (double)a.pos[b * a.pos_batch + (long)t * a.n_axes + axis] * (double)a.inv_freq[p];
      const double part = __builtin_fma(angle, per_turn, -rint(angle * per_turn));   // of a turn, -1/2 .. 1/2
      float s, c;
      sincospif((float)(2.0 * part), &s, &c);
      turn[i] = make_float2(c, a.inverse ? -s : s);
    }
    __syncthreads();
    const unsigned per_row = (unsigned)((a.qh + a.kh) * a.units);
    for (unsigned i = threadIdx.x; i < nrows * per_row; i += ROT_THREADS) {
      unsigned r, rest, h, u;
      udivmod(i, per_row, r, rest);
      udivmod(rest, (unsigned)a.units, h, u);
      unsigned b, t;
      udivmod(t0 + r, (unsigned)a.rows, b, t);
      b += b0;
      const bool is_q = (int)h < a.qh;
      const im_view_t& vi = is_q ? a.q : a.k;
      const im_view_t& vo = is_q ? a.qo : a.ko;
      const int head = is_q ? (int)h : (int)h - a.qh;
      const T* src = (const T*)vi.ptr + b * vi.batch + t * vi.row + head * vi.head;
      T* dst = (T*)vo.ptr + b * vo.batch + t * vo.row + head * vo.head;
      const float2* cs = turn + r * a.P;
      if ((int)u >= a.units_turn) {
        const int at = 2 * a.P + ((int)u - a.units_turn) * E;
        rot_store<T, E>(dst + at, rot_load<T, E>(src + at));
      } else if constexpr (IL && E > 1) {
        const int at = (int)u * E;
        Pack<T, E> x = rot_load<T, E>(src + at), y;
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const float2 w = cs[(at + e) / 2];
          rot_turn(x.v[e], x.v[e + 1], w, y.v[e], y.v[e + 1]);
        }
        rot_store<T, E>(dst + at, y);
      } else {
        const int p = (int)u * E, i0 = IL ? 2 * p : p, i1 = IL ? 2 * p + 1 : a.P + p;
        Pack<T, E> x0 = rot_load<T, E>(src + i0), x1 = rot_load<T, E>(src + i1), y0, y1;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float2 w = cs[p + e];
          rot_turn(x0.v[e], x1.v[e], w, y0.v[e], y1.v[e]);
        }
        rot_store<T, E>(dst + i0, y0);
        rot_store<T, E>(dst + i1, y1);
      }
    }
    __syncthreads();   // the turns are overwritten
  }
}

template <class T>
static void rot_launch(RotArgs a, bool il, bool in16, hipStream_t st) {
  constexpr int V = 16 / (int)sizeof(T);
  const bool vec = in16 && (il ? 2 * a.P % V == 0 : a.P % V == 0);
  const int E = vec ? V : 1;
  a.units_turn = vec && il ? 2 * a.P / V : a.P / E;
  a.units = a.units_turn + (a.dh - 2 * a.P) / E;
  // about four units a thread, as many rows as that takes; their turns fit 32 KB
  const int per_row = (a.qh + a.kh) * a.units;
  a.rows_per_wg = std::max(1, std::min(4 * ROT_THREADS / per_row, 4096 / a.P));
  const dim3 grid((unsigned)std::min<long>((a.rows_total + a.rows_per_wg - 1) / a.rows_per_wg, 1l << 22));
  const size_t lds = (size_t)a.rows_per_wg * a.P * sizeof(float2);
  if (vec) {
    if (il) hipLaunchKernelGGL((rotary_kernel<T, V, true>), grid, dim3(ROT_THREADS), lds, st, a);
    else hipLaunchKernelGGL((rotary_kernel<T, V, false>), grid, dim3(ROT_THREADS), lds, st, a);
  } else {
    if (il) hipLaunchKernelGGL((rotary_kernel<T, 1, true>), grid, dim3(ROT_THREADS), lds, st, a);
    else hipLaunchKernelGGL((rotary_kernel<T, 1, false>), grid, dim3(ROT_THREADS), lds, st, a);
  }
}

}  // namespace imattn

using namespace imattn;

extern "C" int im_rotary_apply(const im_rotary_t* s, const float* pos, int64_t pos_batch, const float* inv_freq, const im_view_t* q,
                               const im_view_t* q_out, const im_view_t* k, const im_view_t* k_out, void* hip_stream) {
  const char* what = "im_rotary_apply";
  if (!s) return refuse(IM_ERR_INVALID, "%s: shape is NULL", what);
  if (s->dtype != IM_DTYPE_F32 && s->dtype != IM_DTYPE_BF16) return refuse(IM_ERR_INVALID, "%s: dtype must be IM_DTYPE_F32 or IM_DTYPE_BF16 (got %d)", what, s->dtype);
  if (s->batch < 0 || s->rows < 0) return refuse(IM_ERR_INVALID, "%s: batch and rows must be >= 0", what);
  if (s->n_axes < 1 || s->n_axes > IM_MAX_AXES) return refuse(IM_ERR_INVALID, "%s: n_axes must be in 1..%d (got %d)", what, IM_MAX_AXES, s->n_axes);
  if (s->head_dim < 2 || s->head_dim > 1024) return refuse(IM_ERR_INVALID, "%s: head_dim must be in 2..1024 (got %d)", what, s->head_dim);
  if (s->q_heads < 1 || s->k_heads < 0 || s->q_heads > 65536 || s->k_heads > 65536) return refuse(IM_ERR_INVALID, "%s: q_heads must be in 1..65536, k_heads in 0..65536", what);
  RotArgs a = {};
  long P = 0;
  for (int x = 0; x < s->n_axes; ++x) {
    if (s->pairs[x] < 0 || s->pairs[x] > s->head_dim) return refuse(IM_ERR_INVALID, "%s: pairs[%d] must be in 0..head_dim / 2", what, x);
    P += s->pairs[x];
    a.end[x] = (int)P;
  }
  if (P < 1 || 2 * P > s->head_dim) return refuse(IM_ERR_INVALID, "%s: the axes' pairs must be 1..head_dim / 2 together (got %ld)", what, P);
  const size_t es = s->dtype == IM_DTYPE_BF16 ? 2 : 4;
  const int64_t nq[3] = {s->batch, s->rows, s->q_heads}, nk[3] = {s->batch, s->rows, s->k_heads};
  if (int rc = check_view(what, "q", q, nq, es, false)) return rc;
  if (int rc = check_view(what, "q_out", q_out, nq, es, true)) return rc;
  if (int rc = check_in_place(what, "q", *q, *q_out, nq)) return rc;
  if (s->k_heads) {
    if (int rc = check_view(what, "k", k, nk, es, false)) return rc;
    if (int rc = check_view(what, "k_out", k_out, nk, es, true)) return rc;
    if (int rc = check_in_place(what, "k", *k, *k_out, nk)) return rc;
  }
  a.rows_total = (long)s->batch * s->rows;
  if (a.rows_total == 0) return IM_OK;
  if (a.rows_total >= (1l << 31)) return refuse(IM_ERR_INVALID, "%s: batch * rows must be < 2^31", what);
  if (!pos || !inv_freq || ((uintptr_t)pos | (uintptr_t)inv_freq) % 4) return refuse(IM_ERR_INVALID, "%s: pos and inv_freq must be aligned device pointers", what);
  if (pos_batch < 0 || pos_batch > (1ll << 40)) return refuse(IM_ERR_INVALID, "%s: pos_batch must be in 0..2^40", what);
  a.rows = s->rows; a.n_axes = s->n_axes; a.P = (int)P; a.dh = s->head_dim; a.qh = s->q_heads; a.kh = s->k_heads; a.inverse = s->inverse != 0;
  a.pos = pos; a.pos_batch = pos_batch; a.inv_freq = inv_freq;
  a.q = *q; a.qo = *q_out;
  bool in16 = view_in_units(a.q, a.dh, es, 16) && view_in_units(a.qo, a.dh, es, 16);
  if (s->k_heads) {
    a.k = *k; a.ko = *k_out;
    in16 = in16 && view_in_units(a.k, a.dh, es, 16) && view_in_units(a.ko, a.dh, es, 16);
  }
  if (s->k_heads) {   // (each may be its own input, not the other's)
    if (q_out->ptr == k->ptr) return refuse(IM_ERR_INVALID, "%s: q_out overlaps k", what);
    if (k_out->ptr == q->ptr) return refuse(IM_ERR_INVALID, "%s: k_out overlaps q", what);
    if (q_out->ptr == k_out->ptr) return refuse(IM_ERR_INVALID, "%s: k_out overlaps q_out", what);
  }
  hipStream_t st = (hipStream_t)hip_stream;
  ProfScope ps(PF_MISC, st);
  if (s->dtype == IM_DTYPE_BF16) rot_launch<bf16_t>(a, s->interleaved, in16, st);
  else rot_launch<float>(a, s->interleaved, in16, st);
  return after_launch(what);
}
