// Kernels of the attention core (include/imattn.h: im_core_attention_*), bf16 and fp32.
//
// One scheme serves the forward, dQ and dK/dV.  A workgroup OWNS rows -- query rows in the forward and for dQ, key rows for
// dK/dV -- as the COLUMNS of 32 x 32 products, one per lane pair (l, l + 32), and STREAMS tiles of the other side through LDS:
//     forward   S^T = K Q^T,                    O^T += V^T P^T
//     dQ        S^T = K Q^T,  dP^T = V dO^T,    dQ^T += K^T dS^T
//     dK/dV     S   = Q K^T,  dP   = dO V^T,    dV^T += dO^T P,  dK^T += Q^T dS
// A lane holds 16 scores of ONE owned row and, by the order perm32 in which the streamed rows are fed, they are two runs of 8
// consecutive streamed rows: what the next product takes as its second operand, so probabilities never leave the
// registers.  Row statistics need one exchange between the two halves of the wave.  The streamed tile is read by rows for the
// first product(s) and transposed for the second: by the LDS transpose read in bf16, by plain reads in fp32, whose
// products run on v_mfma_f32_32x32x2_f32 (exact fp32 multiply-adds; a sixteenth of the bf16 rate).
//
// What bounds them: not the matrix cores but the score arithmetic.  8 x 4608 steps, 8 heads of 64, the diagonal blocks live, scores capped: 590 thousand
// cycles in the forward, 258 us, or 310 where the clock falls under sustained load; the vector units issue in 77 % of the cycles in which a CU has work --
// 11 instructions a score, the softmax's exponential and its share of the cap's polynomial among them -- the matrix units are busy in 25 %.  Training with
// cap and bias: vector 81 / 90 / 63 %, matrix 22 / 23 / 24 % in forward, dQ and dK/dV.  In fp32 at a head of 5 no unit is: vector 50 / 44 / 38 %, matrix
// 27 / 27 / 36 %, segments of 50 rows leave 61 % of a 128-row tile empty; from head dimension 64 on the fp32 matrix rate bounds.  With documents
// the waves wait for copies and each other in 57 / 62 / 64 % of their cycles.  For single tokens against long caches HBM (26 us for 107 MB);
// for the smallest calls (9 us) the chain of loads and the instructions that are met for the first time.
//
// Which streamed tiles are visited is decided from the data, once per workgroup and 64 tiles: a tile in which no owned row
// sees any streamed row is skipped, one in which every owned row sees every streamed row takes the path without
// comparisons.  Both sides carry one number for the order in time: streamed row visible <=> its k_pos <= the owned q_pos
// (or the other way round for dK/dV), with k_pos = -inf for free keys (no causality, prefix), NaN for padding.
//
// Values that are not finite: a masked pair has weight 0, but 0 * inf would still reach the accumulators.  So in a tile with
// masked pairs such values are replaced by 0 when the tile is written to LDS, and the row's pairs that ARE
// visible get a score of NaN.  Tiles without masked pairs need no check.
#pragma once
#include <type_traits>

#include "core_attn.hpp"
#include "mfma_common.hpp"

namespace imattn {

constexpr int CORE_WAVES = 4;
constexpr int CORE_LIST = 64;    // streamed tiles classified at a time
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

typedef float f32x4 __attribute__((ext_vector_type(4)));
struct F8 { float v[8]; };
template <class T> struct CoreT;
template <> struct CoreT<bf16_t> { using Frag = bf16x8; static constexpr int EPC = 8; };
template <> struct CoreT<float> { using Frag = F8; static constexpr int EPC = 4; };

__device__ __forceinline__ f32x16 mfma_f32(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}
// the other half's value of the same column
__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }

// ---- LDS tiles: ROWS rows of ND * 32 elements ----
// bf16: panels of 64 columns, 8 units of 16 bytes a row, swizzled by sw_f.  fp32: rows of 32 ND floats, unit c of row r at c ^ (r % 8).
template <class T, int ND, int ROWS>
struct Tile {
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int SLOTS = BF ? (ND + 1) / 2 * ROWS * 8 : ROWS * ND * 8;   // 16-byte units
  static constexpr int BYTES = SLOTS * 16;
  static constexpr int ROW = BF ? 128 : ND * 128;                              // bytes from row to row
  // row and unit (of the row's data) that slot i of the tile holds
  static __device__ __forceinline__ int row_of(int i) { return BF ? (i >> 3) % ROWS : i / (ND * 8); }
  static __device__ __forceinline__ int unit_of(int i) {
    if constexpr (BF) return ((i & 7) ^ sw_f(row_of(i))) + 8 * (i / (ROWS * 8));
    else return (i % (ND * 8)) ^ (row_of(i) & 7);
  }
};

__device__ __forceinline__ unsigned lds_at(const void* p) { return (unsigned)(uintptr_t)p; }
template <class V>
__device__ __forceinline__ V lds_load(unsigned at, int off) {
  typedef char __attribute__((address_space(3))) * lds_char_ptr;
  typedef V __attribute__((address_space(3))) * lds_v_ptr;
  return *(lds_v_ptr)((lds_char_ptr)at + off);
}

// Where a lane reads its operands, as byte offsets into a tile.
//   by rows: streamed row (in the order perm32) lane % 32 of a 32-row block.  bf16: elements 16 s + 8 h .. + 7 of step s.  fp32: 16 s +
//   4 h .. + 3 and 16 s + 8 + 4 h .. + 3, so that a head of up to 8 elements takes half a step.
//   by columns: column (in the order perm32) lane % 32 of a 32-column block, streamed rows 8 h .. + 7 of a 16-row block.
template <class T, int ND, int ROWS>
struct LaneAt;
template <int ND, int ROWS>
struct LaneAt<bf16_t, ND, ROWS> {
  using TL = Tile<bf16_t, ND, ROWS>;
  unsigned row[ND == 1 ? 2 : 4], col[ND == 1 ? 1 : 2][2];
  __device__ __forceinline__ LaneAt(int lane) {
    const int r = perm32(lane & 31), h = lane >> 5;
#pragma unroll
    for (int j = 0; j < (ND == 1 ? 2 : 4); ++j) row[j] = r * 128 + (((2 * j + h) ^ sw_f(r)) << 4);
    const int j = lane & 15, g = lane >> 4, lrow = 8 * (g >> 1) + (j >> 2), chunk = 2 * (g & 1) + (j & 1), f = sw_f(lrow);
#pragma unroll
    for (int m = 0; m < (ND == 1 ? 1 : 2); ++m) {   // the transpose read's lanes, blocks of four columns exchanged as lds_frag_tr_sw_perm does
      col[m][0] = lrow * 128 + (((4 * m | chunk) ^ f) << 4) + 8 * ((j >> 1) & 1);
      col[m][1] = (lrow + 4) * 128 + (((4 * m | chunk) ^ f ^ 1) << 4) + 8 * ((j >> 1) & 1);
    }
  }
  __device__ __forceinline__ f32x16 rows(unsigned tile, int row32, int s, bf16x8 own, f32x16 c, int) const {
    return mfma32(lds_load<bf16x8>(tile + row[s & 3], (s >> 2) * ROWS * 128 + row32 * 128), own, c);
  }
  __device__ __forceinline__ f32x16 cols(unsigned tile, int row16, int db, bf16x8 p, f32x16 c) const {
    return mfma32(lds_frag_tr_at(tile + col[db & 1][0], tile + col[db & 1][1], (db >> 1) * ROWS * 128 + row16 * 128), p, c);
  }
};
// a and b with the odd rows of 16 lanes of a and the even ones of b exchanged
__device__ __forceinline__ u32x2 swap16(float a, float b) {
  const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return u32x2{s[0], s[1]};
}
template <int ND, int ROWS>
struct LaneAt<float, ND, ROWS> {
  unsigned row[4], col[8], col16[4];
  __device__ __forceinline__ LaneAt(int lane) {
    const int r = perm32(lane & 31), h = lane >> 5;
#pragma unroll
    for (int i = 0; i < 4; ++i) row[i] = r * ND * 128 + (((2 * i + h) ^ (r & 7)) << 4);
#pragma unroll
    for (int j = 0; j < 8; ++j) col[j] = (8 * h + j) * ND * 128 + (((r >> 2) ^ j) << 4) + 4 * (r & 3);
    const int g = (lane >> 4) & 1, c = lane & 15;
#pragma unroll
    for (int j = 0; j < 4; ++j) col16[j] = (8 * h + 2 * j + g) * ND * 128 + (((c >> 2) ^ (2 * j + g)) << 4) + 4 * (c & 3);
  }
  // Heads of up to 16 elements: the second product on 16 x 16 x 4, half of whose time 16 of 32 columns would waste on 32 x 32 x 2.  c[x]: columns
  // 16 x .. + 15 of the owned rows.  Exchanging rows of 16 lanes between the probabilities of two streamed rows gives each of the two products
  // four streamed rows: lanes 16 g .. + 15 hold row 8 (g / 2) + e + g % 2 of the 16-row block.
  __device__ __forceinline__ void cols16(unsigned tile, int row16, const F8& p, f32x4 (&c)[2]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float v = lds_load<float>(tile + col16[j], row16 * ND * 128);
      const u32x2 s = swap16(p.v[2 * j], p.v[2 * j + 1]);
      c[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, __uint_as_float(s[0]), c[0], 0, 0, 0);
      c[1] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, __uint_as_float(s[1]), c[1], 0, 0, 0);
    }
  }
  __device__ __forceinline__ f32x16 rows(unsigned tile, int row32, int s, const F8& own, f32x16 c, int left) const {   // left: elements from this step on
    const int off = (s >> 1) * 128 + row32 * ND * 128;
    const f32x4 u = lds_load<f32x4>(tile + row[2 * (s & 1)], off);
    c = mfma_f32(u[0], own.v[0], c);
    c = mfma_f32(u[1], own.v[1], c);
    c = mfma_f32(u[2], own.v[2], c);
    c = mfma_f32(u[3], own.v[3], c);
    if (left > 8) {
      const f32x4 w = lds_load<f32x4>(tile + row[2 * (s & 1) + 1], off);
      c = mfma_f32(w[0], own.v[4], c);
      c = mfma_f32(w[1], own.v[5], c);
      c = mfma_f32(w[2], own.v[6], c);
      c = mfma_f32(w[3], own.v[7], c);
    }
    return c;
  }
  __device__ __forceinline__ f32x16 cols(unsigned tile, int row16, int db, const F8& p, f32x16 c) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = mfma_f32(lds_load<float>(tile + col[j], db * 128 + row16 * ND * 128), p.v[j], c);
    return c;
  }
};
// The one rounding of probabilities and dS: the second products then run at the bf16 rate.  Errors against 64 bits become 1.4 times those of a result's own
// rounding in dq, dk and dv (0.0024 for 0.0017) and 1.1 times in o (0.0018); a second bf16 part of each would double the second products and their packing.
__device__ __forceinline__ bf16x8 pack_p(const bf16_t*, const float* p) { return pack8(p); }
__device__ __forceinline__ F8 pack_p(const float*, const float* p) {
  F8 f;
#pragma unroll
  for (int j = 0; j < 8; ++j) f.v[j] = p[j];
  return f;
}

// ---- global memory ----
// The asynchronous copies of mfma_common.hpp with five wait states in front: these kernels have more uniform values than scalar registers,
// and a base that v_readlane has just brought back must not be read by a memory instruction earlier (the compiler does not look into
// the statement).
#define CORE_COPY(NAME, INSTRUCTION)                                                                              \
  __device__ __forceinline__ void NAME(const void* gbase, unsigned byte_off, const void* lds_wave_base) {         \
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\t" INSTRUCTION " %1, %2"                                         \
                 :: "s"(lds_offset(lds_wave_base)), "v"(byte_off), "s"(gbase) : "memory");                        \
  }
CORE_COPY(copy16, "global_load_lds_dwordx4")
CORE_COPY(copy4, "global_load_lds_dword")
CORE_COPY(copy1, "global_load_lds_ubyte")
#undef CORE_COPY

// 16 bytes from element `at` of a head of dh elements; units at or behind its end give 0
template <class T>
__device__ __forceinline__ u32x4 load_unit(const T* head, int at, int dh, bool vec) {
  u32x4 u = {0u, 0u, 0u, 0u};
  if (at >= dh) return u;
  if (vec) return *(const u32x4*)(head + at);
  constexpr int E = 16 / (int)sizeof(T);
  T v[E];
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = head[min(at + e, dh - 1)];   // no branches: all loads are in flight together
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const bool is = at + e < dh;
    if constexpr (sizeof(T) == 2) u[e >> 1] |= (is ? (unsigned)v[e] : 0u) << (16 * (e & 1));
    else u[e] = is ? __float_as_uint(v[e]) : 0u;
  }
  return u;
}
// An owned row as operand fragments
template <int ND>
__device__ __forceinline__ void own_frags(const bf16_t* head, bool ok, int dh, bool vec, int h, bf16x8 (&f)[2 * ND]) {
#pragma unroll
  for (int s = 0; s < 2 * ND; ++s) {
    u32x4 u = {0u, 0u, 0u, 0u};
    if (ok) u = load_unit(head, 16 * s + 8 * h, dh, vec);
    f[s] = as_bf16x8(u);
  }
}
template <int ND>
__device__ __forceinline__ void own_frags(const float* head, bool ok, int dh, bool vec, int h, F8 (&f)[2 * ND]) {
#pragma unroll
  for (int s = 0; s < 2 * ND; ++s)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      u32x4 u = {0u, 0u, 0u, 0u};
      if (ok) u = load_unit(head, 16 * s + 8 * i + 4 * h, dh, vec);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[s].v[4 * i + e] = __uint_as_float(u[e]);
    }
}
// the fragments times a power of two
template <int N>
__device__ __forceinline__ void scale_frags(bf16x8 (&f)[N], float by) {
#pragma unroll
  for (int s = 0; s < N; ++s) {
    const u32x4 w = __builtin_bit_cast(u32x4, f[s]);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16) * by;
    f[s] = pack8(v);
  }
}
template <int N>
__device__ __forceinline__ void scale_frags(F8 (&f)[N], float by) {
#pragma unroll
  for (int s = 0; s < N; ++s)
#pragma unroll
    for (int e = 0; e < 8; ++e) f[s].v[e] *= by;
}
// this half's part of the product of an owned row's fragments with a row of dh floats (16-byte aligned if dh % 4 == 0)
template <int ND>
__device__ __forceinline__ float dot_frags(const bf16x8 (&f)[2 * ND], const float* row, int dh, int h) {
  float sum = 0.f;
#pragma unroll
  for (int s = 0; s < 2 * ND; ++s) {
    const u32x4 v = __builtin_bit_cast(u32x4, f[s]);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x4 u = load_unit(row, 16 * s + 8 * h + 4 * i, dh, dh % 4 == 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const unsigned w = v[2 * i + (e >> 1)];
        sum += __uint_as_float(u[e]) * __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
      }
    }
  }
  return sum;
}
template <int ND>
__device__ __forceinline__ float dot_frags(const F8 (&f)[2 * ND], const float* row, int dh, int h) {
  float sum = 0.f;
#pragma unroll
  for (int s = 0; s < 2 * ND; ++s)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x4 u = load_unit(row, 16 * s + 8 * i + 4 * h, dh, dh % 4 == 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += __uint_as_float(u[e]) * f[s].v[4 * i + e];
    }
  return sum;
}
// 8 consecutive results of an owned row from element `at` on
__device__ __forceinline__ void store8(bf16_t* head, int at, int dh, bool vec, const float* v) {
  if (at >= dh) return;
  if (vec) { *(bf16x8*)(head + at) = pack8(v); return; }
#pragma unroll
  for (int e = 0; e < 8; ++e) if (at + e < dh) head[at + e] = f2bf(v[e]);
}
__device__ __forceinline__ void store8(float* head, int at, int dh, bool vec, const float* v) {
  if (vec) {
    if (at < dh) *(float4*)(head + at) = make_float4(v[0], v[1], v[2], v[3]);
    if (at + 4 < dh) *(float4*)(head + at + 4) = make_float4(v[4], v[5], v[6], v[7]);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) if (at + e < dh) head[at + e] = v[e];
}
template <class T, int ND>
__device__ __forceinline__ void store_row(T* head, int dh, bool vec, int h, const f32x16 (&acc)[ND], float f) {
#pragma unroll
  for (int db = 0; db < ND; ++db)
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = acc[db][8 * g + e] * f;
      store8(head, 32 * db + 16 * g + 8 * h, dh, vec, v);
    }
}
template <class T>
__device__ __forceinline__ T* head_of(const im_view_t& v, long b, long row, long head) {
  return (T*)v.ptr + b * v.batch + row * v.row + head * v.head;
}

// ---- scores ----
// The cap, c tanh(s / c).  For |s / c| < 0.4 tanh x is x (1 + u Q(u)), u = x^2, with Q of degree 2 fitted to the smallest relative
// error there (1.2e-7, two half steps of fp32); the raw product r = s / scale takes the place of x, its powers of scale / c are in the
// coefficients (the host sees to it that they are of fp32's range).  That is 6 multiply-adds, where (1 - e) / (1 + e), e = exp(-2 |x|), takes an exponential and a reciprocal, each four times as
// long.  Scores rarely come near half of their cap, so a wave looks at its largest one first (`large`) and
// takes the exponential only if it has to; a score gives the same bits either way.
__device__ __forceinline__ float tanh_small(const CoreArgs& a, float r) {   // tanh(c_in r) / c_in
  const float u = r * r;
  return r * __builtin_fmaf(u, __builtin_fmaf(u, __builtin_fmaf(u, a.tanh_q[2], a.tanh_q[1]), a.tanh_q[0]), 1.f);
}
template <int N>
__device__ __forceinline__ void tanh_of(const CoreArgs& a, float (&x)[N], bool large) {
  if (large) {
#pragma unroll
    for (int r = 0; r < N; ++r) {
      const float ax = fabsf(x[r]), e = fast_exp2(-2.f * LOG2E * a.c_in * ax);
      const float big = __builtin_copysignf((1.f - e) * __builtin_amdgcn_rcpf(1.f + e) * a.inv_c_in, x[r]);
      float small = tanh_small(a, x[r]);
      asm("" : "+v"(small));   // both are computed: a choice, no branch per score
      x[r] = ax >= a.small_to ? big : small;
      if ((r & 3) == 3) __builtin_amdgcn_sched_barrier(0);   // few at a time: registers are what limits the waves in flight
    }
  } else {
#pragma unroll
    for (int r = 0; r < N; ++r) x[r] = tanh_small(a, x[r]);
  }
}

// a b, but 0 where a is 0 whatever b is.  A masked pair has weight 0, but its other factors may be anything: products with the contents of a key that
// nobody sees, statistics and gradients of a query that sees nothing (sums of finite values may overflow too, which no look at the tile shows).
// One instruction, v_mul_legacy_f32; the compiler knows it as an intrinsic without a builtin.
extern "C" __device__ float intrinsic_mul_legacy(float, float) __asm("llvm.amdgcn.fmul.legacy");
__device__ __forceinline__ float mul0(float a, float b) { return intrinsic_mul_legacy(a, b); }

// ---- streamed side ----
enum { TILE_SKIP = 0, TILE_FULL = 1, TILE_PART = 2 };

// per streamed row in LDS
template <int ROWS>
struct __align__(16) RowMeta {
  float pos[ROWS];     // position
  int doc[ROWS];
  float order[ROWS];   // (first the key's padding byte;) k_pos (-inf: free, NaN: no key) when keys are streamed, q_pos (+inf: sees all, NaN: no row) when queries are
  int bad[ROWS];       // == number of the tile: holds a value that is not finite
  int any_bad;
};
template <int ROWS>
struct __align__(16) QueryMeta {     // dK/dV only
  float lse2[ROWS], delta[ROWS];
};

struct RowInfo { float order, pos; int doc; };
struct RowRaw { float pos; int doc; unsigned pad; };

__device__ __forceinline__ RowRaw key_raw(const CoreArgs& a, long b, int row, bool ok) {
  RowRaw r = {0.f, 0, 1u};
  if (ok) {
    const long at = b * a.Tk + row;
    r.pad = 0u;
    if (a.k_doc) r.doc = a.k_doc[at];
    if (a.k_pos) r.pos = a.k_pos[at];
    if (a.key_pad) r.pad = a.key_pad[at];
  }
  return r;
}
__device__ __forceinline__ RowInfo key_info(const CoreArgs& a, float prefix, const RowRaw& r) {
  const float order = a.causal && !(r.pos < prefix) ? r.pos : IM_NEG_INF;
  return {r.pad ? __builtin_nanf("") : order, r.pos, r.doc};
}
__device__ __forceinline__ RowRaw query_raw(const CoreArgs& a, long b, int row, bool ok) {
  RowRaw r = {0.f, 0, 1u};
  if (ok) {
    const long at = b * a.Tq + row;
    r.pad = 0u;
    if (a.q_doc) r.doc = a.q_doc[at];
    if (a.q_pos) r.pos = a.q_pos[at];
  }
  return r;
}
__device__ __forceinline__ RowInfo query_info(const CoreArgs& a, const RowRaw& r) {
  return {r.pad ? __builtin_nanf("") : a.causal ? r.pos : __builtin_inff(), r.pos, r.doc};
}

// Smallest and largest order and document of the rows with ok, over the lanes of a wave
struct Range { float lo, hi; int dlo, dhi; bool all, any; };
__device__ __forceinline__ void range_wave(Range& r) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    r.lo = fminf(r.lo, __shfl_xor(r.lo, o));
    r.hi = fmaxf(r.hi, __shfl_xor(r.hi, o));
    r.dlo = min(r.dlo, __shfl_xor(r.dlo, o));
    r.dhi = max(r.dhi, __shfl_xor(r.dhi, o));
  }
}
// rows in range but without a valid order (padding) clear `all`
__device__ __forceinline__ Range range_of(const RowInfo& i, bool in_range, bool numbers) {   // numbers: more than any and all is asked for
  const bool ok = in_range && i.order == i.order;
  Range r;
  r.lo = ok ? i.order : __builtin_inff();
  r.hi = ok ? i.order : IM_NEG_INF;
  r.dlo = ok ? i.doc : 0x7fffffff;
  r.dhi = ok ? i.doc : (int)0x80000000;
  r.any = __any(ok);
  r.all = __all(ok || !in_range);
  if (numbers) range_wave(r);
  return r;
}
__device__ __forceinline__ int tile_class(const Range& keys, const Range& queries, bool whole, bool numbers) {
  if (!keys.any || !queries.any) return TILE_SKIP;
  bool full = whole && keys.all && queries.all;
  if (numbers) {
    if (keys.lo > queries.hi || keys.dlo > queries.dhi || keys.dhi < queries.dlo) return TILE_SKIP;
    full = full && keys.hi <= queries.lo && keys.dlo == keys.dhi && queries.dlo == queries.dhi && keys.dlo == queries.dlo;
  }
  return full ? TILE_FULL : TILE_PART;
}

template <class T, int ND, bool FEW, CoreKernel WHICH> struct CoreCfg {
  // bf16 dK/dV of the widest heads: the owned rows of V are kept in LDS, not in 32 registers, and tiles are smaller, so that two waves a SIMD hide
  // each other's LDS reads (3 x 3124 steps of 4 heads of 128 with documents: 374 -> 320 us; without masks 361 -> 278 us)
  static constexpr bool OWN_LDS = sizeof(T) == 2 && ND == 4 && WHICH == CORE_DKV;
  static constexpr int ROWS = FEW || (ND == 4 && (sizeof(T) == 4 || OWN_LDS)) ? 32 : 64;   // streamed rows of a tile
  static constexpr int TEAM = FEW ? 64 : 64 * CORE_WAVES;           // threads that load a tile together
  static constexpr int OWN = FEW ? 32 : 32 * CORE_WAVES;            // owned rows of a workgroup
  // four teams' pairs of the widest fp32 tiles do not fit the LDS twice, those of two workgroups in bf16 neither
  static constexpr int BUFS = FEW && ND == 4 && (sizeof(T) == 4 || OWN_LDS) ? 1 : 2;
  static constexpr int N = Tile<T, ND, ROWS>::SLOTS / TEAM;         // 16-byte units a thread and tensor
};

// LDS of one team
template <class T, int ND, bool FEW, CoreKernel WHICH>
struct TeamLds {
  using C = CoreCfg<T, ND, FEW, WHICH>;
  char tile[C::BUFS][2][Tile<T, ND, C::ROWS>::BYTES];   // K, V or Q, dO
  RowMeta<C::ROWS> meta[C::BUFS];
  typename std::conditional<WHICH == CORE_DKV, QueryMeta<C::ROWS>, char>::type qmeta[C::BUFS];
};
template <class T, int ND, bool FEW, CoreKernel WHICH>
struct CoreLds {
  static constexpr int TEAMS = FEW ? CORE_WAVES : 1;
  __align__(16) TeamLds<T, ND, FEW, WHICH> team[TEAMS];
  int4 list[CORE_LIST];       // first row, rows, class | waves that skip it << 8 | waves that see all of it << 12, head of the group (dK/dV)
  Range own[CORE_WAVES];
  bf16x8 own2[CoreCfg<T, ND, FEW, WHICH>::OWN_LDS ? (FEW ? 1 : CORE_WAVES) * 2 * ND * 64 : 1];
};

// A value that the compiler takes for new here: what is made of it is made here, not kept in registers from before the loop.
__device__ __forceinline__ int late(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
template <bool FEW>
__device__ __forceinline__ void team_sync() {
  if constexpr (FEW) {   // one wave: its LDS instructions stay in order, only the compiler must not move them
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  } else __syncthreads();
}

// Exponents that are all ones (infinity, NaN) carry into the sign's place; the bits of other numbers that are added stay below it.
__device__ __forceinline__ unsigned odd_bits(bf16_t, unsigned u) { return (u & 0x7f807f80u) + 0x00800080u; }
__device__ __forceinline__ unsigned odd_bits(float, unsigned u) { return (u & 0x7f800000u) + 0x00800000u; }
__device__ __forceinline__ bool odd(bf16_t, unsigned bits) { return (bits & 0x80008000u) != 0; }
__device__ __forceinline__ bool odd(float, unsigned bits) { return (bits & 0x80000000u) != 0; }
__device__ __forceinline__ unsigned clean_bits(bf16_t, unsigned u) {
  if ((u & 0x7f80u) == 0x7f80u) u &= 0xffff0000u;
  if ((u & 0x7f800000u) == 0x7f800000u) u &= 0x0000ffffu;
  return u;
}
__device__ __forceinline__ unsigned clean_bits(float, unsigned u) { return (u & 0x7f800000u) == 0x7f800000u ? 0u : u; }

// Where a workgroup stands: batch element, key head, owned group, first owned row in it, the group's rows, split.
struct Place { int b, kvh, group, own0, own_n, split; };

template <bool OWN_KEYS, int OWN>
__device__ __forceinline__ Place place_of(const CoreArgs& a) {
  int bx, by, bz;
  xcd_block_index(bx, by, bz);   // 1-d grid
  const int tiles = a.tile_prefix[a.own_groups];
  unsigned rest, tile, bh, split, b, kvh;
  udivmod((unsigned)bx, (unsigned)tiles, rest, tile);
  udivmod(rest, (unsigned)a.splits, bh, split);
  udivmod(bh, (unsigned)a.Hkv, b, kvh);
  int k = 0;
  while (k + 1 < a.own_groups && (int)tile >= a.tile_prefix[k + 1]) ++k;
  Place p;
  p.b = __builtin_amdgcn_readfirstlane((int)b);
  p.kvh = __builtin_amdgcn_readfirstlane((int)kvh);
  p.split = __builtin_amdgcn_readfirstlane((int)split);
  k = __builtin_amdgcn_readfirstlane(k);
  p.group = k;
  p.own_n = OWN_KEYS ? a.own_len[k] : a.own_len[k] * a.G;
  // the last tile of a segment first: under causality it sees most
  p.own0 = (a.tile_prefix[k + 1] - 1 - __builtin_amdgcn_readfirstlane((int)tile)) * OWN;
  return p;
}

// ---- the kernel ----
// Waves a SIMD that the registers are cut for.  Up to head dimension 64 three in bf16 (168 registers each; 8 x 4608 steps, dQ 407 -> 356 us with three
// in place of two) but for dK/dV, whose accumulators are twice as many; two otherwise, and one for wide fp32 heads, where even 256 registers would spill.
template <class T, int ND, CoreKernel WHICH>
constexpr int core_waves() {
  if (ND == 4) return sizeof(T) == 4 ? 1 : 2;
  return WHICH == CORE_DKV || sizeof(T) == 4 ? 2 : 3;
}

// W: head width in units of 32 elements, 0 for fp32 heads of up to 16
template <class T, int W, bool FEW, bool CAP, bool BIAS, CoreKernel WHICH>
__global__ __launch_bounds__(64 * CORE_WAVES, (core_waves<T, (W ? W : 1), WHICH>())) void core_kernel(CoreArgs a) {
  constexpr int ND = W ? W : 1;
  constexpr bool NARROW = W == 0;
  static_assert(!NARROW || sizeof(T) == 4, "");
  using C = CoreCfg<T, ND, FEW, WHICH>;
  using Frag = typename CoreT<T>::Frag;
  using TL = Tile<T, ND, C::ROWS>;
  constexpr int ROWS = C::ROWS, EPC = CoreT<T>::EPC, BUFS = C::BUFS;
  constexpr bool OWN_KEYS = WHICH == CORE_DKV, BWD = WHICH != CORE_FWD;
  extern __shared__ __align__(16) char lds_raw[];   // (nothing but the list and the owned rows' ranges outlives the walk over the tiles)
  auto& lds = *(CoreLds<T, ND, FEW, WHICH>*)lds_raw;
  touch_args<CoreArgs>();
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), h = lane >> 5;
  const int tt = FEW ? lane : (int)threadIdx.x;     // thread of the team
  auto& team = lds.team[FEW ? wave : 0];
  const Place at = place_of<OWN_KEYS, C::OWN>(a);
  const int b = at.b, dh = a.dh;

  // ---- the owned row of this lane ----
  struct OwnRow { int t, row, head; long stat; bool is; };   // position in its group, in the tensor; head; place among the statistics of query rows
  auto own_place = [&](int l) {
    const int col = at.own0 + (FEW ? 0 : 32 * wave) + (l & 31);
    unsigned t = (unsigned)col, g = 0;
    if (!OWN_KEYS && a.G > 1) udivmod((unsigned)col, (unsigned)a.G, t, g);
    OwnRow o;
    o.is = col < at.own_n;
    o.t = (int)t;
    o.row = a.own_row0[at.group] + (int)t;
    o.head = OWN_KEYS ? at.kvh : at.kvh * a.G + (int)g;
    o.stat = ((long)b * a.H + o.head) * a.Tq + o.row;
    return o;
  };
  const OwnRow me = own_place(lane);
  const bool in_range = me.is;
  const int own_row = me.row, own_head = me.head;
  const long own_stat = me.stat;
  bool own_valid = in_range;
  if (OWN_KEYS && a.valid_len) own_valid = in_range && me.t < a.valid_len[b * a.n_seg + a.own_seg[at.group]];
  const float prefix = a.prefix ? a.prefix[b] : IM_NEG_INF;
  const RowInfo own = OWN_KEYS ? key_info(a, prefix, key_raw(a, b, own_row, own_valid)) : query_info(a, query_raw(a, b, own_row, own_valid));

  Frag own1[2 * ND], own2[BWD && !C::OWN_LDS ? 2 * ND : 1];   // Q (and dO), or K and V
  if constexpr (!OWN_KEYS) {
    own_frags<ND>(head_of<const T>(a.q, b, own_row, own_head), in_range, dh, a.vec & VEC_Q, h, own1);
    if constexpr (BWD) own_frags<ND>(head_of<const T>(a.d_o, b, own_row, own_head), in_range, dh, a.vec & VEC_DO, h, own2);
  } else {
    own_frags<ND>(head_of<const T>(a.k, b, own_row, own_head), in_range, dh, a.vec & VEC_K, h, own1);
    if constexpr (C::OWN_LDS) {
      if (!FEW || wave == 0) {
        bf16x8 f[2 * ND];
        own_frags<ND>(head_of<const T>(a.v, b, own_row, own_head), in_range, dh, a.vec & VEC_V, h, f);
#pragma unroll
        for (int s = 0; s < 2 * ND; ++s) lds.own2[(wave * 2 * ND + s) * 64 + lane] = f[s];
      }
    } else own_frags<ND>(head_of<const T>(a.v, b, own_row, own_head), in_range, dh, a.vec & VEC_V, h, own2);
  }
  if (a.own_scale != 1.f) scale_frags(own1, a.own_scale);
  const float own_slope2 = BIAS && !OWN_KEYS && in_range ? a.slope[own_head] * LOG2E : 0.f;

  float own_lse2 = 0.f, own_delta = 0.f;
  if constexpr (WHICH == CORE_DQ) {
    // rows out of range get weight 0 everywhere
    own_lse2 = in_range ? a.lse2[own_stat] : __builtin_inff();
    if (in_range) own_delta = dot_frags<ND>(own2, a.o32 + own_stat * dh, dh, h);
    own_delta += other_half(own_delta);
    if (in_range && h == 0 && (!FEW || wave == 0)) a.delta[own_stat] = own_delta;
  }

  // ---- range of the owned rows, over the workgroup ----
  const bool ranges = a.causal || a.q_doc;   // without them every row's order and document are the same
  {
    const Range r = range_of(own, in_range, ranges);
    if (lane == 0) lds.own[wave] = r;
#pragma unroll
    for (int i = 0; i < BUFS; ++i) {
      for (int r2 = tt; r2 < ROWS; r2 += C::TEAM) team.meta[i].bad[r2] = 0;
      if (tt == 0) team.meta[i].any_bad = 0;
    }
    // columns behind the head's end are never written by the copies
    if (dh < 32 * ND)
      for (int i = tt; i < BUFS * 2 * TL::SLOTS; i += C::TEAM) ((u32x4*)team.tile)[i] = u32x4{0u, 0u, 0u, 0u};
  }
  __syncthreads();
  Range mine = lds.own[0];
  if constexpr (!FEW) {
#pragma unroll
    for (int w = 1; w < CORE_WAVES; ++w) {
      const Range r = lds.own[w];
      mine.lo = fminf(mine.lo, r.lo); mine.hi = fmaxf(mine.hi, r.hi);
      mine.dlo = min(mine.dlo, r.dlo); mine.dhi = max(mine.dhi, r.dhi);
      mine.any |= r.any; mine.all &= r.all;
    }
  }

  // ---- the streamed side ----
  // its rows: keys, or the positions of one query head after another
  const im_view_t& va = OWN_KEYS ? a.q : a.k;
  const im_view_t& vb = OWN_KEYS ? a.d_o : a.v;
  const int head0 = OWN_KEYS ? at.kvh * a.G : at.kvh;
  const T *base_a = head_of<const T>(va, b, 0, head0), *base_b = head_of<const T>(vb, b, 0, head0);
  const bool vec_a = a.vec & (OWN_KEYS ? VEC_Q : VEC_K), vec_b = a.vec & (OWN_KEYS ? VEC_DO : VEC_V);
  const bool words_a = a.words & (OWN_KEYS ? VEC_Q : VEC_K), words_b = a.words & (OWN_KEYS ? VEC_DO : VEC_V);
  const unsigned live = a.own_live[at.group];
  const bool scan = a.causal || a.q_doc || (a.key_pad && !OWN_KEYS);   // classes that depend on the streamed rows' data
  auto stream_len = [&](int j) {   // rows of streamed group j that count
    const int n = a.str_len[j];
    return !OWN_KEYS && a.valid_len ? min(n, max(a.valid_len[b * a.n_seg + a.str_seg[j]], 0)) : n;
  };
  int total = 0;
  for (int j = 0; j < a.str_groups; ++j)
    if ((live >> j) & 1u) total += (stream_len(j) + ROWS - 1) / ROWS * (OWN_KEYS ? a.G : 1);
  if (!mine.any) total = 0;
  const int first = (int)((long)total * at.split / a.splits), last = (int)((long)total * (at.split + 1) / a.splits);

  // ---- accumulators ----
  f32x16 acc1[ND], acc2[WHICH == CORE_DKV ? ND : 1];   // O^T, dQ^T or dK^T; dV^T
#pragma unroll
  for (int d = 0; d < ND; ++d) {
    acc1[d] = zero16();
    if constexpr (WHICH == CORE_DKV) acc2[d] = zero16();
  }
  f32x4 nar1[2] = {}, nar2[2] = {};   // the same of narrow heads
  constexpr float LOWEST = -3.402823466e38f;
  float m = 0.f, l = 0.f, most = LOWEST;   // reference, sum, and by how much a score may exceed the reference
  // A slope's gradient is -sum dS gap.  delta stems from a forward that rounded its probabilities; by how much it is off is what
  // is left of the row's sum of dS (exactly 0 otherwise), and that part is taken back:  -sum (dS - rest P) gap.
  float dslope = 0.f, rest = 0.f, mean_gap = 0.f;

  // Streamed rows go from global memory into LDS by asynchronous copies, one tile ahead, without staging registers.  A thread's
  // unit i of a tile: byte offset off_a / off_b from the tile's first row.
  unsigned off_a[C::N], off_b[C::N];
  bool has[C::N];
#pragma unroll
  for (int i = 0; i < C::N; ++i) {
    const int u = tt + i * C::TEAM, row = TL::row_of(u), c = TL::unit_of(u);
    off_a[i] = (unsigned)(row * va.row * (long)sizeof(T)) + 16 * c;
    off_b[i] = (unsigned)(row * vb.row * (long)sizeof(T)) + 16 * c;
    has[i] = c * EPC < dh;
  }
  int stamp = 0;
  // one tensor's tile; rows behind the n-th repeat the last one (no pair of theirs counts)
  auto copy = [&](const T* from, const im_view_t& view, const unsigned (&off)[C::N], bool vec, bool words, char* to, int n) {
    if (vec) {
#pragma unroll
      for (int i = 0; i < C::N; ++i) {
        unsigned o = off[i];
        if (n < ROWS) {
          const int u = late(tt) + i * C::TEAM;
          o = (unsigned)(min(TL::row_of(u), n - 1) * view.row * (long)sizeof(T)) + 16 * TL::unit_of(u);
        }
        if (has[i]) copy16(from, o, to + (i * C::TEAM + (FEW ? 0 : wave * 64)) * 16);
      }
    } else if (words) {   // 4 bytes a lane
      const int t0 = late(tt);
#pragma unroll(C::N > 2 ? 2 : 4)
      for (int i = 0; i < 4 * C::N; ++i) {
        const int w = t0 + i * C::TEAM, at = 16 * TL::unit_of(w >> 2) + 4 * (w & 3);
        const unsigned o = (unsigned)min(TL::row_of(w >> 2), n - 1) * (unsigned)(view.row * (long)sizeof(T)) + at;
        if (at < dh * (int)sizeof(T)) copy4(from, o, to + (i * C::TEAM + (FEW ? 0 : wave * 64)) * 4);
      }
    } else {   // element by element, through registers
#pragma unroll 1
      for (int i = 0; i < C::N; ++i) {
        const int u = late(tt) + i * C::TEAM;
        *(u32x4*)(to + u * 16) = load_unit(from + min(TL::row_of(u), n - 1) * view.row, TL::unit_of(u) * EPC, dh, false);
      }
    }
  };
  const bool with_pos = a.causal || BIAS;
  const int* docs = OWN_KEYS ? a.q_doc : a.k_doc;
  const float* poss = OWN_KEYS ? a.q_pos : a.k_pos;
  const int own_side = OWN_KEYS ? a.Tq : a.Tk;   // (rows of the streamed side)
  auto fetch = [&](int4 e, int buf) {
    const int row0 = __builtin_amdgcn_readfirstlane(e.x), n = __builtin_amdgcn_readfirstlane(e.y);
    const int g = OWN_KEYS ? __builtin_amdgcn_readfirstlane(e.w) : 0;
    copy(base_a + row0 * va.row + g * va.head, va, off_a, vec_a, words_a, team.tile[buf][0], n);
    copy(base_b + row0 * vb.row + g * vb.head, vb, off_b, vec_b, words_b, team.tile[buf][1], n);
    if (tt < ROWS) {
      const unsigned r = (unsigned)min(tt, n - 1);
      const long at0 = (long)b * own_side + row0;
      if (with_pos) copy4(poss + at0, 4 * r, team.meta[buf].pos);
      if (docs) copy4(docs + at0, 4 * r, team.meta[buf].doc);
      if (!OWN_KEYS && a.key_pad) copy1(a.key_pad + at0, r, team.meta[buf].order);
      if constexpr (OWN_KEYS) {
        const long st = ((long)b * a.H + head0 + g) * a.Tq + row0;
        copy4(a.lse2 + st, 4 * r, team.qmeta[buf].lse2);
        copy4(a.delta + st, 4 * r, team.qmeta[buf].delta);
      }
    }
  };
  // This wave's copies of the tile in `buf` are complete; masks need its rows' order.
  auto arrive = [&](int buf, bool part, int n) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (part && tt < ROWS) {
      RowMeta<ROWS>& meta = team.meta[buf];
      RowRaw raw = {0.f, 0, tt < n ? 0u : 1u};
      if (a.causal) raw.pos = meta.pos[tt];
      if (!OWN_KEYS && a.key_pad && __float_as_uint(meta.order[tt])) raw.pad = 1u;
      meta.order[tt] = OWN_KEYS ? query_info(a, raw).order : key_info(a, prefix, raw).order;
    }
  };
  // values of a tile with masked pairs that are not finite: 0 in their place, and a mark on their row
  auto clean = [&](int buf) {
    u32x4* units = (u32x4*)team.tile[buf];
    const int t0 = late(tt);
    unsigned bits = 0;
#pragma unroll
    for (int i = 0; i < 2 * C::N; ++i) {
      const int u = t0 + i * C::TEAM;
      if (TL::BF && ND == 1 && TL::unit_of(u % TL::SLOTS) >= 4) continue;   // half a panel that nothing reads or writes
      const u32x4 x = units[u];
#pragma unroll
      for (int w = 0; w < 4; ++w) bits |= odd_bits(T(), x[w]);
    }
    if (!odd(T(), bits)) return;
#pragma unroll 1
    for (int i = 0; i < 2 * C::N; ++i) {
      const int u = t0 + i * C::TEAM;
      if (TL::BF && ND == 1 && TL::unit_of(u % TL::SLOTS) >= 4) continue;
      u32x4 x = units[u];
      bits = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w) bits |= odd_bits(T(), x[w]);
      if (!odd(T(), bits)) continue;
#pragma unroll
      for (int w = 0; w < 4; ++w) x[w] = clean_bits(T(), x[w]);
      units[u] = x;
      team.meta[buf].bad[TL::row_of(u % TL::SLOTS)] = stamp;
      team.meta[buf].any_bad = stamp;
    }
  };

  const LaneAt<T, ND, ROWS> at_lane(lane);
  float tile_slope2 = 0.f;   // of the streamed tile's head
  const unsigned own2_at = lds_at(lds.own2) + ((FEW ? 0 : wave) * 2 * ND * 64 + lane) * 16;
  auto products = [&](int buf, int row32, f32x16& sc, f32x16& dp) {
    const unsigned ta = lds_at(team.tile[buf][0]), tb = lds_at(team.tile[buf][1]);
    sc = zero16();
#pragma unroll
    for (int st = 0; st < 2 * ND; ++st)
      if (sizeof(T) == 2 || 16 * st < dh) sc = at_lane.rows(ta, row32, st, own1[st], sc, dh - 16 * st);
    if constexpr (BWD) {
      dp = zero16();
#pragma unroll
      for (int st = 0; st < 2 * ND; ++st)
        if (sizeof(T) == 2 || 16 * st < dh) {
          if constexpr (C::OWN_LDS) dp = at_lane.rows(tb, row32, st, lds_load<bf16x8>(own2_at, st * 1024), dp, 0);
          else dp = at_lane.rows(tb, row32, st, own2[st], dp, dh - 16 * st);
        }
    }
  };
  auto block = [&](int buf, int row32, bool part, bool odd_values, const f32x16& sc, const f32x16& dp) {
    const unsigned ta = lds_at(team.tile[buf][0]), tb = lds_at(team.tile[buf][1]);
    const RowMeta<ROWS>& meta = team.meta[buf];
    const float k = a.to_log2;   // raw score (after the cap, if any) -> units of log2
    bool large = false;
    float top = 0.f;
    if constexpr (CAP) {
      top = fabsf(sc[0]);
#pragma unroll
      for (int r = 1; r < 16; ++r) top = fmaxf(top, fabsf(sc[r]));
      large = __any(top >= a.small_to);
    }
    // Eight rows at a time: register 8 i + e of a product is streamed row row0 + e.  x: score less the reference (forward) or the row's
    // log-sum-exp (backward), -inf where the pair is masked; g: derivative of the cap; gap: distance.
    auto scores = [&](int i, float (&x)[8], float (&g)[CAP && BWD ? 8 : 1], float (&gap)[BIAS ? 8 : 1]) {
      const int row0 = row32 + 16 * i + 8 * h;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = sc[8 * i + e];
      if constexpr (CAP) tanh_of(a, x, large);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (CAP && BWD) g[e] = __builtin_fmaf(-x[e] * a.c_in, x[e] * a.c_in, 1.f);
        float ref = m;
        if constexpr (WHICH == CORE_DQ) ref = own_lse2;
        if constexpr (WHICH == CORE_DKV) ref = team.qmeta[buf].lse2[row0 + e];
        x[e] = __builtin_fmaf(x[e], k, -ref);
        if constexpr (BIAS) {
          float sl = own_slope2;
          if constexpr (OWN_KEYS) sl = tile_slope2;
          gap[e] = fabsf(meta.pos[row0 + e] - own.pos);
          x[e] = __builtin_fmaf(-sl, gap[e], x[e]);
        }
      }
      if (part) {
        if (odd_values) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (meta.bad[row0 + e] == stamp) x[e] = __builtin_nanf("");
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float o = meta.order[row0 + e];
          x[e] = (OWN_KEYS ? own.order <= o : o <= own.order) ? x[e] : IM_NEG_INF;
        }
        if (docs) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = meta.doc[row0 + e] == own.doc ? x[e] : IM_NEG_INF;
        }
      }
    };
    Frag p[2], q[2];
    float x[2][8];   // (forward)
    bool own_heavy = false, heavy = false;
    if constexpr (WHICH == CORE_FWD) {
      float none[1], gap[BIAS ? 8 : 1];
      float mx = IM_NEG_INF;
#pragma unroll
      for (int i = 0; i < 2; ++i) scores(i, x[i], none, gap);
      auto largest = [&]() {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) mx = fmaxf(mx, x[i][e]);
      };
      // A cap makes no score larger: the largest |raw score|, which is known already, bounds it.  (It may be a masked pair's, so a row must not be
      // told from its bound what it does to its own results; with a backward to come the scores' maximum is taken.)
      const bool saving = sizeof(T) == 2 && a.o32;   // (only a backward asks for it)
      const bool bound = CAP && !BIAS && !saving;
      if (bound) mx = __builtin_fmaf(top, k, -m);
      else largest();
      float own_mx = mx;   // this half's part of its row
      // A row's reference is its first block's largest score and moves only when a score exceeds it by 8: probabilities stay below
      // 2^8, and no row's bits depend on another's.
      if (__any(mx > most)) {
        if (bound) {
          mx = IM_NEG_INF;
          largest();
        }
        mx = fmaxf(mx, other_half(mx));
        const float by = mx > most ? mx : 0.f;
        const float f = by > 0.f ? fast_exp2(-by) : 1.f;   // (a first reference below 0 has nothing to scale yet)
        if (mx > most) most = 8.f;
        m += by;
        own_mx -= by;
        l *= f;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) x[i][e] -= by;
        if constexpr (NARROW) {
          const u32x2 s = swap16(f, f);
          nar1[0] *= __uint_as_float(s[0]);
          nar1[1] *= __uint_as_float(s[1]);
        } else {
#pragma unroll
          for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc1[d][r] *= f;
        }
      }
      if constexpr (sizeof(T) == 2) {
        if (saving) {
          own_heavy = 4.f * fast_exp2(own_mx) > l;
          heavy = __any(own_heavy);
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = fast_exp2(x[i][e]);
        // (in pairs: a row of thousands of keys is no chain of thousands of roundings)
        l += ((x[i][0] + x[i][1]) + (x[i][2] + x[i][3])) + ((x[i][4] + x[i][5]) + (x[i][6] + x[i][7]));
        p[i] = pack_p((const T*)nullptr, x[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row0 = row32 + 16 * i + 8 * h;
        float x[8], ds[8], g[CAP ? 8 : 1], gap[BIAS ? 8 : 1];
        scores(i, x, g, gap);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float delta = own_delta;
          if constexpr (OWN_KEYS) delta = team.qmeta[buf].delta[row0 + e];
          x[e] = fast_exp2(x[e]);
          ds[e] = mul0(x[e], dp[8 * i + e] - delta);
        }
        if (BIAS && WHICH == CORE_DQ && a.dslope_rows) {
          float s = 0.f, r = 0.f, g1 = 0.f;   // eight rows' sums first, for the same reason as in the forward
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            s += ds[e] * gap[BIAS ? e : 0];
            r += ds[e];
            g1 += x[e] * gap[BIAS ? e : 0];
          }
          dslope -= s;
          rest += r;
          mean_gap += g1;
        }
        if constexpr (CAP) {
#pragma unroll
          for (int e = 0; e < 8; ++e) ds[e] = mul0(ds[e], g[e]);
        }
        if constexpr (WHICH == CORE_DKV) p[i] = pack_p((const T*)nullptr, x);
        q[i] = pack_p((const T*)nullptr, ds);
        if constexpr (C::OWN_LDS) __builtin_amdgcn_sched_barrier(0);   // one half's scores at a time
      }
    }
    // the second product; for dK/dV both
    if constexpr (NARROW) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if constexpr (WHICH == CORE_FWD) at_lane.cols16(tb, row32 + 16 * i, p[i], nar1);
        else at_lane.cols16(ta, row32 + 16 * i, q[i], nar1);
        if constexpr (WHICH == CORE_DKV) at_lane.cols16(tb, row32 + 16 * i, p[i], nar2);
      }
    } else
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int d = 0; d < ND; ++d)
        if (sizeof(T) == 2 || 32 * d < dh) {
          if constexpr (WHICH == CORE_FWD) acc1[d] = at_lane.cols(tb, row32 + 16 * i, d, p[i], acc1[d]);
          else acc1[d] = at_lane.cols(ta, row32 + 16 * i, d, q[i], acc1[d]);
          if constexpr (WHICH == CORE_DKV) acc2[d] = at_lane.cols(tb, row32 + 16 * i, d, p[i], acc2[d]);
        }
    // The backward takes sum P dP from the saved output.  Where single keys carry a row, the rounding of their probabilities would be off there as much
    // as that of dS; so a row of which one key may be an eighth or more of what it has seen (l: its half) takes what the rounding left in a
    // second product.  (3 x 3124 steps with documents: dQ and dK 1.49 -> 1.43 times the error of one rounding at the end, for 14 us of 620.)
    if constexpr (WHICH == CORE_FWD && sizeof(T) == 2) {
      if (heavy) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const u32x4 w = __builtin_bit_cast(u32x4, p[i]);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[i][e] -= __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
            x[i][e] = own_heavy ? x[i][e] : 0.f;
          }
          const Frag left = pack_p((const T*)nullptr, x[i]);
#pragma unroll
          for (int d = 0; d < ND; ++d) acc1[d] = at_lane.cols(tb, row32 + 16 * i, d, left, acc1[d]);
        }
      }
    }
  };

  for (int lo = first; lo < last; lo += CORE_LIST) {
    const int n = min(CORE_LIST, last - lo);
    // ---- list of the next tiles ----
    if ((int)threadIdx.x < n) {
      int t = lo + (int)threadIdx.x, j = 0, len = 0, g = 0;
      for (; j < a.str_groups; ++j) {
        if (!((live >> j) & 1u)) continue;
        len = stream_len(j);
        const int nt = (len + ROWS - 1) / ROWS, all = OWN_KEYS ? nt * a.G : nt;
        if (t < all) {
          if (OWN_KEYS && a.G > 1) { g = t / nt; t -= g * nt; }
          break;
        }
        t -= all;
      }
      const int row0 = a.str_row0[j] + t * ROWS, rows = min(ROWS, len - t * ROWS);
      const bool full = rows == ROWS && mine.all && !scan;
      lds.list[threadIdx.x] = make_int4(row0, rows, full ? TILE_FULL | 0xf000 : TILE_PART, g);
    }
    __syncthreads();
    if (scan) {
      for (int i = wave; i < n; i += CORE_WAVES) {
        const int4 e = lds.list[i];
        const bool in = lane < e.y;
        const RowInfo info = OWN_KEYS ? query_info(a, query_raw(a, b, e.x + lane, in)) : key_info(a, prefix, key_raw(a, b, e.x + lane, in));
        const Range r = range_of(info, in, ranges);
        // each wave's rows on their own: a wave skips what none of its rows see, or saves the comparisons
        const Range& w = lds.own[FEW ? 0 : lane & (CORE_WAVES - 1)];
        const int cls = OWN_KEYS ? tile_class(w, r, e.y == ROWS, ranges) : tile_class(r, w, e.y == ROWS, ranges);
        const int skip = (int)__ballot(cls == TILE_SKIP) & 15, full = (int)__ballot(cls == TILE_FULL) & 15;
        if (lane == 0) lds.list[i].z = (skip == 15 ? TILE_SKIP : full == 15 ? TILE_FULL : TILE_PART) | skip << 8 | full << 12;
      }
      __syncthreads();
    }
    // ---- walk over it ----
    const int step = FEW ? CORE_WAVES : 1;
    int i = (FEW ? wave : 0) - step;
    auto next = [&]() {   // the next tile to visit; its row count is 0 at the end
      int4 e;
      do {
        i += step;
        e = i < n ? lds.list[i] : make_int4(0, 0, TILE_FULL, 0);
      } while ((__builtin_amdgcn_readfirstlane(e.z) & 3) == TILE_SKIP);
      return make_int4(__builtin_amdgcn_readfirstlane(e.x), __builtin_amdgcn_readfirstlane(e.y), __builtin_amdgcn_readfirstlane(e.z),
                       OWN_KEYS ? __builtin_amdgcn_readfirstlane(e.w) : 0);
    };
    // Tile e is at hand, its copies were asked for one turn ago; those of the tile ahead go into the other buffer meanwhile.  (With one
    // buffer a tile's copies are waited for.)  The first turn only asks for copies.
    int4 e = make_int4(0, 0, 0, 0);
    int buf = BUFS - 1;
    for (;;) {
      const int4 ahead = next();
      if (e.y) {
        arrive(buf, (e.z & 3) == TILE_PART, e.y);
        team_sync<FEW>();   // all waves' copies are there, and nobody reads the other buffer any more
      }
      if (BUFS == 2 && ahead.y) fetch(ahead, buf ^ 1);
      if (e.y) {
        ++stamp;
        bool odd_values = false;   // replaced by 0: the row's mark counts for every wave
        if ((e.z & 3) == TILE_PART) {
          clean(buf);
          team_sync<FEW>();
          odd_values = __builtin_amdgcn_readfirstlane(team.meta[buf].any_bad) == stamp;
        }
        if constexpr (BIAS && OWN_KEYS) {
          typedef const float __attribute__((address_space(4))) * const_ptr;   // (a scalar load: no wait for the copies in flight)
          tile_slope2 = ((const_ptr)(uintptr_t)a.slope)[head0 + e.w] * LOG2E;
        }
        const int w = FEW ? 0 : wave;
        if (!((e.z >> (8 + w)) & 1)) {
          const bool part = odd_values || !((e.z >> (12 + w)) & 1);
#pragma unroll
          for (int r = 0; r < ROWS / 32; ++r) {
            f32x16 sc, dp;
            products(buf, 32 * r, sc, dp);
            block(buf, 32 * r, part, odd_values, sc, dp);
          }
        }
        if constexpr (FEW) team_sync<FEW>();
      }
      if (!ahead.y) break;
      if constexpr (BUFS == 1) {
        // a copy is no LDS instruction: what the wave still reads of the tile has to be there first (with two buffers the list's entry, read
        // after the tile that the copies replace and in order with it, is what their addresses wait for)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        fetch(ahead, 0);
      }
      buf ^= BUFS - 1;
      e = ahead;
    }
    __syncthreads();   // the list is overwritten
  }

  // ---- results ----
  if constexpr (NARROW) {
    // to the layout of the wide accumulators, through LDS of the wave: lane (n, g) holds elements 4 g .. + 3 of owned rows n and 16 + n
    float* mine16 = (float*)lds_raw + wave * 32 * 16;
    auto widen = [&](const f32x4 (&from)[2], f32x16& to) {
#pragma unroll
      for (int x = 0; x < 2; ++x) *(f32x4*)(mine16 + (16 * x + (lane & 15)) * 16 + 4 * (lane >> 4)) = from[x];
      team_sync<true>();
#pragma unroll
      for (int r = 0; r < 8; ++r) to[r] = mine16[(lane & 31) * 16 + 8 * h + r];
      team_sync<true>();
    };
    widen(nar1, acc1[0]);
    if constexpr (WHICH == CORE_DKV) widen(nar2, acc2[0]);
    __syncthreads();
  }
  if constexpr (WHICH == CORE_FWD) {
    l += other_half(l);
    if (most == LOWEST) m = LOWEST;   // nothing seen
  }
  if constexpr (BIAS && WHICH == CORE_DQ) {
    dslope += other_half(dslope);
    rest += other_half(rest);
    mean_gap += other_half(mean_gap);
  }
  if constexpr (FEW) {
    // the waves' parts of the same rows: through LDS to wave 0, in the order of the waves; a wave that no tile fell to has none
    constexpr int NT = WHICH == CORE_DKV ? 2 * ND : ND;
    float* box = (float*)lds_raw;                    // [NT * 16 + 3][64], the tiles are no longer needed
    for (int w = 1; w < min(CORE_WAVES, last - first); ++w) {
      if (wave == w) {
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            box[(16 * d + r) * 64 + lane] = acc1[d][r];
            if constexpr (WHICH == CORE_DKV) box[(16 * (ND + d) + r) * 64 + lane] = acc2[d][r];
          }
        if constexpr (WHICH == CORE_FWD) {
          box[16 * NT * 64 + lane] = m;
          box[(16 * NT + 1) * 64 + lane] = l;
        }
        if constexpr (BIAS && WHICH == CORE_DQ) {
          box[16 * NT * 64 + lane] = dslope;
          box[(16 * NT + 1) * 64 + lane] = rest;
          box[(16 * NT + 2) * 64 + lane] = mean_gap;
        }
      }
      __syncthreads();
      if (wave == 0) {
        float f0 = 1.f, f1 = 1.f;
        if constexpr (WHICH == CORE_FWD) {
          const float m1 = box[16 * NT * 64 + lane], to = fmaxf(m, m1);
          f0 = fast_exp2(m - to); f1 = fast_exp2(m1 - to);
          m = to;
          l = l * f0 + box[(16 * NT + 1) * 64 + lane] * f1;
        }
        if constexpr (BIAS && WHICH == CORE_DQ) {
          dslope += box[16 * NT * 64 + lane];
          rest += box[(16 * NT + 1) * 64 + lane];
          mean_gap += box[(16 * NT + 2) * 64 + lane];
        }
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            acc1[d][r] = acc1[d][r] * f0 + box[(16 * d + r) * 64 + lane] * f1;
            if constexpr (WHICH == CORE_DKV) acc2[d][r] += box[(16 * (ND + d) + r) * 64 + lane];
          }
      }
      __syncthreads();
    }
    if (wave != 0) return;
  }
  const OwnRow to = own_place(late(lane));   // made again rather than kept
  if (!to.is) return;
  if constexpr (WHICH == CORE_FWD) {
    if (a.splits > 1) {
      const long row = ((long)at.split * a.B * a.H * a.Tq) + to.stat;
      store_row<float, ND>(a.part_o + row * dh, dh, dh % 4 == 0, h, acc1, 1.f);
      if (h == 0) { a.part_ml[2 * row] = m; a.part_ml[2 * row + 1] = l; }
      return;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l, lse2 = l == 0.f ? IM_NEG_INF : m + log2f(l);
    store_row<T, ND>(head_of<T>(a.o, b, to.row, to.head), dh, a.vec & VEC_O, h, acc1, inv);
    if (a.o32) store_row<float, ND>(a.o32 + to.stat * dh, dh, dh % 4 == 0, h, acc1, inv);
    if (h == 0) {
      if (a.lse) a.lse[to.stat] = lse2 * LN2;
      if (a.lse2) a.lse2[to.stat] = lse2;
    }
  } else if constexpr (WHICH == CORE_DQ) {
    store_row<T, ND>(head_of<T>(a.dq, b, to.row, to.head), dh, a.vec & VEC_DQ, h, acc1, a.scale);
    if (BIAS && a.dslope_rows && h == 0) a.dslope_rows[to.stat] = dslope + rest * mean_gap;
  } else {
    store_row<T, ND>(head_of<T>(a.dk, b, to.row, to.head), dh, a.vec & VEC_DK, h, acc1, a.scale);
    store_row<T, ND>(head_of<T>(a.dv, b, to.row, to.head), dh, a.vec & VEC_DV, h, acc2, 1.f);
  }
}

// ---- launches ----
template <class T, int ND, bool FEW, CoreKernel WHICH>
constexpr size_t core_lds() {
  constexpr size_t need = sizeof(CoreLds<T, ND, FEW, WHICH>), box = FEW ? ((WHICH == CORE_DKV ? 2 : 1) * ND * 16 + 3) * 64 * 4 : 0;
  static_assert((need > box ? need : box) <= 160 * 1024, "LDS of a CU");
  return need > box ? need : box;
}
template <class T, int W, bool FEW, bool CAP, bool BIAS, CoreKernel WHICH>
static void core_go(const CoreArgs& a, unsigned grid, hipStream_t st) {
  constexpr size_t lds = core_lds<T, (W ? W : 1), FEW, WHICH>();
  auto* fn = core_kernel<T, W, FEW, CAP, BIAS, WHICH>;
  if (lds > 64 * 1024) (void)hipFuncSetAttribute((const void*)fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  hipLaunchKernelGGL(fn, dim3(grid), dim3(64 * CORE_WAVES), lds, st, a);
}
template <class T, int W, bool FEW, CoreKernel WHICH>
static void core_mods(const CoreArgs& a, unsigned grid, hipStream_t st) {
  const bool cap = a.cap > 0.f, bias = a.slope != nullptr;
  if (cap && bias) core_go<T, W, FEW, true, true, WHICH>(a, grid, st);
  else if (cap) core_go<T, W, FEW, true, false, WHICH>(a, grid, st);
  else if (bias) core_go<T, W, FEW, false, true, WHICH>(a, grid, st);
  else core_go<T, W, FEW, false, false, WHICH>(a, grid, st);
}
template <class T, bool FEW, CoreKernel WHICH>
static void core_width(const CoreArgs& a, unsigned grid, hipStream_t st) {
  if constexpr (sizeof(T) == 4)
    if (a.dh <= 16) { core_mods<T, 0, FEW, WHICH>(a, grid, st); return; }
  if (a.dh <= 32) core_mods<T, 1, FEW, WHICH>(a, grid, st);
  else if (a.dh <= 64) core_mods<T, 2, FEW, WHICH>(a, grid, st);
  else core_mods<T, 4, FEW, WHICH>(a, grid, st);
}
template <class T, CoreKernel WHICH>
static void core_widths(bool few, const CoreArgs& a, unsigned grid, hipStream_t st) {
  if (few) core_width<T, true, WHICH>(a, grid, st);
  else core_width<T, false, WHICH>(a, grid, st);
}

}  // namespace imattn
