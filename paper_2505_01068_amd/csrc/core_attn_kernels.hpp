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
// What bounds them: not the matrix cores but the score arithmetic -- with a cap an exponential and a reciprocal per score on top
// of the softmax's exponential, each four times as long as an ordinary instruction -- except in fp32 from head
// dimension 64 on, where the fp32 matrix rate does.
//
// Which streamed tiles are visited is decided from the data, once per workgroup and 256 tiles: a tile in which no owned row
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
constexpr int CORE_LIST = 256;   // streamed tiles classified at a time
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

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
// bf16: panels of 64 columns, swizzled as lds_frag_sw expects.  fp32: rows of 32 ND floats, 16-byte unit c of row r at c ^ (r % 8).
template <class T, int ND, int ROWS>
struct Tile {
  static constexpr int CPR = ND * 32 / CoreT<T>::EPC;   // 16-byte units of a row
  static constexpr int BYTES = sizeof(T) == 2 ? (ND + 1) / 2 * ROWS * 128 : ROWS * ND * 128;
  static __device__ __forceinline__ int unit_at(int row, int c) {   // byte offset of unit c of a row
    if constexpr (sizeof(T) == 2) return (c >> 3) * ROWS * 128 + row * 128 + (((c & 7) ^ sw_f(row & 15)) << 4);
    else return row * ND * 128 + ((c ^ (row & 7)) << 4);
  }
};

// operand by rows: streamed row (in the order perm32) lane % 32 of the 32-row block, contraction step s of 16 elements
template <int ND, int ROWS>
__device__ __forceinline__ bf16x8 row_frag(const bf16_t*, const char* tile, int row32, int s, int lane) {
  const int lrow = perm32(lane & 31);
  return lds_frag_sw((const bf16_t*)(tile + (s >> 2) * ROWS * 128), row32, lrow, 2 * (s & 3) + (lane >> 5));
}
// fp32: elements 16 s + 4 h .. + 3 and 16 s + 8 + 4 h .. + 3, so that a head of up to 8 elements takes half a step
template <int ND, int ROWS>
__device__ __forceinline__ F8 row_frag(const float*, const char* tile, int row32, int s, int lane) {
  const int row = row32 + perm32(lane & 31), h = lane >> 5;
  F8 f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float4 u = *(const float4*)(tile + Tile<float, ND, ROWS>::unit_at(row, 4 * s + 2 * i + h));
    f.v[4 * i] = u.x; f.v[4 * i + 1] = u.y; f.v[4 * i + 2] = u.z; f.v[4 * i + 3] = u.w;
  }
  return f;
}
__device__ __forceinline__ f32x16 mma_rows(bf16x8 a, bf16x8 b, f32x16 c, int) { return mfma32(a, b, c); }
__device__ __forceinline__ f32x16 mma_rows(const F8& a, const F8& b, f32x16 c, int left) {   // left: elements of the head from this step on
#pragma unroll
  for (int j = 0; j < 4; ++j) c = mfma_f32(a.v[j], b.v[j], c);
  if (left > 8) {
#pragma unroll
    for (int j = 4; j < 8; ++j) c = mfma_f32(a.v[j], b.v[j], c);
  }
  return c;
}
// C += (transposed tile, 32 columns from 32 db on in the order perm32) x (16 streamed rows from row16 on), p: the lane's 8 of them
template <int ND, int ROWS>
__device__ __forceinline__ f32x16 mma_cols(const bf16_t*, const char* tile, int row16, int db, bf16x8 p, f32x16 c, int lane) {
  return mfma32(lds_frag_tr_sw_perm((const bf16_t*)(tile + (db >> 1) * ROWS * 128), row16, 32 * (db & 1), lane), p, c);
}
template <int ND, int ROWS>
__device__ __forceinline__ f32x16 mma_cols(const float*, const char* tile, int row16, int db, const F8& p, f32x16 c, int lane) {
  const int col = 32 * db + perm32(lane & 31), row0 = row16 + 8 * (lane >> 5);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    c = mfma_f32(*(const float*)(tile + Tile<float, ND, ROWS>::unit_at(row0 + j, col >> 2) + 4 * (col & 3)), p.v[j], c);
  return c;
}
__device__ __forceinline__ bf16x8 pack_p(const bf16_t*, const float* p) { return pack8(p); }   // the one rounding of probabilities and dS
__device__ __forceinline__ F8 pack_p(const float*, const float* p) {
  F8 f;
#pragma unroll
  for (int j = 0; j < 8; ++j) f.v[j] = p[j];
  return f;
}

// ---- global memory ----
// 16 bytes from element `at` of a head of dh elements; units at or behind its end give 0
template <class T>
__device__ __forceinline__ u32x4 load_unit(const T* head, int at, int dh, bool vec) {
  u32x4 u = {0u, 0u, 0u, 0u};
  if (at >= dh) return u;
  if (vec) return *(const u32x4*)(head + at);
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int e = 0; e < 8; ++e) if (at + e < dh) u[e >> 1] |= (unsigned)head[at + e] << (16 * (e & 1));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) if (at + e < dh) u[e] = __float_as_uint(head[at + e]);
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
// hyperbolic tangent to fp32 accuracy: Taylor series to x^11 below 0.35 (next term 1.3e-8 x), above (1 - e) / (1 + e), e = exp(-2 |x|)
__device__ __forceinline__ float tanh_f32(float x) {
  const float ax = fabsf(x), u = x * x;
  const float e = fast_exp2(-2.f * LOG2E * ax);
  const float big = __builtin_copysignf((1.f - e) * __builtin_amdgcn_rcpf(1.f + e), x);
  const float small = x + x * u * (-1.f / 3 + u * (2.f / 15 + u * (-17.f / 315 + u * (62.f / 2835 + u * (-1382.f / 155925)))));
  return ax < 0.35f ? small : big;
}
// Raw product -> score in units of log2.  With a cap *g is what the derivative needs: bf16 g = r (1 - r) = (1 - tanh^2) / 4
// with r = 1 / (1 + exp(2 x)), tanh x = 1 - 2 r (absolute error 1e-7 of the cap, far below a probability's rounding
// to bf16); fp32 g = 1 - tanh^2.
template <class T, bool CAP, bool GRAD>
__device__ __forceinline__ float score(const CoreArgs& a, float raw, float* g) {
  if constexpr (!CAP) return raw * a.c_in;
  else if constexpr (sizeof(T) == 2) {
    const float r = __builtin_amdgcn_rcpf(1.f + fast_exp2(raw * a.c_in));
    if constexpr (GRAD) *g = r - r * r;
    return a.cap2 - 2.f * a.cap2 * r;
  } else {
    const float t = tanh_f32(raw * a.c_in);
    if constexpr (GRAD) *g = 1.f - t * t;
    return a.cap2 * t;
  }
}

// ---- streamed side ----
enum { TILE_SKIP = 0, TILE_FULL = 1, TILE_PART = 2 };

// per streamed row in LDS
template <int ROWS>
struct __align__(16) RowMeta {
  float order[ROWS];   // k_pos (-inf: free, NaN: no key) when keys are streamed, q_pos (+inf: sees all, NaN: no row) when queries are
  float pos[ROWS];     // position for the bias
  int doc[ROWS];
  int bad[ROWS];       // == number of the tile: holds a value that is not finite
  int any_bad;
};
template <int ROWS>
struct __align__(16) QueryMeta {     // dK/dV only
  float lse2[ROWS], delta[ROWS], slope2[ROWS];
};

struct RowInfo { float order, pos; int doc; };

__device__ __forceinline__ RowInfo key_info(const CoreArgs& a, long b, int row, bool ok) {
  RowInfo i = {__builtin_nanf(""), 0.f, 0};
  if (!ok) return i;
  const long at = b * a.Tk + row;
  if (a.k_doc) i.doc = a.k_doc[at];
  if (a.k_pos) i.pos = a.k_pos[at];
  i.order = a.causal ? i.pos : IM_NEG_INF;
  if (a.prefix && i.pos < a.prefix[b]) i.order = IM_NEG_INF;
  if (a.key_pad && a.key_pad[at]) i.order = __builtin_nanf("");
  return i;
}
__device__ __forceinline__ RowInfo query_info(const CoreArgs& a, long b, int row, bool ok) {
  RowInfo i = {__builtin_nanf(""), 0.f, 0};
  if (!ok) return i;
  const long at = b * a.Tq + row;
  if (a.q_doc) i.doc = a.q_doc[at];
  if (a.q_pos) i.pos = a.q_pos[at];
  i.order = a.causal ? i.pos : __builtin_inff();
  return i;
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
__device__ __forceinline__ Range range_of(const RowInfo& i, bool in_range) {
  const bool ok = in_range && i.order == i.order;
  Range r;
  r.lo = ok ? i.order : __builtin_inff();
  r.hi = ok ? i.order : IM_NEG_INF;
  r.dlo = ok ? i.doc : 0x7fffffff;
  r.dhi = ok ? i.doc : (int)0x80000000;
  r.any = __any(ok);
  r.all = __all(ok || !in_range);
  range_wave(r);
  return r;
}
__device__ __forceinline__ int tile_class(const Range& keys, const Range& queries, bool whole) {
  if (!keys.any || !queries.any) return TILE_SKIP;
  if (keys.lo > queries.hi || keys.dlo > queries.dhi || keys.dhi < queries.dlo) return TILE_SKIP;
  const bool full = whole && keys.all && queries.all && keys.hi <= queries.lo && keys.dlo == keys.dhi && queries.dlo == queries.dhi && keys.dlo == queries.dlo;
  return full ? TILE_FULL : TILE_PART;
}

template <class T, int ND, bool FEW> struct CoreCfg {
  static constexpr int ROWS = FEW || sizeof(T) == 4 ? 32 : 64;      // streamed rows of a tile
  static constexpr int TEAM = FEW ? 64 : 64 * CORE_WAVES;           // threads that load a tile together
  static constexpr int OWN = FEW ? 32 : 32 * CORE_WAVES;            // owned rows of a workgroup
  static constexpr int BUFS = FEW ? 1 : 2;                          // a wave on its own needs no second buffer
  static constexpr int N = ROWS * Tile<T, ND, ROWS>::CPR / TEAM;    // 16-byte units a thread and tensor
};

// LDS of one team
template <class T, int ND, bool FEW, CoreKernel WHICH>
struct TeamLds {
  using C = CoreCfg<T, ND, FEW>;
  char a[C::BUFS][Tile<T, ND, C::ROWS>::BYTES], b[C::BUFS][Tile<T, ND, C::ROWS>::BYTES];   // K, V or Q, dO
  RowMeta<C::ROWS> meta[C::BUFS];
  typename std::conditional<WHICH == CORE_DKV, QueryMeta<C::ROWS>, char>::type qmeta[C::BUFS];
};
template <class T, int ND, bool FEW, CoreKernel WHICH>
struct CoreLds {
  static constexpr int TEAMS = FEW ? CORE_WAVES : 1;
  __align__(16) TeamLds<T, ND, FEW, WHICH> team[TEAMS];
  int2 list[CORE_LIST];       // first row; rows | class << 16
  Range own[CORE_WAVES];
};

template <bool FEW>
__device__ __forceinline__ void team_sync() {
  if constexpr (FEW) {   // one wave: its LDS instructions stay in order, only the compiler must not move them
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  } else __syncthreads();
}

__device__ __forceinline__ bool odd_bits(bf16_t, unsigned u) { return (u & 0x7f80u) == 0x7f80u || (u & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ bool odd_bits(float, unsigned u) { return (u & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ unsigned clean_bits(bf16_t, unsigned u) {
  if ((u & 0x7f80u) == 0x7f80u) u &= 0xffff0000u;
  if ((u & 0x7f800000u) == 0x7f800000u) u &= 0x0000ffffu;
  return u;
}
__device__ __forceinline__ unsigned clean_bits(float, unsigned u) { return (u & 0x7f800000u) == 0x7f800000u ? 0u : u; }

// Where a workgroup stands: batch element, key head, owned segment, first owned row, split.
struct Place { int b, kvh, seg, own0, own_n, split; };

template <bool OWN_KEYS, int OWN>
__device__ __forceinline__ Place place_of(const CoreArgs& a, int nord) {
  int bx, by, bz;
  xcd_block_index(bx, by, bz);   // 1-d grid
  const int tiles = a.tile_prefix[nord];
  unsigned rest, tile, bh, split, b, kvh;
  udivmod((unsigned)bx, (unsigned)tiles, rest, tile);
  udivmod(rest, (unsigned)a.splits, bh, split);
  udivmod(bh, (unsigned)a.Hkv, b, kvh);
  int k = 0;
  while (k + 1 < nord && (int)tile >= a.tile_prefix[k + 1]) ++k;
  Place p;
  p.b = (int)b; p.kvh = (int)kvh; p.split = (int)split; p.seg = a.order[k];
  p.own_n = OWN_KEYS ? a.k_off[p.seg + 1] - a.k_off[p.seg] : (a.q_off[p.seg + 1] - a.q_off[p.seg]) * a.G;
  // the last tile of a segment first: under causality it sees most
  p.own0 = (a.tile_prefix[k + 1] - 1 - (int)tile) * OWN;
  return p;
}

// Streamed tensors as rows; G > 1: row i is position i / G, head i % G of the group
struct Streamed { const char *a, *b; long a_row, a_head, b_row, b_head; };
template <class T>
__device__ __forceinline__ const T* streamed_row(const char* base, long row, long head, int G, int i) {
  if (G == 1) return (const T*)base + i * row;
  unsigned t, g;
  udivmod((unsigned)i, (unsigned)G, t, g);
  return (const T*)base + t * row + g * head;
}

// ---- the kernel ----
template <class T, int ND, bool FEW, bool CAP, bool BIAS, CoreKernel WHICH>
__global__ __launch_bounds__(64 * CORE_WAVES, 1) void core_kernel(CoreArgs a) {
  using C = CoreCfg<T, ND, FEW>;
  using Frag = typename CoreT<T>::Frag;
  constexpr int ROWS = C::ROWS, EPC = CoreT<T>::EPC, CPR = Tile<T, ND, ROWS>::CPR, BUFS = C::BUFS;
  constexpr bool OWN_KEYS = WHICH == CORE_DKV, BWD = WHICH != CORE_FWD;
  extern __shared__ __align__(16) char lds_raw[];
  auto& lds = *(CoreLds<T, ND, FEW, WHICH>*)lds_raw;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
  const int tt = FEW ? lane : (int)threadIdx.x;     // thread of the team
  auto& team = lds.team[FEW ? wave : 0];
  const Place at = place_of<OWN_KEYS, C::OWN>(a, a.n_seg);
  const int b = at.b, dh = a.dh;

  // ---- the owned row of this lane ----
  const int col = at.own0 + (FEW ? 0 : 32 * wave) + (lane & 31);
  const bool in_range = col < at.own_n;
  unsigned own_t = (unsigned)col, own_g = 0;
  if (!OWN_KEYS && a.G > 1) udivmod((unsigned)col, (unsigned)a.G, own_t, own_g);
  const int own_row = (OWN_KEYS ? a.k_off[at.seg] : a.q_off[at.seg]) + (int)own_t;
  const int own_head = OWN_KEYS ? at.kvh : at.kvh * a.G + (int)own_g;
  bool own_valid = in_range;
  if (OWN_KEYS && a.valid_len) own_valid = in_range && (int)own_t < a.valid_len[b * a.n_seg + at.seg];
  const RowInfo own = OWN_KEYS ? key_info(a, b, own_row, own_valid) : query_info(a, b, own_row, own_valid);
  const long own_stat = ((long)b * a.H + own_head) * a.Tq + own_row;   // of a query row

  Frag own1[2 * ND], own2[BWD ? 2 * ND : 1];   // Q (and dO), or K and V
  if constexpr (!OWN_KEYS) {
    own_frags<ND>(head_of<const T>(a.q, b, own_row, own_head), in_range, dh, a.vec & VEC_Q, h, own1);
    if constexpr (BWD) own_frags<ND>(head_of<const T>(a.d_o, b, own_row, own_head), in_range, dh, a.vec & VEC_DO, h, own2);
  } else {
    own_frags<ND>(head_of<const T>(a.k, b, own_row, own_head), in_range, dh, a.vec & VEC_K, h, own1);
    own_frags<ND>(head_of<const T>(a.v, b, own_row, own_head), in_range, dh, a.vec & VEC_V, h, own2);
  }
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
  {
    const Range r = range_of(own, in_range);
    if (lane == 0) lds.own[wave] = r;
#pragma unroll
    for (int i = 0; i < BUFS; ++i) {
      for (int r2 = tt; r2 < ROWS; r2 += C::TEAM) team.meta[i].bad[r2] = 0;
      if (tt == 0) team.meta[i].any_bad = 0;
    }
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
  Streamed s;
  if constexpr (OWN_KEYS) {
    s.a = (const char*)head_of<const T>(a.q, b, 0, (long)at.kvh * a.G);
    s.b = (const char*)head_of<const T>(a.d_o, b, 0, (long)at.kvh * a.G);
    s.a_row = a.q.row; s.a_head = a.q.head; s.b_row = a.d_o.row; s.b_head = a.d_o.head;
  } else {
    s.a = (const char*)head_of<const T>(a.k, b, 0, at.kvh);
    s.b = (const char*)head_of<const T>(a.v, b, 0, at.kvh);
    s.a_row = a.k.row; s.a_head = 0; s.b_row = a.v.row; s.b_head = 0;
  }
  const int G = OWN_KEYS ? a.G : 1;
  const bool vec_a = a.vec & (OWN_KEYS ? VEC_Q : VEC_K), vec_b = a.vec & (OWN_KEYS ? VEC_DO : VEC_V);
  const unsigned live = OWN_KEYS ? a.k_live[at.seg] : a.q_live[at.seg];
  const bool scan = a.causal || a.q_doc || (a.key_pad && !OWN_KEYS);   // classes that depend on the streamed rows' data
  auto stream_len = [&](int j) {   // rows of streamed segment j that count
    if (OWN_KEYS) return (a.q_off[j + 1] - a.q_off[j]) * a.G;
    const int n = a.k_off[j + 1] - a.k_off[j];
    return a.valid_len ? min(n, max(a.valid_len[b * a.n_seg + j], 0)) : n;
  };
  int total = 0;
  for (int j = 0; j < a.n_seg; ++j)
    if ((live >> j) & 1u) total += (stream_len(j) + ROWS - 1) / ROWS;
  if (!mine.any) total = 0;
  const int first = (int)((long)total * at.split / a.splits), last = (int)((long)total * (at.split + 1) / a.splits);

  // ---- accumulators ----
  f32x16 acc1[ND], acc2[WHICH == CORE_DKV ? ND : 1];   // O^T, dQ^T or dK^T; dV^T
#pragma unroll
  for (int d = 0; d < ND; ++d) {
    acc1[d] = zero16();
    if constexpr (WHICH == CORE_DKV) acc2[d] = zero16();
  }
  float m = -3.402823466e38f, l = 0.f;
  // A slope's gradient is -sum dS gap.  delta stems from a forward that rounded its probabilities; by how much it is off is what
  // is left of the row's sum of dS (exactly 0 otherwise), and that part is taken back:  -sum (dS - rest P) gap.
  float dslope = 0.f, rest = 0.f, mean_gap = 0.f;

  u32x4 ra[C::N], rb[C::N];
  RowInfo ri = {0.f, 0.f, 0};
  float r_lse2 = 0.f, r_delta = 0.f, r_slope2 = 0.f;
  int stamp = 0;

  // global -> registers of one list entry
  auto fetch = [&](int2 e) {
    const int row0 = e.x, n = e.y & 0xffff;
#pragma unroll
    for (int i = 0; i < C::N; ++i) {
      const int u = tt + i * C::TEAM, row = u / CPR, c = u % CPR;
      u32x4 z = {0u, 0u, 0u, 0u};
      ra[i] = rb[i] = z;
      if (row < n) {
        ra[i] = load_unit(streamed_row<T>(s.a, s.a_row, s.a_head, G, row0 + row), c * EPC, dh, vec_a);
        rb[i] = load_unit(streamed_row<T>(s.b, s.b_row, s.b_head, G, row0 + row), c * EPC, dh, vec_b);
      }
    }
    if (tt < ROWS) {
      const bool ok = tt < n;
      if constexpr (OWN_KEYS) {
        unsigned t = (unsigned)(row0 + tt), g = 0;
        if (a.G > 1) udivmod(t, (unsigned)a.G, t, g);
        ri = query_info(a, b, (int)t, ok);
        const int head = at.kvh * a.G + (int)g;
        const long st = ((long)b * a.H + head) * a.Tq + (int)t;
        r_lse2 = ok ? a.lse2[st] : __builtin_inff();
        r_delta = ok ? a.delta[st] : 0.f;
        r_slope2 = BIAS && ok ? a.slope[head] * LOG2E : 0.f;
      } else ri = key_info(a, b, row0 + tt, ok);
    }
  };
  // registers -> LDS
  auto put = [&](int buf, int cls) {
    char *ta = team.a[buf], *tb = team.b[buf];
#pragma unroll
    for (int i = 0; i < C::N; ++i) {
      const int u = tt + i * C::TEAM, row = u / CPR, c = u % CPR;
      u32x4 x = ra[i], y = rb[i];
      if (cls == TILE_PART) {
        bool odd = false;
#pragma unroll
        for (int w = 0; w < 4; ++w) odd |= odd_bits(T(), x[w]) | odd_bits(T(), y[w]);
        if (odd) {
#pragma unroll
          for (int w = 0; w < 4; ++w) { x[w] = clean_bits(T(), x[w]); y[w] = clean_bits(T(), y[w]); }
          team.meta[buf].bad[row] = stamp;
          team.meta[buf].any_bad = stamp;
        }
      }
      const int to = Tile<T, ND, ROWS>::unit_at(row, c);
      *(u32x4*)(ta + to) = x;
      *(u32x4*)(tb + to) = y;
    }
    if (tt < ROWS) {
      team.meta[buf].order[tt] = ri.order;
      team.meta[buf].pos[tt] = ri.pos;
      team.meta[buf].doc[tt] = ri.doc;
      if constexpr (OWN_KEYS) {
        team.qmeta[buf].lse2[tt] = r_lse2;
        team.qmeta[buf].delta[tt] = r_delta;
        team.qmeta[buf].slope2[tt] = r_slope2;
      }
    }
  };

  // one block of 32 streamed rows
  auto block = [&](int buf, int row32, bool part) {
    const char *ta = team.a[buf], *tb = team.b[buf];
    const RowMeta<ROWS>& meta = team.meta[buf];
    f32x16 sc = zero16(), dp;
#pragma unroll
    for (int st = 0; st < 2 * ND; ++st)
      if (sizeof(T) == 2 || 16 * st < dh) sc = mma_rows(row_frag<ND, ROWS>((const T*)nullptr, ta, row32, st, lane), own1[st], sc, dh - 16 * st);
    if constexpr (BWD) {
      dp = zero16();
#pragma unroll
      for (int st = 0; st < 2 * ND; ++st)
        if (sizeof(T) == 2 || 16 * st < dh) dp = mma_rows(row_frag<ND, ROWS>((const T*)nullptr, tb, row32, st, lane), own2[st], dp, dh - 16 * st);
    }
    float x[16], g[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = score<T, CAP, BWD>(a, sc[r], &g[r]);
    // register r: streamed row row32 + 16 (r / 8) + 8 h + r % 8
    float gap[BIAS ? 16 : 1];
    if constexpr (BIAS) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int row = row32 + 16 * (r >> 3) + 8 * h + (r & 7);
        gap[r] = fabsf(meta.pos[row] - own.pos);
        float sl = own_slope2;
        if constexpr (OWN_KEYS) sl = team.qmeta[buf].slope2[row];
        x[r] -= sl * gap[r];
      }
    }
    if (part) {
      const bool bad = meta.any_bad == stamp;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int row = row32 + 16 * (r >> 3) + 8 * h + (r & 7);
        const float o = meta.order[row];
        const bool sees = (OWN_KEYS ? own.order <= o : o <= own.order) && meta.doc[row] == own.doc;
        if (bad && meta.bad[row] == stamp) x[r] = __builtin_nanf("");
        x[r] = sees ? x[r] : IM_NEG_INF;
      }
    }
    if constexpr (WHICH == CORE_FWD) {
      float mx = x[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, x[r]);
      mx = fmaxf(mx, other_half(mx));
      // a row's reference moves only when a score exceeds it by 8: probabilities stay below 2^8, and no row's bits depend on another's
      if (__any(mx > m + 8.f)) {
        const float to = mx > m + 8.f ? mx : m, f = fast_exp2(m - to);
        m = to;
        l *= f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc1[d][r] *= f;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) { x[r] = fast_exp2(x[r] - m); l += x[r]; }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const Frag p = pack_p((const T*)nullptr, x + 8 * k);
#pragma unroll
        for (int d = 0; d < ND; ++d)
          if (sizeof(T) == 2 || 32 * d < dh) acc1[d] = mma_cols<ND, ROWS>((const T*)nullptr, tb, row32 + 16 * k, d, p, acc1[d], lane);
      }
    } else {
      float ds[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int row = row32 + 16 * (r >> 3) + 8 * h + (r & 7);
        float lse2 = own_lse2, delta = own_delta;
        if constexpr (OWN_KEYS) { lse2 = team.qmeta[buf].lse2[row]; delta = team.qmeta[buf].delta[row]; }
        // a masked score is -inf, also where the row sees nothing at all (lse2 = -inf)
        x[r] = part && x[r] == IM_NEG_INF ? 0.f : fast_exp2(x[r] - lse2);
        ds[r] = x[r] * (dp[r] - delta);
        const bool none = part && x[r] == 0.f;   // the other product of a masked pair, and its score, may be anything
        if (none) ds[r] = 0.f;
        if constexpr (BIAS && WHICH == CORE_DQ) {
          dslope -= ds[r] * gap[r];
          rest += ds[r];
          mean_gap += x[r] * gap[r];
        }
        if constexpr (CAP) ds[r] = none ? 0.f : ds[r] * g[r];
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const Frag q = pack_p((const T*)nullptr, ds + 8 * k);
#pragma unroll
        for (int d = 0; d < ND; ++d)
          if (sizeof(T) == 2 || 32 * d < dh) acc1[d] = mma_cols<ND, ROWS>((const T*)nullptr, ta, row32 + 16 * k, d, q, acc1[d], lane);
        if constexpr (WHICH == CORE_DKV) {
          const Frag p = pack_p((const T*)nullptr, x + 8 * k);
#pragma unroll
          for (int d = 0; d < ND; ++d)
            if (sizeof(T) == 2 || 32 * d < dh) acc2[d] = mma_cols<ND, ROWS>((const T*)nullptr, tb, row32 + 16 * k, d, p, acc2[d], lane);
        }
      }
    }
  };

  for (int lo = first; lo < last; lo += CORE_LIST) {
    const int n = min(CORE_LIST, last - lo);
    // ---- list of the next tiles ----
    if ((int)threadIdx.x < n) {
      int t = lo + (int)threadIdx.x, j = 0, len = 0;
      for (; j < a.n_seg; ++j) {
        if (!((live >> j) & 1u)) continue;
        len = stream_len(j);
        const int nt = (len + ROWS - 1) / ROWS;
        if (t < nt) break;
        t -= nt;
      }
      const int row0 = (OWN_KEYS ? a.q_off[j] * a.G : a.k_off[j]) + t * ROWS, rows = min(ROWS, len - t * ROWS);
      const bool full = rows == ROWS && mine.all && !scan;
      lds.list[threadIdx.x] = make_int2(row0, rows | (full ? TILE_FULL : TILE_PART) << 16);
    }
    __syncthreads();
    if (scan) {
      for (int i = wave; i < n; i += CORE_WAVES) {
        const int2 e = lds.list[i];
        const int rows = e.y & 0xffff;
        const bool in = lane < rows;
        unsigned t = (unsigned)(e.x + lane), g = 0;
        if (OWN_KEYS && a.G > 1) udivmod(t, (unsigned)a.G, t, g);
        const RowInfo info = OWN_KEYS ? query_info(a, b, (int)t, in) : key_info(a, b, (int)t, in);
        const Range r = range_of(info, in);
        const int cls = OWN_KEYS ? tile_class(mine, r, rows == ROWS) : tile_class(r, mine, rows == ROWS);
        if (lane == 0) lds.list[i].y = rows | cls << 16;
      }
      __syncthreads();
    }
    // ---- walk over it ----
    const int step = FEW ? CORE_WAVES : 1;
    auto next = [&](int i) {
      while (i < n && (lds.list[i].y >> 16) == TILE_SKIP) i += step;
      return i;
    };
    int i = next(FEW ? wave : 0), buf = 0;
    if (i < n) fetch(lds.list[i]);
    while (i < n) {
      const int cls = __builtin_amdgcn_readfirstlane(lds.list[i].y >> 16);
      ++stamp;
      put(buf, cls);
      team_sync<FEW>();
      i = next(i + step);
      if (i < n) fetch(lds.list[i]);
      for (int r = 0; r < ROWS; r += 32) block(buf, r, cls == TILE_PART);
      if constexpr (FEW) team_sync<FEW>();
      buf ^= BUFS - 1;
    }
    __syncthreads();   // the list is overwritten
  }

  // ---- results ----
  if constexpr (WHICH == CORE_FWD) l += other_half(l);
  if constexpr (BIAS && WHICH == CORE_DQ) {
    dslope += other_half(dslope);
    rest += other_half(rest);
    mean_gap += other_half(mean_gap);
  }
  if constexpr (FEW) {
    // the four waves' parts of the same rows: through LDS to wave 0, in the order of the waves
    constexpr int NT = WHICH == CORE_DKV ? 2 * ND : ND;
    float* box = (float*)lds_raw;                    // [NT * 16 + 3][64], the tiles are no longer needed
    for (int w = 1; w < CORE_WAVES; ++w) {
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
  if (!in_range) return;
  if constexpr (WHICH == CORE_FWD) {
    if (a.splits > 1) {
      const long row = ((long)at.split * a.B * a.H + (long)b * a.H + own_head) * a.Tq + own_row;
      store_row<float, ND>(a.part_o + row * dh, dh, dh % 4 == 0, h, acc1, 1.f);
      if (h == 0) { a.part_ml[2 * row] = m; a.part_ml[2 * row + 1] = l; }
      return;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l, lse2 = m + log2f(l);
    store_row<T, ND>(head_of<T>(a.o, b, own_row, own_head), dh, a.vec & VEC_O, h, acc1, inv);
    if (a.o32) store_row<float, ND>(a.o32 + own_stat * dh, dh, dh % 4 == 0, h, acc1, inv);
    if (h == 0) {
      if (a.lse) a.lse[own_stat] = lse2 * LN2;
      if (a.lse2) a.lse2[own_stat] = lse2;
    }
  } else if constexpr (WHICH == CORE_DQ) {
    store_row<T, ND>(head_of<T>(a.dq, b, own_row, own_head), dh, a.vec & VEC_DQ, h, acc1, a.d_scale);
    if (BIAS && a.dslope_rows && h == 0) a.dslope_rows[own_stat] = dslope + rest * mean_gap;
  } else {
    store_row<T, ND>(head_of<T>(a.dk, b, own_row, own_head), dh, a.vec & VEC_DK, h, acc1, a.d_scale);
    store_row<T, ND>(head_of<T>(a.dv, b, own_row, own_head), dh, a.vec & VEC_DV, h, acc2, 1.f);
  }
}

// ---- launches ----
template <class T, int ND, bool FEW, CoreKernel WHICH>
constexpr size_t core_lds() {
  constexpr size_t need = sizeof(CoreLds<T, ND, FEW, WHICH>), box = FEW ? ((WHICH == CORE_DKV ? 2 : 1) * ND * 16 + 3) * 64 * 4 : 0;
  static_assert((need > box ? need : box) <= 160 * 1024, "LDS of a CU");
  return need > box ? need : box;
}
template <class T, int ND, bool FEW, bool CAP, bool BIAS, CoreKernel WHICH>
static void core_go(const CoreArgs& a, unsigned grid, hipStream_t st) {
  constexpr size_t lds = core_lds<T, ND, FEW, WHICH>();
  auto* fn = core_kernel<T, ND, FEW, CAP, BIAS, WHICH>;
  if (lds > 64 * 1024) (void)hipFuncSetAttribute((const void*)fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  hipLaunchKernelGGL(fn, dim3(grid), dim3(64 * CORE_WAVES), lds, st, a);
}
template <class T, int ND, bool FEW, CoreKernel WHICH>
static void core_mods(const CoreArgs& a, unsigned grid, hipStream_t st) {
  const bool cap = a.cap > 0.f, bias = a.slope != nullptr;
  if (cap && bias) core_go<T, ND, FEW, true, true, WHICH>(a, grid, st);
  else if (cap) core_go<T, ND, FEW, true, false, WHICH>(a, grid, st);
  else if (bias) core_go<T, ND, FEW, false, true, WHICH>(a, grid, st);
  else core_go<T, ND, FEW, false, false, WHICH>(a, grid, st);
}
template <class T, CoreKernel WHICH>
static void core_widths(bool few, const CoreArgs& a, unsigned grid, hipStream_t st) {
  if (few) {
    if (a.dh <= 32) core_mods<T, 1, true, WHICH>(a, grid, st);
    else if (a.dh <= 64) core_mods<T, 2, true, WHICH>(a, grid, st);
    else core_mods<T, 4, true, WHICH>(a, grid, st);
  } else {
    if (a.dh <= 32) core_mods<T, 1, false, WHICH>(a, grid, st);
    else if (a.dh <= 64) core_mods<T, 2, false, WHICH>(a, grid, st);
    else core_mods<T, 4, false, WHICH>(a, grid, st);
  }
}

}  // namespace imattn
