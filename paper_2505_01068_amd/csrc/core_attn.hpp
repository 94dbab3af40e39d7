// Attention of projected heads with capped, biased and masked scores: host/device definitions (include/imattn.h).
#pragma once
#include "entry.hpp"

namespace imattn {

// One problem, passed to the kernels by value.  "Query row" below is a pair (position t, head g of the key head's group):
// row t * G + g of a segment, so that the heads that share a key head share its tiles.
struct CoreArgs {
  int B, H, Hkv, G, dh, n_seg, Tq, Tk;
  // The launch's owned rows (queries; keys for dK/dV) and streamed rows in groups of neighbouring segments that the pattern of live blocks
  // treats alike.  Owned groups in launch order, those with most to read first; tile_prefix counts their tiles.  seg: the group's
  // (only) segment, where valid_len needs one.
  int own_groups, own_row0[IM_MAX_SEG], own_len[IM_MAX_SEG], own_seg[IM_MAX_SEG], tile_prefix[IM_MAX_SEG + 1];
  unsigned own_live[IM_MAX_SEG];   // bit per streamed group
  int str_groups, str_row0[IM_MAX_SEG], str_len[IM_MAX_SEG], str_seg[IM_MAX_SEG];
  int splits;                     // workgroups that share the keys of one tile (forward)
  unsigned vec, words;            // bit per tensor (VecBit): heads in aligned units of 16 bytes, of 4 bytes
  int causal;
  float cap;
  float own_scale;                // power of two by which owned rows enter the raw score (1 but where scale or scale / cap is extreme)
  float to_log2;                  // scale / own_scale * log2(e): raw score (after the cap) -> units of log2
  float c_in, inv_c_in;           // scale / own_scale / cap: raw score -> argument of the tangent
  float small_to, tanh_q[3];      // raw scores below small_to take the polynomial 1 + u (q0 + u (q1 + u q2)), u = raw^2
  float scale;
  im_view_t q, k, v, o, d_o, dq, dk, dv;
  const int32_t* valid_len;
  const uint8_t* key_pad;
  const float *q_pos, *k_pos, *slope, *prefix;
  const int32_t *q_doc, *k_doc;
  float* lse;                     // [B, H, Tq], natural logarithm
  float *o32, *lse2;              // saved: [B, H, Tq, dh] and [B, H, Tq] in log2
  float *delta, *dslope_rows;     // [B, H, Tq]
  float *part_o, *part_ml;        // [splits][B, H, Tq][dh], [splits][B, H, Tq][2]
};
enum VecBit { VEC_Q = 1, VEC_K = 2, VEC_V = 4, VEC_O = 8, VEC_DO = 16, VEC_DQ = 32, VEC_DK = 64, VEC_DV = 128 };

enum CoreKernel { CORE_FWD = 0, CORE_DQ = 1, CORE_DKV = 2 };
// Whether the workgroup's four waves take 32 rows each and share every streamed tile (false), or take the same 32 rows and a
// quarter of the streamed tiles each (true).
void launch_core_fwd_f32(bool few, const CoreArgs& a, unsigned grid, hipStream_t st);
void launch_core_fwd_bf16(bool few, const CoreArgs& a, unsigned grid, hipStream_t st);
void launch_core_dq_f32(bool few, const CoreArgs& a, unsigned grid, hipStream_t st);
void launch_core_dq_bf16(bool few, const CoreArgs& a, unsigned grid, hipStream_t st);
void launch_core_dkv_f32(bool few, const CoreArgs& a, unsigned grid, hipStream_t st);
void launch_core_dkv_bf16(bool few, const CoreArgs& a, unsigned grid, hipStream_t st);

}  // namespace imattn
