// Helpers of the entry points: error returns, a view's checks, a kernel's arguments.
#pragma once
#include "common.hpp"

namespace imattn {

template <class... A>
inline int refuse(int code, const char* fmt, A... a) {
  set_error(fmt, a...);
  return code;
}

inline int after_launch(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? IM_OK : refuse(IM_ERR_HIP, "%s launch: %s", what, hipGetErrorString(e));
}

inline size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

// A view of `n[0]` batch elements, `n[1]` rows and `n[2]` heads; an output's elements must not share a place by a stride of 0.
inline int check_view(const char* what, const char* name, const im_view_t* v, const int64_t (&n)[3], size_t es, bool output) {
  if (!v) return refuse(IM_ERR_INVALID, "%s: %s is NULL", what, name);
  if (n[0] == 0 || n[1] == 0 || n[2] == 0) return IM_OK;
  if (!v->ptr) return refuse(IM_ERR_INVALID, "%s: %s has a NULL pointer", what, name);
  if ((uintptr_t)v->ptr % es) return refuse(IM_ERR_INVALID, "%s: %s is not aligned to its elements", what, name);
  const int64_t st[3] = {v->batch, v->row, v->head};
  for (int i = 0; i < 3; ++i) {
    if (n[i] == 1) continue;
    if (st[i] < 0 || st[i] > (1ll << 40)) return refuse(IM_ERR_INVALID, "%s: %s has a stride outside 0..2^40", what, name);
    if (output && st[i] == 0) return refuse(IM_ERR_INVALID, "%s: %s is written and has a stride of 0", what, name);
  }
  return IM_OK;
}

// An output that starts where its input does has to be the same view: elements are read and written in no particular order.
inline int check_in_place(const char* what, const char* name, const im_view_t& in, const im_view_t& out, const int64_t (&n)[3]) {
  if (in.ptr != out.ptr || n[0] == 0 || n[1] == 0 || n[2] == 0) return IM_OK;
  if ((n[0] > 1 && in.batch != out.batch) || (n[1] > 1 && in.row != out.row) || (n[2] > 1 && in.head != out.head))
    return refuse(IM_ERR_INVALID, "%s: %s in place, the strides must be the same", what, name);
  return IM_OK;
}

// Refuses an output that starts where an input or another output does (both with elements).
struct NamedView {
  const char* name;
  const im_view_t* v;
  bool any;
};
template <size_t N, size_t M>
inline int check_apart(const char* what, const NamedView (&outs)[N], const NamedView (&ins)[M]) {
  for (size_t i = 0; i < N; ++i) {
    if (!outs[i].any) continue;
    for (size_t j = 0; j < M; ++j)
      if (ins[j].any && outs[i].v->ptr == ins[j].v->ptr) return refuse(IM_ERR_INVALID, "%s: %s overlaps %s", what, outs[i].name, ins[j].name);
    for (size_t j = 0; j < i; ++j)
      if (outs[j].any && outs[i].v->ptr == outs[j].v->ptr) return refuse(IM_ERR_INVALID, "%s: %s overlaps %s", what, outs[i].name, outs[j].name);
  }
  return IM_OK;
}

// whether every head of the view starts on a multiple of `unit` bytes and is whole units long
inline bool view_in_units(const im_view_t& v, int head_dim, size_t es, size_t unit) {
  return (uintptr_t)v.ptr % unit == 0 && head_dim * es % unit == 0 && v.batch * es % unit == 0 && v.row * es % unit == 0 && v.head * es % unit == 0;
}

// Device side: asks for every 64 bytes of a kernel's arguments (a struct by value, its only one) at once.  They would be read where they are used, one miss
// after the other, and a small call waits for each (24 rows of attention, whose arguments are 15 such lines: 13.5 -> 11.1 us).
template <class Args>
__device__ __forceinline__ void touch_args() {
  typedef const unsigned __attribute__((address_space(4))) * const_ptr;
  const_ptr p = (const_ptr)__builtin_amdgcn_kernarg_segment_ptr();
  unsigned any = 0;
#pragma unroll
  for (unsigned i = 0; i < sizeof(Args) / 4; i += 16) any |= p[i];
  asm volatile("" :: "s"(any));
}

}  // namespace imattn
