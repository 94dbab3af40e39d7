// Entry points of the attention core: validation, launch shapes, workspaces, and the two small kernels that join the parts of
// split keys and sum the slopes' gradients.  See include/imattn.h; the attention kernels are in core_attn_kernels.hpp.
#include "core_attn.hpp"

#include <math.h>
#include <string.h>

#include <algorithm>

namespace imattn {

// One wave a query row: o = sum over splits of 2^(m_s - m) o_s / sum of 2^(m_s - m) l_s.  Bound by latency: a few KB.  Sixteen splits at a time:
// every load of theirs is under way before the first is waited for; lane s holds the reference and the sum of split s.
template <class T, bool WIDE>   // WIDE: heads of more than 64 elements, two a lane
__global__ __launch_bounds__(256) void core_join_kernel(CoreArgs a) {
  const long rows = (long)a.B * a.H * a.Tq, row = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= rows) return;
  constexpr int N = 16;
  float m = -3.402823466e38f, l = 0.f, o0 = 0.f, o1 = 0.f;
  for (int s0 = 0; s0 < a.splits; s0 += N) {
    const int n = a.splits - s0 < N ? a.splits - s0 : N;
    // splits and elements behind the end: the last one again, with weight 0
    const long at = (s0 + (lane < n ? lane : n - 1)) * rows + row;
    float ms = a.part_ml[2 * at], ls = a.part_ml[2 * at + 1], v0[N], v1[WIDE ? N : 1];
#pragma unroll
    for (int s = 0; s < N; ++s) {
      const float* p = a.part_o + ((s0 + (s < n ? s : n - 1)) * rows + row) * a.dh;
      v0[s] = p[lane < a.dh ? lane : a.dh - 1];
      if constexpr (WIDE) v1[s] = p[lane + 64 < a.dh ? lane + 64 : a.dh - 1];
    }
    float to = ms;
#pragma unroll
    for (int o = N / 2; o > 0; o >>= 1) to = fmaxf(to, __shfl_xor(to, o));
    to = fmaxf(__shfl(to, 0), m);
    const float before = __builtin_amdgcn_exp2f(m - to), f = lane < n ? __builtin_amdgcn_exp2f(ms - to) : 0.f;
    m = to;
    ls *= f;
#pragma unroll
    for (int o = N / 2; o > 0; o >>= 1) ls += __shfl_xor(ls, o);
    l = l * before + __shfl(ls, 0);
    o0 *= before;
    o1 *= before;
#pragma unroll
    for (int s = 0; s < N; ++s) {
      const float fs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), s));
      o0 = fs == 0.f ? o0 : o0 + fs * v0[s];
      if constexpr (WIDE) o1 = fs == 0.f ? o1 : o1 + fs * v1[s];
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l, lse2 = l == 0.f ? IM_NEG_INF : m + log2f(l);
  const long bh = row / a.Tq, t = row - bh * a.Tq, b = bh / a.H, head = bh - b * a.H;
  T* o = (T*)a.o.ptr + b * a.o.batch + t * a.o.row + head * a.o.head;
  if (lane < a.dh) stf(o + lane, o0 * inv);
  if (lane + 64 < a.dh) stf(o + lane + 64, o1 * inv);
  if (a.o32) {
    if (lane < a.dh) a.o32[row * a.dh + lane] = o0 * inv;
    if (lane + 64 < a.dh) a.o32[row * a.dh + lane + 64] = o1 * inv;
  }
  if (lane == 0) {
    if (a.lse) a.lse[row] = lse2 * 0.69314718055994530942f;
    if (a.lse2) a.lse2[row] = lse2;
  }
}

// dslope[h] = sum over batch elements and rows of the rows' parts, one workgroup a head, in a fixed order, in fp64.  Bound by latency: eight loads
// of a thread are under way together (8 heads of 32 x 925 rows: 13.6 us with one after the other, 7.7 us).
__global__ __launch_bounds__(1024) void core_dslope_kernel(const float* __restrict__ rows, int B, int H, int Tq, float* dslope) {
  __shared__ double sums[1024];
  constexpr int N = 8;
  const int h = blockIdx.x;
  const long n = (long)B * Tq;
  const unsigned len = Tq > 0 ? Tq : 1, step_b = 1024u / len, step_t = 1024u % len;
  unsigned b = threadIdx.x / len, t = threadIdx.x % len;   // batch element and row of this thread's next part
  double s = 0.0;
  for (long i = threadIdx.x; i < n; i += 1024 * N) {
    float v[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const long at = ((long)b * H + h) * Tq + t;
      v[j] = rows[i + 1024 * j < n ? at : 0];   // (no branch: all eight are under way together)
      b += step_b;
      t += step_t;
      if (t >= len) { t -= len; ++b; }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) s += i + 1024 * j < n ? v[j] : 0.f;
  }
  sums[threadIdx.x] = s;
  __syncthreads();
  for (int o = 512; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o) sums[threadIdx.x] += sums[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) dslope[h] = (float)sums[0];
}

struct CoreLaunch {
  bool few;
  int tiles, splits;
  unsigned grid;
};

static long row_tiles(long n, int own) { return (n + own - 1) / own; }

// Shape of a launch that owns query rows (or key rows), and its groups of rows (written to *a if given).
// Neighbouring segments with the same live partners are one group -- three segments of one new token each are one tile, not three that read the
// cache three times -- unless per-sample lengths cut their ends off, or a tile across the border of two owned segments would mix the times or
// documents by which streamed tiles are skipped (`sparse`; one tile that holds both whole is still better than two).
// few: four waves to 32 rows instead of 128, where 128 rows a workgroup would leave CUs idle or half of the rows empty.  (Head dimension 128, 294
// workgroups of 128 rows: forward 148 us, in workgroups of 32 rows 301; dK/dV with 150: 507 us against 320.)
// splits (forward with few): two workgroups a CU, all at once, each with at least a tile of 32 keys for every wave.  (16 requests against 17408
// keys: 32 us; with four workgroups a CU, in two turns, 41 us.  One request of 8 heads on 2 against 4000 keys: 15.5 us, with at least four
// tiles a wave 18.5; four of head dimension 128 against 2048: 16.1 and 21.7.)
static CoreLaunch core_launch(const im_core_t* s, bool own_keys, bool may_split, bool lengths, bool sparse, CoreArgs* a) {
  CoreLaunch L = {};
  const int G = own_keys ? 1 : s->n_heads / s->n_kv_heads;
  const int32_t* own_len = own_keys ? s->k_len : s->q_len;
  const int32_t* str_len = own_keys ? s->q_len : s->k_len;
  auto live = [&](int own, int str) { return str_len[str] > 0 && ((s->live_mask >> (own_keys ? str * s->n_seg + own : own * s->n_seg + str)) & 1ull); };
  struct Group { int row0, len, seg; unsigned live; long work; } own[IM_MAX_SEG], str[IM_MAX_SEG];
  int n_own = 0, n_str = 0;
  // streamed groups: neighbours that every owned segment sees or does not see together
  for (int j = 0, row = 0; j < s->n_seg; row += str_len[j++]) {
    if (str_len[j] == 0) continue;
    bool alike = n_str > 0 && !(lengths && !own_keys);
    for (int i = 0; i < s->n_seg && alike; ++i) alike = own_len[i] == 0 || live(i, j) == live(i, str[n_str - 1].seg);
    if (alike) str[n_str - 1].len += str_len[j];
    else str[n_str++] = {row, str_len[j], j, 0u, 0};
  }
  for (int i = 0, row = 0; i < s->n_seg; row += own_len[i++]) {
    if (own_len[i] == 0) continue;
    Group g = {row, own_len[i], i, 0u, 0};
    for (int j = 0; j < n_str; ++j)
      if (live(i, str[j].seg)) { g.live |= 1u << j; g.work += str[j].len; }
    if (n_own > 0 && own[n_own - 1].live == g.live && !(lengths && own_keys) && (!sparse || ((long)own[n_own - 1].len + g.len) * G <= 32)) own[n_own - 1].len += g.len;
    else own[n_own++] = g;
  }
  const long groups = (long)s->batch * s->n_kv_heads;
  long t128 = 0, t32 = 0, most = 0;
  for (int i = 0; i < n_own; ++i) {
    t128 += row_tiles((long)own[i].len * G, 128);
    t32 += row_tiles((long)own[i].len * G, 32);
    most = std::max(most, own[i].work);
  }
  L.few = t128 * groups < cu_count() || 4 * t128 > 2 * t32;
  L.tiles = (int)(L.few ? t32 : t128);
  L.splits = 1;
  if (may_split && L.few && L.tiles > 0)
    L.splits = (int)std::max<long>(1, std::min<long>(2l * cu_count() / (L.tiles * groups), most / (4 * 32)));
  const long grid = (long)L.tiles * groups * L.splits;
  L.grid = grid < (1l << 24) ? (unsigned)grid : 0xffffffffu;
  if (a) {
    std::stable_sort(own, own + n_own, [](const Group& x, const Group& y) { return x.work > y.work; });
    a->own_groups = n_own;
    a->str_groups = n_str;
    a->tile_prefix[0] = 0;
    for (int i = 0; i < n_own; ++i) {
      a->own_row0[i] = own[i].row0; a->own_len[i] = own[i].len; a->own_seg[i] = own[i].seg; a->own_live[i] = own[i].live;
      a->tile_prefix[i + 1] = a->tile_prefix[i] + (int)row_tiles((long)own[i].len * G, L.few ? 32 : 128);
    }
    for (int j = 0; j < n_str; ++j) { a->str_row0[j] = str[j].row0; a->str_len[j] = str[j].len; a->str_seg[j] = str[j].seg; }
    a->splits = L.splits;
  }
  return L;
}

static int core_check(const char* what, const im_core_t* s) {
  if (!s) return refuse(IM_ERR_INVALID, "%s: shape is NULL", what);
  if (s->dtype != IM_DTYPE_F32 && s->dtype != IM_DTYPE_BF16) return refuse(IM_ERR_INVALID, "%s: dtype must be IM_DTYPE_F32 or IM_DTYPE_BF16 (got %d)", what, s->dtype);
  if (s->batch < 1 || s->batch > 65535) return refuse(IM_ERR_INVALID, "%s: batch must be in 1..65535 (got %d)", what, s->batch);
  if (s->n_seg < 1 || s->n_seg > IM_MAX_SEG) return refuse(IM_ERR_INVALID, "%s: n_seg must be in 1..%d (got %d)", what, IM_MAX_SEG, s->n_seg);
  if (s->n_heads < 1 || s->n_heads > 65535 || s->n_kv_heads < 1 || s->n_heads % s->n_kv_heads)
    return refuse(IM_ERR_INVALID, "%s: n_heads (%d) must be a positive multiple of n_kv_heads (%d)", what, s->n_heads, s->n_kv_heads);
  if (s->head_dim < 1) return refuse(IM_ERR_INVALID, "%s: head_dim must be >= 1 (got %d)", what, s->head_dim);
  if (s->head_dim > 128) return refuse(IM_ERR_UNSUPPORTED, "%s: head_dim must be <= 128 (got %d)", what, s->head_dim);
  long tq = 0, tk = 0;
  for (int i = 0; i < s->n_seg; ++i) {
    if (s->q_len[i] < 0 || s->k_len[i] < 0) return refuse(IM_ERR_INVALID, "%s: q_len[%d] and k_len[%d] must be >= 0", what, i, i);
    tq += s->q_len[i];
    tk += s->k_len[i];
  }
  if (tq > (1 << 24) || tk > (1 << 24) || tq * (s->n_heads / s->n_kv_heads) > (1l << 30))
    return refuse(IM_ERR_INVALID, "%s: too many rows (Tq = %ld, Tk = %ld; at most 2^24, and 2^30 query rows that share a key head)", what, tq, tk);
  const int nb = s->n_seg * s->n_seg;
  if (nb < 64 && (s->live_mask >> nb) != 0) return refuse(IM_ERR_INVALID, "%s: live_mask has bits set at or above n_seg^2 = %d", what, nb);
  if (!(s->scale >= 0.f) || isinf(s->scale)) return refuse(IM_ERR_INVALID, "%s: scale must be finite and >= 0", what);
  if (s->cap != 0.f && !(s->cap >= 0.01f && s->cap <= 1000.f)) return refuse(IM_ERR_INVALID, "%s: cap must be 0 or in 0.01..1000", what);
  for (int own_keys = 0; own_keys < 2; ++own_keys)
    if (core_launch(s, own_keys, !own_keys, true, true, nullptr).grid == 0xffffffffu)
      return refuse(IM_ERR_INVALID, "%s: problem too large (2^24 workgroups or more)", what);
  return IM_OK;
}

static int core_rules(const char* what, const im_core_t* s, const im_core_rules_t* r) {
  const im_core_rules_t none = {};
  if (!r) r = &none;
  long tq = 0, tk = 0;
  for (int i = 0; i < s->n_seg; ++i) { tq += s->q_len[i]; tk += s->k_len[i]; }
  // arrays without an element may have no address
  if ((r->slope || s->causal) && ((tq && !r->q_pos) || (tk && !r->k_pos))) return refuse(IM_ERR_INVALID, "%s: q_pos and k_pos are needed with slope or causal", what);
  if (!s->causal && r->prefix) return refuse(IM_ERR_INVALID, "%s: prefix needs causal", what);
  if (tq && tk && !r->q_doc != !r->k_doc) return refuse(IM_ERR_INVALID, "%s: q_doc and k_doc: both or neither", what);
  const uintptr_t bits = (uintptr_t)r->valid_len | (uintptr_t)r->q_pos | (uintptr_t)r->k_pos | (uintptr_t)r->slope | (uintptr_t)r->prefix | (uintptr_t)r->q_doc |
                         (uintptr_t)r->k_doc;
  if (bits % 4) return refuse(IM_ERR_INVALID, "%s: an array of the rules is not aligned to its elements", what);
  return IM_OK;
}

static void core_args(const im_core_t* s, const im_core_rules_t* r, CoreArgs* a) {
  memset(a, 0, sizeof(*a));
  a->B = s->batch; a->H = s->n_heads; a->Hkv = s->n_kv_heads; a->G = s->n_heads / s->n_kv_heads; a->dh = s->head_dim; a->n_seg = s->n_seg;
  for (int i = 0; i < s->n_seg; ++i) { a->Tq += s->q_len[i]; a->Tk += s->k_len[i]; }
  a->causal = s->causal != 0;
  a->cap = s->cap;
  if (s->scale == 0.f) a->cap = 0.f;   // every score is 0, capped or not
  // Below scale / cap = 1e-42 a cap changes nothing: no raw score exceeds 3.5e38, and tanh x = x (1 - x^2 / 3 + ..) to half a step of fp32
  // where x < 4e-4.
  if (a->cap != 0.f && (double)s->scale / s->cap < 1e-42) a->cap = 0.f;
  int n = a->cap == 0.f && s->scale > 1e38f ? 2 : 0;   // (scale * log2(e) stays finite: a score of 0 is no 0 times infinity)
  if (a->cap != 0.f) {
    double c = (double)s->scale / s->cap;
    // Coefficients in the raw score hold powers of c up to the sixth.  Where those would leave fp32 the owned rows take a power of two, exactly,
    // and c is that much closer to 1.  (At most 2^32, by which rows below 2^96 stay finite; from c = 2^48 on, where raw scores of 1e-14 are at their
    // cap, every score takes the exponential.)
    if (!(c > 1e-5 && c < 1e5)) n = std::max(-126, std::min(32, ilogb(c)));
    c = ldexp(c, -n);
    const double c2 = c * c;
    a->c_in = (float)c;
    a->inv_c_in = (float)(1.0 / c);
    const bool in = c > 1e-5 && c < 1e5;
    a->small_to = in ? (float)(0.4 / c) : 0.f;
    const double q[3] = {-0.33331882, 0.13277628, -0.0477942};
    for (int i = 0; i < 3; ++i) a->tanh_q[i] = in ? (float)(q[i] * pow(c2, i + 1)) : 0.f;
  }
  a->own_scale = ldexpf(1.f, n);
  a->to_log2 = ldexpf(s->scale, -n) * 1.44269504088896340736f;
  a->scale = s->scale;
  if (r) {
    a->valid_len = r->valid_len; a->key_pad = r->key_pad; a->slope = r->slope; a->prefix = r->prefix;
    a->q_doc = r->q_doc; a->k_doc = r->k_doc;
    if (r->slope || s->causal) { a->q_pos = r->q_pos; a->k_pos = r->k_pos; }
  }
}

// Which tensors lie in units of 16 and of 4 bytes.  Streamed ones are addressed by 32-bit byte offsets within a tile of up to 64 rows.
static void core_units(CoreArgs* a, size_t es) {
  const im_view_t* views[8] = {&a->q, &a->k, &a->v, &a->o, &a->d_o, &a->dq, &a->dk, &a->dv};
  for (int i = 0; i < 8; ++i) {
    if ((uint64_t)views[i]->row * es * 64 >= (1ull << 32)) continue;
    if (view_in_units(*views[i], a->dh, es, 16)) a->vec |= 1u << i;
    if (view_in_units(*views[i], a->dh, es, 4)) a->words |= 1u << i;
  }
}

struct CoreSizes { size_t o32, saved, part_o, fwd, stat, bwd; };
static CoreSizes core_sizes(const im_core_t* s) {
  long tq = 0;
  for (int i = 0; i < s->n_seg; ++i) tq += s->q_len[i];
  const size_t rows = (size_t)s->batch * s->n_heads * tq;
  CoreSizes z;
  z.o32 = round256(rows * s->head_dim * 4);
  z.saved = z.o32 + round256(rows * 4);
  // (documents are not known here: enough for either way of grouping)
  const int splits = std::max(core_launch(s, false, true, false, false, nullptr).splits, core_launch(s, false, true, false, true, nullptr).splits);
  z.part_o = splits > 1 ? round256(splits * rows * s->head_dim * 4) : 0;
  z.fwd = splits > 1 ? z.part_o + round256(splits * rows * 8) : 0;
  z.stat = round256(rows * 4);
  z.bwd = 2 * z.stat;
  return z;
}

static int check_buffer(const char* what, const char* name, const void* p, size_t have, size_t need) {
  if (!need) return IM_OK;
  if (!p || have < need) return refuse(IM_ERR_WORKSPACE, "%s: %s of %zu bytes, %zu needed", what, name, p ? have : (size_t)0, need);
  if ((uintptr_t)p % 16) return refuse(IM_ERR_INVALID, "%s: %s must be 16-byte aligned", what, name);
  return IM_OK;
}

}  // namespace imattn

using namespace imattn;

extern "C" {

int im_core_attention_sizes(const im_core_t* shape, size_t* saved_bytes, size_t* fwd_workspace_bytes, size_t* bwd_workspace_bytes) {
  if (int rc = core_check("im_core_attention_sizes", shape)) return rc;
  const CoreSizes z = core_sizes(shape);
  if (saved_bytes) *saved_bytes = z.saved;
  if (fwd_workspace_bytes) *fwd_workspace_bytes = z.fwd;
  if (bwd_workspace_bytes) *bwd_workspace_bytes = z.bwd;
  return IM_OK;
}

int im_core_attention_fwd(const im_core_t* shape, const im_core_rules_t* rules, const im_view_t* q, const im_view_t* k,
                          const im_view_t* v, const im_view_t* o, float* lse, void* saved, void* workspace,
                          size_t workspace_bytes, void* hip_stream) {
  const char* what = "im_core_attention_fwd";
  if (int rc = core_check(what, shape)) return rc;
  if (int rc = core_rules(what, shape, rules)) return rc;
  CoreArgs a;
  core_args(shape, rules, &a);
  const bool bf = shape->dtype == IM_DTYPE_BF16;
  const size_t es = bf ? 2 : 4;
  const int64_t nq[3] = {a.B, a.Tq, a.H}, nk[3] = {a.B, a.Tk, a.Hkv};
  if (int rc = check_view(what, "q", q, nq, es, false)) return rc;
  if (int rc = check_view(what, "k", k, nk, es, false)) return rc;
  if (int rc = check_view(what, "v", v, nk, es, false)) return rc;
  if (int rc = check_view(what, "o", o, nq, es, true)) return rc;
  if ((uintptr_t)lse % 4) return refuse(IM_ERR_INVALID, "%s: lse is not aligned to its elements", what);
  if ((uintptr_t)saved % 16) return refuse(IM_ERR_INVALID, "%s: saved must be 16-byte aligned", what);
  const CoreSizes z = core_sizes(shape);
  if (int rc = check_buffer(what, "workspace", workspace, workspace_bytes, z.fwd)) return rc;
  const NamedView outs[] = {{"o", o, a.Tq > 0}}, ins[] = {{"q", q, a.Tq > 0}, {"k", k, a.Tk > 0}, {"v", v, a.Tk > 0}};
  if (int rc = check_apart(what, outs, ins)) return rc;
  a.q = *q; a.k = *k; a.v = *v; a.o = *o; a.lse = lse;
  core_units(&a, es);
  if (saved) { a.o32 = (float*)saved; a.lse2 = (float*)((char*)saved + z.o32); }
  a.part_o = (float*)workspace; a.part_ml = (float*)((char*)workspace + z.part_o);
  const CoreLaunch L = core_launch(shape, false, true, a.valid_len != nullptr, a.causal || a.q_doc, &a);
  if (!L.grid) return IM_OK;
  if (L.grid == 0xffffffffu) return refuse(IM_ERR_INVALID, "%s: problem too large (2^24 workgroups or more)", what);
  hipStream_t st = (hipStream_t)hip_stream;
  ProfScope ps(PF_ATTN_FWD, st);
  (bf ? launch_core_fwd_bf16 : launch_core_fwd_f32)(L.few, a, L.grid, st);
  if (L.splits > 1) {
    const dim3 grid((unsigned)(((long)a.B * a.H * a.Tq + 3) / 4));
    auto join = bf ? (a.dh > 64 ? core_join_kernel<bf16_t, true> : core_join_kernel<bf16_t, false>)
                   : (a.dh > 64 ? core_join_kernel<float, true> : core_join_kernel<float, false>);
    hipLaunchKernelGGL(join, grid, dim3(256), 0, st, a);
  }
  return after_launch(what);
}

int im_core_attention_bwd(const im_core_t* shape, const im_core_rules_t* rules, const im_view_t* q, const im_view_t* k,
                          const im_view_t* v, const void* saved, const im_view_t* d_o, const im_view_t* dq,
                          const im_view_t* dk, const im_view_t* dv, float* dslope, void* workspace, size_t workspace_bytes,
                          void* hip_stream) {
  const char* what = "im_core_attention_bwd";
  if (int rc = core_check(what, shape)) return rc;
  if (int rc = core_rules(what, shape, rules)) return rc;
  CoreArgs a;
  core_args(shape, rules, &a);
  const bool bf = shape->dtype == IM_DTYPE_BF16;
  const size_t es = bf ? 2 : 4;
  const int64_t nq[3] = {a.B, a.Tq, a.H}, nk[3] = {a.B, a.Tk, a.Hkv};
  if (int rc = check_view(what, "q", q, nq, es, false)) return rc;
  if (int rc = check_view(what, "k", k, nk, es, false)) return rc;
  if (int rc = check_view(what, "v", v, nk, es, false)) return rc;
  if (int rc = check_view(what, "d_o", d_o, nq, es, false)) return rc;
  if (int rc = check_view(what, "dq", dq, nq, es, true)) return rc;
  if (int rc = check_view(what, "dk", dk, nk, es, true)) return rc;
  if (int rc = check_view(what, "dv", dv, nk, es, true)) return rc;
  if ((uintptr_t)dslope % 4) return refuse(IM_ERR_INVALID, "%s: dslope is not aligned to its elements", what);
  if (dslope && !a.slope) return refuse(IM_ERR_INVALID, "%s: dslope without slope", what);
  const CoreSizes z = core_sizes(shape);
  if (z.saved && !saved) return refuse(IM_ERR_INVALID, "%s: saved is NULL", what);
  if ((uintptr_t)saved % 16) return refuse(IM_ERR_INVALID, "%s: saved must be 16-byte aligned", what);
  if (int rc = check_buffer(what, "workspace", workspace, workspace_bytes, z.bwd)) return rc;
  const NamedView outs[] = {{"dq", dq, a.Tq > 0}, {"dk", dk, a.Tk > 0}, {"dv", dv, a.Tk > 0}};
  const NamedView ins[] = {{"q", q, a.Tq > 0}, {"k", k, a.Tk > 0}, {"v", v, a.Tk > 0}, {"d_o", d_o, a.Tq > 0}};
  if (int rc = check_apart(what, outs, ins)) return rc;
  a.q = *q; a.k = *k; a.v = *v; a.d_o = *d_o; a.dq = *dq; a.dk = *dk; a.dv = *dv;
  core_units(&a, es);
  a.o32 = (float*)saved; a.lse2 = (float*)((char*)saved + z.o32);
  a.delta = (float*)workspace;
  a.dslope_rows = dslope ? (float*)((char*)workspace + z.stat) : nullptr;
  hipStream_t st = (hipStream_t)hip_stream;
  const bool lengths = a.valid_len != nullptr, sparse = a.causal || a.q_doc;
  const CoreLaunch Lk = core_launch(shape, true, false, lengths, sparse, nullptr), Lq = core_launch(shape, false, false, lengths, sparse, &a);
  if (Lq.grid == 0xffffffffu || Lk.grid == 0xffffffffu) return refuse(IM_ERR_INVALID, "%s: problem too large (2^24 workgroups or more)", what);
  if (Lq.grid) {
    ProfScope ps(PF_ATTN_DQ, st);
    (bf ? launch_core_dq_bf16 : launch_core_dq_f32)(Lq.few, a, Lq.grid, st);
  }
  if (dslope) hipLaunchKernelGGL(core_dslope_kernel, dim3(a.H), dim3(1024), 0, st, a.dslope_rows, a.B, a.H, a.Tq, dslope);
  if (Lk.grid) {
    core_launch(shape, true, false, lengths, sparse, &a);
    ProfScope ps(PF_ATTN_DKV, st);
    (bf ? launch_core_dkv_bf16 : launch_core_dkv_f32)(Lk.few, a, Lk.grid, st);
  }
  return after_launch(what);
}

}  // extern "C"
