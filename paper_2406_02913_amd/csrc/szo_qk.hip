// Norms of queries and keys for each head with the position rotation, forward and backward.
//
//   u = x w r,  r = 1 / sqrt(mean(x^2) + eps);   out = R(position) u
//   backward, with du = R^T dout and h = x r:   dx = r (w du - h mean(w du h)),   dw = sum over tokens and heads of du h
//
// Both are bound by memory: a head's features are read once and written once, and everything between stays in registers.
// A head belongs to head_dim / 8 neighbouring lanes, 8 features each as two groups of four, chosen such that the partners
// of a rotation are in one lane: sums over a head are row permutations and the rotation exchanges nothing.  A workgroup takes
// the heads of a token, so that the token's angles are read once and stay in registers.
#include <algorithm>
#include "szo_internal.h"
#include "szo_types.h"

namespace szo {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kMostGroups = 0xFFFFFFFFll / kThreads;     // a launch counts its threads in 32 bits
constexpr int kBwdGroups = 1280;     // workgroups of a backward: what a chip holds at a time; each leaves one partial sum per feature

struct QkArgs {
  szo_qk_desc d;
  szo_qk_grads g;
  float* partials;                   // [workgroups][2][head_dim]
  int lanes_used;                    // head_dim / 8
  int tokens_per_wg, groups_per_token;
  int q_groups;                      // backward: groups of a token that take query heads; the others take key heads
};

// What a lane holds of a head: features f0..f0+3 and f1..f1+3; with the half-split rotation they are partners one by one,
// otherwise neighbours pair up.  Lanes behind the rotated features hold 8 neighbours that stay as they are.
struct LaneFeatures {
  int f0, f1, angle;                 // angle: first of the four angles
  bool on, turned;
  __device__ LaneFeatures(const szo_qk_desc& d, int lane, int lanes_used) {
    const int half = d.rot_dim / 2;
    on = lane < lanes_used;
    turned = on && 4 * lane < half;
    angle = 4 * lane;
    const bool split = turned && !d.interleaved;
    f0 = split ? 4 * lane : 8 * lane;
    f1 = split ? half + 4 * lane : 8 * lane + 4;
  }
};

struct Angles { float c[4], s[4]; };

template <bool VEC>
__device__ __forceinline__ Angles angles_of(const szo_qk_desc& d, int64_t token, const LaneFeatures& f) {
  Angles a;
#pragma unroll
  for (int i = 0; i < 4; ++i) { a.c[i] = 1.f; a.s[i] = 0.f; }
  if (f.turned) {
    const int64_t pos = d.positions[token];
    if (pos >= 0 && pos < d.table_rows) {
      const int64_t at = pos * (d.rot_dim / 2) + f.angle;
      load_f32<SZO_F32, 4, VEC>(d.cos_table, at, a.c);
      load_f32<SZO_F32, 4, VEC>(d.sin_table, at, a.s);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) a.c[i] = a.s[i] = __builtin_nanf("");
    }
  }
  return a;
}

// sign 1: the rotation, -1: its transpose.
__device__ __forceinline__ void rotate(float (&a)[4], float (&b)[4], const Angles& t, float sign, bool interleaved) {
  if (!interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = a[i], y = b[i], s = sign * t.s[i];
      a[i] = x * t.c[i] - y * s;
      b[i] = y * t.c[i] + x * s;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float x = a[2 * i], y = a[2 * i + 1], s = sign * t.s[i];
      a[2 * i] = x * t.c[i] - y * s;
      a[2 * i + 1] = y * t.c[i] + x * s;
      x = b[2 * i], y = b[2 * i + 1], s = sign * t.s[2 + i];
      b[2 * i] = x * t.c[2 + i] - y * s;
      b[2 * i + 1] = y * t.c[2 + i] + x * s;
    }
  }
}

__device__ __forceinline__ float square_sum(const float (&a)[4], const float (&b)[4]) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) { s = fmaf(a[i], a[i], s); s = fmaf(b[i], b[i], s); }
  return s;
}

template <int IN, int OUT, int L, bool VEC>
__global__ void __launch_bounds__(kThreads) qk_norm_rope_kernel(const QkArgs args) {
  const szo_qk_desc& d = args.d;
  const int lane = threadIdx.x % L, group = threadIdx.x / L;
  const int64_t token = (int64_t)blockIdx.x * args.tokens_per_wg + group / args.groups_per_token;
  if (group >= args.tokens_per_wg * args.groups_per_token || token >= d.tokens) return;
  const LaneFeatures f(d, lane, args.lanes_used);
  const Angles t = angles_of<VEC>(d, token, f);
  const int heads = d.q_heads + d.kv_heads;
  float w[2][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[0][i] = w[1][i] = 1.f;
  if (d.norm && f.on) {
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      const float* p = side ? d.k_weight : d.q_weight;
      if (!p) continue;
      float lo[4], hi[4];
      load_f32<SZO_F32, 4, VEC>(p, f.f0, lo);
      load_f32<SZO_F32, 4, VEC>(p, f.f1, hi);
#pragma unroll
      for (int i = 0; i < 4; ++i) { w[side][i] = lo[i]; w[side][4 + i] = hi[i]; }
    }
  }
  for (int h = group % args.groups_per_token; h < heads; h += args.groups_per_token) {
    const bool key = h >= d.q_heads;
    const int head = key ? h - d.q_heads : h;
    const void* x = key ? d.k : d.q;
    const int64_t from = token * (key ? d.k_token_stride : d.q_token_stride) + head * (key ? d.k_head_stride : d.q_head_stride);
    float a[4] = {0.f, 0.f, 0.f, 0.f}, b[4] = {0.f, 0.f, 0.f, 0.f};
    if (f.on) {
      load_f32<IN, 4, VEC>(x, from + f.f0, a);
      load_f32<IN, 4, VEC>(x, from + f.f1, b);
    }
    if (d.norm) {
      const float r = 1.f / sqrtf(lanes_sum<L>(square_sum(a, b)) / (float)d.head_dim + d.eps);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] = a[i] * r * (key ? w[1][i] : w[0][i]);
        b[i] = b[i] * r * (key ? w[1][4 + i] : w[0][4 + i]);
      }
    }
    rotate(a, b, t, 1.f, d.interleaved);
    if (f.on) {
      void* y = key ? d.k_out : d.q_out;
      const int64_t to = token * (key ? d.k_out_token_stride : d.q_out_token_stride) + head * (key ? d.k_out_head_stride : d.q_out_head_stride);
      store_f32<OUT, 4, VEC>(y, to + f.f0, a);
      store_f32<OUT, 4, VEC>(y, to + f.f1, b);
    }
  }
}

// A group of lanes takes query heads or key heads, never both, so that it holds one side's weights and sums.  The weights' gradients: every lane
// adds up its features over the heads and tokens of its workgroup, the workgroup adds its groups in LDS and leaves one partial per feature; a
// second kernel adds those.  No atomics, so the order is fixed.  Small workgroups, five of them on a CU
// by their registers (90; the forms of fp32 inputs with 16-bit gradients keep 8 bytes a lane in memory for it, which has not been measured against four): 4096 tokens
// of 32 + 32 heads of 128 in bf16 47 us (4.3 TB/s; a copy of 4 GB runs at 4.85), with both sides in every lane and workgroups of 1024 threads, one on a CU, 58.
template <int IN, int OUT, int L, bool VEC>
__global__ void __launch_bounds__(kThreads, 5) qk_norm_rope_bwd_kernel(const QkArgs args) {
  constexpr int kGroups = kThreads / L;
  __shared__ float sums[kGroups][8 * L + 1];
  const szo_qk_desc& d = args.d;
  const szo_qk_grads& g = args.g;
  const int lane = threadIdx.x % L, group = threadIdx.x / L, slot = group % args.groups_per_token;
  const LaneFeatures f(d, lane, args.lanes_used);
  const bool used = group < args.tokens_per_wg * args.groups_per_token, key = slot >= args.q_groups;
  const int heads = key ? d.kv_heads : d.q_heads, first_head = key ? slot - args.q_groups : slot;
  const int step = key ? args.groups_per_token - args.q_groups : args.q_groups;
  const void* x = key ? d.k : d.q;
  const void* dy = key ? g.k_out_grad : g.q_out_grad;
  void* dx = key ? g.k_grad : g.q_grad;
  const int64_t x_token = key ? d.k_token_stride : d.q_token_stride, x_head = key ? d.k_head_stride : d.q_head_stride;
  const int64_t dy_token = key ? g.k_out_token_stride : g.q_out_token_stride, dy_head = key ? g.k_out_head_stride : g.q_out_head_stride;
  const int64_t dx_token = key ? g.k_token_stride : g.q_token_stride, dx_head = key ? g.k_head_stride : g.q_head_stride;
  float w[8], dw[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { w[i] = 1.f; dw[i] = 0.f; }
  const float* weight = key ? d.k_weight : d.q_weight;
  if (d.norm && f.on && weight) {
    float lo[4], hi[4];
    load_f32<SZO_F32, 4, VEC>(weight, f.f0, lo);
    load_f32<SZO_F32, 4, VEC>(weight, f.f1, hi);
#pragma unroll
    for (int i = 0; i < 4; ++i) { w[i] = lo[i]; w[4 + i] = hi[i]; }
  }
  for (int64_t first = (int64_t)blockIdx.x * args.tokens_per_wg; first < d.tokens; first += (int64_t)gridDim.x * args.tokens_per_wg) {
    const int64_t token = first + group / args.groups_per_token;
    if (!used || token >= d.tokens) continue;
    const Angles t = angles_of<VEC>(d, token, f);
    for (int head = first_head; head < heads; head += step) {
      float a[4] = {0.f, 0.f, 0.f, 0.f}, b[4] = {0.f, 0.f, 0.f, 0.f}, u[4] = {0.f, 0.f, 0.f, 0.f}, v[4] = {0.f, 0.f, 0.f, 0.f};
      if (f.on) {
        load_f32<OUT, 4, VEC>(dy, token * dy_token + head * dy_head + f.f0, u);
        load_f32<OUT, 4, VEC>(dy, token * dy_token + head * dy_head + f.f1, v);
        if (d.norm) {
          load_f32<IN, 4, VEC>(x, token * x_token + head * x_head + f.f0, a);
          load_f32<IN, 4, VEC>(x, token * x_token + head * x_head + f.f1, b);
        }
      }
      rotate(u, v, t, -1.f, d.interleaved);
      if (d.norm) {
        const float r = 1.f / sqrtf(lanes_sum<L>(square_sum(a, b)) / (float)d.head_dim + d.eps);
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          a[i] *= r;
          b[i] *= r;
          dw[i] = fmaf(u[i], a[i], dw[i]);
          dw[4 + i] = fmaf(v[i], b[i], dw[4 + i]);
          u[i] *= w[i];
          v[i] *= w[4 + i];
          dot = fmaf(u[i], a[i], dot);
          dot = fmaf(v[i], b[i], dot);
        }
        const float mean = lanes_sum<L>(dot) / (float)d.head_dim;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u[i] = r * (u[i] - a[i] * mean);
          v[i] = r * (v[i] - b[i] * mean);
        }
      }
      if (f.on) {
        store_f32<IN, 4, VEC>(dx, token * dx_token + head * dx_head + f.f0, u);
        store_f32<IN, 4, VEC>(dx, token * dx_token + head * dx_head + f.f1, v);
      }
    }
  }
  if (!args.partials) return;
  if (f.on) {
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[group][(i < 4 ? f.f0 : f.f1) + i % 4] = dw[i];      // 0 in groups without work
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * d.head_dim; i += kThreads) {
    const int side = i / d.head_dim, at = i % d.head_dim;
    float s = 0.f;
    for (int first = 0; first < args.tokens_per_wg * args.groups_per_token; first += args.groups_per_token)
      for (int n = side ? args.q_groups : 0; n < (side ? args.groups_per_token : args.q_groups); ++n) s += sums[first + n][at];
    args.partials[(int64_t)blockIdx.x * 2 * d.head_dim + i] = s;
  }
}

// Eight features per workgroup: 128 rows of threads walk the partials, then add each other up in order.
__global__ void __launch_bounds__(1024) qk_weight_grad_kernel(const float* __restrict__ partials, float* q_weight_grad, float* k_weight_grad,
                                                              int head_dim, int count) {
  __shared__ double rows[128][9];
  const int column = threadIdx.x % 8, row = threadIdx.x / 8;
  const int i = blockIdx.x * 8 + column;                  // head_dim is a multiple of 8
  double s = 0.0;
#pragma unroll 4
  for (int p = row; p < count; p += 128) s += (double)partials[(int64_t)p * 2 * head_dim + i];
  rows[row][column] = s;
  __syncthreads();
  for (int half = 64; half; half /= 2) {
    if (row < half) rows[row][column] += rows[row + half][column];
    __syncthreads();
  }
  if (row) return;
  float* to = i < head_dim ? q_weight_grad : k_weight_grad;
  if (to) to[i % head_dim] = (float)rows[0][column];
}

// ---- host ------------------------------------------------------------------------------------------------------------

int lanes_of(int head_dim) { return head_dim <= 64 ? 8 : head_dim <= 128 ? 16 : 32; }

bool stride_ok(int64_t token, int64_t head, int heads, int head_dim) {
  return token >= 0 && head >= 0 && (heads <= 1 || head >= head_dim) && token <= (int64_t)1 << 40 && head <= (int64_t)1 << 40;
}
// Groups of four neighbours at a multiple of their size.
bool four_ok(const void* p, int64_t token, int64_t head, int type) { return aligned_to(p, 4 * type_bytes(type)) && token % 4 == 0 && head % 4 == 0; }

int check(const szo_qk_desc* d) {
  if (!d || d->tokens < 0 || d->q_heads < 0 || d->kv_heads < 0 || d->head_dim <= 0 || d->rot_dim < 0 || d->rot_dim > d->head_dim) return SZO_EINVAL;
  if (!valid_type(d->in_type) || !valid_type(d->out_type) || (d->norm & ~1) || (d->interleaved & ~1) || d->reserved || !(d->eps >= 0.f)) return SZO_EINVAL;
  if (d->head_dim % 8 || d->head_dim > 256 || d->rot_dim % 8 || d->tokens > 0x7FFFFFFF || d->q_heads > 65536 || d->kv_heads > 65536) return SZO_EUNSUPPORTED;
  if (d->tokens == 0 || d->q_heads + d->kv_heads == 0) return SZO_OK;
  if (d->rot_dim && (!d->positions || !d->cos_table || !d->sin_table || d->table_rows < 0)) return SZO_EINVAL;
  if (d->rot_dim && (!aligned_to(d->positions, 4) || !aligned_to(d->cos_table, 4) || !aligned_to(d->sin_table, 4))) return SZO_EINVAL;
  if (!aligned_to(d->q_weight, 4) || !aligned_to(d->k_weight, 4)) return SZO_EINVAL;
  if (!stride_ok(d->q_token_stride, d->q_head_stride, d->q_heads, d->head_dim) || !stride_ok(d->k_token_stride, d->k_head_stride, d->kv_heads, d->head_dim))
    return SZO_EINVAL;
  if ((d->q_heads && !aligned_to(d->q, type_bytes(d->in_type))) || (d->kv_heads && !aligned_to(d->k, type_bytes(d->in_type)))) return SZO_EINVAL;
  return SZO_OK;
}

// Rows that a call writes may not run into each other.
bool written_ok(const void* p, int64_t token, int64_t head, int heads, const szo_qk_desc* d, int type) {
  if (!heads) return true;
  return p && aligned_to(p, type_bytes(type)) && stride_ok(token, head, heads, d->head_dim) && (d->tokens <= 1 || token >= d->head_dim);
}

bool tables_vec(const szo_qk_desc* d) {
  return (!d->rot_dim || (aligned_to(d->cos_table, 16) && aligned_to(d->sin_table, 16))) && aligned_to(d->q_weight, 16) && aligned_to(d->k_weight, 16);
}

// Heads of one token to the groups of lanes of a workgroup; with few heads several tokens share one.
void share(QkArgs* a, int threads) {
  const int groups = threads / lanes_of(a->d.head_dim), heads = a->d.q_heads + a->d.kv_heads;
  a->lanes_used = a->d.head_dim / 8;
  a->groups_per_token = std::min(groups, heads);
  a->tokens_per_wg = std::max(1, groups / heads);
  // as many groups as heads, or in proportion, at least one for each side that has heads (a workgroup has eight at least)
  a->q_groups = heads <= groups ? a->d.q_heads
                                : std::min(std::max((int)((int64_t)groups * a->d.q_heads / heads), a->d.q_heads ? 1 : 0), groups - (a->d.kv_heads ? 1 : 0));
}

template <int IN, int OUT, int L, bool VEC>
void launch(const QkArgs& a, int64_t groups, bool backward, hipStream_t s) {
  if (backward) qk_norm_rope_bwd_kernel<IN, OUT, L, VEC><<<dim3((unsigned)groups), kThreads, 0, s>>>(a);
  else qk_norm_rope_kernel<IN, OUT, L, VEC><<<dim3((unsigned)groups), kThreads, 0, s>>>(a);
}
template <int IN, int OUT>
void launch_lanes(const QkArgs& a, int64_t groups, bool backward, bool vec, hipStream_t s) {
  const int L = lanes_of(a.d.head_dim);
  if (!vec) {                          // element by element: one form for all sizes would idle lanes, but shares are laid out by L
    if (L == 8) launch<IN, OUT, 8, false>(a, groups, backward, s);
    else if (L == 16) launch<IN, OUT, 16, false>(a, groups, backward, s);
    else launch<IN, OUT, 32, false>(a, groups, backward, s);
  } else if (L == 8) launch<IN, OUT, 8, true>(a, groups, backward, s);
  else if (L == 16) launch<IN, OUT, 16, true>(a, groups, backward, s);
  else launch<IN, OUT, 32, true>(a, groups, backward, s);
}
template <int IN>
void launch_out(const QkArgs& a, int64_t groups, bool backward, int out_type, bool vec, hipStream_t s) {
  if (out_type == SZO_F32) launch_lanes<IN, SZO_F32>(a, groups, backward, vec, s);
  else if (out_type == SZO_BF16) launch_lanes<IN, SZO_BF16>(a, groups, backward, vec, s);
  else launch_lanes<IN, SZO_F16>(a, groups, backward, vec, s);
}
void launch_in(const QkArgs& a, int64_t groups, bool backward, int out_type, bool vec, hipStream_t s) {
  if (a.d.in_type == SZO_F32) launch_out<SZO_F32>(a, groups, backward, out_type, vec, s);
  else if (a.d.in_type == SZO_BF16) launch_out<SZO_BF16>(a, groups, backward, out_type, vec, s);
  else launch_out<SZO_F16>(a, groups, backward, out_type, vec, s);
}

}  // namespace
}  // namespace szo

using namespace szo;

extern "C" {

int szo_qk_norm_rope(const szo_qk_desc* d, void* stream) {
  const int rc = check(d);
  if (rc != SZO_OK) return rc;
  if (d->tokens == 0 || d->q_heads + d->kv_heads == 0) return SZO_OK;
  if ((d->q_heads && !d->q) || (d->kv_heads && !d->k)) return SZO_EINVAL;
  if (!written_ok(d->q_out, d->q_out_token_stride, d->q_out_head_stride, d->q_heads, d, d->out_type) ||
      !written_ok(d->k_out, d->k_out_token_stride, d->k_out_head_stride, d->kv_heads, d, d->out_type)) return SZO_EINVAL;
  QkArgs a = {};
  a.d = *d;
  share(&a, kThreads);
  const bool vec = tables_vec(d) && (!d->q_heads || (four_ok(d->q, d->q_token_stride, d->q_head_stride, d->in_type) &&
                                                     four_ok(d->q_out, d->q_out_token_stride, d->q_out_head_stride, d->out_type))) &&
                   (!d->kv_heads || (four_ok(d->k, d->k_token_stride, d->k_head_stride, d->in_type) &&
                                     four_ok(d->k_out, d->k_out_token_stride, d->k_out_head_stride, d->out_type)));
  const int64_t groups = (d->tokens + a.tokens_per_wg - 1) / a.tokens_per_wg;
  if (groups > kMostGroups) return SZO_EUNSUPPORTED;
  launch_in(a, groups, false, d->out_type, vec, (hipStream_t)stream);
  SZO_LAUNCH_CHECK();
  return SZO_OK;
}

size_t szo_qk_workspace_bytes(const szo_qk_desc* d) {
  if (!d || d->head_dim <= 0 || d->head_dim > 256) return 0;
  return sizeof(float) * 2 * (size_t)d->head_dim * kBwdGroups;
}

int szo_qk_norm_rope_bwd(const szo_qk_desc* d, const szo_qk_grads* g, void* workspace, void* stream) {
  const int rc = check(d);
  if (rc != SZO_OK) return rc;
  if (!g || !valid_type(g->out_type) || g->reserved) return SZO_EINVAL;
  const bool weights = g->q_weight_grad || g->k_weight_grad;
  if (weights && (!d->norm || !workspace || !aligned_to(workspace, 16) || !aligned_to(g->q_weight_grad, 4) || !aligned_to(g->k_weight_grad, 4))) return SZO_EINVAL;
  hipStream_t s = (hipStream_t)stream;
  if (d->tokens == 0 || d->q_heads + d->kv_heads == 0) {
    if (g->q_weight_grad && zero_words(g->q_weight_grad, d->head_dim, s)) return SZO_ELAUNCH;
    if (g->k_weight_grad && zero_words(g->k_weight_grad, d->head_dim, s)) return SZO_ELAUNCH;
    return SZO_OK;
  }
  if (d->norm && ((d->q_heads && !d->q) || (d->kv_heads && !d->k))) return SZO_EINVAL;
  if ((d->q_heads && (!g->q_out_grad || !aligned_to(g->q_out_grad, type_bytes(g->out_type)))) ||
      (d->kv_heads && (!g->k_out_grad || !aligned_to(g->k_out_grad, type_bytes(g->out_type))))) return SZO_EINVAL;
  if (!stride_ok(g->q_out_token_stride, g->q_out_head_stride, d->q_heads, d->head_dim) ||
      !stride_ok(g->k_out_token_stride, g->k_out_head_stride, d->kv_heads, d->head_dim)) return SZO_EINVAL;
  if (!written_ok(g->q_grad, g->q_token_stride, g->q_head_stride, d->q_heads, d, d->in_type) ||
      !written_ok(g->k_grad, g->k_token_stride, g->k_head_stride, d->kv_heads, d, d->in_type)) return SZO_EINVAL;
  QkArgs a = {};
  a.d = *d;
  a.g = *g;
  a.partials = weights ? (float*)workspace : nullptr;
  share(&a, kThreads);
  const bool vec = tables_vec(d) &&
                   (!d->q_heads || (four_ok(d->q, d->q_token_stride, d->q_head_stride, d->in_type) &&
                                    four_ok(g->q_out_grad, g->q_out_token_stride, g->q_out_head_stride, g->out_type) &&
                                    four_ok(g->q_grad, g->q_token_stride, g->q_head_stride, d->in_type))) &&
                   (!d->kv_heads || (four_ok(d->k, d->k_token_stride, d->k_head_stride, d->in_type) &&
                                     four_ok(g->k_out_grad, g->k_out_token_stride, g->k_out_head_stride, g->out_type) &&
                                     four_ok(g->k_grad, g->k_token_stride, g->k_head_stride, d->in_type)));
  const int64_t all = (d->tokens + a.tokens_per_wg - 1) / a.tokens_per_wg;
  const int64_t groups = std::min<int64_t>(all, kBwdGroups);
  launch_in(a, groups, true, g->out_type, vec, s);
  SZO_LAUNCH_CHECK();
  if (weights) {
    qk_weight_grad_kernel<<<dim3(2 * d->head_dim / 8), 1024, 0, s>>>(a.partials, g->q_weight_grad, g->k_weight_grad, d->head_dim, (int)groups);
    SZO_LAUNCH_CHECK();
  }
  return SZO_OK;
}

}  // extern "C"
