// Norms after and before a block with its gate and the residual stream, forward and backward (definition: szo.h).
//
//   a = post(y),  h' = h_scale h + y_scale gate a,  x = pre(h');   a norm: unit = (v - mean) r,  r = 1 / sqrt(var + eps),  out = unit w + b
//   (RMS norms: mean 0).  Backward, with u = gx w_pre and unit of h':
//     gh' = gh_out + r (u - [mean u] - unit mean(u unit)),   dw = sum over tokens of gx unit,   db = sum of gx
//     dh = h_scale gh',   dgate = y_scale a gh',   da = y_scale gate gh',   dy from da as gh' from gx
//
// Bound by memory: a row is read once and written once, and everything between stays in registers.  A row belongs to 1 to 16 waves, eight neighbouring
// features of it to a thread (16 above 8192 features), so that a wave's loads are whole lines and a row's statistics are one exchange through LDS: the
// variance comes from each wave's own mean and squares about it, joined as sums of squares about means are, which loses nothing where the mean is large.
//   8192 tokens of 4096, block's output and stream in fp32, post norm and gate: 87 us, 5.4 TB/s of what is read and written once; all in bf16 46 (268 MB at 5.8 TB/s, part of it from the last-level
// cache).  16 tokens: 4.3, a launch.
//   Two kinds of rows keep less in registers, in the backward: above 8192 features 87 to 155 registers a thread are spilled (260 to 380 bytes of scratch), and rows whose eights are not at multiples of 16
// bytes (odd widths, strides and addresses), which are read feature by feature, spill 175 to 383 above 4096 features (0.6 to 1.3 KB).  us of 16 M features in bf16, RMS norm before the block alone / layer norms on
// both sides with biases and a shared gate: 4096 features 38 / 53, 5120 51 / 81, 8192 44 / 74, 11008 115 / 186, 16384 122 / 178; read feature by feature 4095 201 / -, 5001 600 / 949, 12345 681 / 933.  fp32 instead of
// bf16 at 4096 features - / 112, fp32 in and bf16 out - / 99.
#include <algorithm>
#include "szo_internal.h"
#include "szo_types.h"

namespace szo {
namespace {

constexpr int kMostWidth = 16384, kMostWaves = 16;
// Sums over tokens.  Those behind the post norm are of t unit and t with t = y_scale gh' (times the gate where each token has its own): a gate that all tokens share is a factor of
// the gradients by weight and bias, and its own one is weight and bias times the two sums.
constexpr int kSets = 4;
enum Set { kPreWeight, kPreBias, kPostWeight, kPostBias };

struct BlockArgs {
  szo_block_desc d;
  szo_block_grads g;
  float* partials;                   // [workgroups][sets][width]
  int set_at[kSets], sets;           // place of each sum among the partials, -1: not wanted
  int waves;                         // of a row
};

typedef uint32_t words4 __attribute__((ext_vector_type(4)));

// Eight features of a row: neighbours, or with VEC false a row's threads apart.
template <bool VEC> struct Place {
  int first, step, width;
  __device__ __forceinline__ Place() : first(0), step(0), width(0) {}
  __device__ __forceinline__ Place(int chunk, int thread, int threads, int width_)
      : first(VEC ? (chunk * threads + thread) * 8 : chunk * 8 * threads + thread), step(VEC ? 1 : threads), width(width_) {}
  __device__ __forceinline__ int at(int i) const { return first + i * step; }
  __device__ __forceinline__ bool on(int i) const { return VEC ? first < width : at(i) < width; }
};

// As they lie in memory.  Loads and conversions are apart, so that the type, which is the same for the whole launch and not worth 27 kernels, is asked for
// between them without waiting for the first of several loads.
struct Raw { words4 a, b; };

template <bool VEC>
__device__ __forceinline__ Raw fetch(const void* base, int type, int64_t row, const Place<VEC>& p) {
  Raw r = {};
  if constexpr (VEC) {
    if (base && p.first < p.width) {
      if (type == SZO_F32) {
        const char* at = static_cast<const char*>(base) + row * 4;         // the same for the wave: a lane's part of the address stays 32 bits
        r.a = *reinterpret_cast<const words4*>(at + (uint32_t)p.first * 4u);
        r.b = *reinterpret_cast<const words4*>(at + (uint32_t)p.first * 4u + 16u);
      } else {
        const char* at = static_cast<const char*>(base) + row * 2;
        r.a = *reinterpret_cast<const words4*>(at + (uint32_t)p.first * 2u);
      }
    }
  } else {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = 0.f;
      if (base && p.on(i)) {
        const int64_t at = row + p.at(i);
        v[i] = type == SZO_F32 ? static_cast<const float*>(base)[at]
                               : type == SZO_BF16 ? (float)static_cast<const __bf16*>(base)[at] : (float)static_cast<const _Float16*>(base)[at];
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) { r.a[i] = __float_as_uint(v[i]); r.b[i] = __float_as_uint(v[4 + i]); }
  }
  return r;
}

// The first and the second 16 bytes of eight features by themselves (the second ones are there in fp32 alone).
template <bool VEC>
__device__ __forceinline__ words4 fetch_first(const void* base, int type, int64_t row, const Place<VEC>& p) {
  words4 v = {};
  if (base && p.first < p.width) v = *reinterpret_cast<const words4*>(static_cast<const char*>(base) + row * (type == SZO_F32 ? 4 : 2) + (uint32_t)p.first * (type == SZO_F32 ? 4u : 2u));
  return v;
}
template <bool VEC>
__device__ __forceinline__ words4 fetch_second(const void* base, int type, int64_t row, const Place<VEC>& p) {
  words4 v = {};
  if (base && p.first < p.width && type == SZO_F32) v = *reinterpret_cast<const words4*>(static_cast<const char*>(base) + row * 4 + (uint32_t)p.first * 4u + 16u);
  return v;
}

template <bool VEC>
__device__ __forceinline__ void widen(const Raw& r, int type, float (&v)[8]) {
  if (!VEC || type == SZO_F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = __uint_as_float(r.a[i]); v[4 + i] = __uint_as_float(r.b[i]); }
  } else if (type == SZO_BF16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(r.a[i] << 16); v[2 * i + 1] = __uint_as_float(r.a[i] & 0xFFFF0000u); }
  } else {
    const f16x8 h = __builtin_bit_cast(f16x8, r.a);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)h[i];
  }
}

template <bool VEC, int TYPE>
__device__ __forceinline__ void put_as(void* base, int64_t row, const Place<VEC>& p, const float (&v)[8]) {
  if constexpr (VEC) {
    typedef typename TypeOf<TYPE>::type T;
    if (p.first < p.width) store_f32<TYPE, 8, true>(static_cast<T*>(base) + row, (int64_t)(uint32_t)p.first, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (p.on(i)) static_cast<typename TypeOf<TYPE>::type*>(base)[row + p.at(i)] = (typename TypeOf<TYPE>::type)v[i];
  }
}
template <bool VEC>
__device__ __forceinline__ void put(void* base, int type, int64_t row, const Place<VEC>& p, const float (&v)[8]) {
  if (!base) return;
  if (type == SZO_F32) put_as<VEC, SZO_F32>(base, row, p, v);
  else if (type == SZO_BF16) put_as<VEC, SZO_BF16>(base, row, p, v);
  else put_as<VEC, SZO_F16>(base, row, p, v);
}

// A weight's or bias' features; `none` where there is none.
template <bool VEC>
__device__ __forceinline__ void factor(const float* base, int64_t row, const Place<VEC>& p, float none, float (&v)[8]) {
  if (base) {
    const Raw r = fetch<VEC>(base, SZO_F32, row, p);
    widen<VEC>(r, SZO_F32, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = none;
  }
}

// Where the waves of a row meet.  Every exchange of a pass over a row has a slot of its own, and a slot is written again one row later: at least one other
// exchange, with its barrier, lies between (a kernel that makes a single exchange takes a single row).
struct Meeting {
  float (*slots)[kMostWaves][2];     // [exchange][wave]
  int waves, wave, first;            // waves of a row, this one, first one of the row
  float count;                       // features of the wave that this lane adds up for, lane modulo 16; 0: none
};

// Sum over 32 lanes, in every lane of them.
__device__ __forceinline__ float half_sum(float v) {
  v = lanes_sum<16>(v);
#if defined(__HIP_DEVICE_COMPILE__)
  const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
#endif
  return v;
}
__device__ __forceinline__ float from_lane(float v, int lane) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane)); }

// Sums of two values over a row, each in half of the lanes; sixteen lanes take a wave's each where waves meet.
__device__ __forceinline__ void row_sums(const Meeting& m, int slot, float& a, float& b) {
  float v = 0.f;
#if defined(__HIP_DEVICE_COMPILE__)
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  v = half_sum(__uint_as_float(s[0]) + __uint_as_float(s[1]));
#endif
  if (m.waves > 1) {
    const int lane = threadIdx.x % 64, other = lane % 16, half = lane / 32;
    if (lane % 32 == 0) m.slots[slot][m.first + m.wave][half] = v;
    __syncthreads();
    v = lanes_sum<16>(other < m.waves ? m.slots[slot][m.first + other][half] : 0.f);
  }
  a = from_lane(v, 0);
  b = from_lane(v, 32);
}
// Sum of one value.
__device__ __forceinline__ void row_sum(const Meeting& m, int slot, float& a) {
  a = lanes_sum<64>(a);
  if (m.waves == 1) return;
  const int lane = threadIdx.x % 64, other = lane % 16;
  if (lane == 0) m.slots[slot][m.first + m.wave][0] = a;
  __syncthreads();
  a = lanes_sum<16>(other < m.waves ? m.slots[slot][m.first + other][0] : 0.f);
}

// Mean (0 for RMS norms) and 1 / sqrt(var + eps) of a row whose places behind the end hold 0.  `own`: features of this wave.
template <int CH, bool VEC>
__device__ __forceinline__ void row_stats(const Meeting& m, int slot, const float (&v)[CH][8], const Place<VEC> (&at)[CH], bool layer, float own, float inverse_width, float eps,
                                          float& mean, float& r) {
  float square = 0.f;
  if (!layer) {
    mean = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) square = fmaf(v[c][i], v[c][i], square);
    row_sum(m, slot, square);
  } else {
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += v[c][i];
    mean = lanes_sum<64>(sum) / fmaxf(own, 1.f);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const float about = at[c].on(0) ? mean : 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = v[c][i] - (VEC ? about : at[c].on(i) ? mean : 0.f);
        square = fmaf(x, x, square);
      }
    }
    square = lanes_sum<64>(square);
    if (m.waves > 1) {
      const int lane = threadIdx.x % 64, other = lane % 16;
      if (lane == 0) { m.slots[slot][m.first + m.wave][0] = mean; m.slots[slot][m.first + m.wave][1] = square; }
      __syncthreads();
      const bool there = other < m.waves;
      const float its = there ? m.slots[slot][m.first + other][0] : 0.f, squares = there ? m.slots[slot][m.first + other][1] : 0.f;
      mean = lanes_sum<16>(m.count * its) * inverse_width;
      const float off = its - mean;
      square = lanes_sum<16>(there ? fmaf(m.count * off, off, squares) : 0.f);
    }
  }
  r = 1.f / sqrtf(square * inverse_width + eps);
}

// unit = (v - mean) r, and 0 behind the row's end
template <int CH, bool VEC>
__device__ __forceinline__ void to_unit(float (&v)[CH][8], const Place<VEC> (&at)[CH], float mean, float r) {
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const float about = at[c].on(0) ? mean : 0.f, by = at[c].on(0) ? r : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[c][i] = VEC ? (v[c][i] - about) * by : at[c].on(i) ? (v[c][i] - mean) * r : 0.f;
  }
}

// Features of a wave of a row: neighbours with VEC, else runs of 64.
template <int CH, bool VEC>
__device__ __forceinline__ float features_of(int wave, int waves, int width) {
  int n = 0;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if (VEC) n += min(max(width - (c * waves + wave) * 512, 0), 512);
    else
      for (int i = 0; i < 8; ++i) n += min(max(width - ((c * 8 + i) * waves + wave) * 64, 0), 64);
  }
  return (float)n;
}

template <int CH, bool VEC>
__device__ __forceinline__ void find_places(Place<VEC> (&p)[CH], int thread, int threads, int width) {
#pragma unroll
  for (int c = 0; c < CH; ++c) p[c] = Place<VEC>(c, thread, threads, width);
}

template <int CH, bool VEC, int THREADS, bool LAYER, bool POST>
__global__ void __launch_bounds__(THREADS) block_norm_kernel(const BlockArgs args) {
  __shared__ float slots[2][kMostWaves][2];
  const szo_block_desc& d = args.d;
  const int waves = args.waves, threads = waves * 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int row = wave / waves, thread = threadIdx.x - row * threads;
  const float inverse = 1.f / (float)d.width, own = features_of<CH, VEC>(wave - row * waves, waves, d.width);
  const Meeting m = {slots, waves, wave - row * waves, row * waves, (int)(threadIdx.x % 16) < waves ? features_of<CH, VEC>(threadIdx.x % 16, waves, d.width) : 0.f};
  const int64_t token = (int64_t)blockIdx.x * (blockDim.x / threads) + row;
  const bool there = token < d.tokens;                      // rows that are not still take part in the barriers
  Place<VEC> p[CH];
  find_places(p, thread, threads, there ? d.width : 0);
  Raw y_raw[CH], h_raw[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    y_raw[c] = fetch<VEC>(d.y, d.y_type, token * d.y_stride, p[c]);
    h_raw[c] = fetch<VEC>(d.h, d.h_type, token * d.h_stride, p[c]);
  }
  float y[CH][8], h[CH][8], w[8], b[8];
#pragma unroll
  for (int c = 0; c < CH; ++c) widen<VEC>(y_raw[c], d.y_type, y[c]);
  if (POST) {                                               // then there is a block's output
    float mean, r;
    row_stats<CH, VEC>(m, 0, y, p, LAYER, own, inverse, d.eps, mean, r);
    to_unit<CH, VEC>(y, p, mean, r);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      factor<VEC>(d.post_weight, 0, p[c], 1.f, w);
      factor<VEC>(d.post_bias, 0, p[c], 0.f, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[c][i] = fmaf(y[c][i], w[i], b[i]);
    }
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    widen<VEC>(h_raw[c], d.h_type, h[c]);
    factor<VEC>(d.gate, token * d.gate_stride, p[c], 1.f, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[c][i] = d.y ? fmaf(d.y_scale * w[i], y[c][i], d.h_scale * h[c][i]) : d.h_scale * h[c][i];
    put<VEC>(d.h_out, d.h_type, token * d.h_out_stride, p[c], h[c]);
  }
  if (!d.x_out) return;
  float mean, r;
  row_stats<CH, VEC>(m, 1, h, p, LAYER, own, inverse, d.eps, mean, r);
  to_unit<CH, VEC>(h, p, mean, r);
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    factor<VEC>(d.pre_weight, 0, p[c], 1.f, w);
    factor<VEC>(d.pre_bias, 0, p[c], 0.f, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[c][i] = fmaf(h[c][i], w[i], b[i]);
    put<VEC>(d.x_out, d.x_type, token * d.x_out_stride, p[c], h[c]);
  }
}

// Four sets of factors, 128 bytes a thread; wider rows have too many for two workgroups' LDS.
constexpr int kFactors = 4;
__host__ __device__ constexpr bool holds_factors(int ch, bool vec) { return vec && ch == 1; }

// A workgroup walks rows and keeps what it adds up over them in registers, eight features of up to four sums a thread; no atomics, so the order is fixed.
//   Bound by the memory's latency and by instructions: a row has four exchanges between its waves, and two workgroups a CU are all that the sums leave room for.  So the next row's
// first 16 bytes a thread are asked for half a row ahead, what all tokens share lies in LDS (through L2 it was 64 KiB and more a row), and the usual case of one 16-bit type has kernels
// without questions about types (SAME; -1: any types).  4096 tokens of 4096 in bf16, layer norms with biases and a shared gate: 72 us without all that, 67 with types and half of
// the loads ahead, 62 with LDS and without loads ahead, 60 with both: 201 MB and 34 MB of partial sums, written and read.
//   SAME: the type of y, h and x.
template <int CH, bool VEC, int THREADS, bool LAYER, bool POST, int SAME>
__global__ void __launch_bounds__(THREADS, THREADS == 512 && CH == 1 && VEC ? 4 : 1) block_norm_bwd_kernel(const BlockArgs args) {
  __shared__ float slots[4][kMostWaves][2];
  const szo_block_desc& d = args.d;
  const szo_block_grads& g = args.g;
  const int y_type = SAME < 0 ? d.y_type : SAME, h_type = SAME < 0 ? d.h_type : SAME, x_type = SAME < 0 ? d.x_type : SAME;
  const int waves = args.waves, threads = waves * 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int rows = blockDim.x / threads, row = wave / waves, thread = threadIdx.x - row * threads;
  const float inverse = 1.f / (float)d.width, own = features_of<CH, VEC>(wave - row * waves, waves, d.width);
  const Meeting m = {slots, waves, wave - row * waves, row * waves, (int)(threadIdx.x % 16) < waves ? features_of<CH, VEC>(threadIdx.x % 16, waves, d.width) : 0.f};
  constexpr bool kHeld = holds_factors(CH, VEC);
  extern __shared__ __attribute__((aligned(16))) float4 held[];        // [factor][2][thread], each thread's own features
  if constexpr (kHeld) {
    const Place<VEC> at(0, thread, threads, d.width);
    const float* const from[kFactors] = {d.pre_weight, d.post_weight, d.post_bias, d.gate_stride ? nullptr : d.gate};
#pragma unroll
    for (int k = 0; k < kFactors; ++k) {
      if (!from[k]) continue;
      const Raw w = fetch<VEC>(from[k], SZO_F32, 0, at);
      held[2 * k * blockDim.x + threadIdx.x] = __builtin_bit_cast(float4, w.a);
      held[(2 * k + 1) * blockDim.x + threadIdx.x] = __builtin_bit_cast(float4, w.b);
    }
  }
  auto shared_factor = [&](int k, const float* base, const Place<VEC>& at, float none, float (&v)[8]) {
    if (!kHeld || !base) return factor<VEC>(base, 0, at, none, v);
    const float4 lo = held[2 * k * blockDim.x + threadIdx.x], hi = held[(2 * k + 1) * blockDim.x + threadIdx.x];
    v[0] = lo.x; v[1] = lo.y; v[2] = lo.z; v[3] = lo.w; v[4] = hi.x; v[5] = hi.y; v[6] = hi.z; v[7] = hi.w;
  };
  auto gate_factor = [&](int64_t token, const Place<VEC>& at, float (&v)[8]) {
    if (d.gate_stride) factor<VEC>(d.gate, token * d.gate_stride, at, 1.f, v);
    else shared_factor(3, d.gate, at, 1.f, v);
  };
  float sums[kSets][CH][8];
#pragma unroll
  for (int s = 0; s < kSets; ++s)
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) sums[s][c][i] = 0.f;
  constexpr bool kEarly = VEC && CH == 1;               // rows of more have registers for no more
  words4 y_next = {}, h_next = {}, gx_next = {}, gh_next = {};
  auto early = [&](int64_t token) {
    if constexpr (kEarly) {
      const Place<VEC> q(0, thread, threads, token < d.tokens ? d.width : 0);
      y_next = fetch_first<VEC>(d.y, y_type, token * d.y_stride, q);
      h_next = fetch_first<VEC>(g.x_out_grad ? d.h : nullptr, h_type, token * d.h_stride, q);
      gx_next = fetch_first<VEC>(g.x_out_grad, x_type, token * g.x_out_stride, q);
      gh_next = fetch_first<VEC>(g.h_out_grad, h_type, token * g.h_out_stride, q);
    }
  };
  early((int64_t)blockIdx.x * rows + row);
  for (int64_t first = (int64_t)blockIdx.x * rows; first < d.tokens; first += (int64_t)gridDim.x * rows) {
    const int64_t token = first + row;
    const bool there = token < d.tokens;
    Place<VEC> p[CH];
    find_places(p, thread, threads, there ? d.width : 0);
    Raw y_raw[CH], h_raw[CH], gx_raw[CH], gh_raw[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if constexpr (kEarly) {
        y_raw[c] = Raw{y_next, fetch_second<VEC>(d.y, y_type, token * d.y_stride, p[c])};
        h_raw[c] = Raw{h_next, fetch_second<VEC>(g.x_out_grad ? d.h : nullptr, h_type, token * d.h_stride, p[c])};
      } else {
        y_raw[c] = fetch<VEC>(d.y, y_type, token * d.y_stride, p[c]);
        h_raw[c] = fetch<VEC>(g.x_out_grad ? d.h : nullptr, h_type, token * d.h_stride, p[c]);
      }
      if constexpr (kEarly) {
        gx_raw[c] = Raw{gx_next, fetch_second<VEC>(g.x_out_grad, x_type, token * g.x_out_stride, p[c])};
        gh_raw[c] = Raw{gh_next, fetch_second<VEC>(g.h_out_grad, h_type, token * g.h_out_stride, p[c])};
      } else {
        gx_raw[c] = fetch<VEC>(g.x_out_grad, x_type, token * g.x_out_stride, p[c]);
        gh_raw[c] = fetch<VEC>(g.h_out_grad, h_type, token * g.h_out_stride, p[c]);
      }
    }
    float y[CH][8], h[CH][8], gh[CH][8], gate[8], w[8], y_r = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) widen<VEC>(y_raw[c], y_type, y[c]);
    if (POST) {
      float mean;
      row_stats<CH, VEC>(m, 0, y, p, LAYER, own, inverse, d.eps, mean, y_r);
      to_unit<CH, VEC>(y, p, mean, y_r);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      widen<VEC>(h_raw[c], h_type, h[c]);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[c][i] *= d.h_scale;
      if (d.y) {
        float b[8];
        gate_factor(token, p[c], gate);
        shared_factor(1, POST ? d.post_weight : nullptr, p[c], 1.f, w);
        shared_factor(2, POST ? d.post_bias : nullptr, p[c], 0.f, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[c][i] = fmaf(d.y_scale * gate[i], fmaf(y[c][i], w[i], b[i]), h[c][i]);
      }
      widen<VEC>(gh_raw[c], h_type, gh[c]);
    }
    early(token + (int64_t)gridDim.x * rows);
    if (g.x_out_grad) {
      float u[CH][8], mean, r, sum = 0.f, dot = 0.f;
      row_stats<CH, VEC>(m, 1, h, p, LAYER, own, inverse, d.eps, mean, r);
      to_unit<CH, VEC>(h, p, mean, r);
      if (!there) r = 0.f;                                  // with eps 0 it is infinite, and nothing times it would be NaN in the sums
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float pre[8];
        widen<VEC>(gx_raw[c], x_type, u[c]);
        shared_factor(0, d.pre_weight, p[c], 1.f, pre);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          sums[kPreWeight][c][i] = fmaf(u[c][i], h[c][i], sums[kPreWeight][c][i]);
          sums[kPreBias][c][i] += u[c][i];
          u[c][i] *= pre[i];
          sum += u[c][i];
          dot = fmaf(u[c][i], h[c][i], dot);
        }
      }
      row_sums(m, 2, sum, dot);
      sum = LAYER ? sum * inverse : 0.f;
      dot *= inverse;
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) gh[c][i] = fmaf(r, fmaf(-h[c][i], dot, u[c][i] - sum), gh[c][i]);
    }
    if (g.h_grad) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float to[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) to[i] = d.h_scale * gh[c][i];
        put<VEC>(g.h_grad, h_type, token * g.h_stride, p[c], to);
      }
    }
    if (!d.y) continue;
    // from here on gh is the gradient by the norm's output, then by its input.  Gate and weight are read again: kept, they would take registers that are not there (80 -> 76 us).
    float sum = 0.f, dot = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      gate_factor(token, p[c], gate);
      shared_factor(1, POST ? d.post_weight : nullptr, p[c], 1.f, w);
      if (g.gate_grad && d.gate_stride) {
        float into[8];
        shared_factor(2, POST ? d.post_bias : nullptr, p[c], 0.f, into);
#pragma unroll
        for (int i = 0; i < 8; ++i) into[i] = d.y_scale * gh[c][i] * fmaf(y[c][i], w[i], into[i]);
        put<VEC>(g.gate_grad, SZO_F32, token * g.gate_stride, p[c], into);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float t = d.y_scale * gh[c][i];
        gh[c][i] = t * gate[i];
        const float s = d.gate_stride ? gh[c][i] : t;
        sums[kPostWeight][c][i] = fmaf(s, y[c][i], sums[kPostWeight][c][i]);
        sums[kPostBias][c][i] += s;
        if (POST) {
          gh[c][i] *= w[i];
          sum += gh[c][i];
          dot = fmaf(gh[c][i], y[c][i], dot);
        }
      }
    }
    if (POST) {
      row_sums(m, 3, sum, dot);
      sum = LAYER ? sum * inverse : 0.f;
      dot *= inverse;
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) gh[c][i] = y_r * fmaf(-y[c][i], dot, gh[c][i] - sum);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) put<VEC>(g.y_grad, y_type, token * g.y_stride, p[c], gh[c]);
  }
  if (!args.partials) return;
  float* to = args.partials + ((int64_t)blockIdx.x * rows + row) * args.sets * d.width;
  Place<VEC> whole[CH];
  find_places(whole, thread, threads, d.width);
#pragma unroll
  for (int s = 0; s < kSets; ++s)
    if (args.set_at[s] >= 0)
#pragma unroll
      for (int c = 0; c < CH; ++c) put<VEC>(to, SZO_F32, (int64_t)args.set_at[s] * d.width, whole[c], sums[s][c]);
}

// 64 neighbouring sums per workgroup: 16 rows of threads walk the partials, then add each other up in order.
__global__ void __launch_bounds__(1024) block_sums_kernel(const float* __restrict__ partials, int64_t width, int sets, int count, const BlockArgs args) {
  __shared__ double rows[16][65];
  const int column = threadIdx.x % 64, row = threadIdx.x / 64;
  const int64_t i = (int64_t)blockIdx.x * 64 + column;
  auto total = [&](int set) {
    double s = 0.0;
    if (i < width)
#pragma unroll 4
      for (int p = row; p < count; p += 16) s += (double)partials[((int64_t)p * sets + set) * width + i];
    rows[row][column] = s;
    __syncthreads();
    for (int half = 8; half; half /= 2) {
      if (row < half) rows[row][column] += rows[row + half][column];
      __syncthreads();
    }
    return rows[0][column];
  };
  const szo_block_desc& d = args.d;
  const szo_block_grads& g = args.g;
  const int set = blockIdx.y;
  const bool gate_too = set == args.set_at[kPostWeight] && g.gate_grad && d.gate_stride == 0, biased = gate_too && d.post && d.post_bias;
  const double sum = total(set);
  double by_bias = 0.0;
  if (biased) {
    __syncthreads();
    by_bias = total(args.set_at[kPostBias]);
  }
  if (row || i >= width) return;
  const double gate = d.gate && d.gate_stride == 0 ? (double)d.gate[i] : 1.0;
  if (set == args.set_at[kPreWeight]) g.pre_weight_grad[i] = (float)sum;
  else if (set == args.set_at[kPreBias]) g.pre_bias_grad[i] = (float)sum;
  else if (set == args.set_at[kPostBias]) {
    if (g.post_bias_grad) g.post_bias_grad[i] = (float)(gate * sum);
  } else {
    if (g.post_weight_grad) g.post_weight_grad[i] = (float)(gate * sum);
    if (gate_too) g.gate_grad[i] = (float)(sum * (d.post && d.post_weight ? (double)d.post_weight[i] : 1.0) + (biased ? by_bias * (double)d.post_bias[i] : 0.0));
  }
}

// ---- host ------------------------------------------------------------------------------------------------------------

constexpr int64_t kMostStride = (int64_t)1 << 40;
constexpr int64_t kMostGroups = 0xFFFFFFFFll / 1024;

// Eight features a thread up to 512 threads, sixteen beyond: with 1024 threads a thread has 128 registers, and a backward's sums alone take 32 or 64.
int chunks_of(int width) { return width <= 4096 ? 1 : 2; }
int waves_of(int width) { return (width + 512 * chunks_of(width) - 1) / (512 * chunks_of(width)); }
// Rows of a workgroup: it has 256 threads at least where rows have fewer.
int rows_of(int waves) { return waves >= 4 ? 1 : 4 / waves; }

// Workgroups of a backward: what the chip holds at a time.
int64_t bwd_groups(const szo_block_desc* d) {
  const int waves = waves_of(d->width), rows = rows_of(waves);
  const int64_t most = 256 * std::max(1, (chunks_of(d->width) == 1 ? 16 : 8) / (waves * rows));
  return std::max<int64_t>(1, std::min((d->tokens + rows - 1) / rows, most));
}

bool read_ok(const void* p, int64_t stride, int type) { return aligned_to(p, type_bytes(type)) && stride >= 0 && stride <= kMostStride; }
// Rows that a call writes may not run into each other.
bool written_ok(const void* p, int64_t stride, const szo_block_desc* d, int type) {
  return !p || (read_ok(p, stride, type) && (d->tokens <= 1 || stride >= d->width));
}
bool vec_ok(const void* p, int64_t stride, int type) { return !p || (aligned_to(p, 16) && stride % (type == SZO_F32 ? 4 : 8) == 0); }

int check(const szo_block_desc* d) {
  if (!d || d->tokens < 0 || d->width <= 0 || !valid_type(d->y_type) || !valid_type(d->h_type) || !valid_type(d->x_type)) return SZO_EINVAL;
  if ((d->norm != SZO_NORM_RMS && d->norm != SZO_NORM_LAYER) || (d->post & ~1) || d->reserved || !(d->eps >= 0.f)) return SZO_EINVAL;
  if (d->width > kMostWidth) return SZO_EUNSUPPORTED;
  if (d->tokens > 0 && !d->y && !d->h) return SZO_EINVAL;
  if (!read_ok(d->y, d->y_stride, d->y_type) || !read_ok(d->h, d->h_stride, d->h_type) || !read_ok(d->gate, d->gate_stride, SZO_F32)) return SZO_EINVAL;
  if (!aligned_to(d->post_weight, 4) || !aligned_to(d->post_bias, 4) || !aligned_to(d->pre_weight, 4) || !aligned_to(d->pre_bias, 4)) return SZO_EINVAL;
  if (d->tokens > 0 && !d->y && d->gate) return SZO_EINVAL;              // an empty batch may have no addresses
  return SZO_OK;
}

bool inputs_vec(const szo_block_desc* d) {
  return d->width % 8 == 0 && vec_ok(d->y, d->y_stride, d->y_type) && vec_ok(d->h, d->h_stride, d->h_type) && vec_ok(d->gate, d->gate_stride, SZO_F32) &&
         aligned_to(d->post_weight, 16) && aligned_to(d->post_bias, 16) && aligned_to(d->pre_weight, 16) && aligned_to(d->pre_bias, 16);
}

template <int CH, bool VEC, int THREADS, bool LAYER, bool POST, int SAME>
int launch_backward(const BlockArgs& a, int64_t groups, int threads, hipStream_t s) {
  static std::atomic<uint64_t> raised{0};
  const size_t lds = holds_factors(CH, VEC) ? (size_t)threads * kFactors * 2 * sizeof(float4) : 0;
  if (lds > 48 * 1024) {
    const int rc = set_lds_limit_once(raised, (const void*)block_norm_bwd_kernel<CH, VEC, THREADS, LAYER, POST, SAME>, lds);
    if (rc != SZO_OK) return rc;
  }
  block_norm_bwd_kernel<CH, VEC, THREADS, LAYER, POST, SAME><<<dim3((unsigned)groups), threads, lds, s>>>(a);
  SZO_LAUNCH_CHECK();
  return SZO_OK;
}
template <int CH, bool VEC, int THREADS, bool LAYER, bool POST>
int launch(const BlockArgs& a, int64_t groups, bool backward, hipStream_t s) {
  const int threads = 64 * a.waves * rows_of(a.waves);
  if (backward) {
    if constexpr (VEC) {
      const bool same = a.d.y_type == a.d.h_type && a.d.h_type == a.d.x_type;
      if (same && a.d.h_type == SZO_BF16) return launch_backward<CH, VEC, THREADS, LAYER, POST, SZO_BF16>(a, groups, threads, s);
      if (same && a.d.h_type == SZO_F16) return launch_backward<CH, VEC, THREADS, LAYER, POST, SZO_F16>(a, groups, threads, s);
    }
    return launch_backward<CH, VEC, THREADS, LAYER, POST, -1>(a, groups, threads, s);
  }
  block_norm_kernel<CH, VEC, THREADS, LAYER, POST><<<dim3((unsigned)groups), threads, 0, s>>>(a);
  SZO_LAUNCH_CHECK();
  return SZO_OK;
}
template <int CH, bool VEC, int THREADS>
int launch_norm(const BlockArgs& a, int64_t groups, bool backward, hipStream_t s) {
  const bool layer = a.d.norm == SZO_NORM_LAYER, post = a.d.y && a.d.post;
  if (layer) return post ? launch<CH, VEC, THREADS, true, true>(a, groups, backward, s) : launch<CH, VEC, THREADS, true, false>(a, groups, backward, s);
  return post ? launch<CH, VEC, THREADS, false, true>(a, groups, backward, s) : launch<CH, VEC, THREADS, false, false>(a, groups, backward, s);
}
template <bool VEC>
int launch_all(const BlockArgs& a, int64_t groups, bool backward, hipStream_t s) {
  if (a.d.width <= 4096) return launch_norm<1, VEC, 512>(a, groups, backward, s);
  if (a.d.width <= 8192) return launch_norm<2, VEC, 512>(a, groups, backward, s);
  return launch_norm<2, VEC, 1024>(a, groups, backward, s);
}

}  // namespace
}  // namespace szo

using namespace szo;

extern "C" {

int szo_block_norm(const szo_block_desc* d, void* stream) {
  const int rc = check(d);
  if (rc != SZO_OK) return rc;
  if (!written_ok(d->h_out, d->h_out_stride, d, d->h_type) || !written_ok(d->x_out, d->x_out_stride, d, d->x_type)) return SZO_EINVAL;
  if (d->tokens == 0 || (!d->h_out && !d->x_out)) return SZO_OK;
  BlockArgs a = {};
  a.d = *d;
  a.waves = waves_of(d->width);
  const int rows = rows_of(a.waves);
  const int64_t groups = (d->tokens - 1) / rows + 1;
  if (groups > kMostGroups) return SZO_EUNSUPPORTED;
  const bool vec = inputs_vec(d) && vec_ok(d->h_out, d->h_out_stride, d->h_type) && vec_ok(d->x_out, d->x_out_stride, d->x_type);
  return vec ? launch_all<true>(a, groups, false, (hipStream_t)stream) : launch_all<false>(a, groups, false, (hipStream_t)stream);
}

size_t szo_block_workspace_bytes(const szo_block_desc* d) {
  if (check(d) != SZO_OK || d->tokens == 0) return 16;
  return sizeof(float) * kSets * (size_t)d->width * (size_t)(bwd_groups(d) * rows_of(waves_of(d->width)));
}

int szo_block_norm_bwd(const szo_block_desc* d, const szo_block_grads* g, void* workspace, void* stream) {
  const int rc = check(d);
  if (rc != SZO_OK) return rc;
  if (!g || g->reserved) return SZO_EINVAL;
  if (!read_ok(g->x_out_grad, g->x_out_stride, d->x_type) || !read_ok(g->h_out_grad, g->h_out_stride, d->h_type)) return SZO_EINVAL;
  if (!written_ok(g->y_grad, g->y_stride, d, d->y_type) || !written_ok(g->h_grad, g->h_stride, d, d->h_type)) return SZO_EINVAL;
  if (!aligned_to(g->gate_grad, 4) || (d->gate_stride && !written_ok(g->gate_grad, g->gate_stride, d, SZO_F32))) return SZO_EINVAL;
  if (!aligned_to(g->pre_weight_grad, 4) || !aligned_to(g->pre_bias_grad, 4) || !aligned_to(g->post_weight_grad, 4) || !aligned_to(g->post_bias_grad, 4))
    return SZO_EINVAL;
  // a gradient of what has no part in the result is a mistake of the caller's, not zero
  if (d->tokens > 0 && ((!d->y && g->y_grad) || (!d->h && g->h_grad) || (!d->gate && g->gate_grad) ||
                        ((!d->y || !d->post) && (g->post_weight_grad || g->post_bias_grad)))) return SZO_EINVAL;
  BlockArgs a = {};
  a.d = *d;
  a.g = *g;
  a.waves = waves_of(d->width);
  float* const by_gate = d->gate_stride ? nullptr : g->gate_grad;         // a sum over tokens too
  const bool wanted[kSets] = {g->pre_weight_grad != nullptr, g->pre_bias_grad != nullptr, g->post_weight_grad || by_gate, g->post_bias_grad || (by_gate && d->post && d->post_bias)};
  for (int k = 0; k < kSets; ++k) a.set_at[k] = wanted[k] ? a.sets++ : -1;
  if (a.sets && (!workspace || !aligned_to(workspace, 16))) return SZO_EINVAL;
  hipStream_t s = (hipStream_t)stream;
  if (d->tokens == 0) {
    for (float* sums : {g->pre_weight_grad, g->pre_bias_grad, g->post_weight_grad, g->post_bias_grad, by_gate})
      if (sums && zero_words(sums, d->width, s)) return SZO_ELAUNCH;
    return SZO_OK;
  }
  a.partials = a.sets ? (float*)workspace : nullptr;
  const bool vec = inputs_vec(d) && vec_ok(g->x_out_grad, g->x_out_stride, d->x_type) && vec_ok(g->h_out_grad, g->h_out_stride, d->h_type) &&
                   vec_ok(g->y_grad, g->y_stride, d->y_type) && vec_ok(g->h_grad, g->h_stride, d->h_type) &&
                   (!d->gate_stride || vec_ok(g->gate_grad, g->gate_stride, SZO_F32));
  const int64_t groups = bwd_groups(d);
  const int done = vec ? launch_all<true>(a, groups, true, s) : launch_all<false>(a, groups, true, s);
  if (done != SZO_OK) return done;
  if (a.sets) {
    block_sums_kernel<<<dim3((unsigned)((d->width + 63) / 64), (unsigned)a.sets), 1024, 0, s>>>(a.partials, d->width, a.sets, (int)groups * rows_of(a.waves), a);
    SZO_LAUNCH_CHECK();
  }
  return SZO_OK;
}

}  // extern "C"
