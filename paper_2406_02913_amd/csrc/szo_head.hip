// Log probabilities of given tokens from final states x [rows, width] and a head's weight [vocab, width], and their gradients (definition: szo.h).
//
//   logits = x W^T;   logp_t = c logits_t,target - log sum_v exp(c logits_tv)
//   d_tv = c g_t (1[v = target] - p_tv),   dx = d W,   dW = d^T x
//
// The logits stay in the registers of the tile that computes them: a tile of 256 vocabulary entries reduces them to a row's maximum and sum of exponentials (and the target's
// logit, where it has it), and a small kernel joins the tiles of a row.  The backward computes them again, turns them into d, rounded to 16 bits, and multiplies that
// twice.  d is in memory for a piece of the vocabulary at a time.  Three products of the same size, bound by the matrix cores for many rows and by one pass
// over the weight for few.
//   A head of 32000 entries of width 4096 in bf16, several cards, weight in the last-level cache to weight in memory alone: 16 rows 45 to 62 us (262 MB of weight, read at 5.8 to 4.2 TB/s), 300 rows
// 82 to 96, 4096 rows 800 to 852 (1.26 to 1.34 PFLOP/s; fp16 860).  Backward of 4096 rows 2450 to 2600 (fp16 2670): d 824 to 877 with 262 MB written, dx 742 to 793 (1.35 to 1.45 PFLOP/s), dW 819 to 869, the
// copy of x 21.  200 rows of width 2048 in fp16 149 to 166: 45, 50 and 6 for its parts, 57, 4.8 for sizes of rows, 4.1 for the copy.  A vocabulary that does not fill the chip is far from its
// bytes: 16 rows of 8000 x 4096 26 (65 MB: 13), 4 of 4000 x 8192 45.
#include <algorithm>
#include "szo_product.h"

namespace szo {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr int kTileV = 256, kThreads = 512;
constexpr size_t kPieceBytes = (size_t)256 << 20;        // of d, at most
constexpr int64_t kMostGroups = 0xFFFFFFFFll / kThreads, kMostSmallGroups = 0xFFFFFFFFll / 256;      // a launch counts its threads in 32 bits

struct HeadArgs {
  szo_head_desc d;
  int tiles_v, tiles_t;
  float2* parts;                     // [rows][tiles_v]: maximum, sum
  float* hit;                        // [rows]: the target's logit
  // backward
  int64_t first_v, piece_v;          // of this piece of the vocabulary; its columns
  int64_t pitch;                     // columns of d in memory, a multiple of 256
  int64_t rows64;                    // rows, rounded up to a multiple of 64
  uint16_t* grad;                    // d [rows64][pitch]
  const float* row_grad;             // [rows]: scale * gradient, times a factor, 0 where the target is ignored
  const float* row_back;             // [rows]: what a row of d W is multiplied by, 0 where the target is ignored
  const float* back;                 // what d^T x is
  const uint16_t* x_copy;            // x [rows64][width], rows without a target 0
  float* sums;                       // x_grad in parts [splits][rows][width]
  int splits, steps, add;            // parts of a piece, 64-wide steps of it, whether to add to what is there
  void* out;
  int64_t out_stride;
  int out_vec;
};

__device__ __forceinline__ float groups_max(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
  auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
  s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
#endif
  return v;
}
__device__ __forceinline__ float groups_sum(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
  auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
#endif
  return v;
}

// A row's gradient by its scaled logits, 0 where the target is ignored.  Both loads are asked for at once.
__device__ __forceinline__ float gradient_of(const szo_head_desc& d, const float* grad, int64_t row) {
  const int64_t t = d.targets ? d.targets[row] : -1;
  const float g = grad[row] * d.scale;
  return t >= 0 && t < d.vocab ? g : 0.f;
}

template <int TYPE>
__device__ __forceinline__ uint2 rounded4(const f32x4& v, float by) {
  typedef typename TypeOf<TYPE>::type T;
  typedef T four __attribute__((ext_vector_type(4)));
  const four h = {(T)(v[0] * by), (T)(v[1] * by), (T)(v[2] * by), (T)(v[3] * by)};
  return __builtin_bit_cast(uint2, h);
}

// Logits of a tile: vocabulary entries of [v0, v0 + BV) by rows of [t0, t0 + BT).  Tiles of 256 x 256, or of 128 entries by up to 448 rows, so that up to so many rows read the weight
// once, and more CUs do; with few rows LDS holds more steps, which is what hides the memory's latency then.
constexpr int weight_stages(int bv, int bt) { return bv == 256 ? 2 : bt == 128 ? 4 : 3; }
constexpr int row_stages(int bv, int bt) { return bv == 256 ? 2 : bt == 128 ? 4 : bt <= 256 ? 3 : 2; }          // 64 rows: two workgroups a CU
template <int TYPE, int BV, int BT> struct LogitTile : Tile<TYPE, false, false, BV, BT, 2, 4, weight_stages(BV, BT), row_stages(BV, BT)> {
  static constexpr int kWaveV = BV / 2, kWaveT = BT / 4;
};

template <int TYPE, int BV, int BT>
__device__ __forceinline__ void logits_of(LogitTile<TYPE, BV, BT>& tile, const HeadArgs& a, int64_t v0, int64_t t0, lds_at lds, int wave, int lane) {
  const szo_head_desc& d = a.d;
  const Operand w = {static_cast<const uint16_t*>(d.weight) + v0 * d.weight_stride, d.weight_stride, min((int64_t)BV, d.vocab - v0), d.width};
  const Operand x = {static_cast<const uint16_t*>(d.x) + t0 * d.x_stride, d.x_stride, min((int64_t)BT, d.rows - t0), d.width};
  tile.run(w, x, d.width / kStep, lds, wave, lane);
}

template <int TYPE, int BV, int BT>
__global__ void __launch_bounds__(kThreads, 2) head_stats_kernel(const HeadArgs a) {
  extern __shared__ __attribute__((aligned(256))) uint8_t lds[];
  typedef LogitTile<TYPE, BV, BT> L;
  const szo_head_desc& d = a.d;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wi = wave / 4, wj = wave % 4;
  int ti, tj;
  tile_of(blockIdx.x, a.tiles_v, a.tiles_t, ti, tj);
  const int64_t v0 = (int64_t)ti * BV, t0 = (int64_t)tj * BT;
  L tile;
  logits_of<TYPE, BV, BT>(tile, a, v0, t0, (lds_at)lds, wave, lane);
  __syncthreads();
  float2* const meet = reinterpret_cast<float2*>(lds);                 // [2][BT]
  const float by = d.scale * kLog2e;
  const int mine = wi * L::kWaveV + 4 * (lane >> 4);              // this lane's first entry
  const int there = (int)min((int64_t)BV, d.vocab - v0);
  int32_t targets[L::TJ];                                // all of them before the first store, which no load passes
#pragma unroll
  for (int j = 0; j < L::TJ; ++j) {
    const int64_t token = t0 + wj * L::kWaveT + 16 * j + (lane & 15);
    targets[j] = token < d.rows && d.targets ? d.targets[token] : -1;
  }
#pragma unroll
  for (int j = 0; j < L::TJ; ++j) {
    const int column = wj * L::kWaveT + 16 * j + (lane & 15);
    const int64_t token = t0 + column, target = targets[j];
    float most = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < L::TI; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (mine + 16 * i + k >= there) tile.sum[i][j][k] = -__builtin_inff();
        most = fmaxf(most, tile.sum[i][j][k]);
      }
    const int at = (int)(target - v0 - mine);
    if (target >= v0 && target < v0 + there && at >= 0 && at < 16 * L::TI && (at & 15) < 4) {
#pragma unroll
      for (int i = 0; i < L::TI; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (at == 16 * i + k) a.hit[token] = tile.sum[i][j][k];
    }
    most = groups_max(most);
    const float base = most == -__builtin_inff() ? 0.f : most;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < L::TI; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) sum += __builtin_amdgcn_exp2f((tile.sum[i][j][k] - base) * by);
    sum = groups_sum(sum);
    if (lane < 16) meet[wi * BT + column] = make_float2(most, sum);
  }
  __syncthreads();
  for (int column = threadIdx.x; column < BT; column += kThreads) {
    if (t0 + column >= d.rows) break;
    float most = -__builtin_inff(), sum = 0.f;
#pragma unroll
    for (int w = 0; w < 2; ++w) most = fmaxf(most, meet[w * BT + column].x);
    const float base = most == -__builtin_inff() ? 0.f : most;
#pragma unroll
    for (int w = 0; w < 2; ++w) sum += meet[w * BT + column].y * __builtin_amdgcn_exp2f((meet[w * BT + column].x - base) * by);
    a.parts[(t0 + column) * a.tiles_v + ti] = make_float2(most, sum);
  }
}

// A wave joins the tiles of a row.
__global__ void __launch_bounds__(256) head_join_kernel(const HeadArgs a) {
  const szo_head_desc& d = a.d;
  const int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
  const int lane = threadIdx.x & 63;
  if (row >= d.rows) return;
  const float2* parts = a.parts + row * a.tiles_v;
  const int64_t target = d.targets ? d.targets[row] : -1;       // asked for beside the parts
  const float hit = a.hit[row];                                 // nothing that counts without a target
  const float by = d.scale * kLog2e;
  float most = -__builtin_inff(), sum = 0.f;
#pragma unroll 4
  for (int i = lane; i < a.tiles_v; i += 64) {
    const float2 p = parts[i];
    const float up = fmaxf(most, p.x), base = up == -__builtin_inff() ? 0.f : up;
    sum = sum * __builtin_amdgcn_exp2f((most - base) * by) + p.y * __builtin_amdgcn_exp2f((p.x - base) * by);
    most = up;
  }
  const float top = lanes_max<64>(most), base = top == -__builtin_inff() ? 0.f : top;
  sum = lanes_sum<64>(sum * __builtin_amdgcn_exp2f((most - base) * by));
  if (lane) return;
  if (d.stats) { d.stats[2 * row] = top; d.stats[2 * row + 1] = sum; }
  if (!d.logp) return;
  float logp = 0.f;
  if (target >= 0 && target < d.vocab) logp = sum == 0.f ? -__builtin_inff() : (hit - top) * d.scale - logf(sum);
  d.logp[row] = logp;
}

// ---- backward ----------------------------------------------------------------------------------------------------------

// Factors of d.  A common one takes the largest gradient to just below a power of two, where a rounding is smallest relative to the value: most losses have one gradient for all rows, and
// d of an unlikely target is nearly that, so its rounding is the whole row's (1.004 in bf16 would be off by 2^-8, 1.98 is by half of it).  In fp16 each row has a power of two of its own
// beside it, which takes its gradient to between 2^13 and 2^14: with |1 - p| <= 1 nothing overflows, and entries of p from 2^-27 on have all their bits, however small the row's gradient is beside others.
// x_grad's rows are divided by theirs.  weight_grad adds rows up, so the copy of x that it reads is multiplied by the inverse power, and by what takes the largest state of the
// batch to below 2^15: exact but for states below 2^-28 of that, times what the row's gradient is smaller by than the largest.
constexpr int kMostSizes = 256, kMostPlaces = 120;

// Places that an fp16 row is shifted up by; `fill`: the common factor.
__device__ __forceinline__ int places_of(float g, float fill) {
  g = fabsf(g) * fill;
  return g > 0.f && g < __builtin_inff() ? min(14 - __builtin_amdgcn_frexp_expf(g), kMostPlaces) : 0;
}

// Largest gradient and state of the rows that have a finite gradient other than 0, for each workgroup.
__global__ void __launch_bounds__(1024) head_sizes_kernel(const szo_head_desc d, const float* grad, float2* sizes) {
  const uint32_t per = (uint32_t)d.width / 8, all = (uint32_t)d.rows * per;            // below 2^31
  float most = 0.f;
  uint32_t state = 0;
  for (uint32_t i = blockIdx.x * 1024 + threadIdx.x; i < all; i += gridDim.x * 1024) {
    const uint32_t row = i / per;
    const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(d.x) + (int64_t)row * d.x_stride + (i - row * per) * 8);       // beside the gradient
    const float g = fabsf(gradient_of(d, grad, row));
    if (!(g > 0.f && g < __builtin_inff())) continue;
    most = fmaxf(most, g);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t size = w[k / 2] >> (k % 2 * 16) & 0x7FFFu;
      state = max(state, size < 0x7C00u ? size : 0u);
    }
  }
  __shared__ float2 part[16];
  float x = (float)__builtin_bit_cast(_Float16, (uint16_t)state);
  most = lanes_max<64>(most);
  x = lanes_max<64>(x);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = make_float2(most, x);
  __syncthreads();
  if (threadIdx.x) return;
  for (int w = 0; w < 16; ++w) { most = fmaxf(most, part[w].x); x = fmaxf(x, part[w].y); }
  sizes[blockIdx.x] = make_float2(most, x);
}

// The first workgroup: scale * gradient of each row, times its factors, and what undoes them.  Rows without a target have no gradient, whatever the weight holds: what 0 times infinity left of
// theirs is dropped where the row is stored.  The others: the copy of x with rows that have no target as 0, which may hold anything: 0 times infinity would reach the weight's gradient.
// `count`: sizes that were found, fp16 and with weight_grad; else 0.
__global__ void __launch_bounds__(256) head_prepare_kernel(const szo_head_desc d, const float* grad, float* row_grad, float* row_back, float* back, int64_t rows64, uint16_t* x_copy,
                                                           const float2* sizes, int count) {
  __shared__ float2 part[4];
  const bool half = d.type == SZO_F16;
  float most = 0.f, state = 0.f;
  if (count > 0) {
    if ((int)threadIdx.x < count) { most = sizes[threadIdx.x].x; state = sizes[threadIdx.x].y; }
  } else if (blockIdx.x == 0) {
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < d.rows; i += 256) {
      const float g = fabsf(gradient_of(d, grad, i));
      if (g < __builtin_inff()) most = fmaxf(most, g);
    }
  }
  if (half || blockIdx.x == 0) {                         // of the whole workgroup
    most = lanes_max<64>(most);
    state = lanes_max<64>(state);
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = make_float2(most, state);
    __syncthreads();
    for (int w = 0; w < 4; ++w) { most = fmaxf(most, part[w].x); state = fmaxf(state, part[w].y); }
  }
  const float fill = most > 0.f ? 0.992f / __builtin_amdgcn_frexp_mantf(most) : 1.f;
  // fp16: d times 2^places, states times 2^(sum - places)
  const int sum = half && most > 0.f ? places_of(most, fill) + (state > 0.f ? 15 - __builtin_amdgcn_frexp_expf(state) : 0) : 0;
  if (blockIdx.x > 0) {
    const int per = d.width / 8;
    const int64_t i = (int64_t)(blockIdx.x - 1) * 256 + threadIdx.x, row = i / per, at = i % per * 8;
    if (row >= rows64) return;
    const int64_t target = row < d.rows && d.targets ? d.targets[row] : -1;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (target >= 0 && target < d.vocab) {
      v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(d.x) + row * d.x_stride + at);
      const float g = half ? fabsf(gradient_of(d, grad, row)) : 0.f;
      if (g > 0.f && g < __builtin_inff()) {
        const int by = sum - places_of(g, fill);
        f16x8 h = __builtin_bit_cast(f16x8, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) h[k] = (_Float16)__builtin_amdgcn_ldexpf((float)h[k], by);
        v = __builtin_bit_cast(uint4, h);
      }
    }
    *reinterpret_cast<uint4*>(x_copy + row * d.width + at) = v;
    return;
  }
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < d.rows; i += 256) {
    const int64_t t = d.targets ? d.targets[i] : -1;
    const float g = gradient_of(d, grad, i);
    const int by = half ? places_of(g, fill) : 0;
    row_grad[i] = __builtin_amdgcn_ldexpf(g * fill, by);
    row_back[i] = t >= 0 && t < d.vocab ? __builtin_amdgcn_ldexpf(1.f / fill, -by) : 0.f;
  }
  if (threadIdx.x == 0) *back = __builtin_amdgcn_ldexpf(1.f / fill, -sum);
}

// Rows of nothing.
__global__ void __launch_bounds__(256) head_zero_kernel(uint16_t* out, int64_t rows, int64_t stride, int width) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / width;
  if (row < rows) out[row * stride + i % width] = 0;
}

template <int TYPE, int BV, int BT>
__global__ void __launch_bounds__(kThreads, 2) head_grad_kernel(const HeadArgs a) {
  extern __shared__ __attribute__((aligned(256))) uint8_t lds[];
  typedef LogitTile<TYPE, BV, BT> L;
  const szo_head_desc& d = a.d;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wi = wave / 4, wj = wave % 4;
  int ti, tj;
  tile_of(blockIdx.x, a.tiles_v, a.tiles_t, ti, tj);
  const int64_t v0 = a.first_v + (int64_t)ti * BV, t0 = (int64_t)tj * BT;
  L tile;
  logits_of<TYPE, BV, BT>(tile, a, v0, t0, (lds_at)lds, wave, lane);
  const float by = d.scale * kLog2e;
  const int mine = wi * L::kWaveV + 4 * (lane >> 4);
  const int there = (int)min((int64_t)BV, d.vocab - v0);
  float gs[L::TJ], mosts[L::TJ], sums[L::TJ];            // all loads before the first store, which none passes
  int32_t targets[L::TJ];
#pragma unroll
  for (int j = 0; j < L::TJ; ++j) {
    const int64_t token = t0 + wj * L::kWaveT + 16 * j + (lane & 15);
    const bool in = token < d.rows;
    gs[j] = in ? a.row_grad[token] : 0.f;
    mosts[j] = in ? d.stats[2 * token] : 0.f;
    sums[j] = in ? d.stats[2 * token + 1] : 1.f;
    targets[j] = in && d.targets ? d.targets[token] : -1;
  }
#pragma unroll
  for (int j = 0; j < L::TJ; ++j) {
    const int64_t token = t0 + wj * L::kWaveT + 16 * j + (lane & 15), target = targets[j];
    if (token >= a.rows64) continue;
    const float g = gs[j], most = mosts[j], sum = sums[j];
    const bool none = target < 0 || target >= d.vocab || sum == 0.f;
    const int hit = target >= v0 && target < v0 + there ? (int)(target - v0) - mine : -1;
    const float share = g / sum;
    uint16_t* const to = a.grad + token * a.pitch + (v0 - a.first_v) + mine;
#pragma unroll
    for (int i = 0; i < L::TI; ++i) {
      f32x4 y;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float p = share * __builtin_amdgcn_exp2f((tile.sum[i][j][k] - most) * by);
        const float v = hit == 16 * i + k ? g - p : -p;
        y[k] = none || mine + 16 * i + k >= there ? 0.f : v;
      }
      *reinterpret_cast<uint2*>(to + 16 * i) = rounded4<TYPE>(y, 1.f);
    }
  }
}

// dx of a tile: features [k0, k0 + BK) by rows [t0, t0 + BT), over a part of the piece's vocabulary.
template <int TYPE, int BK, int BT>
__global__ void __launch_bounds__(kThreads, 2) head_x_grad_kernel(const HeadArgs a) {
  extern __shared__ __attribute__((aligned(256))) uint8_t lds[];
  typedef Tile<TYPE, true, false, BK, BT, 2, 4, weight_stages(BK, BT), row_stages(BK, BT)> L;
  const szo_head_desc& d = a.d;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wi = wave / 4, wj = wave % 4;
  const int tiles_k = (d.width + BK - 1) / BK, per = tiles_k * a.tiles_t, split = blockIdx.x / per;
  int ti, tj;
  tile_of(blockIdx.x - split * per, tiles_k, a.tiles_t, ti, tj);
  const int k0 = ti * BK, share = (a.steps + a.splits - 1) / a.splits, from = split * share, steps = min(share, a.steps - from);
  const int64_t t0 = (int64_t)tj * BT, r0 = (int64_t)from * kStep;
  L tile;
  if (steps > 0) {
    const Operand w = {static_cast<const uint16_t*>(d.weight) + (a.first_v + r0) * d.weight_stride + k0, d.weight_stride, d.width - k0, a.piece_v - r0};
    const Operand g = {a.grad + t0 * a.pitch + r0, a.pitch, min((int64_t)BT, a.rows64 - t0), a.pitch - r0};
    tile.run(w, g, steps, (lds_at)lds, wave, lane);
  } else {
#pragma unroll
    for (int i = 0; i < L::TI; ++i)
#pragma unroll
      for (int j = 0; j < L::TJ; ++j) tile.sum[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  float by[L::TJ];                                       // all loads before the first store
#pragma unroll
  for (int j = 0; j < L::TJ; ++j) {
    const int64_t token = t0 + wj * (BT / 4) + 16 * j + (lane & 15);
    by[j] = !a.sums && token < d.rows ? a.row_back[token] : 0.f;
  }
#pragma unroll
  for (int j = 0; j < L::TJ; ++j) {
    const int64_t token = t0 + wj * (BT / 4) + 16 * j + (lane & 15);
    if (token >= d.rows) continue;
#pragma unroll
    for (int i = 0; i < L::TI; ++i) {
      const int k = k0 + wi * (BK / 2) + 16 * i + 4 * (lane >> 4);
      if (k >= d.width) continue;
      if (a.sums) {
        float4* const to = reinterpret_cast<float4*>(a.sums + ((int64_t)split * d.rows + token) * d.width + k);
        float4 v = make_float4(tile.sum[i][j][0], tile.sum[i][j][1], tile.sum[i][j][2], tile.sum[i][j][3]);
        if (a.add) {
          const float4 had = *to;
          v.x += had.x; v.y += had.y; v.z += had.z; v.w += had.w;
        }
        *to = v;
      } else {
        uint16_t* const to = static_cast<uint16_t*>(a.out) + token * a.out_stride + k;
        const uint2 v = by[j] == 0.f ? make_uint2(0, 0) : rounded4<TYPE>(tile.sum[i][j], by[j]);
        if (a.out_vec) *reinterpret_cast<uint2*>(to) = v;
        else { to[0] = (uint16_t)v.x; to[1] = (uint16_t)(v.x >> 16); to[2] = (uint16_t)v.y; to[3] = (uint16_t)(v.y >> 16); }
      }
    }
  }
}

// The parts of dx, added up in order.
template <int TYPE>
__global__ void __launch_bounds__(256) head_x_sum_kernel(const HeadArgs a) {
  const szo_head_desc& d = a.d;
  const int per = d.width / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / per, k = i % per * 4;
  if (row >= d.rows) return;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  const float by = a.row_back[row];
#pragma unroll 4
  for (int p = 0; p < a.splits; ++p) {
    const float4 v = *reinterpret_cast<const float4*>(a.sums + ((int64_t)p * d.rows + row) * d.width + k);
    s[0] += v.x; s[1] += v.y; s[2] += v.z; s[3] += v.w;
  }
  uint16_t* const to = static_cast<uint16_t*>(a.out) + row * a.out_stride + k;
  const uint2 v = by == 0.f ? make_uint2(0, 0) : rounded4<TYPE>(s, by);
  if (a.out_vec) *reinterpret_cast<uint2*>(to) = v;
  else { to[0] = (uint16_t)v.x; to[1] = (uint16_t)(v.x >> 16); to[2] = (uint16_t)v.y; to[3] = (uint16_t)(v.y >> 16); }
}

// dW of a tile: features [k0, k0 + SIZE) by vocabulary entries [v0, v0 + SIZE) of the piece.
template <int TYPE, int SIZE>
__global__ void __launch_bounds__(kThreads, 2) head_weight_grad_kernel(const HeadArgs a) {
  extern __shared__ __attribute__((aligned(256))) uint8_t lds[];
  typedef Tile<TYPE, true, true, SIZE, SIZE, 2, 4> L;
  const szo_head_desc& d = a.d;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wi = wave / 4, wj = wave % 4;
  int ti, tj;
  tile_of(blockIdx.x, (d.width + SIZE - 1) / SIZE, a.tiles_v, ti, tj);
  const int k0 = ti * SIZE;
  const int64_t v0 = (int64_t)tj * SIZE;
  const Operand x = {a.x_copy + k0, d.width, d.width - k0, a.rows64};
  const Operand g = {a.grad + v0, a.pitch, a.pitch - v0, a.rows64};
  L tile;
  tile.run(x, g, (int)(a.rows64 / kStep), (lds_at)lds, wave, lane);
  // Through LDS, so that a row's 16-byte pieces go to memory side by side: stored as they lie, 8 bytes a lane and 32 side by side, lines reach memory in parts.
  constexpr int kPitch = SIZE * 2 + 16, kPieces = SIZE / 8;
  static_assert(SIZE * kPitch <= L::kLds, "the operands' place");
  const float by = *a.back;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < L::TJ; ++j)
#pragma unroll
    for (int i = 0; i < L::TI; ++i)
      *reinterpret_cast<uint2*>(lds + (wj * (SIZE / 4) + 16 * j + (lane & 15)) * kPitch + (wi * (SIZE / 2) + 16 * i + 4 * (lane >> 4)) * 2) = rounded4<TYPE>(tile.sum[i][j], by);
  __syncthreads();
  const int piece = threadIdx.x % kPieces, k = k0 + piece * 8;
  if (k >= d.width) return;
  const int rows = (int)min((int64_t)SIZE, a.piece_v - v0);
#pragma unroll 4
  for (int row = threadIdx.x / kPieces; row < rows; row += kThreads / kPieces) {
    const uint4 y = *reinterpret_cast<const uint4*>(lds + row * kPitch + piece * 16);
    uint16_t* const to = static_cast<uint16_t*>(a.out) + (a.first_v + v0 + row) * a.out_stride + k;
    if (a.out_vec) *reinterpret_cast<uint4*>(to) = y;
    else {
      const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int n = 0; n < 8; ++n) to[n] = (uint16_t)(w[n / 2] >> (n % 2 * 16));
    }
  }
}

// ---- host ------------------------------------------------------------------------------------------------------------

constexpr int64_t kMostStride = 1 << 22;

size_t up16(size_t n) { return (n + 15) / 16 * 16; }
int64_t tiles_of(int64_t n, int64_t size) { return (n + size - 1) / size; }
// Tiles of logits, chosen by the time of the rounds in which a CU each takes them, in units of a step of 64 of the width: a tile of 256 x 256 takes 1.33 us a step, one of 128
// entries by n rows 0.27 + 0.0026 n.  That is what a few tiles take; the whole chip at work is up to a fifth slower, all kinds alike.  us for 32000 entries of width 4096, 256 x 256 / 128 by
// 64, 128, 192, 256, 320, 384, 448: 64 rows 97 / 57, 58; 200 rows 103 / 127, 86, -, 74, 85; 300 rows 103 / -, 124, 106, -, 86, 95, 101; 600 rows 187 / -, -, 201, 187, 156, 171; 800 rows 202 / -, -, -,
// 247, 228, -, 201; 8000 entries: 300 rows 88 / -, 40, 49, -, 69, 81, 90; 1000 rows 90 / -, -, -, 64, 74, 82, 91; 2000 rows 102.
struct LogitPlan { int entries, rows; };
LogitPlan logit_plan(int64_t rows, int64_t vocab) {
  LogitPlan best = {256, 256};
  auto rounds = [&](int entries, int n) { return (double)tiles_of(tiles_of(vocab, entries) * tiles_of(rows, n), 256); };
  double least = 1.33 * rounds(256, 256);
  for (int n = 448; n >= 64; n -= 64) {
    const double us = (0.27 + 0.0026 * n) * rounds(128, n);
    if (us <= least) { least = us; best = {128, n}; }
  }
  return best;
}
// Tiles of dx by the same times, in parts of the vocabulary where they do not fill the chip; parts are stored in fp32 and added up by a second kernel (4 TB/s, 3 us).
struct GradPlan { int features, rows, splits; };
GradPlan grad_plan(int64_t rows, int64_t width, int64_t steps, bool pieces) {
  GradPlan best = {};
  double least = 1e30;
  for (int n = 512; n >= 64; n -= 64) {
    const int features = n == 512 ? 256 : 128, count = n == 512 ? 256 : n;
    const int64_t tiles = tiles_of(width, features) * tiles_of(rows, count), splits = std::max<int64_t>(1, std::min<int64_t>(256 / tiles, steps / 8));
    const double step = features == 256 ? 1.33 : 0.27 + 0.0026 * count;
    const double us = (double)tiles_of(tiles * splits, 256) * (double)tiles_of(steps, splits) * step + (splits > 1 || pieces ? 3.0 + (double)(splits * rows * width) * 8 / 4e6 : 0.0);
    if (us <= least) { least = us; best = {features, count, (int)splits}; }
  }
  return best;
}

int check(const szo_head_desc* d) {
  if (!d || d->rows < 0 || d->vocab < 0 || d->width < 0 || (d->type != SZO_BF16 && d->type != SZO_F16) || d->reserved) return SZO_EINVAL;
  if (!(d->scale > 0.f && d->scale <= SZO_MOST_SCALE)) return SZO_EINVAL;
  if (d->width == 0 || d->width % 64 || d->width > 65536 || d->vocab > (1 << 30) || d->rows > 0x7FFFFFFF) return SZO_EUNSUPPORTED;
  if (d->x_stride < 0 || d->weight_stride < 0 || (d->vocab > 1 && d->weight_stride < d->width)) return SZO_EINVAL;
  if (d->x_stride > kMostStride || d->weight_stride > kMostStride || d->x_stride % 8 || d->weight_stride % 8) return SZO_EUNSUPPORTED;
  if ((d->rows && !d->x) || (d->vocab && !d->weight) || !aligned_to(d->x, 16) || !aligned_to(d->weight, 16)) return SZO_EINVAL;
  if (!aligned_to(d->targets, 4) || !aligned_to(d->logp, 4) || !aligned_to(d->stats, 4) || !aligned_to(d->loss_acc, 8)) return SZO_EINVAL;
  if (tiles_of(d->rows, 4) > kMostSmallGroups) return SZO_EUNSUPPORTED;
  if (d->rows) {
    const LogitPlan p = logit_plan(d->rows, d->vocab);
    if (tiles_of(d->vocab, p.entries) * tiles_of(d->rows, p.rows) > kMostGroups) return SZO_EUNSUPPORTED;
  }
  return SZO_OK;
}

// A launch of a kernel whose workgroup takes `bytes` of LDS.
template <typename F, typename... Args>
int launch(F* kernel, std::atomic<uint64_t>& raised, size_t bytes, int64_t groups, hipStream_t s, const Args&... args) {
  const int rc = set_lds_limit_once(raised, (const void*)kernel, bytes);
  if (rc != SZO_OK) return rc;
  kernel<<<dim3((unsigned)groups), kThreads, bytes, s>>>(args...);
  SZO_LAUNCH_CHECK();
  return SZO_OK;
}

template <int TYPE, int BV, int BT>
int logit_launch(const HeadArgs& a, bool backward, hipStream_t s) {
  static std::atomic<uint64_t> raised[2] = {{0}, {0}};
  typedef LogitTile<TYPE, BV, BT> L;
  const int64_t groups = (int64_t)a.tiles_v * a.tiles_t;
  return backward ? launch(head_grad_kernel<TYPE, BV, BT>, raised[1], L::kLds, groups, s, a) : launch(head_stats_kernel<TYPE, BV, BT>, raised[0], L::kLds, groups, s, a);
}
// Logits of `vocab` entries.
template <int TYPE>
int logit_launch(HeadArgs a, int64_t vocab, bool backward, hipStream_t s) {
  const LogitPlan p = logit_plan(a.d.rows, vocab);
  a.tiles_v = (int)tiles_of(vocab, p.entries);
  a.tiles_t = (int)tiles_of(a.d.rows, p.rows);
  if (p.entries == 256) return logit_launch<TYPE, 256, 256>(a, backward, s);
  switch (p.rows) {
    case 64: return logit_launch<TYPE, 128, 64>(a, backward, s);
    case 128: return logit_launch<TYPE, 128, 128>(a, backward, s);
    case 192: return logit_launch<TYPE, 128, 192>(a, backward, s);
    case 256: return logit_launch<TYPE, 128, 256>(a, backward, s);
    case 320: return logit_launch<TYPE, 128, 320>(a, backward, s);
    case 384: return logit_launch<TYPE, 128, 384>(a, backward, s);
    default: return logit_launch<TYPE, 128, 448>(a, backward, s);
  }
}

template <int TYPE, int BK, int BT>
int x_grad_launch(const HeadArgs& a, hipStream_t s) {
  static std::atomic<uint64_t> raised{0};
  const int64_t groups = tiles_of(a.d.width, BK) * a.tiles_t * a.splits;
  return launch(head_x_grad_kernel<TYPE, BK, BT>, raised, Tile<TYPE, true, false, BK, BT, 2, 4, weight_stages(BK, BT), row_stages(BK, BT)>::kLds, groups, s, a);
}
template <int TYPE>
int x_grad_launch(HeadArgs a, const GradPlan& p, hipStream_t s) {
  a.tiles_t = (int)tiles_of(a.d.rows, p.rows);
  if (p.features == 256) return x_grad_launch<TYPE, 256, 256>(a, s);
  switch (p.rows) {
    case 64: return x_grad_launch<TYPE, 128, 64>(a, s);
    case 128: return x_grad_launch<TYPE, 128, 128>(a, s);
    case 192: return x_grad_launch<TYPE, 128, 192>(a, s);
    case 256: return x_grad_launch<TYPE, 128, 256>(a, s);
    case 320: return x_grad_launch<TYPE, 128, 320>(a, s);
    case 384: return x_grad_launch<TYPE, 128, 384>(a, s);
    default: return x_grad_launch<TYPE, 128, 448>(a, s);
  }
}

template <int TYPE, int SIZE>
int weight_grad_launch(HeadArgs a, hipStream_t s) {
  static std::atomic<uint64_t> raised{0};
  a.tiles_v = (int)tiles_of(a.piece_v, SIZE);
  return launch(head_weight_grad_kernel<TYPE, SIZE>, raised, Tile<TYPE, true, true, SIZE, SIZE, 2, 4>::kLds, tiles_of(a.d.width, SIZE) * a.tiles_v, s, a);
}
// Small tiles of dW where large ones would not fill the chip twice, or have a single step: two workgroups share a CU then.  us of a backward, large / small: 16 rows of 32000 x 4096 218 / 216, 200 rows
// 299 / 308, 2000 rows 1310 / 1384; 2000 x 512: 16 rows 26 / 24, 2000 rows 89 / 67.
bool small_weight_tiles(int64_t rows64, int64_t width, int64_t piece_v) { return rows64 <= 64 || tiles_of(width, 256) * tiles_of(piece_v, 256) < 512; }
template <int TYPE>
int weight_grad_launch(const HeadArgs& a, hipStream_t s) {
  return small_weight_tiles(a.rows64, a.d.width, a.piece_v) ? weight_grad_launch<TYPE, 128>(a, s) : weight_grad_launch<TYPE, 256>(a, s);
}

// A backward: columns of d that are in memory at a time, parts of dx, and where things lie in the workspace.
struct Plan {
  int64_t rows64, pitch;
  int pieces;
  GradPlan x;
  size_t grad_at, copy_at, sums_at, rows_at, row_back_at, back_at, sizes_at, bytes;
};
Plan plan_of(const szo_head_desc* d) {
  Plan p;
  p.rows64 = tiles_of(d->rows, 64) * 64;
  const int64_t all = tiles_of(d->vocab, kTileV), fit = std::max<int64_t>(1, (int64_t)(kPieceBytes / 2) / (p.rows64 * kTileV));       // tiles of columns
  p.pieces = (int)tiles_of(all, std::min(all, fit));
  p.pitch = tiles_of(all, p.pieces) * kTileV;
  p.x = grad_plan(d->rows, d->width, tiles_of(std::min(p.pitch, d->vocab), kStep), p.pieces > 1);
  size_t at = 0;
  auto take = [&](size_t n) { const size_t was = at; at = up16(at + n); return was; };
  p.grad_at = take((size_t)p.rows64 * p.pitch * 2);
  p.copy_at = take((size_t)p.rows64 * d->width * 2);
  p.sums_at = take(p.pieces > 1 || p.x.splits > 1 ? (size_t)p.x.splits * d->rows * d->width * sizeof(float) : 0);
  p.rows_at = take((size_t)d->rows * sizeof(float));
  p.row_back_at = take((size_t)d->rows * sizeof(float));
  p.back_at = take(sizeof(float));
  p.sizes_at = take(d->type == SZO_F16 ? kMostSizes * sizeof(float2) : 0);
  p.bytes = at;
  return p;
}

template <int TYPE>
int backward(HeadArgs a, const Plan& p, const float* grad_logp, void* x_grad, int64_t x_grad_stride, void* weight_grad, int64_t weight_grad_stride, char* room, hipStream_t s) {
  const szo_head_desc& d = a.d;
  const int64_t copies = weight_grad ? tiles_of(p.rows64 * (d.width / 8), 256) : 0;
  float2* const sizes = (float2*)(room + p.sizes_at);
  const int count = TYPE == SZO_F16 && weight_grad ? (int)std::min<int64_t>(kMostSizes, tiles_of(d.rows * (d.width / 8), 1024)) : 0;
  if (count) {
    head_sizes_kernel<<<dim3((unsigned)count), 1024, 0, s>>>(d, grad_logp, sizes);
    SZO_LAUNCH_CHECK();
  }
  head_prepare_kernel<<<dim3((unsigned)(1 + copies)), 256, 0, s>>>(d, grad_logp, (float*)(room + p.rows_at), (float*)(room + p.row_back_at), (float*)(room + p.back_at), p.rows64,
                                                                          (uint16_t*)(room + p.copy_at), sizes, count);
  SZO_LAUNCH_CHECK();
  a.rows64 = p.rows64;
  a.pitch = p.pitch;
  a.grad = (uint16_t*)(room + p.grad_at);
  a.row_grad = (const float*)(room + p.rows_at);
  a.row_back = (const float*)(room + p.row_back_at);
  a.back = (const float*)(room + p.back_at);
  a.x_copy = (const uint16_t*)(room + p.copy_at);
  a.splits = p.x.splits;
  float* const sums = p.pieces > 1 || p.x.splits > 1 ? (float*)(room + p.sums_at) : nullptr;
  auto vec = [](const void* q, int64_t stride) { return aligned_to(q, 16) && stride % 8 == 0; };
  int rc = SZO_OK;
  for (int piece = 0; piece < p.pieces; ++piece) {
    a.first_v = (int64_t)piece * p.pitch;
    a.piece_v = std::min(p.pitch, d.vocab - a.first_v);
    a.tiles_v = (int)tiles_of(a.piece_v, kTileV);
    a.steps = (int)tiles_of(a.piece_v, kStep);
    rc = logit_launch<TYPE>(a, a.piece_v, true, s);
    if (rc != SZO_OK) return rc;
    if (x_grad) {                            // before the weight's, which may overwrite the piece's rows of the weight
      a.out = x_grad;
      a.out_stride = x_grad_stride;
      a.out_vec = vec(x_grad, x_grad_stride);
      a.sums = sums;
      a.add = piece > 0;
      rc = x_grad_launch<TYPE>(a, p.x, s);
      if (rc != SZO_OK) return rc;
    }
    if (weight_grad) {
      a.out = weight_grad;
      a.out_stride = weight_grad_stride;
      a.out_vec = vec(weight_grad, weight_grad_stride);
      rc = weight_grad_launch<TYPE>(a, s);
      if (rc != SZO_OK) return rc;
    }
  }
  if (x_grad && sums) {
    a.sums = sums;
    a.out = x_grad;
    a.out_stride = x_grad_stride;
    a.out_vec = vec(x_grad, x_grad_stride);
    head_x_sum_kernel<TYPE><<<dim3((unsigned)tiles_of(d.rows * (d.width / 4), 256)), 256, 0, s>>>(a);
    SZO_LAUNCH_CHECK();
  }
  return SZO_OK;
}

size_t parts_bytes(const szo_head_desc* d) { return up16((size_t)d->rows * tiles_of(d->vocab, logit_plan(d->rows, d->vocab).entries) * sizeof(float2)); }

}  // namespace
}  // namespace szo

using namespace szo;

extern "C" {

size_t szo_head_workspace_bytes(const szo_head_desc* d) {
  if (check(d) != SZO_OK || d->rows == 0) return 16;
  return parts_bytes(d) + up16((size_t)d->rows * sizeof(float));
}

int szo_head_plan(const szo_head_desc* d, int32_t* plan) {
  const int rc = check(d);
  if (rc != SZO_OK) return rc;
  if (!plan) return SZO_EINVAL;
  std::fill(plan, plan + 9, 0);
  if (d->rows == 0 || d->vocab == 0) return SZO_OK;
  const Plan p = plan_of(d);
  const int64_t piece_v = std::min(p.pitch, d->vocab);
  const LogitPlan forward = logit_plan(d->rows, d->vocab), grad = logit_plan(d->rows, piece_v);
  const int32_t says[9] = {forward.entries, forward.rows, p.pieces, grad.entries, grad.rows, p.x.features, p.x.rows, p.x.splits,
                           small_weight_tiles(p.rows64, d->width, piece_v) ? 128 : 256};
  std::copy(says, says + 9, plan);
  return SZO_OK;
}

int szo_head_logprobs(const szo_head_desc* d, void* workspace, void* stream) {
  const int rc = check(d);
  if (rc != SZO_OK) return rc;
  if (d->loss_acc && !d->logp) return SZO_EINVAL;
  if (d->rows == 0) return SZO_OK;
  if (d->vocab == 0 || !workspace || !aligned_to(workspace, 16)) return SZO_EINVAL;
  hipStream_t s = (hipStream_t)stream;
  HeadArgs a = {};
  a.d = *d;
  a.tiles_v = (int)tiles_of(d->vocab, logit_plan(d->rows, d->vocab).entries);             // for the joining kernel
  a.parts = (float2*)workspace;
  a.hit = (float*)((char*)workspace + parts_bytes(d));
  const int done = d->type == SZO_BF16 ? logit_launch<SZO_BF16>(a, d->vocab, false, s) : logit_launch<SZO_F16>(a, d->vocab, false, s);
  if (done != SZO_OK) return done;
  head_join_kernel<<<dim3((unsigned)tiles_of(d->rows, 4)), 256, 0, s>>>(a);
  SZO_LAUNCH_CHECK();
  return d->loss_acc ? add_token_loss(d->logp, d->targets, d->rows, d->vocab, d->loss_scale, d->loss_acc, s) : SZO_OK;
}

size_t szo_head_bwd_workspace_bytes(const szo_head_desc* d) {
  if (check(d) != SZO_OK || d->rows == 0 || d->vocab == 0) return 16;
  return plan_of(d).bytes;
}

int szo_head_logprobs_bwd(const szo_head_desc* d, const float* grad_logp, void* x_grad, int64_t x_grad_stride, void* weight_grad, int64_t weight_grad_stride,
                          void* workspace, void* stream) {
  const int rc = check(d);
  if (rc != SZO_OK) return rc;
  if (!aligned_to(x_grad, 2) || !aligned_to(weight_grad, 2) || !aligned_to(grad_logp, 4)) return SZO_EINVAL;
  if ((x_grad && d->rows > 1 && x_grad_stride < d->width) || (weight_grad && d->vocab > 1 && weight_grad_stride < d->width)) return SZO_EINVAL;
  hipStream_t s = (hipStream_t)stream;
  if (d->rows == 0 || d->vocab == 0) {
    void* const out = d->rows ? x_grad : weight_grad;
    const int64_t rows = d->rows ? d->rows : d->vocab, stride = d->rows ? x_grad_stride : weight_grad_stride, groups = tiles_of(rows * d->width, 256);
    if (!out || rows == 0) return SZO_OK;
    if (groups > kMostSmallGroups) return SZO_EUNSUPPORTED;
    head_zero_kernel<<<dim3((unsigned)groups), 256, 0, s>>>((uint16_t*)out, rows, stride, d->width);
    SZO_LAUNCH_CHECK();
    return SZO_OK;
  }
  if (!d->stats || !grad_logp || !workspace || !aligned_to(workspace, 16)) return SZO_EINVAL;
  if (!x_grad && !weight_grad) return SZO_OK;
  if (tiles_of(tiles_of(d->rows, 64) * 64 * d->width, 4 * 256) >= kMostSmallGroups) return SZO_EUNSUPPORTED;
  HeadArgs a = {};
  a.d = *d;
  const Plan p = plan_of(d);
  if (tiles_of(d->width, p.x.features) * tiles_of(d->rows, p.x.rows) * p.x.splits > kMostGroups || tiles_of(d->width, 128) * (p.pitch / 128) > kMostGroups)
    return SZO_EUNSUPPORTED;
  return d->type == SZO_BF16 ? backward<SZO_BF16>(a, p, grad_logp, x_grad, x_grad_stride, weight_grad, weight_grad_stride, (char*)workspace, s)
                             : backward<SZO_F16>(a, p, grad_logp, x_grad, x_grad_stride, weight_grad, weight_grad_stride, (char*)workspace, s);
}

}  // extern "C"
