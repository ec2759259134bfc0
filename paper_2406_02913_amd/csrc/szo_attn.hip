// Attention over a key/value cache in 8 bits (layout: szo.h).
//
//   s = scale q k,  p = exp(s) where the query sees the key,  out = sum p v / sum p,  in one pass with a running maximum.
//
// A wave takes 32 query rows (a token's query heads of one key head are rows too: they share its keys) and walks blocks of 32 cached
// tokens.  It computes S^T = K Q^T and O^T = V^T P^T in products of 32x32x16: in the result of the first a lane has one query row and 16 of
// the 32 tokens, which is just what the second takes as an operand, so the weights never leave their lane, and the row's maximum is
// one lane exchange away.  The cache is laid out as the two left operands: 16 bytes of a lane are its codes for two products.
//   Numbers: codes are exact in bf16 and fp16.  Keys' exponents go into the factor of the scores.  Values' exponents go into the exponent of the
// weights: with x = log2(e) s + v_exp the running maximum is over x, sum 2^(x - m) code is the output's numerator and
// sum 2^(x - m) 2^-v_exp the denominator, so that the weights, rounded to fp16, are relative to the largest contribution of the row.
#include <algorithm>
#include "szo_internal.h"
#include "szo_kv.h"

namespace szo {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr float kNone = -1e30f;            // running maximum of a row that has seen nothing
constexpr float kSlack = 8.f;              // the maximum may fall behind by this many binary places before sums are scaled: weights up to 2^8 fit fp16

struct AttnArgs {
  szo_attn_desc d;
  int group, blocks_per_page;              // query heads per key head
  int tiles, splits, rows_cap;             // row tiles of a workgroup, parts of the cache, rows kept per wave tile in partial sums
  float to_log2;                           // scale * log2(e)
  float* partial;                          // [sequence][key head][wave tile][split][rows_cap][head_dim + 2]
  bool vec_q, vec_out;
};

struct Rows {
  int n, start, length, first;             // queries of the sequence, its first row of q, its length, first row of the wave's 32
  int count;                               // rows of the sequence for this key head
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

template <int D> struct Raw { uint4 w[D / 32]; };

template <int D>
__device__ __forceinline__ Raw<D> load_block(const uint8_t* codes, int64_t block, int lane) {
  Raw<D> r;
  const uint4* p = reinterpret_cast<const uint4*>(codes + block * (D * kKvBlock)) + (lane % 32) * 2 + lane / 32;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) r.w[i] = p[i * 64];
  return r;
}

template <int TYPE> struct Half;
template <> struct Half<SZO_BF16> {
  typedef bf16x8 vec;
  static __device__ __forceinline__ vec codes(uint32_t lo, uint32_t hi) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return vec{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  }
  static __device__ __forceinline__ f32x16 product(vec a, vec b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Half<SZO_F16> {
  typedef f16x8 vec;
  static __device__ __forceinline__ vec codes(uint32_t lo, uint32_t hi) {
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
    const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
    return vec{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  }
  static __device__ __forceinline__ f32x16 product(vec a, vec b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

// max and sum of a value and its other half's (lane +- 32)
__device__ __forceinline__ float halves_max(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
#endif
  return v;
}
__device__ __forceinline__ float halves_sum(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
#endif
  return v;
}

// 0x80 in each byte of w that is the code of NaN
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

// WR waves side by side over rows, WK = 4 / WR over the cache.
template <int TYPE, int D, int WR>
__global__ void __launch_bounds__(kThreads, D <= 128 ? 2 : 1) attn_cached_kernel(const AttnArgs a) {
  typedef Half<TYPE> H;
  typedef typename H::vec vec;
  constexpr int WK = kWaves / WR, E = D / 32;
  const szo_attn_desc& d = a.d;
  const int lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64), column = lane % 32, half = lane / 32;
  // key heads vary fastest: workgroups are dealt out to the 8 XCDs in turn, so the row tiles of one key head share an L2
  int id = blockIdx.x;
  const int head = id % d.cache.kv_heads;
  id /= d.cache.kv_heads;
  const int split = id % a.splits;
  id /= a.splits;
  const int tile = a.tiles - 1 - id % a.tiles, sequence = id / a.tiles;    // later rows see more: they start first
  const int wave_tile = tile * WR + wave % WR, walker = wave / WR;
  const int start = max(d.q_start[sequence], 0), stop = (int)min((int64_t)d.q_start[sequence + 1], d.tokens);
  const int n = max(0, min(stop - start, d.max_q));
  const int length = (int)max((int64_t)0, min((int64_t)d.cache.lengths[sequence], (int64_t)d.cache.max_pages * d.cache.page_tokens));
  const int whole = d.cache.lengths[sequence], rows = n * a.group, first_row = wave_tile * 32;
  if (tile * WR * 32 >= rows) return;                    // the workgroup as a whole
  const bool active = first_row < rows;

  // this lane's row
  const int row = first_row + column, query = row / a.group, q_head = head * a.group + row % a.group;
  const bool valid = row < rows;
  const int behind = whole - (stop - start);             // position of the sequence's first query
  const int position = behind + query;
  const int see_to = !valid ? 0 : d.causal ? min(length, position + 1) : length;
  const int see_from = d.window > 0 ? position - d.window + 1 : 0;

  vec q[E][2];
  if (active) {
    const int64_t at = (int64_t)(start + query) * d.q_token_stride + (int64_t)q_head * d.q_head_stride;
#pragma unroll
    for (int s = 0; s < E; ++s)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        vec x = {};
        if (valid) {
          const auto* p = static_cast<const typename TypeOf<TYPE>::type*>(d.q) + at + 32 * s + 16 * half + 8 * u;
          if (a.vec_q) x = *reinterpret_cast<const vec*>(p);
          else
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = p[i];
        }
        q[s][u] = x;
      }
  }

  // blocks that some row of the wave's tile sees, the part of them that is this split's, and this wave's share of that
  const int pos_first = behind + first_row / a.group, pos_last = behind + (min(first_row + 32, rows) - 1) / a.group;
  const int reach = d.causal ? min(length, pos_last + 1) : length;
  const int lo = d.window > 0 ? max(0, pos_first - d.window + 1) / kKvBlock : 0, hi = active && reach > 0 ? (reach + kKvBlock - 1) / kKvBlock : 0;
  const int share = (max(hi - lo, 0) + a.splits - 1) / a.splits;
  const int j0 = lo + split * share + walker, j1 = min(hi, lo + (split + 1) * share);
  const int see_all = d.causal ? min(length, pos_first + 1) : length;     // tokens before this one are seen by every row, but for the window
  const int see_all_from = d.window > 0 ? pos_last - d.window + 1 : 0;

  f32x16 o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = f32x16{};
  float m = kNone, l = 0.f;

  int64_t block = j0 < j1 ? block_of(d.cache, sequence, j0, head, a.blocks_per_page) : -1;
  Raw<D> k;
  if (block >= 0) k = load_block<D>(d.cache.k, block, lane);
  for (int j = j0; j < j1; j += WK) {
    const int64_t next = j + WK < j1 ? block_of(d.cache, sequence, j + WK, head, a.blocks_per_page) : -1;
    if (block >= 0) {
      Raw<D> v = load_block<D>(d.cache.v, block, lane);
      const int ke = (int)d.cache.k_exp[block] - kExpBias, ve = (int)d.cache.v_exp[block] - kExpBias;
      f32x16 s = {};
#pragma unroll
      for (int i = 0; i < E; ++i) {
        s = H::product(H::codes(k.w[i].x, k.w[i].y), q[i][0], s);
        s = H::product(H::codes(k.w[i].z, k.w[i].w), q[i][1], s);
      }
      if (next >= 0) k = load_block<D>(d.cache.k, next, lane);
      const float factor = a.to_log2 * power_of_two(min(max(ke, kExpMin), kExpMax)), shift = (float)min(max(ve, kExpMin), kExpMax);
      const float unshift = power_of_two(-min(max(ve, kExpMin), kExpMax));
      float x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = fmaf(s[i], factor, shift);
      const int token = j * kKvBlock + 4 * half;           // of x[0]; x[i] is 8 (i / 4) + i % 4 further
      const bool all = (j + 1) * kKvBlock <= see_all && j * kKvBlock >= see_all_from;
      if (!all) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int t = token + 8 * (i / 4) + i % 4;
          x[i] = t < see_to && t >= see_from ? x[i] : -__builtin_inff();
        }
      }
      float most = x[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) most = fmaxf(most, x[i]);
      most = halves_max(most);
      if (__any(most > m + kSlack)) {
        const float to = fmaxf(m, most), scale = exp2f(m - to);
        m = to;
        l *= scale;
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[e][i] *= scale;
      }
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) { x[i] = __builtin_amdgcn_exp2f(x[i] - m); sum += x[i]; }
      l = fmaf(sum, unshift, l);
      f16x8 p[2];
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i / 8][i % 8] = (_Float16)x[i];
      if (!all) {
        // A masked token's weight is 0, and 0 times NaN would be NaN: such codes are taken out, and the rows that do see them get their NaN
        uint32_t bad = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) bad |= nan_codes(v.w[e].x) | nan_codes(v.w[e].y) | nan_codes(v.w[e].z) | nan_codes(v.w[e].w);
        if (__any(bad != 0)) {
          f16x8 seen[2];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int t = token + 8 * (i / 4) + i % 4;
            seen[i / 8][i % 8] = t < see_to && t >= see_from ? (_Float16)1.f : (_Float16)0.f;
          }
#pragma unroll
          for (int e = 0; e < E; ++e) {
            uint32_t w[4] = {v.w[e].x, v.w[e].y, v.w[e].z, v.w[e].w}, mark[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const uint32_t ones = nan_codes(w[c]) >> 7;
              w[c] &= ~(ones * 0xFFu);
              mark[c] = ones * 0x38u;                      // the code of 1
            }
            v.w[e] = make_uint4(w[0], w[1], w[2], w[3]);
            f32x16 hits = {};
            hits = Half<SZO_F16>::product(Half<SZO_F16>::codes(mark[0], mark[1]), seen[0], hits);
            hits = Half<SZO_F16>::product(Half<SZO_F16>::codes(mark[2], mark[3]), seen[1], hits);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[e][i] = hits[i] > 0.f ? __builtin_nanf("") : o[e][i];
          }
        }
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        o[e] = Half<SZO_F16>::product(Half<SZO_F16>::codes(v.w[e].x, v.w[e].y), p[0], o[e]);
        o[e] = Half<SZO_F16>::product(Half<SZO_F16>::codes(v.w[e].z, v.w[e].w), p[1], o[e]);
      }
    } else if (next >= 0) {
      k = load_block<D>(d.cache.k, next, lane);
    }
    block = next;
  }
  l = halves_sum(l);

  if constexpr (WK > 1) {
    // the walkers' sums meet in the first one's registers
    extern __shared__ __attribute__((aligned(16))) float meet[];
    constexpr int kPer = 64 * (D / 2 + 2);
    if (walker > 0) {
      float* to = meet + ((walker - 1) * WR + wave % WR) * kPer;
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<float4*>(to + (e * 4 + i / 4) * 256 + lane * 4) = make_float4(o[e][i], o[e][i + 1], o[e][i + 2], o[e][i + 3]);
      to[D / 2 * 64 + lane] = m;
      to[D / 2 * 64 + 64 + lane] = l;
    }
    __syncthreads();
    if (walker > 0) return;
    float top = m;
#pragma unroll
    for (int w = 1; w < WK; ++w) top = fmaxf(top, meet[((w - 1) * WR + wave % WR) * kPer + D / 2 * 64 + lane]);
    const float scale = exp2f(m - top);
    l *= scale;
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[e][i] *= scale;
#pragma unroll
    for (int w = 1; w < WK; ++w) {
      const float* from = meet + ((w - 1) * WR + wave % WR) * kPer;
      const float part = exp2f(from[D / 2 * 64 + lane] - top);
      l = fmaf(from[D / 2 * 64 + 64 + lane], part, l);
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const float4 x = *reinterpret_cast<const float4*>(from + (e * 4 + i / 4) * 256 + lane * 4);
          o[e][i] = fmaf(x.x, part, o[e][i]);
          o[e][i + 1] = fmaf(x.y, part, o[e][i + 1]);
          o[e][i + 2] = fmaf(x.z, part, o[e][i + 2]);
          o[e][i + 3] = fmaf(x.w, part, o[e][i + 3]);
        }
    }
    m = top;
  }
  if (!valid) return;

  if (a.splits > 1) {
    const int64_t tiles = (int64_t)a.tiles * WR;
    float* to = a.partial + ((((int64_t)sequence * d.cache.kv_heads + head) * tiles + wave_tile) * a.splits + split) * a.rows_cap * (D + 2);
    float* mine = to + (int64_t)column * D;
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<float4*>(mine + 32 * e + 2 * i + 4 * half) = make_float4(o[e][i], o[e][i + 1], o[e][i + 2], o[e][i + 3]);
    if (half == 0) {
      to[(int64_t)a.rows_cap * D + 2 * column] = m;
      to[(int64_t)a.rows_cap * D + 2 * column + 1] = l;
    }
    return;
  }
  const float by = l == 0.f ? 0.f : 1.f / l;
  const int64_t at = (int64_t)(start + query) * d.out_token_stride + (int64_t)q_head * d.out_head_stride;
#pragma unroll
  for (int e = 0; e < E; ++e)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const float y[4] = {o[e][i] * by, o[e][i + 1] * by, o[e][i + 2] * by, o[e][i + 3] * by};
      if (a.vec_out) store_f32<TYPE, 4, true>(d.out, at + 32 * e + 2 * i + 4 * half, y);
      else store_f32<TYPE, 4, false>(d.out, at + 32 * e + 2 * i + 4 * half, y);
    }
  if (d.lse && half == 0)
    d.lse[(int64_t)(start + query) * d.q_heads + q_head] = l == 0.f ? -__builtin_inff() : (m + __log2f(l)) * 0.693147180559945309f;
}

// Joins the parts of a row: one workgroup per sequence, key head and wave tile, D / 4 lanes a row.
template <int TYPE, int D>
__global__ void __launch_bounds__(kThreads) attn_join_kernel(const AttnArgs a, int wave_tiles) {
  const szo_attn_desc& d = a.d;
  int64_t id = blockIdx.x;
  const float* from = a.partial + id * a.splits * a.rows_cap * (D + 2);
  const int wave_tile = (int)(id % wave_tiles);
  id /= wave_tiles;
  const int head = (int)(id % d.cache.kv_heads), sequence = (int)(id / d.cache.kv_heads);
  const int start = max(d.q_start[sequence], 0), stop = (int)min((int64_t)d.q_start[sequence + 1], d.tokens);
  const int rows = min(max(0, min(stop - start, d.max_q)) * a.group - wave_tile * 32, 32);
  for (int i = threadIdx.x; i < rows * (D / 4); i += kThreads) {
    const int column = i / (D / 4), f = i % (D / 4) * 4, row = wave_tile * 32 + column, query = row / a.group, q_head = head * a.group + row % a.group;
    float m = kNone, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.splits; ++s) {
      const float* part = from + (int64_t)s * a.rows_cap * (D + 2);
      const float ms = part[(int64_t)a.rows_cap * D + 2 * column], ls = part[(int64_t)a.rows_cap * D + 2 * column + 1];
      const float4 x = *reinterpret_cast<const float4*>(part + (int64_t)column * D + f);
      const float top = fmaxf(m, ms), keep = exp2f(m - top), add = exp2f(ms - top);
      m = top;
      l = l * keep + ls * add;
      o[0] = o[0] * keep + x.x * add;
      o[1] = o[1] * keep + x.y * add;
      o[2] = o[2] * keep + x.z * add;
      o[3] = o[3] * keep + x.w * add;
    }
    const float by = l == 0.f ? 0.f : 1.f / l;
    const float y[4] = {o[0] * by, o[1] * by, o[2] * by, o[3] * by};
    const int64_t at = (int64_t)(start + query) * d.out_token_stride + (int64_t)q_head * d.out_head_stride + f;
    if (a.vec_out) store_f32<TYPE, 4, true>(d.out, at, y);
    else store_f32<TYPE, 4, false>(d.out, at, y);
    if (d.lse && f == 0)
      d.lse[(int64_t)(start + query) * d.q_heads + q_head] = l == 0.f ? -__builtin_inff() : (m + __log2f(l)) * 0.693147180559945309f;
  }
}

// ---- host ------------------------------------------------------------------------------------------------------------

struct Plan { int wr, tiles, splits, rows_cap; };

Plan plan_of(const szo_attn_desc* d) {
  Plan p;
  const int64_t rows = (int64_t)d->max_q * (d->q_heads / d->cache.kv_heads);
  p.wr = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
  p.tiles = (int)((rows + 32 * p.wr - 1) / (32 * p.wr));
  p.rows_cap = (int)std::min<int64_t>(32, rows);
  const int64_t base = (int64_t)d->cache.sequences * d->cache.kv_heads * p.tiles;
  const int64_t blocks = ((int64_t)std::max(d->max_len, 1) + kKvBlock - 1) / kKvBlock;
  const int64_t most = std::max<int64_t>(1, blocks / (kWaves / p.wr));
  p.splits = (int)std::min<int64_t>(std::max<int64_t>(1, 512 / base), std::min<int64_t>(most, 64));
  return p;
}

int check(const szo_attn_desc* d) {
  if (!d) return SZO_EINVAL;
  const int rc = check_cache(&d->cache);
  if (rc != SZO_OK) return rc;
  const szo_kv_cache& c = d->cache;
  if ((d->type != SZO_BF16 && d->type != SZO_F16) || (d->causal & ~1) || d->reserved || d->q_heads < 0 || d->window < 0 || d->max_q < 0 || d->max_len < 0 ||
      d->tokens < 0) return SZO_EINVAL;
  if (!(d->scale > -3.4e38f && d->scale < 3.4e38f)) return SZO_EINVAL;
  if (d->tokens > 0x7FFFFFFF) return SZO_EUNSUPPORTED;
  if (c.kv_heads == 0 ? d->q_heads != 0 : d->q_heads % c.kv_heads != 0) return SZO_EINVAL;
  if (c.sequences == 0 || d->q_heads == 0 || d->tokens == 0 || d->max_q == 0) return SZO_OK;
  if (!d->q || !d->out || !d->q_start || !aligned_to(d->q_start, 4) || !aligned_to(d->q, 2) || !aligned_to(d->out, 2) || !aligned_to(d->lse, 4)) return SZO_EINVAL;
  if (!c.lengths || !c.page_table) return SZO_EINVAL;
  if (d->q_token_stride < 0 || d->q_head_stride < 0 || (d->tokens > 1 && d->out_token_stride < c.head_dim) || (d->q_heads > 1 && d->out_head_stride < c.head_dim))
    return SZO_EINVAL;
  if ((int64_t)d->max_q * (d->q_heads / c.kv_heads) > 0x3FFFFFFF) return SZO_EUNSUPPORTED;
  const Plan p = plan_of(d);
  if ((int64_t)c.sequences * c.kv_heads * p.tiles * p.wr * p.splits > 0x7FFFFFFF) return SZO_EUNSUPPORTED;
  return SZO_OK;
}
bool nothing(const szo_attn_desc* d) { return d->cache.sequences == 0 || d->q_heads == 0 || d->tokens == 0 || d->max_q == 0; }

template <int TYPE, int D, int WR>
int launch(const AttnArgs& a, int64_t groups, hipStream_t s) {
  constexpr size_t lds = WR == kWaves ? 0 : (size_t)(kWaves - WR) * 64 * (D / 2 + 2) * sizeof(float);
  static std::atomic<uint64_t> raised{0};
  if (lds > 64 * 1024) {
    const int rc = set_lds_limit_once(raised, (const void*)attn_cached_kernel<TYPE, D, WR>, lds);
    if (rc != SZO_OK) return rc;
  }
  attn_cached_kernel<TYPE, D, WR><<<dim3((unsigned)groups), kThreads, lds, s>>>(a);
  SZO_LAUNCH_CHECK();
  return SZO_OK;
}

template <int TYPE, int D>
int launch_all(const AttnArgs& a, const Plan& p, hipStream_t s) {
  const int64_t groups = (int64_t)a.d.cache.sequences * a.d.cache.kv_heads * p.tiles * p.splits;
  const int rc = p.wr == 1 ? launch<TYPE, D, 1>(a, groups, s) : p.wr == 2 ? launch<TYPE, D, 2>(a, groups, s) : launch<TYPE, D, 4>(a, groups, s);
  if (rc != SZO_OK || p.splits == 1) return rc;
  attn_join_kernel<TYPE, D><<<dim3((unsigned)(groups / p.splits * p.wr)), kThreads, 0, s>>>(a, p.tiles * p.wr);
  SZO_LAUNCH_CHECK();
  return SZO_OK;
}

template <int TYPE>
int launch_dim(const AttnArgs& a, const Plan& p, hipStream_t s) {
  switch (a.d.cache.head_dim) {
    case 64: return launch_all<TYPE, 64>(a, p, s);
    case 96: return launch_all<TYPE, 96>(a, p, s);
    case 128: return launch_all<TYPE, 128>(a, p, s);
    default: return launch_all<TYPE, 256>(a, p, s);
  }
}

}  // namespace
}  // namespace szo

using namespace szo;

extern "C" {

size_t szo_attn_workspace_bytes(const szo_attn_desc* d) {
  if (check(d) != SZO_OK || nothing(d)) return 16;
  const Plan p = plan_of(d);
  if (p.splits == 1) return 16;
  return (size_t)d->cache.sequences * d->cache.kv_heads * p.tiles * p.wr * p.splits * p.rows_cap * (d->cache.head_dim + 2) * sizeof(float);
}

int szo_attn_cached(const szo_attn_desc* d, void* workspace, void* stream) {
  const int rc = check(d);
  if (rc != SZO_OK) return rc;
  if (nothing(d)) return SZO_OK;
  const Plan p = plan_of(d);
  if (p.splits > 1 && (!workspace || !aligned_to(workspace, 16))) return SZO_EINVAL;
  AttnArgs a = {};
  a.d = *d;
  a.group = d->q_heads / d->cache.kv_heads;
  a.blocks_per_page = d->cache.page_tokens / kKvBlock;
  a.tiles = p.tiles;
  a.splits = p.splits;
  a.rows_cap = p.rows_cap;
  a.to_log2 = d->scale * 1.44269504088896341f;
  a.partial = (float*)workspace;
  a.vec_q = aligned_to(d->q, 16) && d->q_token_stride % 8 == 0 && d->q_head_stride % 8 == 0;
  a.vec_out = aligned_to(d->out, 8) && d->out_token_stride % 4 == 0 && d->out_head_stride % 4 == 0;
  return d->type == SZO_BF16 ? launch_dim<SZO_BF16>(a, p, (hipStream_t)stream) : launch_dim<SZO_F16>(a, p, (hipStream_t)stream);
}

}  // extern "C"
