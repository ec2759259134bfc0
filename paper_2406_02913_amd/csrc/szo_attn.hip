// Attention over a key/value cache in 8 bits (layout: szo.h).
//
//   s = scale q k,  p = exp(s) where the query sees the key,  out = sum p v / sum p,  in one pass with a running maximum.
//
// A wave takes 32 query rows (a token's query heads of one key head are rows too: they share its keys) and walks blocks of 32 cached
// tokens.  It computes S^T = K Q^T and O^T = V^T P^T in products of 32 x 32: in the result of the first a lane has one query row and 16 of
// the 32 tokens, which is just what the second takes as an operand, so the weights never leave their lane, and the row's maximum is
// one lane exchange away.  The cache is laid out as the two left operands: 16 bytes of a lane are its codes.
//   Scores: codes become bf16 or fp16, like the queries, exactly; the block's exponent goes into the factor of its scores.  (The matrix cores'
// 8-bit products would take the codes as they are, with a query in two or three 8-bit parts; but they add up to fewer than fp32's bits:
// scores of 20 were off by 1e-4.)
//   Values: codes become fp16, exactly; weights are rounded to fp16.  A block's exponent goes into the exponent of its weights: with
// x = log2(e) s + v_exp the running maximum is over x, sum 2^(x - m) code is the output's numerator and sum 2^(x - m) 2^-v_exp the
// denominator, so that the weights are relative to the largest contribution of the row.  A block whose exponent is far below that of others may add nothing to the
// numerator and all the same most of the denominator (a block of zeros has exponent -32, others up to 120): its 2^(x - m) leaves fp32's range,
// 2^(x - m - v_exp) does not, and is what is added up there (attn_walk_kernel: `apart`).
//   A maximum is held as two numbers, log2(e) s of the token that sets it and the exponent of its block: their sum would lose the exponent where scores are large.
#include <algorithm>
#include "szo_internal.h"
#include "szo_kv.h"

namespace szo {
namespace {

constexpr int kThreads = 256;              // of the joining kernel
constexpr float kNone = -3.402823466e38f;  // running maximum of a row that has seen nothing: the lowest finite value, so that differences stay defined
constexpr float kSlack = 4.f;              // the maximum may fall behind by this many binary places before sums are scaled
constexpr float kLift = 11.f;              // weights are held times 2^11: up to 2^15 with the slack, and all 11 bits of fp16 down to 2^-25 of the largest
// The denominator is held times 2^40 beside that.  Its largest term is the one of the block with exponent e that sets the maximum, 2^(51 - e), from 2^-73 (with the slack)
// on: what is 2^-50 of it is still a normal number; no term is above 2^(15 + 32 + 40), so that 2^31 of them are finite.
constexpr int kSumLift = 40;
constexpr int kApart = 90;                 // exponents of values further apart than this: terms of the denominator may leave fp32's range on the way
constexpr float kFar = 1048576.f;          // maxima beyond 2^20: a fused product minus the rounded maximum is no longer a difference of rounded products

struct AttnArgs {
  szo_attn_desc d;
  int group, blocks_per_page;              // query heads per key head
  int tiles, splits, rows_cap;             // row tiles of a workgroup, parts of the cache, rows kept per wave tile in partial sums
  float to_log2;                           // |scale| * log2(e)
  bool negate;                             // scale < 0: queries change sign
  float* partial;                          // [sequence][key head][wave tile][split] of part_floats()
  bool vec_q, vec_out;
};

// A part's sums: rows_cap rows of head_dim numerators, then maximum (two floats) and denominator of each.  A multiple of 16 bytes, which rows are stored
// and read in.
__host__ __device__ constexpr int part_floats(int rows_cap, int head_dim) { return (rows_cap * (head_dim + 3) + 3) / 4 * 4; }

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

template <int D> struct Raw { uint4 w[D / 32]; };

// ONCE: nobody else reads it, so it may pass the caches by.
template <int D, bool ONCE>
__device__ __forceinline__ Raw<D> load_block(const uint8_t* codes, int block, int lane) {
  typedef uint32_t words __attribute__((ext_vector_type(4)));
  Raw<D> r;
  const words* p = reinterpret_cast<const words*>(codes + (int64_t)block * (D * kKvBlock)) + (lane % 32) * 2 + lane / 32;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    words w;
    if constexpr (ONCE) w = __builtin_nontemporal_load(p + i * 64);
    else w = p[i * 64];
    r.w[i] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return r;
}

// Eight codes as fp16.
__device__ __forceinline__ f16x8 halves(uint32_t lo, uint32_t hi) {
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
  return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ f32x16 product(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

// Operands of the scores, in the queries' type.
template <int TYPE> struct Score;
template <> struct Score<SZO_BF16> {
  typedef bf16x8 vec;
  static __device__ __forceinline__ vec codes(uint32_t lo, uint32_t hi) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return vec{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  }
  static __device__ __forceinline__ f32x16 add(vec k, vec q, f32x16 s) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q, s, 0, 0, 0); }
};
template <> struct Score<SZO_F16> {
  typedef f16x8 vec;
  static __device__ __forceinline__ vec codes(uint32_t lo, uint32_t hi) { return halves(lo, hi); }
  static __device__ __forceinline__ f32x16 add(vec k, vec q, f32x16 s) { return product(k, q, s); }
};

// A lane's row of queries, in the order of the features that a block of keys has: 32 s + 16 half + 8 u .. + 7.
template <int TYPE, int D> struct Query {
  typename Score<TYPE>::vec part[D / 32][2];
  __device__ __forceinline__ void load(const void* base, int64_t at, bool valid, bool aligned, bool negate, int half) {
    typedef typename Score<TYPE>::vec vec;
    const auto* p = static_cast<const typename TypeOf<TYPE>::type*>(base) + at + 16 * half;
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        vec x = {};
        if (valid) {
          if (aligned) x = *reinterpret_cast<const vec*>(p + 32 * s + 8 * u);
          else
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = p[32 * s + 8 * u + i];
        }
        uint4 w = __builtin_bit_cast(uint4, x);
        const uint32_t flip = negate ? 0x80008000u : 0u;
        w.x ^= flip; w.y ^= flip; w.z ^= flip; w.w ^= flip;
        part[s][u] = __builtin_bit_cast(vec, w);
      }
  }
};

// Factor of a block's scores, in powers of two; never 0, so that masked ones stay -inf, and finite, so that scores of 0 stay 0.
__device__ __forceinline__ float score_factor(float to_log2, int key_exp) {
  return __builtin_amdgcn_fmed3f(to_log2 * power_of_two(min(max(key_exp - kExpBias, kExpMin), kExpMax)), 1e-37f, -kNone);
}

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

// Sums are scaled by 2^by in two steps of half of it: a denominator may be so large that it matters where 2^by by itself is 0 (by from -152 on).
__device__ __forceinline__ float half_of(float by) { return __builtin_amdgcn_exp2f(0.5f * by); }
// What the numerators are multiplied by, and log sum exp: the exponents of maximum and denominator cancel, so they go first.
__device__ __forceinline__ float inverse_sum(float l) { return l == 0.f ? 0.f : power_of_two(kSumLift) / l; }
__device__ __forceinline__ float log_sum(float m, float m_exp, float l) {
  if (l == 0.f) return -__builtin_inff();
  const float e = (float)__builtin_amdgcn_frexp_expf(l) - (kLift + (float)kSumLift);
  return ((m + (m_exp + e)) + __log2f(__builtin_amdgcn_frexp_mantf(l))) * 0.693147180559945309f;
}

__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

// 0x80 in each byte of w that is the code of NaN
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

// Where a sequence's blocks lie, walked forward: the page table is read one step before the block's codes are asked for.
struct Walk {
  int page_at, sub;
  __device__ __forceinline__ Walk(int block, int blocks_per_page) : page_at(block / blocks_per_page), sub(block - page_at * blocks_per_page) {}
  __device__ __forceinline__ void step(int by, int blocks_per_page) {
    sub += by;
    while (sub >= blocks_per_page) { sub -= blocks_per_page; ++page_at; }
  }
  // Number of the block in the cache; -1: no page.  Below the sequence's length, so inside the page table.
  __device__ __forceinline__ int at(const szo_kv_cache& c, const int32_t* table, int head, int blocks_per_page) const {
    return on(c, table[page_at], head, blocks_per_page);
  }
  __device__ __forceinline__ int on(const szo_kv_cache& c, int page, int head, int blocks_per_page) const {
    return (uint32_t)page >= (uint32_t)c.pages ? -1 : (page * c.kv_heads + head) * blocks_per_page + sub;
  }
};

// A lane's half of a row: finished, or as this split's partial sum.  Of WK waves each has the features 32 e .. + 31 with e = walker modulo WK.
template <int TYPE, int D, int WK>
__device__ __forceinline__ void put_row(const AttnArgs& a, const f32x16 (&o)[D / 32], float m, float m_exp, float l, int sequence, int head, int64_t tiles, int wave_tile, int split,
                                        int walker, int token, int q_head, int column, int half) {
  const szo_attn_desc& d = a.d;
  if (a.splits > 1) {
    float* to = a.partial + ((((int64_t)sequence * d.cache.kv_heads + head) * tiles + wave_tile) * a.splits + split) * part_floats(a.rows_cap, D);
    float* mine = to + (int64_t)column * D;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) {
      if (e % WK != walker) continue;
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<float4*>(mine + 32 * e + 2 * i + 4 * half) = make_float4(o[e][i], o[e][i + 1], o[e][i + 2], o[e][i + 3]);
    }
    if (half == 0 && walker == 0) {
      to[(int64_t)a.rows_cap * D + 3 * column] = m;
      to[(int64_t)a.rows_cap * D + 3 * column + 1] = m_exp;
      to[(int64_t)a.rows_cap * D + 3 * column + 2] = l;
    }
    return;
  }
  const float by = inverse_sum(l);
  const int64_t at = (int64_t)token * d.out_token_stride + (int64_t)q_head * d.out_head_stride;
#pragma unroll
  for (int e = 0; e < D / 32; ++e) {
    if (e % WK != walker) continue;
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const float y[4] = {o[e][i] * by, o[e][i + 1] * by, o[e][i + 2] * by, o[e][i + 3] * by};
      if (a.vec_out) store_f32<TYPE, 4, true>(d.out, at + 32 * e + 2 * i + 4 * half, y);
      else store_f32<TYPE, 4, false>(d.out, at + 32 * e + 2 * i + 4 * half, y);
    }
  }
  if (d.lse && half == 0 && walker == 0) d.lse[(int64_t)token * d.q_heads + q_head] = log_sum(m, m_exp, l);
}

// WR waves side by side over rows, WK over the cache, every wave with what it reads straight from memory.
//   A step computes the weights of block j and its share of the output beside the scores of block j + 1: matrix and vector instructions of
// one step do not depend on each other.  The arguments that the first loads need come first, where they are in registers when a wave starts; the page of the
// first block is read along with the lengths, for the case that it starts there.  Codes are asked for a step before they are used (two steps: 562 -> 596 us for a prompt of 8192,
// registers run out).
//   A prompt of 8192 tokens with 32 query and 8 key heads of 128, causal: 577 us, 953 TFLOP/s, bound by the issue of instructions: matrix products take 44 % of
// the cycles, and a step has 186 vector instructions beside 16 products.  One token of each of 64 sequences of up to 8192: 108 us, 5.73 TB/s of the cache.
// 4096 tokens in bf16 with head dimensions of 64, 96, 128, 256: 124, 138, 168, 393 us (556, 748, 820, 699 TFLOP/s), in fp16 110, 140, 166, 383.
template <int TYPE, int D, int WR, int WK, bool ONCE>
__global__ void __launch_bounds__(64 * WR * WK, D <= 128 ? 2 : 1) attn_walk_kernel(const int32_t* q_start, const int32_t* lengths, const int32_t* page_table,
                                                                                   int max_pages, int bpp, int splits, int tiles, const AttnArgs a) {
  constexpr int E = D / 32;
  const szo_attn_desc& d = a.d;
  const int lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64), column = lane % 32, half = lane / 32;
  // key heads vary fastest: workgroups are dealt out to the 8 XCDs in turn, so the row tiles of one key head share an L2
  const int head = blockIdx.x, sequence = blockIdx.z;
  const int split = splits == 1 ? 0 : blockIdx.y % splits;
  const int tile = tiles - 1 - (splits == 1 ? blockIdx.y : blockIdx.y / splits);          // later rows see more: they start first
  const int wave_tile = tile * WR + wave % WR, walker = WK == 1 ? 0 : wave / WR;
  const int32_t* table = page_table + (int64_t)sequence * max_pages;
  const int whole = lengths[sequence], guess = max_pages > walker / bpp ? table[walker / bpp] : -1;
  const int start = max(q_start[sequence], 0), stop = max((int)min((int64_t)q_start[sequence + 1], d.tokens), 0);      // differences of both fit
  const int n = max(0, min(stop - start, d.max_q));
  const int length = (int)max((int64_t)0, min((int64_t)whole, (int64_t)max_pages * bpp * kKvBlock));
  const int rows = n * a.group, first_row = wave_tile * 32;
  if (tile * WR * 32 >= rows) return;                    // the workgroup as a whole
  const int behind = max(whole, 0) - (stop - start);     // position of the sequence's first query
  // First position of the window of a query at `position`: 0 where the window is wider; no difference leaves 32 bits.  What a wave has in common is kept in scalar
  // registers (a prompt of 8192 636 us otherwise, 577 so).
  auto window_from = [&](int position) { return d.window > 0 ? max(position + 1, d.window) - d.window : 0; };

  // this lane's row
  const int row = first_row + column, query = row / a.group, q_head = head * a.group + row % a.group;
  const bool valid = row < rows;
  const int see_to = !valid ? 0 : d.causal ? min(length, behind + query + 1) : length;
  const int see_from = window_from(behind + query);
  Query<TYPE, D> q;
  q.load(d.q, (int64_t)(start + query) * d.q_token_stride + (int64_t)q_head * d.q_head_stride, valid, a.vec_q, a.negate, half);

  // blocks that some row of the wave sees, the part of them that is this split's, and this wave's share of that
  const int pos_first = behind + first_row / a.group, pos_last = behind + (min(first_row + 32, rows) - 1) / a.group;
  const int reach = first_row >= rows || d.cache.pages == 0 ? 0 : d.causal ? min(length, pos_last + 1) : length;
  const int lo = uniform(window_from(pos_first)) / kKvBlock, hi = reach > 0 ? (reach + kKvBlock - 1) / kKvBlock : 0;
  const int share = splits == 1 ? max(hi - lo, 0) : (max(hi - lo, 0) + splits - 1) / splits;
  const int j0 = lo + split * share + walker, j1 = min(hi, lo + (split + 1) * share);
  const int see_all = d.causal ? min(length, pos_first + 1) : length;     // tokens before this one are seen by every row, but for the window
  const int see_all_from = uniform(window_from(pos_last));

  f32x16 o[E], s = {};
  float m = kNone, m_exp = 0.f, l = 0.f;
  bool far = false;                        // some row's maximum is beyond kFar
  uint32_t poison[(E + 1) / 2];            // one bit for each of the lane's sums: it is NaN
#pragma unroll
  for (int e = 0; e < E; ++e) { o[e] = f32x16{}; poison[e / 2] = 0; }

  if (j0 < j1) {
    // A block without a page is read as block 0 and masked as a whole; behind the last block the last one stands in, for nothing.
    Walk walk(j0, bpp);
    int now = j0 == walker ? walk.on(d.cache, guess, head, bpp) : walk.at(d.cache, table, head, bpp), next = now;
    if (j0 + WK < j1) { walk.step(WK, bpp); next = walk.at(d.cache, table, head, bpp); }
    auto known = [](int b) { return max(b, 0); };
    auto scores = [&](const Raw<D>& k) {
      s = f32x16{};
#pragma unroll
      for (int i = 0; i < E; ++i) {
        s = Score<TYPE>::add(Score<TYPE>::codes(k.w[i].x, k.w[i].y), q.part[i][0], s);
        s = Score<TYPE>::add(Score<TYPE>::codes(k.w[i].z, k.w[i].w), q.part[i][1], s);
      }
    };
    Raw<D> k = load_block<D, ONCE>(d.cache.k, known(now), lane), v = load_block<D, ONCE>(d.cache.v, known(now), lane);
    int ke = d.cache.k_exp[known(now)], ve = d.cache.v_exp[known(now)], most_vexp = kExpMin;
    scores(k);
    k = load_block<D, ONCE>(d.cache.k, known(next), lane);
    for (int j = j0; j < j1; j += WK) {        // k: keys of the next step, v: values of this one
      const bool there = now >= 0;
      now = next;
      if (j + 2 * WK < j1) { walk.step(WK, bpp); next = walk.at(d.cache, table, head, bpp); }
      float factor = score_factor(a.to_log2, ke);
      const int vexp = uniform(min(max(ve - kExpBias, kExpMin), kExpMax));
      const float shift = (float)vexp;
      float unshift = power_of_two(kSumLift - vexp);
      most_vexp = max(most_vexp, vexp);
      const bool apart = most_vexp - vexp > kApart;
      ke = d.cache.k_exp[known(now)], ve = d.cache.v_exp[known(now)];
      const int token = j * kKvBlock + 4 * half, to = there ? see_to - token : 0, from = see_from - token;      // of s[0]; s[i] is 8 (i / 4) + i % 4 further
      const bool all = there && (j + 1) * kKvBlock <= see_all && j * kKvBlock >= see_all_from;
      if (!all) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int at = 8 * (i / 4) + i % 4;
          s[i] = at < to && at >= from ? s[i] : -__builtin_inff();
        }
      }
      float most = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) most = fmaxf(most, s[i]);
      most = rounded_product(halves_max(most), factor);
      const float over = (most - m) + (shift - m_exp);
      if (__any(over > kSlack)) {
        const bool up = over > 0.f;
        const float by_half = half_of(up ? -over : 0.f), scale = by_half * by_half;
        l = l * by_half * by_half;
        m = up ? most : m;
        m_exp = up ? shift : m_exp;
        far |= __any(up && fabsf(m) > kFar);
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[e][i] *= scale;
      }
      if (!all) {
        // A masked token's weight is 0, and 0 times NaN would be NaN: such codes are taken out, and the rows that do see them get their NaN
        uint32_t bad = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) bad |= nan_codes(v.w[e].x) | nan_codes(v.w[e].y) | nan_codes(v.w[e].z) | nan_codes(v.w[e].w);
        if (__any(bad != 0)) {
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
            f16x8 seen[2];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int at = 8 * (i / 4) + i % 4;
              seen[i / 8][i % 8] = at < to && at >= from ? (_Float16)1.f : (_Float16)0.f;
            }
            f32x16 hits = {};
            hits = product(halves(mark[0], mark[1]), seen[0], hits);
            hits = product(halves(mark[2], mark[3]), seen[1], hits);
#pragma unroll
            for (int i = 0; i < 16; ++i) poison[e / 2] |= hits[i] > 0.f ? 1u << (e % 2 * 16 + i) : 0u;
          }
        }
      }
      // Half of the weights beside the scores, the other half beside the first half of the output: there are vector instructions for every product to run beside
      // (all of them first: 576 us instead of 556 for a prompt of 8192).
      f16x8 p[2];
      const float step = shift - m_exp;
      float base = step - m + kLift, sum = 0.f;
      if (apart || far) {      // the terms of the denominator by themselves, of products that are rounded as the maximum is; what follows adds those of the numerator alone
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float x = rounded_product(s[i], factor) - m + step;
          l += __builtin_amdgcn_exp2f(x - shift + (kLift + (float)kSumLift));
          s[i] = x;
        }
        factor = 1.f;
        base = kLift;
        unshift = 0.f;
      }
      const f32x16 x = s;
      auto weigh = [&](int c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float w = __builtin_amdgcn_exp2f(fmaf(x[8 * c + i], factor, base));
          sum += w;
          p[c][i] = (_Float16)w;
        }
      };
      weigh(0);
      scores(k);
      if (WK == 1) k = load_block<D, ONCE>(d.cache.k, known(next), lane);       // one path of instructions up to here: no condition
      weigh(1);
      l = fmaf(sum, unshift, l);
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = product(halves(v.w[e].x, v.w[e].y), p[0], o[e]);
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = product(halves(v.w[e].z, v.w[e].w), p[1], o[e]);
      if (WK == 1 || j + WK < j1) v = load_block<D, ONCE>(d.cache.v, known(now), lane);
      if (WK > 1 && j + 2 * WK < j1) k = load_block<D, ONCE>(d.cache.k, known(next), lane);
    }
  }

  l = halves_sum(l);
  uint32_t any = 0;
#pragma unroll
  for (int e = 0; e < E; e += 2) any |= poison[e / 2];
  if (__any(any != 0)) {
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[e][i] = poison[e / 2] >> (e % 2 * 16 + i) & 1 ? __builtin_nanf("") : o[e][i];
  }

  if constexpr (WK > 1) {
    // the walkers' sums meet: each adds up every WK-th tile of 32 features (one of them all: 16 short answers 26.2 -> 25.8 us, one token behind 1000 10.3 -> 9.9)
    extern __shared__ __attribute__((aligned(16))) float meet[];
    constexpr int kPer = 64 * (D / 2 + 3);
    static_assert(WR == 1, "one tile of rows");
    {
      float* to = meet + walker * kPer;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (e % WK == walker) continue;
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<float4*>(to + (e * 4 + i / 4) * 256 + lane * 4) = make_float4(o[e][i], o[e][i + 1], o[e][i + 2], o[e][i + 3]);
      }
      to[D / 2 * 64 + lane] = m;
      to[D / 2 * 64 + 64 + lane] = m_exp;
      to[D / 2 * 64 + 128 + lane] = l;
    }
    __syncthreads();
    // the largest of the first numbers, and of the second ones relative to it: no walker's maximum is above the two, and one is equal to them
    float top = kNone, top_exp = kNone, part[WK];
#pragma unroll
    for (int w = 0; w < WK; ++w) top = fmaxf(top, meet[w * kPer + D / 2 * 64 + lane]);
#pragma unroll
    for (int w = 0; w < WK; ++w) {
      part[w] = meet[w * kPer + D / 2 * 64 + lane] - top + meet[w * kPer + D / 2 * 64 + 64 + lane];
      top_exp = fmaxf(top_exp, part[w]);
    }
    l = 0.f;
#pragma unroll
    for (int w = 0; w < WK; ++w) {
      const float by_half = half_of(part[w] - top_exp);
      part[w] = by_half * by_half;
      l = fmaf(meet[w * kPer + D / 2 * 64 + 128 + lane] * by_half, by_half, l);
    }
    const float own_half = half_of(m - top + m_exp - top_exp), own = own_half * own_half;
    m = top;
    m_exp = top_exp;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (e % WK != walker) continue;
#pragma unroll
      for (int i = 0; i < 16; ++i) o[e][i] *= own;
#pragma unroll
      for (int w = 0; w < WK; ++w) {
        if (w == walker) continue;
        const float* from = meet + w * kPer;
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const float4 x = *reinterpret_cast<const float4*>(from + (e * 4 + i / 4) * 256 + lane * 4);
          o[e][i] = fmaf(x.x, part[w], o[e][i]);
          o[e][i + 1] = fmaf(x.y, part[w], o[e][i + 1]);
          o[e][i + 2] = fmaf(x.z, part[w], o[e][i + 2]);
          o[e][i + 3] = fmaf(x.w, part[w], o[e][i + 3]);
        }
      }
    }
  }
  if (valid) put_row<TYPE, D, WK>(a, o, m, m_exp, l, sequence, head, (int64_t)a.tiles * WR, wave_tile, split, walker, start + query, q_head, column, half);
}

// Joins the parts of a row, four features of it at a time, by G neighbouring lanes: each takes every G-th part and they add each other up by row
// permutations.  One lane, up to four parts on the way, for up to five parts and for full tiles, 16 lanes otherwise (1 sequence of 8000 in 32 parts 12.4 -> 10.5 us,
// 32 rows of it in 8 parts 18.7 -> 19.2).  Workgroups go over sequences, key heads, wave tiles and a tile's pieces.
template <int TYPE, int D, int G>
__global__ void __launch_bounds__(kThreads) attn_join_kernel(const int32_t* q_start, const float* partial, int wave_tiles, int splits, int rows_cap, const AttnArgs a) {
  const szo_attn_desc& d = a.d;
  const int wave_tile = blockIdx.x % wave_tiles, head = blockIdx.y, sequence = blockIdx.z;
  const float* from = partial + (((int64_t)sequence * gridDim.y + head) * wave_tiles + wave_tile) * splits * part_floats(rows_cap, D);
  const int start = max(q_start[sequence], 0), stop = max((int)min((int64_t)q_start[sequence + 1], d.tokens), 0);
  const int rows = min(max(0, min(stop - start, d.max_q)) * a.group - wave_tile * 32, 32);
  const int i = (blockIdx.x / wave_tiles * kThreads + threadIdx.x) / G, g = threadIdx.x % G;
  const int column = i / (D / 4), f = i % (D / 4) * 4, row = wave_tile * 32 + column, query = row / a.group, q_head = head * a.group + row % a.group;
  if (column >= rows) return;                  // G lanes at once
  float m = kNone, m_exp = 0.f, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  constexpr int kAhead = G == 1 ? 4 : 2;
#pragma unroll kAhead
  for (int s = g; s < splits; s += G) {
    const float* part = from + (int64_t)s * part_floats(rows_cap, D);
    const float* stats = part + (int64_t)rows_cap * D + 3 * column;
    const float ms = stats[0], es = stats[1], ls = stats[2];
    const float4 x = *reinterpret_cast<const float4*>(part + (int64_t)column * D + f);
    const float over = (ms - m) + (es - m_exp), keep_half = half_of(fminf(-over, 0.f)), add_half = half_of(fminf(over, 0.f));
    const float keep = keep_half * keep_half, add = add_half * add_half;
    l = fmaf(l * keep_half, keep_half, ls * add_half * add_half);
    m = over > 0.f ? ms : m;
    m_exp = over > 0.f ? es : m_exp;
    o[0] = o[0] * keep + x.x * add;
    o[1] = o[1] * keep + x.y * add;
    o[2] = o[2] * keep + x.z * add;
    o[3] = o[3] * keep + x.w * add;
  }
  if constexpr (G > 1) {
    const float top = lanes_max<G>(m), rest = m - top + m_exp, top_exp = lanes_max<G>(rest), keep_half = half_of(rest - top_exp), keep = keep_half * keep_half;
    l = lanes_sum<G>(l * keep_half * keep_half);
    m = top;
    m_exp = top_exp;
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = lanes_sum<G>(o[k] * keep);
    if (g) return;
  }
  const float by = inverse_sum(l);
  const float y[4] = {o[0] * by, o[1] * by, o[2] * by, o[3] * by};
  const int64_t at = (int64_t)(start + query) * d.out_token_stride + (int64_t)q_head * d.out_head_stride + f;
  if (a.vec_out) store_f32<TYPE, 4, true>(d.out, at, y);
  else store_f32<TYPE, 4, false>(d.out, at, y);
  if (d.lse && f == 0)
    d.lse[(int64_t)(start + query) * d.q_heads + q_head] = log_sum(m, m_exp, l);
}

// ---- host ------------------------------------------------------------------------------------------------------------

// How rows and cache go to waves.
//   Four waves of a workgroup take rows side by side (wr 4) or share the cache of one tile of 32 rows (wr 1), and meet in LDS.  Side by side from
// 2048 tiles on, which fill the chip's 2048 waves by themselves, or from half of that where there is no cache to share, eight blocks at most.  us of
// one pass, 32 query and 8 key heads of 128, side by side / shared: one prompt of 1024 tokens (1032 tiles) 31 / 21, of 2048 54 / 57, 4 of 512 26 / 32,
// 4 of 1024 57 / 76, 16 of 256 31 / 50, 16 of 64 7.9 / 13.1.
//   With few workgroups a tile's cache is split over several, and a second kernel joins the parts.  That costs 2 us where a tile has few rows and 4 to 6
// with 32, whose parts are 16 KiB each, and every workgroup 5 us to begin and to end: few rows go to up to 512 workgroups with a single block a wave (from 64
// workgroups on with four), full tiles to 256 with four blocks a wave, and to twice as many of either only in caches of thousands.  us of parts 1, 2, 4, 8, 16, 32,
// one token each: 1 sequence of 1000 10.7, 10.6, 9.0, 8.5, 8.5, 8.6; 1 of 8000 54, 33, 21, 15.2, 11.8, 10.4; 8 of 4000 35, 24, 17, 18, 21, 27; 16 of 8000 81, 50, 46,
// 51, 58, 74; 32 of 1000 14, 18, 21; 64 of 500 to 8192 111, 107, 106.  64 tokens of one sequence (8 tiles for each key head) behind 2000 17.2, 16.1, 14.7, 19.7;
// behind 8000 60, 38, 25, 25, 34; 200 tokens, four waves a tile, behind 4000 29, 32, 39, behind 8000 60, 47, 55.  All with 32 query heads of 128 in bf16: the rule counts
// blocks and tiles, and has not been measured for other head dimensions.
//   Between 65 and 256 workgroups, a CU each, eight waves share a tile's cache of 1000 tokens or more instead of four (wk): 8 x 29 answers behind up to 2000
// 20.3 -> 16.4 us, 200 tokens behind 2000 17.0 -> 15.5, behind 8000 47 -> 40; with fewer workgroups parts are better (one token behind 8000 10.2 -> 10.6),
// and short tiles read enough at once when three quarters of the CUs have one (32 sequences of 1000 14.2 -> 15.2).
//   Blocks that one workgroup alone reads, 128 MiB of them or more, pass the caches by (once): 64 sequences of 500 to 8192 121 -> 106 us, 16 of 8000 52 -> 46,
// 32 of 1000 (64 MiB) 14.2 -> 15.4.
struct Plan { int wr, wk, tiles, splits, rows_cap; bool once; };

Plan plan_of(const szo_attn_desc* d) {
  Plan p;
  const int64_t group = d->q_heads / d->cache.kv_heads, rows = (int64_t)d->max_q * group;
  const int64_t pairs = (int64_t)d->cache.sequences * d->cache.kv_heads;
  const int64_t seen = d->window > 0 ? std::min<int64_t>(d->max_len, (int64_t)d->window + d->max_q) : d->max_len;       // tokens of a sequence, at most
  const int64_t blocks = (std::max<int64_t>(seen, 1) + kKvBlock - 1) / kKvBlock;
  // tiles of 32 rows that hold something, about: a sequence's last one is partly filled
  const int64_t held = std::min<int64_t>(d->tokens * group / 32 + d->cache.sequences, (int64_t)d->cache.sequences * ((rows + 31) / 32)) * d->cache.kv_heads;
  p.wr = rows > 32 && (held >= 2048 || (held >= 1024 && blocks <= 8)) ? 4 : 1;
  p.tiles = (int)((rows + 32 * p.wr - 1) / (32 * p.wr));
  p.rows_cap = (int)std::min<int64_t>(32, rows);
  p.once = p.wr == 1 && p.tiles == 1 && blocks * kKvBlock * 2 * d->cache.head_dim >= ((int64_t)128 << 20) / pairs;
  const int64_t some = std::max<int64_t>(1, std::min(held / p.wr, pairs * p.tiles));          // workgroups that hold something
  p.wk = p.wr == 4 ? 1 : d->cache.head_dim <= 128 && !p.once && some > 64 && some <= (p.tiles == 1 ? 192 : 256) && blocks >= 32 ? 8 : 4;
  const int64_t walkers = p.wk;
  const bool few = rows <= 16;
  const bool single = few && some <= 64;                // a block a wave
  const int64_t chip = few ? 512 : 256, step = single ? walkers : 4 * walkers, parts = blocks < (single ? 24 : 48) ? 1 : std::min<int64_t>((blocks + step - 1) / step, 32);
  const int64_t fill = p.wk == 8 ? std::min(256 / some, blocks / 32) : few && chip / some < 3 ? 1 : std::min(chip / some, parts), even = p.wk == 8 ? 1 : std::min(2 * chip / some, blocks / (walkers * (few ? 15 : 20)));
  p.splits = (int)std::min<int64_t>(std::max<int64_t>({1, fill, even}), 64);
  return p;
}

int check(const szo_attn_desc* d) {
  if (!d) return SZO_EINVAL;
  const int rc = check_cache(&d->cache);
  if (rc != SZO_OK) return rc;
  const szo_kv_cache& c = d->cache;
  if ((d->type != SZO_BF16 && d->type != SZO_F16) || (d->causal & ~1) || d->reserved || d->q_heads < 0 || d->window < 0 || d->max_q < 0 || d->max_len < 0 ||
      d->tokens < 0) return SZO_EINVAL;
  if (!(d->scale >= -SZO_MOST_SCALE && d->scale <= SZO_MOST_SCALE)) return SZO_EINVAL;
  if (d->tokens > 0x7FFFFFFF) return SZO_EUNSUPPORTED;
  if (c.kv_heads == 0 ? d->q_heads != 0 : d->q_heads % c.kv_heads != 0) return SZO_EINVAL;
  if (c.sequences == 0 || d->q_heads == 0 || d->tokens == 0 || d->max_q == 0) return SZO_OK;
  if (!d->q || !d->out || !d->q_start || !aligned_to(d->q_start, 4) || !aligned_to(d->q, 2) || !aligned_to(d->out, 2) || !aligned_to(d->lse, 4)) return SZO_EINVAL;
  if (!c.lengths || !c.page_table) return SZO_EINVAL;
  if (d->q_token_stride < 0 || d->q_head_stride < 0 || (d->tokens > 1 && d->out_token_stride < c.head_dim) || (d->q_heads > 1 && d->out_head_stride < c.head_dim))
    return SZO_EINVAL;
  if ((int64_t)d->max_q * (d->q_heads / c.kv_heads) > 0x3FFFFFFF) return SZO_EUNSUPPORTED;
  if ((int64_t)c.pages * c.kv_heads * (c.page_tokens / kKvBlock) > 0x7FFFFFFF) return SZO_EUNSUPPORTED;
  const Plan p = plan_of(d);
  if ((int64_t)c.sequences * c.kv_heads * p.tiles * p.wr * p.splits > 0x7FFFFFFF || (int64_t)p.tiles * p.splits > 65535 || c.sequences > 65535) return SZO_EUNSUPPORTED;
  return SZO_OK;
}
bool nothing(const szo_attn_desc* d) { return d->cache.sequences == 0 || d->q_heads == 0 || d->tokens == 0 || d->max_q == 0; }

template <int TYPE, int D, int WR, int WK, bool ONCE>
int launch(const AttnArgs& a, hipStream_t s) {
  constexpr size_t lds = WK == 1 ? 0 : (size_t)WK * 64 * (D / 2 + 3) * sizeof(float);
  static std::atomic<uint64_t> raised{0};
  if (lds > 64 * 1024) {
    const int rc = set_lds_limit_once(raised, (const void*)attn_walk_kernel<TYPE, D, WR, WK, ONCE>, lds);
    if (rc != SZO_OK) return rc;
  }
  const dim3 grid((unsigned)a.d.cache.kv_heads, (unsigned)(a.tiles * a.splits), (unsigned)a.d.cache.sequences);
  attn_walk_kernel<TYPE, D, WR, WK, ONCE><<<grid, 64 * WR * WK, lds, s>>>(a.d.q_start, a.d.cache.lengths, a.d.cache.page_table, a.d.cache.max_pages, a.blocks_per_page,
                                                                     a.splits, a.tiles, a);
  SZO_LAUNCH_CHECK();
  return SZO_OK;
}

template <int TYPE, int D, int G>
int join(const AttnArgs& a, const Plan& p, hipStream_t s) {
  const int pieces = (a.rows_cap * (D / 4) * G + kThreads - 1) / kThreads;            // of a tile
  const dim3 grid((unsigned)(p.tiles * p.wr * pieces), (unsigned)a.d.cache.kv_heads, (unsigned)a.d.cache.sequences);
  attn_join_kernel<TYPE, D, G><<<grid, kThreads, 0, s>>>(a.d.q_start, a.partial, p.tiles * p.wr, a.splits, a.rows_cap, a);
  SZO_LAUNCH_CHECK();
  return SZO_OK;
}

template <int TYPE, int D>
int launch_all(const AttnArgs& a, const Plan& p, hipStream_t s) {
  int rc;
  if (p.wr == 4) rc = launch<TYPE, D, 4, 1, false>(a, s);
  else if (p.wk == 8) rc = launch<TYPE, D <= 128 ? D : 128, 1, 8, false>(a, s);           // 134 KiB of LDS at 128
  else if (p.once) rc = launch<TYPE, D, 1, 4, true>(a, s);
  else rc = launch<TYPE, D, 1, 4, false>(a, s);
  if (rc != SZO_OK || p.splits == 1) return rc;
  return p.splits < 6 || a.rows_cap > 16 ? join<TYPE, D, 1>(a, p, s) : join<TYPE, D, 16>(a, p, s);
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
  return (size_t)d->cache.sequences * d->cache.kv_heads * p.tiles * p.wr * p.splits * part_floats(p.rows_cap, d->cache.head_dim) * sizeof(float);
}

int szo_attn_plan(const szo_attn_desc* d, int32_t* plan) {
  const int rc = check(d);
  if (rc != SZO_OK) return rc;
  if (!plan) return SZO_EINVAL;
  const Plan p = nothing(d) ? Plan{} : plan_of(d);
  plan[0] = p.wr;
  plan[1] = p.wk;
  plan[2] = p.splits;
  plan[3] = p.once;
  return SZO_OK;
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
  a.to_log2 = (d->scale < 0.f ? -d->scale : d->scale) * 1.44269504088896341f;
  a.negate = d->scale < 0.f;
  a.partial = (float*)workspace;
  a.vec_q = aligned_to(d->q, 16) && d->q_token_stride % 8 == 0 && d->q_head_stride % 8 == 0;
  a.vec_out = aligned_to(d->out, 8) && d->out_token_stride % 4 == 0 && d->out_head_stride % 4 == 0;
  return d->type == SZO_BF16 ? launch_dim<SZO_BF16>(a, p, (hipStream_t)stream) : launch_dim<SZO_F16>(a, p, (hipStream_t)stream);
}

}  // extern "C"
