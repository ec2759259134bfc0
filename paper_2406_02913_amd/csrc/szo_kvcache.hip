// Writing a key/value cache in 8 bits, and reading it back.
//
//   e = smallest integer with max|x| <= 448 * 2^e over a block of 32 tokens of a head;   code = e4m3(x 2^-e)
//
// Bound by memory: new keys and values are read once and 1 byte each is written.  One workgroup owns one block of one head, keys and
// values, so the maximum is a workgroup's and nothing is shared between workgroups.  The block's elements are held in registers between
// the maximum and the conversion.  Values lie transposed in the cache (the order of a matrix operand): whole blocks go through LDS, so that
// both sides of the transposition are wide and contiguous.  A few tokens into a block that is there already take their bytes one by one: a decoding
// step moves a few hundred bytes per head and is bound by latency, not by them.
//   Eight prompts, 4096 tokens together, 32 heads of 128, from fp32: 34.9 us, 4.8 TB/s of what is read and written (a copy of 2 GiB runs at 4.85); one token to each of
// 64 sequences, 8 heads: 4.9 us, four reads that wait for each other; 8192 tokens of 8 heads back as bf16: 10.2 us, 4.9 TB/s.
#include <algorithm>
#include "szo_internal.h"
#include "szo_kv.h"

namespace szo {
namespace {

constexpr int kThreads = 256;
constexpr int kRow = kKvBlock + 4;         // bytes of a feature's row of values in LDS: odd in words, so that rows start in different banks

struct KvArgs {
  szo_kv_cache c;
  szo_kv_tokens t;
  int blocks_per_page;
};

// The block that a workgroup owns, and the tokens of it that the call is about: slots [first, end), slot s being row from + s.
struct Share {
  int head, index, first, end;
  int64_t row, block;
  __device__ bool find(const int32_t* token_start, const int32_t* lengths, int64_t tokens, const KvArgs& a) {
    const int sequence = blockIdx.z, nth = blockIdx.y;
    head = blockIdx.x;
    const int start = max(token_start[sequence], 0), stop = max((int)min((int64_t)token_start[sequence + 1], tokens), 0);      // rows that there are
    const int64_t length = lengths[sequence], had = length - (int64_t)(stop - start);
    if (stop <= start || length <= 0) return false;
    const int64_t at = (had > 0 ? had : 0) / kKvBlock + nth;             // tokens before position 0 have no place
    if (at * kKvBlock >= length) return false;
    index = (int)at;
    first = (int)max((int64_t)0, had - at * kKvBlock);
    end = (int)min((int64_t)kKvBlock, length - at * kKvBlock);
    row = start + (at * kKvBlock - had);
    block = block_of(a.c, sequence, index, head, a.blocks_per_page);
    return true;
  }
};

__device__ __forceinline__ int exponent_for(float most) {
  const uint32_t b = __float_as_uint(most);
  // most = m 2^x, m in [1, 2): 448 = 1.75 * 2^8; values below the normal range end at the lower limit anyway
  const int x = (int)(b >> 23) - 127, e = x - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return min(max(e, kExpMin), kExpMax);
}

// Four values as codes, times 2^-e: nearest even, what is not finite as NaN.  |x 2^-e| <= 448, so nothing overflows.
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d, float down) {
  int w = 0;
  w = __builtin_amdgcn_cvt_pk_fp8_f32(finite_or_nan(a) * down, finite_or_nan(b) * down, w, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(finite_or_nan(c) * down, finite_or_nan(d) * down, w, true);
  return (uint32_t)w;
}

__device__ __forceinline__ void values_of(uint32_t w, float (&v)[4]) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  v[0] = lo[0]; v[1] = lo[1]; v[2] = hi[0]; v[3] = hi[1];
}

// Codes of the block that the call does not write, moved down to a larger exponent: by dwords, byte by byte where new ones lie between.
template <int D, bool VALUES>
__device__ __forceinline__ void move_down(uint8_t* block, int first, int end, float down) {
  for (int i = threadIdx.x; i < D * kKvBlock / 4; i += kThreads) {
    uint32_t* at = reinterpret_cast<uint32_t*>(block) + i;
    // a dword holds four features of one token (keys), or tokens t..t+3 of one feature (values)
    int t;
    if (VALUES) { const int p = (i % 8) * 4; t = ((p >> 3) & 1) * 16 + ((p >> 2) & 1) * 8 + (p >> 4) * 4; }
    else t = (i / 8) % kKvBlock;
    const int last = VALUES ? t + 3 : t;
    if (t >= first && last < end) continue;
    float v[4];
    values_of(*at, v);
    const uint32_t w = codes_of(v[0], v[1], v[2], v[3], down);
    if (last < first || t >= end) {
      *at = w;
    } else {
      for (int r = 0; r < 4; ++r)
        if (t + r < first || t + r >= end) reinterpret_cast<uint8_t*>(at)[r] = (uint8_t)(w >> (8 * r));
    }
  }
}

// What the first loads need comes first in the arguments, where it is in registers when a wave starts.  VEC: groups of four features lie at multiples of their size.
template <int TYPE, int D, bool VEC>
__global__ void __launch_bounds__(kThreads) kv_cache_write_kernel(const int32_t* token_start, const int32_t* lengths, int64_t tokens, const KvArgs a) {
  __shared__ float maxima[2][kThreads / 64];
  __shared__ __attribute__((aligned(16))) uint8_t tile[D * kRow];
  Share s;
  if (!s.find(token_start, lengths, tokens, a) || s.block < 0) return;
  constexpr int kKeys = D * kKvBlock / 8, kValues = D * kKvBlock / 16;          // units: 8 features of a token; 4 features of 4 tokens
  constexpr int kPerK = (kKeys + kThreads - 1) / kThreads, kPerV = (kValues + kThreads - 1) / kThreads;
  float k[kPerK][8], v[kPerV][4][4];
  float kmost = 0.f, vmost = 0.f;
#pragma unroll
  for (int n = 0; n < kPerK; ++n) {
    const int u = threadIdx.x + n * kThreads, t = u / (D / 8), f = u % (D / 8) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) k[n][i] = 0.f;
    if (u < kKeys && t >= s.first && t < s.end) {
      const int64_t at = (s.row + t) * a.t.k_token_stride + s.head * a.t.k_head_stride + f;
      float lo[4], hi[4];
      load_f32<TYPE, 4, VEC>(a.t.k, at, lo);
      load_f32<TYPE, 4, VEC>(a.t.k, at + 4, hi);
#pragma unroll
      for (int i = 0; i < 4; ++i) { k[n][i] = lo[i]; k[n][4 + i] = hi[i]; }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) kmost = fmaxf(kmost, finite_size(k[n][i]));
  }
#pragma unroll
  for (int n = 0; n < kPerV; ++n) {
    const int u = threadIdx.x + n * kThreads, t0 = u / (D / 4) * 4, f = u % (D / 4) * 4;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int t = t0 + r;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[n][r][i] = 0.f;
      if (u < kValues && t >= s.first && t < s.end)
        load_f32<TYPE, 4, VEC>(a.t.v, (s.row + t) * a.t.v_token_stride + s.head * a.t.v_head_stride + f, v[n][r]);
#pragma unroll
      for (int i = 0; i < 4; ++i) vmost = fmaxf(vmost, finite_size(v[n][r][i]));
    }
  }
  kmost = lanes_max<64>(kmost);
  vmost = lanes_max<64>(vmost);
  if (threadIdx.x % 64 == 0) { maxima[0][threadIdx.x / 64] = kmost; maxima[1][threadIdx.x / 64] = vmost; }
  const bool whole = s.first == 0;
  int kold = kExpMin, vold = kExpMin;
  if (!whole) { kold = (int)a.c.k_exp[s.block] - kExpBias; vold = (int)a.c.v_exp[s.block] - kExpBias; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) { kmost = fmaxf(kmost, maxima[0][w]); vmost = fmaxf(vmost, maxima[1][w]); }
  const int ke = max(exponent_for(kmost), min(max(kold, kExpMin), kExpMax)), ve = max(exponent_for(vmost), min(max(vold, kExpMin), kExpMax));
  const float kdown = power_of_two(-ke), vdown = power_of_two(-ve);
  uint8_t* kb = a.c.k + s.block * (D * kKvBlock);
  uint8_t* vb = a.c.v + s.block * (D * kKvBlock);
  if (threadIdx.x == 0) { a.c.k_exp[s.block] = (uint8_t)(ke + kExpBias); a.c.v_exp[s.block] = (uint8_t)(ve + kExpBias); }
  if (!whole) {
    // up to 152 binary places; from 2^-126 on nothing is left of a code either way
    if (ke > kold) move_down<D, false>(kb, s.first, s.end, power_of_two(max(kold - ke, -126)));
    if (ve > vold) move_down<D, true>(vb, s.first, s.end, power_of_two(max(vold - ve, -126)));
  }
#pragma unroll
  for (int n = 0; n < kPerK; ++n) {
    const int u = threadIdx.x + n * kThreads, t = u / (D / 8), f = u % (D / 8) * 8;
    if (u < kKeys && (whole || (t >= s.first && t < s.end))) {
      const uint2 w = make_uint2(codes_of(k[n][0], k[n][1], k[n][2], k[n][3], kdown), codes_of(k[n][4], k[n][5], k[n][6], k[n][7], kdown));
      *reinterpret_cast<uint2*>(kb + (f / 32) * 1024 + t * 32 + f % 32) = w;
    }
  }
#pragma unroll
  for (int n = 0; n < kPerV; ++n) {
    const int u = threadIdx.x + n * kThreads, t0 = u / (D / 4) * 4, f = u % (D / 4) * 4;
    if (u >= kValues) break;
    if (!whole && (t0 + 4 <= s.first || t0 >= s.end)) continue;
    uint32_t w[4];                         // one token's four features, then turned into one feature's four tokens
#pragma unroll
    for (int r = 0; r < 4; ++r) w[r] = codes_of(v[n][r][0], v[n][r][1], v[n][r][2], v[n][r][3], vdown);
    const int p = value_place(t0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400 + 0x0101 * i), hi = __builtin_amdgcn_perm(w[3], w[2], 0x0c0c0400 + 0x0101 * i);
      const uint32_t four = lo | (hi << 16);
      if (whole) *reinterpret_cast<uint32_t*>(tile + (f + i) * kRow + p) = four;
      else {
        for (int r = 0; r < 4; ++r)
          if (t0 + r >= s.first && t0 + r < s.end) vb[(f + i) * 32 + p + r] = (uint8_t)(four >> (8 * r));
      }
    }
  }
  if (!whole) return;
  __syncthreads();
  for (int i = threadIdx.x; i < D * 2; i += kThreads) {          // 16 bytes each
    const uint32_t* from = reinterpret_cast<const uint32_t*>(tile + (i / 2) * kRow + (i % 2) * 16);
    reinterpret_cast<uint4*>(vb)[i] = make_uint4(from[0], from[1], from[2], from[3]);
  }
}

template <int TYPE, int D, bool VEC>
__global__ void __launch_bounds__(kThreads) kv_cache_read_kernel(const int32_t* token_start, const int32_t* lengths, int64_t tokens, const KvArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t tile[D * kRow];
  Share s;
  if (!s.find(token_start, lengths, tokens, a)) return;
  constexpr int kKeys = D * kKvBlock / 8, kValues = D * kKvBlock / 16;
  const bool there = s.block >= 0;
  const uint8_t* kb = a.c.k + (there ? s.block * (D * kKvBlock) : 0);
  const uint8_t* vb = a.c.v + (there ? s.block * (D * kKvBlock) : 0);
  float kup = 0.f, vup = 0.f;
  if (there) {
    kup = power_of_two(min(max((int)a.c.k_exp[s.block] - kExpBias, kExpMin), kExpMax));
    vup = power_of_two(min(max((int)a.c.v_exp[s.block] - kExpBias, kExpMin), kExpMax));
  }
  for (int i = threadIdx.x; i < D * 2; i += kThreads) {
    const uint4 w = there ? reinterpret_cast<const uint4*>(vb)[i] : make_uint4(0, 0, 0, 0);
    uint32_t* to = reinterpret_cast<uint32_t*>(tile + (i / 2) * kRow + (i % 2) * 16);
    to[0] = w.x; to[1] = w.y; to[2] = w.z; to[3] = w.w;
  }
  for (int u = threadIdx.x; u < kKeys; u += kThreads) {
    const int t = u / (D / 8), f = u % (D / 8) * 8;
    if (t < s.first || t >= s.end) continue;
    const uint2 w = there ? *reinterpret_cast<const uint2*>(kb + (f / 32) * 1024 + t * 32 + f % 32) : make_uint2(0, 0);
    float lo[4], hi[4];
    values_of(w.x, lo);
    values_of(w.y, hi);
#pragma unroll
    for (int i = 0; i < 4; ++i) { lo[i] *= kup; hi[i] *= kup; }
    const int64_t at = (s.row + t) * a.t.k_token_stride + s.head * a.t.k_head_stride + f;
    store_f32<TYPE, 4, VEC>(a.t.k, at, lo);
    store_f32<TYPE, 4, VEC>(a.t.k, at + 4, hi);
  }
  __syncthreads();
  for (int u = threadIdx.x; u < kValues; u += kThreads) {
    const int t0 = u / (D / 4) * 4, f = u % (D / 4) * 4, p = value_place(t0);
    if (t0 + 4 <= s.first || t0 >= s.end) continue;
    float v[4][4];                         // [feature][token]
#pragma unroll
    for (int i = 0; i < 4; ++i) values_of(*reinterpret_cast<const uint32_t*>(tile + (f + i) * kRow + p), v[i]);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (t0 + r < s.first || t0 + r >= s.end) continue;
      const float x[4] = {v[0][r] * vup, v[1][r] * vup, v[2][r] * vup, v[3][r] * vup};
      store_f32<TYPE, 4, VEC>(a.t.v, (s.row + t0 + r) * a.t.v_token_stride + s.head * a.t.v_head_stride + f, x);
    }
  }
}

template <int TYPE, int D>
void launch_type(const KvArgs& a, dim3 grid, bool vec, bool write, hipStream_t s) {
  if (write) {
    if (vec) kv_cache_write_kernel<TYPE, D, true><<<grid, kThreads, 0, s>>>(a.t.token_start, a.c.lengths, a.t.tokens, a);
    else kv_cache_write_kernel<TYPE, D, false><<<grid, kThreads, 0, s>>>(a.t.token_start, a.c.lengths, a.t.tokens, a);
  } else {
    if (vec) kv_cache_read_kernel<TYPE, D, true><<<grid, kThreads, 0, s>>>(a.t.token_start, a.c.lengths, a.t.tokens, a);
    else kv_cache_read_kernel<TYPE, D, false><<<grid, kThreads, 0, s>>>(a.t.token_start, a.c.lengths, a.t.tokens, a);
  }
}
template <int D>
void launch_dim(const KvArgs& a, dim3 grid, bool vec, bool write, hipStream_t s) {
  if (a.t.type == SZO_F32) launch_type<SZO_F32, D>(a, grid, vec, write, s);
  else if (a.t.type == SZO_BF16) launch_type<SZO_BF16, D>(a, grid, vec, write, s);
  else launch_type<SZO_F16, D>(a, grid, vec, write, s);
}

int move_tokens(const szo_kv_cache* c, const szo_kv_tokens* t, bool write, hipStream_t s) {
  const int rc = check_cache(c);
  if (rc != SZO_OK) return rc;
  if (!t || !valid_type(t->type) || t->reserved || t->max_new < 0 || t->tokens < 0) return SZO_EINVAL;
  if (t->k_token_stride < 0 || t->k_head_stride < 0 || t->v_token_stride < 0 || t->v_head_stride < 0) return SZO_EINVAL;
  if (!write) {                            // rows that are written may not run into each other
    if (t->k_token_stride < c->head_dim || t->v_token_stride < c->head_dim) return SZO_EINVAL;
    if (c->kv_heads > 1 && (t->k_head_stride < c->head_dim || t->v_head_stride < c->head_dim)) return SZO_EINVAL;
  }
  if (c->sequences == 0 || t->max_new == 0 || c->kv_heads == 0) return SZO_OK;
  if (!t->token_start || !t->k || !t->v || !aligned_to(t->token_start, 4) || !aligned_to(t->k, type_bytes(t->type)) || !aligned_to(t->v, type_bytes(t->type)))
    return SZO_EINVAL;
  KvArgs a;
  a.c = *c;
  a.t = *t;
  a.blocks_per_page = c->page_tokens / kKvBlock;
  const int64_t room = (int64_t)c->max_pages * a.blocks_per_page;            // blocks behind the page table hold nothing
  const int64_t most = std::min<int64_t>({t->max_new, t->tokens, 0x7FFFFFFF});          // new tokens of a sequence; rows are counted in 32 bits
  if (most == 0) return SZO_OK;
  int64_t touched = (most + kKvBlock - 2) / kKvBlock + 1;
  if (write) touched = std::min(touched, room);
  if (touched == 0) return SZO_OK;
  if (touched > 65535 || c->sequences > 65535) return SZO_EUNSUPPORTED;
  const dim3 grid((unsigned)c->kv_heads, (unsigned)touched, (unsigned)c->sequences);
  const size_t four = 4 * type_bytes(t->type);
  const bool vec = aligned_to(t->k, four) && aligned_to(t->v, four) && t->k_token_stride % 4 == 0 && t->k_head_stride % 4 == 0 && t->v_token_stride % 4 == 0 &&
                   t->v_head_stride % 4 == 0;
  switch (c->head_dim) {
    case 64: launch_dim<64>(a, grid, vec, write, s); break;
    case 96: launch_dim<96>(a, grid, vec, write, s); break;
    case 128: launch_dim<128>(a, grid, vec, write, s); break;
    default: launch_dim<256>(a, grid, vec, write, s); break;
  }
  SZO_LAUNCH_CHECK();
  return SZO_OK;
}

}  // namespace

int check_cache(const szo_kv_cache* c) {
  if (!c || c->pages < 0 || c->kv_heads < 0 || c->sequences < 0 || c->max_pages < 0 || c->page_tokens <= 0 || c->head_dim <= 0) return SZO_EINVAL;
  if (c->page_tokens % kKvBlock) return SZO_EINVAL;
  if (c->kv_heads > 65535) return SZO_EUNSUPPORTED;            // a side of a grid
  if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128 && c->head_dim != 256) return SZO_EUNSUPPORTED;
  if ((int64_t)c->max_pages * c->page_tokens > 0x7FFFFFFF) return SZO_EUNSUPPORTED;
  if (c->sequences && (!c->lengths || !aligned_to(c->lengths, 4))) return SZO_EINVAL;          // read for every sequence, with or without pages
  if (c->sequences && c->max_pages && (!c->page_table || !aligned_to(c->page_table, 4))) return SZO_EINVAL;
  if (c->pages && c->kv_heads && (!c->k || !c->v || !c->k_exp || !c->v_exp || !aligned_to(c->k, 16) || !aligned_to(c->v, 16))) return SZO_EINVAL;
  return SZO_OK;
}

}  // namespace szo

using namespace szo;

extern "C" {

int szo_kv_cache_write(const szo_kv_cache* cache, const szo_kv_tokens* tokens, void* stream) {
  return move_tokens(cache, tokens, true, (hipStream_t)stream);
}

int szo_kv_cache_read(const szo_kv_cache* cache, const szo_kv_tokens* tokens, void* stream) {
  return move_tokens(cache, tokens, false, (hipStream_t)stream);
}

}  // extern "C"
