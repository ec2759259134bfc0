// Log probabilities of given tokens with entropy and the best alternatives, and their gradient.
//
//   u = scale (x - max x),  S = sum exp(u):   logp = u_target - log S,   entropy = log S - sum u exp(u) / S
//   gradient = scale (g ([v = target] - p) - h p (log p + entropy)),  p = exp(u) / S
//
// Bound by reading the logits: once, with a running maximum and two running sums in every thread.  The alternatives cost the stream nothing:
// the threads' own maxima are there already, and the top-th largest of them is a lower bound of the top-th largest logit that
// only the elements of as many threads can reach.  Those threads' elements (about top / 512 of the row) are read again, from cache, and ranked.
#include <algorithm>
#include "szo_internal.h"
#include "szo_types.h"

namespace szo {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kCandidates = 1024;
constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLowest = -3.402823466e38f;

// 16 bytes of logits at any element; gfx950 loads them at any address.
template <int TYPE> struct Chunk {
  typedef typename TypeOf<TYPE>::type T;
  static constexpr int N = 16 / sizeof(T);
  typedef T vec __attribute__((ext_vector_type(N)));
  typedef vec loose __attribute__((aligned(sizeof(T))));
  static __device__ __forceinline__ void load(const void* base, int64_t at, float (&v)[N]) {
    const vec x = *reinterpret_cast<const loose*>(static_cast<const T*>(base) + at);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (float)x[i];
  }
  static __device__ __forceinline__ void store(void* base, int64_t at, const float (&v)[N]) {
    vec x;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (T)v[i];
    *reinterpret_cast<loose*>(static_cast<T*>(base) + at) = x;
  }
  static __device__ __forceinline__ float one(const void* base, int64_t at) { return (float)static_cast<const T*>(base)[at]; }
};

// Running statistics: sums relative to the maximum so far, which starts at the lowest finite value so that differences stay defined.
struct Running {
  float m, s, t;                     // maximum, sum exp(u), sum u exp(u)
  __device__ Running() : m(kLowest), s(0.f), t(0.f) {}
  // to a maximum that is not smaller
  __device__ void rebase(float to, float scale) {
    const float du = (m - to) * scale, f = exp2f(du * kLog2e);
    t = f * (t + (du > -200.f ? du : -200.f) * s);             // u becomes u + du; below -200 the factor is 0 anyway
    s *= f;
    m = to;
  }
  __device__ void add(float x, float scale) {
    const float u = (x - m) * scale, e = exp2f(u * kLog2e);
    s += e;
    t = fmaf(e, fmaxf(u, -200.f), t);                          // -inf: 0 times a finite number
  }
};

// Order of alternatives: larger first, NaN before everything, zeros of both signs alike.
__device__ __forceinline__ uint32_t order_of(float x) {
  if (x != x) return 0xFFFFFFFFu;
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

struct LogpArgs { szo_logprobs_desc d; };

template <int TYPE>
__global__ void __launch_bounds__(kThreads) token_logprobs_kernel(const LogpArgs a) {
  typedef Chunk<TYPE> C;
  constexpr int N = C::N;
  __shared__ float red[3][kWaves];
  __shared__ float maxima[kThreads];
  __shared__ uint64_t found[kCandidates];
  __shared__ int count, winners, more;
  __shared__ float bound;
  __shared__ short winner[kThreads];
  const szo_logprobs_desc& d = a.d;
  const int64_t row = blockIdx.x, from = row * d.row_stride;
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int vocab = (int)d.vocab, chunks = vocab / N;
  Running r;
  int c = tid;
  constexpr int U = 4;
  for (; c + (U - 1) * kThreads < chunks; c += U * kThreads) {
    float v[U][N];
#pragma unroll
    for (int i = 0; i < U; ++i) C::load(d.logits, from + (int64_t)(c + i * kThreads) * N, v[i]);
    float most = r.m;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int n = 0; n < N; ++n) most = fmaxf(most, v[i][n]);
    r.rebase(most, d.scale);
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int n = 0; n < N; ++n) r.add(v[i][n], d.scale);
  }
  for (; c < chunks; c += kThreads) {
    float v[N];
    C::load(d.logits, from + (int64_t)c * N, v);
    float most = r.m;
#pragma unroll
    for (int n = 0; n < N; ++n) most = fmaxf(most, v[n]);
    r.rebase(most, d.scale);
#pragma unroll
    for (int n = 0; n < N; ++n) r.add(v[n], d.scale);
  }
  const int tail = chunks * N + tid;                           // fewer than N elements
  if (tail < vocab) {
    const float x = C::one(d.logits, from + tail);
    r.rebase(fmaxf(r.m, x), d.scale);
    r.add(x, d.scale);
  }
  maxima[tid] = r.m;
  float m = lanes_max<64>(r.m);
  if (lane == 0) red[0][wave] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) m = fmaxf(m, red[0][w]);
  r.rebase(m, d.scale);
  float s = lanes_sum<64>(r.s), t = lanes_sum<64>(r.t);
  if (lane == 0) { red[1][wave] = s; red[2][wave] = t; }
  if (tid == 0) { count = 0; winners = 0; more = 0; }
  __syncthreads();
  s = t = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) { s += red[1][w]; t += red[2][w]; }
  const float log_s = logf(s);                                 // a row of -inf alone: s is 0
  const bool empty = s == 0.f;
  if (tid == 0) {
    const int target = d.targets ? d.targets[row] : -1;
    if (d.logp) {
      float y = 0.f;
      if (target >= 0 && target < vocab) y = empty ? -__builtin_inff() : (C::one(d.logits, from + target) - m) * d.scale - log_s;
      d.logp[row] = y;
    }
    if (d.entropy) d.entropy[row] = empty ? 0.f : log_s - t / s;
    if (d.stats) { d.stats[2 * row] = empty ? -__builtin_inff() : m; d.stats[2 * row + 1] = s; }
  }
  const int top = d.top;
  if (!top || !(d.top_logp || d.top_index)) return;

  auto put = [&](int rank, float x, int index) {
    if (d.top_logp) d.top_logp[row * top + rank] = empty ? -__builtin_inff() : (x - m) * d.scale - log_s;
    if (d.top_index) d.top_index[row * top + rank] = index;
  };
  const bool plain = s - s == 0.f && !empty;                   // NaN or infinite logits make s NaN
  if (plain) {
    // the top-th largest of the threads' maxima, by halving in one wave
    if (wave == 0) {
      uint32_t key[kWaves];
#pragma unroll
      for (int i = 0; i < kWaves; ++i) key[i] = order_of(maxima[i * 64 + lane]);
      uint32_t lo = 0, hi = order_of(m);                       // at least top keys are >= lo
      while (lo < hi) {
        const uint32_t mid = lo + (hi - lo + 1) / 2;
        int n = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) n += __popcll(__ballot(key[i] >= mid));
        if (n >= top) lo = mid; else hi = mid - 1;
        if (n == top) break;
      }
      if (lane == 0) bound = __uint_as_float(lo & 0x80000000u ? lo & 0x7FFFFFFFu : ~lo);
    }
    __syncthreads();
    const float least = bound;
    if (maxima[tid] >= least) winner[atomicAdd(&winners, 1)] = (short)tid;
    __syncthreads();
    const int per = (chunks + kThreads - 1) / kThreads, items = winners * per;
    for (int i = tid; i < items; i += kThreads) {
      const int at = winner[i / per] + i % per * kThreads;
      if (at >= chunks) continue;
      float v[N];
      C::load(d.logits, from + (int64_t)at * N, v);
#pragma unroll
      for (int n = 0; n < N; ++n)
        if (v[n] >= least) {
          const int to = atomicAdd(&count, 1);
          if (to < kCandidates) found[to] = (uint64_t)order_of(v[n]) << 32 | (uint32_t)~(at * N + n);
        }
    }
    if (tail < vocab) {
      const float x = C::one(d.logits, from + tail);
      if (x >= least) {
        const int to = atomicAdd(&count, 1);
        if (to < kCandidates) found[to] = (uint64_t)order_of(x) << 32 | (uint32_t)~tail;
      }
    }
    __syncthreads();
    if (count >= top && count <= kCandidates) {      // fewer: most of the row is -inf
      for (int i = tid; i < count; i += kThreads) {
        const uint64_t mine = found[i];
        int rank = 0;
        for (int j = 0; j < count; ++j) rank += found[j] > mine;
        if (rank < top) {
          const int index = (int)~(uint32_t)mine;
          put(rank, C::one(d.logits, from + index), index);
        }
      }
      return;
    }
  }
  // Rows with NaN, infinities or very many equal logits: one pass over the row for each alternative.
  uint64_t last = ~0ull;
  for (int rank = 0; rank < top; ++rank) {
    uint64_t best = 0;
    for (int i = tid; i < vocab; i += kThreads) {
      const uint64_t key = (uint64_t)order_of(C::one(d.logits, from + i)) << 32 | (uint32_t)~i;
      if (key < last && key > best) best = key;
    }
#pragma unroll
    for (int step = 32; step; step /= 2) {
      const uint64_t other = __shfl_xor(best, step);
      best = other > best ? other : best;
    }
    __syncthreads();
    if (lane == 0) found[wave] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) best = found[w] > best ? found[w] : best;
    if (tid == 0) {
      const int index = (int)~(uint32_t)best;
      put(rank, C::one(d.logits, from + index), index);
    }
    last = best;
  }
}

// loss_acc += scale * sum of -logp over rows with a target: fp64, one workgroup, fixed order.
__global__ void __launch_bounds__(1024) logp_loss_kernel(const float* __restrict__ logp, const int32_t* __restrict__ targets, int64_t rows, int64_t vocab,
                                                         double scale, double* loss_acc) {
  __shared__ double part[16];
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < rows; i += 1024) {
    const int t = targets ? targets[i] : -1;
    if (t >= 0 && t < vocab) s -= (double)logp[i];
  }
  s = wave_sum(s);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = s;
  __syncthreads();
  if (threadIdx.x) return;
  for (int w = 1; w < 16; ++w) s += part[w];
  *loss_acc += scale * s;
}

struct GradArgs { szo_logprobs_desc d; const float *g_logp, *g_entropy; void* out; int64_t out_stride; int parts; };

constexpr int kGradThreads = 256;
constexpr int kGradChunks = 4;             // 16-byte pieces of a thread

template <int TYPE>
__global__ void __launch_bounds__(kGradThreads) token_logprobs_bwd_kernel(const GradArgs a) {
  typedef Chunk<TYPE> C;
  constexpr int N = C::N;
  const szo_logprobs_desc& d = a.d;
  const int64_t row = blockIdx.x / a.parts;
  const int part = blockIdx.x % a.parts, vocab = (int)d.vocab, chunks = vocab / N;
  const float m = d.stats[2 * row], s = d.stats[2 * row + 1];
  const int target = d.targets ? d.targets[row] : -1;
  const float g = a.g_logp && target >= 0 && target < vocab ? a.g_logp[row] : 0.f, h = a.g_entropy ? a.g_entropy[row] : 0.f;
  const bool empty = s == 0.f;
  const float by = 1.f / s, log_s = logf(s), entropy = a.g_entropy ? d.entropy[row] : 0.f;
  const int64_t from = row * d.row_stride, to = row * a.out_stride;
  auto gradient = [&](float x, int v) {
    const float u = (x - m) * d.scale, p = exp2f(u * kLog2e) * by;
    float y = -g * p;
    if (a.g_entropy) y = fmaf(-h * p, fmaxf(u, -200.f) - log_s + entropy, y);
    if (v == target) y += g;
    return empty ? 0.f : y * d.scale;
  };
  const int first = part * kGradThreads * kGradChunks + threadIdx.x;
#pragma unroll
  for (int i = 0; i < kGradChunks; ++i) {
    const int c = first + i * kGradThreads;
    if (c >= chunks) break;
    float v[N];
    C::load(d.logits, from + (int64_t)c * N, v);
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = gradient(v[n], c * N + n);
    C::store(a.out, to + (int64_t)c * N, v);
  }
  const int tail = chunks * N + threadIdx.x;
  if (part == 0 && tail < vocab) {
    typedef typename TypeOf<TYPE>::type T;
    static_cast<T*>(a.out)[to + tail] = (T)gradient(C::one(d.logits, from + tail), tail);
  }
}

int check(const szo_logprobs_desc* d) {
  if (!d || d->rows < 0 || d->vocab < 0 || !valid_type(d->type) || d->reserved) return SZO_EINVAL;
  if (d->top < 0 || d->top > d->vocab || !(d->scale > 0.f && d->scale < 3.4e38f)) return SZO_EINVAL;
  if (d->top > SZO_LOGPROBS_MAX_TOP || d->vocab > (1 << 30) || d->rows > 0x7FFFFFFF) return SZO_EUNSUPPORTED;
  if (d->rows > 1 && d->row_stride < 0) return SZO_EINVAL;
  if (d->rows && d->vocab && (!d->logits || !aligned_to(d->logits, type_bytes(d->type)))) return SZO_EINVAL;
  if (!aligned_to(d->targets, 4) || !aligned_to(d->logp, 4) || !aligned_to(d->entropy, 4) || !aligned_to(d->stats, 4) || !aligned_to(d->top_logp, 4) ||
      !aligned_to(d->top_index, 4) || !aligned_to(d->loss_acc, 8)) return SZO_EINVAL;
  return SZO_OK;
}

}  // namespace
}  // namespace szo

using namespace szo;

extern "C" {

size_t szo_logprobs_workspace_bytes(const szo_logprobs_desc* d) {
  (void)d;
  return 16;
}

int szo_token_logprobs(const szo_logprobs_desc* d, void* workspace, void* stream) {
  (void)workspace;
  const int rc = check(d);
  if (rc != SZO_OK) return rc;
  if (d->loss_acc && !d->logp) return SZO_EINVAL;
  if (d->rows == 0) return SZO_OK;
  if (d->vocab == 0) return SZO_EINVAL;
  hipStream_t s = (hipStream_t)stream;
  const LogpArgs a = {*d};
  const dim3 grid((unsigned)d->rows);
  if (d->type == SZO_F32) token_logprobs_kernel<SZO_F32><<<grid, kThreads, 0, s>>>(a);
  else if (d->type == SZO_BF16) token_logprobs_kernel<SZO_BF16><<<grid, kThreads, 0, s>>>(a);
  else token_logprobs_kernel<SZO_F16><<<grid, kThreads, 0, s>>>(a);
  SZO_LAUNCH_CHECK();
  if (d->loss_acc) {
    logp_loss_kernel<<<1, 1024, 0, s>>>(d->logp, d->targets, d->rows, d->vocab, d->loss_scale, d->loss_acc);
    SZO_LAUNCH_CHECK();
  }
  return SZO_OK;
}

int szo_token_logprobs_bwd(const szo_logprobs_desc* d, const float* grad_logp, const float* grad_entropy, void* grad_logits, int64_t grad_row_stride,
                           void* stream) {
  const int rc = check(d);
  if (rc != SZO_OK) return rc;
  if (d->rows == 0 || d->vocab == 0) return SZO_OK;
  if (!d->stats || (grad_entropy && !d->entropy) || !grad_logits || !aligned_to(grad_logits, type_bytes(d->type)) || !aligned_to(grad_logp, 4) ||
      !aligned_to(grad_entropy, 4)) return SZO_EINVAL;
  if (d->rows > 1 && grad_row_stride < d->vocab) return SZO_EINVAL;
  GradArgs a = {*d, grad_logp, grad_entropy, grad_logits, grad_row_stride, 0};
  const int64_t pieces = d->vocab / (16 / (int64_t)type_bytes(d->type)), per = (int64_t)kGradThreads * kGradChunks;
  a.parts = (int)std::max<int64_t>(1, (pieces + per - 1) / per);
  if (d->rows * a.parts > 0x7FFFFFFF) return SZO_EUNSUPPORTED;
  hipStream_t s = (hipStream_t)stream;
  const dim3 grid((unsigned)(d->rows * a.parts));
  if (d->type == SZO_F32) token_logprobs_bwd_kernel<SZO_F32><<<grid, kGradThreads, 0, s>>>(a);
  else if (d->type == SZO_BF16) token_logprobs_bwd_kernel<SZO_BF16><<<grid, kGradThreads, 0, s>>>(a);
  else token_logprobs_bwd_kernel<SZO_F16><<<grid, kGradThreads, 0, s>>>(a);
  SZO_LAUNCH_CHECK();
  return SZO_OK;
}

}  // extern "C"
