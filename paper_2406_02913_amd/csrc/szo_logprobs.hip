// Log probabilities of given tokens with entropy and the best alternatives, and their gradient.
//
//   u = scale (x - max x),  S = sum exp(u):   logp = u_target - log S,   entropy = log S - sum u exp(u) / S
//   gradient = scale (g ([v = target] - p) - h p (log p + entropy)),  p = exp(u) / S
//
// Bound by reading the logits: once, with a running maximum and two running sums in every thread.  The alternatives cost the stream nothing:
// the threads' own maxima are there already.  The top-th largest among the maxima of groups of 8 threads bounds the top-th largest logit from below, and
// few others reach it (of 32 groups, 31 logits for 20 alternatives): the threads whose maximum does look through their elements again, and what they
// find is ranked.
// With few rows a row is split over workgroups, whose parts a second kernel joins.
//   Rows with NaN or infinities, with fewer finite logits than alternatives, or with more than 1024 that reach the bound are gone through once for each alternative instead,
// element by element: with 5 of 32000 logits not masked and 20 alternatives 400 us for 16 rows (9 without a mask), 2330 for 4096 (97).
#include <algorithm>
#include "szo_internal.h"
#include "szo_types.h"

namespace szo {
namespace {

constexpr int kCandidates = 1024;
constexpr int kThreads = 256;
constexpr int kMostParts = 32;
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
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

// Running statistics in powers of two, u = (x - m) scale log2(e): relative to the maximum so far, which starts at the lowest finite value so that
// differences stay defined.
struct Running {
  float m, s, t;                     // maximum, sum 2^u, sum u 2^u
  __device__ Running() : m(kLowest), s(0.f), t(0.f) {}
  // to a maximum that is not smaller
  __device__ void rebase(float to, float scale) {
    const float du = (m - to) * scale, f = __builtin_amdgcn_exp2f(du);
    t = f * fmaf(fmaxf(du, -300.f), s, t);                     // u becomes u + du; below -300 the factor is 0 anyway
    s *= f;
    m = to;
  }
  __device__ void add(float x, float scale) {
    const float u = (x - m) * scale, e = __builtin_amdgcn_exp2f(u);
    s += e;
    t = fmaf(e, fmaxf(u, -300.f), t);                          // -inf: 0 times a finite number
  }
};

// Order of alternatives: larger first, NaN before everything, zeros of both signs alike.
__device__ __forceinline__ uint32_t order_of(float x) {
  if (x != x) return 0xFFFFFFFFu;
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t key_of(float x, int index) { return (uint64_t)order_of(x) << 32 | (uint32_t)~index; }
__device__ __forceinline__ int index_of(uint64_t key) { return (int)~(uint32_t)key; }
__device__ __forceinline__ float value_of(uint64_t key) {
  const uint32_t k = (uint32_t)(key >> 32);
  return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);         // 0xFFFFFFFF is a NaN as well
}

// Parts of rows: statistics [row][part][3], then the keys of the part's best [row][part][top], 0 where there are fewer.
struct LogpArgs { szo_logprobs_desc d; int parts; float* stats; uint64_t* best; };

// A row's results, from its statistics.
struct Finish {
  float m, s, log_s, scale;
  bool empty;
  __device__ Finish(float m_, float s_, float scale_) : m(m_), s(s_), log_s(logf(s_)), scale(scale_), empty(s_ == 0.f) {}     // a row of -inf alone: s is 0
  __device__ float logp(float x) const { return empty ? -__builtin_inff() : (x - m) * scale - log_s; }
  template <int TYPE>
  __device__ void write(const szo_logprobs_desc& d, int64_t row, float t) const {
    const int target = d.targets ? d.targets[row] : -1;
    if (d.logp) d.logp[row] = target >= 0 && target < d.vocab ? logp(Chunk<TYPE>::one(d.logits, row * d.row_stride + target)) : 0.f;
    if (d.entropy) d.entropy[row] = empty ? 0.f : log_s - t / s * kLn2;
    if (d.stats) { d.stats[2 * row] = empty ? -__builtin_inff() : m; d.stats[2 * row + 1] = s; }
  }
  __device__ void put(const szo_logprobs_desc& d, int64_t row, int rank, uint64_t key) const {
    if (d.top_logp) d.top_logp[row * d.top + rank] = logp(value_of(key));
    if (d.top_index) d.top_index[row * d.top + rank] = index_of(key);
  }
};

// 256 threads with four pieces each on the way.  4096 rows of 32000 in fp32: 95 us with 20 alternatives (5.5 TB/s), 89 without; 512 threads 93 and 88, but
// rows of 2000 43 instead of 24, of 8000 61 instead of 54.
template <int TYPE>
__global__ void __launch_bounds__(kThreads) token_logprobs_kernel(const LogpArgs a) {
  typedef Chunk<TYPE> C;
  constexpr int N = C::N, U = 4, kWaves = kThreads / 64, kGroups = kThreads / 8;      // U: pieces of a thread on the way; as many groups as alternatives
  __shared__ float red[3][kWaves];
  __shared__ __attribute__((aligned(16))) float maxima[kGroups];
  __shared__ uint64_t found[kCandidates];
  __shared__ int count, winners;
  __shared__ short winner[kThreads];
  const szo_logprobs_desc& d = a.d;
  const int64_t row = blockIdx.x / a.parts, from = row * d.row_stride;
  const int part = blockIdx.x % a.parts, tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int vocab = (int)d.vocab, all = vocab / N, share = (all + a.parts - 1) / a.parts;
  const int c0 = min(all, part * share), chunks = min(all, (part + 1) * share);        // this part's pieces; the last part has what is behind them
  const float scale = d.scale * kLog2e;
  Running r;
  float own = kLowest, second = kLowest;                       // the largest logit of this thread, and of its other pieces
  int piece = -1;                                              // where the largest is
  float v[U][N];
  for (int c = c0 + tid; c < chunks; c += U * kThreads) {
#pragma unroll
    for (int i = 0; i < U; ++i) C::load(d.logits, from + (int64_t)min(c + i * kThreads, chunks - 1) * N, v[i]);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const bool in = c + i * kThreads < chunks;
      float here = -__builtin_inff();
#pragma unroll
      for (int n = 0; n < N; ++n) {
        v[i][n] = in ? v[i][n] : -__builtin_inff();
        here = fmaxf(here, v[i][n]);
      }
      second = fmaxf(second, fminf(own, here));
      piece = here > own ? c + i * kThreads : piece;
      own = fmaxf(own, here);
    }
    r.rebase(own, scale);
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int n = 0; n < N; ++n) r.add(v[i][n], scale);
  }
  const int tail = part == a.parts - 1 ? all * N + tid : vocab;                        // fewer than N elements
  if (tail < vocab) {
    const float x = C::one(d.logits, from + tail);
    r.rebase(fmaxf(r.m, x), scale);
    r.add(x, scale);
  }
  own = r.m;                                                   // its element behind the pieces among them
  float m = lanes_max<8>(own);
  if (lane % 8 == 0) maxima[tid / 8] = m;
  m = lanes_max<64>(own);
  if (lane == 0) red[0][wave] = m;
  if (tid == 0) { count = 0; winners = 0; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) m = fmaxf(m, red[0][w]);
  r.rebase(m, scale);
  float s = lanes_sum<64>(r.s), t = lanes_sum<64>(r.t);
  if (lane == 0) { red[1][wave] = s; red[2][wave] = t; }
  __syncthreads();
  s = t = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) { s += red[1][w]; t += red[2][w]; }
  const Finish f(m, s, d.scale);
  if (tid == 0) {
    if (a.parts == 1) f.write<TYPE>(d, row, t);
    else {
      float* to = a.stats + (row * a.parts + part) * 3;
      to[0] = m; to[1] = s; to[2] = t;
    }
  }
  const int top = d.top;
  if (!top || !(d.top_logp || d.top_index)) return;

  auto put = [&](int rank, uint64_t key) {
    if (a.parts == 1) f.put(d, row, rank, key);
    else a.best[(row * a.parts + part) * top + rank] = key;
  };
  const bool plain = s - s == 0.f && !f.empty;                 // NaN or infinite logits make s NaN
  if (plain) {
    // the smallest of the groups' maxima that fewer than top of them exceed; every wave for itself
    const float mine = maxima[lane % kGroups];
    int above = 0;
#pragma unroll
    for (int i = 0; i < kGroups; i += 4) {
      const float4 g = *reinterpret_cast<const float4*>(maxima + i);
      above += (g.x > mine) + (g.y > mine) + (g.z > mine) + (g.w > mine);
    }
    const float least = -lanes_max<64>(above < top ? -mine : -__builtin_inff());
    auto take = [&](float x, int index) {
      if (x >= least) {
        const int to = atomicAdd(&count, 1);
        if (to < kCandidates) found[to] = key_of(x, index);
      }
    };
    if (chunks - c0 <= U * kThreads) {                          // still in registers
      if (own >= least) {
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (c0 + tid + i * kThreads < chunks)
#pragma unroll
            for (int n = 0; n < N; ++n) take(v[i][n], (c0 + tid + i * kThreads) * N + n);
      }
    } else {
      // most find one piece with such elements and know it; others look through all of theirs, together
      float y[N];
      if (own >= least && second >= least) winner[atomicAdd(&winners, 1)] = (short)tid;
      else if (own >= least && piece >= 0) {
        C::load(d.logits, from + (int64_t)piece * N, y);
#pragma unroll
        for (int n = 0; n < N; ++n) take(y[n], piece * N + n);
      }
      __syncthreads();
      const int per = (chunks - c0 + kThreads - 1) / kThreads, items = winners * per;
      for (int i = tid; i < items; i += kThreads) {
        const int at = c0 + winner[i / per] + i % per * kThreads;
        if (at >= chunks) continue;
        C::load(d.logits, from + (int64_t)at * N, y);
#pragma unroll
        for (int n = 0; n < N; ++n) take(y[n], at * N + n);
      }
    }
    if (tail < vocab) take(C::one(d.logits, from + tail), tail);
    __syncthreads();
    if (count >= top && count <= kCandidates) {
      for (int i = tid; i < count; i += kThreads) {
        const uint64_t mine = found[i];
        const int n = count;
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) rank += found[j] > mine;
        if (rank < top) put(rank, mine);
      }
      return;
    }
  }
  // Rows with NaN, infinities, very many equal logits or fewer finite ones than are asked for: one pass for each alternative.
  const int begin = c0 * N, end = part == a.parts - 1 ? vocab : chunks * N;
  uint64_t last = 0;                                           // of the alternative before; the first has none (a NaN at index 0 is the largest key there is)
  for (int rank = 0; rank < top; ++rank) {
    uint64_t best = 0;
    for (int i = begin + tid; i < end; i += kThreads) {
      const uint64_t key = key_of(C::one(d.logits, from + i), i);
      if ((rank == 0 || key < last) && key > best) best = key;
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
    if (tid == 0) put(rank, best);                             // 0 where the part has no further element
    last = best;
  }
}

// Parts of a row to its results: one workgroup a row.
template <int TYPE>
__global__ void __launch_bounds__(256) token_logprobs_join_kernel(const LogpArgs a) {
  __shared__ uint64_t keys[kMostParts * SZO_LOGPROBS_MAX_TOP];
  const szo_logprobs_desc& d = a.d;
  const int64_t row = blockIdx.x;
  const float* part = a.stats + row * a.parts * 3;
  const float scale = d.scale * kLog2e;
  Running r;
  for (int i = 0; i < a.parts; ++i) r.m = fmaxf(r.m, part[3 * i]);
  for (int i = 0; i < a.parts; ++i) {
    Running p;
    p.m = part[3 * i]; p.s = part[3 * i + 1]; p.t = part[3 * i + 2];
    p.rebase(r.m, scale);
    r.s += p.s;
    r.t += p.t;
  }
  const Finish f(r.m, r.s, d.scale);
  if (threadIdx.x == 0) f.write<TYPE>(d, row, r.t);
  if (!d.top || !(d.top_logp || d.top_index)) return;
  const int n = a.parts * d.top;
  for (int i = threadIdx.x; i < n; i += 256) keys[i] = a.best[row * n + i];
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += 256) {
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += keys[j] > keys[i];
    if (rank < d.top && keys[i]) f.put(d, row, rank, keys[i]);
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

}  // namespace

int add_token_loss(const float* logp, const int32_t* targets, int64_t rows, int64_t vocab, double scale, double* loss_acc, hipStream_t s) {
  logp_loss_kernel<<<1, 1024, 0, s>>>(logp, targets, rows, vocab, scale, loss_acc);
  SZO_LAUNCH_CHECK();
  return SZO_OK;
}

namespace {

struct GradArgs { szo_logprobs_desc d; const float *g_logp, *g_entropy; void* out; int64_t out_stride; int parts; };

constexpr int kGradThreads = 256;
constexpr int kGradChunks = 4;             // 16-byte pieces of a thread, one after the other

// dx = scale (g (1[v = target] - p) - h p (log p + H)), p from the row's maximum and sum: logits are read once and as much is written, 16 bytes a
// lane, several workgroups a row.  A thread's four pieces come one after the other: the output may be the input, so no load passes a store.  Bound by memory:
// 4096 rows of 32000 in bf16 96 us, 5.5 TB/s of both.
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
    const float u = (x - m) * d.scale, p = __builtin_amdgcn_exp2f(u * kLog2e) * by;
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
  if (d->top < 0 || d->top > d->vocab || !(d->scale > 0.f && d->scale <= SZO_MOST_SCALE)) return SZO_EINVAL;
  if (d->top > SZO_LOGPROBS_MAX_TOP || d->vocab > (1 << 30) || d->rows > 0x7FFFFFFF) return SZO_EUNSUPPORTED;
  if (d->rows > 1 && d->row_stride < 0) return SZO_EINVAL;
  if (d->rows && d->vocab && (!d->logits || !aligned_to(d->logits, type_bytes(d->type)))) return SZO_EINVAL;
  if (!aligned_to(d->targets, 4) || !aligned_to(d->logp, 4) || !aligned_to(d->entropy, 4) || !aligned_to(d->stats, 4) || !aligned_to(d->top_logp, 4) ||
      !aligned_to(d->top_index, 4) || !aligned_to(d->loss_acc, 8)) return SZO_EINVAL;
  return SZO_OK;
}

// With few rows a row goes to several workgroups, 64 KiB of it at least to each.  us of 1 / 16 / 64 rows of fp32 with 5 alternatives, whole and in parts:
// vocabulary of 131072 17, 18, 25 -> 9.5, 10.1, 13.4; of 50257 9.4, 10.2, 12.5 -> 9.0, 9.8, 11.1; of 32000 7.2, 7.7, 8.2 whole, 8.0, 8.9, 9.3 in parts of 32 KiB.
struct Plan { int parts; };
Plan plan_of(const szo_logprobs_desc* d) {
  Plan p;
  const int64_t pieces = d->vocab * (int64_t)type_bytes(d->type) / 16;
  p.parts = d->rows == 0 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>({pieces / 4096, 512 / d->rows, kMostParts}));
  return p;
}
size_t best_at(const szo_logprobs_desc* d, const Plan& p) { return ((size_t)d->rows * p.parts * 3 * sizeof(float) + 15) / 16 * 16; }

template <int TYPE>
void launch(const LogpArgs& a, const Plan& p, hipStream_t s) {
  token_logprobs_kernel<TYPE><<<dim3((unsigned)(a.d.rows * p.parts)), kThreads, 0, s>>>(a);
  if (p.parts > 1) token_logprobs_join_kernel<TYPE><<<dim3((unsigned)a.d.rows), 256, 0, s>>>(a);
}

}  // namespace
}  // namespace szo

using namespace szo;

extern "C" {

size_t szo_logprobs_workspace_bytes(const szo_logprobs_desc* d) {
  if (check(d) != SZO_OK) return 16;
  const Plan p = plan_of(d);
  return p.parts == 1 ? 16 : best_at(d, p) + (size_t)d->rows * p.parts * d->top * sizeof(uint64_t);
}

int szo_token_logprobs(const szo_logprobs_desc* d, void* workspace, void* stream) {
  const int rc = check(d);
  if (rc != SZO_OK) return rc;
  if (d->loss_acc && !d->logp) return SZO_EINVAL;
  if (d->rows == 0) return SZO_OK;
  if (d->vocab == 0) return SZO_EINVAL;
  const Plan p = plan_of(d);
  if (d->rows * p.parts > 0xFFFFFFFFll / kThreads) return SZO_EUNSUPPORTED;            // a launch counts its threads in 32 bits
  if (p.parts > 1 && (!workspace || !aligned_to(workspace, 16))) return SZO_EINVAL;
  hipStream_t s = (hipStream_t)stream;
  const LogpArgs a = {*d, p.parts, (float*)workspace, p.parts > 1 ? (uint64_t*)((char*)workspace + best_at(d, p)) : nullptr};
  if (d->type == SZO_F32) launch<SZO_F32>(a, p, s);
  else if (d->type == SZO_BF16) launch<SZO_BF16>(a, p, s);
  else launch<SZO_F16>(a, p, s);
  SZO_LAUNCH_CHECK();
  return d->loss_acc ? add_token_loss(d->logp, d->targets, d->rows, d->vocab, d->loss_scale, d->loss_acc, s) : SZO_OK;
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
  if (d->rows * a.parts > 0xFFFFFFFFll / kGradThreads) return SZO_EUNSUPPORTED;
  hipStream_t s = (hipStream_t)stream;
  const dim3 grid((unsigned)(d->rows * a.parts));
  if (d->type == SZO_F32) token_logprobs_bwd_kernel<SZO_F32><<<grid, kGradThreads, 0, s>>>(a);
  else if (d->type == SZO_BF16) token_logprobs_bwd_kernel<SZO_BF16><<<grid, kGradThreads, 0, s>>>(a);
  else token_logprobs_bwd_kernel<SZO_F16><<<grid, kGradThreads, 0, s>>>(a);
  SZO_LAUNCH_CHECK();
  return SZO_OK;
}

}  // extern "C"
