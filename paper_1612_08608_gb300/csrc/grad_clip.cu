// asap_clip_grads and asap_sgd_clipped: the norm of each worker's gradient over
// many tensors, and the gradients scaled to a largest norm or the SGD step
// (Eq. A.1, first line) taken with them.
//
//   norm_k  = sqrt(sum over the tensors of group k of g^2)
//   scale_k = max_norm / norm_k where norm_k > max_norm, else 1
//   out     = scale_k g                                   (clip)
//   w       = (1 - lr l2) w - lr scale_k g; copy = w      (step)
//
// Two launches: every gradient is read for the norms, then once more to be
// scaled.  Tensors are cut into chunks of kChunk elements, sorted by group; block
// b takes the chunks [b per, (b + 1) per), so that the partial sum of (block b,
// group k) has the slot b + k: no two share one, a group's lie side by side, and
// no ticket, atomic or clearing of the workspace is needed.  Each block of the
// second launch adds up the slots of the groups that it meets, all in the same
// order.  The second launch walks the chunks backwards: what the first one read
// last is still in L2.
//
// Squares are added in fp32 per thread and chunk, the chunks' sums as
// float-float pairs, and the threads' sums in fp64.  Where fp32 squares overflow
// or vanish, the thread adds its elements of the chunk again in fp64.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "asap_internal.h"

namespace asap {
void set_thread_error(const char* msg);
}

namespace {

using namespace asap;

constexpr int kThreads = 256;
constexpr int kBlocksPerSm = 6;
constexpr int kChunk = 16384;                // elements
constexpr int kStepUnroll = 2;             // groups of eight elements of the step in flight, a thread
constexpr int kMaxBlocks = 1024;             // slots for partial sums: this and one for each group
constexpr int kMaxGroups = 65536;

struct Tensor {
  const void* g;
  void* a;               // clip: the scaled gradient; step: the fp32 parameters
  void* c;               // step: their 16-bit copy (may be NULL)
  long long n;
  int chunk0;            // number of the first chunk
  int group;
  int gchunk0, gchunk1;  // chunks of the whole group
  unsigned char type;    // of g (and of a, for a clip)
  unsigned char ctype;   // of c
  unsigned char head;    // elements before the first chunk's vectors
  unsigned char vec;     // a and c are aligned there too
};

// The tables travel as kernel arguments: nothing is copied, and a captured
// launch keeps its own.  A small one keeps the launch of a small call short.
template <int T>
struct Args {
  Tensor t[T];
  int count;
  int chunk_begin, chunk_end;   // of this launch
  int per;                      // chunks per block
  int first_block;
  float max_norm;
  float decay, lr;              // step
  double* partial;
  float* norms;
};

constexpr int kSmallTable = 32, kLargeTable = 576;
static_assert(sizeof(Args<kLargeTable>) <= 32764, "kernel arguments");

struct Pair {
  float hi, lo;
};

// Knuth's two-sum: the rounding error of the high parts' sum is kept in lo.
__device__ __forceinline__ Pair pair_add(Pair a, float b) {
  const float s = a.hi + b;
  const float bv = s - a.hi;
  const float e = ((a.hi - (s - bv)) + (b - bv)) + a.lo;
  const float hi = s + e;
  return Pair{hi, e - (hi - s)};
}

__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float as_float(__half v) { return __half2float(v); }
template <typename E>
__device__ __forceinline__ E from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// 16 bytes of E.
template <typename E>
struct alignas(16) Vec {
  static constexpr int kN = 16 / sizeof(E);
  E e[kN];
};

template <typename E>
__device__ __forceinline__ Vec<E> load_vec(const E* p) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  Vec<E> v;
  *reinterpret_cast<uint4*>(&v) = u;
  return v;
}

template <typename E>
__device__ __forceinline__ void store_vec(E* p, const Vec<E>& v) {
  *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(&v);
}

// Elements [begin, end) of chunk j of a tensor; the part from `body` on starts
// at a 16-byte boundary of g.
struct Range {
  long long begin, body, end;
};

__device__ __forceinline__ Range chunk_range(const Tensor& t, int j) {
  Range r;
  const long long aligned = t.head + static_cast<long long>(j) * kChunk;
  r.begin = j ? aligned : 0;
  r.body = aligned < t.n ? aligned : t.n;
  r.end = aligned + kChunk < t.n ? aligned + kChunk : t.n;
  return r;
}

template <int T>
__device__ __forceinline__ int tensor_of(const Args<T>& a, int chunk) {
  int lo = 0, hi = a.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.t[mid].chunk0 <= chunk) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Sum over the block in a fixed order, in every thread.
__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  double t = 0.0;
  for (int w = 0; w < kThreads / 32; ++w) t += red[w];
  return t;
}

// This thread's sum of squares of a chunk.
template <typename E>
__device__ __forceinline__ double chunk_squares(const E* g, const Range& r, Pair& total) {
  constexpr int kN = Vec<E>::kN;
  const long long nv = (r.end - r.body) / kN;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  bool seen = false;     // an element that is not zero
  const E* body = g + r.body;
  long long v = threadIdx.x;
  for (; v + 3 * kThreads < nv; v += 4 * kThreads) {
    Vec<E> x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] = load_vec(body + (v + u * kThreads) * kN);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int e = 0; e < kN; ++e) {
        const float f = as_float(x[u].e[e]);
        s[u] = fmaf(f, f, s[u]);
        seen |= f != 0.f;
      }
  }
  for (; v < nv; v += kThreads) {
    const Vec<E> x = load_vec(body + v * kN);
#pragma unroll
    for (int e = 0; e < kN; ++e) {
      const float f = as_float(x.e[e]);
      s[e & 3] = fmaf(f, f, s[e & 3]);
      seen |= f != 0.f;
    }
  }
  const long long tail = r.body + nv * kN;
  const long long loose = (r.body - r.begin) + (r.end - tail);     // fewer than 2 kN
  const long long at = threadIdx.x < r.body - r.begin ? r.begin + threadIdx.x : tail + (threadIdx.x - (r.body - r.begin));
  if (threadIdx.x < loose) {
    const float f = as_float(g[at]);
    s[0] = fmaf(f, f, s[0]);
    seen |= f != 0.f;
  }
  const float sum = (s[0] + s[1]) + (s[2] + s[3]);
  // What squares below 2^-126 lose is nothing beside a sum above 2^-100, and the
  // sums of 2^27 chunks below 2^100 do not overflow.
  if (!seen || (sum >= 0x1p-100f && sum < 0x1p+100f)) {
    total = pair_add(total, sum);
    return 0.0;
  }
  double w = 0.0;
  for (v = threadIdx.x; v < nv; v += kThreads)
    for (int e = 0; e < kN; ++e) {
      const double f = as_float(body[v * kN + e]);
      w += f * f;
    }
  if (threadIdx.x < loose) {
    const double f = as_float(g[at]);
    w += f * f;
  }
  return w;
}

template <int T>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) k_grad_squares(const __grid_constant__ Args<T> a) {
  __shared__ double red[kThreads / 32];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int b = a.first_block + blockIdx.x;
  const int begin = max(a.chunk_begin, b * a.per);
  const int end = static_cast<int>(min(static_cast<long long>(a.chunk_end), (b + 1LL) * a.per));
  if (begin >= end) return;
  int ti = tensor_of(a, begin);
  Pair total{0.f, 0.f};
  double wide = 0.0;
  auto flush = [&](int i) {
    const Tensor& t = a.t[i];
    const double sum = block_sum(static_cast<double>(total.hi) + static_cast<double>(total.lo) + wide, red);
    // the part of this (block, group) that an earlier launch summed
    const bool more = max(b * a.per, t.gchunk0) < a.chunk_begin;
    if (threadIdx.x == 0) a.partial[b + t.group] = more ? a.partial[b + t.group] + sum : sum;
    total = Pair{0.f, 0.f};
    wide = 0.0;
  };
  for (int c = begin; c < end; ++c) {
    while (ti + 1 < a.count && a.t[ti + 1].chunk0 <= c) {
      if (a.t[ti + 1].group != a.t[ti].group) flush(ti);
      ++ti;
    }
    const Tensor& t = a.t[ti];
    const Range r = chunk_range(t, c - t.chunk0);
    switch (t.type) {
      case ASAP_F32: wide += chunk_squares(static_cast<const float*>(t.g), r, total); break;
      case ASAP_BF16: wide += chunk_squares(static_cast<const __nv_bfloat16*>(t.g), r, total); break;
      default: wide += chunk_squares(static_cast<const __half*>(t.g), r, total); break;
    }
  }
  flush(ti);
}

// The norm of a group, the same in every thread and block.
template <int T>
__device__ __forceinline__ float group_norm(const Args<T>& a, const Tensor& t, double* red) {
  double v = 0.0;
  const int b1 = (t.gchunk1 - 1) / a.per;
  for (int b = t.gchunk0 / a.per + threadIdx.x; b <= b1; b += kThreads) v += __ldcg(a.partial + b + t.group);
  return static_cast<float>(sqrt(block_sum(v, red)));
}

__device__ __forceinline__ float group_scale(float norm, float max_norm) {
  return norm > max_norm && norm < INFINITY ? max_norm / norm : 1.f;
}

template <typename E>
__device__ __forceinline__ void scale_chunk(const Tensor& t, const Range& r, float scale) {
  constexpr int kN = Vec<E>::kN;
  const E* g = static_cast<const E*>(t.g);
  E* o = static_cast<E*>(t.a);
  if (!t.vec) {
    for (long long i = r.begin + threadIdx.x; i < r.end; i += kThreads) o[i] = from_float<E>(as_float(g[i]) * scale);
    return;
  }
  const long long nv = (r.end - r.body) / kN;
  const E* gb = g + r.body;
  E* ob = o + r.body;
  long long v = threadIdx.x;
  for (; v + 3 * kThreads < nv; v += 4 * kThreads) {
    Vec<E> x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] = load_vec(gb + (v + u * kThreads) * kN);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
#pragma unroll
      for (int e = 0; e < kN; ++e) x[u].e[e] = from_float<E>(as_float(x[u].e[e]) * scale);
      store_vec(ob + (v + u * kThreads) * kN, x[u]);
    }
  }
  for (; v < nv; v += kThreads) {
    Vec<E> x = load_vec(gb + v * kN);
#pragma unroll
    for (int e = 0; e < kN; ++e) x.e[e] = from_float<E>(as_float(x.e[e]) * scale);
    store_vec(ob + v * kN, x);
  }
  const long long tail = r.body + nv * kN, head = r.body - r.begin;
  if (threadIdx.x < head + (r.end - tail)) {
    const long long at = threadIdx.x < head ? r.begin + threadIdx.x : tail + (threadIdx.x - head);
    o[at] = from_float<E>(as_float(g[at]) * scale);
  }
}

// 32 bytes at a time: two vectors.
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  uint32_t u[8];
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]) : "l"(p));
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(u[e]);
}

__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               :: "l"(p), "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])),
                  "r"(__float_as_uint(v[3])), "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])),
                  "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7])) : "memory");
}

template <typename E>
__device__ __forceinline__ void load8(const E* p, float (&v)[8]) {
  const Vec<E> x = load_vec(p);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = as_float(x.e[e % Vec<E>::kN]);
}

template <typename E, typename H, bool kCopy>
__device__ __forceinline__ void step_chunk(const Tensor& t, const Range& r, float decay, float rate) {
  constexpr int kN = 8;                             // 32 bytes of parameters
  const E* g = static_cast<const E*>(t.g);
  float* w = static_cast<float*>(t.a);
  H* c = static_cast<H*>(t.c);
  auto one = [&](long long i) {
    const float x = fmaf(-rate, as_float(g[i]), decay * w[i]);
    w[i] = x;
    if (kCopy) c[i] = from_float<H>(x);
  };
  if (!t.vec) {
    for (long long i = r.begin + threadIdx.x; i < r.end; i += kThreads) one(i);
    return;
  }
  const long long nv = (r.end - r.body) / kN;
  auto step = [&](long long i, const float (&gv)[8], float (&p)[8]) {
#pragma unroll
    for (int e = 0; e < kN; ++e) p[e] = fmaf(-rate, gv[e], decay * p[e]);
    store8(w + i, p);
    if (kCopy) {
      Vec<H> q;
#pragma unroll
      for (int e = 0; e < kN; ++e) q.e[e] = from_float<H>(p[e]);
      store_vec(c + i, q);
    }
  };
  long long v = threadIdx.x;
  for (; v + (kStepUnroll - 1) * kThreads < nv; v += kStepUnroll * kThreads) {
    float gv[kStepUnroll][8], p[kStepUnroll][8];
#pragma unroll
    for (int u = 0; u < kStepUnroll; ++u) {
      load8(g + r.body + (v + u * kThreads) * kN, gv[u]);
      load8(w + r.body + (v + u * kThreads) * kN, p[u]);
    }
#pragma unroll
    for (int u = 0; u < kStepUnroll; ++u) step(r.body + (v + u * kThreads) * kN, gv[u], p[u]);
  }
  for (; v < nv; v += kThreads) {
    float gv[8], p[8];
    load8(g + r.body + v * kN, gv);
    load8(w + r.body + v * kN, p);
    step(r.body + v * kN, gv, p);
  }
  const long long tail = r.body + nv * kN, head = r.body - r.begin;
  if (threadIdx.x < head + (r.end - tail)) one(threadIdx.x < head ? r.begin + threadIdx.x : tail + (threadIdx.x - head));
}

template <typename E>
__device__ __forceinline__ void step_any(const Tensor& t, const Range& r, float decay, float rate) {
  if (!t.c) step_chunk<E, __nv_bfloat16, false>(t, r, decay, rate);
  else if (t.ctype == ASAP_BF16) step_chunk<E, __nv_bfloat16, true>(t, r, decay, rate);
  else step_chunk<E, __half, true>(t, r, decay, rate);
}

enum Mode { kNormOnly, kClip, kStep };

template <int T, int M>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) k_grad_apply(const __grid_constant__ Args<T> a) {
  __shared__ double red[kThreads / 32];
  const int b = a.first_block + blockIdx.x;
  const int begin = max(a.chunk_begin, b * a.per);
  const int end = static_cast<int>(min(static_cast<long long>(a.chunk_end), (b + 1LL) * a.per));
  if (begin >= end) return;
  int ti = tensor_of(a, end - 1);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  int group = -1;
  float scale = 1.f;
  bool skip = false;
  for (int c = end - 1; c >= begin; --c) {
    while (a.t[ti].chunk0 > c) --ti;
    const Tensor& t = a.t[ti];
    if (t.group != group) {
      group = t.group;
      const float norm = group_norm(a, t, red);
      scale = group_scale(norm, a.max_norm);
      skip = M == kNormOnly || (M == kStep && !(norm < INFINITY));   // a gradient that is not finite takes no step
      // the block with the group's first chunk reports its norm
      if (t.gchunk0 >= b * a.per && threadIdx.x == 0) a.norms[group] = norm;
    }
    if (skip || (M == kClip && scale == 1.f && t.a == t.g)) continue;
    const Range r = chunk_range(t, c - t.chunk0);
    if (M == kClip) {
      switch (t.type) {
        case ASAP_F32: scale_chunk<float>(t, r, scale); break;
        case ASAP_BF16: scale_chunk<__nv_bfloat16>(t, r, scale); break;
        default: scale_chunk<__half>(t, r, scale); break;
      }
    } else if (M == kStep) {
      switch (t.type) {
        case ASAP_F32: step_any<float>(t, r, a.decay, a.lr * scale); break;
        case ASAP_BF16: step_any<__nv_bfloat16>(t, r, a.decay, a.lr * scale); break;
        default: step_any<__half>(t, r, a.decay, a.lr * scale); break;
      }
    }
  }
}

asap_status reject(const char* msg) {
  set_thread_error(msg);
  return ASAP_ERR_ARG;
}

inline int bytes_of(int type) { return type == ASAP_F32 ? 4 : 2; }

struct Call {
  int count;
  const void* const* grads;
  void* const* a;
  void* const* c;
  const int64_t* numel;
  const int32_t* dtypes;
  const int32_t* cdtypes;
  const int32_t* groups;
  int n_groups;
  float max_norm, decay, lr;
  float* norms;
  void* workspace;
  size_t workspace_bytes;
  cudaStream_t stream;
  int mode;
};

size_t workspace_of(int n_groups) { return 8 * (static_cast<size_t>(kMaxBlocks) + static_cast<size_t>(n_groups)); }

// Written ranges must not meet each other, nor a gradient other than the one
// that the same tensor is scaled in place from.
bool ranges_meet(const Call& k) {
  struct R {
    uintptr_t begin, end;
    int tensor;
    bool written;
  };
  std::vector<R> v;
  v.reserve(3 * static_cast<size_t>(k.count));
  for (int i = 0; i < k.count; ++i) {
    if (k.numel[i] == 0) continue;
    const uintptr_t n = static_cast<uintptr_t>(k.numel[i]), g = reinterpret_cast<uintptr_t>(k.grads[i]);
    const int es = bytes_of(k.dtypes[i]);
    const uintptr_t a = reinterpret_cast<uintptr_t>(k.a[i]);
    if (k.mode == kClip && a == g) {
      v.push_back({g, g + n * es, i, true});
      continue;
    }
    v.push_back({g, g + n * es, i, false});
    v.push_back({a, a + n * (k.mode == kClip ? es : 4), i, true});
    if (k.c && k.c[i]) {
      const uintptr_t c = reinterpret_cast<uintptr_t>(k.c[i]);
      v.push_back({c, c + n * 2, i, true});
    }
  }
  std::sort(v.begin(), v.end(), [](const R& x, const R& y) { return x.begin < y.begin; });
  uintptr_t end = 0, wend = 0;                       // furthest ends of any range, and of a written one
  for (const R& r : v) {
    if (r.begin < wend || (r.written && r.begin < end)) return true;
    end = std::max(end, r.end);
    if (r.written) wend = std::max(wend, r.end);
  }
  return false;
}

template <int T>
cudaError_t launch(const Call& k, const std::vector<Tensor>& tensors, int chunks, int per) {
  Args<T> a;
  a.per = per;
  a.max_norm = k.max_norm;
  a.decay = k.decay;
  a.lr = k.lr;
  a.partial = static_cast<double*>(k.workspace);
  a.norms = k.norms;
  const int total = static_cast<int>(tensors.size());
  const int parts = (total + T - 1) / T;
  for (int pass = 0; pass < 2; ++pass)
    for (int q = 0; q < parts; ++q) {
      const int part = pass ? parts - 1 - q : q;     // the second pass goes backwards
      const int t0 = part * T;
      a.count = std::min(T, total - t0);
      std::copy(tensors.begin() + t0, tensors.begin() + t0 + a.count, a.t);
      a.chunk_begin = a.t[0].chunk0;
      a.chunk_end = t0 + a.count < total ? tensors[t0 + a.count].chunk0 : chunks;
      a.first_block = a.chunk_begin / per;
      const int blocks = (a.chunk_end - 1) / per - a.first_block + 1;
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3(blocks);
      cfg.blockDim = dim3(kThreads);
      cfg.stream = k.stream;
      cudaLaunchAttribute attr[1];
      attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
      attr[0].val.programmaticStreamSerializationAllowed = 1;
      cfg.attrs = attr;
      cfg.numAttrs = pass && q == 0 ? 1 : 0;         // the first launch after the squares' last
      cudaError_t e;
      if (pass == 0) e = cudaLaunchKernelEx(&cfg, k_grad_squares<T>, a);
      else if (k.mode == kNormOnly) e = cudaLaunchKernelEx(&cfg, k_grad_apply<T, kNormOnly>, a);
      else if (k.mode == kClip) e = cudaLaunchKernelEx(&cfg, k_grad_apply<T, kClip>, a);
      else e = cudaLaunchKernelEx(&cfg, k_grad_apply<T, kStep>, a);
      if (e != cudaSuccess) return e;
    }
  return cudaSuccess;
}

asap_status run(const Call& k, const char* const* why) {
  if (k.count < 0 || k.n_groups < 1 || k.n_groups > kMaxGroups) return reject(why[0]);
  if (!k.norms || !k.workspace || (k.count > 0 && (!k.grads || !k.numel || !k.dtypes || (k.mode != kNormOnly && !k.a))))
    return reject(why[1]);
  if (k.workspace_bytes < workspace_of(k.n_groups) || (reinterpret_cast<uintptr_t>(k.workspace) & 7u) ||
      (reinterpret_cast<uintptr_t>(k.norms) & 3u))
    return reject(why[2]);
  if (!(k.max_norm > 0.f)) return reject(why[3]);
  std::vector<int> order;
  order.reserve(k.count);
  std::vector<char> has(k.n_groups, 0);
  bool sorted = true;
  long long chunks = 0;
  for (int i = 0; i < k.count; ++i) {
    const int type = k.dtypes[i], group = k.groups ? k.groups[i] : 0;
    if (type != ASAP_F32 && type != ASAP_BF16 && type != ASAP_F16) return reject(why[4]);
    if (group < 0 || group >= k.n_groups) return reject(why[5]);
    if (k.numel[i] < 0 || k.numel[i] > (1LL << 40)) return reject(why[6]);
    if (k.numel[i] == 0) continue;
    uintptr_t low = reinterpret_cast<uintptr_t>(k.grads[i]) & (bytes_of(type) - 1);
    if (!k.grads[i]) return reject(why[1]);
    if (k.mode != kNormOnly) {
      if (!k.a[i]) return reject(why[1]);
      low |= reinterpret_cast<uintptr_t>(k.a[i]) & ((k.mode == kClip ? bytes_of(type) : 4) - 1);
    }
    if (k.c && k.c[i]) {
      if (!k.cdtypes || (k.cdtypes[i] != ASAP_BF16 && k.cdtypes[i] != ASAP_F16)) return reject(why[4]);
      low |= reinterpret_cast<uintptr_t>(k.c[i]) & 1u;
    }
    if (low) return reject(why[7]);
    if (!order.empty() && k.groups && k.groups[order.back()] > group) sorted = false;
    has[group] = 1;
    order.push_back(i);
  }
  if (k.mode != kNormOnly && ranges_meet(k)) return reject(why[8]);
  if (!sorted)
    std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return k.groups[x] < k.groups[y]; });
  std::vector<Tensor> tensors(order.size());
  for (size_t j = 0; j < order.size(); ++j) {
    const int i = order[j];
    Tensor& t = tensors[j];
    t.g = k.grads[i];
    t.a = k.mode == kNormOnly ? nullptr : k.a[i];
    t.c = k.c ? k.c[i] : nullptr;
    t.n = k.numel[i];
    t.group = k.groups ? k.groups[i] : 0;
    t.type = static_cast<unsigned char>(k.dtypes[i]);
    t.ctype = static_cast<unsigned char>(t.c ? k.cdtypes[i] : 0);
    const int es = bytes_of(t.type);
    // The first element from which g and whatever the second pass moves beside it
    // are aligned (the step takes eight elements at a time); none: g's own boundary.
    const uintptr_t g = reinterpret_cast<uintptr_t>(t.g), w = reinterpret_cast<uintptr_t>(t.a),
                    c = reinterpret_cast<uintptr_t>(t.c);
    auto aligned = [&](uintptr_t h) {
      if (k.mode != kStep) return ((g + h * es) & 15u) == 0 && (k.mode == kNormOnly || ((w + h * es) & 15u) == 0);
      return ((g + h * es) & (8 * es - 1)) == 0 && ((w + h * 4) & 31u) == 0 && (!t.c || ((c + h * 2) & 15u) == 0);
    };
    uintptr_t head = 0;
    while (head < 16 && !aligned(head)) ++head;
    t.vec = head < 16;
    if (!t.vec) head = ((16 - (g & 15u)) & 15u) / es;
    t.head = static_cast<unsigned char>(std::min<long long>(static_cast<long long>(head), t.n));
    t.chunk0 = static_cast<int>(chunks);
    chunks += std::max<long long>(1, (t.n - t.head + kChunk - 1) / kChunk);
    if (chunks > INT32_MAX / 2) return reject(why[6]);
  }
  for (size_t j = 0; j < tensors.size();) {
    size_t e = j;
    while (e < tensors.size() && tensors[e].group == tensors[j].group) ++e;
    const int c1 = e < tensors.size() ? tensors[e].chunk0 : static_cast<int>(chunks);
    const int c0 = tensors[j].chunk0;
    for (; j < e; ++j) {
      tensors[j].gchunk0 = c0;
      tensors[j].gchunk1 = c1;
    }
  }
  // groups without an element have the norm 0
  for (int g = 0; g < k.n_groups; ++g)
    if (!has[g]) {
      if (cudaMemsetAsync(k.norms, 0, 4 * static_cast<size_t>(k.n_groups), k.stream) != cudaSuccess) {
        set_thread_error("clearing the norms failed");
        return ASAP_ERR_CUDA;
      }
      break;
    }
  if (tensors.empty()) return ASAP_OK;
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1) {
    set_thread_error("no usable current device");
    return ASAP_ERR_CUDA;
  }
  const int blocks = std::min(kMaxBlocks, kBlocksPerSm * sms);
  const int per = static_cast<int>((chunks + blocks - 1) / blocks);
  const cudaError_t e = tensors.size() <= kSmallTable ? launch<kSmallTable>(k, tensors, static_cast<int>(chunks), per)
                                                      : launch<kLargeTable>(k, tensors, static_cast<int>(chunks), per);
  if (e != cudaSuccess) {
    cudaGetLastError();
    set_thread_error(cudaGetErrorString(e));
    return ASAP_ERR_CUDA;
  }
  return ASAP_OK;
}

asap_status guarded(const Call& k, const char* const* why) {
  try {
    return run(k, why);
  } catch (const std::bad_alloc&) {
    set_thread_error("out of host memory");
    return ASAP_ERR_OOM;
  } catch (...) {
    set_thread_error("unexpected error on the host");
    return ASAP_ERR_CUDA;
  }
}

#define ASAP_CLIP_REASONS(f)                                                                                    \
  {f ": need count >= 0 and 1 <= n_groups <= 65536", f ": NULL pointer",                                        \
   f ": workspace too small, or workspace or norms not aligned", f ": need max_norm > 0", f ": unknown type",   \
   f ": group out of range", f ": element count out of range", f ": a tensor is not aligned to its type",       \
   f ": written tensors overlap each other or a gradient"}

}  // namespace

extern "C" asap_status asap_clip_workspace(int n_groups, uint64_t* bytes) {
  if (!bytes || n_groups < 1 || n_groups > kMaxGroups)
    return reject("asap_clip_workspace: need bytes and 1 <= n_groups <= 65536");
  *bytes = workspace_of(n_groups);
  return ASAP_OK;
}

extern "C" asap_status asap_clip_grads(int count, const void* const* grads, void* const* out, const int64_t* numel,
                                       const int32_t* dtypes, const int32_t* groups, int n_groups, float max_norm,
                                       float* norms_out, void* workspace, uint64_t workspace_bytes, void* cuda_stream) {
  static const char* const why[] = ASAP_CLIP_REASONS("asap_clip_grads");
  Call k = {count, grads, out, nullptr, numel, dtypes, nullptr, groups, n_groups, max_norm, 0.f, 0.f, norms_out,
            workspace, static_cast<size_t>(workspace_bytes), static_cast<cudaStream_t>(cuda_stream),
            out ? kClip : kNormOnly};
  return guarded(k, why);
}

extern "C" asap_status asap_sgd_clipped(int count, float* const* params, void* const* copies,
                                        const int32_t* copy_dtypes, const void* const* grads, const int64_t* numel,
                                        const int32_t* dtypes, const int32_t* groups, int n_groups, float max_norm,
                                        float lr, float l2, float* norms_out, void* workspace,
                                        uint64_t workspace_bytes, void* cuda_stream) {
  static const char* const why[] = ASAP_CLIP_REASONS("asap_sgd_clipped");
  if (!(lr > 0.f) || !(l2 >= 0.f) || !(lr * l2 < 1.f))
    return reject("asap_sgd_clipped: need lr > 0, l2 >= 0 and lr*l2 < 1");
  if (count > 0 && !params) return reject(why[1]);
  Call k = {count, grads, reinterpret_cast<void* const*>(params), copies, numel, dtypes, copy_dtypes, groups, n_groups,
            max_norm, 1.f - lr * l2, lr, norms_out, workspace, static_cast<size_t>(workspace_bytes),
            static_cast<cudaStream_t>(cuda_stream), kStep};
  return guarded(k, why);
}
