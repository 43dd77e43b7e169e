// Logits adjusted before a label is taken from them: penalties for repeated labels, biases,
// masks (a bit per label, or the labels that leave a state of a decoding graph), and
// optionally the log-softmax of what is left.
//
// One workgroup takes up to `per` columns of a row: its logits are asked for first and stay in
// registers (16 bytes a lane and access); meanwhile the counts of the row's history and the
// bits of its state's arcs are gathered in LDS, from which each lane takes its columns'.  The
// history and the arcs are read again by each workgroup of a row, for the columns of its own.
// Bound: memory (a logit is read and written once; MI355X, 2,048 x 5,000 fp32 with a history of 120,
// a graph and the log-softmax 22 us: 82 MB, which repeated passes find in part in the last-level
// cache), the scan of long histories (512 x 46,340 bf16 with up to 2,000 labels each 37 us, 23
// without), and for few rows latency: state, arc range, arcs, and the history are dependent round
// trips (128 x 500 4.6 us).  A log-softmax over more columns than a workgroup holds takes two
// passes: sums first, then everything again with the row's normaliser (512 x 46,340 bf16 48 us, 23
// without it).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "internal.h"
#include "types.h"

namespace tbs {
namespace {

constexpr int kThreads = 256;
constexpr int kCols = 8192;  // most columns of a workgroup: 32 per lane, counts in 32 KiB

__device__ __forceinline__ float ninff() { return -__builtin_inff(); }

// (m, s) stands for e^m s; s may be NaN, m never is
struct LogSum {
  float m, s;
  __device__ __forceinline__ void add(LogSum o) {
    const float mm = fmaxf(m, o.m);
    s = (m == mm ? s : s * __expf(m - mm)) + (o.m == mm ? o.s : o.s * __expf(o.m - mm));
    m = mm;
  }
  // log of e^x over it, for x a term that is not -inf (an empty sum has none): x - m loses little or
  // nothing, as m + log(s) would where m is large
  struct Log {
    float m, logs;
    __device__ __forceinline__ float of(float x) const { return (x - m) - logs; }
  };
  __device__ __forceinline__ Log log() const { return Log{m, logf(s)}; }
};

__device__ __forceinline__ LogSum workgroup_sum(LogSum v, LogSum* red) {
  for (int d = 32; d; d >>= 1) v.add(LogSum{__shfl_xor(v.m, d), __shfl_xor(v.s, d)});
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) v.add(red[w]);
  return v;
}

// kDirect: everything in one pass (a log-softmax: the row in one workgroup); kSums, kApply: the
// two passes of a log-softmax in parts.
enum { kDirect, kSums, kApply };

// Q: accesses of a lane, Q * E * kThreads >= p.per
template <class T, int Q, int PASS>
__global__ __launch_bounds__(kThreads) void k_adjust(AdjustArgs p) {
  constexpr int E = 16 / (int)sizeof(T), W = Q * E * kThreads;
  __shared__ __align__(16) int count[W];
  __shared__ uint32_t arcs[W / 32];
  __shared__ LogSum red[kThreads / 64];
  const int r = blockIdx.x / p.parts, part = blockIdx.x % p.parts, tid = threadIdx.x;
  const int c0 = part * p.per, n = min(p.per, p.V - c0);
  const T* z = (const T*)p.logits + (size_t)r * p.ldz + c0;
  // the lane's columns: q-th access at (q * kThreads + tid) * E
  Vec<T, E> in[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int c = (q * kThreads + tid) * E;
    in[q] = Vec<T, E>{};
    if (c + E <= n) {
      in[q] = load_vec<T, E>(z + c);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (c + e < n) in[q].v[e] = z[c + e];
    }
  }
  bool masked = false;
  int lo = 0, hi = 0;
  if (p.graph_rp) {
    const int s = p.states[r];
    masked = s >= 0 && s < p.S;
    if (masked) {
      lo = p.graph_rp[s];
      hi = p.graph_rp[s + 1];
    }
  }
  const int* hist = p.history ? p.history + (size_t)r * p.ldh : nullptr;
  const int len = !hist ? 0 : p.hlen ? min(max(p.hlen[r], 0), p.L) : p.L;
  float rep = p.repetition, pres = p.presence, freq = p.frequency;
  if (p.row_penalties) {
    rep = p.row_penalties[3 * (size_t)r];
    pres = p.row_penalties[3 * (size_t)r + 1];
    freq = p.row_penalties[3 * (size_t)r + 2];
  }
  if (len > 0 || masked) {  // (alike for the whole workgroup)
    if (len > 0)
#pragma unroll
      for (int q = 0; q < W / 4 / kThreads; ++q)
        *reinterpret_cast<int4*>(count + 4 * (q * kThreads + tid)) = make_int4(0, 0, 0, 0);
    for (int i = tid; i < W / 32; i += kThreads) arcs[i] = 0;
    __syncthreads();
    for (unsigned i = 4 * tid; i < (unsigned)len; i += 4 * kThreads) {
      Vec<int, 4> h = {{-1, -1, -1, -1}};
      if (i + 4 <= (unsigned)len) {
        h = load_vec<int, 4>(hist + i);
      } else {
#pragma unroll
        for (unsigned k = 0; k < 4; ++k)
          if (i + k < (unsigned)len) h.v[k] = hist[i + k];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const unsigned c = (unsigned)h.v[k] - (unsigned)c0;
        if (h.v[k] >= 0 && c < (unsigned)n) atomicAdd(&count[c], 1);
      }
    }
    for (unsigned i = (unsigned)lo + tid; i < (unsigned)hi; i += kThreads) {
      const unsigned c = (unsigned)p.graph_label[i] - (unsigned)c0;
      if (c < (unsigned)n) atomicOr(&arcs[c / 32], 1u << (c % 32));
    }
    if (masked && tid == 0 && c0 == 0) atomicOr(&arcs[0], 1u);  // blank keeps the state
    __syncthreads();
  }
  const float* bias = p.bias ? p.bias + (size_t)r * p.ldb + c0 : nullptr;
  const uint32_t* allowed = p.allowed ? p.allowed + (size_t)r * p.ldm + c0 / 32 : nullptr;

  float v[Q][E];
  LogSum sum{ninff(), 0.f};
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int c = (q * kThreads + tid) * E;
    const bool whole = c + E <= n;
    Vec<float, E> add = {};
    Vec<int, E> k = {};
    uint32_t bits = 0xffffffffu;  // (E divides 32: a word holds the columns of an access)
    if (c < n) {
      if (bias) {
        if (whole) {
          add = load_vec<float, E>(bias + c);
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (c + e < n) add.v[e] = bias[c + e];
        }
      }
      if (len > 0) k = load_vec<int, E>(count + c);
      if (allowed) bits = allowed[c / 32];
      if (masked) bits &= arcs[c / 32];
    }
    bits >>= c % 32;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float x = to_float(in[q].v[e]);
      if (k.v[e] > 0) x = (x > 0.f ? x / rep : x * rep) - pres - freq * (float)k.v[e];
      x += add.v[e];
      if (!(bits >> e & 1) || c + e >= n) x = ninff();
      v[q][e] = x;
      sum.m = fmaxf(sum.m, x);
    }
  }
  LogSum::Log norm{0.f, 0.f};
  if (PASS == kSums || (PASS == kDirect && p.normalize)) {
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (v[q][e] != ninff()) sum.s += __expf(v[q][e] - sum.m);  // (a NaN stays)
    sum = workgroup_sum(sum, red);
    if (PASS == kSums) {
      if (tid == 0) p.stats[(size_t)r * p.parts + part] = make_float2(sum.m, sum.s);
      return;
    }
    norm = sum.log();
  }
  if (PASS == kApply) {
    LogSum all{ninff(), 0.f};
    for (int i = tid; i < p.parts; i += kThreads) {
      const float2 s = p.stats[(size_t)r * p.parts + i];
      all.add(LogSum{s.x, s.y});
    }
    norm = workgroup_sum(all, red).log();
  }
  T* out = (T*)p.out + (size_t)r * p.ldo + c0;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int c = (q * kThreads + tid) * E;
    Vec<T, E> o;
#pragma unroll
    for (int e = 0; e < E; ++e) o.v[e] = from_float<T>(v[q][e] == ninff() ? ninff() : norm.of(v[q][e]));
    if (c + E <= n) {
      store_vec(out + c, o);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (c + e < n) out[c + e] = o.v[e];
    }
  }
}

template <class T, int PASS>
hipError_t launch_pass(const AdjustArgs& p, hipStream_t st) {
  constexpr int one = 16 / (int)sizeof(T) * kThreads;  // columns of one access
  const dim3 grid((unsigned)(p.R * p.parts)), block(kThreads);
  auto launch = [&](auto q) {
    hipLaunchKernelGGL((k_adjust<T, decltype(q)::value, PASS>), grid, block, 0, st, p);
    return hipGetLastError();
  };
  // (a whole row takes what it needs: 2,048 x 5,000 fp32 28 us by 8 accesses, 25 by 5; seven go by
  // eight, whose last is the one that is left out)
  const int q = (p.per - 1) / one + 1;
  if (q == 1) return launch(std::integral_constant<int, 1>());
  if (q == 2) return launch(std::integral_constant<int, 2>());
  if constexpr (PASS == kDirect) {
    if (q == 3) return launch(std::integral_constant<int, 3>());
    if constexpr (4 * one < kCols) {
      if (q == 5) return launch(std::integral_constant<int, 5>());
      if (q == 6) return launch(std::integral_constant<int, 6>());
    }
  }
  if (q <= 4) return launch(std::integral_constant<int, 4>());
  if constexpr (4 * one < kCols) return launch(std::integral_constant<int, 8>());
  return hipErrorInvalidValue;  // (not reached)
}

template <class T>
hipError_t launch_t(const AdjustArgs& p, hipStream_t st) {
  if (p.parts == 1 || !p.normalize) return launch_pass<T, kDirect>(p, st);
  const hipError_t e = launch_pass<T, kSums>(p, st);
  return e == hipSuccess ? launch_pass<T, kApply>(p, st) : e;
}

}  // namespace

// Columns per workgroup: the whole row where a workgroup holds it and a log-softmax wants it
// (one pass); else as many as leave two workgroups per CU, since each reads the history again.
bool plan_adjust(AdjustArgs& p, int dtype) {
  if (p.V > 1 << 30) return false;
  const int one = (dtype == kF32 ? 4 : 8) * kThreads;
  const int cus = device_cus() > 0 ? device_cus() : 256;
  auto parts = [&](int per) { return (p.V - 1) / per + 1; };
  p.per = kCols;
  if (!p.normalize || p.V > kCols)
    while (p.per > one && (long long)p.R * parts(p.per) < 2 * cus) p.per /= 2;
  p.parts = parts(p.per);
  if (p.parts == 1) p.per = p.V;
  return (long long)p.R * p.parts <= 1 << 23;  // (a launch holds less than 2^32 threads)
}

hipError_t launch_adjust(const AdjustArgs& p, int dtype, hipStream_t st) {
  if (p.R == 0) return hipSuccess;
  if (dtype == kF32) return launch_t<float>(p, st);
  if (dtype == kBF16) return launch_t<bf16>(p, st);
  return launch_t<_Float16>(p, st);
}

}  // namespace tbs
