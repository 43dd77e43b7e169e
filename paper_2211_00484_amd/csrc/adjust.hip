// Logits adjusted before a label is taken from them: penalties for repeated labels, biases,
// masks (a bit per label, or the labels that leave a state of a decoding graph), and
// optionally the log-softmax of what is left.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "internal.h"
#include "types.h"

namespace tbs {
namespace {

constexpr int kThreads = 256;
constexpr int kCols = 4096;  // columns whose counts and masks are in LDS at a time

__device__ __forceinline__ float ninff() { return -__builtin_inff(); }

template <class T>
__global__ __launch_bounds__(kThreads) void k_adjust(AdjustArgs p) {
  __shared__ int count[kCols];
  __shared__ uint32_t arcs[kCols / 32];
  __shared__ float red[2][kThreads / 64];
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const T* z = (const T*)p.logits + (size_t)r * p.ldz;
  T* out = (T*)p.out + (size_t)r * p.ldo;
  const int* hist = p.history ? p.history + (size_t)r * p.ldh : nullptr;
  const int len = !hist ? 0 : p.hlen ? min(max(p.hlen[r], 0), p.L) : p.L;
  float rep = p.repetition, pres = p.presence, freq = p.frequency;
  if (p.row_penalties) {
    rep = p.row_penalties[3 * (size_t)r];
    pres = p.row_penalties[3 * (size_t)r + 1];
    freq = p.row_penalties[3 * (size_t)r + 2];
  }
  int lo = 0, hi = 0;
  bool masked = false;
  if (p.graph_rp) {
    const int s = p.states[r];
    masked = s >= 0 && s < p.S;
    if (masked) {
      lo = p.graph_rp[s];
      hi = p.graph_rp[s + 1];
    }
  }
  const float* bias = p.bias ? p.bias + (size_t)r * p.ldb : nullptr;
  const uint32_t* allowed = p.allowed ? p.allowed + (size_t)r * p.ldm : nullptr;

  // the adjusted logits of columns [c0, c0 + kCols), one at a time, to f(column, value)
  auto columns = [&](int c0, auto f) {
    const int n = min(kCols, p.V - c0);
    for (int i = tid; i < kCols; i += kThreads) count[i] = 0;
    for (int i = tid; i < kCols / 32; i += kThreads) arcs[i] = 0;
    __syncthreads();
    for (int i = tid; i < len; i += kThreads) {
      const unsigned c = (unsigned)(hist[i] - c0);
      if (hist[i] >= 0 && c < (unsigned)n) atomicAdd(&count[c], 1);
    }
    if (masked) {
      for (int i = lo + tid; i < hi; i += kThreads) {
        const unsigned c = (unsigned)(p.graph_label[i] - c0);
        if (c < (unsigned)n) atomicOr(&arcs[c / 32], 1u << (c % 32));
      }
      if (tid == 0 && c0 == 0) atomicOr(&arcs[0], 1u);  // blank keeps the state
    }
    __syncthreads();
    for (int c = tid; c < n; c += kThreads) {
      const int col = c0 + c;
      float v = to_float(z[col]);
      const int k = count[c];
      if (k > 0) v = (v > 0.f ? v / rep : v * rep) - pres - freq * (float)k;
      if (bias) v += bias[col];
      if (allowed && !(allowed[col / 32] >> (col % 32) & 1)) v = ninff();
      if (masked && !(arcs[c / 32] >> (c % 32) & 1)) v = ninff();
      f(col, v);
    }
    __syncthreads();
  };

  float shift = 0.f;
  if (p.normalize) {
    float m = ninff(), s = 0.f;
    for (int c0 = 0; c0 < p.V; c0 += kCols)
      columns(c0, [&](int, float v) {
        if (v > m) {
          s *= __expf(m - v);
          m = v;
        }
        if (v != ninff()) s += __expf(v - m);  // (NaN stays)
      });
    for (int d = 32; d; d >>= 1) {
      const float om = __shfl_xor(m, d), os = __shfl_xor(s, d), mm = fmaxf(m, om);
      s = (m == mm ? s : s * __expf(m - mm)) + (om == mm ? os : os * __expf(om - mm));
      m = mm;
    }
    if (lane == 0) {
      red[0][wave] = m;
      red[1][wave] = s;
    }
    __syncthreads();
    m = red[0][0];
    s = red[1][0];
    for (int w = 1; w < kThreads / 64; ++w) {
      const float om = red[0][w], os = red[1][w], mm = fmaxf(m, om);
      s = (m == mm ? s : s * __expf(m - mm)) + (om == mm ? os : os * __expf(om - mm));
      m = mm;
    }
    shift = m == ninff() && s == 0.f ? 0.f : m + logf(s);
  }
  for (int c0 = 0; c0 < p.V; c0 += kCols)
    columns(c0, [&](int col, float v) { out[col] = from_float<T>(v == ninff() ? v : v - shift); });
}

}  // namespace

bool plan_adjust(AdjustArgs& p, int) {
  p.parts = 1;
  p.per = p.V;
  return p.R <= 1 << 23;  // (a launch holds less than 2^32 threads)
}

hipError_t launch_adjust(const AdjustArgs& p, int dtype, hipStream_t st) {
  if (p.R == 0) return hipSuccess;
  if (dtype == kF32) hipLaunchKernelGGL(k_adjust<float>, dim3(p.R), dim3(kThreads), 0, st, p);
  else if (dtype == kBF16) hipLaunchKernelGGL(k_adjust<bf16>, dim3(p.R), dim3(kThreads), 0, st, p);
  else hipLaunchKernelGGL(k_adjust<_Float16>, dim3(p.R), dim3(kThreads), 0, st, p);
  return hipGetLastError();
}

}  // namespace tbs
