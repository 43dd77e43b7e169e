// Linear layers with a fused epilogue, and their gradients:
//   out = act(x W^T + bias + residual)   or   act(x W^T + bias) + residual,
//   dz = dy act'(pre),  dx = dz W,  dW = dz^T x,  dbias = sum over rows of dz.
// One tiled product serves all three: C[m][n] = sum_k A(m, k) B(n, k), where an operand is
// stored with k along its rows (KC: x and W of the forward product, dz of dx) or with k down
// its columns (W of dx, both operands of dW).  Sums are fp32 on the matrix units: bf16 and
// fp16 operands by 16x16x32 products, fp32 operands by 16x16x4 products.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "internal.h"
#include "types.h"

namespace tbs {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// ---------------------------------------------------------------------------
// activations, in fp32

// tanh to about 2e-7 of it: odd series below 1/4 (the next term is 1e-8 of x), else
// (1 - e) / (1 + e) with e = exp(-2 |x|).
__device__ __forceinline__ float tanh_f32(float x) {
  const float a = fabsf(x), s = x * x;
  float p = 62.f / 2835.f;
  p = __builtin_fmaf(p, s, -17.f / 315.f);
  p = __builtin_fmaf(p, s, 2.f / 15.f);
  p = __builtin_fmaf(p, s, -1.f / 3.f);
  p = __builtin_fmaf(p * s, x, x);
  const float e = __expf(-2.f * a);
  const float t = copysignf((1.f - e) * __builtin_amdgcn_rcpf(1.f + e), x);
  return a < 0.25f ? p : t;
}
// (expf and not the bare hardware exponential: that loses |x| 2^-24 of it, 2e-6 at x = -30)
__device__ __forceinline__ float sigmoid_f32(float x) { return __builtin_amdgcn_rcpf(1.f + expf(-x)); }

__device__ __forceinline__ float activate(float z, int act) {
  switch (act) {
    case kActRelu: return z < 0.f ? 0.f : z;  // (a NaN stays)
    case kActTanh: return tanh_f32(z);
    case kActSilu: return z * sigmoid_f32(z);
    case kActGelu: return 0.5f * z * (1.f + erff(z * 0.70710678f));
    default: return z;
  }
}
__device__ __forceinline__ float slope(float z, int act) {
  switch (act) {
    case kActRelu: return z <= 0.f ? 0.f : 1.f;
    case kActTanh: {
      // 1 - tanh^2 = 4 e / (1 + e)^2, which loses nothing where tanh is near 1
      const float e = expf(-2.f * fabsf(z)), r = __builtin_amdgcn_rcpf(1.f + e);
      return 4.f * e * r * r;
    }
    case kActSilu: {
      const float s = sigmoid_f32(z);
      return s * (1.f + z * (1.f - s));
    }
    case kActGelu:
      return 0.5f * (1.f + erff(z * 0.70710678f)) + z * 0.39894228f * expf(-0.5f * z * z);
    default: return 1.f;
  }
}

// out (and pre) of four consecutive columns n .. n+3 of row m from their sums
template <class T>
__device__ __forceinline__ void epilogue4(const LinearEpilogue& e, f32x4 z, int m, int n, int N) {
  T* out = (T*)e.out + (size_t)m * e.ldo + n;
  const T* res = e.res ? (const T*)e.res + (size_t)m * e.ldr + n : nullptr;
  const T* bias = e.bias ? (const T*)e.bias + n : nullptr;
  T* pre = e.pre ? (T*)e.pre + (size_t)m * e.ldp + n : nullptr;
  if (n + 4 <= N) {
    f32x4 r = {0.f, 0.f, 0.f, 0.f};
    if (res) {
      const Vec<T, 4> t = load_vec<T, 4>(res);
#pragma unroll
      for (int v = 0; v < 4; ++v) r[v] = to_float(t.v[v]);
    }
    if (bias) {
      const Vec<T, 4> t = load_vec<T, 4>(bias);
#pragma unroll
      for (int v = 0; v < 4; ++v) z[v] += to_float(t.v[v]);
    }
    if (!e.res_after)
#pragma unroll
      for (int v = 0; v < 4; ++v) z[v] += r[v];
    Vec<T, 4> o;
    if (pre) {
#pragma unroll
      for (int v = 0; v < 4; ++v) o.v[v] = from_float<T>(z[v]);
      store_vec(pre, o);
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      float y = activate(z[v], e.act);
      if (e.res_after) y += r[v];
      o.v[v] = from_float<T>(y);
    }
    store_vec(out, o);
  } else {
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      if (n + v >= N) break;
      float y = z[v];
      const float r = res ? to_float(res[v]) : 0.f;
      if (bias) y += to_float(bias[v]);
      if (!e.res_after) y += r;
      if (pre) pre[v] = from_float<T>(y);
      y = activate(y, e.act);
      if (e.res_after) y += r;
      out[v] = from_float<T>(y);
    }
  }
}

// ---------------------------------------------------------------------------
// staging of an operand's slice: ROWS rows (m or n) x 64 bytes of k, as 16-byte chunks

template <class T>
constexpr int kChunkElems = 16 / (int)sizeof(T);
template <class T>
constexpr int kSlice = 64 / (int)sizeof(T);  // k per slice

// Elements [k, k + a chunk) of a row of n, zeros past its end.  A chunk that crosses the end
// is read from the row's last whole chunk and shifted.
template <class T>
__device__ __forceinline__ uint4 load_chunk_guarded(const T* row, int k, int n) {
  constexpr int CH = kChunkElems<T>;
  uint4 v = make_uint4(0, 0, 0, 0);
  if (k >= n) return v;
  if (n >= CH) {
    const int d = max(k + CH - n, 0);
    __builtin_memcpy(&v, row + k - d, 16);
    unsigned __int128 x = __builtin_bit_cast(unsigned __int128, v);
    x >>= d * 8 * (int)sizeof(T);
    return __builtin_bit_cast(uint4, x);
  }
  Vec<T, CH> r = {};
#pragma unroll
  for (int i = 0; i < CH; ++i)
    if (k + i < n) r.v[i] = row[k + i];
  __builtin_memcpy(&v, &r, 16);
  return v;
}

// Byte offset in an operand's stage of chunk c of tile row r (KC), or of chunk c of k row r
// (not KC).  The chunks are permuted so that the lanes that read together meet different
// banks: KC, 16 rows of one chunk; not KC, 16-bit, 4 k rows x 16 columns; fp32, the k rows
// r and r + 4, r + 8, r + 12 of 16 columns.
template <class T, bool KC, int ROWS>
__device__ __forceinline__ int chunk_at(int r, int c) {
  if (KC) return r * 64 + ((c ^ ((r >> 1) & 3)) * 16);
  const int x = sizeof(T) == 2 ? (r & 3) << 1 : ((r >> 2) & 3) << 2;
  return r * ROWS * (int)sizeof(T) + ((c ^ x) * 16);
}

template <class T, bool KC, int ROWS, int THREADS>
struct Stager {
  static constexpr int CH = kChunkElems<T>, N = ROWS * 4 / THREADS;
  uint4 r[N];
  // slice from k0 on of rows row0 .. (of `rows`), contraction length kc
  __device__ __forceinline__ void load(const T* p, long long ld, int row0, int rows, int k0, int kc) {
    const bool tail = k0 + kSlice<T> > kc;
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const int id = threadIdx.x + q * THREADS;
      if (KC) {
        const int gr = min(row0 + id / 4, rows - 1), k = k0 + id % 4 * CH;
        const T* row = p + (size_t)gr * ld;
        if (tail) r[q] = load_chunk_guarded(row, k, kc);
        else __builtin_memcpy(&r[q], row + k, 16);
      } else {
        constexpr int CPR = ROWS / CH;
        const int k = k0 + id / CPR, col = row0 + id % CPR * CH;
        const T* row = p + (size_t)min(k, kc - 1) * ld;
        if (row0 + ROWS > rows) r[q] = load_chunk_guarded(row, col, rows);
        else __builtin_memcpy(&r[q], row + col, 16);
        if (tail && k >= kc) r[q] = make_uint4(0, 0, 0, 0);
      }
    }
  }
  __device__ __forceinline__ void store(char* stage) const {
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const int id = threadIdx.x + q * THREADS;
      constexpr int CPR = KC ? 4 : ROWS / CH;
      *reinterpret_cast<uint4*>(stage + chunk_at<T, KC, ROWS>(id / CPR, id % CPR)) = r[q];
    }
  }
};

// ---------------------------------------------------------------------------
// fragments: lane l holds row l & 15 of a 16-row block; g = l >> 4 its share of k

template <class T, bool KC, int ROWS>
__device__ __forceinline__ uint4 fragment(const char* stage, int row0, int lane) {
  const int i = lane & 15, g = lane >> 4;
  if (KC) {
    return *reinterpret_cast<const uint4*>(stage + chunk_at<T, true, ROWS>(row0 + i, g));
  } else if (sizeof(T) == 2) {
    // k rows 8 g .. 8 g + 7 of 16 columns: two transposing reads of 4 k rows each, in which
    // lane i of 16 addresses 4 columns of one k row and receives column i of the four
    union {
      s16x4 h[2];
      uint4 v;
    } u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = 8 * g + 4 * h + (i >> 2);
      const char* at = stage + chunk_at<T, false, ROWS>(k, row0 / 8 + ((i & 3) >> 1)) + (i & 1) * 8;
      u.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
    }
    return u.v;
  } else {
    union {
      float f[4];
      uint4 v;
    } u;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      u.f[j] = *reinterpret_cast<const float*>(stage + chunk_at<T, false, ROWS>(4 * g + j, row0 / 4 + (i >> 2)) +
                                               (i & 3) * 4);
    return u.v;
  }
}

// acc += B-side block (rows of the result's lanes' registers) x A-side block (its lanes)
__device__ __forceinline__ f32x4 mma(bf16, const uint4& b, const uint4& a, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a), c,
                                                 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(_Float16, const uint4& b, const uint4& a, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, b), __builtin_bit_cast(f16x8, a), c,
                                                0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(float, const uint4& b, const uint4& a, f32x4 c) {
  const f32x4 x = __builtin_bit_cast(f32x4, b), y = __builtin_bit_cast(f32x4, a);
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
  return c;
}
__device__ __forceinline__ uint4 ones_fragment(float) {
  return __builtin_bit_cast(uint4, f32x4{1.f, 1.f, 1.f, 1.f});
}
__device__ __forceinline__ uint4 ones_fragment(bf16) {
  return make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
}
__device__ __forceinline__ uint4 ones_fragment(_Float16) {
  return make_uint4(0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u);
}

// ---------------------------------------------------------------------------
// the tiled product

// One workgroup: a BM x BN tile of C over slices [first, last) of one of `splits` parts of k;
// each wave WM x WN of it.  splits > 1: fp32 partial sums to part [splits][M][N] (and, rsum,
// the sums over k of A's rows to rpart [splits][M]); else the epilogue (rsum: to rout).
template <class T, bool AKC, bool BKC, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * (BM / WM) * (BN / WN)) void k_product(ProductArgs p) {
  constexpr int THREADS = 64 * (BM / WM) * (BN / WN);
  constexpr int MB = WM / 16, NB = WN / 16;
  constexpr int kStage = (BM + BN) * 64;
  __shared__ __align__(16) char lds[2 * kStage];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // Tiles in row-major order with each XCD on a run of neighbours (workgroup i is handed to
  // XCD i mod 8), so that the tiles of one row of A meet in one L2.
  const int tiles = p.tiles_m * p.tiles_n * p.splits;
  const int per = tiles / 8, more = tiles % 8, x = blockIdx.x % 8;
  int id = x * per + min(x, more) + blockIdx.x / 8;
  const int tn = id % p.tiles_n;
  id /= p.tiles_n;
  const int tm = id % p.tiles_m, split = id / p.tiles_m;
  const int m0 = tm * BM, n0 = tn * BN;
  const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN) * WN;
  const int slices = (p.K + kSlice<T> - 1) / kSlice<T>;
  const int first = split * p.slices_per, last = min(first + p.slices_per, slices);
  const T* a = (const T*)p.a;
  const T* b = (const T*)p.b;

  f32x4 acc[MB][NB], rs[MB];
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    rs[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const bool rsum = p.rsum && tn == 0 && wn == 0;
  Stager<T, AKC, BM, THREADS> sa;
  Stager<T, BKC, BN, THREADS> sb;
  if (first < last) {
    sa.load(a, p.lda, m0, p.M, first * kSlice<T>, p.K);
    sb.load(b, p.ldb, n0, p.N, first * kSlice<T>, p.K);
    sa.store(lds);
    sb.store(lds + BM * 64);
  }
  __syncthreads();
  for (int s = first; s < last; ++s) {
    const char* cur = lds + ((s - first) & 1) * kStage;
    char* next = lds + (~(s - first) & 1) * kStage;
    if (s + 1 < last) {
      sa.load(a, p.lda, m0, p.M, (s + 1) * kSlice<T>, p.K);
      sb.load(b, p.ldb, n0, p.N, (s + 1) * kSlice<T>, p.K);
    }
    uint4 fa[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) fa[i] = fragment<T, AKC, BM>(cur, wm + 16 * i, lane);
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const uint4 fb = fragment<T, BKC, BN>(cur + BM * 64, wn + 16 * j, lane);
#pragma unroll
      for (int i = 0; i < MB; ++i) acc[i][j] = mma(T{}, fb, fa[i], acc[i][j]);
    }
    if (rsum) {
#pragma unroll
      for (int i = 0; i < MB; ++i) rs[i] = mma(T{}, ones_fragment(T{}), fa[i], rs[i]);
    }
    if (s + 1 < last) {
      sa.store(next);
      sb.store(next + BM * 64);
    }
    __syncthreads();
  }
  const int mi = lane & 15, ni = 4 * (lane >> 4);
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    const int m = m0 + wm + 16 * i + mi;
    if (m >= p.M) continue;
    if (rsum && lane < 16) {
      if (p.splits > 1) p.rpart[(size_t)split * p.M + m] = rs[i][0];
      else if (p.rout) ((T*)p.rout)[m] = from_float<T>(rs[i][0]);
    }
    if (!p.epi.out) continue;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int n = n0 + wn + 16 * j + ni;
      if (n >= p.N) continue;
      if (p.splits > 1) {
        float* q = p.part + ((size_t)split * p.M + m) * p.N + n;
        if (n + 4 <= p.N) {
          __builtin_memcpy(q, &acc[i][j], 16);
        } else {
          for (int v = 0; n + v < p.N; ++v) q[v] = acc[i][j][v];
        }
      } else {
        epilogue4<T>(p.epi, acc[i][j], m, n, p.N);
      }
    }
  }
}

// Sum of the parts of a split product, in the parts' order, and the epilogue; the last
// workgroups sum the rows' sums.
template <class T>
__global__ __launch_bounds__(256) void k_join_parts(ProductArgs p) {
  const int quads = (p.N + 3) / 4;
  const long long total = p.epi.out ? (long long)p.M * quads : 0;
  long long id = (long long)blockIdx.x * 256 + threadIdx.x;
  if (id < total) {
    const int m = (int)(id / quads), n = (int)(id - (long long)m * quads) * 4;
    f32x4 z = {0.f, 0.f, 0.f, 0.f};
    const float* q = p.part + (size_t)m * p.N + n;
    const size_t step = (size_t)p.M * p.N;
    if (n + 4 <= p.N) {
      for (int s = 0; s < p.splits; ++s) {
        f32x4 t;
        __builtin_memcpy(&t, q + s * step, 16);
        z += t;
      }
    } else {
      for (int s = 0; s < p.splits; ++s)
        for (int v = 0; n + v < p.N; ++v) z[v] += q[s * step + v];
    }
    epilogue4<T>(p.epi, z, m, n, p.N);
    return;
  }
  id -= total;
  if (p.rsum && p.rout && id < p.M) {
    float r = 0.f;
    for (int s = 0; s < p.splits; ++s) r += p.rpart[(size_t)s * p.M + id];
    ((T*)p.rout)[id] = from_float<T>(r);
  }
}

// dz = dy act'(pre), four elements per thread
template <class T>
__global__ __launch_bounds__(256) void k_act_grad(const T* __restrict__ dy, long long ldy, const T* __restrict__ pre,
                                                  long long ldp, T* __restrict__ dz, long long ldz, int M, int N,
                                                  int act) {
  constexpr int E = kChunkElems<T>;
  const int per = (N + E - 1) / E;
  const long long total = (long long)M * per;
  for (long long id = (long long)blockIdx.x * 256 + threadIdx.x; id < total; id += (long long)gridDim.x * 256) {
    const int m = (int)(id / per), n = (int)(id - (long long)m * per) * E;
    const T* y = dy + (size_t)m * ldy + n;
    const T* z = pre + (size_t)m * ldp + n;
    T* o = dz + (size_t)m * ldz + n;
    if (n + E <= N) {
      const Vec<T, E> vy = load_vec<T, E>(y), vz = load_vec<T, E>(z);
      Vec<T, E> r;
#pragma unroll
      for (int v = 0; v < E; ++v) r.v[v] = from_float<T>(to_float(vy.v[v]) * slope(to_float(vz.v[v]), act));
      store_vec(o, r);
    } else {
      for (int v = 0; n + v < N; ++v) o[v] = from_float<T>(to_float(y[v]) * slope(to_float(z[v]), act));
    }
  }
}

// ---------------------------------------------------------------------------
// launches

constexpr long long kMaxTiles = 1 << 23;  // (a launch holds less than 2^32 threads)

template <class T, bool AKC, bool BKC, int BM, int BN, int WM, int WN>
hipError_t launch_tile(const ProductArgs& p, hipStream_t st) {
  const int tiles = p.tiles_m * p.tiles_n * p.splits;
  hipLaunchKernelGGL((k_product<T, AKC, BKC, BM, BN, WM, WN>), dim3(tiles), dim3(64 * (BM / WM) * (BN / WN)), 0,
                     st, p);
  return hipGetLastError();
}

template <class T>
hipError_t launch_product_t(ProductArgs p, bool akc, bool bkc, hipStream_t st) {
  hipError_t e;
  if (akc && bkc) e = launch_tile<T, true, true, 64, 64, 32, 32>(p, st);
  else if (akc) e = launch_tile<T, true, false, 64, 64, 32, 32>(p, st);
  else e = launch_tile<T, false, false, 64, 64, 32, 32>(p, st);
  if (e != hipSuccess || p.splits == 1) return e;
  const long long items = (p.epi.out ? (long long)p.M * ((p.N + 3) / 4) : 0) + (p.rsum && p.rout ? p.M : 0);
  hipLaunchKernelGGL(k_join_parts<T>, dim3((unsigned)((items + 255) / 256)), dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace

bool plan_product(ProductArgs& p, int dtype, bool akc, bool bkc) {
  constexpr int kMost = 1 << 30;  // (indices a tile past the end are still int)
  if (p.M > kMost || p.N > kMost || p.K > kMost) return false;
  const int ks = dtype == kF32 ? kSlice<float> : kSlice<_Float16>;
  const int slices = (p.K + ks - 1) / ks;
  p.tiles_m = (p.M + 63) / 64;
  p.tiles_n = (p.N + 63) / 64;
  p.splits = 1;
  p.slices_per = std::max(slices, 1);
  return (long long)p.tiles_m * p.tiles_n <= kMaxTiles;
}

hipError_t launch_product(const ProductArgs& p, int dtype, bool akc, bool bkc, hipStream_t st) {
  if (p.M == 0 || p.N == 0) return hipSuccess;
  if (dtype == kF32) return launch_product_t<float>(p, akc, bkc, st);
  if (dtype == kBF16) return launch_product_t<bf16>(p, akc, bkc, st);
  return launch_product_t<_Float16>(p, akc, bkc, st);
}

template <class T>
static hipError_t launch_act_grad_t(const void* dy, long long ldy, const void* pre, long long ldp, void* dz,
                                    long long ldz, int M, int N, int act, hipStream_t st) {
  const long long items = (long long)M * ((N + kChunkElems<T> - 1) / kChunkElems<T>);
  const long long blocks = std::min<long long>((items + 255) / 256, 1 << 20);
  hipLaunchKernelGGL(k_act_grad<T>, dim3((unsigned)blocks), dim3(256), 0, st, (const T*)dy, ldy, (const T*)pre, ldp,
                     (T*)dz, ldz, M, N, act);
  return hipGetLastError();
}

hipError_t launch_act_grad(int dtype, const void* dy, long long ldy, const void* pre, long long ldp, void* dz,
                           long long ldz, int M, int N, int act, hipStream_t st) {
  if (M == 0 || N == 0) return hipSuccess;
  if (ldy == N && ldp == N && ldz == N && (long long)M * N < (1ll << 30)) {  // one long row
    N *= M;
    M = 1;
    ldy = ldp = ldz = N;
  }
  if (dtype == kF32) return launch_act_grad_t<float>(dy, ldy, pre, ldp, dz, ldz, M, N, act, st);
  if (dtype == kBF16) return launch_act_grad_t<bf16>(dy, ldy, pre, ldp, dz, ldz, M, N, act, st);
  return launch_act_grad_t<_Float16>(dy, ldy, pre, ldp, dz, ldz, M, N, act, st);
}

}  // namespace tbs
