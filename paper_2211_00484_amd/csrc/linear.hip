// Linear layers with a fused epilogue, and their gradients:
//   out = act(x W^T + bias + residual)   or   act(x W^T + bias) + residual,
//   dz = dy act'(pre),  dx = dz W,  dW = dz^T x,  dbias = sum over rows of dz.
// One tiled product serves all three: C[m][n] = sum_k A(m, k) B(n, k), where an operand is
// stored with k along its rows (KC: x and W of the forward product, dz of dx) or with k down
// its columns (W of dx, both operands of dW).  Sums are fp32 on the matrix units: bf16 and
// fp16 operands by 16x16x32 products, fp32 operands by 16x16x4 products.
//
// dz of 16-bit layers is a product of its own and has more bits than a matrix instruction takes
// of an operand: dx, dW and dbias take it in two parts of the element type, so that they are
// rounded once, as the forward product is (from the rounded dz alone their errors are 1.4 times
// those of one rounding, and dz below fp16's range is lost to the sums over rows).  It costs their
// products twice (40,000 x 512, N = 500 bf16 with tanh 152 us, 100 from the rounded dz).
//
// Bound, MI355X: 16-bit, the matrix units (in the main loop of 128 x 128 tiles they are busy 86%
// of its cycles, of 256 x 256 tiles 70%) and, for K of a few hundred, what is not the main loop:
// 64,000 x 512, K = 2,048 fp16 with a residual 150 us, 895 TFLOP/s (the library's product alone
// 111); 6,000 x 5,000, K = 512 bf16 47 us, 650 TFLOP/s (76).  At K = 512 a 256 x 256 tile's main loop
// takes 14 us and its results 6, written at 5.6 TB/s while every CU writes.  fp32: the fp32 matrix
// instructions, 8,000 x 512, K = 384 33 us (32), 8,192 x 2,048, K = 2,048 138 TFLOP/s (137).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

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

// The normal distribution at z: its upper tail at s = |z| is e^(-s^2 / 2) G(s), where G falls as 1 / s
// and is t times a polynomial in t = 1 / (1 + 0.35 s), fitted here to within 5e-8 of it up to s = 14.5
// (so that a small tail keeps its digits, which 1 + erf does not).  density: e^(-s^2 / 2), whose
// argument's rounding is made good.
__device__ __forceinline__ float normal_cdf(float z, float& density) {
  const float s = fminf(fabsf(z), 20.f), h = s * s, l = __builtin_fmaf(s, s, -h);
  constexpr float kHi = -0.7213475f, kLo = -9.629815e-9f;  // -log2(e) / 2
  const float p = h * kHi, d = __builtin_fmaf(h, kHi, -p) + __builtin_fmaf(h, kLo, l * kHi);
  const float e = __builtin_amdgcn_exp2f(p);
  density = __builtin_fmaf(e * 0.69314718f, d, e);
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.35f, s, 1.f));
  float g = -0.029163932f;
  g = __builtin_fmaf(g, t, 0.14406084f);
  g = __builtin_fmaf(g, t, -0.25590193f);
  g = __builtin_fmaf(g, t, 0.15939298f);
  g = __builtin_fmaf(g, t, -0.023263881f);
  g = __builtin_fmaf(g, t, 0.10557482f);
  g = __builtin_fmaf(g, t, 0.11981549f);
  g = __builtin_fmaf(g, t, 0.13986434f);
  g = __builtin_fmaf(g, t, 0.13962126f);
  const float tail = g * t * density;
  return z < 0.f ? tail : 1.f - tail;
}

__device__ __forceinline__ float activate(float z, int act) {
  switch (act) {
    case kActRelu: return z < 0.f ? 0.f : z;  // (a NaN stays)
    case kActTanh: return tanh_f32(z);
    case kActSilu: return z * sigmoid_f32(z);
    case kActGelu: {
      float density;
      return z * normal_cdf(z, density);
    }
    default: return z;
  }
}
// z, but for values so large that what a slope multiplies them by is 0: an infinite z, which pre
// holds where the type's range ends, has its limit too.
__device__ __forceinline__ float limited(float z) { return fabsf(z) > 1e4f ? copysignf(1e4f, z) : z; }
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
      return s * (1.f + limited(z) * (1.f - s));
    }
    case kActGelu: {
      float density;
      const float cdf = normal_cdf(z, density);
      return cdf + limited(z) * 0.39894228f * density;
    }
    default: return 1.f;
  }
}

// out (and pre) of E consecutive columns n .. of row m from their sums, biases and residuals
// (FULL: all of them lie inside the row).
template <class T, int E, bool FULL>
__device__ __forceinline__ void finish(const LinearEpilogue& e, Vec<float, E> z, const Vec<T, E>& bias,
                                       const Vec<T, E>& r, int m, int n, int N) {
  T* out = (T*)e.out + (size_t)m * e.ldo + n;
  T* pre = e.pre ? (T*)e.pre + (size_t)m * e.ldp + n : nullptr;
  const bool whole = FULL || n + E <= N;
  Vec<T, E> o;
#pragma unroll
  for (int v = 0; v < E; ++v) {
    z.v[v] += to_float(bias.v[v]);
    if (!e.res_after) z.v[v] += to_float(r.v[v]);
  }
  auto put = [&](T* to) {
#pragma unroll
    for (int v = 0; v < E; ++v) o.v[v] = from_float<T>(z.v[v]);
    if (whole) {
      store_vec(to, o);
    } else {
#pragma unroll
      for (int v = 0; v < E; ++v)
        if (n + v < N) to[v] = o.v[v];
    }
  };
  if (pre) put(pre);
  switch (e.act) {
    case kActRelu:
#pragma unroll
      for (int v = 0; v < E; ++v) z.v[v] = activate(z.v[v], kActRelu);
      break;
    case kActTanh:
#pragma unroll
      for (int v = 0; v < E; ++v) z.v[v] = activate(z.v[v], kActTanh);
      break;
    case kActSilu:
#pragma unroll
      for (int v = 0; v < E; ++v) z.v[v] = activate(z.v[v], kActSilu);
      break;
    case kActGelu:
#pragma unroll
      for (int v = 0; v < E; ++v) z.v[v] = activate(z.v[v], kActGelu);
      break;
  }
  if (e.res_after)
#pragma unroll
    for (int v = 0; v < E; ++v) z.v[v] += to_float(r.v[v]);
  put(out);
}
// Columns n .. of a row of N (p; null: zeros, as past the row's end)
template <class T, int E>
__device__ __forceinline__ Vec<T, E> load_columns(const T* p, int n, int N) {
  Vec<T, E> b = {};
  if (!p) return b;
  if (n + E <= N) return load_vec<T, E>(p + n);
#pragma unroll
  for (int v = 0; v < E; ++v)
    if (n + v < N) b.v[v] = p[n + v];
  return b;
}
template <class T, int E>
__device__ __forceinline__ Vec<T, E> load_residual(const LinearEpilogue& e, int m, int n, int N) {
  return load_columns<T, E>(e.res ? (const T*)e.res + (size_t)m * e.ldr : nullptr, n, N);
}

// ---------------------------------------------------------------------------
// staging of an operand's slice: ROWS rows (m or n) x 128 bytes of k, as 16-byte chunks
// (a whole cache line of each row: 64,000 x 512, K = 2,048 fp16 165 us, 197 in slices of 64 bytes)

template <class T>
constexpr int kChunkElems = 16 / (int)sizeof(T);
template <class T>
constexpr int kSlice = 128 / (int)sizeof(T);  // k per slice

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

// Places of a slice's chunks in LDS, numbered in the order in which direct copies fill them: 64 in
// a row by a wave, 16 bytes a lane.  Bank conflicts are kept off by sharing the rows out to blocks
// with a pad behind each, so that a fragment's address is its lane's constant plus constants
// (permuting the chunks of a row instead measured the same):
//  - KC: row r to block r % 8, pads of 16 bytes: 8 rows of a fragment meet 8 places;
//  - not KC, 16-bit: k row r to block r % 4, pads of 32: a transposing read's 4 k rows x 32 bytes;
//  - not KC, fp32: k row r to block r / 4 % 4, pads of 64: rows of two lane groups x 64 bytes.
template <class T, bool KC, int ROWS>
struct Layout {
  static constexpr int CH = kChunkElems<T>;
  static constexpr int CPR = KC ? 8 : ROWS / CH;           // chunks per row (of k, or of m)
  static constexpr int BLOCKS = KC ? 8 : 4, CPB = ROWS * 8 / BLOCKS;
  static constexpr int PAD = KC ? 16 : sizeof(T) == 2 ? 32 : 64;
  static constexpr int BLOCK = CPB * 16 + PAD, BYTES = BLOCKS * BLOCK;
  static_assert(CPB % 64 == 0, "a wave's copy stays in a block");
  __device__ static __forceinline__ int at(int id) { return id / CPB * BLOCK + id % CPB * 16; }
  __device__ static __forceinline__ int row(int id) {
    const int block = id / CPB, r = id % CPB / CPR;
    return KC || sizeof(T) == 2 ? r * BLOCKS + block : r / 4 * 16 + block * 4 + r % 4;
  }
  __device__ static __forceinline__ int chunk(int id) { return id % CPR; }
};

template <class T, bool KC, int ROWS, int THREADS>
struct Stager {
  typedef Layout<T, KC, ROWS> L;
  static constexpr int CH = kChunkElems<T>, N = ROWS * 8 / THREADS;
  uint4 r[N];
  // slice from k0 on of rows row0 .. (of `rows`), contraction length kc
  __device__ __forceinline__ void load(const T* p, long long ld, int row0, int rows, int k0, int kc) {
    const bool tail = k0 + kSlice<T> > kc;
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const int id = threadIdx.x + q * THREADS;
      if (KC) {
        const int gr = min(row0 + L::row(id), rows - 1), k = k0 + L::chunk(id) * CH;
        const T* row = p + (size_t)gr * ld;
        if (tail) r[q] = load_chunk_guarded(row, k, kc);
        else __builtin_memcpy(&r[q], row + k, 16);
      } else {
        const int k = k0 + L::row(id), col = row0 + L::chunk(id) * CH;
        const T* row = p + (size_t)min(k, kc - 1) * ld;
        if (row0 + ROWS > rows) r[q] = load_chunk_guarded(row, col, rows);
        else __builtin_memcpy(&r[q], row + col, 16);
        if (tail && k >= kc) r[q] = make_uint4(0, 0, 0, 0);
      }
    }
  }
  __device__ __forceinline__ void store(char* stage) const {
#pragma unroll
    for (int q = 0; q < N; ++q) *reinterpret_cast<uint4*>(stage + L::at(threadIdx.x + q * THREADS)) = r[q];
  }
};

// Copies straight into LDS: a wave's 64 chunks land in 1 KiB from `to` on, lane l's at 16 l.
// Written as assembly (with no register to receive anything) because the compiler lets every
// later LDS read wait for all copies of its own; the waits are in wait_copies.
__device__ __forceinline__ void copy_chunks(unsigned to, const char* base, unsigned offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(to), "v"(offset), "s"(base)
               : "memory", "m0");
}
// Waits until at most N of the wave's copies are in flight and its LDS accesses are done, then
// for the workgroup.
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(N) : "memory");
}

// The same slices as Stager's by direct copies.  Chunks of rows past the operand's end are
// those of its last row (KC) or begin in its last whole or partial chunk (not KC; what is read
// behind a row's end is the start of the next, which exists in every slice but the last):
// they only reach results that are not stored.
template <class T, bool KC, int ROWS, int THREADS>
struct Copier {
  typedef Layout<T, KC, ROWS> L;
  static constexpr int CH = kChunkElems<T>, N = ROWS * 8 / THREADS;
  unsigned offset[N];
  const char* base;
  long long step;
  __device__ __forceinline__ void init(const T* p, long long ld, int row0, int rows, int k0) {
    base = (const char*)(p + (KC ? (size_t)row0 * ld + k0 : (size_t)k0 * ld + row0));
    step = KC ? 128 : (long long)kSlice<T> * ld * (int)sizeof(T);
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const int id = threadIdx.x + q * THREADS, r = L::row(id), c = L::chunk(id);
      if (KC) offset[q] = (unsigned)((long long)min(r, rows - 1 - row0) * ld * (int)sizeof(T)) + c * 16;
      else offset[q] = (unsigned)((long long)r * ld * (int)sizeof(T)) + min(c, (rows - 1 - row0) / CH) * 16;
    }
  }
  __device__ __forceinline__ void copy(unsigned stage, int wave) {
#pragma unroll
    for (int q = 0; q < N; ++q) copy_chunks(stage + L::at(q * THREADS + wave * 64), base, offset[q]);
    base += step;
  }
};

// ---------------------------------------------------------------------------
// fragments of half a slice (64 bytes of k): lane l holds row l & 15 of a 16-row block;
// g = l >> 4 its share of k

template <class T, bool KC, int ROWS>
__device__ __forceinline__ uint4 fragment(const char* stage, int row0, int half, int lane) {
  typedef Layout<T, KC, ROWS> L;
  const int i = lane & 15, g = lane >> 4;
  if (KC) {
    return *reinterpret_cast<const uint4*>(stage + (i & 7) * L::BLOCK + (i >> 3) * 128 + g * 16 + row0 * 16 +
                                           half * 64);
  } else if (sizeof(T) == 2) {
    // k rows 8 g .. 8 g + 7 of 16 columns: two transposing reads of 4 k rows each, in which
    // lane i of 16 addresses 4 columns of one k row and receives column i of the four
    union {
      s16x4 h[2];
      uint4 v;
    } u;
    const char* at = stage + (i >> 2) * L::BLOCK + 2 * g * (ROWS * 2) + (i & 3) * 8 + row0 * 2 + half * 8 * (ROWS * 2);
#pragma unroll
    for (int h = 0; h < 2; ++h)
      u.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + h * (ROWS * 2)));
    return u.v;
  } else {
    union {
      float f[4];
      uint4 v;
    } u;
    const char* at = stage + g * L::BLOCK + (row0 + i) * 4 + half * 4 * (ROWS * 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) u.f[j] = *reinterpret_cast<const float*>(at + j * (ROWS * 4));
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

// Orders a wave's LDS accesses before and after it (the hardware runs them in order).
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A 16-bit value's second part, what its rounding took off, is held times 2^kLowBits: fp16 has no
// exponents to spare for it, bf16 has.
template <class T>
constexpr int kLowBits = 0;
template <>
constexpr int kLowBits<_Float16> = 11;

// One workgroup: a BM x BN tile of C over slices [first, last) of one of `splits` parts of k;
// each wave WM x WN of it.  splits > 1: fp32 partial sums to part [splits][M][N] (and, rsum,
// the sums over k of A's rows to rpart [splits][M]); else the epilogue (rsum: to rout).
// DIRECT: operands whose rows are 4-byte aligned are copied straight into a ring of ST
// slices, ST - 1 of them in flight while one is used; the last slice, where it is not whole, and
// other operands go through registers.
// LOW: A is a + a_low 2^-kLowBits; the part's slices are gone through twice, those of a_low first,
// whose sums are scaled before those of a are added.
template <class T, bool AKC, bool BKC, int BM, int BN, int WM, int WN, int ST, bool DIRECT, bool LOW>
__global__ __launch_bounds__(64 * (BM / WM) * (BN / WN)) void k_product(ProductArgs p) {
  constexpr int THREADS = 64 * (BM / WM) * (BN / WN);
  constexpr int MB = WM / 16, NB = WN / 16;
  constexpr int kA = Layout<T, AKC, BM>::BYTES, kStage = kA + Layout<T, BKC, BN>::BYTES;
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
  const bool rsum = !AKC && p.rsum && tn == 0 && wn == 0;
  // fp32: the sums of half slices are added in fp64 (each by the next, so that nothing waits for
  // it): a column of 64,000 in one fp32 sum is off by 4e-6, which 16-bit results do not show
  constexpr bool kWide = sizeof(T) == 4;
  double rt[MB] = {};
  // The fragments of a half slice, and their products.  The second half's products are left
  // until the first half of the next slice has been asked for, so that its LDS reads (and the
  // wait for the workgroup before them) have products to hide behind.
  struct Half {
    uint4 a[MB], b[NB];
  };
  Half h0, h1;
  auto read = [&](const char* cur, int h, Half& f) {
#pragma unroll
    for (int i = 0; i < MB; ++i) f.a[i] = fragment<T, AKC, BM>(cur, wm + 16 * i, h, lane);
#pragma unroll
    for (int j = 0; j < NB; ++j) f.b[j] = fragment<T, BKC, BN>(cur + kA, wn + 16 * j, h, lane);
  };
  auto multiply = [&](const Half& f) {
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int i = 0; i < MB; ++i) acc[i][j] = mma(T{}, f.b[j], f.a[i], acc[i][j]);
    if (!AKC && rsum) {
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        if (kWide) {
          rt[i] += (double)rs[i][0];
          rs[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        rs[i] = mma(T{}, ones_fragment(T{}), f.a[i], rs[i]);
      }
    }
  };
  constexpr bool kDeep = MB * NB <= 16;  // (larger tiles have no registers for two halves)
  auto slice = [&](const char* cur, bool any) {
    read(cur, 0, h0);
    if (kDeep) {
      if (any) multiply(h1);
      read(cur, 1, h1);
    } else {
      multiply(h0);
      read(cur, 1, h0);
    }
    multiply(h0);
  };
  Stager<T, AKC, BM, THREADS> sa;
  Stager<T, BKC, BN, THREADS> sb;
  const T* a_now = LOW ? (const T*)p.a_low : a;  // the part of A that is staged
  long long lda_now = LOW ? p.lda_low : p.lda;
  auto load = [&](int s) {
    sa.load(a_now, lda_now, m0, p.M, s * kSlice<T>, p.K);
    sb.load(b, p.ldb, n0, p.N, s * kSlice<T>, p.K);
  };
  Copier<T, AKC, BM, THREADS> ca;
  Copier<T, BKC, BN, THREADS> cb;
  constexpr int kCopies = ca.N + cb.N;
  const unsigned base = (unsigned)(size_t)(__attribute__((address_space(3))) char*)lds;
  // slices that copies may take: all, but for a last one that is not whole
  const bool partial = p.K % kSlice<T> != 0 || (!AKC && p.M % kChunkElems<T> != 0) ||
                       (!BKC && p.N % kChunkElems<T> != 0);
  const int whole = partial ? min(last, slices - 1) : last;
  const int count = last - first, total = LOW ? 2 * count : count;  // turns: slices of either part
  int in = 0;  // stage that the next turn's slice goes to
  auto begin = [&]() {
    ca.init(a_now, lda_now, m0, p.M, first * kSlice<T>);
    cb.init(b, p.ldb, n0, p.N, first * kSlice<T>);
  };
  auto slice_of = [&](int turn) { return first + (LOW && turn >= count ? turn - count : turn); };
  auto request = [&](int turn) {
    if (LOW && turn == count) {
      a_now = a;
      lda_now = p.lda;
      begin();
    }
    const int s = slice_of(turn);
    if (s < whole && (!LOW || turn < total)) {
      ca.copy(base + in * kStage, wave);
      cb.copy(base + in * kStage + kA, wave);
    } else if (turn < total) {
      load(s);
      sa.store(lds + in * kStage);
      sb.store(lds + in * kStage + kA);
    }
    in = in == ST - 1 ? 0 : in + 1;
  };
  int turn = 0, out = 0;
  if (DIRECT) {
    begin();
#pragma unroll
    for (int i = 0; i < ST - 1; ++i) request(i);
  }
  for (int pass = LOW ? 1 : 0; pass >= 0; --pass) {
    if (DIRECT) {
      for (int s = first; s < last; ++s, ++turn) {
        // (ST - 2 slices behind this one may be in flight, if the last of them was copied)
        if (slice_of(turn + ST - 2) < whole && (!LOW || turn + ST - 2 < total)) wait_copies<(ST - 2) * kCopies>();
        else wait_copies<0>();
        request(turn + ST - 1);  // (to the place of the slice before, which every wave has read)
        slice(lds + out * kStage, s > first);
        out = out == ST - 1 ? 0 : out + 1;
      }
    } else {
      if (LOW && pass == 0) {
        a_now = a;
        lda_now = p.lda;
      }
      if (first < last) {
        load(first);
        sa.store(lds);
        sb.store(lds + kA);
      }
      __syncthreads();
      for (int s = first; s < last; ++s) {
        char* next = lds + (~(s - first) & 1) * kStage;
        if (s + 1 < last) load(s + 1);
        slice(lds + ((s - first) & 1) * kStage, s > first);
        if (s + 1 < last) {
          sa.store(next);
          sb.store(next + kA);
        }
        __syncthreads();
      }
    }
    if (kDeep && first < last) multiply(h1);
    if (LOW && pass == 1) {
      // (an infinity or NaN of the other operand comes again with a, and with a's sign)
      constexpr float kScale = 1.f / (float)(1 << kLowBits<T>);
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        rs[i] *= kScale;
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const float t = acc[i][j][v] * kScale;
            acc[i][j][v] = fabsf(t) < INFINITY ? t : 0.f;
          }
      }
    }
  }
  if (rsum && lane < 16) {
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      const int m = m0 + wm + 16 * i + lane;
      if (m >= p.M) continue;
      const float r = kWide ? (float)(rt[i] + (double)rs[i][0]) : rs[i][0];
      if (p.splits > 1) p.rpart[(size_t)split * p.M + m] = r;
      else if (p.rout) ((T*)p.rout)[m] = from_float<T>(r);
    }
  }
  if (!p.epi.out) return;
  // Results leave through LDS, 16 rows of the wave's columns at a time: a lane holds 4 columns
  // of a row, but stores (and reads the residual) in 16-byte pieces, a row's side by side.  The
  // rows are rolled in one loop, with the registers picked by a switch: unrolled, the five
  // activations take more code than the instruction cache holds.
  constexpr int E = kChunkElems<T>, LPR = WN / E, RPP = 64 / LPR, RS = WN + 4;
  __syncthreads();  // the waves have read their last slices
  float* tile = reinterpret_cast<float*>(lds) + wave * 16 * RS;
  const int row = lane / LPR, col = lane % LPR * E;
  const int n = n0 + wn + col;
  const bool parts = p.splits > 1;
  const Vec<T, E> bias = load_columns<T, E>(parts ? nullptr : (const T*)p.epi.bias, n, p.N);
  // Tiles that lie inside C whole take no branch per row, and those without a residual hold no
  // loads: a wait for a load also waits for the stores before it, where a branch keeps the
  // compiler from counting them (10.7 us for a 256 x 256 tile's results before).
  auto leave = [&](auto full_c, auto res_c) __attribute__((always_inline)) {
    constexpr bool FULL = decltype(full_c)::value, RES = decltype(res_c)::value;
    constexpr int Q = 16 / RPP;
    const T* r0 = RES ? (const T*)p.epi.res + (size_t)(m0 + wm + row) * p.epi.ldr + n : nullptr;
    Vec<T, E> res[Q] = {};  // of the rows to come, asked for one block ahead
    auto ask = [&](int i) {
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const int off = 16 * min(i, MB - 1) + q * RPP, m = m0 + wm + row + off;
        if (FULL) res[q] = load_vec<T, E>(r0 + (size_t)off * p.epi.ldr);
        else if (m < p.M && !parts) res[q] = load_residual<T, E>(p.epi, m, n, p.N);
      }
    };
    if (RES) ask(0);
#pragma unroll 1
    for (int i = 0; i < MB; ++i) {
      // (each case ends in its own comment to the assembler: alike, the compiler merges the cases
      // and makes acc an indexed array in scratch memory)
      auto put = [&](const f32x4(&r)[NB]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NB; ++j)
          *reinterpret_cast<f32x4*>(tile + (lane & 15) * RS + 16 * j + 4 * (lane >> 4)) = r[j];
      };
      static_assert(MB <= 8, "cases");
      switch (i) {
        case 0: put(acc[0]); asm volatile("; rows 0"); break;
        case 1: put(acc[1 % MB]); asm volatile("; rows 1"); break;
        case 2: put(acc[2 % MB]); asm volatile("; rows 2"); break;
        case 3: put(acc[3 % MB]); asm volatile("; rows 3"); break;
        case 4: put(acc[4 % MB]); asm volatile("; rows 4"); break;
        case 5: put(acc[5 % MB]); asm volatile("; rows 5"); break;
        case 6: put(acc[6 % MB]); asm volatile("; rows 6"); break;
        default: put(acc[7 % MB]); asm volatile("; rows 7");
      }
      wave_sync();
      Vec<T, E> now[Q];
#pragma unroll
      for (int q = 0; q < Q; ++q) now[q] = res[q];
      if (RES) ask(i + 1);
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const int r = row + q * RPP, m = m0 + wm + 16 * i + r;
        Vec<float, E> z;
#pragma unroll
        for (int v = 0; v < E; v += 4)
          *reinterpret_cast<f32x4*>(z.v + v) = *reinterpret_cast<const f32x4*>(tile + r * RS + col + v);
        if (!FULL && (m >= p.M || n >= p.N)) continue;
        if ((!RES || !FULL) && parts) {
          float* to = p.part + ((size_t)split * p.M + m) * p.N + n;
          if (FULL || n + E <= p.N) {
            store_vec(to, z);
          } else {
#pragma unroll
            for (int v = 0; v < E; ++v)
              if (n + v < p.N) to[v] = z.v[v];
          }
        } else {
          finish<T, E, FULL>(p.epi, z, bias, now[q], m, n, p.N);
        }
      }
      wave_sync();
    }
  };
  const bool full = m0 + BM <= p.M && n0 + BN <= p.N;
  if (!full) leave(std::false_type(), std::true_type());
  else if (p.epi.res && !parts) leave(std::true_type(), std::true_type());
  else leave(std::true_type(), std::false_type());
}

// Few rows (M <= 32: a decoder's step, a short chunk), both operands with k along their rows: a
// workgroup per 16 columns, its four waves taking turns at the 64-byte pieces of k, straight from
// memory to fragments with four pieces of each row in flight; their sums meet in LDS.  Bound by
// the latency of a launch and of two or three memory round trips.
template <class T, int MB>
__global__ __launch_bounds__(256) void k_product_rows(ProductArgs p) {
  constexpr int CH = kChunkElems<T>, STEP = 4 * CH, AHEAD = 4;
  __shared__ f32x4 sums[4][MB][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x * 16;
  const T* b = (const T*)p.b + (size_t)min(n0 + i, p.N - 1) * p.ldb;
  const T* a[MB];
  f32x4 acc[MB];
#pragma unroll
  for (int m = 0; m < MB; ++m) {
    a[m] = (const T*)p.a + (size_t)min(16 * m + i, p.M - 1) * p.lda;
    acc[m] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int whole = p.K / STEP;  // pieces without an end of a row in them
  for (int s = wave; s < whole; s += 4 * AHEAD) {
    uint4 fb[AHEAD], fa[AHEAD][MB];
#pragma unroll
    for (int t = 0; t < AHEAD; ++t) {
      const int k = min(s + 4 * t, whole - 1) * STEP + g * CH;  // (a piece too many is dropped below)
      __builtin_memcpy(&fb[t], b + k, 16);
#pragma unroll
      for (int m = 0; m < MB; ++m) __builtin_memcpy(&fa[t][m], a[m] + k, 16);
    }
#pragma unroll
    for (int t = 0; t < AHEAD; ++t)
      if (s + 4 * t < whole)
#pragma unroll
        for (int m = 0; m < MB; ++m) acc[m] = mma(T{}, fb[t], fa[t][m], acc[m]);
  }
  if (whole * STEP < p.K && wave == whole % 4) {
    const int k = whole * STEP + g * CH;
    const uint4 fb = load_chunk_guarded(b, k, p.K);
#pragma unroll
    for (int m = 0; m < MB; ++m) acc[m] = mma(T{}, fb, load_chunk_guarded(a[m], k, p.K), acc[m]);
  }
#pragma unroll
  for (int m = 0; m < MB; ++m) sums[wave][m][lane] = acc[m];
  __syncthreads();
  const int n = n0 + 4 * g;
  if (n >= p.N) return;
  const Vec<T, 4> bias = load_columns<T, 4>((const T*)p.epi.bias, n, p.N);
  if (const int m = wave; m < MB) {
    const int r = 16 * m + i;
    if (r >= p.M) return;
    Vec<float, 4> z;
    f32x4 t = sums[0][m][lane];
#pragma unroll
    for (int w = 1; w < 4; ++w) t += sums[w][m][lane];
#pragma unroll
    for (int v = 0; v < 4; ++v) z.v[v] = t[v];
    finish<T, 4, false>(p.epi, z, bias, load_residual<T, 4>(p.epi, r, n, p.N), r, n, p.N);
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
    Vec<float, 4> z = {};
    const float* q = p.part + (size_t)m * p.N + n;
    const size_t step = (size_t)p.M * p.N;
    if (n + 4 <= p.N) {
      for (int s = 0; s < p.splits; s += 8) {  // (eight parts in flight)
        Vec<float, 4> t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = load_vec<float, 4>(q + min(s + i, p.splits - 1) * step);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (s + i < p.splits)
#pragma unroll
            for (int v = 0; v < 4; ++v) z.v[v] += t[i].v[v];
      }
    } else {
      for (int s = 0; s < p.splits; ++s)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (n + v < p.N) z.v[v] += q[s * step + v];
    }
    finish<T, 4, false>(p.epi, z, load_columns<T, 4>((const T*)p.epi.bias, n, p.N), load_residual<T, 4>(p.epi, m, n, p.N), m,
                 n, p.N);
    return;
  }
  id -= total;
  if (p.rsum && p.rout && id < p.M) {
    double r = 0.0;
    for (int s = 0; s < p.splits; ++s) r += (double)p.rpart[(size_t)s * p.M + id];
    ((T*)p.rout)[id] = from_float<T>((float)r);
  }
}

// dz = dy act'(pre), 16 bytes a thread and turn; low (rows of ldl), unless null: what dz's rounding
// took off, times 2^kLowBits (0 where dz is beyond the type's range).  Bound: memory (8,000 x 512 fp32 10.4 us, 4.7 TB/s).
template <class T>
__global__ __launch_bounds__(256) void k_act_grad(const T* __restrict__ dy, long long ldy, const T* __restrict__ pre,
                                                  long long ldp, T* __restrict__ dz, long long ldz,
                                                  T* __restrict__ low, long long ldl, int M, int N, int act) {
  constexpr int E = kChunkElems<T>;
  const int per = (N + E - 1) / E;
  const long long total = (long long)M * per;
  for (long long id = (long long)blockIdx.x * 256 + threadIdx.x; id < total; id += (long long)gridDim.x * 256) {
    const int m = (int)(id / per), n = (int)(id - (long long)m * per) * E;
    const T* y = dy + (size_t)m * ldy + n;
    const T* z = pre + (size_t)m * ldp + n;
    T* o = dz + (size_t)m * ldz + n;
    T* l = sizeof(T) == 2 && low ? low + (size_t)m * ldl + n : nullptr;
    // (both parts go by one rounding: the compiler may round a product to fp16 without fp32 between,
    // and another time with it, a step apart at a tie)
    auto parts = [&](float d, T& r, T& rl) {
      r = from_float<T>(d);
      asm("" : "+v"(r));
      const float t = d - to_float(r);
      rl = from_float<T>(fabsf(t) < INFINITY ? t * (float)(1 << kLowBits<T>) : 0.f);
    };
    if (n + E <= N) {
      const Vec<T, E> vy = load_vec<T, E>(y), vz = load_vec<T, E>(z);
      Vec<T, E> r, rl;
#pragma unroll
      for (int v = 0; v < E; ++v) {
        parts(to_float(vy.v[v]) * slope(to_float(vz.v[v]), act), r.v[v], rl.v[v]);
      }
      store_vec(o, r);
      if (l) store_vec(l, rl);
    } else {
      for (int v = 0; n + v < N; ++v) {
        T r, rl;
        parts(to_float(y[v]) * slope(to_float(z[v]), act), r, rl);
        o[v] = r;
        if (l) l[v] = rl;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// launches

constexpr long long kMaxTiles = 1 << 23;  // (a launch holds less than 2^32 threads)

// Whether direct copies may take an operand: rows that start on 4 bytes, offsets within a tile
// that fit 32 bits, and, with k down its columns, rows of a chunk at least.
template <class T>
bool direct_ok(const void* p, long long ld, bool kc, int rows) {
  return (uintptr_t)p % 4 == 0 && ld * (long long)sizeof(T) % 4 == 0 && ld < (1 << 20) &&
         (kc || rows >= kChunkElems<T>);
}

template <class T, bool AKC, bool BKC, int BM, int BN, int WM, int WN, int ST, bool DIRECT, bool LOW>
hipError_t launch_tile_d(const ProductArgs& p, hipStream_t st) {
  constexpr size_t lds = (DIRECT ? ST : 2) * (Layout<T, AKC, BM>::BYTES + Layout<T, BKC, BN>::BYTES);
  if (lds > 65536) {
    static LdsGrant grant;
    const hipError_t e = grant((const void*)k_product<T, AKC, BKC, BM, BN, WM, WN, ST, DIRECT, LOW>, lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((k_product<T, AKC, BKC, BM, BN, WM, WN, ST, DIRECT, LOW>), dim3(p.tiles_m * p.tiles_n * p.splits),
                     dim3(64 * (BM / WM) * (BN / WN)), lds, st, p);
  return hipGetLastError();
}

template <class T, bool AKC, bool BKC, bool LOW>
hipError_t launch_shape(const ProductArgs& p, hipStream_t st) {
  const bool direct = direct_ok<T>(p.a, p.lda, AKC, p.M) && direct_ok<T>(p.b, p.ldb, BKC, p.N) &&
                      (!LOW || direct_ok<T>(p.a_low, p.lda_low, AKC, p.M));
  if (p.shape == 0)
    return direct ? launch_tile_d<T, AKC, BKC, 64, 64, 32, 32, 3, true, LOW>(p, st)
                  : launch_tile_d<T, AKC, BKC, 64, 64, 32, 32, 3, false, LOW>(p, st);
  if (p.shape == 1 || sizeof(T) == 4)
    return direct ? launch_tile_d<T, AKC, BKC, 128, 128, 64, 64, 2, true, LOW>(p, st)
                  : launch_tile_d<T, AKC, BKC, 128, 128, 64, 64, 2, false, LOW>(p, st);
  if constexpr (sizeof(T) == 2)
    return direct ? launch_tile_d<T, AKC, BKC, 256, 256, 128, 64, 2, true, LOW>(p, st)
                  : launch_tile_d<T, AKC, BKC, 256, 256, 128, 64, 2, false, LOW>(p, st);
  return hipErrorInvalidValue;  // (not reached)
}
// (only gradients have an operand in two parts, and only 16-bit ones)
template <class T, bool AKC>
hipError_t launch_gradient(const ProductArgs& p, hipStream_t st) {
  if constexpr (sizeof(T) == 2)
    if (p.a_low) return launch_shape<T, AKC, false, true>(p, st);
  return launch_shape<T, AKC, false, false>(p, st);
}

constexpr int kRowsShape = 3;

template <class T>
hipError_t launch_rows(const ProductArgs& p, hipStream_t st) {
  const dim3 grid(p.tiles_n), block(256);
  if (p.M <= 16) hipLaunchKernelGGL((k_product_rows<T, 1>), grid, block, 0, st, p);
  else hipLaunchKernelGGL((k_product_rows<T, 2>), grid, block, 0, st, p);
  return hipGetLastError();
}

template <class T>
hipError_t launch_product_t(const ProductArgs& p, bool akc, bool bkc, hipStream_t st) {
  if (p.shape == kRowsShape) return launch_rows<T>(p, st);
  hipError_t e;
  if (akc && bkc) e = launch_shape<T, true, true, false>(p, st);
  else if (akc) e = launch_gradient<T, true>(p, st);
  else e = launch_gradient<T, false>(p, st);
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
  if (((long long)p.M + 63) / 64 * (((long long)p.N + 63) / 64) > kMaxTiles) return false;
  const int cus = device_cus() > 0 ? device_cus() : 256;
  p.splits = 1;
  // (64 rows, K = 2,048: 12.2 us by rows, 7.7 by tiles in parts; 16 rows, K = 512, N = 5,000 4.0)
  // (a workgroup per 16 columns, so that a launch takes a quarter of the columns that tiles would)
  if (akc && bkc && (p.M <= 16 || (p.M <= 32 && p.K <= 1024)) && (p.N + 15) / 16 <= kMaxTiles) {
    p.shape = kRowsShape;
    p.tiles_m = 1;
    p.tiles_n = (p.N + 15) / 16;
    p.slices_per = std::max(slices, 1);
    return true;
  }
  static const int bm[] = {64, 128, 256}, bn[] = {64, 128, 256};
  auto tiles = [&](int s) {
    return (long long)((p.M + bm[s] - 1) / bm[s]) * ((p.N + bn[s] - 1) / bn[s]);
  };
  // 256 x 256 tiles (16-bit operands) where they fill their last round of a tile per CU to three
  // quarters: 64,000 x 512, K = 2,048 155 us against 177 by 128 x 128; 40,000 x 512, K = 500, a
  // quarter of a second round, 46.8 against 42.9.  fp32 operands, bound by their matrix
  // instructions, spread best in small tiles: 8,000 x 384, K = 512 31.8 us by 64 x 64, 47.2 by
  // 128 x 128.
  // A tile no more than twice as wide as the result.
  const long long rounds = (tiles(2) + cus - 1) / cus;
  const int least = std::min(p.M, p.N);
  if (dtype == kF32) p.shape = least > 64 && tiles(1) >= 4 * cus ? 1 : 0;
  else if (least > 128 && 4 * tiles(2) >= 3 * rounds * cus) p.shape = 2;
  else p.shape = least > 64 && tiles(1) * slices >= 8 * cus ? 1 : 0;
  p.tiles_m = (p.M + bm[p.shape] - 1) / bm[p.shape];
  p.tiles_n = (p.N + bn[p.shape] - 1) / bn[p.shape];
  const long long n = tiles(p.shape);
  long long splits = 1;
  // Fewer tiles than CUs: k in parts of 8 slices at least, as many as the CUs hold at once (three
  // workgroups of 64 x 64 tiles each, two of 128 x 128): dW of 512 x 384 fp32 over 8,000 rows, 48
  // tiles, 41 us in 16 parts, 51 in 11, whose CUs have two or three; of 500 x 512 bf16 over 40,000,
  // 16 tiles, 41 in 32, 66 in 8.  Shorter parts do not pay for the join (512 x 512, K = 512 bf16
  // 15.5 us whole, 19 in 2), but for fp32, whose slices take longest, down to 4 slices while no CU
  // has two (369 x 256, K = 512 11.4 us in 2 parts, 9.2 in 4; 935 x 500, K = 640 14.8 in 2, 18.8 in 5).
  if (n < cus) {
    splits = std::max(1ll, std::min((p.shape == 0 ? 3 : 2) * cus / n, (long long)slices / 8));
    if (dtype == kF32) splits = std::max(splits, std::min(cus / n, (long long)slices / 4));
  }
  p.slices_per = std::max(1, (int)((slices + splits - 1) / splits));
  p.splits = std::max(1, (slices + p.slices_per - 1) / p.slices_per);
  return true;
}

hipError_t launch_product(const ProductArgs& p, int dtype, bool akc, bool bkc, hipStream_t st) {
  if (p.M == 0 || p.N == 0) return hipSuccess;
  if (dtype == kF32) return launch_product_t<float>(p, akc, bkc, st);
  if (dtype == kBF16) return launch_product_t<bf16>(p, akc, bkc, st);
  return launch_product_t<_Float16>(p, akc, bkc, st);
}

template <class T>
static hipError_t launch_act_grad_t(const void* dy, long long ldy, const void* pre, long long ldp, void* dz,
                                    long long ldz, void* low, long long ldl, int M, int N, int act, hipStream_t st) {
  const long long items = (long long)M * ((N + kChunkElems<T> - 1) / kChunkElems<T>);
  const long long blocks = std::min<long long>((items + 255) / 256, 1 << 20);
  hipLaunchKernelGGL(k_act_grad<T>, dim3((unsigned)blocks), dim3(256), 0, st, (const T*)dy, ldy, (const T*)pre, ldp,
                     (T*)dz, ldz, (T*)low, ldl, M, N, act);
  return hipGetLastError();
}

hipError_t launch_act_grad(int dtype, const void* dy, long long ldy, const void* pre, long long ldp, void* dz,
                           long long ldz, void* low, long long ldl, int M, int N, int act, hipStream_t st) {
  if (M == 0 || N == 0) return hipSuccess;
  if (ldy == N && ldp == N && ldz == N && (!low || ldl == N) && (long long)M * N < (1ll << 30)) {  // one long row
    N *= M;
    M = 1;
    ldy = ldp = ldz = ldl = N;
  }
  if (dtype == kF32) return launch_act_grad_t<float>(dy, ldy, pre, ldp, dz, ldz, low, ldl, M, N, act, st);
  if (dtype == kBF16) return launch_act_grad_t<bf16>(dy, ldy, pre, ldp, dz, ldz, low, ldl, M, N, act, st);
  return launch_act_grad_t<_Float16>(dy, ldy, pre, ldp, dz, ldz, low, ldl, M, N, act, st);
}

}  // namespace tbs
