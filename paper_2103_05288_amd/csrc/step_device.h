// Device code of what a decoder's step runs around its attention: the norm that adds the residual and leaves 8-bit
// rows with scales, and its gradient; products of few rows with 4-bit weights; the check of drafted tokens.  Compiled
// through hipRTC once per registration, with what never changes between calls as macros; rows, widths, vocabularies and
// strides are arguments.
//
//   DISC_NORM:    DISC_T, DISC_STORAGE (1: i8, 2: e4m3), DISC_EPS, DISC_OFFSET
//   DISC_LINEAR4: DISC_T_F16 (0: bf16), DISC_ROWS (0: as the results, 1: i8, 2: e4m3), DISC_GROUP (32, 64, 128), DISC_ZEROS
//   DISC_VERIFY:  DISC_T
#pragma once
typedef unsigned char u8;
typedef unsigned short u16;
typedef unsigned int u32;
typedef long long i64;
typedef unsigned long long u64;
typedef u32 u32x2 __attribute__((ext_vector_type(2)));
typedef u32 u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
#define DISC_DEV __device__ __forceinline__

// wide accesses at any element's address (the operands' strides and pointers are the caller's)
typedef u32x4 u32x4_u __attribute__((aligned(1)));
typedef u32x2 u32x2_u __attribute__((aligned(1)));
template <bool kNt, class V>
DISC_DEV V fetch(const V* p) {
  if (kNt) return __builtin_nontemporal_load(p);
  return *p;
}
template <bool kNt, class V>
DISC_DEV void put(V* p, V x) {
  if (kNt) __builtin_nontemporal_store(x, p);
  else *p = x;
}

#ifdef DISC_NORM
// =================================================================================================
// s = x + residual (32 bits), total = s rounded, y = s w / sqrt(mean(s^2) + eps) with w = weight + offset, and y as codes
// of 8 bits with a scale for the row.  The row's root cancels in its codes,
//   code = round(s w (Q / a)), scale = a / (sqrt(mean(s^2) + eps) Q), a = max |s w|,
// so that both reductions (a, and the sum of squares, which only the scale needs) are one.
// Squares are summed in 64 bits: no finite row overflows, and the sum is not what limits the result.
// =================================================================================================
typedef DISC_T T;
constexpr int kV = 16 / (int)sizeof(T);                     // elements of one access
constexpr float kMost = DISC_STORAGE == 1 ? 127.f : 448.f;  // largest code
constexpr int kMostWaves = 16;
typedef T vec_t __attribute__((ext_vector_type(kV)));
typedef vec_t vec_u __attribute__((aligned(alignof(T))));

// `n` elements of a row from p on (the rest zeros): one access, or the ragged end of a row by single elements
template <bool kNt>
DISC_DEV vec_t take(const T* p, i64 n) {
  if (n >= kV) return (vec_t)fetch<kNt>((const vec_u*)p);
  vec_t v = {};
#pragma unroll
  for (int e = 0; e < kV - 1; ++e)
    if (e < n) v[e] = p[e];
  return v;
}
template <bool kNt>
DISC_DEV void give(T* p, vec_t v, i64 n) {
  if (n >= kV) {
    put<kNt>((vec_u*)p, (vec_u)v);
    return;
  }
#pragma unroll
  for (int e = 0; e < kV - 1; ++e)
    if (e < n) p[e] = v[e];
}

DISC_DEV double shuffled(double x, int by) {
  const u64 b = __builtin_bit_cast(u64, x);
  const u32 lo = (u32)__shfl_xor((int)(u32)b, by), hi = (u32)__shfl_xor((int)(u32)(b >> 32), by);
  return __builtin_bit_cast(double, ((u64)hi << 32) | lo);
}
DISC_DEV u32 magnitude(float x) { return __builtin_bit_cast(u32, x) & 0x7fffffffu; }   // (orders as |x| does, NaN above infinity)

// Sums of `lanes` neighbouring threads (a power of two; above 64, whole wavefronts through LDS), the same in all of them.
struct Group {
  int lanes, first_wave, waves;
  DISC_DEV Group(int l) : lanes(l), first_wave(0), waves(0) {
    if (lanes > 64) {
      waves = lanes / 64;
      first_wave = (int)threadIdx.x / lanes * waves;
    }
  }
  template <class X, class F>
  DISC_DEV X over(X x, X* kept, F f) const {
    for (int s = 1; s < lanes && s < 64; s *= 2) x = f(x, shuffle(x, s));
    if (waves) {
      __syncthreads();
      if (threadIdx.x % 64 == 0) kept[threadIdx.x / 64] = x;
      __syncthreads();
      x = kept[first_wave];
      for (int w = 1; w < waves; ++w) x = f(x, kept[first_wave + w]);
    }
    return x;
  }
  DISC_DEV static double shuffle(double x, int s) { return shuffled(x, s); }
  DISC_DEV static u32 shuffle(u32 x, int s) { return (u32)__shfl_xor((int)x, s); }
};

struct NormArgs {
  const T *x, *residual, *weight;
  T* total;
  u8* codes;
  float* scales;
  i64 x_row, residual_row, total_row, codes_row, rows;
  int width, lanes;         // lanes: threads of a row
};

DISC_DEV u32 code4(float a, float b, float c, float d) {
  const float y[4] = {__builtin_amdgcn_fmed3f(a, -kMost, kMost), __builtin_amdgcn_fmed3f(b, -kMost, kMost), __builtin_amdgcn_fmed3f(c, -kMost, kMost),
                      __builtin_amdgcn_fmed3f(d, -kMost, kMost)};
#if DISC_STORAGE == 2
  int p = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return (u32)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], p, true);
#else
  u32 p = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) p |= ((u32)(int)__builtin_rintf(y[e]) & 0xffu) << (8 * e);
  return p;
#endif
}

template <bool kNt, int kN>
DISC_DEV void norm_body(const NormArgs& A) {
  __shared__ double sums[kMostWaves], most64[kMostWaves];
  __shared__ u32 most[kMostWaves];
  const Group group(A.lanes);
  const int lane = (int)threadIdx.x % A.lanes;
  const i64 at = (i64)blockIdx.x * ((int)blockDim.x / A.lanes) + (int)threadIdx.x / A.lanes;
  const bool live = at < A.rows;
  const i64 row = live ? at : A.rows - 1;                  // (all threads reach the barriers)
  float s[kN][kV], w[kN][kV];
  double squares = 0;
  u32 a = 0;
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const int c = (i * A.lanes + lane) * kV;
    const int n = A.width - c;
    if (n > 0) {
      const vec_t x = take<kNt>(A.x + row * A.x_row + c, n), v = take<false>(A.weight + c, n);
      vec_t r = {};
      if (A.residual) r = take<kNt>(A.residual + row * A.residual_row + c, n);
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        s[i][e] = (float)x[e] + (float)r[e];
        w[i][e] = (float)v[e] + (e < n ? (float)DISC_OFFSET : 0.f);
      }
    } else {
#pragma unroll
      for (int e = 0; e < kV; ++e) s[i][e] = w[i][e] = 0.f;
    }
#pragma unroll
    for (int e = 0; e < kV; ++e) {
      squares += (double)s[i][e] * (double)s[i][e];
      a = max(a, magnitude(s[i][e] * w[i][e]));
    }
  }
  if (A.total && live) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int c = (i * A.lanes + lane) * kV;
      vec_t t;
#pragma unroll
      for (int e = 0; e < kV; ++e) t[e] = (T)s[i][e];
      if (c < A.width) give<kNt>(A.total + row * A.total_row + c, t, A.width - c);
    }
  }
  squares = group.over(squares, sums, [](double p, double q) { return p + q; });
  a = group.over(a, most, [](u32 p, u32 q) { return max(p, q); });
  const double root = 1.0 / sqrt(squares / (double)A.width + (double)DISC_EPS);
  // Where a product leaves what 32 bits hold well -- above their range, or so small that Q / a would be infinite -- they
  // are formed in 64.  (By the whole block, for the barriers.)
  float largest = __builtin_bit_cast(float, a);
  const bool wide = !(largest >= 0x1p-100f && largest < __builtin_inff());
  double largest64 = (double)largest;
  if (__syncthreads_or(wide)) {
    double m = 0;
#pragma unroll
    for (int i = 0; i < kN; ++i)
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        const double y = __builtin_fabs((double)s[i][e] * (double)w[i][e]);
        m = !(y <= m) ? y : m;                              // (a NaN replaces whatever was there, and stays below)
        if (!(m < __builtin_inf())) m = __builtin_inf();
      }
    m = group.over(m, most64, [](double p, double q) { return p > q ? p : q; });
    if (wide) largest64 = m;                                // (a row's scale does not depend on its neighbours)
  }
  if (!live) return;
  const double scale = largest64 > 0 ? largest64 * root / (double)kMost : 0.0;
  const bool fine = (float)scale < __builtin_inff();         // (not NaN either)
  if (lane == 0) A.scales[row] = fine ? (float)scale : __builtin_nanf("");
  const float inverse = kMost / largest;
  const double inverse64 = fine && largest64 > 0 ? (double)kMost / largest64 : 0.0;
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const int c = (i * A.lanes + lane) * kV;
    const int n = A.width - c;
    if (n <= 0) break;
    float y[kV];
#pragma unroll
    for (int e = 0; e < kV; ++e) y[e] = s[i][e] * w[i][e] * inverse;
    if (wide) {
#pragma unroll
      for (int e = 0; e < kV; ++e) y[e] = fine ? (float)((double)s[i][e] * (double)w[i][e] * inverse64) : 0.f;
    }
    u8* to = A.codes + row * A.codes_row + c;
    u32 code[kV / 4];
#pragma unroll
    for (int k = 0; k < kV / 4; ++k) code[k] = code4(y[4 * k], y[4 * k + 1], y[4 * k + 2], y[4 * k + 3]);
    if (n >= kV) {
      typedef u32 words __attribute__((ext_vector_type(kV / 4)));
      typedef words words_u __attribute__((aligned(1)));
      words p;
#pragma unroll
      for (int k = 0; k < kV / 4; ++k) p[k] = code[k];
      put<kNt>((words_u*)to, (words_u)p);
    } else {
#pragma unroll
      for (int e = 0; e < kV - 1; ++e)
        if (e < n) to[e] = (u8)(code[e / 4] >> (8 * (e % 4)));
    }
  }
}

// The gradient.  With u = s / root(s), g = w dy:  dx = (g - u mean(g u)) / root(s) + dtotal,  dweight = sum over rows of dy u.
// (The rounding to codes counts as the identity.)  A block has a share of the rows and keeps its columns' part of dweight
// in registers; the parts, a row of the workspace for each group of threads, are summed by a second launch in a fixed order.
struct NormBackwardArgs {
  const T *total, *weight, *dy, *dtotal;
  T* dx;
  float *dweight, *part;
  i64 total_row, dy_row, dtotal_row, dx_row, rows;
  int width, lanes, parts;
};

template <bool kNt, int kN>
DISC_DEV void norm_backward_body(const NormBackwardArgs& A) {
  __shared__ double sums[kMostWaves], alongs[kMostWaves];
  const Group group(A.lanes);
  const int lane = (int)threadIdx.x % A.lanes, groups = (int)blockDim.x / A.lanes;
  const int mine = (int)blockIdx.x * groups + (int)threadIdx.x / A.lanes;
  float dw[kN][kV] = {};
  for (i64 at = mine; at - (int)threadIdx.x / A.lanes < A.rows; at += A.parts) {
    const bool live = at < A.rows;                          // (all threads reach the barriers)
    const i64 row = live ? at : A.rows - 1;
    vec_t h[kN], d[kN], v[kN], t[kN];
    double squares = 0, along = 0;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int c = (i * A.lanes + lane) * kV;
      const int n = A.width - c;
      h[i] = d[i] = v[i] = t[i] = vec_t{};
      if (n <= 0) continue;
      h[i] = take<kNt>(A.total + row * A.total_row + c, n);
      d[i] = take<kNt>(A.dy + row * A.dy_row + c, n);
      v[i] = take<false>(A.weight + c, n);
      if (A.dtotal) t[i] = take<kNt>(A.dtotal + row * A.dtotal_row + c, n);
    }
#pragma unroll
    for (int i = 0; i < kN; ++i)
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        const double x = (double)(float)h[i][e];
        squares += x * x;
        along += x * (double)((float)d[i][e]) * (double)((float)v[i][e] + (float)DISC_OFFSET);
      }
    squares = group.over(squares, sums, [](double p, double q) { return p + q; });
    along = group.over(along, alongs, [](double p, double q) { return p + q; });
    if (!live) continue;
    const double root = 1.0 / sqrt(squares / (double)A.width + (double)DISC_EPS);
    const float r = (float)root, k = (float)(root * along / (double)A.width);
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int c = (i * A.lanes + lane) * kV;
      if (c >= A.width) break;
      vec_t y;
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        const float u = (float)h[i][e] * r, dy = (float)d[i][e], g = dy * ((float)v[i][e] + (float)DISC_OFFSET);
        dw[i][e] += dy * u;
        y[e] = (T)(r * (g - u * k) + (float)t[i][e]);
      }
      give<kNt>(A.dx + row * A.dx_row + c, y, A.width - c);
    }
  }
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const int c = (i * A.lanes + lane) * kV;
#pragma unroll
    for (int e = 0; e < kV; ++e)
      if (c + e < A.width) A.part[(i64)mine * A.width + c + e] = dw[i][e];
  }
}

#define DISC_NORM_KERNELS(N)                                                                                                              \
  extern "C" __global__ void __launch_bounds__(1024) disc_norm##N##_k(NormArgs A) { norm_body<false, N>(A); }                             \
  extern "C" __global__ void __launch_bounds__(1024) disc_norm##N##_nt_k(NormArgs A) { norm_body<true, N>(A); }                           \
  extern "C" __global__ void __launch_bounds__(512) disc_norm_backward##N##_k(NormBackwardArgs A) { norm_backward_body<false, N>(A); }     \
  extern "C" __global__ void __launch_bounds__(512) disc_norm_backward##N##_nt_k(NormBackwardArgs A) { norm_backward_body<true, N>(A); }
DISC_NORM_KERNELS(1)
DISC_NORM_KERNELS(2)
DISC_NORM_KERNELS(4)
DISC_NORM_KERNELS(8)

// dweight: a block has 64 columns, four threads each of a quarter of the parts.
extern "C" __global__ void __launch_bounds__(256) disc_norm_join_k(NormBackwardArgs A) {
  __shared__ float kept[4][64];
  const int c = (int)blockIdx.x * 64 + (int)threadIdx.x % 64, q = (int)threadIdx.x / 64;
  float sum = 0;
  if (c < A.width)
    for (int p = q; p < A.parts; p += 4) sum += A.part[(i64)p * A.width + c];
  kept[q][threadIdx.x % 64] = sum;
  __syncthreads();
  if (q == 0 && c < A.width) A.dweight[c] = (kept[0][threadIdx.x] + kept[1][threadIdx.x]) + (kept[2][threadIdx.x] + kept[3][threadIdx.x]);
}
#endif  // DISC_NORM

#ifdef DISC_LINEAR4
// =================================================================================================
// y[m, n] = r[m] sum_k x[m, k] s[n, k / G] (c[n, k] - z[n, k / G]) + bias[n] with codes c of 4 bits.
// =================================================================================================
#if DISC_T_F16
typedef _Float16 T;
#else
typedef __bf16 T;
#endif
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef long i8x8;
constexpr int kG = DISC_GROUP;
constexpr int kBlockK = 128;                               // elements of a row that a wavefront takes at once: 16 bytes a lane
constexpr int kGroups = kBlockK / kG;                      // groups of them
// what is multiplied: 0 bf16, 1 f16 (e4m3 rows are brought to it, exactly), 2 i8
constexpr int kKind = DISC_ROWS == 1 ? 2 : DISC_ROWS == 2 || DISC_T_F16 ? 1 : 0;
constexpr int kRowSize = DISC_ROWS ? 1 : 2;

struct LinearArgs {
  const u8* x;
  const u8* weights;
  const T* scales;
  const float* row_scales;
  const u8* zeros;
  const T* bias;
  T* out;
  i64 x_row, out_row;
  int rows, n, k, groups;                                  // groups: of a row of weights
};

// Where the eight elements of dword j of a lane (with q = lane / 16) stand in a block of 128 (see arrange()).
DISC_DEV int place(int j, int q) {
  return kG == 128 ? q * 32 + j * 8 : kG == 64 ? (j >> 1) * 64 + (q & 1) * 32 + (q >> 1) * 16 + (j & 1) * 8 : j * 32 + q * 8;
}
// A lane reads 32 neighbouring codes, dword j of them goes to product j.  A product sums over the four lanes q = 0 .. 3 of a
// row, which have to be of one group: lanes swap dwords, halves of the wavefront for groups of 64, rows of 16 lanes too for 32.
DISC_DEV u32x4 arrange(u32x4 d) {
  if (kG <= 64) {
    const auto a = __builtin_amdgcn_permlane32_swap(d[0], d[2], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(d[1], d[3], false, false);
    d = u32x4{a[0], b[0], a[1], b[1]};
  }
  if (kG == 32) {
    const auto a = __builtin_amdgcn_permlane16_swap(d[0], d[1], false, false);
    const auto b = __builtin_amdgcn_permlane16_swap(d[2], d[3], false, false);
    d = u32x4{a[0], a[1], b[0], b[1]};
  }
  return d;
}

// Eight codes as an operand, in the order 0 4 1 5 2 6 3 7.
// bf16: 128 + c by setting the exponent's bits; what that adds to the sum is taken off with the zero point.
// f16:  1024 + c and 1024 + 16 c, from which c - 8 is exact.
DISC_DEV u32x4 widen(u32 d) {
  if (kKind == 0) return (u32x4{d, d >> 4, d >> 8, d >> 12} & 0x000f000fu) | 0x43004300u;
  const u32 e = d >> 8;
  const u32x4 raw = {(d & 0x000f000fu) | 0x64006400u, (d & 0x00f000f0u) | 0x64006400u, (e & 0x000f000fu) | 0x64006400u, (e & 0x00f000f0u) | 0x64006400u};
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const u32 pair = raw[i];                                // (a bit cast of a vector's element itself takes its first one)
    const f16x2 h = __builtin_bit_cast(f16x2, pair);
    const f16x2 w = i & 1 ? h * f16x2{(_Float16)0.0625f, (_Float16)0.0625f} - f16x2{(_Float16)72.f, (_Float16)72.f} : h - f16x2{(_Float16)1032.f, (_Float16)1032.f};
    r[i] = __builtin_bit_cast(u32, w);
  }
  return r;
}
// Eight elements of x in that order.
DISC_DEV u32x4 reorder(u32x4 d) {
  return u32x4{__builtin_amdgcn_perm(d[2], d[0], 0x05040100u), __builtin_amdgcn_perm(d[2], d[0], 0x07060302u), __builtin_amdgcn_perm(d[3], d[1], 0x05040100u),
               __builtin_amdgcn_perm(d[3], d[1], 0x07060302u)};
}
DISC_DEV u32 pack16(float a, float b) { return __builtin_bit_cast(u32, f16x2{(_Float16)a, (_Float16)b}); }
// ... of eight e4m3 codes, in half precision (each is a number of it)
DISC_DEV u32x4 reorder8(u32x2 d) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)d[0], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)d[0], true);
  const auto c = __builtin_amdgcn_cvt_pk_f32_fp8((int)d[1], false), e = __builtin_amdgcn_cvt_pk_f32_fp8((int)d[1], true);
  return u32x4{pack16(a[0], c[0]), pack16(a[1], c[1]), pack16(b[0], e[0]), pack16(b[1], e[1])};
}

// What a lane has of a block of 128 elements of kTiles tiles of 16 rows of x: by dword of codes.  i8: two dwords, even
// elements and odd ones.
template <int kM>
struct Rows {
  u32x4 v[kM][4];
};

template <int kM>
DISC_DEV void take_rows(const LinearArgs& A, int row0, int block, int q, int m, Rows<kM>& r) {
#pragma unroll
  for (int t = 0; t < kM; ++t) {
    const int row = min(row0 + t * 16 + m, A.rows - 1);     // (rows behind the last: a copy, not stored)
    const u8* p = A.x + (i64)row * A.x_row * kRowSize;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int k = block * kBlockK + place(j, q);
      u32x4 v = {0, 0, 0, 0};
      if (k < A.k) {
        if (kRowSize == 2) {
          v = *(const u32x4_u*)(p + (i64)k * 2);
        } else {
          const u32x2 c = *(const u32x2_u*)(p + k);
          v[0] = c[0];
          v[1] = c[1];
        }
      }
      r.v[t][j] = v;
    }
  }
}

template <int kM, int kWaves>
DISC_DEV void linear_body(const LinearArgs& A) {
  __shared__ float kept[kWaves][kM][256];
  const int lane = (int)threadIdx.x % 64, wave = (int)threadIdx.x / 64;
  const int c = lane % 16, q = lane / 16;
  const int n = (int)blockIdx.x * 16 + c, row0 = (int)blockIdx.y * 16 * kM;
  const i64 nn = min(n, A.n - 1);
  const u8* w = A.weights + nn * (A.k / 2);
  const T* scales = A.scales + nn * A.groups;
  const u8* zeros = DISC_ZEROS ? A.zeros + nn * A.groups : nullptr;
  f32x4 total[kM] = {};
  const int blocks = (A.k + kBlockK - 1) / kBlockK;
  for (int b = wave; b < blocks; b += kWaves) {
    u32x4 d = {0, 0, 0, 0};
    if (b * kBlockK + q * 32 < A.k) d = *(const u32x4*)(w + (i64)b * (kBlockK / 2) + q * 16);
    Rows<kM> x;
    take_rows<kM>(A, row0, b, q, c, x);
    d = arrange(d);
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int group = min(b * kGroups + g, A.groups - 1);
      const float s = (float)scales[group];
      const int z = DISC_ZEROS ? (int)zeros[group] : 8;
#pragma unroll
      for (int t = 0; t < kM; ++t) {
        if constexpr (kKind == 2) {
          i32x4 acc = {}, sum = {};
          const u32 ones = 0x01010101u;
#pragma unroll
          for (int j = g * 4 / kGroups; j < (g + 1) * 4 / kGroups; ++j) {
            const u32 lo = d[j] & 0x0f0f0f0fu, hi = (d[j] >> 4) & 0x0f0f0f0fu;
            const u32 even = __builtin_amdgcn_perm(x.v[t][j][1], x.v[t][j][0], 0x06040200u), odd = __builtin_amdgcn_perm(x.v[t][j][1], x.v[t][j][0], 0x07050301u);
            const i8x8 xs = (i8x8)(((u64)odd << 32) | even), ws = (i8x8)(((u64)hi << 32) | lo), os = (i8x8)(((u64)ones << 32) | ones);
            acc = __builtin_amdgcn_mfma_i32_16x16x32_i8(xs, ws, acc, 0, 0, 0);
            sum = __builtin_amdgcn_mfma_i32_16x16x32_i8(xs, os, sum, 0, 0, 0);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) total[t][i] += s * (float)(acc[i] - z * sum[i]);
        } else {
          f32x4 acc = {}, sum = {};
#pragma unroll
          for (int j = g * 4 / kGroups; j < (g + 1) * 4 / kGroups; ++j) {
            const u32x4 v = kRowSize == 1 ? reorder8(u32x2{x.v[t][j][0], x.v[t][j][1]}) : reorder(x.v[t][j]), u = widen(d[j]);
            if constexpr (kKind == 0) {
              const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
              acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, u), acc, 0, 0, 0);
              sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, ones), sum, 0, 0, 0);
            } else {
              const u32x4 ones = {0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u};
              acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, v), __builtin_bit_cast(f16x8, u), acc, 0, 0, 0);
              if (DISC_ZEROS) sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, v), __builtin_bit_cast(f16x8, ones), sum, 0, 0, 0);
            }
          }
          const float off = kKind == 0 ? 128.f + (float)z : (float)(z - 8);
#pragma unroll
          for (int i = 0; i < 4; ++i) total[t][i] += s * (kKind == 0 || DISC_ZEROS ? acc[i] - off * sum[i] : acc[i]);
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < kM; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) kept[wave][t][(q * 4 + i) * 16 + c] = total[t][i];
  __syncthreads();
  for (int o = (int)threadIdx.x; o < kM * 256; o += kWaves * 64) {
    const int m = row0 + o / 16, col = (int)blockIdx.x * 16 + o % 16;
    if (m >= A.rows || col >= A.n) continue;
    float y = 0;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) y += kept[v][o / 256][o % 256];
    if (DISC_ROWS) y *= A.row_scales[m];
    if (A.bias) y += (float)A.bias[col];
    A.out[m * A.out_row + col] = (T)y;
  }
}
extern "C" __global__ void __launch_bounds__(512) disc_linear1_k(LinearArgs A) { linear_body<1, 8>(A); }
extern "C" __global__ void __launch_bounds__(512) disc_linear2_k(LinearArgs A) { linear_body<2, 8>(A); }
extern "C" __global__ void __launch_bounds__(512) disc_linear4_k(LinearArgs A) { linear_body<4, 8>(A); }
#endif  // DISC_LINEAR4

#ifdef DISC_VERIFY
// =================================================================================================
// Drafted tokens x_0 .. x_{n-1} against the target's probabilities p_0 .. p_n: x_i is kept while u_i q_i(x_i) < p_i(x_i).
// The token behind the kept ones is drawn from max(p - q, 0) of the first place that was not kept, or from p_n:
// the first whose running sum passes u times the whole.  Products of two 32-bit numbers and differences are formed, and
// sums kept, in 64 bits, in a fixed order.
// =================================================================================================
typedef DISC_T T;
constexpr int kV = 16 / (int)sizeof(T);
typedef T vec_t __attribute__((ext_vector_type(kV)));
typedef vec_t vec_u __attribute__((aligned(alignof(T))));
constexpr int kChunk = 4096;                               // elements of a row that a block sums

struct VerifyArgs {
  const T *target, *draft;
  const int *drafted, *lengths;
  const float* uniforms;
  int *tokens, *accepted;
  double* part;                                            // [batch][chunks][2]: sums of max(p - q, 0), and of p
  i64 target_batch, target_row, draft_batch, draft_row;
  int batch, drafts, vocabulary, chunks;
};

DISC_DEV double weight(double x) { return x > 0 && x < __builtin_inf() ? x : 0.0; }

// The drafted tokens of sequence b that are kept, by one wavefront: the same in all of its lanes.
DISC_DEV int kept_of(const VerifyArgs& A, i64 b, int lane) {
  const int n = A.lengths ? min(max(A.lengths[b], 0), A.drafts) : A.drafts;
  for (int first = 0; first < n; first += 64) {
    const int i = first + lane;
    bool bad = false;
    if (i < n) {
      const int x = A.drafted[b * A.drafts + i];
      bad = true;
      if (x >= 0 && x < A.vocabulary) {
        const double p = (double)(float)A.target[b * A.target_batch + i * A.target_row + x];
        const double q = A.draft ? (double)(float)A.draft[b * A.draft_batch + i * A.draft_row + x] : 1.0;
        bad = !((double)A.uniforms[b * (A.drafts + 1) + i] * q < p);
      }
    }
    const u64 mask = __ballot(bad);
    if (mask) return first + __builtin_ctzll(mask);
  }
  return n;
}

// What the last token's weights are made of.
struct Place {
  const T *p, *q;       // q: null where nothing is taken off
  int removed;          // the token without weight (no draft probabilities: the drafted one); -1
  DISC_DEV Place(const VerifyArgs& A, i64 b, int kept) {
    const int n = A.lengths ? min(max(A.lengths[b], 0), A.drafts) : A.drafts;
    p = A.target + b * A.target_batch + kept * A.target_row;
    q = kept < n && A.draft ? A.draft + b * A.draft_batch + kept * A.draft_row : nullptr;
    removed = kept < n && !A.draft ? A.drafted[b * A.drafts + kept] : -1;
  }
  DISC_DEV bool less() const { return q != nullptr || removed >= 0; }
};
DISC_DEV double sum_of(double x, double* kept, int threads) {
  for (int s = 1; s < 64; s *= 2) {
    const u64 b = __builtin_bit_cast(u64, x);
    const u32 lo = (u32)__shfl_xor((int)(u32)b, s), hi = (u32)__shfl_xor((int)(u32)(b >> 32), s);
    x += __builtin_bit_cast(double, ((u64)hi << 32) | lo);
  }
  __syncthreads();
  if (threadIdx.x % 64 == 0) kept[threadIdx.x / 64] = x;
  __syncthreads();
  x = 0;
  for (int w = 0; w < threads / 64; ++w) x += kept[w];
  return x;
}

extern "C" __global__ void __launch_bounds__(256) disc_verify_sum_k(VerifyArgs A) {
  __shared__ double kept_sums[4];
  __shared__ int kept_s;
  const i64 b = blockIdx.x / (u32)A.chunks;
  const int chunk = (int)(blockIdx.x - (u32)b * (u32)A.chunks);
  if (threadIdx.x < 64) {
    const int k = kept_of(A, b, (int)threadIdx.x);
    if (threadIdx.x == 0) {
      kept_s = k;
      if (chunk == 0) A.accepted[b] = k;
    }
  }
  __syncthreads();
  const Place at(A, b, kept_s);
  const int first = chunk * kChunk, end = min(A.vocabulary - first, kChunk);
  double less = 0, all = 0;
  for (int i = (int)threadIdx.x; i < end; i += 256) {
    const double p = weight((double)(float)at.p[first + i]);
    all += p;
    if (at.q) less += weight((double)(float)at.p[first + i] - (double)(float)at.q[first + i]);
    else if (first + i != at.removed) less += p;
  }
  less = sum_of(less, kept_sums, 256);
  all = sum_of(all, kept_sums, 256);
  if (threadIdx.x == 0) {
    double* to = A.part + (b * A.chunks + chunk) * 2;
    to[0] = less;
    to[1] = all;
  }
}

extern "C" __global__ void __launch_bounds__(256) disc_verify_pick_k(VerifyArgs A) {
  __shared__ double kept_sums[4];
  __shared__ double upto[256];
  __shared__ int found, last, chunk_s, column_s;
  __shared__ double before_s, goal_s;
  const i64 b = blockIdx.x;
  const int kept = A.accepted[b];
  const Place at(A, b, kept);
  const double* part = A.part + b * A.chunks * 2;
  if (threadIdx.x == 0) {
    double less = 0, all = 0;
    for (int i = 0; i < A.chunks; ++i) {
      less += part[2 * i];
      all += part[2 * i + 1];
    }
    const int column = at.less() && less > 0 ? 0 : 1;
    const double whole = column ? all : less, u = (double)A.uniforms[b * (A.drafts + 1) + A.drafts];
    const double goal = (u > 0 ? u : 0.0) * whole;
    double before = 0, sum = 0;
    int chunk = -1;
    for (int i = 0; i < A.chunks; ++i) {
      const double x = part[2 * i + column];
      if (x > 0) {
        chunk = i;
        before = sum;
        if (sum + x > goal) break;
      }
      sum += x;
    }
    chunk_s = chunk;
    column_s = column;
    before_s = before;
    goal_s = goal;
    found = 0x7fffffff;
    last = -1;
  }
  __syncthreads();
  const int chunk = chunk_s, column = column_s;
  if (chunk >= 0) {
    // (a thread has neighbouring elements of the chunk)
    constexpr int kEach = kChunk / 256;
    const int first = chunk * kChunk + (int)threadIdx.x * kEach;
    double x[kEach], sum = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int i = first + e;
      x[e] = 0;
      if (i < A.vocabulary) {
        const double p = (double)(float)at.p[i];
        x[e] = weight(column == 0 && at.q ? p - (double)(float)at.q[i] : p);
        if (column == 0 && i == at.removed) x[e] = 0;
      }
      sum += x[e];
    }
    upto[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
      double s = before_s;
      for (int t = 0; t < 256; ++t) {
        const double y = upto[t];
        upto[t] = s;
        s += y;
      }
    }
    __syncthreads();
    double s = upto[threadIdx.x];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      s += x[e];
      if (x[e] > 0) {
        atomicMax(&last, first + e);
        if (s > goal_s) atomicMin(&found, first + e);
      }
    }
  }
  __syncthreads();
  const int token = found != 0x7fffffff ? found : last;
  for (int i = (int)threadIdx.x; i <= A.drafts; i += 256) A.tokens[b * (A.drafts + 1) + i] = i < kept ? A.drafted[b * A.drafts + i] : i == kept ? token : -1;
}
#endif  // DISC_VERIFY
