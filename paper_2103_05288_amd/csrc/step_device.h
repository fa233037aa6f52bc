// Device code of what a decoder's step runs around its attention: the norm that adds the residual and leaves 8-bit
// rows with scales, and its gradient; products of few rows with 4-bit weights; the check of drafted tokens.  Compiled
// through hipRTC once per registration, with what never changes between calls as macros; rows, widths, vocabularies and
// strides are arguments.
//
//   DISC_NORM:    DISC_T, DISC_STORAGE (1: i8, 2: e4m3)
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
typedef u32 u32_u __attribute__((aligned(1)));
typedef u16 u16_u __attribute__((aligned(1)));
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
// Bound by memory: a row is read once and stays in registers between its sums and its codes, 16 bytes a lane and access, so rows of up to
// 512 bytes a part of a wavefront each and longer ones a block.  16384 x 8192 bf16 with a residual to e4m3 154 us a call, 6.1 TB/s (a copy 5.4).
// Few rows are bound by a chain of one trip to memory and one exchange (333 x 1001: 3.8 us of kernel).
// =================================================================================================
typedef DISC_T T;
constexpr int kV = 16 / (int)sizeof(T);                     // elements of one access
constexpr float kMost = DISC_STORAGE == 1 ? 127.f : 448.f;  // largest code
constexpr int kMostWaves = 16;
typedef T vec_t __attribute__((ext_vector_type(kV)));
typedef vec_t vec_u __attribute__((aligned(alignof(T))));

// `n` elements of a row of `width` from p on (n is 1 at least): one access, which at the ragged end of a row is its last kV elements
// (rows shorter than that: single ones).  settle() puts them in place, with zeros behind them, once every load is on its way (with the
// end's elements loaded one by one, a block's loads waited for each other: 9179 x 6879 fp16 151 us, 6880 80).
template <bool kNt>
DISC_DEV vec_t take(const T* p, int n, int width) {
  if (width >= kV) return (vec_t)fetch<kNt>((const vec_u*)(p - max(kV - n, 0)));
  vec_t v = {};
#pragma unroll
  for (int e = 0; e < kV - 1; ++e)
    if (e < n) v[e] = p[e];
  return v;
}
DISC_DEV void settle(vec_t& v, int n, int width) {
  if (n >= kV || n <= 0 || width < kV) return;
  typedef u64 halves __attribute__((ext_vector_type(2)));
  halves h = __builtin_bit_cast(halves, v);
  const int by = (kV - n) * (128 / kV);                     // bits: 16 .. 112
  const u64 lo = h[0], hi = h[1];
  h[0] = by >= 64 ? hi >> (by - 64) : lo >> by | hi << (64 - by);
  h[1] = by >= 64 ? 0 : hi >> by;
  v = __builtin_bit_cast(vec_t, h);
}
template <bool kNt>
DISC_DEV void give(T* p, vec_t v, int n) {
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

// What `lanes` neighbouring threads have, brought together, the same in all of them: a power of two of up to 64, or (kBlock) the
// whole block through LDS.
DISC_DEV double exchanged(double x, int s) { return shuffled(x, s); }
DISC_DEV u32 exchanged(u32 x, int s) { return (u32)__shfl_xor((int)x, s); }
template <bool kBlock, class X, class F>
DISC_DEV X over_lanes(X x, int lanes, F f) {
  for (int s = 1; s < (kBlock ? 64 : lanes); s *= 2) x = f(x, exchanged(x, s));
  return x;
}
template <class X, class F>
DISC_DEV X over_waves(const X* kept, F f) {
  X x = kept[0];
  for (int w = 1; w < (int)blockDim.x / 64; ++w) x = f(x, kept[w]);
  return x;
}
struct Plus {
  DISC_DEV double operator()(double a, double b) const { return a + b; }
};
struct Most {
  DISC_DEV u32 operator()(u32 a, u32 b) const { return max(a, b); }
  DISC_DEV double operator()(double a, double b) const { return a > b ? a : b; }
};

struct NormArgs {
  const T *x, *residual, *weight;
  T* total;
  u8* codes;
  float* scales;
  i64 x_row, residual_row, total_row, codes_row, rows;
  int width, lanes;         // lanes: threads of a row
  float offset;
  double eps;
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

// kLean: the weight is read again where it is used (its registers are needed for the widest rows).
template <bool kNt, bool kBlock, int kN, bool kLean>
DISC_DEV void norm_body(const NormArgs& A) {
  __shared__ double sums[kMostWaves], most64[kMostWaves];
  __shared__ u32 most[kMostWaves];
  const int lanes = kBlock ? (int)blockDim.x : A.lanes, lane = (int)threadIdx.x % lanes;
  const i64 row = kBlock ? (i64)blockIdx.x : (i64)blockIdx.x * ((int)blockDim.x / lanes) + (int)threadIdx.x / lanes;
  if (row >= A.rows) return;                                // (not of a whole block: no barrier follows)
  vec_t x[kN], r[kN], v[kN];
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const int c = (i * lanes + lane) * kV, n = A.width - c;
    x[i] = r[i] = v[i] = vec_t{};
    if (n <= 0) continue;
    x[i] = take<kNt>(A.x + row * A.x_row + c, n, A.width);
    if (A.residual) r[i] = take<kNt>(A.residual + row * A.residual_row + c, n, A.width);
    v[i] = take<false>(A.weight + c, n, A.width);
  }
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const int n = A.width - (i * lanes + lane) * kV;
    settle(x[i], n, A.width);
    settle(r[i], n, A.width);
    settle(v[i], n, A.width);
  }
  float s[kN][kV];
  double squares = 0;
  u32 a = 0;
  const auto weight = [&](int i, int e) { return (float)v[i][e] + A.offset; };   // (behind a row's end s is 0)
  const auto weights_again = [&](int i) {
    const int c = (i * lanes + lane) * kV;
    if (!kLean || c >= A.width) return;
    v[i] = take<false>(A.weight + c, A.width - c, A.width);
    settle(v[i], A.width - c, A.width);
  };
#pragma unroll
  for (int i = 0; i < kN; ++i)
#pragma unroll
    for (int e = 0; e < kV; ++e) {
      s[i][e] = (float)x[i][e] + (float)r[i][e];
      squares += (double)s[i][e] * (double)s[i][e];
      a = max(a, magnitude(s[i][e] * weight(i, e)));
    }
  if (A.total) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int c = (i * lanes + lane) * kV;
      vec_t t;
#pragma unroll
      for (int e = 0; e < kV; ++e) t[e] = (T)s[i][e];
      if (c < A.width) give<kNt>(A.total + row * A.total_row + c, t, A.width - c);
    }
  }
  squares = over_lanes<kBlock>(squares, lanes, Plus());
  a = over_lanes<kBlock>(a, lanes, Most());
  if (kBlock) {
    if (threadIdx.x % 64 == 0) {
      sums[threadIdx.x / 64] = squares;
      most[threadIdx.x / 64] = a;
    }
    __syncthreads();
    a = over_waves(most, Most());
    if (lane == 0) squares = over_waves(sums, Plus());
  }
  // Where a product leaves what 32 bits hold well -- above their range, or so small that Q / a would be infinite -- they
  // are formed in 64.
  float largest = __builtin_bit_cast(float, a);
  const bool wide = !(largest >= 0x1p-100f && largest < __builtin_inff());   // (the same for the whole row)
  double largest64 = (double)largest;
  if (wide) {
    double m = 0;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      weights_again(i);
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        const double y = __builtin_fabs((double)s[i][e] * (double)weight(i, e));
        m = !(y <= m) ? y : m;                              // (a NaN replaces whatever was there, and becomes an infinity)
        if (!(m < __builtin_inf())) m = __builtin_inf();
      }
    }
    m = over_lanes<kBlock>(m, lanes, Most());
    if (kBlock) {
      if (threadIdx.x % 64 == 0) most64[threadIdx.x / 64] = m;
      __syncthreads();
      m = over_waves(most64, Most());
    }
    largest64 = m;
  }
  // The scale is NaN where the row holds an infinity or a NaN: the largest is, or (an infinity times a weight of 0) the squares are.
  const bool fine = largest64 < __builtin_inf();
  if (lane == 0) {
    const double root = 1.0 / sqrt(squares / (double)A.width + A.eps);
    const float scale = (float)(largest64 > 0 ? largest64 * root / (double)kMost : 0.0);
    A.scales[row] = fine ? scale : __builtin_nanf("");
  }
  const float inverse = kMost / largest;
  const double inverse64 = fine && largest64 > 0 ? (double)kMost / largest64 : 0.0;
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const int c = (i * lanes + lane) * kV;
    const int n = A.width - c;
    if (n <= 0) break;
    weights_again(i);
    float y[kV];
#pragma unroll
    for (int e = 0; e < kV; ++e) y[e] = s[i][e] * weight(i, e) * inverse;
    if (wide) {
#pragma unroll
      for (int e = 0; e < kV; ++e) y[e] = fine ? (float)((double)s[i][e] * (double)weight(i, e) * inverse64) : 0.f;
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
// in registers; the blocks' parts, a row of the workspace each, are summed by a second launch in a fixed order.
// Bound by memory and by the exchange between a row's reads and its writes, of which only as many blocks hide as the registers leave room
// for: 16384 x 4096 bf16 with dtotal 107 us, 5.0 TB/s, and the parts' sum 5.9; 500 x 1280 fp32 6.4 and 3.9.
struct NormBackwardArgs {
  const T *total, *weight, *dy, *dtotal;
  T* dx;
  float *dweight, *part;
  i64 total_row, dy_row, dtotal_row, dx_row, rows;
  int width, lanes, parts, groups;   // parts: blocks; groups: of threads that have a row, of all blocks
  float offset;
  double eps;
};

// kLean: weight and dtotal are read again where they are used (their registers are needed for wide rows).
template <bool kNt, bool kBlock, int kN, bool kLean>
DISC_DEV void norm_backward_body(const NormBackwardArgs& A) {
  __shared__ double sums[2][kMostWaves], alongs[2][kMostWaves];
  const int lanes = kBlock ? (int)blockDim.x : A.lanes, lane = (int)threadIdx.x % lanes;
  const int mine = kBlock ? (int)blockIdx.x : (int)blockIdx.x * ((int)blockDim.x / lanes) + (int)threadIdx.x / lanes;
  float dw[kN][kV] = {};
  int turn = 0;
  for (i64 row = mine; row < A.rows; row += A.groups, turn ^= 1) {
    vec_t h[kN], d[kN], v[kN], t[kLean ? 1 : kN];
    double squares = 0, along = 0;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int c = (i * lanes + lane) * kV;
      const int n = A.width - c;
      h[i] = d[i] = v[i] = vec_t{};
      if (!kLean) t[i] = vec_t{};
      if (n <= 0) continue;
      h[i] = take<kNt>(A.total + row * A.total_row + c, n, A.width);
      d[i] = take<kNt>(A.dy + row * A.dy_row + c, n, A.width);
      v[i] = take<false>(A.weight + c, n, A.width);
      if (!kLean && A.dtotal) t[i] = take<kNt>(A.dtotal + row * A.dtotal_row + c, n, A.width);
    }
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int n = A.width - (i * lanes + lane) * kV;
      settle(h[i], n, A.width);
      settle(d[i], n, A.width);
      settle(v[i], n, A.width);
      if (!kLean) settle(t[i], n, A.width);
    }
#pragma unroll
    for (int i = 0; i < kN; ++i)
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        const double x = (double)(float)h[i][e];
        squares += x * x;
        along += x * (double)((float)d[i][e]) * (double)((float)v[i][e] + A.offset);
      }
    squares = over_lanes<kBlock>(squares, lanes, Plus());
    along = over_lanes<kBlock>(along, lanes, Plus());
    if (kBlock) {                                           // (two sets in turn: the next row's are written while some read these)
      if (threadIdx.x % 64 == 0) {
        sums[turn][threadIdx.x / 64] = squares;
        alongs[turn][threadIdx.x / 64] = along;
      }
      __syncthreads();
      squares = over_waves(sums[turn], Plus());
      along = over_waves(alongs[turn], Plus());
    }
    const double root = 1.0 / sqrt(squares / (double)A.width + A.eps);
    const float r = (float)root, k = (float)(root * along / (double)A.width);
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int c = (i * lanes + lane) * kV;
      if (c >= A.width) break;
      vec_t y, last = {};
      if (kLean) {
        v[i] = take<false>(A.weight + c, A.width - c, A.width);
        if (A.dtotal) last = take<kNt>(A.dtotal + row * A.dtotal_row + c, A.width - c, A.width);
        settle(v[i], A.width - c, A.width);
        settle(last, A.width - c, A.width);
      } else {
        last = t[i];
      }
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        const float u = (float)h[i][e] * r, dy = (float)d[i][e], g = dy * ((float)v[i][e] + A.offset);
        dw[i][e] += dy * u;
        y[e] = (T)(r * (g - u * k) + (float)last[e]);
      }
      give<kNt>(A.dx + row * A.dx_row + c, y, A.width - c);
    }
  }
  if (!kBlock) {                                            // the groups of a block, one after the other
    __shared__ float parts[kBlock ? 1 : 256 * kN * kV];
    const int count = (int)blockDim.x / lanes, span = kN * lanes * kV, group = (int)threadIdx.x / lanes;
#pragma unroll
    for (int i = 0; i < kN; ++i)
#pragma unroll
      for (int e = 0; e < kV; ++e) parts[group * span + (i * lanes + lane) * kV + e] = dw[i][e];
    __syncthreads();
    for (int c = (int)threadIdx.x; c < A.width; c += 256) {
      float sum = 0;
      for (int g = 0; g < count; ++g) sum += parts[g * span + c];
      A.part[(i64)blockIdx.x * A.width + c] = sum;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const int c = (i * lanes + lane) * kV;
#pragma unroll
    for (int e = 0; e < kV; ++e)
      if (c + e < A.width) A.part[(i64)blockIdx.x * A.width + c + e] = dw[i][e];
  }
}

// accesses of a thread: a part of a wavefront has a row (_s), 256 threads, or the whole block of up to 1024 (_b)
#define DISC_NORM_KERNEL(NAME, THREADS, NT, BLOCK, N) \
  extern "C" __global__ void __launch_bounds__(THREADS) disc_norm##NAME(NormArgs A) { norm_body<NT, BLOCK, N, (THREADS > 512 && N > 1)>(A); }
#define DISC_NORM_BACKWARD_KERNEL(NAME, THREADS, NT, BLOCK, N) \
  extern "C" __global__ void __launch_bounds__(THREADS) disc_norm_backward##NAME(NormBackwardArgs A) { norm_backward_body<NT, BLOCK, N, (THREADS > 256)>(A); }
DISC_NORM_KERNEL(1_s, 256, false, false, 1)
DISC_NORM_KERNEL(4_s, 256, false, false, 4)
DISC_NORM_KERNEL(4_s_nt, 256, true, false, 4)
DISC_NORM_KERNEL(4, 512, false, true, 4)
DISC_NORM_KERNEL(4_nt, 512, true, true, 4)
DISC_NORM_KERNEL(1_b, 1024, false, true, 1)
DISC_NORM_KERNEL(4_b, 1024, false, true, 4)
DISC_NORM_BACKWARD_KERNEL(1_s, 256, false, false, 1)
DISC_NORM_BACKWARD_KERNEL(4_s, 256, false, false, 4)
DISC_NORM_BACKWARD_KERNEL(4_s_nt, 256, true, false, 4)
DISC_NORM_BACKWARD_KERNEL(4, 256, false, true, 4)
DISC_NORM_BACKWARD_KERNEL(4_nt, 256, true, true, 4)
DISC_NORM_BACKWARD_KERNEL(2_b, 1024, true, true, 2)
DISC_NORM_BACKWARD_KERNEL(4_b, 1024, true, true, 4)

// dweight: a block has 16 columns, 64 threads each of every 64th part.
extern "C" __global__ void __launch_bounds__(1024) disc_norm_join_k(NormBackwardArgs A) {
  __shared__ float kept[16][16];
  const int c = (int)blockIdx.x * 16 + (int)threadIdx.x % 16;
  float sum = 0;
  if (c < A.width) {
    int p = (int)threadIdx.x / 16;
    for (; p + 192 < A.parts; p += 256) {
      float x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) x[u] = A.part[(i64)(p + 64 * u) * A.width + c];
      sum += (x[0] + x[1]) + (x[2] + x[3]);
    }
    for (; p < A.parts; p += 64) sum += A.part[(i64)p * A.width + c];
  }
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  if (threadIdx.x % 64 < 16) kept[threadIdx.x / 64][threadIdx.x % 16] = sum;
  __syncthreads();
  if (threadIdx.x < 16 && c < A.width) {
    sum = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) sum += kept[w][threadIdx.x];
    A.dweight[c] = sum;
  }
}
#endif  // DISC_NORM

#ifdef DISC_LINEAR4
// =================================================================================================
// y[m, n] = r[m] sum_k x[m, k] s[n, k / G] (c[n, k] - z[n, k / G]) + bias[n] with codes c of 4 bits.
// A group's products are summed with the codes less their zero point, c - z: whole numbers of at most eight bits, which both 16-bit types
// hold, so that an element whose code is its zero point adds nothing, however large x is.  (Codes as they are, with the zero point taken off
// by the group's sum of x, cost half as many instructions and round relative to sum |x| (c + z).)  i8 sums are whole numbers, exact
// in that form too, with the sum of x from a product with ones:  sum x (c - z) = sum x c - z sum x.
// The groups' sums, in 32 bits, are multiplied by s and added up in 32 bits.
// Bound by the weights' bytes where there are few rows, and with more by what a CU's memory pipe takes to bring x to the lanes: a load
// of 16 bytes a lane costs it the same whether the lanes' addresses differ or not.  So x of up to 4 rows is loaded in whole wavefronts
// and turned into place (linear_body), and of more rows goes through LDS, where a block's 16 .. 128 columns share it (linear_wide_body).
// Unpacking is 17 instructions for eight codes of bf16 and shows where a lane has few rows to use them for (with one in their place,
// 1 x 8192 x 131072 takes 121 us, not 133, 1 x 4096 x 28672 17, not 20, and 64 x 4096 x 28672 31, not 33).
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

// (d & mask) | bits in one instruction: one of two constants has to be in a vector register
DISC_DEV u32 with_bits(u32 d, u32 mask, u32 bits) {
  asm("" : "+v"(bits));
  return (d & mask) | bits;
}
// Eight codes less their zero point as an operand, in the order 0 4 1 5 2 6 3 7: 1024 + c and 1024 + 16 c in half precision by setting the
// exponent's bits, from which one multiply-add takes the rest, exactly (f16: two numbers at once; bf16: twice the difference, whose eight
// bits are in the upper half of its 32).
struct Zero {
  f16x2 one, sixteen;     // 1024 + z and 64 + z
  float one32, sixteen32; // -2 (1024 + z) and -2 (64 + z)
  DISC_DEV explicit Zero(u32 z) {
    if (kKind == 0) {
      one32 = (float)z * -2.f - 2048.f;
      sixteen32 = (float)z * -2.f - 128.f;
    } else {
      const u32 bits = (z | z << 16) | 0x64006400u;
      one = __builtin_bit_cast(f16x2, bits);
      sixteen = one - f16x2{(_Float16)960.f, (_Float16)960.f};
    }
  }
};
DISC_DEV u32x4 widen(u32 d, const Zero& z) {
  const u32 e = d >> 8;
  const u32x4 raw = {with_bits(d, 0x000f000fu, 0x64006400u), with_bits(d, 0x00f000f0u, 0x64006400u), with_bits(e, 0x000f000fu, 0x64006400u),
                     with_bits(e, 0x00f000f0u, 0x64006400u)};
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const u32 pair = raw[i];                                // (a bit cast of a vector's element itself takes its first one)
    const f16x2 h = __builtin_bit_cast(f16x2, pair);
    if (kKind == 0) {
      const float by = i & 1 ? 0.125f : 2.f, less = i & 1 ? z.sixteen32 : z.one32;
      const float a = __builtin_fmaf((float)h[0], by, less), b = __builtin_fmaf((float)h[1], by, less);
      r[i] = __builtin_amdgcn_perm(__builtin_bit_cast(u32, b), __builtin_bit_cast(u32, a), 0x07060302u);
    } else {
      const f16x2 w = i & 1 ? h * f16x2{(_Float16)0.0625f, (_Float16)0.0625f} - z.sixteen : h - z.one;
      r[i] = __builtin_bit_cast(u32, w);
    }
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

// `n` 16-bit numbers or bytes at any address, as words
template <int kBytes>
struct Words {
  u32 w[(kBytes + 3) / 4];
  DISC_DEV void take(const u8* p) {
    if constexpr (kBytes == 1) w[0] = *p;
    if constexpr (kBytes == 2) w[0] = *(const u16_u*)p;
    if constexpr (kBytes == 4) w[0] = *(const u32_u*)p;
    if constexpr (kBytes == 8) {
      const u32x2 v = *(const u32x2_u*)p;
      w[0] = v[0], w[1] = v[1];
    }
    if constexpr (kBytes >= 16)
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i) {
        const u32x4 v = *(const u32x4_u*)(p + 16 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[4 * i + e] = v[e];
      }
  }
};

// What a lane has of kRun neighbouring blocks of 128 elements: 32 neighbouring codes of a row and block of kN tiles of 16 rows of
// weights, with their groups' scales and zero points (loaded for the run at once: a load of 2 bytes from each of 16 rows costs as much
// as one of 16 bytes; 28672 rows of 4096, one of x: 20.4 us with runs of one block, 18.7 of two).
constexpr int kXs = kKind == 2 ? 2 : 4;                     // operands of a block: 16 bytes a lane (8 of e4m3 in memory)
template <int kN, int kRun>
struct Weights {
  u32x4 w[kRun][kN];
  Words<2 * kGroups * kRun> scale[kN];
  Words<kGroups * kRun> zero[kN];
};

struct Lane {
  const u8 *w, *s, *z;     // the team's first row of weights, of scales, of zero points
  u32 w_row[4], s_row[4];  // from there to its row of each tile: bytes of codes, groups
  int c, q, k, groups;
};

// kWhole: all of the blocks is there; else one block is taken, the last, which may have 32, 64 or 96 elements.
template <bool kWhole, int kN, int kRun>
DISC_DEV void take_weights(const Lane& L, int b, Weights<kN, kRun>& B) {
  static_assert(kWhole || kRun == 1, "");
  const int q = L.q;
#pragma unroll
  for (int r = 0; r < kRun; ++r)
#pragma unroll
    for (int t = 0; t < kN; ++t) {
      B.w[r][t] = u32x4{0, 0, 0, 0};
      if (kWhole || b * kBlockK + q * 32 < L.k) B.w[r][t] = *(const u32x4*)(L.w + (L.w_row[t] + (u32)((b + r) * (kBlockK / 2) + q * 16)));
    }
#pragma unroll
  for (int t = 0; t < kN; ++t) {
    const u8* s = L.s + 2 * (L.s_row[t] + (u32)(b * kGroups));
    const u8* z = L.z + (L.s_row[t] + (u32)(b * kGroups));
    if (kWhole) {
      B.scale[t].take(s);
      if (DISC_ZEROS) B.zero[t].take(z);
    } else {
      B.zero[t].w[0] = 0;
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        const int at = min(g, L.groups - 1 - b * kGroups);
        const u32 v = *(const u16*)(s + 2 * at);
        B.scale[t].w[g / 2] = g % 2 ? B.scale[t].w[g / 2] | v << 16 : v;
        if (DISC_ZEROS) B.zero[t].w[0] |= (u32)z[at] << (8 * g);
      }
    }
  }
}

// bf16 rows times 2^-32 (see finish)
DISC_DEV u32x4 lowered(u32x4 v) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const u32 d = v[i];
    const float lo = __builtin_bit_cast(float, d << 16) * 0x1p-32f, hi = __builtin_bit_cast(float, d & 0xffff0000u) * 0x1p-32f;
    const __bf16 a = (__bf16)lo, b = (__bf16)hi;
    r[i] = (u32)__builtin_bit_cast(u16, a) | (u32)__builtin_bit_cast(u16, b) << 16;
  }
  return r;
}

struct Yes {
  static constexpr bool value = true;
};
struct No {
  static constexpr bool value = false;
};
template <int K>
struct Sum {
  typedef f32x4 type;
};
template <>
struct Sum<2> {
  typedef i32x4 type;
};
// acc += products of the elements of one group: operands of x times w(j), [16 rows][8]
template <class F, class A>
DISC_DEV A multiply(const u32x4* x, F w, int j0, A acc) {
#pragma unroll
  for (int j = j0; j < j0 + 4 / kGroups; ++j) {
    if constexpr (kKind == 2 && kG > 32) {
      if (j % 2) continue;
      const u32x4 b = {w(j)[0], w(j)[1], w(j + 1)[0], w(j + 1)[1]};
      acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, x[j / 2]), __builtin_bit_cast(i32x4, b), acc, 0, 0, 0);
    } else if constexpr (kKind == 2) {
      acc = __builtin_amdgcn_mfma_i32_16x16x32_i8((i8x8)((u64)x[j / 2][j % 2 * 2 + 1] << 32 | x[j / 2][j % 2 * 2]), (i8x8)((u64)w(j)[1] << 32 | w(j)[0]), acc, 0, 0, 0);
    } else if constexpr (kKind == 1) {
      acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x[j]), __builtin_bit_cast(f16x8, w(j)), acc, 0, 0, 0);
    } else {
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x[j]), __builtin_bit_cast(bf16x8, w(j)), acc, 0, 0, 0);
    }
  }
  return acc;
}

// 16 bytes of x for a product (8 of e4m3; of i8 for two of groups of 32, whose elements are 32 apart).  `here`, `too`: whether they are
// in the row.
DISC_DEV u32x4 load_x(const u8* p, bool here, bool too) {
  u32x4 v = {0, 0, 0, 0};
  if (kRowSize == 2 || (kKind == 2 && kG > 32)) {
    if (here) v = *(const u32x4_u*)p;
  } else {
    if (here) {
      const u32x2 h = *(const u32x2_u*)p;
      v[0] = h[0], v[1] = h[1];
    }
    if (kKind == 2 && too) {
      const u32x2 h = *(const u32x2_u*)(p + 32);
      v[2] = h[0], v[3] = h[1];
    }
  }
  return v;
}
// What was loaded of x as operands: in the order of the codes, e4m3 in half precision.
DISC_DEV u32x4 operand(u32x4 v, bool down) {
  if (kKind == 2)
    return u32x4{__builtin_amdgcn_perm(v[1], v[0], 0x06040200u), __builtin_amdgcn_perm(v[1], v[0], 0x07050301u), __builtin_amdgcn_perm(v[3], v[2], 0x06040200u),
                 __builtin_amdgcn_perm(v[3], v[2], 0x07050301u)};
  if (kRowSize == 1) return reorder8(u32x2{v[0], v[1]});
  return reorder(kKind == 0 && down ? lowered(v) : v);
}
// total += a block's products: codes w of each tile of weights with the scales and zero points from number `at` on, x(t, i) the operands
template <int kM, int kN, class X, class S, class Z>
DISC_DEV void add_products(const u32x4 (&codes)[kN], const S* scale, const Z* zero, int at0, X x, float lower, f32x4 (&total)[kM][kN]) {
  constexpr int kEach = 4 / kGroups;                        // dwords of codes of a group
  typedef typename Sum<kKind>::type acc_t;
  const auto zero_of = [&](int n, int at) { return DISC_ZEROS ? (zero[n].w[at / 4] >> (8 * (at % 4))) & 0xffu : 8u; };
  u32x4 w[kN][4];
#pragma unroll
  for (int n = 0; n < kN; ++n) {
    const u32x4 d = arrange(codes[n]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const u32 c = d[j];
      if (kKind == 2) {
        w[n][j][0] = c & 0x0f0f0f0fu;
        w[n][j][1] = (c >> 4) & 0x0f0f0f0fu;
      } else {
        w[n][j] = widen(c, Zero(zero_of(n, at0 + j / kEach)));
      }
    }
  }
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    float s[kN];
    int z[kN];
#pragma unroll
    for (int n = 0; n < kN; ++n) {
      const int at = at0 + g;
      const u32 pair = scale[n].w[at / 2];
      const u16 bits = (u16)(at % 2 ? pair >> 16 : pair);
      s[n] = (float)__builtin_bit_cast(T, bits) * (kKind == 0 ? 0.5f * lower : lower);
      z[n] = (int)zero_of(n, at);
    }
#pragma unroll
    for (int t = 0; t < kM; ++t) {
      constexpr int kUnits = kKind == 2 && kGroups == 4 ? 1 : kXs / kGroups;   // operands of a group (i8 of groups of 32: half a one)
      const int first = g * kXs / kGroups;
      u32x4 v[kUnits];
#pragma unroll
      for (int i = 0; i < kUnits; ++i) v[i] = x(t, first + i);
      const int j0 = kKind == 2 && kGroups == 4 ? g % 2 : 0;
      // (i8) the sum of the rows' elements over the group, in the results' layout: what the codes' zero points are taken off with
      acc_t sum = {};
      if (kKind == 2) sum = multiply(v, [&](int) { return u32x4{0x01010101u, 0x01010101u, 0x01010101u, 0x01010101u}; }, j0, sum);
#pragma unroll
      for (int n = 0; n < kN; ++n) {
        const acc_t acc = multiply(v, [&](int j) { return w[n][g * kEach + j - j0]; }, j0, acc_t{});
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (kKind == 2) total[t][n][i] += s[n] * (float)(acc[i] - z[n] * sum[i]);
          else total[t][n][i] += s[n] * acc[i];
        }
      }
    }
  }
}

// The lane's rows of a team's tiles of weights, from column col0 on.
template <int kN>
DISC_DEV Lane lane_of(const LinearArgs& A, int col0) {
  Lane L;
  L.c = (int)threadIdx.x % 16;
  L.q = (int)threadIdx.x % 64 / 16;
  const int from = min(col0, A.n - 1);
  L.w = A.weights + (i64)from * (A.k / 2);
  L.s = (const u8*)(A.scales + (i64)from * A.groups);
  L.z = DISC_ZEROS ? A.zeros + (i64)from * A.groups : nullptr;
#pragma unroll
  for (int t = 0; t < kN; ++t) {
    const int n = min(t * 16 + L.c, A.n - 1 - from);        // (rows behind the last: copies of it, not stored)
    L.w_row[t] = (u32)n * (u32)(A.k / 2);
    L.s_row[t] = (u32)n * (u32)A.groups;
  }
  L.k = A.k;
  L.groups = A.groups;
  return L;
}

// A team's sums brought together and written.  Where a result is no finite number, the sums on the way to it may have passed 32 bits:
// false, and the whole block forms it again of scales times 2^-32 and of bf16 rows times 2^-32 (what was finite stays).
template <int kM, int kN, int kSplit, int kTeams>
DISC_DEV bool finish(const LinearArgs& A, const f32x4 (&total)[kM][kN], float* kept, int team, int share, int row0, int col0, bool again) {
  const int lane = (int)threadIdx.x % 64, c = lane % 16, q = lane / 16, wave = team * kSplit + share;
  bool lost = false;
  const auto write = [&](int m, int col, float y) {
    if (m >= A.rows || col >= A.n) return;
    if (DISC_ROWS) y *= A.row_scales[m];
    if (again) y *= 0x1p32f * (kKind == 0 ? 0x1p32f : 1.f);
    if (!again) lost |= !(__builtin_fabsf(y) < __builtin_inff());
    if (A.bias) y += (float)A.bias[col];
    T* to = A.out + (m * A.out_row + col);
    if (!again || !(__builtin_fabsf((float)*to) < __builtin_inff())) *to = (T)y;
  };
  if (kSplit == 1) {
#pragma unroll
    for (int t = 0; t < kM; ++t)
#pragma unroll
      for (int n = 0; n < kN; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) write(row0 + t * 16 + q * 4 + i, col0 + n * 16 + c, total[t][n][i]);
    return again || !__any(lost);                           // (its wavefronts have nothing to do with each other)
  }
#pragma unroll
  for (int t = 0; t < kM; ++t)
#pragma unroll
    for (int n = 0; n < kN; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) kept[(wave * kM * kN + t * kN + n) * 256 + (q * 4 + i) * 16 + c] = total[t][n][i];
  __syncthreads();
  for (int o = share * 64 + lane; o < kM * kN * 256; o += kSplit * 64) {
    float y = 0;
#pragma unroll
    for (int v = 0; v < kSplit; ++v) y += kept[(team * kSplit + v) * kM * kN * 256 + o];
    write(row0 + o / (kN * 256) * 16 + o % 256 / 16, col0 + o / 256 % kN * 16 + o % 16, y);
  }
  return !__syncthreads_or(lost) || again;
}

// ---- few rows ---------------------------------------------------------------------------------------
// A product takes its x from the first kR of each 16 lanes (the others' results are not used).  Where kR is less than 16, a load
// fetches what 16 / kR products take, one behind the other in the 16 lanes, and each is turned to the front when its product is due
// (one row x 4096 x 28672: 22.2 us with a load for each product, 18.5; x 12288 10.5, 8.9).
constexpr int kRun = 2;                                     // blocks of a run
template <int kR>
constexpr int loads_of(int run) {
  return (run * kXs * kR + 15) / 16;
}
template <int kN, int kR, int kBlocks>
struct Run : Weights<kN, kBlocks> {
  u32x4 x[loads_of<kR>(kBlocks)];
};
template <bool kWhole, int kN, int kR, int kBlocks>
DISC_DEV void take_run(const Lane& L, const u8* x, int b, Run<kN, kR, kBlocks>& B) {
  const int q = L.q;
  take_weights<kWhole, kN, kBlocks>(L, b, B);
#pragma unroll
  for (int i = 0; i < loads_of<kR>(kBlocks); ++i) {
    // the operand that this lane loads: the n-th of the run
    const int n = kR == 16 ? i : min(i * (16 / kR) + L.c / kR, kBlocks * kXs - 1), j = kKind == 2 ? n % kXs * 2 : n % kXs;
    const int k = n / kXs * kBlockK + place(j, q);
    const bool here = kWhole || b * kBlockK + k < L.k, too = kWhole || b * kBlockK + k + 32 < L.k;
    B.x[i] = load_x(x + ((i64)b * kBlockK + k) * kRowSize, here, too);
  }
}
// v of the lanes kBy behind, among 16
template <int kBy>
DISC_DEV u32x4 turned(u32x4 v) {
  if constexpr (kBy != 0) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32 d = v[i];
      r[i] = (u32)__builtin_amdgcn_update_dpp(0, (int)d, 0x120 + 16 - kBy, 0xf, 0xf, false);   // row_ror
    }
    return r;
  }
  return v;
}
template <int kR, int kAt, int kCount>
DISC_DEV void operands_of(const u32x4* v, u32x4* x) {
  if constexpr (kCount > 0) {
    x[0] = turned<kAt * kR % 16>(v[kAt * kR / 16]);
    operands_of<kR, kAt + 1, kCount - 1>(v, x + 1);
  }
}
// total += the run's products from block kAt on (x as operands already)
template <int kAt, int kN, int kR, int kBlocks>
DISC_DEV void add_blocks(const Run<kN, kR, kBlocks>& B, float lower, f32x4 (&total)[1][kN]) {
  if constexpr (kAt < kBlocks) {
    u32x4 x[kXs];
    operands_of<kR, kAt * kXs, kXs>(B.x, x);
    add_products<1, kN>(B.w[kAt], B.scale, B.zero, kAt * kGroups, [&](int, int i) { return x[i]; }, lower, total);
    add_blocks<kAt + 1>(B, lower, total);
  }
}
template <int kN, int kR, int kBlocks>
DISC_DEV void add_run(Run<kN, kR, kBlocks>& B, bool down, f32x4 (&total)[1][kN]) {
#pragma unroll
  for (int i = 0; i < loads_of<kR>(kBlocks); ++i) B.x[i] = operand(B.x[i], down);
  add_blocks<0>(B, down ? 0x1p-32f : 1.f, total);
}

// kSplit wavefronts share the elements of a row, in runs of blocks, and add up what they have through LDS: a team.  kTeams of them in
// a block have kN tiles of weights each, and the same tile of x.
template <int kN, int kR, int kSplit, int kTeams>
DISC_DEV void linear_body(const LinearArgs& A) {
  __shared__ float kept[kSplit > 1 ? kTeams * kSplit * kN * 256 : 1];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64), team = wave / kSplit, share = wave % kSplit;
  const int col0 = ((int)blockIdx.x * kTeams + team) * 16 * kN, row0 = (int)blockIdx.y * 16;
  const bool idle = col0 >= A.n;                            // (a team behind the last tile; it reaches the barriers)
  const Lane L = lane_of<kN>(A, col0);
  const u8* x = A.x + (i64)min(row0 + L.c % kR, A.rows - 1) * A.x_row * kRowSize;   // (rows behind the last: a copy, not stored)
  const int runs = A.k / (kBlockK * kRun), count = idle || runs <= share ? 0 : (runs - share + kSplit - 1) / kSplit;
  for (int again = 0;; ++again) {
    f32x4 total[1][kN];
#pragma unroll
    for (int n = 0; n < kN; ++n) total[0][n] = f32x4{0, 0, 0, 0};
    // (behind the wavefront's last run, that again: nothing depends on how many there are, so that loads are waited for one by one)
    if (count > 0) {
      Run<kN, kR, kRun> B;
      take_run<true>(L, x, share * kRun, B);
#pragma unroll 1
      for (int i = 1; i <= count; ++i) {
        add_run(B, again != 0, total);
        take_run<true>(L, x, (share + min(i, count - 1) * kSplit) * kRun, B);
      }
    }
    if (!idle)                                              // the blocks behind the last whole run
#pragma unroll 1
      for (int b = runs * kRun + share; b * kBlockK < A.k; b += kSplit) {
        Run<kN, kR, 1> last;
        take_run<false>(L, x, b, last);
        add_run(last, again != 0, total);
      }
    if (finish<1, kN, kSplit, kTeams>(A, total, kept, team, share, row0, col0, again != 0)) break;
  }
}
// tiles of weights, rows of x, wavefronts of a team, teams
#define DISC_LINEAR_KERNEL(N, R, S, W) \
  extern "C" __global__ void __launch_bounds__(S * W * 64) disc_linear_##N##_##R##_##S##_##W##_k(LinearArgs A) { linear_body<N, R, S, W>(A); }
DISC_LINEAR_KERNEL(1, 1, 1, 8)
DISC_LINEAR_KERNEL(1, 1, 16, 1)
DISC_LINEAR_KERNEL(1, 1, 8, 1)
DISC_LINEAR_KERNEL(2, 1, 8, 1)
DISC_LINEAR_KERNEL(1, 4, 1, 8)
DISC_LINEAR_KERNEL(1, 4, 8, 1)
DISC_LINEAR_KERNEL(1, 16, 8, 1)

// ---- more rows --------------------------------------------------------------------------------------
// kM tiles of 16 rows of x through LDS, in chunks of kSplit * kBlocksEach blocks: one in use, the next one in LDS, the one behind it on
// its way in registers.  An operand of a product is 16 bytes a lane; its 16 rows are turned by a number that differs between the
// operands of a row, so that neither the writes (a row's operands) nor the reads (16 rows of one) meet in a bank.
// (us without LDS, a wavefront's x of 16 rows from memory, and with it: 16 x 4096 x 28672 38.5 / 19.6.  A wavefront's blocks of a chunk, 1 / 2, which
// share a load of scales: 64 x 8192 x 8192 29.7 / 27.6, 32 x 8192 x 28672 51 / 47, 64 x 12288 x 12288 of e4m3 57 / 48; in blocks of 64 x 128, where more of
// x would stay in LDS, 64 x 4096 x 28672 32.3 / 33.4.)  Bound by the weights' way to the wavefronts: a step's
// loads are waited for between two barriers.  (us of 61 x 8192 x 8192 in blocks of 32 x 64 and of 64 x 4096 x 28672 in blocks of 64 x 128, 27 and
// 33: without the loads of weights and scales 14 and 24, without widening codes 26 and 31, without reads of LDS 27 and 32, without products 28 and 36.)
template <int kM, int kN, int kSplit, int kTeams, int kBlocksEach>
DISC_DEV void linear_wide_body(const LinearArgs& A) {
  constexpr int kThreads = kSplit * kTeams * 64, kBlocks = kSplit * kBlocksEach, kRowUnits = 4 * kXs, kUnits = kBlocks * 16 * kM * kRowUnits;
  constexpr int kHold = kUnits / kThreads, kKept = kTeams * kSplit * kM * kN * 64;
  static_assert(kHold * kThreads == kUnits, "");
  __shared__ u32x4 xs[2 * kUnits > kKept ? 2 * kUnits : kKept];
  const int lane = (int)threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64), team = wave / kSplit, share = wave % kSplit;
  const int c = lane % 16, q = lane / 16;
  const int col0 = ((int)blockIdx.x * kTeams + team) * 16 * kN, row0 = (int)blockIdx.y * 16 * kM;
  const Lane L = lane_of<kN>(A, col0);                      // (a team behind the last tile goes along, and writes nothing)
  // the units that this thread brings: number p of a row's in a block, which are operand i of the lanes q
  u32x4 held[kHold];
  const auto unit = [&](int h, int& row, int& block, int& k, int& to) {
    const int u = (int)threadIdx.x + h * kThreads, p = u % kRowUnits;
    row = u / kRowUnits % (16 * kM);
    block = u / (kRowUnits * 16 * kM);
    int i, r;
    if (kKind == 2) {
      i = kG == 128 ? p & 1 : p >> 2;
      r = kG == 128 ? p >> 1 : kG == 64 ? (p >> 1 & 1) | (p & 1) << 1 : p & 3;
    } else {
      i = kG == 128 ? p & 3 : kG == 64 ? p >> 3 << 1 | (p & 1) : p >> 2;
      r = kG == 128 ? p >> 2 : kG == 64 ? (p >> 2 & 1) | (p >> 1 & 1) << 1 : p & 3;
    }
    k = block * kBlockK + place(kKind == 2 ? 2 * i : i, r);
    to = ((block * kM + row / 16) * kXs + i) * 64 + r * 16 + ((row % 16) ^ (i * 4 + r));
  };
  const u8* from[kHold];
#pragma unroll
  for (int h = 0; h < kHold; ++h) {
    int row, block, k, to;
    unit(h, row, block, k, to);
    from[h] = A.x + ((i64)min(row0 + row, A.rows - 1) * A.x_row + k) * kRowSize;   // (rows behind the last: a copy, not stored)
  }
  // Yes: all of the chunk is there
  const auto bring = [&](int chunk, auto whole_chunk) {
#pragma unroll
    for (int h = 0; h < kHold; ++h) {
      int row, block, k, to;
      unit(h, row, block, k, to);
      k += chunk * kBlocks * kBlockK;
      const u8* p = from[h] + (i64)chunk * (kBlocks * kBlockK * kRowSize);
      const bool here = decltype(whole_chunk)::value || k < A.k, too = decltype(whole_chunk)::value || k + 32 < A.k;
      held[h] = load_x(p, here, too);
    }
  };
  const auto keep = [&](int chunk, bool down) {
    if (kKind == 0 && down) {
#pragma unroll
      for (int h = 0; h < kHold; ++h) held[h] = lowered(held[h]);
    }
#pragma unroll
    for (int h = 0; h < kHold; ++h) {
      int row, block, k, to;
      unit(h, row, block, k, to);
      xs[(chunk & 1) * kUnits + to] = operand(held[h], false);
    }
  };
  const int full = A.k / (kBlocks * kBlockK), blocks = (A.k + kBlockK - 1) / kBlockK;
  const auto operands = [&](int chunk, int r) {
    const u32x4* at = xs + (chunk & 1) * kUnits + (share * kBlocksEach + r) * kM * kXs * 64 + q * 16;
    return [=](int t, int i) { return at[(t * kXs + i) * 64 + (c ^ (i * 4 + q))]; };
  };
  for (int again = 0;; ++again) {
    const float lower = again ? 0x1p-32f : 1.f;
    f32x4 total[kM][kN];
#pragma unroll
    for (int t = 0; t < kM; ++t)
#pragma unroll
      for (int n = 0; n < kN; ++n) total[t][n] = f32x4{0, 0, 0, 0};
    if (full > 0) {
      // (nothing depends on which chunk it is, so that loads are waited for one by one; behind the last one, that again)
      Weights<kN, kBlocksEach> B;
      // (... and in the same order before the loop as in it)
      bring(0, Yes());
      keep(0, again != 0);
      bring(min(1, full - 1), Yes());
      take_weights<true, kN, kBlocksEach>(L, share * kBlocksEach, B);
      __syncthreads();
#pragma unroll 1
      for (int chunk = 0; chunk < full; ++chunk) {
        keep(chunk + 1, again != 0);
        bring(min(chunk + 2, full - 1), Yes());
#pragma unroll
        for (int r = 0; r < kBlocksEach; ++r) add_products<kM, kN>(B.w[r], B.scale, B.zero, r * kGroups, operands(chunk, r), lower, total);
        take_weights<true, kN, kBlocksEach>(L, (min(chunk + 1, full - 1) * kSplit + share) * kBlocksEach, B);
        __syncthreads();
      }
    }
    if (full * kBlocks < blocks) {                          // what is left, up to a chunk
      bring(full, No());
      keep(full, again != 0);
      __syncthreads();
#pragma unroll 1
      for (int r = 0; r < kBlocksEach; ++r) {
        const int b = full * kBlocks + share * kBlocksEach + r;
        if (b < blocks) {
          Weights<kN, 1> last;
          take_weights<false, kN, 1>(L, b, last);
          add_products<kM, kN>(last.w[0], last.scale, last.zero, 0, operands(full, r), lower, total);
        }
      }
      __syncthreads();
    }
    if (finish<kM, kN, kSplit, kTeams>(A, total, (float*)xs, team, share, row0, col0, again != 0)) break;
  }
}
// tiles of x, of weights, wavefronts of a team, teams, blocks of a wavefront and chunk
#define DISC_LINEAR_WIDE_KERNEL(M, N, S, W, B) \
  extern "C" __global__ void __launch_bounds__(S * W * 64) disc_linear_wide_##M##_##N##_##S##_##W##_##B##_k(LinearArgs A) { linear_wide_body<M, N, S, W, B>(A); }
DISC_LINEAR_WIDE_KERNEL(1, 2, 2, 4, 2)
DISC_LINEAR_WIDE_KERNEL(1, 1, 8, 1, 2)
DISC_LINEAR_WIDE_KERNEL(1, 1, 4, 2, 2)
DISC_LINEAR_WIDE_KERNEL(1, 1, 2, 4, 4)
DISC_LINEAR_WIDE_KERNEL(1, 1, 2, 8, 4)
DISC_LINEAR_WIDE_KERNEL(2, 1, 8, 1, 1)
DISC_LINEAR_WIDE_KERNEL(2, 1, 4, 2, 1)
DISC_LINEAR_WIDE_KERNEL(2, 2, 4, 2, 2)
DISC_LINEAR_WIDE_KERNEL(2, 2, 2, 4, 2)
DISC_LINEAR_WIDE_KERNEL(4, 1, 2, 4, 2)
DISC_LINEAR_WIDE_KERNEL(4, 1, 2, 8, 1)
#endif  // DISC_LINEAR4

#ifdef DISC_VERIFY
// =================================================================================================
// Drafted tokens x_0 .. x_{n-1} against the target's probabilities p_0 .. p_n: x_i is kept while u_i q_i(x_i) < p_i(x_i).
// The token behind the kept ones is drawn from max(p - q, 0) of the first place that was not kept, or from p_n:
// the first whose running sum passes u times the whole.  Products of two 32-bit numbers and differences are formed, and
// sums kept, in 64 bits, in a fixed order.
// Only the row that the last token comes from is read, once for its chunks' sums by as many blocks as it has chunks, and one chunk again.
// Bound by memory where rows are long (64 x 8 x 131072 fp32: 13 us of 67 MB, and 7 for the second launch; bf16 17 for both), by two chains of trips to memory
// (accepted, place, part, row) where there is little to read (1 x 4 x 32000: 4 and 4 us).
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

DISC_DEV int length_of(const VerifyArgs& A, i64 b) { return A.lengths ? min(max(A.lengths[b], 0), A.drafts) : A.drafts; }

// The drafted tokens of sequence b that are kept, by a wavefront: the same in all of its lanes.
DISC_DEV int kept_of(const VerifyArgs& A, i64 b, int lane) {
  const int n = length_of(A, b);
  for (int first = 0; first < A.drafts; first += 64) {
    const int i = first + lane;
    bool bad = false;
    if (i < A.drafts) {
      // (what does not depend on each other is read before anything is waited for)
      const int x = A.drafted[b * A.drafts + i];
      const float u = A.uniforms[b * (A.drafts + 1) + i];
      bad = true;
      if (x >= 0 && x < A.vocabulary) {
        const double p = (double)(float)A.target[b * A.target_batch + i * A.target_row + x];
        const double q = A.draft ? (double)(float)A.draft[b * A.draft_batch + i * A.draft_row + x] : 1.0;
        bad = !((double)u * q < p);
      }
    }
    const u64 mask = __ballot(bad || i >= n);
    if (mask) return min(first + (int)__builtin_ctzll(mask), n);
  }
  return n;
}

// What the last token's weights are made of.
struct Place {
  const T *p, *q;       // q: null where nothing is taken off
  int removed;          // the token without weight (no draft probabilities: the drafted one); -1
  DISC_DEV Place(const VerifyArgs& A, i64 b, int kept) {
    const int n = length_of(A, b);
    p = A.target + b * A.target_batch + kept * A.target_row;
    q = kept < n && A.draft ? A.draft + b * A.draft_batch + kept * A.draft_row : nullptr;
    removed = kept < n && !A.draft ? A.drafted[b * A.drafts + kept] : -1;
  }
  DISC_DEV bool less() const { return q != nullptr || removed >= 0; }
};

// x of another lane (0 where there is none), by the data-parallel moves of a wavefront
template <int kControl, int kRows>
DISC_DEV double moved(double x) {
  const u64 b = __builtin_bit_cast(u64, x);
  const u32 lo = (u32)__builtin_amdgcn_update_dpp(0, (int)(u32)b, kControl, kRows, 0xf, false);
  const u32 hi = (u32)__builtin_amdgcn_update_dpp(0, (int)(u32)(b >> 32), kControl, kRows, 0xf, false);
  return __builtin_bit_cast(double, ((u64)hi << 32) | lo);
}
// x of one lane, the same number for all of them
DISC_DEV double of_lane(double x, int lane) {
  const u64 b = __builtin_bit_cast(u64, x);
  const u32 lo = (u32)__builtin_amdgcn_readlane((int)(u32)b, lane), hi = (u32)__builtin_amdgcn_readlane((int)(u32)(b >> 32), lane);
  return __builtin_bit_cast(double, ((u64)hi << 32) | lo);
}
// the running sum over a wavefront, this lane's among it (moves of 1, 2, 4, 8 lanes among 16, then of a 16's last and a 32's last)
DISC_DEV double wave_running(double x) {
  x += moved<0x111, 0xf>(x);
  x += moved<0x112, 0xf>(x);
  x += moved<0x114, 0xf>(x);
  x += moved<0x118, 0xf>(x);
  x += moved<0x142, 0xa>(x);
  x += moved<0x143, 0xc>(x);
  return x;
}
DISC_DEV double wave_sum(double x) { return of_lane(wave_running(x), 63); }

// The weights of kV neighbouring tokens from i on (`end`: behind the last): what is left of p beside q, and p.
struct Pair {
  float p[kV], q[kV];
  DISC_DEV void take(const Place& at, i64 i, i64 end) {
    vec_t a = {}, b = {};
    if (i + kV <= end) {
      a = *(const vec_u*)(at.p + i);
      if (at.q) b = *(const vec_u*)(at.q + i);
    } else {
#pragma unroll
      for (int e = 0; e < kV - 1; ++e)
        if (i + e < end) {
          a[e] = at.p[i + e];
          if (at.q) b[e] = at.q[i + e];
        }
    }
#pragma unroll
    for (int e = 0; e < kV; ++e) p[e] = (float)a[e], q[e] = (float)b[e];
  }
  DISC_DEV double all(int e) const { return weight((double)p[e]); }
  DISC_DEV double less(const Place& at, i64 i, int e) const {
    if (i + e == at.removed) return 0;
    return at.q ? weight((double)p[e] - (double)q[e]) : weight((double)p[e]);
  }
};
// Sums of tokens first + kV j, j = begin, begin + step ..., below `end`: added to `less` and `all`.
template <int kAtOnce>
DISC_DEV void sum_tokens(const Place& at, i64 begin, int step, i64 end, double& less, double& all) {
  for (; begin < end; begin += (i64)step * kAtOnce) {
    Pair x[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) x[u].take(at, min(begin + (i64)u * step, end), end);
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        all += x[u].all(e);
        less += x[u].less(at, begin + (i64)u * step, e);
      }
  }
}

// Which of up to 64 ranges, a lane each with its sums, u of the whole falls into, and what is in front of it: by a wavefront.
struct Range {
  int range;              // -1: nothing has any weight
  bool from_less;
  double before, goal;
  DISC_DEV Range(bool takes_less, float uniform, double less, double all) {
    const double upto_less = wave_running(less), upto_all = wave_running(all);
    const double whole_less = of_lane(upto_less, 63);
    from_less = takes_less && whole_less > 0;
    const double own = from_less ? less : all, upto = from_less ? upto_less : upto_all, whole = of_lane(upto, 63), u = (double)uniform;
    goal = (u > 0 ? u : 0.0) * whole;
    const double front = moved<0x138, 0xf>(upto);           // (the lane's before it)
    // (by the lane's own sum: each lane's running sum is added up in another order, so that of a lane without weight can be above the one before)
    const u64 some = __ballot(own > 0), over = __ballot(own > 0 && upto > goal);
    range = over ? (int)__builtin_ctzll(over) : some ? 63 - (int)__builtin_clzll(some) : -1;
    before = of_lane(front, max(range, 0));
  }
};

// The token of `count` tokens, at most 16 a thread, from `first` on at which the running sum, `before` in front of them, passes the
// goal (where rounding leaves none, the last with any weight): written by the thread that has it.
constexpr int kEach = 16, kPairs = kEach / kV;
template <int kWaves>
DISC_DEV void pick(const Place& at, const Range& r, i64 first, int count, double* kept, int* over, int* some, int* to) {
  const int lane = (int)threadIdx.x % 64, wave = (int)threadIdx.x / 64;
  const i64 begin = first + (int)threadIdx.x * kEach, end = first + count;
  Pair x[kPairs];
#pragma unroll
  for (int u = 0; u < kPairs; ++u) x[u].take(at, min(begin + u * kV, end), end);
  const auto weight_of = [&](int e) { return r.from_less ? x[e / kV].less(at, begin + e / kV * kV, e % kV) : x[e / kV].all(e % kV); };
  double sum = 0;
#pragma unroll
  for (int e = 0; e < kEach; ++e) sum += weight_of(e);
  double s = wave_running(sum);
  if (lane == 63) kept[wave] = s;
  __syncthreads();
  double in_front = r.before;
  for (int w = 0; w < wave; ++w) in_front += kept[w];
  s += in_front;
  const u64 has = __ballot(sum > 0), passes = __ballot(sum > 0 && s > r.goal);
  if (lane == 0) {
    over[wave] = passes ? wave * 64 + (int)__builtin_ctzll(passes) : -1;
    some[wave] = has ? wave * 64 + 63 - (int)__builtin_clzll(has) : -1;
  }
  __syncthreads();
  int who = -1;
  for (int w = 0; w < kWaves; ++w)
    if (who < 0) who = over[w];
  if (who < 0)
    for (int w = 0; w < kWaves; ++w) who = max(who, some[w]);
  if ((int)threadIdx.x != who) return;
  s -= sum;
  int token = -1;
  bool done = false;
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const double y = weight_of(e);
    s += y;
    if (y > 0 && !done) {
      token = (int)(begin + e);
      done = s > r.goal;
    }
  }
  *to = token;
}
DISC_DEV void write_tokens(const VerifyArgs& A, i64 b, int kept, bool nothing, int threads) {
  for (int i = (int)threadIdx.x; i <= A.drafts; i += threads)
    if (i != kept || nothing) A.tokens[b * (A.drafts + 1) + i] = i < kept ? A.drafted[b * A.drafts + i] : -1;
}

// A block a chunk of a row: what is kept (each block for itself), and the chunk's sums.
extern "C" __global__ void __launch_bounds__(256) disc_verify_sum_k(VerifyArgs A) {
  __shared__ double kept_sums[2][4];
  const i64 b = blockIdx.x / (u32)A.chunks;
  const int chunk = (int)(blockIdx.x - (u32)b * (u32)A.chunks);
  const int kept = kept_of(A, b, (int)threadIdx.x % 64);    // (each wavefront for itself)
  if (threadIdx.x == 0 && chunk == 0) A.accepted[b] = kept;
  const Place at(A, b, kept);
  const i64 first = (i64)chunk * kChunk;
  double less = 0, all = 0;
  sum_tokens<kChunk / (256 * kV)>(at, first + (int)threadIdx.x * kV, 256 * kV, min((i64)A.vocabulary, first + kChunk), less, all);
  less = wave_sum(less);
  all = wave_sum(all);
  if (threadIdx.x % 64 == 0) {
    kept_sums[0][threadIdx.x / 64] = less;
    kept_sums[1][threadIdx.x / 64] = all;
  }
  __syncthreads();
  if (threadIdx.x < 2) {
    const double* k = kept_sums[threadIdx.x];
    A.part[(b * A.chunks + chunk) * 2 + threadIdx.x] = (k[0] + k[1]) + (k[2] + k[3]);
  }
}

extern "C" __global__ void __launch_bounds__(256) disc_verify_pick_k(VerifyArgs A) {
  __shared__ double kept_sums[4];
  __shared__ int over[4], some[4];
  const i64 b = blockIdx.x;
  const int lane = (int)threadIdx.x % 64;
  const int kept = A.accepted[b];
  const float uniform = A.uniforms[b * (A.drafts + 1) + A.drafts];
  const double* part = A.part + b * A.chunks * 2;
  const Place at(A, b, kept);
  // (each wavefront for itself: first a lane a group of chunks, then the chunks of the group)
  const int each = (A.chunks + 63) / 64;
  double less = 0, all = 0;
  for (int i = lane * each; i < min((lane + 1) * each, A.chunks); ++i) less += part[2 * i], all += part[2 * i + 1];
  Range r(at.less(), uniform, less, all);
  if (r.range >= 0) {
    int chunk = r.range * each;
    if (each > 1) {
      int last = chunk;
      double upto = r.before;                               // of the chunks so far; r.before stays what is in front of the last of them
      for (int i = chunk; i < min(chunk + each, A.chunks); ++i) {
        const double x = part[2 * i + (r.from_less ? 0 : 1)];
        if (!(x > 0)) continue;
        last = i;
        r.before = upto;
        upto += x;
        if (upto > r.goal) break;
      }
      chunk = last;
    }
    pick<4>(at, r, (i64)chunk * kChunk, min(kChunk, A.vocabulary - chunk * kChunk), kept_sums, over, some, A.tokens + b * (A.drafts + 1) + kept);
  }
  write_tokens(A, b, kept, r.range < 0, 256);
}
#endif  // DISC_VERIFY
