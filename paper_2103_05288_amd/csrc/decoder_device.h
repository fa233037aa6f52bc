// Device code of the operators around a decoder's attention: rotary positions, the cache of keys and
// values in pages, attention over it.  Compiled through hipRTC once per registration, with what never
// changes between calls as macros (element types, head size, softmax scale, the rotation's frequencies);
// batch, heads, lengths, page size and strides are arguments.
//
//   DISC_ROTARY:  DISC_T, DISC_D, DISC_R, DISC_INTERLEAVED, DISC_MAGNITUDE, kTurns[DISC_R / 2]
//   DISC_CACHE:   DISC_T_F16 (0: bf16), DISC_STORAGE (0: as the activations, 1: i8, 2: e4m3), DISC_D, DISC_SCALE_LOG2E
#pragma once
typedef unsigned char u8;
typedef unsigned short u16;
typedef unsigned int u32;
typedef long long i64;
typedef unsigned long long u64;
typedef u32 u32x2 __attribute__((ext_vector_type(2)));
typedef u32 u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
#define DISC_DEV __device__ __forceinline__

// wide accesses at any element's address (the operands' strides and pointers are the caller's)
typedef u32x2 u32x2_u __attribute__((aligned(1)));
typedef u32x4 u32x4_u __attribute__((aligned(1)));
// ... and past the caches, where a call moves more than they keep for whoever comes next
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

#ifdef DISC_ROTARY
// =================================================================================================
// Rotary positions.  Pair j of a head's first R elements turns by the angle p f_j of its token's
// position p and is scaled by the magnitude; the gradient is the turn back with the same magnitude.
//   y_a = m (x_a cos - x_b sin),  y_b = m (x_b cos + x_a sin),   (a, b) = (j, j + R/2) or (2j, 2j + 1)
// kTurns[j] = f_j / (pi/2): quarter turns a position.  p kTurns[j] is formed in 64 bits (in 32 the angle
// of position 10^6 would be off by 0.06), reduced to an eighth of a turn each side of a quarter, and only
// then rounded to 32 bits.
// A block has one token: its sines are computed once for all heads and kept in LDS, then the heads' rows stream by.
// Bound by memory traffic (one read, one write); blocks of more tokens share nothing more and leave a longer last
// round (us at 1, 2, 4, 8 tokens a block: 32768 x 40 x 128 bf16 121, 124, 128, 133; 16007 x 24 x 80 fp32 55, 57, 59, 64).
// Past the caches they take 106 us (6.3 TB/s) and 43 us (5.8 TB/s).
// =================================================================================================
constexpr int kMaxTensors = 4;
struct RotaryTensor {
  const DISC_T* x;
  DISC_T* y;
  i64 x_token, x_head, y_token, y_head;   // strides in elements
  int heads;
};
struct RotaryArgs {
  RotaryTensor t[kMaxTensors];
  const void* positions;
  int n, position_bytes, backward, pad;
};

constexpr int kD = DISC_D, kR = DISC_R, kH = kR / 2;

// Elements of one access: 16 bytes, or less where it would not divide what it goes over -- each half of the turning
// elements, or all of them where the pairs are neighbours; and the rest of the head.
constexpr int width_of(int n) {
  int w = 16 / (int)sizeof(DISC_T);
  while (n % w) w /= 2;
  return w;
}
constexpr int kW = width_of(DISC_INTERLEAVED ? kR : kH), kV = width_of(kD - kR);
constexpr int kTurnUnits = (DISC_INTERLEAVED ? kR : kH) / kW, kUnits = kTurnUnits + (kD - kR) / kV;
static_assert(kUnits <= 256, "a head is one pass of a block at most");

typedef DISC_T turn_t __attribute__((ext_vector_type(kW)));
typedef turn_t turn_u __attribute__((aligned(alignof(DISC_T))));
typedef DISC_T rest_t __attribute__((ext_vector_type(kV)));
typedef rest_t rest_u __attribute__((aligned(alignof(DISC_T))));

template <bool kNt>
DISC_DEV void rotary_body(const RotaryArgs& A) {
  __shared__ float cs[kH], sn[kH];
  const i64 t = blockIdx.x;
  for (int j = threadIdx.x; j < kH; j += 256) {
    const double p = A.position_bytes == 8 ? (double)((const i64*)A.positions)[t] : (double)((const int*)A.positions)[t];
    const double turns = p * kTurns[j], quarter = rint(turns);
    float s, c;
    sincospif((float)(turns - quarter) * 0.5f, &s, &c);
    const int q = (int)((i64)quarter & 3);
    const float sq = q & 1 ? c : s, cq = q & 1 ? s : c;      // sin, cos of the angle up to their signs
    const float m = (float)DISC_MAGNITUDE;
    cs[j] = (q == 1 || q == 2 ? -cq : cq) * m;
    sn[j] = ((q & 2) != 0) != (A.backward != 0) ? -sq * m : sq * m;
  }
  __syncthreads();
  for (int k = 0; k < A.n; ++k) {
    const RotaryTensor& X = A.t[k];
    // in place, the rest of a head is there already
    const int units = X.x != X.y ? kUnits : kTurnUnits, rows = 256 / units, u = threadIdx.x % units;
    // blockIdx.y: a share of the heads, for calls of few tokens
    const int h_lo = (int)((i64)X.heads * blockIdx.y / gridDim.y), h_hi = (int)((i64)X.heads * (blockIdx.y + 1) / gridDim.y);
    const DISC_T* xt = X.x + t * X.x_token;
    DISC_T* yt = X.y + t * X.y_token;
    for (int h = h_lo + (int)threadIdx.x / units; h < h_hi && (int)threadIdx.x < rows * units; h += rows) {
      const DISC_T* x = xt + h * X.x_head;
      DISC_T* y = yt + h * X.y_head;
      if (u < kTurnUnits) {
        const int j = u * kW;
        if (DISC_INTERLEAVED) {
          const turn_t v = fetch<kNt>((const turn_u*)(x + j));
          turn_t r;
#pragma unroll
          for (int e = 0; e + 1 < kW; e += 2) {
            const float c = cs[(j + e) / 2], s = sn[(j + e) / 2], p0 = (float)v[e], p1 = (float)v[e + 1];
            r[e] = (DISC_T)(p0 * c - p1 * s);
            r[e + 1] = (DISC_T)(p1 * c + p0 * s);
          }
          put<kNt>((turn_u*)(y + j), (turn_u)r);
        } else {
          const turn_t a = fetch<kNt>((const turn_u*)(x + j)), b = fetch<kNt>((const turn_u*)(x + kH + j));
          turn_t ra, rb;
#pragma unroll
          for (int e = 0; e < kW; ++e) {
            const float c = cs[j + e], s = sn[j + e], p0 = (float)a[e], p1 = (float)b[e];
            ra[e] = (DISC_T)(p0 * c - p1 * s);
            rb[e] = (DISC_T)(p1 * c + p0 * s);
          }
          put<kNt>((turn_u*)(y + j), (turn_u)ra);
          put<kNt>((turn_u*)(y + kH + j), (turn_u)rb);
        }
      } else {
        const int j = kR + (u - kTurnUnits) * kV;
        put<kNt>((rest_u*)(y + j), (rest_u)fetch<kNt>((const rest_u*)(x + j)));
      }
    }
  }
}
extern "C" __global__ void __launch_bounds__(256) disc_rotary_k(RotaryArgs A) { rotary_body<false>(A); }
extern "C" __global__ void __launch_bounds__(256) disc_rotary_nt_k(RotaryArgs A) { rotary_body<true>(A); }
#endif  // DISC_ROTARY

#ifdef DISC_CACHE
// =================================================================================================
// The cache: keys and values in pages [page][kv head][place][D], and where they are quantised a scale
// for every row [page][kv head][place].  A slot is page * page_size + place.
// =================================================================================================
#if DISC_T_F16
typedef _Float16 T;
#else
typedef __bf16 T;
#endif
typedef T Tx2 __attribute__((ext_vector_type(2)));
typedef T Tx8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
constexpr int kD = DISC_D;
constexpr bool kQuantised = DISC_STORAGE != 0;
constexpr int kSize = kQuantised ? 1 : 2;                  // bytes of a stored element
constexpr float kMost = DISC_STORAGE == 1 ? 127.f : 448.f; // largest code

struct RowsArgs {
  const i64* slots;
  T* k;                     // rows of activations (read by the store, written by the load)
  T* v;
  u8* kp;
  u8* vp;
  float* ks;
  float* vs;
  i64 k_token, k_head, v_token, v_head;
  i64 tokens, slots_end;    // slots_end = pages * page_size
  int heads, shift;         // page_size = 1 << shift
};

// First row of a slot in the pages, in rows: (page * heads + head) * page_size + place.
DISC_DEV i64 page_row(i64 slot, int head, int heads, int shift) {
  return ((((slot >> shift) * heads) + head) << shift) + (slot & ((1ll << shift) - 1));
}

constexpr int kLanes = kD <= 16 ? 2 : kD <= 32 ? 4 : kD <= 64 ? 8 : kD <= 128 ? 16 : 32;   // lanes of a row, eight elements each

DISC_DEV float f32_of(u32 pair, int hi) {
  return (float)__builtin_bit_cast(Tx2, pair)[hi];
}

// Eight values to eight codes.  x * up * inverse is rounded once to 32 bits (`up` is a power of two) and once to the code
// (half to even).
DISC_DEV u32x2 encode(const u32x4& x, float up, float inverse) {
  u32x2 c;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = __builtin_amdgcn_fmed3f(f32_of(x[w * 2 + e / 2], e & 1) * up * inverse, -kMost, kMost);
#if DISC_STORAGE == 2
    int p = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    c[w] = (u32)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], p, true);
#else
    u32 p = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) p |= ((u32)(int)__builtin_rintf(y[e]) & 0xffu) << (8 * e);
    c[w] = p;
#endif
  }
  return c;
}

// Stores rows of keys and values.  Scale of a row: a / kMost with a its largest magnitude; code of an
// element: round(x * (kMost / a)).  The magnitude is compared as the bits of |x|, so that a NaN counts as
// larger than an infinity: a row that holds either gets the scale NaN and codes of zero, and reads back as
// NaN.  A row of zeros has the scale 0.  kMost / a is no number of 32 bits below kMost / 2^128: bf16 rows of less than 2^-100
// are brought up by 2^100 before (fp16 has none).  Slots outside the pages are left out.
// Keys and values of a (token, head) are one lane group's, so that two loads are in flight a lane.
template <bool kNt>
DISC_DEV void store_body(const RowsArgs& A) {
  const i64 row = ((i64)blockIdx.x * 256 + threadIdx.x) / kLanes;
  const int lane = threadIdx.x % kLanes;
  const i64 t = row / A.heads;
  const int h = (int)(row - t * A.heads);
  if (t >= A.tokens) return;
  const i64 slot = A.slots[t];
  if (slot < 0 || slot >= A.slots_end) return;
  const i64 to = page_row(slot, h, A.heads, A.shift);
  const bool mine = lane * 8 < kD;
  u32x4 x[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
  if (mine) {
    x[0] = fetch<kNt>((const u32x4_u*)(A.k + t * A.k_token + h * A.k_head + lane * 8));
    x[1] = fetch<kNt>((const u32x4_u*)(A.v + t * A.v_token + h * A.v_head + lane * 8));
  }
  if (!kQuantised) {
    if (mine) {
      put<kNt>((u32x4*)(A.kp + (to * kD + lane * 8) * 2), x[0]);
      put<kNt>((u32x4*)(A.vp + (to * kD + lane * 8) * 2), x[1]);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    // (the bits of 16-bit magnitudes order as the magnitudes do, NaN above infinity)
    u32 a = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const u32 lo = x[i][w] & 0x7fffu, hi = (x[i][w] >> 16) & 0x7fffu;
      a = max(a, max(lo, hi));
    }
#pragma unroll
    for (int s = 1; s < kLanes; s *= 2) a = max(a, (u32)__shfl_xor((int)a, s));
    const float m = (float)__builtin_bit_cast(T, (u16)a);
    const bool fine = m < __builtin_inff();
    const float up = !DISC_T_F16 && m < 0x1p-100f ? 0x1p100f : 1.f;
    const float inverse = fine && m > 0.f ? kMost / (m * up) : 0.f;
    u32x2 c = {0, 0};
    if (fine) c = encode(x[i], up, inverse);
    if (mine) put<kNt>((u32x2*)((i ? A.vp : A.kp) + to * kD + lane * 8), c);
    if (lane == 0) (i ? A.vs : A.ks)[to] = fine ? m / kMost : __builtin_nanf("");
  }
}

// Reads rows back: code * scale, rounded once.  A slot outside the pages gives a row of zeros.
template <bool kNt>
DISC_DEV void load_body(const RowsArgs& A) {
  const i64 row = ((i64)blockIdx.x * 256 + threadIdx.x) / kLanes;
  const int lane = threadIdx.x % kLanes;
  const i64 t = row / A.heads;
  const int h = (int)(row - t * A.heads);
  if (t >= A.tokens || lane * 8 >= kD) return;
  const i64 slot = A.slots[t];
  const bool there = slot >= 0 && slot < A.slots_end;
  const i64 from = there ? page_row(slot, h, A.heads, A.shift) : 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    u32x4 y = {0, 0, 0, 0};
    if (there) {
      if (!kQuantised) {
        y = fetch<kNt>((const u32x4*)((i ? A.vp : A.kp) + (from * kD + lane * 8) * 2));
      } else {
        const u32x2 c = fetch<kNt>((const u32x2*)((i ? A.vp : A.kp) + from * kD + lane * 8));
        const float s = (i ? A.vs : A.ks)[from];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          float f[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int at = (w * 2 + e) % 4;
#if DISC_STORAGE == 2
            f[e] = at == 0   ? __builtin_amdgcn_cvt_f32_fp8((int)c[w / 2], 0)
                   : at == 1 ? __builtin_amdgcn_cvt_f32_fp8((int)c[w / 2], 1)
                   : at == 2 ? __builtin_amdgcn_cvt_f32_fp8((int)c[w / 2], 2)
                             : __builtin_amdgcn_cvt_f32_fp8((int)c[w / 2], 3);
#else
            f[e] = (float)(signed char)(c[w / 2] >> (8 * at));
#endif
          }
          const Tx2 p = {(T)(f[0] * s), (T)(f[1] * s)};
          y[w] = __builtin_bit_cast(u32, p);
        }
      }
    }
    T* to = i ? A.v + t * A.v_token + h * A.v_head : A.k + t * A.k_token + h * A.k_head;
    put<kNt>((u32x4_u*)(to + lane * 8), (u32x4_u)y);
  }
}
// Bound by memory traffic, small calls by their launch.  (Past the caches in large calls: 40009 x 8 x 128 bf16 to e4m3 49 -> 47
// us, 65536 x 8 x 128 from i8 89 -> 80.5, both 5.0 TB/s.)
extern "C" __global__ void __launch_bounds__(256) disc_store_k(RowsArgs A) { store_body<false>(A); }
extern "C" __global__ void __launch_bounds__(256) disc_store_nt_k(RowsArgs A) { store_body<true>(A); }
extern "C" __global__ void __launch_bounds__(256) disc_load_k(RowsArgs A) { load_body<false>(A); }
extern "C" __global__ void __launch_bounds__(256) disc_load_nt_k(RowsArgs A) { load_body<true>(A); }

// =================================================================================================
// Attention of one query token a sequence over its pages:
//   o = sum_t p_t v_t / sum_t p_t,   p_t = 2^(c q.k_t - m),   c = softmax scale * log2(e)
// in one pass over the keys and values with a running reference m: the maximum, but for kLag powers of two by which
// the scores may pass it before it moves (and with it what was summed).
//
// Products on the matrix cores, 16 x 16 x 32.  A step is 32 tokens; the 16 columns are the query heads
// that share a kv head.  S^T = K Q^T: row i of tile mt takes the key of token 8 (i / 4) + 4 mt + i % 4, so
// that a lane's results are the scores of eight neighbouring tokens 8 g + 0..7 (g = lane / 16) -- which is
// what the second product O^T = V^T P^T wants as its operand: the probabilities never leave their
// registers.  A lane reads, of those eight tokens, E neighbouring elements of the values; what is row
// d of V^T in the matrix product is then spread over eight registers of the same lane, and byte permutes
// put it together: the values need no LDS either.
//
// 8-bit codes are exact in half precision and in bf16; a key's scale multiplies its score, a value's scale its
// probability.  Those products p * scale, the weights, are taken to half precision relative to a power of two of their own
// row's, which follows the largest of them (neither the largest score nor the largest scale: a token that scores high may
// have a value of zero, and one with a huge value no weight).
// Where the weights would have no more bits than the result they are held as a sum of two 16-bit numbers (hi + lo), so
// that of all but the smallest the only rounding that counts is the result's.  bf16 has the range of 32 bits.  Half
// precision ends at 2^-25, which is 2^-34 of the largest weight over 8-bit rows and 2^-35 of the largest probability over
// fp16 ones: a smaller weight is off by up to that much.
//
// A block is four wavefronts; they take the steps of a stretch of tokens in turn and join in LDS at its end.
// The stretches are cut from the lengths, on the device, so that all blocks have the same share.
//
// Long caches are bound by their reads: 64 sequences of up to 8192 tokens (8 kv heads of 128, i8) 101 us, 5.5 TB/s; two of
// 131072 (bf16) 116 us, 5.7 TB/s.  Short ones by the chain lengths -> page table -> first rows -> end, about 5 us, and by the
// joining launch, 4 to 8 us: one sequence of 300 5.9 us, four of 4000 17.
// =================================================================================================
constexpr int kStep = 32;                     // tokens of a step
constexpr int kMostPages = 1024;              // pages of a stretch that are kept in LDS at a time
constexpr int kDirectPages = 64;              // pages of a sequence that is one chunk
constexpr int kE = kD % 128 == 0 ? 8 : kD % 64 == 0 ? 4 : 8;    // neighbouring elements of a value that a lane reads
constexpr int kNB = (kD + 16 * kE - 1) / (16 * kE);             // such groups of 16 lanes
constexpr int kND = kE * kNB;                                   // 16-row tiles of O^T
constexpr int kKE = 16 / kSize;                                 // elements of a key that a lane reads at once
constexpr int kNK = (kD + 4 * kKE - 1) / (4 * kKE);             // such reads
constexpr int kVW = kE * kSize / 4;                             // registers of one value read
// type of the second product, and whether its probabilities are split
#if DISC_T_F16
constexpr bool kSplit = true;
#else
constexpr bool kSplit = !kQuantised;
#endif

struct AttendArgs {
  const T* q;
  const int* lengths;
  const int* table;
  const u8* kp;
  const u8* vp;
  const float* ks;
  const float* vs;
  const int* prefix_table;
  T* out;
  float* part;              // results of the chunks [part][heads of q of the kv heads][D], as if there were no others
  float* part_m;            // their reference (-infinity where there was no score) and sum, two floats a row
  i64 q_row, q_head, o_row, o_head;
  int batch, heads, kv_heads, group, pages, shift, width, tiles;
  int target;               // blocks a kv head that the sequences' tokens are shared out to
  int parts;                // chunks there can be at most: target + batch
  int direct;               // every sequence is one chunk, whatever its length: chunk b
  int join_ways;            // wavefronts of a row of disc_join_k: 1 or 4
  int prefix_len, prefix_chunk, prefix_parts;
  int prefix_tiles;         // the prefix's blocks of 16 query rows a kv head in disc_attend_k (0: disc_prefix_k has it)
  int prefix_inline;        // a short prefix: every sequence's own block goes through it too, and nothing is joined
};

DISC_DEV int clamp_length(int n, int width, int shift) {
  const i64 most = (i64)width << shift;
  return n < 0 ? 0 : n > most ? (int)most : n;
}

// Number of the wavefront in its block: the same for its lanes, which the compiler has to be told, so that what depends
// on it is a scalar and its branches are no masks.
DISC_DEV int wavefront() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// Sum of the lanes up to this one.
DISC_DEV u32 scan64(u32 x) {
  x += (u32)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false);   // row_shr:1
  x += (u32)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false);
  x += (u32)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false);
  x += (u32)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false);
  x += (u32)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);   // row_bcast:15
  x += (u32)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);   // row_bcast:31
  return x;
}

// How the sequences' tokens are shared out: in units of four steps, the sequences one after the other, every one of
// `target` blocks takes the same number of units (one more or less).  A block so has a stretch of one sequence, or the
// end of one, whole ones and the beginning of another; what block j has of sequence b is chunk j + b, which no two of
// them share.  Every wavefront finds out for itself, from the lengths.
struct Shares {
  u64 each;                 // units of a block; the first `more` blocks have one more
  u32 more;
  DISC_DEV u64 first(u32 j) const { return (u64)j * each + (j < more ? j : more); }
  DISC_DEV u32 block_of(u64 unit) const {
    const u64 edge = (u64)more * (each + 1);
    if (unit < edge) return divide(unit, each + 1);
    return more + divide(unit - edge, each);
  }
  static DISC_DEV u32 divide(u64 a, u64 b) { return (a | b) < 1ull << 32 ? (u32)a / (u32)b : (u32)(a / b); }
};
constexpr int kUnit = 4 * kStep;
DISC_DEV u32 units_of(int n) { return (u32)(n + kUnit - 1) / kUnit; }

// Lengths of the sequences b0 + lane.
DISC_DEV int length_of(const AttendArgs& A, int b0) {
  const int b = b0 + (threadIdx.x & 63);
  return b < A.batch ? clamp_length(A.lengths[b], A.width, A.shift) : 0;
}

DISC_DEV Shares shares_of(const AttendArgs& A, int& n) {      // n: the last 64 lengths that were read
  u64 total = 0;
  for (int b0 = 0; b0 < A.batch; b0 += 64) {
    n = length_of(A, b0);
    total += (u32)__builtin_amdgcn_readlane((int)scan64(units_of(n)), 63);   // (64 x 2^23 at most)
  }
  Shares S;
  S.each = total < 1ull << 32 ? (u32)total / (u32)A.target : total / (u32)A.target;
  S.more = (u32)(total - S.each * (u32)A.target);
  return S;
}

// The stretches of a block, one after the other.
struct Walk {
  u64 lo, hi, before;       // the block's units; units of the sequences before b0
  u64 who;                  // the sequences b0 + 0..63 that it has something of and has not been at
  int b0, n;
  u32 first, units;         // of sequence b0 + lane, from `before` on
  int b, begin, end;        // the stretch: tokens [begin, end) of sequence b
  bool whole;               // it is all of the sequence

  DISC_DEV void start(const AttendArgs& A, u32 block) {
    const Shares S = shares_of(A, n);
    lo = S.first(block);
    hi = S.first(block + 1);
    before = 0;
    b0 = -64;
    who = 0;
    units = 0;
  }
  DISC_DEV bool next(const AttendArgs& A) {
    while (!who) {
      if (b0 >= 0) before += (u32)__builtin_amdgcn_readlane((int)(first + units), 63);
      b0 += 64;
      if (b0 >= A.batch || before >= hi) return false;
      if (A.batch > 64) n = length_of(A, b0);
      units = units_of(n);
      first = scan64(units) - units;
      who = __ballot(units > 0 && before + first < hi && before + first + units > lo);
    }
    const int l = __ffsll((unsigned long long)who) - 1;
    who &= who - 1;
    const u64 f = before + (u32)__builtin_amdgcn_readlane((int)first, l);
    const u32 u = (u32)__builtin_amdgcn_readlane((int)units, l);
    const int len = __builtin_amdgcn_readlane(n, l);
    const u32 from = lo > f ? (u32)(lo - f) : 0, to = hi < f + u ? (u32)(hi - f) : u;
    b = b0 + l;
    begin = (int)(from * kUnit);
    end = to == u ? len : (int)(to * kUnit);
    whole = from == 0 && to == u;
    return true;
  }
};

// The chunks of sequence b: the first, and how many.
DISC_DEV void chunks_of(const AttendArgs& A, int b, int& chunk, int& count) {
  int n = 0;
  const Shares S = shares_of(A, n);
  u64 before = 0;
  for (int b0 = 0;; b0 += 64) {
    if (A.batch > 64) n = length_of(A, b0);
    const u32 incl = scan64(units_of(n));
    if (b < b0 + 64) {
      const u32 u = (u32)__builtin_amdgcn_readlane((int)units_of(n), b - b0);
      const u64 f = before + (u32)__builtin_amdgcn_readlane((int)incl, b - b0) - u;
      chunk = count = 0;
      if (u) {
        const u32 j = S.block_of(f);
        chunk = (int)j + b;
        count = (int)(S.block_of(f + u - 1) - j) + 1;
      }
      return;
    }
    before += (u32)__builtin_amdgcn_readlane((int)incl, 63);
  }
}

// Products: in half precision over codes and fp16, else in bf16.
DISC_DEV f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  if (kQuantised || DISC_T_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
#if !DISC_T_F16
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Tx8, a), __builtin_bit_cast(Tx8, b), c, 0, 0, 0);
#else
  return c;
#endif
}

// Codes as half-precision numbers: kCode times the code.  A signed code plus 128, in the low byte of a half, is that
// many times its smallest number 2^-24; one multiply-add makes it (code + 128) 2^-9 - 128 2^-9, exactly.
constexpr float kCode = DISC_STORAGE == 1 ? 1.f / 512.f : 1.f;
constexpr u32 kBias = DISC_STORAGE == 1 ? 0x80808080u : 0u;    // x ^ kBias: four signed codes plus 128
template <bool kHigh>
DISC_DEV u32 half_of_floats(u32 x) {
#if DISC_STORAGE == 2
  return __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x, 1.f, kHigh));
#else
  return 0;
#endif
}
DISC_DEV u32 half_of_codes(u32 x) {                            // of the low bytes of its halves, the others are 0
  const f16x2 scale = {(_Float16)32768.f, (_Float16)32768.f}, offset = {(_Float16)-0.25f, (_Float16)-0.25f};
  return __builtin_bit_cast(u32, __builtin_elementwise_fma(__builtin_bit_cast(f16x2, x), scale, offset));
}

// Eight neighbouring codes (two registers) of a key.  (In half precision, 72 operations for a step's keys; bf16 queries are
// brought to it once.  As bf16 numbers they take 96: 64 x 8192 i8 of heads of 128, 64 and 80 109, 66 and 96 us, where this
// takes 106, 62 and 91; e4m3 of 128 and 256 100 and 103, here 100 and 105.)
DISC_DEV u32x4 keys_of_codes(u32 a, u32 b) {
  u32x4 r;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const u32 x = (w ? b : a) ^ kBias;
    if (DISC_STORAGE == 2) {
      r[2 * w] = half_of_floats<false>(x);
      r[2 * w + 1] = half_of_floats<true>(x);
    } else {
      r[2 * w] = half_of_codes(__builtin_amdgcn_perm(x, x, 0x0c010c00u));
      r[2 * w + 1] = half_of_codes(__builtin_amdgcn_perm(x, x, 0x0c030c02u));
    }
  }
  return r;
}

template <int RT>
struct Rows {                                // RT x 16 query rows of a wavefront
  u32x4 q[RT][kNK * (kKE / 8)];
  f32x4 o[RT][kND];
  float use[RT], l[RT];                      // what the scores are taken relative to, this lane's share of the sum
  float lim[RT];                             // how far a score may pass it: kLag, or -infinity as long as there was none
  float grow[RT], room[RT];                  // power of two on the weights (0: none yet), log2 of what they may be without it
  float factor;                              // on the scores: softmax scale, log2(e), and what q and the keys were scaled by
  int row[RT];                               // ... without that, where `uneven`: rows have powers of two of their own, these
  bool uneven;
};
struct Keys {
  u32x4 k[2][kNK];
};
struct Values {
  u32 v[8][kNB * kVW];
};

// `rows`: of the stretch's pages in LDS, from the page of its first token (number `base`) on, the first row of this kv
// head, or kNoPage.  Rows are counted in 32 bits (the host checks that there are no more); their addresses have 64.
constexpr u32 kNoPage = 0xffffffffu;
DISC_DEV u32 row_of(const AttendArgs& A, const u32* rows, int base, int t, bool& there) {
  const u32 first = rows[(t >> A.shift) - base];
  there = first != kNoPage;
  return (there ? first : 0) + (u32)(t & ((1 << A.shift) - 1));
}

template <bool kNt>
DISC_DEV void read_keys(const u8* p, int g, Keys& K) {
#pragma unroll
  for (int mt = 0; mt < 2; ++mt)
#pragma unroll
    for (int i = 0; i < kNK; ++i) {
      if ((i + 1) * 64 <= kD * kSize || i * 64 + g * 16 < kD * kSize) K.k[mt][i] = fetch<kNt>((const u32x4*)(p + mt * 4 * (kD * kSize) + i * 64));
      else K.k[mt][i] = (u32x4){0, 0, 0, 0};
    }
}

template <bool kNt>
DISC_DEV void load_keys(const AttendArgs& A, const u32* rows, int base, int last, int t0, Keys& K) {
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  bool there;
  const u32 row = row_of(A, rows, base, min(t0 + (m >> 2) * 8, last), there) + (m & 3);
  read_keys<kNt>(A.kp + (u64)row * (kD * kSize) + g * 16, g, K);
}

template <bool kNt>
DISC_DEV void read_values(const u8* first, int c, Values& V) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
#pragma unroll
    for (int n = 0; n < kNB; ++n) {
      const u8* p = first + j * (kD * kSize) + n * 16 * kE * kSize;
      const bool mine = (n + 1) * 16 * kE <= kD || (n * 16 + c) * kE < kD;
      if (kVW == 4) {
        u32x4 x = {0, 0, 0, 0};
        if (mine) x = fetch<kNt>((const u32x4*)p);
#pragma unroll
        for (int w = 0; w < 4; ++w) V.v[j][n * kVW + w % kVW] = x[w];
      } else if (kVW == 2) {
        u32x2 x = {0, 0};
        if (mine) x = fetch<kNt>((const u32x2*)p);
#pragma unroll
        for (int w = 0; w < 2; ++w) V.v[j][n * kVW + w % kVW] = x[w];
      } else {
        V.v[j][n * kVW] = mine ? fetch<kNt>((const u32*)p) : 0u;
      }
    }
  }
}

template <bool kNt>
DISC_DEV bool load_values(const AttendArgs& A, const u32* rows, int base, int last, int t0, Values& V) {
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  bool there;
  const u32 row = row_of(A, rows, base, min(t0 + g * 8, last), there);
  read_values<kNt>(A.vp + (u64)row * (kD * kSize) + c * kE * kSize, c, V);
  return there;
}

// The scales of a step: lanes 0..31 those of its keys, 32..63 those of its values.
DISC_DEV float load_scale(const AttendArgs& A, const u32* rows, int base, int last, int t0) {
  const int lane = threadIdx.x & 63;
  bool there;
  return (lane < 32 ? A.ks : A.vs)[row_of(A, rows, base, min(t0 + (lane & 31), last + 7), there)];
}

// Row d of V^T: element i of the lane's eight tokens, as the second product's operand.
DISC_DEV u32x4 column_of(const Values& V, int n, int i) {
  u32x4 r;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (!kQuantised) {
      const u32 a = V.v[2 * w][n * kVW + i / 2], b = V.v[2 * w + 1][n * kVW + i / 2];
      r[w] = __builtin_amdgcn_perm(b, a, i & 1 ? 0x07060302u : 0x05040100u);
    } else {
      const u32 a = V.v[2 * w][n * kVW + i / 4] ^ kBias, b = V.v[2 * w + 1][n * kVW + i / 4] ^ kBias;
      const u32 e = i & 3;
      if (DISC_STORAGE == 2) r[w] = half_of_floats<false>(__builtin_amdgcn_perm(b, a, 0x0c0c0400u + 0x0101u * e));
      else r[w] = half_of_codes(__builtin_amdgcn_perm(b, a, 0x0c040c00u + 0x00010001u * e));
    }
  }
  return r;
}

DISC_DEV float max_of_groups(float x) {      // over the four lane groups that share a query row
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

template <int RT>
DISC_DEV void scores(const Rows<RT>& R, const Keys& K, f32x4 (&s)[RT][2]) {
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) s[rt][mt] = (f32x4){0, 0, 0, 0};
#pragma unroll
  for (int mt = 0; mt < 2; ++mt)
#pragma unroll
    for (int i = 0; i < kNK; ++i) {
      if (!kQuantised) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt][mt] = mfma(K.k[mt][i], R.q[rt][i], s[rt][mt]);
      } else {
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          const u32x4 k = keys_of_codes(K.k[mt][i][2 * f], K.k[mt][i][2 * f + 1]);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) s[rt][mt] = mfma(k, R.q[rt][(i * 2 + f) % (kNK * (kKE / 8))], s[rt][mt]);
        }
      }
    }
}

constexpr float kLag = !kQuantised && DISC_T_F16 ? 4.f : 8.f;   // a score may pass the running maximum by this many powers of two
constexpr float kNone = -__builtin_inff();
// The largest probability is 2^kBase when the reference moves (or half of that: it moves by powers of two).  Results add up
// to 2^31 probabilities times values, which must not pass 32 bits where the result does not: of bf16 values, which may be as
// large as those, far below 1 (bf16 has the range); of fp16 values and codes there is room.  Probabilities over fp16 values
// are their weights: they begin at the upper end of half precision, 2^15 with the lag.
constexpr float kBase = kQuantised ? 0.f : DISC_T_F16 ? 11.f : -40.f;
constexpr float kWeight = 11.f, kMostWeight = 15.f;   // log2 of the largest weight when its power of two is set, and at any time

// A step's scores, scaled, relative to the reference of their row and masked; where they pass it by more than the lag
// (or it is the first time that there are any), the reference moves up to them, and sum and result with it.
template <int RT>
DISC_DEV void bound_step(Rows<RT>& R, f32x4 (&s)[RT][2], float (&ks)[8], float (&vs)[8], int live) {
  if (R.uneven) {
    asm volatile("");                             // (a branch, as below)
#pragma unroll
    for (int j = 0; j < 8; ++j) {                 // (exponents added up: a score is out of range only if all of it is)
      const int e = __builtin_amdgcn_frexp_expf(ks[j]);
      ks[j] = __builtin_amdgcn_frexp_mantf(ks[j]);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt][j / 4][j % 4] = __builtin_ldexpf(s[rt][j / 4][j % 4], R.row[rt] + e);
    }
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int j = 0; j < 8; ++j) s[rt][j / 4][j % 4] = __builtin_fmaf(s[rt][j / 4][j % 4], ks[j], -R.use[rt]);
  if (__ballot(live < 8)) {                       // some token of the step is not there
    asm volatile("");                             // (a branch, and not a select for every score of every step)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt][j / 4][j % 4] = j < live ? s[rt][j / 4][j % 4] : kNone;
      vs[j] = j < live ? vs[j] : 0.f;
    }
  }
  bool late = false;
  float top[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    top[rt] = kNone;
#pragma unroll
    for (int j = 0; j < 8; ++j) top[rt] = fmaxf(top[rt], s[rt][j / 4][j % 4]);
    late |= top[rt] > R.lim[rt];
  }
  if (kQuantised) {
    float vtop = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) vtop = fmaxf(vtop, fabsf(vs[j]));
    // (a bound of the weights, of the largest score and the largest scale of eight tokens; times 2^32, so that it is no
    // subnormal number, of which the hardware has no logarithm)
    const float v = __builtin_amdgcn_logf(vtop * 0x1p32f) - 32.f;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) late |= top[rt] + v > R.room[rt];
  }
  if (__ballot(late)) {                           // seldom after the first steps
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const float t = max_of_groups(top[rt]);
      const bool first = R.lim[rt] == kNone;
      const float past = t - kBase, shift = past > (first ? kNone : 0.f) ? ceilf(past) : 0.f;
      const float alpha = first ? 0.f : __builtin_amdgcn_exp2f(-shift);
      float turn = alpha;                         // on the results
      if (kQuantised) {
        // The weights' power of two makes up for the reference's move, so that the results stay as they are, unless the
        // step's largest weight has no room.  (By the scales' exponents: one too many at most.)
        float w = kNone;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float e = (float)__builtin_amdgcn_frexp_expf(vs[j]);
          w = fmaxf(w, vs[j] != 0.f ? s[rt][j / 4][j % 4] + e : kNone);
        }
        w = max_of_groups(w) - shift;
        const float before = kMostWeight - R.room[rt] + shift;       // (infinity: there is none yet)
        float e = fminf(before, 100.f);
        if (w + e > kMostWeight) e = fmaxf(kWeight - ceilf(w), -120.f);
        const bool any = w > kNone || R.grow[rt] > 0.f;
        turn = R.grow[rt] > 0.f ? __builtin_ldexpf(1.f, (int)(e - before)) : 0.f;
        R.grow[rt] = any ? __builtin_ldexpf(1.f, (int)e) : 0.f;
        R.room[rt] = any ? kMostWeight - e : kNone;
      }
      R.use[rt] += shift;
      R.lim[rt] = t > kNone ? kBase + kLag : R.lim[rt];
      if (__ballot(!first)) {                     // (nothing was summed before the first time)
        asm volatile("");
        R.l[rt] *= alpha;
#pragma unroll
        for (int d = 0; d < kND; ++d) R.o[rt][d] *= turn;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) s[rt][j / 4][j % 4] -= shift;
    }
  }
}

// The step's weights, in place of its scores.
template <int RT>
DISC_DEV void weigh_step(Rows<RT>& R, f32x4 (&s)[RT][2], const float (&vs)[8]) {
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float p = __builtin_amdgcn_exp2f(s[rt][j / 4][j % 4]);
      sum += p;
      if (kQuantised) p *= vs[j] * R.grow[rt];
      s[rt][j / 4][j % 4] = p;
    }
    R.l[rt] += sum;
  }
}

#if DISC_T_F16 || DISC_STORAGE != 0
typedef _Float16 P;
#else
typedef __bf16 P;
#endif
typedef P Px2 __attribute__((ext_vector_type(2)));

// The probabilities as the second product's operand.
template <int RT>
DISC_DEV void split(const f32x4 (&s)[RT][2], u32x4 (&hi)[RT], u32x4 (&lo)[RT]) {
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float a = s[rt][w / 2][(2 * w) % 4], b = s[rt][w / 2][(2 * w + 1) % 4];
      const Px2 both = {(P)a, (P)b};
      u32 x = __builtin_bit_cast(u32, both);
      if (kSplit) {
        // (What is left of the very numbers that are multiplied: the compiler may form another (P)a from what `a` is a product
        // of, which is rounded once and differs now and then by a unit of its last place, and `lo` by as much.)
        asm("" : "+v"(x));
        const Px2 h = __builtin_bit_cast(Px2, x), r = {(P)(a - (float)h[0]), (P)(b - (float)h[1])};
        lo[rt][w] = __builtin_bit_cast(u32, r);
      }
      hi[rt][w] = x;
    }
}

template <int RT>
DISC_DEV void accumulate(Rows<RT>& R, const f32x4 (&s)[RT][2], Values& V, int live) {
  if (__ballot(live < 8)) {                       // what is behind the end may hold anything: 0 * NaN is no 0
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int w = 0; w < kNB * kVW; ++w) V.v[j][w] = j < live ? V.v[j][w] : 0u;
  }
  u32x4 hi[RT], lo[RT];
  split<RT>(s, hi, lo);
#pragma unroll
  for (int n = 0; n < kNB; ++n)
#pragma unroll
    for (int i = 0; i < kE; ++i) {
      const u32x4 v = column_of(V, n, i);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        R.o[rt][n * kE + i] = mfma(v, hi[rt], R.o[rt][n * kE + i]);
        if (kSplit) R.o[rt][n * kE + i] = mfma(v, lo[rt], R.o[rt][n * kE + i]);
      }
    }
}

// The tokens begin + first, + stride, ... (steps of 32) up to end, for the rows of one wavefront.
template <int RT, bool kNt>
DISC_DEV void attend_tokens(const AttendArgs& A, const u32* rows, float* scales, int begin, int end, int first, int stride, Rows<RT>& R) {
  const int lane = threadIdx.x & 63, g = lane >> 4, base = begin >> A.shift;
  int t0 = begin + first;
  if (t0 >= end) return;
  // (places behind the chunk's last token are read at its last group of eight: in the page, masked below)
  const int last = (end - 1) & ~7;
  Keys K;
  Values V;
  float scale = 0.f;
  load_keys<kNt>(A, rows, base, last, t0, K);
  if (kQuantised) scale = load_scale(A, rows, base, last, t0);
  bool there = load_values<kNt>(A, rows, base, last, t0, V);
  do {
    f32x4 s[RT][2];
    const int n = end - (t0 + g * 8);
    const int live = !there || n <= 0 ? 0 : n < 8 ? n : 8;
    scores<RT>(R, K, s);
    // (this wavefront's 64 floats of LDS: the lanes' eight tokens' scales from the lanes that read them)
    float ks[8], vs[8];
    if (kQuantised) scales[lane] = lane < 32 ? scale * R.factor : scale;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      ks[j] = kQuantised ? scales[g * 8 + j] : R.factor;
      vs[j] = kQuantised ? scales[32 + g * 8 + j] : 1.f;
    }
    // The next step's keys are read while this one's probabilities and second product run, its values after that, in
    // the registers that are free then.  (Behind the end the last rows come again: a load that only some steps make
    // would have every step wait for all loads before it.)
    const int next = t0 + stride;
    load_keys<kNt>(A, rows, base, last, next, K);
    if (kQuantised) scale = load_scale(A, rows, base, last, next);
    __builtin_amdgcn_sched_barrier(0);
    bound_step<RT>(R, s, ks, vs, live);
    weigh_step<RT>(R, s, vs);
    accumulate<RT>(R, s, V, live);
    there = load_values<kNt>(A, rows, base, last, next, V);
    __builtin_amdgcn_sched_barrier(0);
    t0 = next;
  } while (t0 < end);
}

template <int RT>
DISC_DEV void clear_rows(Rows<RT>& R) {
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    R.lim[rt] = kNone;
    R.use[rt] = R.l[rt] = R.grow[rt] = 0.f;
    R.room[rt] = kNone;
#pragma unroll
    for (int d = 0; d < kND; ++d) R.o[rt][d] = (f32x4){0, 0, 0, 0};
  }
  R.factor = (float)(DISC_SCALE_LOG2E);
  R.uneven = false;
}

// The query rows' operand: lane (n, g) holds row n, the elements that the keys' lanes hold of theirs.
template <int RT>
DISC_DEV void load_query(Rows<RT>& R, int rt, const T* p) {      // p: this lane's row, or null
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int i = 0; i < kNK; ++i)
#pragma unroll
    for (int f = 0; f < kKE / 8; ++f) {
      const int d = i * 4 * kKE + g * kKE + f * 8;
      R.q[rt][i * (kKE / 8) + f] = p && d < kD ? *(const u32x4_u*)(p + d) : (u32x4){0, 0, 0, 0};
    }
}

// bf16 queries for keys that are codes, in half precision: 2^15 is the power of two of the largest of them all, of the
// wavefront or of the block (`most`: its bits).  What is below 2^-39 of it is lost, and a row of 2^-16 of it has an error
// of 2^-24 of its own largest: of a score, 2^-24 of the row's largest |q| times the sum of |k|, as much as its sum of D
// products is rounded by.  A row that is smaller still has a power of two of its own, so that nothing another sequence or
// head brings along takes its bits; rows that hold a NaN or an infinity are not asked for theirs, and keep them.
template <int RT>
DISC_DEV u32 largest_queries(const Rows<RT>& R, u32 (&top)[RT]) {     // bits of |q|: of this lane's rows, of all finite ones
  u32 most = 0;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    top[rt] = 0;
#pragma unroll
    for (int i = 0; i < kNK * (kKE / 8); ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) top[rt] = max(top[rt], max(R.q[rt][i][w] & 0x7fffu, (R.q[rt][i][w] >> 16) & 0x7fffu));
    top[rt] = max(top[rt], (u32)__shfl_xor((int)top[rt], 16));
    top[rt] = max(top[rt], (u32)__shfl_xor((int)top[rt], 32));
    if (top[rt] < 0x7f80u) most = max(most, top[rt]);
  }
#pragma unroll
  for (int d = 1; d < 16; d *= 2) most = max(most, (u32)__shfl_xor((int)most, d));
  return most;
}
// By biased exponents: 2^15 is brought to by 2^(142 - e), or the largest power of two there is; its exponent.
DISC_DEV int up_of(int e) { return min(142 - max(e, 1), 127); }
DISC_DEV bool far_below(u32 top, int e) { return top != 0 && (int)(top >> 7) + 16 < e; }
// Whether some row of this lane's asks for its own (or the largest, or the softmax scale, is so large that its power of two
// and the scale might have no product).
template <int RT>
DISC_DEV bool uneven_queries(const u32 (&top)[RT], u32 most) {
  const int e = (int)(most >> 7);
  bool uneven = e > 200 || DISC_SCALE_LOG2E > 0x1p60 || DISC_SCALE_LOG2E < -0x1p60;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) uneven |= far_below(top[rt], e);
  return !DISC_T_F16 && uneven;
}
DISC_DEV float power(int e) { return __builtin_bit_cast(float, (u32)(127 + e) << 23); }    // 2^e, -126 .. 127
template <int RT>
DISC_DEV void halve_query(Rows<RT>& R, const u32 (&top)[RT], u32 most, bool uneven) {
#if !DISC_T_F16
  const int e = (int)(most >> 7);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int up = up_of(far_below(top[rt], e) ? (int)(top[rt] >> 7) : e);
    const float f = power(up);
    R.row[rt] = (DISC_STORAGE == 1 ? 9 : 0) - up;           // (and 1 / kCode)
#pragma unroll
    for (int i = 0; i < kNK * (kKE / 8); ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const u32 x = R.q[rt][i][w];
        const f16x2 y = {(_Float16)(__builtin_bit_cast(float, x << 16) * f), (_Float16)(__builtin_bit_cast(float, x & 0xffff0000u) * f)};
        R.q[rt][i][w] = __builtin_bit_cast(u32, y);
      }
  }
  R.uneven = uneven;
  if (uneven) return;
  R.factor *= 1.f / power(up_of(e));
#endif
  R.factor *= 1.f / kCode;
}

// Rows of the pages of the tokens [begin, end), for a kv head, into LDS, by `of` threads.
DISC_DEV void stage_pages(const AttendArgs& A, const int* table, int width, int begin, int end, int h, u32* rows, int thread, int of) {
  const int base = begin >> A.shift, n = ((end - 1) >> A.shift) - base + 1;
  for (int i = thread; i < n; i += of) {
    const int p = base + i < width ? table[base + i] : -1;
    rows[i] = p >= 0 && p < A.pages ? ((u32)p * (u32)A.kv_heads + (u32)h) << A.shift : kNoPage;
  }
}

// Element of O^T that register r of a lane's tile (n, i) holds.
DISC_DEV int element_of(int n, int i, int r) {
  return (n * 16 + (((threadIdx.x & 63) >> 4) * 4 + r)) * kE + i;
}

DISC_DEV void store4(T* p, f32x4 x) {
  const Tx2 a = {(T)x[0], (T)x[1]}, b = {(T)x[2], (T)x[3]};
  *(u32x2_u*)p = (u32x2){__builtin_bit_cast(u32, a), __builtin_bit_cast(u32, b)};
}

// Row of the partial results: a chunk's (first the sequences', then the prefix's), for a query head.
DISC_DEV i64 part_row(const AttendArgs& A, int chunk, int head) { return (i64)chunk * A.heads + head; }
DISC_DEV i64 prefix_row(const AttendArgs& A, int part, int b, int head) {
  return (i64)A.parts * A.heads + ((i64)part * A.batch + b) * A.heads + head;
}

// What wavefronts have of the same rows, put together: each leaves its registers in LDS, four neighbouring elements of the
// result (register r of four tiles) a piece, and finishes a share of the registers r of all of them.  (Two and two, then the
// two, with one of them finishing all: eight sequences of 100 x 256 elements 9.2 us where this takes 8.3.)
constexpr int kPieces = kND / 4;
static_assert(kND % 4 == 0 && kE % 4 == 0, "a piece is of one group of tiles");
struct Other {
  f32x4 o[4][kPieces][64];
  float use[64], l[64], unit[kQuantised ? 64 : 1];   // use: -infinity where there was no score
};
// One over the weights' power of two: results times this (and one over kCode) are the values'.  It is multiplied in last,
// when they are divided by their sum: before, a power of two close to the largest would make them infinite.
template <int RT>
DISC_DEV float unit_of(const Rows<RT>& R, int rt) { return kQuantised ? (R.grow[rt] > 0.f ? 1.f / R.grow[rt] : 0.f) : 1.f; }
DISC_DEV float reference(const Rows<1>& R) { return R.lim[0] > kNone ? R.use[0] : kNone; }
// (no reference: the sum is 0, or NaN where every score was)
DISC_DEV float weight(float use, float top, float l) { return use > kNone ? __builtin_amdgcn_exp2f(use - top) : l; }
DISC_DEV f32x4 piece_of(const Rows<1>& R, int r, int q) {
  return (f32x4){R.o[0][4 * q][r], R.o[0][4 * q + 1][r], R.o[0][4 * q + 2][r], R.o[0][4 * q + 3][r]};
}
DISC_DEV void hand_over(const Rows<1>& R, Other& X) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int q = 0; q < kPieces; ++q) X.o[r][q][lane] = piece_of(R, r, q);
  X.use[lane] = reference(R);
  X.l[lane] = R.l[0];
  if (kQuantised) X.unit[lane] = unit_of(R, 0);
}

// `kWays` wavefronts work on the same rows, 4 / kWays rows sets a block.
// Four: a block's share of the sequences' tokens, for one kv head and 16 of its query heads at most; or, where the query
// rows of all sequences are few, one chunk of the prefix for 16 of them.  One or two: all of a short sequence, where
// there are so many that blocks of four would come in several rounds, each with its latency of five steps.
template <int kWays, bool kNt>
DISC_DEV void attend_body(const AttendArgs& A) {
  constexpr int kSets = 4 / kWays, kIds = kWays == 4 ? kMostPages + 1 : kDirectPages;   // (a stretch need not begin with a page)
  __shared__ u32 all_pages[kSets][kIds];
  __shared__ Other other[kWays == 1 ? 1 : 4];
  __shared__ __align__(16) float scales[4][64];
  const int w = wavefront(), n = threadIdx.x & 15, set = w / kWays, turn = w % kWays;
  u32* pages = all_pages[set];
  const int shared_blocks = kWays == 4 ? A.prefix_tiles * A.prefix_parts * A.kv_heads : 0;
  const bool shared = (int)blockIdx.x < shared_blocks;
  int part, h, row0, rows;                // rows: of this set; the first is number row0 of the kv head's
  Walk I;
  I.b = I.begin = 0;
  I.whole = !shared;
  if (shared) {
    const int per = A.prefix_parts * A.kv_heads, tile = blockIdx.x / per, rest = blockIdx.x - tile * per;
    part = rest / A.kv_heads;
    h = rest - part * A.kv_heads;
    row0 = tile * 16;
    rows = min(A.batch * A.group - row0, 16);
    I.begin = part * A.prefix_chunk;
    I.end = min(A.prefix_len, I.begin + A.prefix_chunk);
  } else {
    const int block = (blockIdx.x - shared_blocks) * kSets + set, per = A.kv_heads * A.tiles;
    part = block / per;
    const int rest = block - part * per;
    h = rest / A.tiles;
    row0 = (rest - h * A.tiles) * 16;
    rows = min(A.group - row0, 16);
    if (kWays < 4 || A.direct) {
      if (kWays < 4 && part >= A.batch) part = rows = 0;       // (behind the last sequence: the barriers are for all)
      // (all of the sequence's table, which is short, without waiting for its length)
      I.b = part;
      stage_pages(A, A.table + (i64)part * A.width, A.width, 0, A.width << A.shift, h, pages, turn * 64 + (threadIdx.x & 63), kWays * 64);
      if (kWays == 4 && A.prefix_inline)
        stage_pages(A, A.prefix_table, (A.prefix_len + (1 << A.shift) - 1) >> A.shift, 0, A.prefix_len, h, pages + kDirectPages, threadIdx.x, 256);
      I.end = rows ? clamp_length(A.lengths[part], A.width, A.shift) : 0;
    } else {
      I.start(A, part);
      if (!I.next(A)) return;
    }
  }
  const int width = shared ? (A.prefix_len + (1 << A.shift) - 1) >> A.shift : A.width;
  while (true) {
    const int* table = shared ? A.prefix_table : A.table + (i64)I.b * A.width;
    // sequence and query head of this lane's row
    const int b = shared ? (row0 + n) / A.group : I.b, head = h * A.group + (shared ? row0 + n - b * A.group : row0 + n);
    Rows<1> R;
    clear_rows<1>(R);
    load_query<1>(R, 0, n < rows ? A.q + b * A.q_row + head * A.q_head : nullptr);
    if (kQuantised) {
      u32 top[1];
      const u32 largest = largest_queries<1>(R, top);
      halve_query<1>(R, top, largest, __ballot(uneven_queries<1>(top, largest)) != 0);
    }
    const int most = kMostPages << A.shift;
    bool ahead = kWays == 4 && A.prefix_inline;                // the prefix, in front of the sequence's own
    for (int at = ahead ? 0 : I.begin;;) {
      const int end = ahead ? A.prefix_len : I.end, to = end - at > most ? at + most : end;
      if (kWays == 4 && at < end && (shared || !A.direct)) stage_pages(A, table, width, at, to, h, pages, threadIdx.x, 256);
      __syncthreads();
      attend_tokens<1, kNt>(A, ahead ? pages + kDirectPages : pages, scales[w], at, to, turn * kStep, kWays * kStep, R);
      at = to;
      if (ahead) {
        ahead = false;
        at = I.begin;
        continue;
      }
      if (kWays < 4 || at >= end) break;
      __syncthreads();
    }
    R.l[0] += __shfl_xor(R.l[0], 16);
    R.l[0] += __shfl_xor(R.l[0], 32);
    // register r of this wavefront's share, of all that work on these rows
    constexpr int kShare = 4 / kWays;
    f32x4 done[kShare][kPieces];
    float top = reference(R), l = R.l[0], unit = unit_of(R, 0);
    if (kWays == 1) {
#pragma unroll
      for (int i = 0; i < kShare; ++i)
#pragma unroll
        for (int q = 0; q < kPieces; ++q) done[i][q] = piece_of(R, i, q);
    } else {
      const int lane = threadIdx.x & 63;
      hand_over(R, other[w]);
      __syncthreads();
      const Other* all = other + set * kWays;
      float use[kWays], sum[kWays], units[kWays];
#pragma unroll
      for (int i = 0; i < kWays; ++i) {
        use[i] = all[i].use[lane], sum[i] = all[i].l[lane], top = fmaxf(top, use[i]);
        if (kQuantised) units[i] = all[i].unit[lane], unit = fmaxf(unit, units[i]);
      }
      const float per = kQuantised && unit > 0.f ? 1.f / unit : 0.f;
      l = 0.f;
#pragma unroll
      for (int i = 0; i < kWays; ++i) {
        float f = weight(use[i], top, sum[i]);
        l += use[i] > kNone ? sum[i] * f : sum[i];
        if (kQuantised) f *= units[i] * per;
#pragma unroll
        for (int j = 0; j < kShare; ++j)
#pragma unroll
          for (int q = 0; q < kPieces; ++q) {
            const f32x4 o = all[i].o[turn + j * kWays][q][lane] * f;
            done[j][q] = i ? done[j][q] + o : o;
          }
      }
    }
    if (n < rows) {
      const bool alone = I.whole && A.prefix_parts == 0;
      // (the sum is 2^(kBase - 1) or more where it is not 0: its reciprocal is rounded to 32 bits, of which the result keeps 11 at most)
      const float inverse = 1.f / kCode / l;
      const i64 at = shared ? prefix_row(A, part, b, head) : part_row(A, A.direct ? b : part + b, head);
      T* out = A.out + b * A.o_row + head * A.o_head;
#pragma unroll
      for (int q = 0; q < kPieces; ++q)
#pragma unroll
        for (int j = 0; j < kShare; ++j) {
          const int d = element_of(q / (kE / 4), q % (kE / 4) * 4, turn + j * kWays);
          if (d >= kD) continue;
          f32x4 x = l != 0.f ? done[j][q] * inverse : (f32x4){0, 0, 0, 0};
          if (kQuantised) x *= unit;
          if (alone) store4(out + d, x);
          else *(f32x4*)(A.part + at * kD + d) = x;
        }
      if (!alone && turn == 0 && (threadIdx.x & 63) < 16) A.part_m[2 * at] = top, A.part_m[2 * at + 1] = l;
    }
    if (kWays < 4 || shared || A.direct || !I.next(A)) return;
    __syncthreads();                      // (what was handed over is still being read)
  }
}
// (wavefronts a SIMD by the registers that they take, few of which are spilled: 2 to 4 of 168 over 16-bit rows of 128, outside
// the loop over tokens; 16-bit rows of 256 do not fit 256: 31 spilled ones cost 60 us where one wavefront takes 36, four
// sequences of 15000; heads of up to 48 have the tiles of 128, three wavefronts and none spilled 39 us, four 52, 64 sequences
// of 4000 x 32)
constexpr int kWavesPerSimd = kD <= 64 && kND <= 4 ? 4 : kD <= 128 ? 3 : kQuantised ? 2 : 1;
#define DISC_ATTEND(NAME, WAYS, NT) \
  extern "C" __global__ void __launch_bounds__(256, kWavesPerSimd) NAME(AttendArgs A) { attend_body<WAYS, NT>(A); }
DISC_ATTEND(disc_attend_k, 4, false)
DISC_ATTEND(disc_attend2_k, 2, false)
DISC_ATTEND(disc_attend1_k, 1, false)
DISC_ATTEND(disc_attend_nt_k, 4, true)
DISC_ATTEND(disc_attend2_nt_k, 2, true)
DISC_ATTEND(disc_attend1_nt_k, 1, true)

// One chunk of the shared prefix for one kv head, where the batch has many query rows: each of the eight wavefronts
// has 16 x RT rows of its own, and all go through the same tokens.  A tile of them is read once a block, brought into
// the matrix operands' form -- codes to 16-bit numbers, values transposed -- and kept in LDS in the order in which a
// wavefront reads an operand (16 bytes a lane, one row after the other); the next tile's loads are in flight
// meanwhile, and two tiles take turns.  1024 rows x 16384 tokens x 8 heads of 128, i8: 98 to 100 us, 0.69 PFLOP/s (bf16 and
// fp16, twice the second product: 127 to 130).  Bound by issue: the matrix cores are busy for 29 % of the cycles, the vector ALU
// for 49 % (sixteen powers of two at a quarter of the rate, and what goes round them, a step), little of it at once; wavefronts
// wait for 33 % of their time.  Of heads of 256 and over e4m3 up to 5 registers of 256 are spilled.
constexpr int kPrefixRT = kD <= 128 ? 2 : 1;
constexpr int kPrefixSteps = kD <= 128 ? 4 : 2;               // steps of a tile
constexpr int kNF = kNK * (kKE / 8);                          // operands of a step's keys, a 16-row tile
struct PrefixTile {
  u32x4 k[kPrefixSteps][2 * kNF][64];
  u32x4 v[kPrefixSteps][kND][64];
  float ks[kPrefixSteps * kStep], vs[kPrefixSteps * kStep];
  int live[kPrefixSteps * 4];                                 // tokens that are there, of every eight
};
extern "C" __global__ void __launch_bounds__(512, 2) disc_prefix_k(AttendArgs A) {
  __shared__ PrefixTile tiles[2];
  __shared__ u32 pages[kMostPages + 1];
  __shared__ u32 tops[8], uneven[8];
  const int lane = threadIdx.x & 63, w = wavefront(), n = lane & 15, g = lane >> 4;
  // (blocks of the same chunk and kv head are a multiple of eight apart where there are that many: on one XCD)
  const int all = A.batch * A.group, per = A.prefix_parts * A.kv_heads;
  const int block = blockIdx.x / per, rest = blockIdx.x - block * per, part = rest / A.kv_heads, h = rest - part * A.kv_heads;
  const int begin = part * A.prefix_chunk, end = min(A.prefix_len, begin + A.prefix_chunk);
  const int base = begin >> A.shift, last = (end - 1) & ~7;
  stage_pages(A, A.prefix_table, (A.prefix_len + (1 << A.shift) - 1) >> A.shift, begin, end, h, pages, threadIdx.x, 512);
  const int row0 = (block * 8 + w) * kPrefixRT * 16;
  Rows<kPrefixRT> R;
  clear_rows<kPrefixRT>(R);
#pragma unroll
  for (int rt = 0; rt < kPrefixRT; ++rt) {
    const int row = row0 + rt * 16 + n, b = row / A.group, i = row - b * A.group;
    load_query<kPrefixRT>(R, rt, row < all ? A.q + b * A.q_row + (h * A.group + i) * A.q_head : nullptr);
  }
  if (kQuantised) {                                           // (one power of two for the block: its keys' scales are shared)
    u32 top[kPrefixRT], largest = largest_queries<kPrefixRT>(R, top);
    tops[w] = largest;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) largest = max(largest, tops[i]);
    uneven[w] = __ballot(uneven_queries<kPrefixRT>(top, largest)) != 0;
    __syncthreads();
    u32 some = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) some |= uneven[i];
    halve_query<kPrefixRT>(R, top, largest, __builtin_amdgcn_readfirstlane(some) != 0);
  }
  const bool keys = w < kPrefixSteps, values = !keys && w < 2 * kPrefixSteps;
  const int step = keys ? w : w - kPrefixSteps;               // this wavefront's share of a tile
  // (either of them, in the same registers)
  constexpr int kKeyWords = 2 * kNK * 4, kValueWords = 8 * kNB * kVW;
  u32 held[kKeyWords > kValueWords ? kKeyWords : kValueWords];
  float scale = 0.f;                                          // of token `lane` of the step
  int live = 0;
  auto fetch_tile = [&](int t0) {                                  // t0: the tile's first token
    t0 += step * kStep;
    bool there;
    if (keys) {
      Keys K;
      load_keys<false>(A, pages, base, last, t0, K);
#pragma unroll
      for (int x = 0; x < kKeyWords; ++x) held[x] = K.k[x / (4 * kNK)][x / 4 % kNK][x % 4];
    }
    if (values) {
      Values V;
      there = load_values<false>(A, pages, base, last, t0, V);
      const int m = end - (t0 + g * 8);
      live = !there || m <= 0 ? 0 : m < 8 ? m : 8;
#pragma unroll
      for (int x = 0; x < kValueWords; ++x) held[x] = V.v[x / (kNB * kVW)][x % (kNB * kVW)];
    }
    if (kQuantised && (keys || values)) {
      const int t = min(t0 + (lane & 31), last + 7);
      scale = (keys ? A.ks : A.vs)[row_of(A, pages, base, t, there)];
    }
  };
  auto put_tile = [&](PrefixTile& T) {
    if (keys) {
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int i = 0; i < kNK; ++i) {
          const u32* x = held + (mt * kNK + i) * 4;
          if (!kQuantised) {
            T.k[step][mt * kNF + i][lane] = (u32x4){x[0], x[1], x[2], x[3]};
          } else {
            T.k[step][mt * kNF + 2 * i][lane] = keys_of_codes(x[0], x[1]);
            T.k[step][mt * kNF + (2 * i + 1) % kNF][lane] = keys_of_codes(x[2], x[3]);
          }
        }
      if (kQuantised && lane < kStep) T.ks[step * kStep + lane] = scale * R.factor;
    }
    if (values) {
      Values V;
#pragma unroll
      for (int j = 0; j < 8; ++j)                             // (what is behind the end may hold anything)
#pragma unroll
        for (int x = 0; x < kNB * kVW; ++x) V.v[j][x] = j < live ? held[j * kNB * kVW + x] : 0u;
      if (n == 0) T.live[step * 4 + g] = live;
      if (kQuantised) {
        const int alive = __shfl(live, ((lane & 31) >> 3) * 16);
        if (lane < kStep) T.vs[step * kStep + lane] = (lane & 7) < alive ? scale : 0.f;
      }
#pragma unroll
      for (int x = 0; x < kNB; ++x)
#pragma unroll
        for (int i = 0; i < kE; ++i) T.v[step][x * kE + i][lane] = column_of(V, x, i);
    }
  };
  __syncthreads();
  fetch_tile(begin);
  put_tile(tiles[0]);
  __syncthreads();
  constexpr int kTile = kPrefixSteps * kStep;
  for (int t0 = begin, turn = 0; t0 < end; t0 += kTile, turn ^= 1) {
    const PrefixTile& T = tiles[turn];
    if (t0 + kTile < end) fetch_tile(t0 + kTile);
    if (row0 < all) {
      // The next step's scores are in the matrix cores while this one's probabilities are formed.  (Steps behind the end
      // have no token that is there.)
      f32x4 s[2][kPrefixRT][2];
      u32x4 kf[2 * kNF];
      auto read_keys = [&](int st) {
#pragma unroll
        for (int i = 0; i < 2 * kNF; ++i) kf[i] = T.k[st][i][lane];
      };
      auto score = [&](int st) {
        f32x4(&x)[kPrefixRT][2] = s[st & 1];
#pragma unroll
        for (int rt = 0; rt < kPrefixRT; ++rt) x[rt][0] = x[rt][1] = (f32x4){0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < kNF; ++i)
#pragma unroll
          for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int rt = 0; rt < kPrefixRT; ++rt) x[rt][mt] = mfma(kf[mt * kNF + i], R.q[rt][i], x[rt][mt]);
      };
      read_keys(0);
      score(0);
#pragma unroll
      for (int st = 0; st < kPrefixSteps; ++st) {
        float ks[8], vs[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          ks[j] = kQuantised ? T.ks[st * kStep + g * 8 + j] : R.factor;
          vs[j] = kQuantised ? T.vs[st * kStep + g * 8 + j] : 1.f;
        }
        const int live = T.live[st * 4 + g];
        if (st + 1 < kPrefixSteps) read_keys(st + 1);
        __builtin_amdgcn_sched_barrier(0);
        bound_step<kPrefixRT>(R, s[st & 1], ks, vs, live);
        __builtin_amdgcn_s_setprio(1);
        if (st + 1 < kPrefixSteps) score(st + 1);
        weigh_step<kPrefixRT>(R, s[st & 1], vs);
        u32x4 hi[kPrefixRT], lo[kPrefixRT];
        split<kPrefixRT>(s[st & 1], hi, lo);
        __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int d = 0; d < kND; ++d) {
          const u32x4 v = T.v[st][d][lane];
#pragma unroll
          for (int rt = 0; rt < kPrefixRT; ++rt) {
            R.o[rt][d] = mfma(v, hi[rt], R.o[rt][d]);
            if (kSplit) R.o[rt][d] = mfma(v, lo[rt], R.o[rt][d]);
          }
        }
      }
    }
    if (t0 + kTile < end) put_tile(tiles[turn ^ 1]);
    __syncthreads();
  }
#pragma unroll
  for (int rt = 0; rt < kPrefixRT; ++rt) {
    R.l[rt] += __shfl_xor(R.l[rt], 16);
    R.l[rt] += __shfl_xor(R.l[rt], 32);
    const int row = row0 + rt * 16 + n, b = row / A.group, i = row - b * A.group;
    if (row >= all) continue;
    const i64 at = prefix_row(A, part, b, h * A.group + i);
    const float l = R.l[rt], f = l != 0.f ? 1.f / kCode / l : 0.f, unit = unit_of(R, rt);
#pragma unroll
    for (int x = 0; x < kNB; ++x)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int d = element_of(x, 0, r);
        if (d < kD) {
#pragma unroll
          for (int e = 0; e < kE; e += 4) {
            f32x4 y = {R.o[rt][x * kE + e][r] * f, R.o[rt][x * kE + e + 1][r] * f, R.o[rt][x * kE + e + 2][r] * f, R.o[rt][x * kE + e + 3][r] * f};
            if (kQuantised) y *= unit;
            *(f32x4*)(A.part + at * kD + d + e) = y;
          }
        }
      }
    if (g == 0) A.part_m[2 * at] = R.lim[rt] > kNone ? R.use[rt] : kNone, A.part_m[2 * at + 1] = R.l[rt];
  }
}

// Joins the chunks of a sequence and of the prefix, for a (sequence, query head) a wavefront, or where the rows are few
// and their chunks many, a block.  The chunks' maxima and sums are read 64 at a time, a lane each, so that the reads
// of the results themselves do not wait for each other.  A chain of trips to memory, 3 to 12 us: more wavefronts a row do not
// shorten it (sixteen 8.2 us where four take 7.1).
extern "C" __global__ void __launch_bounds__(256) disc_join_k(AttendArgs A) {
  __shared__ float so[4][kD], sm[4], sl[4];
  const int w = wavefront(), lane = threadIdx.x & 63, ways = A.join_ways;
  const i64 row = ways == 1 ? (i64)blockIdx.x * 4 + w : (i64)blockIdx.x;
  const int b = (int)(row / A.heads), head = (int)(row - (i64)b * A.heads);
  if (b >= A.batch) return;                                   // (one wavefront a row: no barrier comes)
  int chunk = b, count = 1;
  if (!A.direct) {
    chunks_of(A, b, chunk, count);
    if (count == 1 && A.prefix_parts == 0) return;            // the chunk's own block wrote the result
  }
  const int n = count + A.prefix_parts;
  constexpr int kPer = (kD + 63) / 64;
  float o[kPer], m = kNone, l = 0.f;
#pragma unroll
  for (int e = 0; e < kPer; ++e) o[e] = 0.f;
  // this wavefront's chunks: n0 + x * ways
  const int first = ways == 1 ? 0 : w;
  for (int i0 = first; i0 < n; i0 += 64 * ways) {
    const int i = i0 + lane * ways;
    const i64 at = i < count ? part_row(A, chunk + i, head) : prefix_row(A, min(i, n - 1) - count, b, head);
    const float pm = i < n ? A.part_m[2 * at] : kNone, pl = i < n ? A.part_m[2 * at + 1] : 0.f;
    const int most = min(64, (n - i0 + ways - 1) / ways);
    float v[8][kPer];
    auto read = [&](int x0) {
#pragma unroll
      for (int x = 0; x < 8; ++x) {                           // (the last one again, with a weight of 0, behind the end)
        const int j = i0 + min(x0 + x, most - 1) * ways;
        const i64 slot = j < count ? part_row(A, chunk + j, head) : prefix_row(A, j - count, b, head);
#pragma unroll
        for (int e = 0; e < kPer; ++e) v[x][e] = e * 64 + lane < kD ? A.part[slot * kD + e * 64 + lane] : 0.f;
      }
    };
    read(0);                                                  // (on their way while the weights are formed)
    __builtin_amdgcn_sched_barrier(0);
    float top = fmaxf(m, pm);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    // A chunk's result counts by its sum.  (No reference: nothing was there, or every score was NaN and so is the sum.  The
    // sums are at most 2^(kBase + kLag + 31): their weights are brought below 1, so that no result grows on the way.)
    const float f = pm > kNone ? pl * __builtin_amdgcn_exp2f(pm - top - (kBase + kLag + 32.f)) : pl;
    float sum = f;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    const float before = m > kNone ? __builtin_amdgcn_exp2f(m - top) : l;
    l = (m > kNone ? l * before : l) + sum;
    m = top;
#pragma unroll
    for (int e = 0; e < kPer; ++e) o[e] *= before;
    for (int x0 = 0; x0 < most; x0 += 8) {
      if (x0) read(x0);
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const float fx = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), min(x0 + x, 63)));
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[e] = x0 + x < most ? o[e] + v[x][e] * fx : o[e];
      }
    }
  }
  if (ways > 1) {
#pragma unroll
    for (int e = 0; e < kPer; ++e)
      if (e * 64 + lane < kD) so[w][e * 64 + lane] = o[e];
    if (lane == 0) sm[w] = m, sl[w] = l;
    __syncthreads();
    if (w > 0) return;
    float top = kNone;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = fmaxf(top, sm[i]);
    l = 0.f;
#pragma unroll
    for (int e = 0; e < kPer; ++e) o[e] = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float f = sm[i] > kNone ? __builtin_amdgcn_exp2f(sm[i] - top) : sl[i];
      l += sm[i] > kNone ? sl[i] * f : sl[i];
#pragma unroll
      for (int e = 0; e < kPer; ++e)
        if (e * 64 + lane < kD) o[e] += so[i][e * 64 + lane] * f;
    }
  }
#pragma unroll
  for (int e = 0; e < kPer; ++e)
    if (e * 64 + lane < kD) A.out[b * A.o_row + head * A.o_head + e * 64 + lane] = (T)(l != 0.f ? o[e] / l : 0.f);
}
#endif  // DISC_CACHE
