// Host side of the operators around a decoder's attention (decoder_device.h): registration, the checks
// of a launch, its launch dimensions.  No allocation and no lookup on a launch that succeeds.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <new>
#include <stdexcept>

#include "disc_internal.hpp"

namespace disc {

extern const char* const kDecoderHeader;   // decoder_device.h, embedded at build time

namespace {

// ---- what the device code takes; the layouts mirror decoder_device.h -------------------------------
struct RotaryTensor {
  const void* x;
  void* y;
  int64_t x_token, x_head, y_token, y_head;
  int32_t heads, pad;
};
struct RotaryArgs {
  RotaryTensor t[DISC_ROTARY_TENSORS];
  const void* positions;
  int32_t n, position_bytes, backward, pad;
};
struct RowsArgs {
  const void* slots;
  const void *k, *v;
  const void *kp, *vp, *ks, *vs;
  int64_t k_token, k_head, v_token, v_head, tokens, slots_end;
  int32_t heads, shift;
};
struct AttendArgs {
  const void *q, *lengths, *table, *kp, *vp, *ks, *vs, *prefix_table;
  void* out;
  float *part, *part_m;
  int64_t q_row, q_head, o_row, o_head;
  int32_t batch, heads, kv_heads, group, pages, shift, width, tiles;
  int32_t target, parts, direct, join_ways, prefix_len, prefix_chunk, prefix_parts, prefix_tiles, prefix_inline;
};
constexpr int kMostPages = 1024;
constexpr int64_t kNonTemporalBytes = 64 << 20;   // from here on past the caches, as the fused patterns
constexpr int64_t kAttendStreamBytes = 128 << 20;
constexpr int kUnit = 128;              // tokens that a block's four wavefronts take at once
constexpr int64_t kDirectTokens = 512;  // sequences no longer than this are one chunk each (kDirectPages of the smallest size)
// A prefix no longer than this is gone through by every sequence's own block, where these run all at once: nothing is joined
// then (us, joined / in line, 8 heads, by the bytes of a row: 128 bytes 32 sequences of 100 behind 300 11.5 / 10.1, behind 500
// 11.6 / 10.9, but 90 of 64 behind 500 16.7 / 19.5; 256 bytes 32 of 100 behind 200 11.7 / 9.6, behind 500 12.0 / 11.8, 90 of 64
// 16.6 / 24.6; 512 bytes 20 of 100 behind 200 12.9 / 14.8).
constexpr int64_t inline_tokens(int64_t row_bytes) { return row_bytes <= 128 ? 512 : row_bytes <= 256 ? 256 : 0; }
// disc_attend_k has the prefix too, 16 query rows a block, up to so many of their units of 128 tokens: a launch less, but
// keys and values are read, and codes brought into the operands' form, once for 16 rows and not for 256 (us, there / in
// disc_prefix_k: 64 sequences of 32 and 8 heads x 128 behind 1000 tokens 19 / 30, behind 4000 30 / 40, 16000 61 / 52 of
// 8-bit rows, 21 / 28, 38 / 38 and 88 / 58 of 16-bit ones, which take two products where codes take one).
constexpr int64_t kFewUnits8 = 6144, kFewUnits16 = 4096;

enum { FN_ROTARY = 0, FN_ROTARY_NT, FN_ROTARY_COUNT };
enum { FN_STORE = 0, FN_STORE_NT, FN_LOAD, FN_LOAD_NT, FN_ATTEND, FN_ATTEND2, FN_ATTEND1, FN_ATTEND_NT, FN_PREFIX = FN_ATTEND_NT + 3, FN_JOIN, FN_CACHE_COUNT };

constexpr int64_t kMostElements = (int64_t)1 << 60;
constexpr int64_t kMostThreads = ((int64_t)1 << 32) - 1;     // of one launch, by axis; calls of more tokens are several launches

int refuse(disc_ctx* c, int code, const char* what) { return context_fail(c, code, what); }
int refuse(disc_ctx* c, int code, const char* what, long long got) {
  char buf[160];
  snprintf(buf, sizeof buf, "%s (got %lld)", what, got);
  return context_fail(c, code, buf);
}

// a * b of two sizes, or -1 where that is more than any memory holds
int64_t times(int64_t a, int64_t b) {
  if (a < 0 || b < 0) return -1;
  if (a == 0 || b == 0) return 0;
  return a > kMostElements / b ? -1 : a * b;
}

// rows [tokens][heads] of `d` elements: every stride is a size, and the extent fits
bool strides_ok(int64_t tokens, int64_t token, int64_t heads, int64_t head, int64_t d) {
  if (token < 0 || head < 0) return false;
  const int64_t a = times(tokens - 1, token), b = times(heads - 1, head);
  return a >= 0 && b >= 0 && a + b + d <= kMostElements;
}
// ... and no two of them overlap
bool rows_apart(int64_t tokens, int64_t token, int64_t heads, int64_t head, int64_t d) {
  if (tokens <= 1) return heads <= 1 || head >= d;
  if (heads <= 1) return token >= d;
  return (head >= d && token >= (heads - 1) * head + d) || (token >= d && head >= (tokens - 1) * token + d);
}
bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

Operator* get_operator(disc_ctx* c, int32_t id, Operator::Kind kind) {
  auto& all = *context_operators(c);
  if (id < 0 || id >= (int)all.size() || all[id]->kind != kind) return nullptr;
  return all[id].get();
}

// The context's device is the current one while kernels are enqueued (the default stream is the current device's).
struct OnDevice {
  int before = -1;
  bool ok = true;
  explicit OnDevice(int device) {
    int now = -1;
    ok = hipGetDevice(&now) == hipSuccess;
    if (ok && now != device) {
      ok = hipSetDevice(device) == hipSuccess;
      before = now;
    }
  }
  ~OnDevice() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

int enqueue(disc_ctx* c, void* fn, uint64_t blocks, uint32_t y, uint32_t threads, const void* args, size_t size, void* stream) {
  void* extra[] = {HIP_LAUNCH_PARAM_BUFFER_POINTER, const_cast<void*>(args), HIP_LAUNCH_PARAM_BUFFER_SIZE, &size, HIP_LAUNCH_PARAM_END};
  const hipError_t e = hipModuleLaunchKernel((hipFunction_t)fn, (uint32_t)blocks, y, 1, threads, 1, 1, 0, (hipStream_t)stream, nullptr, extra);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    char buf[128];
    snprintf(buf, sizeof buf, "hipModuleLaunchKernel: %s", hipGetErrorString(e));
    return context_fail(c, DISC_ERR_HIP, buf);
  }
  return DISC_OK;
}

// Compiles the operator and enters it, or finds the one that was made of the same description.  `measured`: the kernel
// whose blocks a CU are asked for.
int enter(disc_ctx* c, std::unique_ptr<Operator> o, const std::string& macros, const char* const* names, int n, int measured, int32_t* id_out) {
  auto& all = *context_operators(c);
  for (size_t i = 0; i < all.size(); ++i)
    if (all[i]->key == o->key) {
      *id_out = (int32_t)i;
      return DISC_OK;
    }
  std::vector<char> code;
  const int rc = context_compile(c, macros + kDecoderHeader, &code);
  if (rc) return rc;
  all.reserve(all.size() + 1);
  const int device = context_device(c);
  if (device >= 0) {
    OnDevice on(device);
    if (!on.ok) return refuse(c, DISC_ERR_HIP, "hipSetDevice failed");
    hipModule_t m = nullptr;
    if (hipModuleLoadData(&m, code.data()) != hipSuccess) {
      (void)hipGetLastError();
      return refuse(c, DISC_ERR_HIP, "hipModuleLoadData failed");
    }
    o->module = m;
    for (int i = 0; i < n; ++i) {
      hipFunction_t f = nullptr;
      if (hipModuleGetFunction(&f, m, names[i]) != hipSuccess) {
        (void)hipGetLastError();
        (void)hipModuleUnload(m);
        return refuse(c, DISC_ERR_HIP, "hipModuleGetFunction failed");
      }
      o->fn[i] = f;
    }
    int blocks = 0;
    if (hipModuleOccupancyMaxActiveBlocksPerMultiprocessor(&blocks, (hipFunction_t)o->fn[measured], 256, 0) == hipSuccess && blocks > 0)
      o->resident = blocks;
    else
      (void)hipGetLastError();
  }
  *id_out = (int32_t)all.size();
  all.push_back(std::move(o));
  return DISC_OK;
}

std::string text(const char* format, double x) {
  char buf[64];
  snprintf(buf, sizeof buf, format, x);
  return buf;
}

// ---- rotary positions ------------------------------------------------------------------------------

// accesses of one head, as the device code has them
int rotary_units(const Operator& o) {
  const auto accesses = [&](int n) {
    int w = 16 / dtype_bytes(o.dtype);
    while (n % w) w /= 2;
    return n / w;
  };
  return accesses(o.layout == DISC_ROTARY_INTERLEAVED ? o.rotary_dim : o.rotary_dim / 2) + accesses(o.head_dim - o.rotary_dim);
}

int register_rotary(disc_ctx* c, const disc_rotary_desc* d, int32_t* id_out) {
  if (!c) return DISC_ERR_INVALID_ARG;
  if (!d || !id_out || !d->frequencies) return refuse(c, DISC_ERR_INVALID_ARG, "null pointer");
  if (!is_float_dtype(d->dtype)) return refuse(c, DISC_ERR_INVALID_ARG, "rotary takes f32, f16 or bf16");
  if (d->head_dim < 2 || d->head_dim > 256) return refuse(c, DISC_ERR_SHAPE, "head_dim is 2 .. 256", d->head_dim);
  if (d->rotary_dim < 2 || d->rotary_dim > d->head_dim || d->rotary_dim % 2)
    return refuse(c, DISC_ERR_SHAPE, "rotary_dim is even, 2 .. head_dim", d->rotary_dim);
  if (d->layout != DISC_ROTARY_HALF && d->layout != DISC_ROTARY_INTERLEAVED) return refuse(c, DISC_ERR_INVALID_ARG, "bad rotary layout");
  if (!std::isfinite((float)d->magnitude)) return refuse(c, DISC_ERR_INVALID_ARG, "magnitude is no finite number of 32 bits");
  std::string macros = "#define DISC_ROTARY 1\n";
  macros += std::string("#define DISC_T ") + dtype_ctype(d->dtype) + "\n";
  macros += "#define DISC_D " + std::to_string(d->head_dim) + "\n#define DISC_R " + std::to_string(d->rotary_dim) + "\n";
  macros += "#define DISC_INTERLEAVED " + std::to_string(d->layout) + "\n#define DISC_MAGNITUDE " + text("%a", d->magnitude) + "\n";
  macros += "__device__ const double kTurns[DISC_R / 2] = {";
  for (int j = 0; j < d->rotary_dim / 2; ++j) {
    const double f = d->frequencies[j];
    if (!std::isfinite(f) || std::fabs(f) > 3.2) return refuse(c, DISC_ERR_INVALID_ARG, "a frequency is finite and at most half a turn a position");
    macros += text("%a,", f * 0.63661977236758134308);   // quarter turns: f / (pi / 2)
  }
  macros += "};\n";
  std::unique_ptr<Operator> o(new Operator);
  o->kind = Operator::ROTARY;
  o->key = macros;
  o->dtype = d->dtype;
  o->head_dim = d->head_dim;
  o->rotary_dim = d->rotary_dim;
  o->layout = d->layout;
  static const char* const names[] = {"disc_rotary_k", "disc_rotary_nt_k"};
  return enter(c, std::move(o), macros, names, FN_ROTARY_COUNT, FN_ROTARY, id_out);
}

int launch_rotary(disc_ctx* c, int32_t id, const int64_t* dims, int n_dims, const void* const* in, int n_in, void* const* out, int n_out,
                  void* stream) {
  if (!c) return DISC_ERR_INVALID_ARG;
  const Operator* o = get_operator(c, id, Operator::ROTARY);
  if (!o) return refuse(c, DISC_ERR_INVALID_ARG, "bad rotary id");
  if (!dims || !in || !out) return refuse(c, DISC_ERR_INVALID_ARG, "null pointer array");
  if (n_out < 1 || n_out > DISC_ROTARY_TENSORS || n_in != n_out + 1 || n_dims != 3 + 5 * n_out)
    return refuse(c, DISC_ERR_INVALID_ARG, "rotary takes positions and 1 .. 4 tensors, as many results, and 3 + 5 dims a tensor");
  RotaryArgs a;
  memset(&a, 0, sizeof a);
  const int64_t tokens = dims[0];
  a.position_bytes = dims[1] == 8 ? 8 : 4;
  a.backward = dims[2] != 0;
  a.n = n_out;
  if (tokens < 0 || tokens >= (int64_t)1 << 31) return refuse(c, DISC_ERR_SHAPE, "tokens is 0 .. 2^31 - 1", tokens);
  if (dims[1] != 4 && dims[1] != 8) return refuse(c, DISC_ERR_INVALID_ARG, "positions have 4 or 8 bytes", dims[1]);
  const int size = dtype_bytes(o->dtype);
  int64_t most = 0, moved = 0;
  for (int k = 0; k < n_out; ++k) {
    const int64_t* s = dims + 3 + 5 * k;
    if (s[0] < 0 || s[0] > 1 << 20) return refuse(c, DISC_ERR_SHAPE, "heads is 0 .. 2^20", s[0]);
    if (tokens > 0 && s[0] > 0) {
      if (!strides_ok(tokens, s[1], s[0], s[2], o->head_dim) || !strides_ok(tokens, s[3], s[0], s[4], o->head_dim))
        return refuse(c, DISC_ERR_SHAPE, "a stride is negative or an extent overflows");
      if (!rows_apart(tokens, s[3], s[0], s[4], o->head_dim)) return refuse(c, DISC_ERR_SHAPE, "rows of a result overlap");
      if (!in[1 + k] || !out[k]) return refuse(c, DISC_ERR_INVALID_ARG, "null tensor pointer");
      if (!aligned(in[1 + k], size) || !aligned(out[k], size)) return refuse(c, DISC_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
      if (in[1 + k] == out[k] && ((tokens > 1 && s[1] != s[3]) || (s[0] > 1 && s[2] != s[4])))
        return refuse(c, DISC_ERR_INVALID_ARG, "in place, both sides have the same strides");
    }
    a.t[k] = {in[1 + k], out[k], s[1], s[2], s[3], s[4], (int32_t)s[0], 0};
    most = most > s[0] ? most : s[0];
    moved += tokens * s[0] * o->head_dim;   // (2^59 at most)
  }
  if (tokens == 0 || most == 0) return context_device(c) < 0 ? refuse(c, DISC_ERR_INVALID_ARG, "host-only context cannot launch") : DISC_OK;
  if (!in[0] || !aligned(in[0], a.position_bytes)) return refuse(c, DISC_ERR_INVALID_ARG, "positions: null or not aligned");
  a.positions = in[0];
  if (context_device(c) < 0) return refuse(c, DISC_ERR_INVALID_ARG, "host-only context cannot launch");
  // A token a block; where they are few, the heads are shared out too, one pass of a block's rows each.
  const int64_t rows = 256 / rotary_units(*o), passes = (most + rows - 1) / rows;
  const uint32_t y = tokens * 2 <= context_cus(c) ? (uint32_t)(passes < 64 ? passes : 64) : 1;
  const bool nt = moved >= kNonTemporalBytes / (2 * size);
  OnDevice on(context_device(c));
  if (!on.ok) return refuse(c, DISC_ERR_HIP, "hipSetDevice failed");
  int rc = DISC_OK, n = 0;
  for (int64_t left = tokens; rc == DISC_OK && left > 0; ++n) {
    const int64_t now = std::min(left, kMostThreads / 256);
    rc = enqueue(c, o->fn[nt ? FN_ROTARY_NT : FN_ROTARY], (uint64_t)now, y, 256, &a, sizeof a, stream);
    left -= now;
    a.positions = (const char*)a.positions + now * a.position_bytes;
    for (int k = 0; k < a.n; ++k) {
      if (a.t[k].heads == 0) continue;
      a.t[k].x = (const char*)a.t[k].x + now * a.t[k].x_token * size;
      a.t[k].y = (char*)a.t[k].y + now * a.t[k].y_token * size;
    }
  }
  if (rc == DISC_OK) context_count(c, n);
  return rc;
}

// ---- the cache -------------------------------------------------------------------------------------

int register_cache(disc_ctx* c, const disc_cache_desc* d, int32_t* id_out) {
  if (!c) return DISC_ERR_INVALID_ARG;
  if (!d || !id_out) return refuse(c, DISC_ERR_INVALID_ARG, "null pointer");
  if (d->dtype != DISC_F16 && d->dtype != DISC_BF16) return refuse(c, DISC_ERR_INVALID_ARG, "a cache takes f16 or bf16 rows");
  if (d->storage < DISC_STORAGE_SAME || d->storage > DISC_STORAGE_E4M3) return refuse(c, DISC_ERR_INVALID_ARG, "bad storage");
  if (d->head_dim < 16 || d->head_dim > 256 || d->head_dim % 16) return refuse(c, DISC_ERR_SHAPE, "head_dim is a multiple of 16, 16 .. 256", d->head_dim);
  // (times 512 for fp16 queries over i8: what undoes the size of its codes in half precision)
  if (!std::isfinite((float)(d->softmax_scale * 1.44269504088896340736 * (d->dtype == DISC_F16 && d->storage == DISC_STORAGE_I8 ? 512.0 : 1.0))))
    return refuse(c, DISC_ERR_INVALID_ARG, "softmax_scale is no finite number of 32 bits");
  const double scale = d->softmax_scale != 0.0 ? d->softmax_scale : 1.0 / std::sqrt((double)d->head_dim);
  std::string macros = "#define DISC_CACHE 1\n#define DISC_T_F16 " + std::to_string(d->dtype == DISC_F16 ? 1 : 0) + "\n";
  macros += "#define DISC_STORAGE " + std::to_string(d->storage) + "\n#define DISC_D " + std::to_string(d->head_dim) + "\n";
  macros += "#define DISC_SCALE_LOG2E " + text("%a", scale * 1.44269504088896340736) + "\n";
  std::unique_ptr<Operator> o(new Operator);
  o->kind = Operator::CACHE;
  o->key = macros;
  o->dtype = d->dtype;
  o->storage = d->storage;
  o->head_dim = d->head_dim;
  static const char* const names[] = {"disc_store_k", "disc_store_nt_k", "disc_load_k", "disc_load_nt_k", "disc_attend_k", "disc_attend2_k", "disc_attend1_k",
                                      "disc_attend_nt_k", "disc_attend2_nt_k", "disc_attend1_nt_k", "disc_prefix_k", "disc_join_k"};
  return enter(c, std::move(o), macros, names, FN_CACHE_COUNT, FN_ATTEND, id_out);
}

// page_size = 1 << shift; -1: no page size
int page_shift(int64_t page_size) {
  for (int s = 3; s <= 16; ++s)
    if (page_size == (int64_t)1 << s) return s;
  return -1;
}

int check_pages(disc_ctx* c, const Operator& o, int64_t heads, int64_t pages, int64_t page_size, int* shift) {
  if (heads < 1 || heads > 1 << 16) return refuse(c, DISC_ERR_SHAPE, "kv_heads is 1 .. 65536", heads);
  *shift = page_shift(page_size);
  if (*shift < 0) return refuse(c, DISC_ERR_SHAPE, "page_size is a power of two, 8 .. 65536", page_size);
  if (pages < 1 || pages >= (int64_t)1 << 31) return refuse(c, DISC_ERR_SHAPE, "pages is 1 .. 2^31 - 1", pages);
  const int64_t rows = times(times(pages, heads), page_size);
  if (rows < 0 || times(rows, o.head_dim) < 0) return refuse(c, DISC_ERR_SHAPE, "the pages are larger than any memory");
  return DISC_OK;
}

int launch_rows(disc_ctx* c, int32_t id, const int64_t* dims, int n_dims, const void* const* in, int n_in, void* const* out, int n_out,
                void* stream, bool store) {
  if (!c) return DISC_ERR_INVALID_ARG;
  const Operator* o = get_operator(c, id, Operator::CACHE);
  if (!o) return refuse(c, DISC_ERR_INVALID_ARG, "bad cache id");
  if (!dims || !in || !out) return refuse(c, DISC_ERR_INVALID_ARG, "null pointer array");
  const bool scaled = o->storage != DISC_STORAGE_SAME;
  const int n_pages = scaled ? 4 : 2;
  if (n_dims != 8 || n_in != (store ? 3 : 1 + n_pages) || n_out != (store ? n_pages : 2))
    return refuse(c, DISC_ERR_INVALID_ARG, "a store or load takes 8 dims, slots, keys and values, the pages and with 8-bit storage their scales");
  RowsArgs a;
  memset(&a, 0, sizeof a);
  a.tokens = dims[0];
  if (a.tokens < 0 || a.tokens >= (int64_t)1 << 31) return refuse(c, DISC_ERR_SHAPE, "tokens is 0 .. 2^31 - 1", a.tokens);
  int shift = 0;
  if (const int rc = check_pages(c, *o, dims[1], dims[2], dims[3], &shift)) return rc;
  a.heads = (int32_t)dims[1];
  a.shift = shift;
  a.slots_end = dims[2] << shift;
  a.k_token = dims[4];
  a.k_head = dims[5];
  a.v_token = dims[6];
  a.v_head = dims[7];
  if (a.tokens == 0) return context_device(c) < 0 ? refuse(c, DISC_ERR_INVALID_ARG, "host-only context cannot launch") : DISC_OK;
  if (!strides_ok(a.tokens, a.k_token, a.heads, a.k_head, o->head_dim) || !strides_ok(a.tokens, a.v_token, a.heads, a.v_head, o->head_dim))
    return refuse(c, DISC_ERR_SHAPE, "a stride is negative or an extent overflows");
  if (!store && (!rows_apart(a.tokens, a.k_token, a.heads, a.k_head, o->head_dim) || !rows_apart(a.tokens, a.v_token, a.heads, a.v_head, o->head_dim)))
    return refuse(c, DISC_ERR_SHAPE, "rows of a result overlap");
  a.slots = in[0];
  a.k = store ? in[1] : out[0];
  a.v = store ? in[2] : out[1];
  const void* pages[4] = {nullptr, nullptr, nullptr, nullptr};
  for (int i = 0; i < n_pages; ++i) {
    pages[i] = store ? out[i] : in[1 + i];
    if (!pages[i] || !aligned(pages[i], 16)) return refuse(c, DISC_ERR_INVALID_ARG, "pages or scales: null or not 16-byte aligned");
  }
  a.kp = pages[0];
  a.vp = pages[1];
  a.ks = pages[2];
  a.vs = pages[3];
  if (!a.slots || !aligned(a.slots, 8)) return refuse(c, DISC_ERR_INVALID_ARG, "slots: null or not 8-byte aligned");
  if (!a.k || !a.v || !aligned(a.k, 2) || !aligned(a.v, 2)) return refuse(c, DISC_ERR_INVALID_ARG, "keys or values: null or not aligned to their elements");
  int lanes = 2;
  while (lanes * 8 < o->head_dim) lanes *= 2;
  if (context_device(c) < 0) return refuse(c, DISC_ERR_INVALID_ARG, "host-only context cannot launch");
  OnDevice on(context_device(c));
  if (!on.ok) return refuse(c, DISC_ERR_HIP, "hipSetDevice failed");
  const bool nt = times(a.tokens, a.heads) * o->head_dim * (2 + (scaled ? 1 : 2)) * 2 >= kNonTemporalBytes;
  const int64_t each = kMostThreads / 256 * 256 / ((int64_t)a.heads * lanes);   // tokens of a launch (2047 at least)
  int rc = DISC_OK, n = 0;
  for (int64_t left = a.tokens; rc == DISC_OK && left > 0; ++n) {
    a.tokens = std::min(left, each);
    rc = enqueue(c, o->fn[(store ? FN_STORE : FN_LOAD) + (nt ? 1 : 0)], (uint64_t)((a.tokens * a.heads * lanes + 255) / 256), 1, 256, &a, sizeof a, stream);
    left -= a.tokens;
    a.slots = (const int64_t*)a.slots + a.tokens;
    a.k = (const char*)a.k + a.tokens * a.k_token * 2;
    a.v = (const char*)a.v + a.tokens * a.v_token * 2;
  }
  if (rc == DISC_OK) context_count(c, n);
  return rc;
}

// The sizes of an attention call: its chunks, its rows of partial results.  (Pure host.)
struct AttendPlan {
  AttendArgs a;
  int64_t attend_blocks, prefix_blocks, join_blocks;
  int ways;                 // wavefronts of a sequence
  bool nt;
  size_t workspace, reserve;   // bytes that this call takes, and that any of a smaller batch, prefix or table does
};

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Rows of query tokens that a block of a prefix has (`few`: in disc_attend_k), and blocks that are there at once.
struct PrefixBlocks {
  int64_t rows, slots;
  PrefixBlocks(const Operator& o, int64_t cus, bool few) : rows(few ? 16 : o.head_dim <= 128 ? 256 : 128), slots((few ? o.resident : 1) * cus) {}
};
// Rounds of them that a chunk of the prefix may be made for: those that one chunk takes, or one more, three at most.
int64_t most_rounds(int64_t blocks, int64_t slots) { return std::min<int64_t>(3, ceil_div(blocks, slots) + 1); }

// `one_chunk`: every sequence of up to kDirectTokens is one chunk, whatever is faster (it takes less workspace).
int plan_attend(disc_ctx* c, const Operator& o, const int64_t* d, int n_dims, bool one_chunk, AttendPlan* p) {
  if (!d || n_dims != 12) return refuse(c, DISC_ERR_INVALID_ARG, "an attention call takes 12 dims");
  AttendArgs& a = p->a;
  memset(&a, 0, sizeof a);
  const int64_t batch = d[0], heads = d[1], kv = d[2], width = d[5], prefix = d[6], prefix_width = d[7];
  int shift = 0;
  if (const int rc = check_pages(c, o, kv, d[3], d[4], &shift)) return rc;
  if (times(times(d[3], kv), d[4]) >= (int64_t)1 << 32) return refuse(c, DISC_ERR_SHAPE, "attention counts rows of a cache in 32 bits", d[3]);
  if (batch < 0 || batch > 1 << 20) return refuse(c, DISC_ERR_SHAPE, "batch is 0 .. 2^20", batch);
  if (heads < kv || heads % kv || heads > 1 << 20) return refuse(c, DISC_ERR_SHAPE, "q_heads is a multiple of kv_heads, at most 2^20", heads);
  if (width < 0 || times(width, d[4]) < 0 || times(width, d[4]) > (int64_t)1 << 30)
    return refuse(c, DISC_ERR_SHAPE, "table_width * page_size is 0 .. 2^30", width);
  if (prefix < 0 || prefix > (int64_t)1 << 30) return refuse(c, DISC_ERR_SHAPE, "prefix_length is 0 .. 2^30", prefix);
  if (prefix_width < ceil_div(prefix, d[4])) return refuse(c, DISC_ERR_SHAPE, "the prefix's table is shorter than the prefix", prefix_width);
  a.batch = (int32_t)batch;
  a.heads = (int32_t)heads;
  a.kv_heads = (int32_t)kv;
  a.group = (int32_t)(heads / kv);
  a.pages = (int32_t)d[3];
  a.shift = shift;
  a.width = (int32_t)width;
  a.tiles = (int32_t)ceil_div(a.group, 16);
  a.prefix_len = (int32_t)prefix;
  const int64_t cus = context_cus(c), per = kv * a.tiles;
  // Sequences' own tokens: as many blocks as run at once share all of them, so that they end together whatever the
  // lengths are.
  const int64_t at_once = cus * o.resident;
  a.target = (int32_t)(at_once / per > 1 ? at_once / per : 1);
  int64_t parts = batch + a.target;
  // (16-bit rows above 128: where the blocks are few, two steps more cost more than the join, 8 or 16 blocks of 500 tokens x
  // 256 14.4 us joined / 16.0 as one chunk each, 120 20.0 / 18.3; 8-bit ones 14.2 / 12.8, 18.0 / 13.7)
  const int64_t direct_tokens = o.head_dim <= 128 || o.storage != DISC_STORAGE_SAME || times(batch, per) >= cus / 4 || one_chunk ? kDirectTokens : kDirectTokens / 2;
  if ((width << shift) <= direct_tokens) {
    a.direct = 1;
    parts = batch;
  }
  a.prefix_inline = prefix > 0 && a.direct && prefix <= inline_tokens(o.head_dim * (o.storage != DISC_STORAGE_SAME ? 1 : 2)) && times(batch, per) <= at_once;
  // Keys and values go past the caches where they are more than those keep until the next step, and one block reads
  // them (us, through them / past them, four caches in turn: i8 549 MB 108 / 101, 230 55 / 54, 137 40 / 40, 70 30 / 32; bf16
  // 553 MB 110 / 98, 234 56 / 52, 141 42 / 40, 74 18 / 20).  By what the tables and the pages hold: the lengths are the device's.
  const int64_t own = times(std::min(d[3], times(batch, width)) << shift, kv * 2 * o.head_dim * (o.storage != DISC_STORAGE_SAME ? 1 : 2));
  p->nt = a.tiles == 1 && !a.prefix_inline && (own < 0 || own >= kAttendStreamBytes);
  const int64_t rows = batch * a.group;
  int64_t prefix_blocks = 0;
  if (prefix > 0 && batch > 0 && !a.prefix_inline) {
    const int64_t units = ceil_div(prefix, kUnit), tile_units = times(times(ceil_div(rows, 16), units), kv);
    const bool few = tile_units >= 0 && tile_units <= (o.storage != DISC_STORAGE_SAME ? kFewUnits8 : kFewUnits16);
    const PrefixBlocks at(o, cus, few);
    const int64_t row_blocks = ceil_div(rows, at.rows), slots = at.slots;
    // Chunks of the prefix: as many as make the shortest run, in rounds of the blocks that are there at once times the
    // units of a chunk and a block's own cost of about four.
    // (Of the rounds that one chunk takes, or one more, the most chunks that fit; nothing is gained where those are many.)
    const int64_t blocks = kv * row_blocks, rounds = ceil_div(blocks, slots);
    int64_t units_each = units, best = rounds * (units + 4);
    for (int64_t r = rounds; r <= most_rounds(blocks, slots); ++r) {
      const int64_t each = ceil_div(units, std::min(units, r * slots / blocks)), cost = r * (each + 4);
      if (cost < best) best = cost, units_each = each;
    }
    int64_t chunk = units_each * kUnit;
    const int64_t most = (int64_t)kMostPages << shift;
    chunk = chunk > most ? most : chunk;
    a.prefix_chunk = (int32_t)chunk;
    a.prefix_parts = (int32_t)ceil_div(prefix, chunk);
    prefix_blocks = times(a.prefix_parts, blocks);
    if (few) a.prefix_tiles = (int32_t)row_blocks;
  }
  if (parts >= (int64_t)1 << 31) return refuse(c, DISC_ERR_SHAPE, "too many chunks for one call");
  const bool alone = a.direct && (prefix == 0 || a.prefix_inline);   // every chunk's block writes the result itself
  p->attend_blocks = times(a.direct ? batch : a.target, per);
  p->ways = 4;
  if (a.direct && a.prefix_tiles == 0) {
    // Short sequences: four wavefronts each while all of them run at once, else two, else one.
    if (p->attend_blocks > 2 * at_once)
      p->ways = 1;
    else if (p->attend_blocks > at_once)
      p->ways = 2;
    if (p->attend_blocks > 0) p->attend_blocks = ceil_div(p->attend_blocks, 4 / p->ways);
  }
  a.parts = (int32_t)(parts = alone ? 0 : parts);
  if (p->attend_blocks >= 0 && a.prefix_tiles) {
    p->attend_blocks += prefix_blocks;
    prefix_blocks = 0;
  }
  p->prefix_blocks = prefix_blocks;
  // A block a row where there are few rows to join, so that their chunks, which are many then, are read by four wavefronts.
  a.join_ways = times(batch, heads) <= 4 * cus ? 4 : 1;
  p->join_blocks = alone ? 0 : ceil_div(times(batch, heads), 4 / a.join_ways);
  const int64_t partial = times(parts, heads) + times(a.prefix_parts, times(batch, heads));
  if (times(batch, heads) >= (int64_t)1 << 31 || p->attend_blocks < 0 || p->prefix_blocks < 0 || p->attend_blocks > kMostThreads / 256 ||
      p->prefix_blocks > kMostThreads / 512 || p->join_blocks > kMostThreads / 256 || times(partial, 4 * 256 + 8) < 0)
    return refuse(c, DISC_ERR_SHAPE, "too many rows for one call");
  const size_t row = (size_t)o.head_dim * 4 + 8;
  p->workspace = batch > 0 ? (size_t)partial * row : 0;
  // Fewer query rows make more chunks of a prefix, so that a smaller call may take more than this one does.  What none
  // takes more than: a chunk for every unit; and the rows of as many blocks as the chunks are made for, or where those are
  // fewer than one chunk's, one, or as many as the pages of a chunk ask for.
  int64_t chunks = a.direct ? (alone ? 0 : batch) : batch + a.target;
  if (prefix > 0 && !a.prefix_inline) {
    int64_t most = 0;
    for (const bool few : {false, true}) {
      const PrefixBlocks at(o, cus, few);
      most = std::max(most, most_rounds(kv * ceil_div(rows, at.rows), at.slots) * at.slots * at.rows / heads);
    }
    chunks += std::max(std::min(most, times(batch, ceil_div(prefix, kUnit))), times(batch, ceil_div(prefix, (int64_t)kMostPages << shift)));
  }
  p->reserve = batch > 0 ? std::max(p->workspace, (size_t)(chunks * heads) * row) : 0;
  return DISC_OK;
}

int launch_attend(disc_ctx* c, int32_t id, const int64_t* dims, int n_dims, const void* const* in, int n_in, void* const* out, int n_out,
                  void* workspace, size_t workspace_bytes, void* stream) {
  if (!c) return DISC_ERR_INVALID_ARG;
  const Operator* o = get_operator(c, id, Operator::CACHE);
  if (!o) return refuse(c, DISC_ERR_INVALID_ARG, "bad cache id");
  if (!dims || !in || !out) return refuse(c, DISC_ERR_INVALID_ARG, "null pointer array");
  AttendPlan p;
  if (const int rc = plan_attend(c, *o, dims, n_dims, false, &p)) return rc;
  // (a workspace asked for at a larger batch, where sequences are one chunk each, does not hold the chunks of this one)
  if (p.workspace > workspace_bytes && !p.a.direct)
    if (const int rc = plan_attend(c, *o, dims, n_dims, true, &p)) return rc;
  AttendArgs& a = p.a;
  const bool scaled = o->storage != DISC_STORAGE_SAME;
  const int want = 5 + (scaled ? 2 : 0) + (a.prefix_len > 0 ? 1 : 0);
  if (n_in != want || n_out != 1)
    return refuse(c, DISC_ERR_INVALID_ARG, "an attention call takes q, lengths, table, the pages, with 8-bit storage their scales, with a prefix its table, and one result");
  a.q_row = dims[8];
  a.q_head = dims[9];
  a.o_row = dims[10];
  a.o_head = dims[11];
  if (a.batch == 0) return context_device(c) < 0 ? refuse(c, DISC_ERR_INVALID_ARG, "host-only context cannot launch") : DISC_OK;
  if (!strides_ok(a.batch, a.q_row, a.heads, a.q_head, o->head_dim) || !strides_ok(a.batch, a.o_row, a.heads, a.o_head, o->head_dim))
    return refuse(c, DISC_ERR_SHAPE, "a stride is negative or an extent overflows");
  if (!rows_apart(a.batch, a.o_row, a.heads, a.o_head, o->head_dim)) return refuse(c, DISC_ERR_SHAPE, "rows of a result overlap");
  a.q = in[0];
  a.lengths = in[1];
  a.table = in[2];
  a.kp = in[3];
  a.vp = in[4];
  a.ks = scaled ? in[5] : nullptr;
  a.vs = scaled ? in[6] : nullptr;
  a.prefix_table = a.prefix_len > 0 ? in[n_in - 1] : nullptr;
  a.out = out[0];
  if (!a.q || !a.out || !aligned(a.q, 2) || !aligned(a.out, 2)) return refuse(c, DISC_ERR_INVALID_ARG, "q or out: null or not aligned to its elements");
  if (!a.lengths || !aligned(a.lengths, 4) || (a.width > 0 && !a.table) || !aligned(a.table, 4) || (a.prefix_len > 0 && !a.prefix_table) ||
      !aligned(a.prefix_table, 4))
    return refuse(c, DISC_ERR_INVALID_ARG, "lengths or a table: null or not 4-byte aligned");
  if (!a.kp || !a.vp || !aligned(a.kp, 16) || !aligned(a.vp, 16) || (scaled && (!a.ks || !a.vs)) || !aligned(a.ks, 16) || !aligned(a.vs, 16))
    return refuse(c, DISC_ERR_INVALID_ARG, "pages or scales: null or not 16-byte aligned");
  if (p.workspace > 0 && (!workspace || workspace_bytes < p.workspace)) return refuse(c, DISC_ERR_WORKSPACE, "workspace missing or too small");
  if (!aligned(workspace, 16)) return refuse(c, DISC_ERR_INVALID_ARG, "the workspace is not 16-byte aligned");
  a.part = (float*)workspace;
  const int64_t partial = (int64_t)a.parts * a.heads + (int64_t)a.prefix_parts * a.batch * a.heads;
  a.part_m = a.part + partial * o->head_dim;
  if (context_device(c) < 0) return refuse(c, DISC_ERR_INVALID_ARG, "host-only context cannot launch");
  OnDevice on(context_device(c));
  if (!on.ok) return refuse(c, DISC_ERR_HIP, "hipSetDevice failed");
  int rc = DISC_OK, n = 0;
  if (p.prefix_blocks > 0) {
    rc = enqueue(c, o->fn[FN_PREFIX], (uint64_t)p.prefix_blocks, 1, 512, &a, sizeof a, stream);
    ++n;
  }
  if (rc == DISC_OK && p.attend_blocks > 0) {
    rc = enqueue(c, o->fn[(p.ways == 4 ? FN_ATTEND : p.ways == 2 ? FN_ATTEND2 : FN_ATTEND1) + (p.nt ? FN_ATTEND_NT - FN_ATTEND : 0)], (uint64_t)p.attend_blocks, 1, 256, &a, sizeof a, stream);
    ++n;
  }
  if (rc == DISC_OK && p.join_blocks > 0) {
    rc = enqueue(c, o->fn[FN_JOIN], (uint64_t)p.join_blocks, 1, 256, &a, sizeof a, stream);
    ++n;
  }
  if (rc == DISC_OK) context_count(c, n);
  return rc;
}

int fail_inside(disc_ctx* c, const char* what) noexcept {
  char buf[160];
  snprintf(buf, sizeof buf, "internal error: %s", what);
  if (c) context_fail(c, DISC_ERR_INTERNAL, buf);
  return DISC_ERR_INTERNAL;
}

// Nothing leaves a C function by exception.
template <class F>
int guarded(disc_ctx* c, F f) noexcept {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return fail_inside(c, "out of host memory");
  } catch (const std::exception& e) {
    return fail_inside(c, e.what());
  } catch (...) {
    return fail_inside(c, "unknown exception");
  }
}

}  // namespace
}  // namespace disc

using namespace disc;

extern "C" {

int disc_register_rotary(disc_ctx* ctx, const disc_rotary_desc* desc, int32_t* id_out) {
  return guarded(ctx, [&] { return register_rotary(ctx, desc, id_out); });
}
int disc_register_cache(disc_ctx* ctx, const disc_cache_desc* desc, int32_t* id_out) {
  return guarded(ctx, [&] { return register_cache(ctx, desc, id_out); });
}
int disc_rotary(disc_ctx* ctx, int32_t id, const int64_t* dims, int n_dims, const void* const* inputs, int n_in, void* const* outputs, int n_out,
                void*, size_t, void* hip_stream) {
  return guarded(ctx, [&] { return launch_rotary(ctx, id, dims, n_dims, inputs, n_in, outputs, n_out, hip_stream); });
}
int disc_cache_store(disc_ctx* ctx, int32_t id, const int64_t* dims, int n_dims, const void* const* inputs, int n_in, void* const* outputs,
                     int n_out, void*, size_t, void* hip_stream) {
  return guarded(ctx, [&] { return launch_rows(ctx, id, dims, n_dims, inputs, n_in, outputs, n_out, hip_stream, true); });
}
int disc_cache_load(disc_ctx* ctx, int32_t id, const int64_t* dims, int n_dims, const void* const* inputs, int n_in, void* const* outputs,
                    int n_out, void*, size_t, void* hip_stream) {
  return guarded(ctx, [&] { return launch_rows(ctx, id, dims, n_dims, inputs, n_in, outputs, n_out, hip_stream, false); });
}
int disc_cache_attend(disc_ctx* ctx, int32_t id, const int64_t* dims, int n_dims, const void* const* inputs, int n_in, void* const* outputs,
                      int n_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return guarded(ctx, [&] { return launch_attend(ctx, id, dims, n_dims, inputs, n_in, outputs, n_out, workspace, workspace_bytes, hip_stream); });
}
int disc_cache_workspace_bytes(disc_ctx* ctx, int32_t id, const int64_t* dims, int n_dims, size_t* out) {
  return guarded(ctx, [&] {
    if (!ctx || !out) return (int)DISC_ERR_INVALID_ARG;
    const Operator* o = get_operator(ctx, id, Operator::CACHE);
    if (!o) return refuse(ctx, DISC_ERR_INVALID_ARG, "bad cache id");
    AttendPlan p;
    const int rc = plan_attend(ctx, *o, dims, n_dims, false, &p);
    if (rc == DISC_OK) *out = p.reserve;
    return rc;
  });
}

}  // extern "C"
