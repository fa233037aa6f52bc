// Host side of what a decoder's step runs around its attention (step_device.h): a norm into 8-bit rows and its gradient,
// products with 4-bit weights, the check of drafted tokens.  Registration, the checks of a launch, its launch dimensions.
// No allocation and no lookup on a launch that succeeds.
#include "operators.hpp"

namespace disc {

extern const char* const kStepHeader;   // step_device.h, embedded at build time

namespace {

// ---- what the device code takes; the layouts mirror step_device.h ----------------------------------
struct NormArgs {
  const void *x, *residual, *weight;
  void *total, *codes, *scales;
  int64_t x_row, residual_row, total_row, codes_row, rows;
  int32_t width, lanes;
};
struct NormBackwardArgs {
  const void *total, *weight, *dy, *dtotal;
  void *dx, *dweight;
  float* part;
  int64_t total_row, dy_row, dtotal_row, dx_row, rows;
  int32_t width, lanes, parts, pad;
};
struct LinearArgs {
  const void *x, *weights, *scales, *row_scales, *zeros, *bias;
  void* out;
  int64_t x_row, out_row;
  int32_t rows, n, k, groups;
};
struct VerifyArgs {
  const void *target, *draft, *drafted, *lengths, *uniforms;
  void *tokens, *accepted, *part;
  int64_t target_batch, target_row, draft_batch, draft_row;
  int32_t batch, drafts, vocabulary, chunks;
};

// the kernels of 1, 2, 4 and 8 accesses a thread, each through the caches and past them
enum { FN_NORM = 0, FN_NORM_BACKWARD = 8, FN_NORM_JOIN = 16, FN_NORM_COUNT };
enum { FN_LINEAR1 = 0, FN_LINEAR2, FN_LINEAR4, FN_LINEAR_COUNT };
enum { FN_VERIFY_SUM = 0, FN_VERIFY_PICK, FN_VERIFY_COUNT };

constexpr int64_t kMostRows = ((int64_t)1 << 31) - 1;
constexpr int kVerifyChunk = 4096;   // step_device.h's kChunk

int on_host(disc_ctx* c) { return refuse(c, DISC_ERR_INVALID_ARG, "host-only context cannot launch"); }

// rows of `width` elements, `stride` apart: the extent fits
bool extent_ok(int64_t rows, int64_t stride, int64_t width) { return strides_ok(rows, stride, 1, 0, width); }
bool apart(int64_t rows, int64_t stride, int64_t width) { return rows <= 1 || stride >= width; }

int64_t power_of_two(int64_t n) {   // the next one
  int64_t p = 1;
  while (p < n) p *= 2;
  return p;
}
int log2_of(int64_t p) {
  int k = 0;
  while (p >> (k + 1)) ++k;
  return k;
}

// ---- norm ------------------------------------------------------------------------------------------

int register_norm(disc_ctx* c, const disc_norm_desc* d, int32_t* id_out) {
  if (!c) return DISC_ERR_INVALID_ARG;
  if (!d || !id_out) return refuse(c, DISC_ERR_INVALID_ARG, "null pointer");
  if (!is_float_dtype(d->dtype)) return refuse(c, DISC_ERR_INVALID_ARG, "a norm takes f32, f16 or bf16");
  if (d->storage != DISC_STORAGE_I8 && d->storage != DISC_STORAGE_E4M3) return refuse(c, DISC_ERR_INVALID_ARG, "a norm's rows are stored as i8 or e4m3");
  if (!(d->eps > 0.0) || !std::isfinite((float)d->eps) || (float)d->eps == 0.f) return refuse(c, DISC_ERR_INVALID_ARG, "eps is a positive number of 32 bits");
  if (!std::isfinite((float)d->weight_offset)) return refuse(c, DISC_ERR_INVALID_ARG, "weight_offset is no finite number of 32 bits");
  std::string macros = std::string("#define DISC_NORM 1\n#define DISC_T ") + dtype_ctype(d->dtype) + "\n#define DISC_STORAGE " + std::to_string(d->storage) + "\n";
  macros += "#define DISC_EPS " + text("%a", d->eps) + "\n#define DISC_OFFSET " + text("%a", d->weight_offset) + "\n";
  std::unique_ptr<Operator> o(new Operator);
  o->kind = Operator::NORM;
  o->key = macros;
  o->dtype = d->dtype;
  o->storage = d->storage;
  static const char* const names[] = {"disc_norm1_k",          "disc_norm1_nt_k",          "disc_norm2_k",          "disc_norm2_nt_k",
                                      "disc_norm4_k",          "disc_norm4_nt_k",          "disc_norm8_k",          "disc_norm8_nt_k",
                                      "disc_norm_backward1_k", "disc_norm_backward1_nt_k", "disc_norm_backward2_k", "disc_norm_backward2_nt_k",
                                      "disc_norm_backward4_k", "disc_norm_backward4_nt_k", "disc_norm_backward8_k", "disc_norm_backward8_nt_k",
                                      "disc_norm_join_k"};
  return enter(c, std::move(o), macros, kStepHeader, names, FN_NORM_COUNT, FN_NORM, id_out);
}

// Threads of a row and accesses of a thread.
struct RowShape {
  int lanes, each, block;
  RowShape(const Operator& o, int64_t width, int most_lanes, bool wide) {
    const int64_t accesses = ceil_div(width * dtype_bytes(o.dtype), 16);
    const int64_t want = wide ? most_lanes : 256;
    int64_t l = std::max<int64_t>(8, std::min(power_of_two(accesses), want));
    int64_t n = power_of_two(ceil_div(accesses, l));
    while (n > 4 && l < most_lanes) {
      l *= 2;
      n /= 2;
    }
    lanes = (int)l;
    each = (int)n;
    block = lanes > 256 ? lanes : 256;
  }
};
constexpr int kNormLanes = 1024, kBackwardLanes = 512;

int check_rows(disc_ctx* c, const Operator& o, int64_t rows, int64_t width) {
  if (rows < 0 || rows > kMostRows) return refuse(c, DISC_ERR_SHAPE, "rows is 0 .. 2^31 - 1", rows);
  const int64_t most = 512 * 8 * 16 / dtype_bytes(o.dtype);
  if (width < 1 || width > most) return refuse(c, DISC_ERR_SHAPE, "width is 1 .. 32768, 16384 of fp32", width);
  return DISC_OK;
}

int launch_norm(disc_ctx* c, int32_t id, const int64_t* dims, int n_dims, const void* const* in, int n_in, void* const* out, int n_out, void* stream) {
  if (!c) return DISC_ERR_INVALID_ARG;
  const Operator* o = get_operator(c, id, Operator::NORM);
  if (!o) return refuse(c, DISC_ERR_INVALID_ARG, "bad norm id");
  if (!dims || !in || !out) return refuse(c, DISC_ERR_INVALID_ARG, "null pointer array");
  const bool adds = n_in == 3;
  if (n_dims != 6 || (n_in != 2 && n_in != 3) || n_out != n_in) return refuse(c, DISC_ERR_INVALID_ARG, "a norm takes 6 dims, x, weight and with a residual that, codes, scales and with a residual the total");
  NormArgs a;
  memset(&a, 0, sizeof a);
  if (const int rc = check_rows(c, *o, dims[0], dims[1])) return rc;
  a.rows = dims[0];
  a.width = (int32_t)dims[1];
  a.x_row = dims[2];
  a.residual_row = dims[3];
  a.total_row = dims[4];
  a.codes_row = dims[5];
  if (a.rows == 0) return context_device(c) < 0 ? on_host(c) : DISC_OK;
  const int size = dtype_bytes(o->dtype);
  if (!extent_ok(a.rows, a.x_row, a.width) || !extent_ok(a.rows, a.codes_row, a.width) ||
      (adds && (!extent_ok(a.rows, a.residual_row, a.width) || !extent_ok(a.rows, a.total_row, a.width))))
    return refuse(c, DISC_ERR_SHAPE, "a stride is negative or an extent overflows");
  if (!apart(a.rows, a.codes_row, a.width) || (adds && !apart(a.rows, a.total_row, a.width))) return refuse(c, DISC_ERR_SHAPE, "rows of a result overlap");
  a.x = in[0];
  a.weight = in[1];
  a.residual = adds ? in[2] : nullptr;
  a.codes = out[0];
  a.scales = out[1];
  a.total = adds ? out[2] : nullptr;
  if (!a.x || !a.weight || !a.codes || !a.scales || (adds && (!a.residual || !a.total))) return refuse(c, DISC_ERR_INVALID_ARG, "null tensor pointer");
  if (!aligned(a.x, size) || !aligned(a.weight, size) || !aligned(a.residual, size) || !aligned(a.total, size) || !aligned(a.scales, 4))
    return refuse(c, DISC_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
  if (a.rows > 1 && adds && ((a.total == a.x && a.total_row != a.x_row) || (a.total == a.residual && a.total_row != a.residual_row)))
    return refuse(c, DISC_ERR_INVALID_ARG, "in place, both sides have the same strides");
  if (context_device(c) < 0) return on_host(c);
  const RowShape s(*o, a.width, kNormLanes, a.rows <= context_cus(c));
  a.lanes = s.lanes;
  const int64_t moved = times(a.rows * a.width, size * (adds ? 3 : 1) + 1);
  const bool nt = moved < 0 || moved >= kNonTemporalBytes;
  const int64_t groups = s.block / s.lanes, each = kMostThreads / s.block * groups;   // rows of a launch
  OnDevice on(context_device(c));
  if (!on.ok) return refuse(c, DISC_ERR_HIP, "hipSetDevice failed");
  int rc = DISC_OK, n = 0;
  for (int64_t left = a.rows; rc == DISC_OK && left > 0; ++n) {
    a.rows = std::min(left, each);
    rc = enqueue(c, o->fn[FN_NORM + 2 * log2_of(s.each) + (nt ? 1 : 0)], (uint64_t)ceil_div(a.rows, groups), 1, (uint32_t)s.block, &a, sizeof a, stream);
    left -= a.rows;
    a.x = (const char*)a.x + a.rows * a.x_row * size;
    a.codes = (char*)a.codes + a.rows * a.codes_row;
    a.scales = (char*)a.scales + a.rows * 4;
    if (adds) {
      a.residual = (const char*)a.residual + a.rows * a.residual_row * size;
      a.total = (char*)a.total + a.rows * a.total_row * size;
    }
  }
  if (rc == DISC_OK) context_count(c, n);
  return rc;
}

// Groups of threads that share a gradient's rows, each with a row of partial sums.
int64_t backward_blocks(disc_ctx* c, const RowShape& s, int64_t rows) { return std::min<int64_t>(ceil_div(rows, s.block / s.lanes), 2 * context_cus(c)); }
size_t backward_bytes(disc_ctx* c, const Operator& o, int64_t rows, int64_t width) {
  const RowShape s(o, width, kBackwardLanes, false);
  return (size_t)(backward_blocks(c, s, rows) * (s.block / s.lanes) * width) * 4;
}

int launch_norm_backward(disc_ctx* c, int32_t id, const int64_t* dims, int n_dims, const void* const* in, int n_in, void* const* out, int n_out,
                         void* workspace, size_t workspace_bytes, void* stream) {
  if (!c) return DISC_ERR_INVALID_ARG;
  const Operator* o = get_operator(c, id, Operator::NORM);
  if (!o) return refuse(c, DISC_ERR_INVALID_ARG, "bad norm id");
  if (!dims || !in || !out) return refuse(c, DISC_ERR_INVALID_ARG, "null pointer array");
  const bool adds = n_in == 4;
  if (n_dims != 6 || (n_in != 3 && n_in != 4) || n_out != 2)
    return refuse(c, DISC_ERR_INVALID_ARG, "a norm's gradient takes 6 dims, total, weight, dy and where there is one dtotal, dx and dweight");
  NormBackwardArgs a;
  memset(&a, 0, sizeof a);
  if (const int rc = check_rows(c, *o, dims[0], dims[1])) return rc;
  a.rows = dims[0];
  a.width = (int32_t)dims[1];
  a.total_row = dims[2];
  a.dy_row = dims[3];
  a.dtotal_row = dims[4];
  a.dx_row = dims[5];
  const int size = dtype_bytes(o->dtype);
  a.total = in[0];
  a.weight = in[1];
  a.dy = in[2];
  a.dtotal = adds ? in[3] : nullptr;
  a.dx = out[0];
  a.dweight = out[1];
  if (!a.dweight || !aligned(a.dweight, 4)) return refuse(c, DISC_ERR_INVALID_ARG, "dweight: null or not aligned to its elements");
  if (a.rows > 0) {
    if (!extent_ok(a.rows, a.total_row, a.width) || !extent_ok(a.rows, a.dy_row, a.width) || !extent_ok(a.rows, a.dx_row, a.width) ||
        (adds && !extent_ok(a.rows, a.dtotal_row, a.width)))
      return refuse(c, DISC_ERR_SHAPE, "a stride is negative or an extent overflows");
    if (!apart(a.rows, a.dx_row, a.width)) return refuse(c, DISC_ERR_SHAPE, "rows of a result overlap");
    if (!a.total || !a.weight || !a.dy || !a.dx || (adds && !a.dtotal)) return refuse(c, DISC_ERR_INVALID_ARG, "null tensor pointer");
    if (!aligned(a.total, size) || !aligned(a.weight, size) || !aligned(a.dy, size) || !aligned(a.dtotal, size) || !aligned(a.dx, size))
      return refuse(c, DISC_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
    if (a.rows > 1 && ((a.dx == a.total && a.dx_row != a.total_row) || (a.dx == a.dy && a.dx_row != a.dy_row) || (a.dx == a.dtotal && a.dx_row != a.dtotal_row)))
      return refuse(c, DISC_ERR_INVALID_ARG, "in place, both sides have the same strides");
  }
  const RowShape s(*o, a.width, kBackwardLanes, false);
  const int64_t blocks = backward_blocks(c, s, a.rows);
  a.lanes = s.lanes;
  a.parts = (int32_t)(blocks * (s.block / s.lanes));
  if (a.parts > 0 && (!workspace || workspace_bytes < (size_t)a.parts * a.width * 4)) return refuse(c, DISC_ERR_WORKSPACE, "workspace missing or too small");
  if (!aligned(workspace, 16)) return refuse(c, DISC_ERR_INVALID_ARG, "the workspace is not 16-byte aligned");
  a.part = (float*)workspace;
  if (context_device(c) < 0) return on_host(c);
  const int64_t moved = times(a.rows * a.width, size * (adds ? 4 : 3));
  const bool nt = moved < 0 || moved >= kNonTemporalBytes;
  OnDevice on(context_device(c));
  if (!on.ok) return refuse(c, DISC_ERR_HIP, "hipSetDevice failed");
  int rc = DISC_OK, n = 0;
  if (blocks > 0) {
    rc = enqueue(c, o->fn[FN_NORM_BACKWARD + 2 * log2_of(s.each) + (nt ? 1 : 0)], (uint64_t)blocks, 1, (uint32_t)s.block, &a, sizeof a, stream);
    ++n;
  }
  if (rc == DISC_OK) {   // (no rows: zeros)
    rc = enqueue(c, o->fn[FN_NORM_JOIN], (uint64_t)ceil_div(a.width, 64), 1, 256, &a, sizeof a, stream);
    ++n;
  }
  if (rc == DISC_OK) context_count(c, n);
  return rc;
}

// ---- products with 4-bit weights -------------------------------------------------------------------

int register_linear4(disc_ctx* c, const disc_linear4_desc* d, int32_t* id_out) {
  if (!c) return DISC_ERR_INVALID_ARG;
  if (!d || !id_out) return refuse(c, DISC_ERR_INVALID_ARG, "null pointer");
  if (d->dtype != DISC_F16 && d->dtype != DISC_BF16) return refuse(c, DISC_ERR_INVALID_ARG, "a product gives f16 or bf16 rows");
  if (d->rows < DISC_STORAGE_SAME || d->rows > DISC_STORAGE_E4M3) return refuse(c, DISC_ERR_INVALID_ARG, "bad storage of the rows");
  if (d->group != 32 && d->group != 64 && d->group != 128) return refuse(c, DISC_ERR_SHAPE, "group is 32, 64 or 128", d->group);
  std::string macros = "#define DISC_LINEAR4 1\n#define DISC_T_F16 " + std::to_string(d->dtype == DISC_F16 ? 1 : 0) + "\n";
  macros += "#define DISC_ROWS " + std::to_string(d->rows) + "\n#define DISC_GROUP " + std::to_string(d->group) + "\n#define DISC_ZEROS " + (d->zeros ? "1\n" : "0\n");
  std::unique_ptr<Operator> o(new Operator);
  o->kind = Operator::LINEAR4;
  o->key = macros;
  o->dtype = d->dtype;
  o->storage = d->rows;
  o->group = d->group;
  o->zeros = d->zeros != 0;
  static const char* const names[] = {"disc_linear1_k", "disc_linear2_k", "disc_linear4_k"};
  return enter(c, std::move(o), macros, kStepHeader, names, FN_LINEAR_COUNT, FN_LINEAR1, id_out);
}

int launch_linear4(disc_ctx* c, int32_t id, const int64_t* dims, int n_dims, const void* const* in, int n_in, void* const* out, int n_out, void* stream) {
  if (!c) return DISC_ERR_INVALID_ARG;
  const Operator* o = get_operator(c, id, Operator::LINEAR4);
  if (!o) return refuse(c, DISC_ERR_INVALID_ARG, "bad product id");
  if (!dims || !in || !out) return refuse(c, DISC_ERR_INVALID_ARG, "null pointer array");
  const bool scaled = o->storage != DISC_STORAGE_SAME;
  const int least = 3 + (scaled ? 1 : 0) + (o->zeros ? 1 : 0);
  if (n_dims != 5 || (n_in != least && n_in != least + 1) || n_out != 1)
    return refuse(c, DISC_ERR_INVALID_ARG, "a product takes 5 dims, x, weights, scales, with 8-bit rows their scales, with zero points those, where there is one a bias, and one result");
  LinearArgs a;
  memset(&a, 0, sizeof a);
  const int64_t rows = dims[0], n = dims[1], k = dims[2];
  if (rows < 0 || rows > 1 << 20) return refuse(c, DISC_ERR_SHAPE, "rows is 0 .. 2^20", rows);
  if (n < 1 || n > 1 << 26) return refuse(c, DISC_ERR_SHAPE, "n is 1 .. 2^26", n);
  if (k < o->group || k > 1 << 24 || k % o->group) return refuse(c, DISC_ERR_SHAPE, "k is a multiple of the group, at most 2^24", k);
  a.rows = (int32_t)rows;
  a.n = (int32_t)n;
  a.k = (int32_t)k;
  a.groups = (int32_t)(k / o->group);
  a.x_row = dims[3];
  a.out_row = dims[4];
  if (rows == 0) return context_device(c) < 0 ? on_host(c) : DISC_OK;
  if (!extent_ok(rows, a.x_row, k) || !extent_ok(rows, a.out_row, n)) return refuse(c, DISC_ERR_SHAPE, "a stride is negative or an extent overflows");
  if (!apart(rows, a.out_row, n)) return refuse(c, DISC_ERR_SHAPE, "rows of a result overlap");
  int i = 3;
  a.x = in[0];
  a.weights = in[1];
  a.scales = in[2];
  a.row_scales = scaled ? in[i++] : nullptr;
  a.zeros = o->zeros ? in[i++] : nullptr;
  a.bias = n_in > least ? in[i] : nullptr;
  a.out = out[0];
  if (!a.x || !a.weights || !a.scales || (scaled && !a.row_scales) || (o->zeros && !a.zeros) || (n_in > least && !a.bias) || !a.out)
    return refuse(c, DISC_ERR_INVALID_ARG, "null tensor pointer");
  if (!aligned(a.weights, 16)) return refuse(c, DISC_ERR_INVALID_ARG, "the weights are not 16-byte aligned");
  if (!aligned(a.x, scaled ? 1 : 2) || !aligned(a.scales, 2) || !aligned(a.row_scales, 4) || !aligned(a.bias, 2) || !aligned(a.out, 2))
    return refuse(c, DISC_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
  if (context_device(c) < 0) return on_host(c);
  const int tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  OnDevice on(context_device(c));
  if (!on.ok) return refuse(c, DISC_ERR_HIP, "hipSetDevice failed");
  const int rc = enqueue(c, o->fn[tiles == 1 ? FN_LINEAR1 : tiles == 2 ? FN_LINEAR2 : FN_LINEAR4], (uint64_t)ceil_div(n, 16), (uint32_t)ceil_div(rows, 16 * tiles), 512, &a,
                         sizeof a, stream);
  if (rc == DISC_OK) context_count(c, 1);
  return rc;
}

// ---- drafted tokens --------------------------------------------------------------------------------

int register_verify(disc_ctx* c, const disc_verify_desc* d, int32_t* id_out) {
  if (!c) return DISC_ERR_INVALID_ARG;
  if (!d || !id_out) return refuse(c, DISC_ERR_INVALID_ARG, "null pointer");
  if (!is_float_dtype(d->dtype)) return refuse(c, DISC_ERR_INVALID_ARG, "probabilities are f32, f16 or bf16");
  const std::string macros = std::string("#define DISC_VERIFY 1\n#define DISC_T ") + dtype_ctype(d->dtype) + "\n";
  std::unique_ptr<Operator> o(new Operator);
  o->kind = Operator::VERIFY;
  o->key = macros;
  o->dtype = d->dtype;
  static const char* const names[] = {"disc_verify_sum_k", "disc_verify_pick_k"};
  return enter(c, std::move(o), macros, kStepHeader, names, FN_VERIFY_COUNT, FN_VERIFY_SUM, id_out);
}

int check_verify(disc_ctx* c, int64_t batch, int64_t drafts, int64_t vocabulary) {
  if (batch < 0 || batch > 1 << 20) return refuse(c, DISC_ERR_SHAPE, "batch is 0 .. 2^20", batch);
  if (drafts < 0 || drafts > 4096) return refuse(c, DISC_ERR_SHAPE, "drafts is 0 .. 4096", drafts);
  if (vocabulary < 1 || vocabulary > 1 << 30) return refuse(c, DISC_ERR_SHAPE, "vocabulary is 1 .. 2^30", vocabulary);
  if (batch * ceil_div(vocabulary, kVerifyChunk) > kMostThreads / 256) return refuse(c, DISC_ERR_SHAPE, "too many rows for one call");
  return DISC_OK;
}

int launch_verify(disc_ctx* c, int32_t id, const int64_t* dims, int n_dims, const void* const* in, int n_in, void* const* out, int n_out,
                  void* workspace, size_t workspace_bytes, void* stream) {
  if (!c) return DISC_ERR_INVALID_ARG;
  const Operator* o = get_operator(c, id, Operator::VERIFY);
  if (!o) return refuse(c, DISC_ERR_INVALID_ARG, "bad verification id");
  if (!dims || !in || !out) return refuse(c, DISC_ERR_INVALID_ARG, "null pointer array");
  if (n_dims != 9) return refuse(c, DISC_ERR_INVALID_ARG, "a verification takes 9 dims");
  const bool drafted = dims[7] != 0, ragged = dims[8] != 0;
  if (n_in != 3 + (drafted ? 1 : 0) + (ragged ? 1 : 0) || n_out != 2)
    return refuse(c, DISC_ERR_INVALID_ARG, "a verification takes the target's probabilities, the drafted tokens, uniforms, where there are some the draft's probabilities and lengths, tokens and accepted");
  VerifyArgs a;
  memset(&a, 0, sizeof a);
  if (const int rc = check_verify(c, dims[0], dims[1], dims[2])) return rc;
  a.batch = (int32_t)dims[0];
  a.drafts = (int32_t)dims[1];
  a.vocabulary = (int32_t)dims[2];
  a.chunks = (int32_t)ceil_div(a.vocabulary, kVerifyChunk);
  a.target_batch = dims[3];
  a.target_row = dims[4];
  a.draft_batch = dims[5];
  a.draft_row = dims[6];
  if (a.batch == 0) return context_device(c) < 0 ? on_host(c) : DISC_OK;
  if (!strides_ok(a.batch, a.target_batch, a.drafts + 1, a.target_row, a.vocabulary) ||
      (drafted && a.drafts > 0 && !strides_ok(a.batch, a.draft_batch, a.drafts, a.draft_row, a.vocabulary)))
    return refuse(c, DISC_ERR_SHAPE, "a stride is negative or an extent overflows");
  a.target = in[0];
  a.drafted = in[1];
  a.uniforms = in[2];
  a.draft = drafted ? in[3] : nullptr;
  a.lengths = ragged ? in[n_in - 1] : nullptr;
  a.tokens = out[0];
  a.accepted = out[1];
  if (!a.target || !a.uniforms || !a.tokens || !a.accepted || (a.drafts > 0 && (!a.drafted || (drafted && !a.draft))) || (ragged && !a.lengths))
    return refuse(c, DISC_ERR_INVALID_ARG, "null tensor pointer");
  const int size = dtype_bytes(o->dtype);
  if (!aligned(a.target, size) || !aligned(a.draft, size) || !aligned(a.drafted, 4) || !aligned(a.uniforms, 4) || !aligned(a.lengths, 4) || !aligned(a.tokens, 4) ||
      !aligned(a.accepted, 4))
    return refuse(c, DISC_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
  if (!workspace || workspace_bytes < (size_t)a.batch * a.chunks * 16) return refuse(c, DISC_ERR_WORKSPACE, "workspace missing or too small");
  if (!aligned(workspace, 16)) return refuse(c, DISC_ERR_INVALID_ARG, "the workspace is not 16-byte aligned");
  a.part = workspace;
  if (context_device(c) < 0) return on_host(c);
  OnDevice on(context_device(c));
  if (!on.ok) return refuse(c, DISC_ERR_HIP, "hipSetDevice failed");
  int rc = enqueue(c, o->fn[FN_VERIFY_SUM], (uint64_t)a.batch * a.chunks, 1, 256, &a, sizeof a, stream);
  if (rc == DISC_OK) rc = enqueue(c, o->fn[FN_VERIFY_PICK], (uint64_t)a.batch, 1, 256, &a, sizeof a, stream);
  if (rc == DISC_OK) context_count(c, 2);
  return rc;
}

}  // namespace
}  // namespace disc

using namespace disc;

extern "C" {

int disc_register_norm(disc_ctx* ctx, const disc_norm_desc* desc, int32_t* id_out) {
  return guarded(ctx, [&] { return register_norm(ctx, desc, id_out); });
}
int disc_norm(disc_ctx* ctx, int32_t id, const int64_t* dims, int n_dims, const void* const* inputs, int n_in, void* const* outputs, int n_out, void*, size_t,
              void* hip_stream) {
  return guarded(ctx, [&] { return launch_norm(ctx, id, dims, n_dims, inputs, n_in, outputs, n_out, hip_stream); });
}
int disc_norm_backward(disc_ctx* ctx, int32_t id, const int64_t* dims, int n_dims, const void* const* inputs, int n_in, void* const* outputs, int n_out,
                       void* workspace, size_t workspace_bytes, void* hip_stream) {
  return guarded(ctx, [&] { return launch_norm_backward(ctx, id, dims, n_dims, inputs, n_in, outputs, n_out, workspace, workspace_bytes, hip_stream); });
}
int disc_norm_workspace_bytes(disc_ctx* ctx, int32_t id, const int64_t* dims, int n_dims, size_t* out) {
  return guarded(ctx, [&] {
    if (!ctx || !out) return (int)DISC_ERR_INVALID_ARG;
    const Operator* o = get_operator(ctx, id, Operator::NORM);
    if (!o) return refuse(ctx, DISC_ERR_INVALID_ARG, "bad norm id");
    if (!dims || n_dims != 6) return refuse(ctx, DISC_ERR_INVALID_ARG, "a norm's gradient takes 6 dims");
    const int rc = check_rows(ctx, *o, dims[0], dims[1]);
    if (rc == DISC_OK) *out = backward_bytes(ctx, *o, dims[0], dims[1]);
    return rc;
  });
}
int disc_register_linear4(disc_ctx* ctx, const disc_linear4_desc* desc, int32_t* id_out) {
  return guarded(ctx, [&] { return register_linear4(ctx, desc, id_out); });
}
int disc_linear4(disc_ctx* ctx, int32_t id, const int64_t* dims, int n_dims, const void* const* inputs, int n_in, void* const* outputs, int n_out, void*, size_t,
                 void* hip_stream) {
  return guarded(ctx, [&] { return launch_linear4(ctx, id, dims, n_dims, inputs, n_in, outputs, n_out, hip_stream); });
}
int disc_register_verify(disc_ctx* ctx, const disc_verify_desc* desc, int32_t* id_out) {
  return guarded(ctx, [&] { return register_verify(ctx, desc, id_out); });
}
int disc_verify(disc_ctx* ctx, int32_t id, const int64_t* dims, int n_dims, const void* const* inputs, int n_in, void* const* outputs, int n_out,
                void* workspace, size_t workspace_bytes, void* hip_stream) {
  return guarded(ctx, [&] { return launch_verify(ctx, id, dims, n_dims, inputs, n_in, outputs, n_out, workspace, workspace_bytes, hip_stream); });
}
int disc_verify_workspace_bytes(disc_ctx* ctx, int32_t id, const int64_t* dims, int n_dims, size_t* out) {
  return guarded(ctx, [&] {
    if (!ctx || !out) return (int)DISC_ERR_INVALID_ARG;
    if (!get_operator(ctx, id, Operator::VERIFY)) return refuse(ctx, DISC_ERR_INVALID_ARG, "bad verification id");
    if (!dims || n_dims != 9) return refuse(ctx, DISC_ERR_INVALID_ARG, "a verification takes 9 dims");
    const int rc = check_verify(ctx, dims[0], dims[1], dims[2]);
    if (rc == DISC_OK) *out = (size_t)(dims[0] * ceil_div(dims[2], kVerifyChunk)) * 16;
    return rc;
  });
}

}  // extern "C"
