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
  float offset, pad;
  double eps;
};
struct NormBackwardArgs {
  const void *total, *weight, *dy, *dtotal;
  void *dx, *dweight;
  float* part;
  int64_t total_row, dy_row, dtotal_row, dx_row, rows;
  int32_t width, lanes, parts, groups;
  float offset;
  double eps;
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

// the norm's kernels and its gradient's (with _nt behind: past the caches), and what joins the gradient's parts
enum { FN_NORM_S1 = 0, FN_NORM_S4, FN_NORM_S4_NT, FN_NORM_4, FN_NORM_4_NT, FN_NORM_B1, FN_NORM_B4, FN_BACKWARD_S1, FN_BACKWARD_S4, FN_BACKWARD_S4_NT, FN_BACKWARD_4,
       FN_BACKWARD_4_NT, FN_BACKWARD_B2, FN_BACKWARD_B4, FN_NORM_JOIN, FN_NORM_COUNT };
struct LinearKernel {
  const char* name;
  int m, n, split, teams;   // tiles of 16 rows of x and of weights, wavefronts of a team, teams of a block
};
#define FEW(N, R, S, W) {"disc_linear_" #N "_" #R "_" #S "_" #W "_k", 1, N, S, W}
#define WIDE(M, N, S, W, B) {"disc_linear_wide_" #M "_" #N "_" #S "_" #W "_" #B "_k", M, N, S, W}
constexpr LinearKernel kLinear[] = {
    FEW(1, 1, 1, 8),     FEW(1, 1, 16, 1),    FEW(1, 1, 8, 1),     FEW(2, 1, 8, 1),     FEW(1, 4, 1, 8),     FEW(1, 4, 8, 1),
    FEW(1, 16, 8, 1),    WIDE(1, 2, 2, 4, 2), WIDE(1, 1, 8, 1, 2), WIDE(1, 1, 4, 2, 2), WIDE(1, 1, 2, 4, 4), WIDE(1, 1, 2, 8, 4),
    WIDE(2, 1, 8, 1, 1), WIDE(2, 1, 4, 2, 1), WIDE(2, 2, 4, 2, 2), WIDE(2, 2, 2, 4, 2), WIDE(4, 1, 2, 4, 2), WIDE(4, 1, 2, 8, 1),
};
#undef FEW
#undef WIDE
constexpr int kLinearCount = sizeof kLinear / sizeof kLinear[0];
static_assert(kLinearCount <= (int)(sizeof(Operator::fn) / sizeof(void*)) && FN_NORM_COUNT <= kLinearCount, "an operator holds as many kernels");
// Which of them, by rows x k x n (us).  Of one row, the first four: a team's wavefronts take 256 elements each at a time, so that rows
// are shared out by as many as leave each something; where columns are many, two tiles share what is loaded of x.
//   1 x 512 x 32768 4.8, 17.3, 7.9, 7.2; 1 x 1024 x 32768 7.1, 18.3, 8.7, 8.3; 1 x 4096 x 4096 18.9, 5.1, 5.2, 6.8;
//   1 x 16384 x 1024 67, 10.5, 11.3, 17; 1 x 4096 x 12288 19.5, 12.3, 8.9, 10.5; 1 x 8192 x 131072 170, 190, 133, 123.
// (x through LDS, the last of those for 16 rows, is a seventh faster than the fourth at 1 x 4096 x 28672, 17.0 for 19.3, as fast at 1 x 8192 x 32768, 36.1
// for 36.5, and slower at 1 x 8192 x 131072, 134; it is not among the choices for one row.)
// Of more, the smallest block by which every CU has no more than one: a block of more columns takes less a column, and a CU two blocks of a
// kind twice as long as one.  Columns of a block 16, 32, 64, 128, of 16 rows of x:
//   16 x 4096 x 4096 7.1, 7.6, 10.5, 16.0; 16 x 4096 x 8192 12.8, 8.1, 10.6, 15.9; 16 x 4096 x 12288 18.3, 14.2, 10.8, 15.9; 16 x 4096 x 28672 45, 30, 22, 19.8;
//   16 x 8192 x 131072 307, 198, 152, 146; of 32 rows of x: 32 x 4096 x 4096 9.3, 10.5, 14.4, 21.1; 32 x 14336 x 4096 22.6, 27, 37, 63; 32 x 4096 x 12288
//   -, 20.3, 14.7, 21.1; 32 x 4096 x 28672 -, 43, 31, 24.5; 64 x 4096 x 4096 16.4, 10.6, 14.2, 20.8; 64 x 8192 x 8192 -, 36.4, 26.3, 41.8;
//   64 and 128 columns of 64 rows: 64 x 4096 x 12288 19.7, 26.5; 64 x 12288 x 12288 57, 76 (128 of 32 rows 62); 64 x 4096 x 28672 43, 30.8.
// Of up to 16 rows and a short k, or few columns and rows, x comes without LDS, or a wavefront has two tiles of columns:
//   16 x 512 x 8192 4.0 (6.9 by 16 columns, 4.1 by 32); 5 x 4096 x 4096 6.1 (6.7); 8 x 4096 x 4096 6.6 (6.7); 16 x 512 x 32768 6.4 (7.8 by 128); 16 x 512 x 131072 21 (28).
// Two to four rows of many columns as more: 3 x 8192 x 131072 160 without LDS, 138; 3 x 4096 x 28672 20.5, 17.9; 3 x 4096 x 12288 9.3, 15.7.
int linear_kernel(int64_t rows, int64_t n, int64_t k, int64_t cus) {
  const int64_t tiles = ceil_div(n, 16);
  if (rows > 32) {
    const int64_t pairs = tiles * 4 * ceil_div(rows, 64);   // tiles of x times those of weights
    return pairs <= 2 * cus ? 12 : pairs <= 4 * cus ? 13 : pairs <= 8 * cus ? 14 : pairs <= 16 * cus ? 16 : 17;
  }
  if (rows > 16) return tiles <= cus ? 12 : tiles <= 2 * cus ? 13 : tiles <= 4 * cus ? 14 : 15;
  if (rows > 4) {
    if (tiles <= cus) return k <= 1024 || (rows <= 8 && k <= 4096) ? 6 : 8;
    if (tiles <= 2 * cus) return k <= 512 ? 6 : 9;
    return tiles <= 4 * cus ? 10 : k <= 1024 ? 7 : 11;
  }
  if (rows > 1) return k <= 1024 ? 4 : tiles <= 4 * cus ? 5 : 11;
  return k <= 1024 ? 0 : tiles <= cus ? 1 : tiles <= 4 * cus ? 2 : 3;
}
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

// ---- norm ------------------------------------------------------------------------------------------

int register_norm(disc_ctx* c, const disc_norm_desc* d, int32_t* id_out) {
  if (!c) return DISC_ERR_INVALID_ARG;
  if (!d || !id_out) return refuse(c, DISC_ERR_INVALID_ARG, "null pointer");
  if (!is_float_dtype(d->dtype)) return refuse(c, DISC_ERR_INVALID_ARG, "a norm takes f32, f16 or bf16");
  if (d->storage != DISC_STORAGE_I8 && d->storage != DISC_STORAGE_E4M3) return refuse(c, DISC_ERR_INVALID_ARG, "a norm's rows are stored as i8 or e4m3");
  if (!(d->eps > 0.0) || !std::isfinite((float)d->eps) || (float)d->eps == 0.f) return refuse(c, DISC_ERR_INVALID_ARG, "eps is a positive number of 32 bits");
  if (!std::isfinite((float)d->weight_offset)) return refuse(c, DISC_ERR_INVALID_ARG, "weight_offset is no finite number of 32 bits");
  const std::string macros = std::string("#define DISC_NORM 1\n#define DISC_T ") + dtype_ctype(d->dtype) + "\n#define DISC_STORAGE " + std::to_string(d->storage) + "\n";
  std::unique_ptr<Operator> o(new Operator);
  o->kind = Operator::NORM;
  o->key = macros + text("%a ", d->eps) + text("%a", d->weight_offset);
  o->dtype = d->dtype;
  o->storage = d->storage;
  o->eps = d->eps;
  o->offset = (float)d->weight_offset;
  static const char* const names[] = {"disc_norm1_s",          "disc_norm4_s",          "disc_norm4_s_nt",          "disc_norm4",          "disc_norm4_nt",
                                      "disc_norm1_b",          "disc_norm4_b",          "disc_norm_backward1_s",    "disc_norm_backward4_s", "disc_norm_backward4_s_nt",
                                      "disc_norm_backward4",   "disc_norm_backward4_nt", "disc_norm_backward2_b", "disc_norm_backward4_b", "disc_norm_join_k"};
  return enter(c, std::move(o), macros, kStepHeader, names, FN_NORM_COUNT, FN_NORM_4, id_out);
}

// Who has a row: `lanes` threads, a part of a wavefront or all of a block, and which kernel.
struct RowShape {
  int lanes, block, fn;
  int per_cu = 0;           // (the gradient's) blocks a CU that the rows are shared out to
  int groups() const { return block / lanes; }
};
RowShape norm_shape(const Operator& o, int64_t width, bool few, bool nt) {
  const int64_t accesses = ceil_div(width * dtype_bytes(o.dtype), 16);
  if (accesses <= 64) return {(int)std::max<int64_t>(8, power_of_two(accesses)), 256, FN_NORM_S1};
  if (few && accesses <= 1024) return {(int)ceil_div(accesses, 64) * 64, (int)ceil_div(accesses, 64) * 64, FN_NORM_B1};
  if (accesses <= 256) return {(int)power_of_two(ceil_div(accesses, 4)), 256, nt ? FN_NORM_S4_NT : FN_NORM_S4};
  const int block = (int)ceil_div(accesses, 256) * 64;
  return {block, block, accesses > 2048 ? FN_NORM_B4 : nt ? FN_NORM_4_NT : FN_NORM_4};
}
// Blocks of a gradient: enough that a CU has rows under way while others are being summed, and few enough that the parts, a row of
// 32 bits each, stay small beside the rows (us with 1, 2, 3, 4, 6 a CU: 65536 x 512 bf16 134, 80, 66, 62, 63; 16384 x 1024 41, 32,
// 34, 36, 38; 16384 x 4096 214, 144, 117, 119, 132; 8192 x 8192 148, 115, 133, 125, 136; 4096 x 16384 133, 145, 158, 172, 200).
RowShape backward_shape(const Operator& o, int64_t width, bool nt) {
  const int64_t accesses = ceil_div(width * dtype_bytes(o.dtype), 16);
  if (accesses <= 64) return {(int)std::max<int64_t>(8, power_of_two(accesses)), 256, FN_BACKWARD_S1, 4};
  if (accesses <= 256) return {(int)power_of_two(ceil_div(accesses, 4)), 256, nt ? FN_BACKWARD_S4_NT : FN_BACKWARD_S4, 2};
  if (accesses > 2048) return {1024, 1024, FN_BACKWARD_B4, 1};
  const int block = (int)(accesses > 1024 ? ceil_div(accesses, 128) : ceil_div(accesses, 256)) * 64;
  if (accesses > 1024) return {block, block, FN_BACKWARD_B2, 1};
  return {block, block, nt ? FN_BACKWARD_4_NT : FN_BACKWARD_4, block <= 128 ? 3 : 2};
}

int check_rows(disc_ctx* c, const Operator& o, int64_t rows, int64_t width) {
  if (rows < 0 || rows > kMostRows) return refuse(c, DISC_ERR_SHAPE, "rows is 0 .. 2^31 - 1", rows);
  const int64_t most = 1024 * 4 * 16 / dtype_bytes(o.dtype);
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
  a.offset = o->offset;
  a.eps = o->eps;
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
  const int64_t moved = times(a.rows * a.width, size * (adds ? 3 : 1) + 1);
  const RowShape s = norm_shape(*o, a.width, a.rows <= 2 * context_cus(c), moved < 0 || moved >= kNonTemporalBytes);
  a.lanes = s.lanes;
  const int64_t groups = s.groups(), each = kMostThreads / s.block * groups;   // rows of a launch
  OnDevice on(context_device(c));
  if (!on.ok) return refuse(c, DISC_ERR_HIP, "hipSetDevice failed");
  int rc = DISC_OK, n = 0;
  for (int64_t left = a.rows; rc == DISC_OK && left > 0; ++n) {
    a.rows = std::min(left, each);
    rc = enqueue(c, o->fn[s.fn], (uint64_t)ceil_div(a.rows, groups), 1, (uint32_t)s.block, &a, sizeof a, stream);
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

// Blocks that share a gradient's rows, each with a row of partial sums.
int64_t backward_blocks(disc_ctx* c, const RowShape& s, int64_t rows) {
  const int64_t all = ceil_div(rows, s.groups()), most = s.per_cu * context_cus(c);
  return all > 0 ? ceil_div(all, ceil_div(all, most)) : 0;   // (each as many rows, within one)
}
size_t backward_bytes(disc_ctx* c, const Operator& o, int64_t rows, int64_t width) {
  const RowShape s = backward_shape(o, width, false);
  return (size_t)(std::min<int64_t>(ceil_div(rows, s.groups()), s.per_cu * context_cus(c)) * width) * 4;   // (any fewer rows too)
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
  a.offset = o->offset;
  a.eps = o->eps;
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
  const int64_t moved = times(a.rows * a.width, size * (adds ? 4 : 3));
  const RowShape s = backward_shape(*o, a.width, moved < 0 || moved >= kNonTemporalBytes);
  const int64_t blocks = backward_blocks(c, s, a.rows);
  a.lanes = s.lanes;
  a.parts = (int32_t)blocks;
  a.groups = (int32_t)(blocks * s.groups());
  if (a.parts > 0 && (!workspace || workspace_bytes < (size_t)a.parts * a.width * 4)) return refuse(c, DISC_ERR_WORKSPACE, "workspace missing or too small");
  if (!aligned(workspace, 16)) return refuse(c, DISC_ERR_INVALID_ARG, "the workspace is not 16-byte aligned");
  a.part = (float*)workspace;
  if (context_device(c) < 0) return on_host(c);
  OnDevice on(context_device(c));
  if (!on.ok) return refuse(c, DISC_ERR_HIP, "hipSetDevice failed");
  int rc = DISC_OK, n = 0;
  if (blocks > 0) {
    rc = enqueue(c, o->fn[s.fn], (uint64_t)blocks, 1, (uint32_t)s.block, &a, sizeof a, stream);
    ++n;
  }
  if (rc == DISC_OK) {   // (no rows: zeros)
    rc = enqueue(c, o->fn[FN_NORM_JOIN], (uint64_t)ceil_div(a.width, 16), 1, 1024, &a, sizeof a, stream);
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
  const char* names[kLinearCount];
  for (int i = 0; i < kLinearCount; ++i) names[i] = kLinear[i].name;
  return enter(c, std::move(o), macros, kStepHeader, names, kLinearCount, 0, id_out);
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
  const int at = linear_kernel(rows, n, k, context_cus(c));
  const LinearKernel& f = kLinear[at];
  OnDevice on(context_device(c));
  if (!on.ok) return refuse(c, DISC_ERR_HIP, "hipSetDevice failed");
  const int rc = enqueue(c, o->fn[at], (uint64_t)ceil_div(n, 16 * f.n * f.teams), (uint32_t)ceil_div(rows, 16 * f.m), (uint32_t)(f.split * f.teams) * 64, &a, sizeof a, stream);
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
