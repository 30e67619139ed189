// C ABI of the operators on data (include/morello_mi355x.h): descriptor checks, workspace, and the
// products and passes that a call is made of.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdarg>
#include <cstdio>

#include "../../include/morello_mi355x.h"
#include "operators.h"

using namespace mrl;

namespace {

int32_t refuse(int32_t code, const char* fmt, ...) {
  char text[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(text, sizeof text, fmt, ap);
  va_end(ap);
  return fail_with(code, text);
}
#define CHECK(cond, ...) do { if (!(cond)) return refuse(MRL_E_INVAL, __VA_ARGS__); } while (0)

int32_t hip_status(hipError_t e) { return e == hipSuccess ? MRL_OK : refuse(MRL_E_HIP, "launch: %s", hipGetErrorString(e)); }

constexpr uint32_t kSizeEnd = 1u << 31;
size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

// A matrix of b x rows x columns.  written: elements must not share a place.
int32_t check_matrix(const char* name, const mrl_matrix& x, uint64_t b, uint64_t rows, uint64_t columns, bool written, bool column_major_too) {
  CHECK(x.dtype <= MRL_BF16, "%s: unknown type %u", name, x.dtype);
  CHECK(x.layout == MRL_ROW_MAJOR || (x.layout == MRL_COLUMN_MAJOR && column_major_too), "%s: unsupported layout %u", name, x.layout);
  if (!b || !rows || !columns) return MRL_OK;
  CHECK(x.data, "%s is NULL", name);
  CHECK((uintptr_t)x.data % (x.dtype == MRL_BF16 ? 2 : 4) == 0, "%s is not aligned to its elements", name);
  const uint64_t lines = x.layout ? columns : rows, width = x.layout ? rows : columns;
  CHECK(x.ld >= 0 && x.batch >= 0, "%s: negative stride", name);
  // the last element's offset, which products of 64 bits may not hold: the kernels' and those below do what it allows
  CHECK(x.ld < (int64_t)1 << 40 && x.batch < (int64_t)1 << 40 && ((unsigned __int128)(lines - 1) * x.ld + (unsigned __int128)(b - 1) * x.batch) >> 56 == 0,
        "%s: stride too large", name);
  if (written) {
    const bool rows_apart = lines == 1 || (uint64_t)x.ld >= width;
    const uint64_t one = (lines - 1) * (uint64_t)x.ld + width;                     // elements that a batch spans
    const bool inside = b == 1 || (uint64_t)x.batch >= one;                        // batch after batch,
    const bool across = b > 1 && (uint64_t)x.batch >= width && (lines == 1 || (uint64_t)x.ld >= (b - 1) * (uint64_t)x.batch + width);   // or row after row
    CHECK((rows_apart && inside) || across, "%s: rows or batches overlap", name);
  }
  return MRL_OK;
}
int32_t check_vector(const char* name, const mrl_matrix& x, uint64_t n) {
  CHECK(x.dtype <= MRL_BF16, "%s: unknown type %u", name, x.dtype);
  if (n) CHECK((uintptr_t)x.data % (x.dtype == MRL_BF16 ? 2 : 4) == 0, "%s is not aligned to its elements", name);
  return MRL_OK;
}

RowsOf rows_of(const mrl_matrix& x) { return RowsOf{x.data, x.ld, x.batch, x.dtype == MRL_BF16}; }

Drop drop_of(uint32_t drop, uint64_t seed, uint64_t offset) {
  return Drop{drop, drop < 65536 ? (float)(65536.0 / (65536 - drop)) : 0.0f, {(uint32_t)seed, (uint32_t)(seed >> 32)}, {(uint32_t)offset, (uint32_t)(offset >> 32)}};
}

int32_t check_common(uint32_t b, uint32_t m, uint32_t k, uint32_t n, uint32_t activation, uint32_t drop) {
  CHECK(b < kSizeEnd && m < kSizeEnd && k < kSizeEnd && n < kSizeEnd && (uint64_t)b * m < kSizeEnd, "sizes %u x %u x %u x %u: each, and b * m, must be below 2^31", b, m, k, n);
  CHECK(activation <= MRL_ACT_SILU, "unknown activation %u", activation);
  CHECK(drop <= 65536, "drop %u is above 65536", drop);
  return MRL_OK;
}

// An operand of a product over k: lines along the other index where its neighbours along k are adjacent.
struct Side { const void* data; uint32_t kc; int64_t ld, batch; };

// Workgroups and steps are counted in 32 bits.
int32_t check_product(const Product& p, const ProductPlan& plan) {
  CHECK(plan.blocks <= UINT32_MAX && (uint64_t)p.segs * ((p.K + 31ull) / 32) <= UINT32_MAX, "the product is too large for one call");
  return MRL_OK;
}

int32_t linear_product(const mrl_linear_desc& d, Product* out) {
  int32_t rc = check_common(d.b, d.m, d.k, d.n, d.activation, d.drop);
  if (rc) return rc;
  CHECK(d.lhs.dtype == d.rhs.dtype, "lhs and rhs of two types");
  const uint64_t b = d.b, work = d.k ? 1 : 0;
  if (!rc) rc = check_matrix("lhs", d.lhs, d.n ? b : 0, d.m, d.k, false, true);
  if (!rc) rc = check_matrix("rhs", d.rhs, (uint64_t)d.m * work ? b : 0, d.k, d.n, false, true);
  if (!rc && d.bias.data) rc = check_vector("bias", d.bias, d.n);
  if (!rc && d.residual.data) rc = check_matrix("residual", d.residual, b, d.m, d.n, false, false);
  if (!rc) rc = check_matrix("out", d.out, b, d.m, d.n, true, false);
  if (!rc && d.pre.data) rc = check_matrix("pre", d.pre, b, d.m, d.n, true, false);
  if (rc) return rc;
  Product p{};
  p.a = d.lhs.data;
  p.b = d.rhs.data;
  p.bf16 = d.lhs.dtype == MRL_BF16;
  p.a_kc = d.lhs.layout == MRL_ROW_MAJOR;
  p.b_kc = d.rhs.layout == MRL_COLUMN_MAJOR;
  p.lda = d.lhs.ld;
  p.ldb = d.rhs.ld;
  p.batch_a = d.lhs.batch;
  p.batch_b = d.rhs.batch;
  p.batches = d.b;
  p.segs = 1;
  p.M = d.m;
  p.N = d.n;
  p.K = d.k;
  p.e.out = rows_of(d.out);
  p.e.residual = rows_of(d.residual);
  p.e.pre = rows_of(d.pre);
  p.e.bias = d.bias.data;
  p.e.bias_bf16 = d.bias.dtype == MRL_BF16;
  p.e.activation = d.activation;
  p.e.drop = drop_of(d.drop, d.seed, d.offset);
  // batches that share rhs and follow each other are rows of one Matmul (the random bits count rows over the batches)
  const auto follows = [&](const RowsOf& r) { return !r.data || (uint64_t)r.batch == (uint64_t)d.m * (uint64_t)r.ld; };
  if (d.b > 1 && !d.rhs.batch && p.a_kc && (uint64_t)d.lhs.batch == (uint64_t)d.m * (uint64_t)d.lhs.ld && follows(p.e.out) && follows(p.e.residual) && follows(p.e.pre)) {
    p.M = d.b * d.m;
    p.batches = 1;
  }
  p.wa = p.a_kc ? p.K : p.M;
  p.wb = p.b_kc ? p.K : p.N;
  *out = p;
  return MRL_OK;
}

// What a gradient is made of: dz (rows without gaps, starting at multiples of 8 elements), then the two products.  dz is rounded to the
// operands' type, which both products need it in: a bf16 gradient is then within 0.0024 of its norm, where one rounding at the end leaves 0.0017,
// and a dz in f32 (or in two bf16 parts) would double what is written, read and multiplied.
struct GradPlan {
  bool pass;                       // dz differs from grad (or has another type): a pass over the rows makes it
  bool lhs, rhs;                   // wanted
  GradRows rows;
  Product by_lhs, by_rhs;
  ProductPlan plan_lhs, plan_rhs;
  size_t dz_bytes, sums_bytes, lhs_bytes, rhs_bytes;      // workspace, in this order
  size_t bytes() const { return dz_bytes + sums_bytes + lhs_bytes + rhs_bytes; }
};

int32_t plan_grad(const mrl_linear_grad_desc& d, GradPlan* out) {
  int32_t rc = check_common(d.b, d.m, d.k, d.n, d.activation, d.drop);
  if (rc) return rc;
  GradPlan g{};
  g.lhs = d.d_lhs.data && d.b && d.m && d.k;
  const bool sum = d.b != 1 && !d.d_rhs.batch;           // d_rhs is the sum over the batches (0 where there are none)
  g.rhs = d.d_rhs.data && (d.b || sum) && d.k && d.n;
  const uint32_t act = d.activation;
  CHECK(d.lhs.dtype == d.rhs.dtype, "lhs and rhs of two types");
  rc = check_matrix("grad", d.grad, d.b, d.m, d.n, false, false);
  if (!rc && act != MRL_ACT_NONE) rc = check_matrix("pre", d.pre, d.b, d.m, d.n, false, false);
  if (!rc) rc = check_matrix("rhs", d.rhs, g.lhs ? d.b : 0, d.k, d.n, false, true);
  if (!rc) rc = check_matrix("lhs", d.lhs, g.rhs ? d.b : 0, d.m, d.k, false, true);
  if (!rc && d.d_lhs.data) rc = check_matrix("d_lhs", d.d_lhs, d.b, d.m, d.k, true, false);
  if (!rc && d.d_rhs.data) rc = check_matrix("d_rhs", d.d_rhs, sum ? 1 : d.b, d.k, d.n, true, true);
  if (!rc && d.d_bias.data) rc = check_vector("d_bias", d.d_bias, d.n);
  if (rc) return rc;

  const uint32_t is_bf16 = d.lhs.dtype == MRL_BF16;
  const Drop drop = drop_of(d.drop, d.seed, d.offset);
  const uint64_t pitch = (d.n + 7ull) / 8 * 8;
  g.pass = (g.lhs || g.rhs) && (act != MRL_ACT_NONE || drop.drop || d.grad.dtype != d.lhs.dtype);
  g.dz_bytes = g.pass ? align_up((size_t)d.b * d.m * pitch * (is_bf16 ? 2 : 4)) : 0;
  RowsOf dz = rows_of(d.grad);
  if (g.pass) dz = RowsOf{nullptr, (int64_t)pitch, (int64_t)(d.m * pitch), is_bf16};
  g.rows.grad = rows_of(d.grad);
  if (act != MRL_ACT_NONE) g.rows.pre = rows_of(d.pre);
  g.rows.dz = dz;
  g.rows.batches = d.b;
  g.rows.M = d.m;
  g.rows.N = d.n;
  g.rows.activation = act;
  g.rows.drop = drop;
  g.rows.dbias = d.d_bias.data;
  g.rows.dbias_bf16 = d.d_bias.dtype == MRL_BF16;
  g.sums_bytes = align_up(grad_rows_bytes(d.b, d.m, d.n, d.d_bias.data));

  if (g.lhs) {                     // d_lhs = dz rhs^T: m x k, the sum over n
    Product& p = g.by_lhs;
    p.a = dz.data;
    p.b = d.rhs.data;
    p.bf16 = is_bf16;
    p.a_kc = 1;
    p.b_kc = d.rhs.layout == MRL_ROW_MAJOR;
    p.lda = dz.ld;
    p.ldb = d.rhs.ld;
    p.batch_a = dz.batch;
    p.batch_b = d.rhs.batch;
    p.batches = d.b;
    p.segs = 1;
    p.M = d.m;
    p.N = d.k;
    p.K = d.n;
    p.e.out = rows_of(d.d_lhs);
    if (d.b > 1 && !d.rhs.batch && (uint64_t)dz.batch == (uint64_t)d.m * (uint64_t)dz.ld && (uint64_t)d.d_lhs.batch == (uint64_t)d.m * (uint64_t)d.d_lhs.ld) {
      p.M = d.b * d.m;
      p.batches = 1;
    }
    p.wa = g.pass ? pitch : p.K;
    p.wb = p.b_kc ? p.K : p.N;
    g.plan_lhs = plan_product(p);
    if ((rc = check_product(p, g.plan_lhs))) return rc;
    g.lhs_bytes = align_up(g.plan_lhs.bytes());
  }
  if (g.rhs) {                     // d_rhs = lhs^T dz: k x n (column-major: its transpose, dz^T lhs), the sum over m
    Product& p = g.by_rhs;
    const Side lhs{d.lhs.data, d.lhs.layout == MRL_COLUMN_MAJOR, d.lhs.ld, d.lhs.batch}, z{dz.data, 0, dz.ld, dz.batch};
    const bool turned = d.d_rhs.layout == MRL_COLUMN_MAJOR;
    const Side &a = turned ? z : lhs, &b = turned ? lhs : z;
    p.a = a.data;
    p.b = b.data;
    p.bf16 = is_bf16;
    p.a_kc = a.kc;
    p.b_kc = b.kc;
    p.lda = a.ld;
    p.ldb = b.ld;
    p.batches = sum ? 1 : d.b;
    p.segs = sum ? d.b : 1;
    p.batch_a = p.seg_a = a.batch;
    p.batch_b = p.seg_b = b.batch;
    p.M = turned ? d.n : d.k;
    p.N = turned ? d.k : d.n;
    p.K = d.b ? d.m : 0;           // (of no batches there is nothing to sum, nor to copy)
    p.e.out = RowsOf{d.d_rhs.data, d.d_rhs.ld, d.d_rhs.batch, d.d_rhs.dtype == MRL_BF16};
    // batches whose rows follow each other are one sum
    if (sum && !lhs.kc && (uint64_t)lhs.batch == (uint64_t)d.m * (uint64_t)lhs.ld && (uint64_t)z.batch == (uint64_t)d.m * (uint64_t)z.ld) {
      p.K = d.b * d.m;
      p.segs = 1;
    }
    const uint32_t width_lhs = lhs.kc ? p.K : d.k, width_z = g.pass ? pitch : d.n;
    p.wa = turned ? width_z : width_lhs;
    p.wb = turned ? width_lhs : width_z;
    g.plan_rhs = plan_product(p);
    if ((rc = check_product(p, g.plan_rhs))) return rc;
    g.rhs_bytes = align_up(g.plan_rhs.bytes());
  }
  *out = g;
  return MRL_OK;
}

int32_t check_workspace(const void* d_workspace, size_t have, size_t need) {
  if (!need) return MRL_OK;
  if (have < need) return refuse(MRL_E_NOMEM, "workspace of %zu bytes, %zu are needed", have, need);
  CHECK(d_workspace && (uintptr_t)d_workspace % 256 == 0, "workspace is NULL or not aligned to 256 bytes");
  return MRL_OK;
}

}  // namespace

extern "C" {

int32_t mrl_linear_bytes(const mrl_linear_desc* desc, size_t* bytes) {
  CHECK(desc && bytes, "NULL argument");
  Product p;
  const int32_t rc = linear_product(*desc, &p);
  if (rc) return rc;
  *bytes = plan_product(p).bytes();
  return MRL_OK;
}

int32_t mrl_linear(const mrl_linear_desc* desc, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  CHECK(desc, "NULL argument");
  Product p;
  int32_t rc = linear_product(*desc, &p);
  if (rc) return rc;
  const ProductPlan plan = plan_product(p);
  if ((rc = check_product(p, plan))) return rc;
  if ((rc = check_workspace(d_workspace, workspace_bytes, plan.bytes()))) return rc;
  const hipStream_t st = (hipStream_t)hip_stream;
  hipError_t e = launch_product(p, plan, d_workspace, st);
  const Product* const products[2] = {&p, nullptr};
  const ProductPlan* const plans[2] = {&plan, nullptr};
  const float* const partials[2] = {plan.partial(d_workspace), nullptr};
  if (e == hipSuccess && plan.splits > 1) e = launch_rest(products, plans, partials, nullptr, nullptr, st);
  return hip_status(e);
}

int32_t mrl_linear_grad_bytes(const mrl_linear_grad_desc* desc, size_t* bytes) {
  CHECK(desc && bytes, "NULL argument");
  GradPlan g;
  const int32_t rc = plan_grad(*desc, &g);
  if (rc) return rc;
  *bytes = g.bytes();
  return MRL_OK;
}

int32_t mrl_linear_grad(const mrl_linear_grad_desc* desc, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  CHECK(desc, "NULL argument");
  GradPlan g;
  int32_t rc = plan_grad(*desc, &g);
  if (rc) return rc;
  if ((rc = check_workspace(d_workspace, workspace_bytes, g.bytes()))) return rc;
  float* const sums = (float*)((char*)d_workspace + g.dz_bytes);
  char* const for_lhs = (char*)sums + g.sums_bytes;
  char* const for_rhs = for_lhs + g.lhs_bytes;
  const hipStream_t st = (hipStream_t)hip_stream;
  if (g.pass) {
    g.rows.dz.data = d_workspace;
    g.by_lhs.a = d_workspace;
    (desc->d_rhs.layout == MRL_COLUMN_MAJOR ? g.by_rhs.a : g.by_rhs.b) = d_workspace;
  } else {
    g.rows.dz.data = nullptr;      // grad is dz
  }
  hipError_t e = hipSuccess;
  if (g.pass || g.rows.dbias) e = launch_grad_rows(g.rows, sums, st);
  if (e == hipSuccess && g.lhs) e = launch_product(g.by_lhs, g.plan_lhs, for_lhs, st);
  if (e == hipSuccess && g.rhs) e = launch_product(g.by_rhs, g.plan_rhs, for_rhs, st);
  const Product* const products[2] = {g.lhs ? &g.by_lhs : nullptr, g.rhs ? &g.by_rhs : nullptr};
  const ProductPlan* const plans[2] = {&g.plan_lhs, &g.plan_rhs};
  const float* const partials[2] = {g.plan_lhs.partial(for_lhs), g.plan_rhs.partial(for_rhs)};
  if (e == hipSuccess) e = launch_rest(products, plans, partials, &g.rows, sums, st);
  return hip_status(e);
}

int32_t mrl_dropout(const mrl_dropout_desc* desc, void* hip_stream) {
  CHECK(desc, "NULL argument");
  const mrl_dropout_desc& d = *desc;
  int32_t rc = check_common(1, d.m, 0, d.n, MRL_ACT_NONE, d.drop);
  if (!rc) rc = check_matrix("x", d.x, 1, d.m, d.n, false, false);
  if (!rc && d.residual.data) rc = check_matrix("residual", d.residual, 1, d.m, d.n, false, false);
  if (!rc) rc = check_matrix("out", d.out, 1, d.m, d.n, true, false);
  if (rc) return rc;
  return hip_status(launch_drop(DropRows{rows_of(d.x), rows_of(d.residual), rows_of(d.out), d.m, d.n, drop_of(d.drop, d.seed, d.offset)}, (hipStream_t)hip_stream));
}

}  // extern "C"
