// Internal: the operators on data (include/morello_mi355x.h, mrl_linear and what follows): what the
// kernels get, the random bits of a dropout, the activations, and loads and stores of eight neighbouring elements.
#pragma once
#include <stdint.h>
#include <string.h>
#include <hip/hip_runtime.h>

namespace mrl {

using bf16 = __bf16;
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

enum : uint32_t { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };

// A matrix of rows as an epilogue reads or writes it: unit stride along n.
struct RowsOf {
  void* data;          // nullptr: there is none
  int64_t ld, batch;   // elements from a row to the next, from a batch to the next
  uint32_t bf16;       // 1 bf16, 0 f32
};

// D: an element whose 16 random bits are below `drop` counts 0, any other `scale`.  drop = 0: there is no dropout.
struct Drop {
  uint32_t drop;
  float scale;
  uint32_t seed[2], offset[2];
};

// out = residual + D f(z), z = sum + bias
struct Epilogue {
  RowsOf out, residual, pre;
  const void* bias;
  uint32_t bias_bf16, activation;
  Drop drop;
};

// The 16 random bits of elements (row, 8 group .. 8 group + 7), two to a word, the first in the low half: Philox4x32
// with seven rounds (Salmon, Moraes, Dror, Shaw: Parallel random numbers, as easy as 1, 2, 3; SC 2011), the fewest
// with which they found it to pass every test of their batteries.  16 bits an element: the probability is a multiple of 2^-16 and the scale
// is the inverse of exactly that, so the expectation is kept; with 32 bits an element a block serves four elements and the
// generator, not memory, bounds the kernel (14 wide products, a quarter of the rate of other operations, per block).
__device__ __forceinline__ u32x4 random_block(const Drop& d, uint32_t row, uint32_t group) {
  uint32_t c0 = group, c1 = row, c2 = d.offset[0], c3 = d.offset[1], k0 = d.seed[0], k1 = d.seed[1];
#pragma unroll
  for (int r = 0; r < 7; r++) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return u32x4{c0, c1, c2, c3};
}

// v <- D v.  A dropped element is 0 whatever it was (a product would keep NaN and infinities).
__device__ __forceinline__ void drop8(const Drop& d, uint32_t row, uint32_t n0, float (&v)[8]) {
  const u32x4 w = random_block(d, row, n0 >> 3);
#pragma unroll
  for (int e = 0; e < 8; e++) {
    const uint32_t bits = e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xFFFFu;
    v[e] = bits < d.drop ? 0.0f : v[e] * d.scale;
  }
}

// The logistic function of z, given -z / ln 2; 2^x overflows to infinity for very negative z, which gives the right 0.
__device__ __forceinline__ float logistic(float x) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x)); }

// GELU in its tanh form is z times the logistic function of 2 u, u = sqrt(2 / pi) (z + 0.044715 z^3), since
// (1 + tanh u) / 2 = logistic(2 u).
constexpr float kGelu = 1.5957691216057308f, kGelu3 = 0.07135481627159741f;      // 2 sqrt(2 / pi), and 0.044715 of that
constexpr float kLog2e = 1.4426950408889634f;

// v <- f(v).  A product with a logistic value of 0 would be NaN for z = -inf, where the limit is 0.  (Each branch holds all eight
// elements: a branch per element keeps their exponentials from overlapping, 60 us instead of 18 on 134 M elements.)
__device__ __forceinline__ void activate8(uint32_t act, float (&v)[8]) {
  if (act == kActGelu) {
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const float z = v[e], s = logistic(z * (-kLog2e * kGelu - kLog2e * kGelu3 * (z * z)));
      v[e] = s == 0.0f ? 0.0f : z * s;
    }
  } else if (act == kActSilu) {
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const float z = v[e], s = logistic(-kLog2e * z);
      v[e] = s == 0.0f ? 0.0f : z * s;
    }
  } else if (act == kActRelu) {
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = v[e] < 0.0f ? 0.0f : v[e];       // (NaN stays)
  }
}

// v <- v f'(z).  The logistic value s times 1 - s falls off faster than any power of z grows, so where either is 0 the second
// term of s + z u s (1 - s) is 0 too.  ReLU selects: where z <= 0 the result is 0 whatever v is (a product would keep NaN and infinities);
// where z is NaN it is NaN, as f(z) is.
__device__ __forceinline__ void slope8(uint32_t act, const float (&z)[8], float (&v)[8]) {
  if (act == kActGelu) {
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const float z2 = z[e] * z[e], s = logistic(z[e] * (-kLog2e * kGelu - kLog2e * kGelu3 * z2)), t = s * (1.0f - s);
      v[e] *= t == 0.0f ? s : s + z[e] * (kGelu + 3.0f * kGelu3 * z2) * t;
    }
  } else if (act == kActSilu) {
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const float s = logistic(-kLog2e * z[e]), t = s * (1.0f - s);
      v[e] *= t == 0.0f ? s : s + z[e] * t;
    }
  } else if (act == kActRelu) {
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = z[e] > 0.0f ? v[e] : z[e] == z[e] ? 0.0f : z[e];
  }
}

// Eight elements from p on, of which `valid` are there (the others come as 0).  Rows may start at any element: the hardware
// takes wide loads and stores at any address.
template <class T>
__device__ __forceinline__ void load8(const T* p, uint32_t valid, float (&v)[8]) {
  if (valid >= 8) {
    T t[8];
    __builtin_memcpy(t, p, sizeof t);
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = (float)t[e];
  } else {
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = (uint32_t)e < valid ? (float)p[e] : 0.0f;
  }
}
template <class T>
__device__ __forceinline__ void store8(T* p, uint32_t valid, const float (&v)[8]) {
  if (valid >= 8) {
    T t[8];
#pragma unroll
    for (int e = 0; e < 8; e++) t[e] = (T)v[e];
    __builtin_memcpy(p, t, sizeof t);
  } else {
#pragma unroll
    for (int e = 0; e < 8; e++) if ((uint32_t)e < valid) p[e] = (T)v[e];
  }
}
__device__ __forceinline__ void load8(const void* data, uint32_t is_bf16, int64_t at, uint32_t valid, float (&v)[8]) {
  if (is_bf16) load8((const bf16*)data + at, valid, v);
  else load8((const float*)data + at, valid, v);
}
__device__ __forceinline__ void store8(void* data, uint32_t is_bf16, int64_t at, uint32_t valid, const float (&v)[8]) {
  if (is_bf16) store8((bf16*)data + at, valid, v);
  else store8((float*)data + at, valid, v);
}

// The epilogue of eight sums: elements (batch, m, n0 .. n0 + 7), n0 a multiple of 8; rows of one batch: M; bias: these columns'.  The sums and all
// that is done to them are f32 and rounded once, to the type of what is stored.
__device__ __forceinline__ void bias8(const Epilogue& e, uint32_t n0, uint32_t valid, float (&b)[8]) {
  if (e.bias) {
    load8(e.bias, e.bias_bf16, n0, valid, b);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) b[i] = 0.0f;
  }
}
__device__ __forceinline__ void finish8(const Epilogue& e, uint32_t batch, uint32_t M, uint32_t m, uint32_t n0, uint32_t valid, const float (&bias)[8], float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i++) v[i] += bias[i];
  float r[8];
  if (e.residual.data) load8(e.residual.data, e.residual.bf16, (int64_t)batch * e.residual.batch + (int64_t)m * e.residual.ld + n0, valid, r);
  if (e.pre.data) store8(e.pre.data, e.pre.bf16, (int64_t)batch * e.pre.batch + (int64_t)m * e.pre.ld + n0, valid, v);
  activate8(e.activation, v);
  if (e.drop.drop) drop8(e.drop, batch * M + m, n0, v);
  if (e.residual.data) {
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] += r[i];
  }
  store8(e.out.data, e.out.bf16, (int64_t)batch * e.out.batch + (int64_t)m * e.out.ld + n0, valid, v);
}

// A product sum over k of A(m, k) B(k, n), for every batch, with an epilogue.  The sum may run over several segments of K
// (the batches of a gradient that they share).
struct Product {
  const void *a, *b;
  uint32_t bf16;                 // type of both
  uint32_t a_kc, b_kc;           // 1: neighbours along k are adjacent, 0: along m (n)
  int64_t lda, ldb;              // elements between lines: rows of A where a_kc, columns of A else; likewise B
  int64_t batch_a, batch_b;      // elements between batches
  int64_t seg_a, seg_b;          // and between segments
  uint32_t batches, segs, M, N, K;
  uint32_t wa, wb;               // elements of a line that are there: K, or M (N); more where a line is followed by zeros
  Epilogue e;
};

// How it is launched.
enum : uint32_t { kFast256, kFast256x128, kFast128, kFast128Alone, kFast64, kRows, kRowsWide, kWide128, kWide64, kAny64 };
struct ProductPlan {
  uint32_t kernel;
  uint32_t splits;               // workgroups along k
  uint32_t steps, per_split;     // steps of 128 bytes along k: in all, per split
  uint64_t blocks;               // workgroups
  // workspace, in this order: the operands' copies to lines that start at multiples of 16 bytes (0: not copied), the sums over splits
  uint64_t copy_a_bytes, copy_b_bytes, partial_bytes;
  uint64_t bytes() const { return copy_a_bytes + copy_b_bytes + partial_bytes; }
  float* partial(void* workspace) const { return (float*)((char*)workspace + copy_a_bytes + copy_b_bytes); }
};
ProductPlan plan_product(const Product& p);
hipError_t launch_product(const Product& p, const ProductPlan& plan, void* workspace, hipStream_t st);     // without the sum over splits

// dz = D f'(z) grad of `rows` x N elements (rows over all batches of M) and its column sums.
struct GradRows {
  RowsOf grad, pre, dz;
  uint32_t batches, M, N, activation;
  Drop drop;
  void* dbias;                   // nullptr: not wanted
  uint32_t dbias_bf16;
};
uint64_t grad_rows_bytes(uint32_t batches, uint32_t M, uint32_t N, bool dbias);
hipError_t launch_grad_rows(const GradRows& g, float* sums, hipStream_t st);       // dz, and the column sums of blocks of rows
// What is left, in one launch: the products' sums over splits (nullptr: no such product), dbias from the blocks' sums.
hipError_t launch_rest(const Product* const p[2], const ProductPlan* const plan[2], const float* const partial[2], const GradRows* rows, const float* sums, hipStream_t st);

// out = residual + D x
struct DropRows {
  RowsOf x, residual, out;
  uint32_t M, N;
  Drop drop;
};
hipError_t launch_drop(const DropRows& d, hipStream_t st);

// Layer normalisation of the rows of `batches` x M x N (N elements each), and what its gradient needs of them (mean, r) in `stats`, two f32 a row
struct NormRows {
  RowsOf x, out;
  const void *weight, *bias;     // nullptr: 1, 0
  uint32_t weight_bf16, bias_bf16;
  float* stats;                  // nullptr: not wanted
  uint32_t batches, M, N;
  float eps;
};
hipError_t launch_norm(const NormRows& p, hipStream_t st);

struct NormGrad {
  RowsOf grad, x, residual, dx;  // dx.data nullptr: not wanted
  const void* weight;
  const float* stats;
  void *dweight, *dbias;         // nullptr: not wanted
  uint32_t weight_bf16, dweight_bf16, dbias_bf16;
  uint32_t batches, M, N;
};
uint64_t norm_grad_bytes(const NormGrad& p);
hipError_t launch_norm_grad(const NormGrad& p, float* partial, hipStream_t st);

// `batches` matrices of `lines` lines of k values in blocks of 32 along k: 4 bits a value, a byte of scale a block (the header of the ABI has
// the format).  Lines are whole steps of 128 values, 64 bytes; scales come for 64 lines and a step at a time.
constexpr uint32_t mx_steps(uint32_t k) { return (k + 127) / 128; }
constexpr uint64_t mx_code_bytes(uint32_t lines, uint32_t k) { return (uint64_t)lines * mx_steps(k) * 64; }
constexpr uint64_t mx_scale_bytes(uint32_t lines, uint32_t k) { return ((uint64_t)lines + 63) / 64 * mx_steps(k) * 256; }

// between x and its blocks, either way.  kc: x's neighbours along k are adjacent (RowsOf's rows are lines), else those along the lines (its rows are k).
struct MxRows {
  RowsOf x;
  uint8_t *codes, *scales;
  uint32_t kc, batches, lines, k;
  uint32_t shared;               // blocks -> x: every batch is the same matrix
};
hipError_t launch_mx_quantize(const MxRows& p, hipStream_t st);
hipError_t launch_mx_dequantize(const MxRows& p, hipStream_t st);

// A product of operands in blocks.  p.a and p.b are codes, counted in units of four values (two bytes), K a multiple of 32 of them
struct MxProduct {
  Product p;
  MxRows lhs;                    // where x.data is given: a's values, which the kernel puts into blocks itself (mx_takes_rows)
  const uint8_t *scales_a, *scales_b;
  int64_t scales_batch_a, scales_batch_b;
  float* partial;                // (set by launch_mx)
};
ProductPlan plan_mx(const MxProduct& p);
bool mx_takes_rows(const MxProduct& p, const ProductPlan& plan, const MxRows& lhs);
hipError_t launch_mx(const MxProduct& p, const ProductPlan& plan, float* partial, hipStream_t st);       // without the sum over splits

int32_t fail_with(int32_t code, const char* message);      // sets mrl_last_error, returns code

}  // namespace mrl
