// Layer normalisation of rows and its gradients (operators.h): kernels and launches.
//
//   mean = S x / n,  var = S (x - mean)^2 / n,  r = 1 / sqrt(var + eps),  h = (x - mean) r,  out = h w + b
//   g = grad w,  dx = residual + r (g - S g / n - h S(g h) / n),  dw = S_rows grad h,  db = S_rows grad
#include <hip/hip_runtime.h>

#include <algorithm>

#include "tiles.h"

namespace mrl {
namespace {

constexpr uint32_t kThreads = 1024;        // of a workgroup that goes over a row in passes
constexpr uint32_t kLaunchRows = kLaunch / (kThreads / 512);       // such workgroups of a launch

// The sums of two values over the workgroup, in every thread.  Their order is that of the threads.
__device__ __forceinline__ f32x2 sum_block(f32x2 v) {
  __shared__ f32x2 sums[kThreads / 64];
#pragma unroll
  for (int i = 32; i; i >>= 1) {
    v[0] += __shfl_xor(v[0], i);
    v[1] += __shfl_xor(v[1], i);
  }
  __syncthreads();                 // (the sums of the call before have been read)
  if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = v;
  __syncthreads();
  v = sums[0];
#pragma unroll
  for (uint32_t w = 1; w < kThreads / 64; w++) {
    v[0] += sums[w][0];
    v[1] += sums[w][1];
  }
  return v;
}

__device__ __forceinline__ int64_t start(const RowsOf& x, uint32_t row, uint32_t M, uint32_t batches) {
  const uint32_t batch = batches == 1 ? 0 : row / M;
  return (int64_t)batch * x.batch + (int64_t)(row - batch * M) * x.ld;
}

// 1 / sqrt(var + eps), given the mean of the squares of what `rest` is the mean of.  rest^2 is not rounded, nor infinite, by itself: where the squares' sum is, the
// variance is infinite and this is 0.  NaN stays.
__device__ __forceinline__ float inverse(float squares, float rest, float eps) {
  const float var = __builtin_fmaf(-rest, rest, squares);
  return 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps);
}

template <int CTRL>
__device__ __forceinline__ float moved(float x) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, true)); }
// The sum over sixteen neighbouring lanes, in each of them.
__device__ __forceinline__ float sum16(float x) {
  x += moved<0xB1>(x);             // lanes 1, 0, 3, 2
  x += moved<0x4E>(x);             // lanes 2, 3, 0, 1
  x += moved<0x141>(x);            // mirrored in eight
  return x + moved<0x140>(x);      // and in sixteen
}
// The sum over a wave, in every lane: the four sixteens' one after the other.
__device__ __forceinline__ float sum_wave(float x) {
  const int v = __float_as_int(sum16(x));
  return (__int_as_float(__builtin_amdgcn_readlane(v, 0)) + __int_as_float(__builtin_amdgcn_readlane(v, 16))) +
         (__int_as_float(__builtin_amdgcn_readlane(v, 32)) + __int_as_float(__builtin_amdgcn_readlane(v, 48)));
}

// ---- rows that are kept in registers
//
// A thread has eight neighbouring elements, R times.  Those that would end past the row are moved back to its last eight, so that no load waits for a
// branch; `skip` of them are then another thread's (8 or more: all) and count nothing.  Rows have eight elements at least.  WHOLE: a multiple of eight, so that
// skip is 0 or 8.
struct Chunk {
  uint32_t at, skip;
  __device__ __forceinline__ Chunk(uint32_t n, uint32_t N) : at(min(n, N - 8)), skip(n - min(n, N - 8)) {}
};

// Eight elements as they are stored.
template <class T> struct Raw {
  T v[8];
  __device__ __forceinline__ void load(const void* data, int64_t at) { __builtin_memcpy(v, (const T*)data + at, sizeof v); }
  template <bool WHOLE>
  __device__ __forceinline__ void clear(uint32_t skip) {
    if (WHOLE) {
      u32x4 w[sizeof v / 16];
      __builtin_memcpy(w, v, sizeof v);
#pragma unroll
      for (uint32_t i = 0; i < sizeof v / 16; i++)
#pragma unroll
        for (int e = 0; e < 4; e++) w[i][e] = skip ? 0u : w[i][e];
      __builtin_memcpy(v, w, sizeof v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; e++) v[e] = (uint32_t)e < skip ? (T)0.0f : v[e];
    }
  }
};
// Eight elements of either type, without a branch: bf16 takes the first 16 bytes of the two loads.  other: what takes their place where there is no data (the
// loads then go to `any`, 32 bytes that are there).
struct Either {
  u32x4 w[2];
  __device__ __forceinline__ void load(const void* data, uint32_t is_bf16, int64_t at, const void* any) {
    const char* const from = data ? (const char*)data + (at << (is_bf16 ? 1 : 2)) : (const char*)any;
    __builtin_memcpy(&w[0], from, 16);
    __builtin_memcpy(&w[1], from + (data && !is_bf16 ? 16 : 0), 16);
  }
  __device__ __forceinline__ void values(const void* data, uint32_t is_bf16, float other, float (&v)[8]) const {
    const uint32_t flat[8] = {w[0][0], w[0][1], w[0][2], w[0][3], w[1][0], w[1][1], w[1][2], w[1][3]};
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const uint32_t half = e & 1 ? w[0][e >> 1] & 0xFFFF0000u : w[0][e >> 1] << 16;
      v[e] = data ? __uint_as_float(is_bf16 ? half : flat[e]) : other;
    }
  }
};

constexpr uint32_t kRowThreads = 1024;     // of a workgroup that keeps rows
constexpr uint32_t kKeep = 2;              // R at most: rows of up to 16384 elements
constexpr uint32_t kNarrow = 128;          // elements of a row that sixteen lanes have

// Which threads a row has: LANES of them, 16 for rows of up to 128 elements, or 64 for `waves` waves.
template <int LANES>
struct Team {
  uint32_t waves, size, group, groups, t;          // threads of a row; the thread's row of the workgroup's; its place in it
  __device__ __forceinline__ Team(uint32_t waves) : waves(waves) {
    size = LANES == 64 ? waves * 64 : LANES;
    group = LANES == 64 ? (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / waves : threadIdx.x / LANES;
    groups = blockDim.x / size;
    t = threadIdx.x - group * size;
  }
  // The sums over the row's threads, in each of them, added in one order.  `sums` may be written again behind the next such exchange.
  __device__ __forceinline__ f32x2 sum(f32x2 v, f32x2* sums) const;
};
template <int LANES>
__device__ __forceinline__ f32x2 Team<LANES>::sum(f32x2 v, f32x2* sums) const {
  if (LANES == 16) return f32x2{sum16(v[0]), sum16(v[1])};
  v = f32x2{sum_wave(v[0]), sum_wave(v[1])};
  if (waves == 1) return v;
  if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = v;
  __syncthreads();
  v = f32x2{0.0f, 0.0f};
  for (uint32_t i = 0; i < waves; i++) {
    v[0] += sums[group * waves + i][0];
    v[1] += sums[group * waves + i][1];
  }
  return v;
}

// `waves` waves a row; a workgroup's groups of waves take a row each, then the rows that follow those of all workgroups.  Memory bounds it, so the next
// row's loads go out before this one's sums are made; weight and bias are read once.  8192 x 2048 in bf16 12.9 us, 5.2 TB/s (21.8 by workgroups of a row each whose loads wait
// for branches); f32 22.4 us, 6.0 TB/s.
template <class T, int R, int LANES, bool WHOLE>
__global__ __launch_bounds__(kRowThreads) void norm_rows_kernel(const NormRows p, uint32_t waves) {
  __shared__ f32x2 sums[2][kRowThreads / 64];
  const Team<LANES> team(waves);
  const uint32_t rows = p.batches * p.M, t = team.t, pitch = team.size * 8, stride = gridDim.x * team.groups;
  uint64_t row = (uint64_t)blockIdx.x * team.groups + team.group;
  Raw<T> next[R];
  const auto load = [&](uint64_t row) {
    const int64_t x = start(p.x, (uint32_t)min(row, rows - 1ull), p.M, p.batches);        // (past the last row it is read again)
#pragma unroll
    for (int i = 0; i < R; i++) next[i].load(p.x.data, x + Chunk(i * pitch + t * 8, p.N).at);
  };
  load(row);
  float w[R][8], b[R][8];
  {
    Either ew[R], eb[R];
    const void* const any = (const char*)p.x.data;         // (eight elements: 16 bytes of bf16, which both loads of Either take)
#pragma unroll
    for (int i = 0; i < R; i++) {
      const Chunk c(i * pitch + t * 8, p.N);
      ew[i].load(p.weight, p.weight_bf16, c.at, any);
      eb[i].load(p.bias, p.bias_bf16, c.at, any);
    }
#pragma unroll
    for (int i = 0; i < R; i++) {
      ew[i].values(p.weight, p.weight_bf16, 1.0f, w[i]);
      eb[i].values(p.bias, p.bias_bf16, 0.0f, b[i]);
    }
  }
  const float one = 1.0f / (float)p.N;
  const bool past = p.out.bf16 && goes_past((uint64_t)rows * p.N * 2);           // (f32, 32 bytes a lane, is not faster so)
  for (uint64_t row0 = row - team.group; row0 < rows; row0 += stride, row += stride) {
    float v[R][8];
    f32x2 s = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < R; i++)
#pragma unroll
      for (int e = 0; e < 8; e++) v[i][e] = (float)next[i].v[e];
    if (row0 + stride < rows) load(row + stride);
#pragma unroll
    for (int i = 0; i < R; i++) {
      const Chunk c(i * pitch + t * 8, p.N);
      if (WHOLE && c.skip) continue;
#pragma unroll
      for (int e = 0; e < 8; e++) s[0] += WHOLE || (uint32_t)e >= c.skip ? v[i][e] : 0.0f;
    }
    float about = team.sum(f32x2{s[0], 0.0f}, sums[0])[0] * one;
    asm volatile("" : "+v"(about));        // (rounded here and nowhere else: folded into the subtractions below it would be another number in each of them)
    // the sum of what is left puts the mean right: where it is far from 0, its own sum has lost that much
    s[0] = 0.0f;
#pragma unroll
    for (int i = 0; i < R; i++) {
      const Chunk c(i * pitch + t * 8, p.N);
#pragma unroll
      for (int e = 0; e < 8; e++) v[i][e] -= about;
      if (WHOLE && c.skip) continue;
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const float d = WHOLE || (uint32_t)e >= c.skip ? v[i][e] : 0.0f;
        s[0] += d;
        s[1] += d * d;
      }
    }
    s = team.sum(s, sums[1]);
    const float rest = s[0] * one, r = inverse(s[1] * one, rest, p.eps);
    if (row >= rows) continue;
    if (p.stats && t == 0) {
      p.stats[2 * row] = about + rest;
      p.stats[2 * row + 1] = r;
    }
    const int64_t out = start(p.out, (uint32_t)row, p.M, p.batches);
#pragma unroll
    for (int i = 0; i < R; i++) {
      const uint32_t n = i * pitch + t * 8;
      if (n >= p.N) continue;
#pragma unroll
      for (int e = 0; e < 8; e++) v[i][e] = (v[i][e] - rest) * r * w[i][e] + b[i][e];
      // (what is another thread's too is the same there)
      if (past) store8_past((bf16*)p.out.data + out + Chunk(n, p.N).at, v[i]);
      else store8(p.out.data, p.out.bf16, out + Chunk(n, p.N).at, 8, v[i]);
    }
  }
}

// ---- rows of fewer than eight elements: a row a thread (65536 x 4 in bf16 3.2 us; a workgroup a row took 943)

__global__ __launch_bounds__(256) void norm_few_kernel(const NormRows p, uint32_t first) {
  const uint64_t row = (uint64_t)(first + blockIdx.x) * 256 + threadIdx.x;
  if (row >= (uint64_t)p.batches * p.M) return;
  float v[8], w[8];
  load8(p.x.data, p.x.bf16, start(p.x, (uint32_t)row, p.M, p.batches), p.N, v);
  float about = 0.0f, rest = 0.0f, squares = 0.0f;
#pragma unroll
  for (uint32_t e = 0; e < 7; e++) about += e < p.N ? v[e] : 0.0f;
  about /= (float)p.N;
#pragma unroll
  for (uint32_t e = 0; e < 7; e++) {
    const float d = e < p.N ? v[e] - about : 0.0f;
    rest += d;
    squares += d * d;
  }
  rest /= (float)p.N;
  const float r = inverse(squares / (float)p.N, rest, p.eps);
  if (p.stats) {
    p.stats[2 * row] = about + rest;
    p.stats[2 * row + 1] = r;
  }
#pragma unroll
  for (int e = 0; e < 8; e++) v[e] = (v[e] - about - rest) * r;
  if (p.weight) {
    load8(p.weight, p.weight_bf16, 0, p.N, w);
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] *= w[e];
  }
  if (p.bias) {
    load8(p.bias, p.bias_bf16, 0, p.N, w);
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] += w[e];
  }
  store8(p.out.data, p.out.bf16, start(p.out, (uint32_t)row, p.M, p.batches), p.N, v);
}

__global__ __launch_bounds__(256) void norm_grad_few_kernel(const NormGrad p, uint32_t first) {
  const uint64_t at = (uint64_t)(first + blockIdx.x) * 256 + threadIdx.x;
  if (at >= (uint64_t)p.batches * p.M) return;
  const uint32_t row = (uint32_t)at;
  const float mean = p.stats[2 * at], r = p.stats[2 * at + 1];
  float h[8], g[8], w[8];
  load8(p.x.data, p.x.bf16, start(p.x, row, p.M, p.batches), p.N, h);
  load8(p.grad.data, p.grad.bf16, start(p.grad, row, p.M, p.batches), p.N, g);
  if (p.weight) {
    load8(p.weight, p.weight_bf16, 0, p.N, w);
#pragma unroll
    for (int e = 0; e < 8; e++) g[e] *= w[e];
  }
  float a = 0.0f, b = 0.0f;
#pragma unroll
  for (uint32_t e = 0; e < 7; e++) {
    h[e] = (h[e] - mean) * r;
    a += e < p.N ? g[e] : 0.0f;
    b += e < p.N ? g[e] * h[e] : 0.0f;
  }
  a /= (float)p.N;
  b /= (float)p.N;
#pragma unroll
  for (int e = 0; e < 8; e++) h[e] = r * (g[e] - a - h[e] * b);
  if (p.residual.data) {
    load8(p.residual.data, p.residual.bf16, start(p.residual, row, p.M, p.batches), p.N, w);
#pragma unroll
    for (int e = 0; e < 8; e++) h[e] += w[e];
  }
  store8(p.dx.data, p.dx.bf16, start(p.dx, row, p.M, p.batches), p.N, h);
}

// ---- rows that are longer than registers hold: a row a workgroup, in passes

// A thread's chunks of a pass, kAhead at a time.
constexpr uint32_t kAhead = 4;
__device__ __forceinline__ void load_chunks(const RowsOf& x, int64_t row, uint32_t n, uint32_t N, float (&v)[kAhead][8]) {
  const auto load = [&](auto type) {
    Raw<decltype(type)> t[kAhead];
#pragma unroll
    for (uint32_t u = 0; u < kAhead; u++) t[u].load(x.data, row + Chunk(n + u * kThreads * 8, N).at);
#pragma unroll
    for (uint32_t u = 0; u < kAhead; u++)
#pragma unroll
      for (int e = 0; e < 8; e++) v[u][e] = (float)t[u].v[e];
  };
  if (x.bf16) load(bf16());
  else load(float());
}
// Eight results, without the `skip` that are another thread's: in place of x that thread may have stored them before this one read them.
__device__ __forceinline__ void store_chunk(const RowsOf& x, int64_t row, const Chunk& c, const float (&v)[8]) {
  if (c.skip == 0) return store8(x.data, x.bf16, row + c.at, 8, v);
#pragma unroll
  for (uint32_t e = 1; e < 8; e++) {
    if (e < c.skip) continue;
    if (x.bf16) ((bf16*)x.data)[row + c.at + e] = (bf16)v[e];
    else ((float*)x.data)[row + c.at + e] = v[e];
  }
}

// Three passes over the row: 1000 x 20000 in f32 47 to 50 us, 4096 x 32768 337 (209 to read and write it once), 1 x 1048576 268 (what one compute unit loads bounds that).
__global__ __launch_bounds__(kThreads) void norm_kernel(const NormRows p, uint32_t first) {
  const uint32_t row = first + blockIdx.x;
  const int64_t x = start(p.x, row, p.M, p.batches), out = start(p.out, row, p.M, p.batches);
  const float N = (float)p.N;
  float v[kAhead][8];
  const auto over = [&](auto f) {
    for (uint32_t n = threadIdx.x * 8; n < p.N; n += kAhead * kThreads * 8) {
      load_chunks(p.x, x, n, p.N, v);
#pragma unroll
      for (uint32_t u = 0; u < kAhead; u++) f(Chunk(n + u * kThreads * 8, p.N), v[u]);
    }
  };
  f32x2 s = {0.0f, 0.0f};
  over([&](const Chunk& at, const float (&v)[8]) {
#pragma unroll
    for (uint32_t e = 0; e < 8; e++) s[0] += e >= at.skip ? v[e] : 0.0f;
  });
  const float about = sum_block(s)[0] / N;         // (and put right, as in norm_rows_kernel)
  s = f32x2{0.0f, 0.0f};
  over([&](const Chunk& at, const float (&v)[8]) {
#pragma unroll
    for (uint32_t e = 0; e < 8; e++) {
      const float d = e >= at.skip ? v[e] - about : 0.0f;
      s[0] += d;
      s[1] += d * d;
    }
  });
  s = sum_block(s);
  const float rest = s[0] / N, r = inverse(s[1] / N, rest, p.eps);
  if (p.stats && threadIdx.x == 0) {
    p.stats[2 * (uint64_t)row] = about + rest;
    p.stats[2 * (uint64_t)row + 1] = r;
  }
  over([&](const Chunk& at, float (&v)[8]) {
    if (at.skip >= 8) return;
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = (v[e] - about - rest) * r;
    if (p.weight) {
      load8(p.weight, p.weight_bf16, at.at, 8, w);
#pragma unroll
      for (int e = 0; e < 8; e++) v[e] *= w[e];
    }
    if (p.bias) {
      load8(p.bias, p.bias_bf16, at.at, 8, w);
#pragma unroll
      for (int e = 0; e < 8; e++) v[e] += w[e];
    }
    store_chunk(p.out, out, at, v);
  });
}

// dx: two passes over the row.  With the column sums before it 1000 x 20000 in f32 takes 98 us, 4096 x 32768 671 (313 to read and write it once), 1 x 1048576 340.
__global__ __launch_bounds__(kThreads) void norm_grad_kernel(const NormGrad p, uint32_t first) {
  const uint32_t row = first + blockIdx.x;
  const int64_t x = start(p.x, row, p.M, p.batches), grad = start(p.grad, row, p.M, p.batches), dx = start(p.dx, row, p.M, p.batches);
  const float mean = p.stats[2 * (uint64_t)row], r = p.stats[2 * (uint64_t)row + 1];
  float h[kAhead][8], g[kAhead][8];
  const auto over = [&](auto f) {                  // f(place, h, g)
    for (uint32_t n = threadIdx.x * 8; n < p.N; n += kAhead * kThreads * 8) {
      load_chunks(p.x, x, n, p.N, h);
      load_chunks(p.grad, grad, n, p.N, g);
#pragma unroll
      for (uint32_t u = 0; u < kAhead; u++) {
        const Chunk at(n + u * kThreads * 8, p.N);
        if (at.skip >= 8) continue;
#pragma unroll
        for (int e = 0; e < 8; e++) h[u][e] = (h[u][e] - mean) * r;
        if (p.weight) {
          float w[8];
          load8(p.weight, p.weight_bf16, at.at, 8, w);
#pragma unroll
          for (int e = 0; e < 8; e++) g[u][e] *= w[e];
        }
        f(at, h[u], g[u]);
      }
    }
  };
  f32x2 s = {0.0f, 0.0f};
  over([&](const Chunk& at, const float (&h)[8], const float (&g)[8]) {
#pragma unroll
    for (uint32_t e = 0; e < 8; e++) {
      s[0] += e >= at.skip ? g[e] : 0.0f;
      s[1] += e >= at.skip ? g[e] * h[e] : 0.0f;
    }
  });
  s = sum_block(s);
  const float a = s[0] / (float)p.N, b = s[1] / (float)p.N;
  over([&](const Chunk& at, float (&h)[8], const float (&g)[8]) {
#pragma unroll
    for (int e = 0; e < 8; e++) h[e] = r * (g[e] - a - h[e] * b);
    if (p.residual.data) {
      float y[8];
      load8(p.residual.data, p.residual.bf16, start(p.residual, row, p.M, p.batches) + at.at, 8, y);
#pragma unroll
      for (int e = 0; e < 8; e++) h[e] += y[e];
    }
    store_chunk(p.dx, dx, at, h);
  });
}

// The gradient of such rows: each workgroup's groups take its `each` rows in turn and keep the columns' sums, which they add in their order at the end.
// partial: the workgroups' sums (2 x N each: dw, db), nullptr where there is one workgroup.  8192 x 2048 in bf16 with a residual 28 us, and 3.9 for norm_sums_kernel, of 26
// that memory takes for what has to be read and written.
template <class TX, class TG, int R, int LANES, bool WHOLE>
__global__ __launch_bounds__(kRowThreads) void norm_grad_rows_kernel(const NormGrad p, uint32_t waves, uint32_t each, uint32_t first, float* __restrict__ partial) {
  constexpr bool AHEAD = R == 1 || (WHOLE && sizeof(TX) + sizeof(TG) == 4);      // (else there are no registers for it)
  __shared__ f32x2 sums[2][kRowThreads / 64];
  __shared__ float columns[R == 1 ? 2 * kRowThreads * 8 : 8];            // (rows of two chunks a thread take all waves)
  const uint32_t block = first + blockIdx.x, rows = p.batches * p.M;
  const Team<LANES> team(waves);
  const uint32_t group = team.group, groups = team.groups, t = team.t, pitch = team.size * 8;
  const uint64_t begin = (uint64_t)block * each;
  const uint32_t end = (uint32_t)min(begin + each, (uint64_t)rows);
  const bool wants = p.dweight || p.dbias;

  Raw<TX> x1[R];
  Raw<TG> g1[R];
  float mean1 = 0.0f, r1 = 0.0f;
  const auto load = [&](uint32_t at) {
    const uint32_t row = min(at, end - 1);         // (past the last row it is read again)
    const int64_t at_x = start(p.x, row, p.M, p.batches), at_g = start(p.grad, row, p.M, p.batches);
    mean1 = p.stats[2 * (uint64_t)row];
    r1 = p.stats[2 * (uint64_t)row + 1];
#pragma unroll
    for (int i = 0; i < R; i++) {
      const Chunk c(i * pitch + t * 8, p.N);
      x1[i].load(p.x.data, at_x + c.at);
      g1[i].load(p.grad.data, at_g + c.at);
    }
  };
  float w[R][8], dw[R][8], db[R][8];
#pragma unroll
  for (int i = 0; i < R; i++)
#pragma unroll
    for (int e = 0; e < 8; e++) { w[i][e] = 1.0f; dw[i][e] = db[i][e] = 0.0f; }
  if (begin < end) {
    if (AHEAD) load((uint32_t)begin + group);
    if (p.weight) {
      Either ew[R];
#pragma unroll
      for (int i = 0; i < R; i++) ew[i].load(p.weight, p.weight_bf16, Chunk(i * pitch + t * 8, p.N).at, p.weight);
#pragma unroll
      for (int i = 0; i < R; i++) ew[i].values(p.weight, p.weight_bf16, 1.0f, w[i]);
    }
  }
  const float one = 1.0f / (float)p.N;
  uint32_t turn = 0;
  for (uint64_t row0 = begin; row0 < end; row0 += groups, turn ^= 1) {
    const uint32_t row = (uint32_t)row0 + group;
    if (!AHEAD) load(row);
    Raw<TX> x[R];
    Raw<TG> g[R];
    const float mean = mean1, r = r1;
#pragma unroll
    for (int i = 0; i < R; i++) {
      x[i] = x1[i];
      g[i] = g1[i];
      g[i].template clear<WHOLE>(Chunk(i * pitch + t * 8, p.N).skip);
    }
    if (AHEAD && row0 + groups < end) load(row + groups);
    float s0 = 0.0f, s1 = 0.0f;
    if (row < end) {
#pragma unroll
      for (int i = 0; i < R; i++)
#pragma unroll
        for (int e = 0; e < 8; e++) {
          const float grad = (float)g[i].v[e], h = ((float)x[i].v[e] - mean) * r, gw = grad * w[i][e];
          s0 += gw;
          s1 += gw * h;
          dw[i][e] += grad * h;
          db[i][e] += grad;
        }
    }
    if (!p.dx.data) continue;
    Either z[R];
    if (p.residual.data && row < end) {            // (asked for before the sums go around)
      const int64_t at = start(p.residual, row, p.M, p.batches);
#pragma unroll
      for (int i = 0; i < R; i++) z[i].load(p.residual.data, p.residual.bf16, at + Chunk(i * pitch + t * 8, p.N).at, p.residual.data);
    }
    const f32x2 s = team.sum(f32x2{s0, s1}, sums[turn]);
    if (row >= end) continue;
    const float a = s[0] * one, b = s[1] * one;
    const int64_t dx = start(p.dx, row, p.M, p.batches);
#pragma unroll
    for (int i = 0; i < R; i++) {
      const Chunk c(i * pitch + t * 8, p.N);
      if (c.skip >= 8) continue;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; e++) v[e] = r * ((float)g[i].v[e] * w[i][e] - a - ((float)x[i].v[e] - mean) * r * b);
      if (p.residual.data) {
        float y[8];
        z[i].values(p.residual.data, p.residual.bf16, 0.0f, y);
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] += y[e];
      }
      if (WHOLE || c.skip == 0) {
        store8(p.dx.data, p.dx.bf16, dx + c.at, 8, v);
        // (past the caches, 8192 x 2048 takes 35.9 us instead of 34.8 from memory and 29.9 instead of 30.7 from the cache there; with mx_quantize of d_x behind it 45.0 instead
        // of 43.0, and 41.9 instead of 40.7)
      } else {
#pragma unroll
        for (int e = 1; e < 8; e++) {
          if ((uint32_t)e < c.skip) continue;
          if (p.dx.bf16) ((bf16*)p.dx.data)[dx + c.at + e] = (bf16)v[e];
          else ((float*)p.dx.data)[dx + c.at + e] = v[e];
        }
      }
    }
  }
  if (!wants) return;
  float* const mine = partial + (uint64_t)block * 2 * p.N;
  if (R == 1 && groups > 1) {      // a column a thread, the groups' sums in their order
    float* const at = columns + group * pitch + t * 8;
#pragma unroll
    for (int e = 0; e < 8; e++) { at[e] = dw[0][e]; at[kRowThreads * 8 + e] = db[0][e]; }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < 2 * pitch; i += blockDim.x) {
      const uint32_t which = i >= pitch, n = i - which * pitch;
      const Chunk c(n & ~7u, p.N);
      if ((n & 7) < c.skip) continue;
      float s = 0.0f;
      for (uint32_t k = 0; k < groups; k++) s += columns[which * kRowThreads * 8 + k * pitch + n];
      const uint32_t column = c.at + (n & 7), is_bf16 = which ? p.dbias_bf16 : p.dweight_bf16;
      void* const to = which ? p.dbias : p.dweight;
      if (partial) mine[which * p.N + column] = s;
      else if (to && is_bf16) ((bf16*)to)[column] = (bf16)s;
      else if (to) ((float*)to)[column] = s;
    }
    return;
  }
  const auto put = [&](void* to, uint32_t is_bf16, const Chunk& c, const float (&v)[8]) {
    if (!to) return;
    if (c.skip == 0) return store8(to, is_bf16, (int64_t)c.at, 8, v);
#pragma unroll
    for (int e = 1; e < 8; e++) {
      if ((uint32_t)e < c.skip) continue;
      if (is_bf16) ((bf16*)to)[c.at + e] = (bf16)v[e];
      else ((float*)to)[c.at + e] = v[e];
    }
  };
#pragma unroll
  for (int i = 0; i < R; i++) {
    const Chunk c(i * pitch + t * 8, p.N);
    if (c.skip >= 8) continue;
    put(partial ? mine : p.dweight, partial ? 0 : p.dweight_bf16, c, dw[i]);
    put(partial ? mine + p.N : p.dbias, partial ? 0 : p.dbias_bf16, c, db[i]);
  }
}

// The sums over columns alone, for rows too long for registers: 256 columns, eight a thread, `each` rows, eight at a time.
__global__ __launch_bounds__(256) void norm_columns_kernel(const NormGrad p, uint32_t each, uint32_t first, float* __restrict__ partial) {
  __shared__ float sums[2][8][256];
  const uint32_t blocks_n = (p.N + 255) / 256, id = first + blockIdx.x, bn = id % blocks_n, br = id / blocks_n;
  const uint32_t c = threadIdx.x & 31, l = threadIdx.x >> 5, n = bn * 256 + c * 8, rows = p.batches * p.M;
  float dw[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f}, db[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  if (n < p.N) {
    for (uint32_t i = l; i < each; i += 8) {
      const uint64_t at = (uint64_t)br * each + i;
      if (at >= rows) break;
      const uint32_t row = (uint32_t)at;
      float x[8], g[8];
      load8(p.grad.data, p.grad.bf16, start(p.grad, row, p.M, p.batches) + n, p.N - n, g);
#pragma unroll
      for (int e = 0; e < 8; e++) db[e] += g[e];
      if (!p.dweight) continue;
      load8(p.x.data, p.x.bf16, start(p.x, row, p.M, p.batches) + n, p.N - n, x);
      const float mean = p.stats[2 * at], r = p.stats[2 * at + 1];
#pragma unroll
      for (int e = 0; e < 8; e++) dw[e] += g[e] * ((x[e] - mean) * r);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; e++) { sums[0][l][c * 8 + e] = dw[e]; sums[1][l][c * 8 + e] = db[e]; }
  __syncthreads();
  const uint32_t at = bn * 256 + threadIdx.x;
  if (at >= p.N) return;
  float s[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < 8; i++) { s[0] += sums[0][i][threadIdx.x]; s[1] += sums[1][i][threadIdx.x]; }
  if (partial) {
    partial[(uint64_t)br * 2 * p.N + at] = s[0];
    partial[((uint64_t)br * 2 + 1) * p.N + at] = s[1];
    return;
  }
  if (p.dweight && p.dweight_bf16) ((bf16*)p.dweight)[at] = (bf16)s[0];
  else if (p.dweight) ((float*)p.dweight)[at] = s[0];
  if (p.dbias && p.dbias_bf16) ((bf16*)p.dbias)[at] = (bf16)s[1];
  else if (p.dbias) ((float*)p.dbias)[at] = s[1];
}

// dw and db from `blocks` workgroups' sums: 32 columns of the two side by side, 32 workgroups' at a time.
__global__ __launch_bounds__(1024) void norm_sums_kernel(const NormGrad p, uint32_t blocks, const float* __restrict__ partial) {
  __shared__ float sums[32][33];
  const uint32_t c = threadIdx.x & 31, l = threadIdx.x >> 5;
  const uint64_t at = (uint64_t)blockIdx.x * 32 + c;
  float s = 0.0f;
  if (at < 2ull * p.N) {
#pragma unroll 8
    for (uint32_t i = l; i < blocks; i += 32) s += partial[(uint64_t)i * 2 * p.N + at];
  }
  sums[l][c] = s;
  __syncthreads();
  if (l || at >= 2ull * p.N) return;
  for (int i = 1; i < 32; i++) s += sums[i][c];
  const uint32_t n = (uint32_t)(at < p.N ? at : at - p.N), is_bf16 = at < p.N ? p.dweight_bf16 : p.dbias_bf16;
  void* const to = at < p.N ? p.dweight : p.dbias;
  if (!to) return;
  if (is_bf16) ((bf16*)to)[n] = (bf16)s;
  else ((float*)to)[n] = s;
}

// How a gradient is launched, by its sizes alone (and whether column sums are wanted).  A workgroup a compute unit where they are: more of them write and read more sums, and
// take longer from the start (8192 x 2048 in bf16 256 workgroups 34 us, 512 36, 1024 42; 4096 x 16384 99, 108, 141).
struct GradPlan {
  uint32_t keep, waves, groups;            // R and the waves of a row (0: too long to be kept), rows at a time of a workgroup
  uint32_t each, blocks;                   // rows of a workgroup (of a block of rows), how many of them
};
GradPlan plan_grad(const NormGrad& p) {
  const uint64_t rows = (uint64_t)p.batches * p.M;
  const bool sums = p.dweight || p.dbias;
  GradPlan g{};
  if (p.N >= 8 && p.N <= kRowThreads * 8 * kKeep) {
    g.keep = p.N <= kRowThreads * 8 ? 1 : 2;
    g.waves = (p.N + 512 * g.keep - 1) / (512 * g.keep);
    g.groups = kRowThreads / (p.N <= kNarrow ? 16 : 64 * g.waves);
    const uint64_t want = sums ? 256 : 4096;                   // workgroups
    g.each = (uint32_t)((rows + want * g.groups - 1) / (want * g.groups)) * g.groups;
    // Up to four rows a group are one workgroup's, which saves the second launch where there are sums: 16 x 1024 in bf16 6.8 us, spread over workgroups 7.4; where a row is narrow or
    // takes all waves it costs time, 4 x 16384 14.9 and 10.7, 64 x 512 8.6 and 6.9, 256 x 128 8.2 and 6.5, and d_x alone has no second launch to save: 12.7 and 5.3, 7.6 and 3.8, 7.3 and 3.5.
    if (rows <= 4 * g.groups) g.each = 4 * g.groups;
  } else {
    const uint64_t blocks_n = (p.N + 255) / 256;
    g.each = 64;
    while (g.each < rows && (rows + g.each - 1) / g.each * blocks_n > 4096) g.each *= 2;
  }
  if (!g.each) g.each = 8;
  g.blocks = rows ? (uint32_t)((rows + g.each - 1) / g.each) : 1;           // (of no rows the sums are 0)
  return g;
}

template <class TX, class TG>
hipError_t launch_rows(const NormGrad& p, const GradPlan& g, float* partial, hipStream_t st) {
  return in_launches(g.blocks, [&](uint64_t first, uint32_t n) {
    const auto go = [&](auto kernel) { kernel<<<n, g.groups * (p.N <= kNarrow ? 16 : 64 * g.waves), 0, st>>>(p, g.waves, g.each, (uint32_t)first, g.blocks > 1 ? partial : nullptr); };
    // (rows of two types, and narrow ones, are taken to end anywhere)
    constexpr bool MAY = sizeof(TX) == sizeof(TG);
    const bool whole = MAY && p.N % 8 == 0;
    if (p.N <= kNarrow) go(norm_grad_rows_kernel<TX, TG, 1, 16, false>);
    else if (g.keep == 1) whole ? go(norm_grad_rows_kernel<TX, TG, 1, 64, MAY>) : go(norm_grad_rows_kernel<TX, TG, 1, 64, false>);
    else whole ? go(norm_grad_rows_kernel<TX, TG, 2, 64, MAY>) : go(norm_grad_rows_kernel<TX, TG, 2, 64, false>);
  });
}

// How rows are normalised: two chunks a thread where a wave would have more than one (8192 x 2048 in bf16 16.2 us with one, 14.2 with two; 32768 x 512 13.8 and 16).
struct NormPlan { uint32_t keep, waves, groups, blocks; };     // keep: R, 0: too long (or short) to be kept
NormPlan plan_norm(uint64_t rows, uint32_t N) {
  NormPlan g{};
  if (N < 8 || N > kRowThreads * 8 * kKeep) return g;
  g.keep = N <= 512 ? 1 : 2;
  g.waves = (N + 512 * g.keep - 1) / (512 * g.keep);
  g.groups = N <= kNarrow ? 16 : std::max(1u, 4 / g.waves);
  const uint32_t waves = N <= kNarrow ? 4 : g.groups * g.waves;
  g.blocks = (uint32_t)std::min<uint64_t>((rows + g.groups - 1) / g.groups, 8192 / waves);        // (as many waves as the card has room for)
  return g;
}

template <class T>
void launch_norm_rows(const NormRows& p, const NormPlan& g, hipStream_t st) {
  const auto go = [&](auto kernel) { kernel<<<g.blocks, g.groups * (p.N <= kNarrow ? 16 : 64 * g.waves), 0, st>>>(p, g.waves); };
  const bool whole = p.N % 8 == 0;
  if (p.N <= kNarrow) go(norm_rows_kernel<T, 1, 16, false>);
  else if (g.keep == 1) whole ? go(norm_rows_kernel<T, 1, 64, true>) : go(norm_rows_kernel<T, 1, 64, false>);
  else whole ? go(norm_rows_kernel<T, 2, 64, true>) : go(norm_rows_kernel<T, 2, 64, false>);
}

}  // namespace

hipError_t launch_norm(const NormRows& p, hipStream_t st) {
  const uint64_t rows = (uint64_t)p.batches * p.M;
  if (!p.N || !rows) return hipSuccess;
  const NormPlan g = plan_norm(rows, p.N);
  if (p.N < 8) return in_launches((rows + 255) / 256, [&](uint64_t first, uint32_t n) { norm_few_kernel<<<n, 256, 0, st>>>(p, (uint32_t)first); });
  if (!g.keep) return in_launches(rows, [&](uint64_t first, uint32_t n) { norm_kernel<<<n, kThreads, 0, st>>>(p, (uint32_t)first); }, kLaunchRows);
  if (p.x.bf16) launch_norm_rows<bf16>(p, g, st);
  else launch_norm_rows<float>(p, g, st);
  return hipGetLastError();
}

uint64_t norm_grad_bytes(const NormGrad& p) {
  if (!p.dweight && !p.dbias) return 0;
  const GradPlan g = plan_grad(p);
  return g.blocks > 1 ? (uint64_t)g.blocks * 2 * p.N * 4 : 0;
}

hipError_t launch_norm_grad(const NormGrad& p, float* partial, hipStream_t st) {
  const bool sums = p.dweight || p.dbias;
  if (!p.N || (!sums && !p.dx.data)) return hipSuccess;
  const GradPlan g = plan_grad(p);
  hipError_t e = hipSuccess;
  if (g.keep) {
    if (p.x.bf16) e = p.grad.bf16 ? launch_rows<bf16, bf16>(p, g, partial, st) : launch_rows<bf16, float>(p, g, partial, st);
    else e = p.grad.bf16 ? launch_rows<float, bf16>(p, g, partial, st) : launch_rows<float, float>(p, g, partial, st);
  } else {
    // (the sums first: d_x may be x or grad itself)
    if (sums) e = in_launches((uint64_t)g.blocks * ((p.N + 255) / 256), [&](uint64_t first, uint32_t n) {
      norm_columns_kernel<<<n, 256, 0, st>>>(p, g.each, (uint32_t)first, g.blocks > 1 ? partial : nullptr);
    });
    const uint64_t rows = (uint64_t)p.batches * p.M;
    if (e == hipSuccess && p.dx.data && p.N < 8)
      e = in_launches((rows + 255) / 256, [&](uint64_t first, uint32_t n) { norm_grad_few_kernel<<<n, 256, 0, st>>>(p, (uint32_t)first); });
    else if (e == hipSuccess && p.dx.data)
      e = in_launches(rows, [&](uint64_t first, uint32_t n) { norm_grad_kernel<<<n, kThreads, 0, st>>>(p, (uint32_t)first); }, kLaunchRows);
  }
  if (e == hipSuccess && sums && g.blocks > 1) {
    norm_sums_kernel<<<(uint32_t)((2ull * p.N + 31) / 32), 1024, 0, st>>>(p, g.blocks, partial);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace mrl
