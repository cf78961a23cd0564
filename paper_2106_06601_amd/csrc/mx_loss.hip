// Softmax cross entropy over a vocabulary, and its gradient:
//
//     L = alpha X W^^T,  lse = log sum_j exp(L_j),  loss = lse - L_target
//     G_j = dloss (exp(L_j - lse) - [j = target])
//
// The products are the library's; these kernels are what stands between them, where the
// logits of a piece of the vocabulary are in memory (few rows, or a sum that is split).
// A row's statistics are kept by chunks of columns and joined by another kernel.  Bound by memory, or by
// launches: 13 rows over 65536 words 4.7 us and 4.6 joining; 4096 rows 8 joining 256 chunks.
#include <algorithm>

#include "mx_layer.hpp"
#include "mx_loss.hpp"
#include "mx_rows.hpp"

namespace costa {
namespace {

// Eight logits from column c of the piece on; those past it -infinity.
__device__ inline void logits8(const LogitsPart& p, int64_t row, int64_t c, float x[8]) {
  const float* part = p.sums + row * p.n + c;
  const bool all = c + 8 <= p.n;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = 0.0f;
  for (int s = 0; s < p.splits; ++s, part += p.m * p.n) {
    if (all) {
      float w[8];
      __builtin_memcpy(w, part, sizeof w);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] += w[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < p.n) x[i] += part[i];
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = c + i < p.n ? (p.splits > 0 ? p.alpha * x[i] : 0.0f) : -__builtin_inff();
}

// A workgroup has a chunk of a row, eight columns a lane.
__global__ __launch_bounds__(256) void loss_stats(LogitsPart p, LossStat* stats, float* at, int64_t row0,
                                                  int64_t chunk0) {
  __shared__ float red[2][4];
  const int64_t row = row0 + blockIdx.x, chunk = chunk0 + blockIdx.y, c = chunk * kLossChunk + threadIdx.x * 8;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  float x[8];
  logits8(p, row, c, x);
  float top = x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i]);
#pragma unroll
  for (int by = 32; by > 0; by /= 2) top = fmaxf(top, __shfl_xor(top, by));
  if (lane == 0) red[0][wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  const float from = top == -__builtin_inff() ? 0.0f : top;
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) sum += exp_of(x[i] - from);
#pragma unroll
  for (int by = 32; by > 0; by /= 2) sum += __shfl_xor(sum, by);
  if (lane == 0) red[1][wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) stats[chunk * p.m + row] = LossStat{top, (red[1][0] + red[1][1]) + (red[1][2] + red[1][3])};
  const int64_t t = p.target[row] - p.col0 - c;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (t == i && c + i < p.n) at[row] = x[i];
}

// A workgroup has 64 rows; 16 lanes of each take every 16th chunk, and one joins theirs.
__global__ __launch_bounds__(1024) void loss_join(int64_t m, int64_t n, int64_t chunks, const LossStat* stats,
                                                  const float* at, const int64_t* target, float* loss, float* lse) {
  __shared__ LossStat red[16][64];
  const int in = threadIdx.x % 64, mine = threadIdx.x / 64;
  for (int64_t row0 = (int64_t)blockIdx.x * 64; row0 < m; row0 += (int64_t)gridDim.x * 64) {
    const int64_t row = row0 + in;
    LossStat all{-__builtin_inff(), 0.0f};
    if (row < m)
#pragma unroll 4
      for (int64_t c = mine; c < chunks; c += 16) all = join_stats(all, stats[c * m + row]);
    red[mine][in] = all;
    __syncthreads();
    if (mine == 0 && row < m) {
#pragma unroll
      for (int i = 1; i < 16; ++i) all = join_stats(all, red[i][in]);
      const float tail = logf(all.sum);
      const int64_t t = target[row];
      lse[row] = all.top == -__builtin_inff() ? tail : all.top + tail;
      // (from the largest logit, not from lse: of a row that is nearly sure nothing is lost)
      loss[row] = t >= 0 && t < n ? (all.top - at[row]) + tail : 0.0f;
    }
    __syncthreads();
  }
}

template <int GSRC>
__global__ __launch_bounds__(256) void loss_grad(LogitsPart p, int64_t vocabulary, const float* lse,
                                                 const float* dloss, const float* factor, void* g) {
  const int64_t upr = (p.n + 7) / 8, units = p.m * upr;
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < units; u += (int64_t)gridDim.x * 256) {
    const int64_t row = ((u | upr) >> 32) == 0 ? (int64_t)((uint32_t)u / (uint32_t)upr) : u / upr, c = (u - row * upr) * 8;
    float x[8];
    logits8(p, row, c, x);
    const int64_t t = p.target[row];
    const bool counts = t >= 0 && t < vocabulary;
    const float d = counts ? (dloss ? dloss[row] : 1.0f) / (factor ? factor[row] : 1.0f) : 1.0f, l = lse[row];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = counts ? d * (exp_of(x[i] - l) - (t - p.col0 - c == i ? 1.0f : 0.0f)) : 0.0f;
    put8<GSRC>(static_cast<Elem<GSRC>*>(g) + row * p.n, c, p.n, x);
  }
}

// A wave has a row: the target's logit again, and from it how far the row is from sure.  Bound by reading x and the
// targets' rows of w: 4096 rows of 4096 in bfloat16 by 4 bits 9 us.
template <int SRC, int BITS, bool WIDE>
__global__ __launch_bounds__(256) void loss_factors(int64_t m, int64_t k, RowsView x, MxView w, float alpha,
                                                    const int64_t* target, const float* lse, const float* dloss,
                                                    float* factor) {
  const int lane = threadIdx.x % 64;
  for (int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 64; row < m; row += (int64_t)gridDim.x * 4) {
    const int64_t t = target[row];
    if (t < 0 || t >= w.rows) {
      if (lane == 0) factor[row] = 1.0f;
      continue;
    }
    const void* const xl = line_of<SRC>(x, row);
    const uint8_t* const data = w.data + t * w.row_bytes;
    const uint8_t* const scales = w.scales + t * w.row_scales;
    float sum = 0.0f;
#pragma unroll 4
    for (int64_t c = lane * 8; c < k; c += 512) {  // (a row of w is padded with zeros to whole steps of eight)
      Raw8<SRC> raw;
      get8<SRC, WIDE>(raw, xl, c, k);
      v2u d = {0u, 0u};
      if (BITS == 4) d.x = *reinterpret_cast<const uint32_t*>(data + c / 2);
      else d = *reinterpret_cast<const v2u*>(data + c);
      float a[8], b[8];
      mx_decode8<BITS>(d, scales[c / kMxBlock], b);
      floats8<SRC, WIDE>(raw, c, k, a);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(a[i], b[i], sum);
    }
#pragma unroll
    for (int by = 32; by > 0; by /= 2) sum += __shfl_xor(sum, by);
    const float rest = fminf(fmaxf(1.0f - exp_of(alpha * sum - lse[row]), 0x1p-24f), 1.0f);  // (NaN: 2^-24)
    const float f = (dloss ? __builtin_fabsf(dloss[row]) : 1.0f) * rest;
    if (lane == 0) factor[row] = f > 0.0f && f < __builtin_inff() ? f : 1.0f;
  }
}

__global__ __launch_bounds__(1024) void loss_scale(int64_t m, int64_t n, const int64_t* target, const float* dloss,
                                                   float* factor) {
  __shared__ uint32_t red[16];
  uint32_t top = 0;  // (magnitudes' bits: NaN above infinity above the finite ones)
  if (dloss)
#pragma unroll 8
    for (int64_t i = threadIdx.x; i < m; i += 1024) {
      const int64_t t = target[i];
      const uint32_t d = magnitude(dloss[i]);
      top = max(top, t >= 0 && t < n ? d : 0u);
    }
#pragma unroll
  for (int by = 32; by > 0; by /= 2) top = max(top, (uint32_t)__shfl_xor((int)top, by));
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, red[i]);
  const float all = top == 0 || top >= 0x7f800000u ? 1.0f : __builtin_bit_cast(float, top);
  for (int64_t i = threadIdx.x; i < m; i += 1024) factor[i] = all;
}

template <int SRC>
__global__ __launch_bounds__(256) void round_rows(int64_t m, int64_t n, const float* x, const float* factor, RowsView y) {
  const int64_t upr = (n + 7) / 8;
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < m * upr; u += (int64_t)gridDim.x * 256) {
    const int64_t row = u / upr, c = (u - row * upr) * 8;
    const float by = factor ? factor[row] : 1.0f;
    float v[8] = {};
    if (c + 8 <= n) __builtin_memcpy(v, x + row * n + c, sizeof v);
    else
      for (int i = 0; i < 8; ++i)
        if (c + i < n) v[i] = x[row * n + c + i];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= by;
    put8<SRC>(line_to<SRC>(y, row), c, n, v);
  }
}

constexpr int64_t kGroups = 1 << 20;
dim3 groups_for(int64_t units) { return dim3((unsigned)std::min(up_div(units, 256), kGroups)); }

}  // namespace

hipError_t launch_mx_loss_stats(const LogitsPart& p, LossStat* stats, float* at, hipStream_t stream) {
  constexpr int64_t kRows = 1 << 18, kChunks = 1 << 5;  // of a launch: below 2^32 lanes
  const int64_t chunks = up_div(p.n, kLossChunk);
  for (int64_t j = 0; j < chunks; j += kChunks)
    for (int64_t i = 0; i < p.m; i += kRows) {
      const dim3 grid((unsigned)std::min(kRows, p.m - i), (unsigned)std::min(kChunks, chunks - j));
      loss_stats<<<grid, 256, 0, stream>>>(p, stats, at, i, j);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  return hipSuccess;
}

hipError_t launch_mx_loss_join(int64_t m, int64_t n, int64_t chunks, const LossStat* stats, const float* at,
                               const int64_t* target, float* loss, float* lse, hipStream_t stream) {
  loss_join<<<dim3((unsigned)std::min<int64_t>(up_div(m, 64), 1 << 16)), 1024, 0, stream>>>(m, n, chunks, stats, at, target,
                                                                                          loss, lse);
  return hipGetLastError();
}

hipError_t launch_mx_loss_scale(int64_t m, int64_t n, const int64_t* target, const float* dloss, float* factor,
                                hipStream_t stream) {
  loss_scale<<<1, 1024, 0, stream>>>(m, n, target, dloss, factor);
  return hipGetLastError();
}

template <int SRC>
static void launch_factors(const ProductArgs& x, const int64_t* target, const float* lse, const float* dloss, float* factor,
                           hipStream_t stream) {
  const dim3 grid((unsigned)std::min<int64_t>(up_div(x.m, 4), 1 << 16));
  auto go = [&](auto bits, auto wide) {
    loss_factors<SRC, decltype(bits)::value, decltype(wide)::value><<<grid, 256, 0, stream>>>(
        x.m, x.k, RowsView{const_cast<void*>(x.real), x.a_rs}, x.b, x.alpha, target, lse, dloss, factor);
  };
  auto of = [&](auto bits) { x.k >= 8 ? go(bits, std::true_type{}) : go(bits, std::false_type{}); };
  if (x.b.bits == 4) of(std::integral_constant<int, 4>{});
  else of(std::integral_constant<int, 8>{});
}
hipError_t launch_mx_loss_factors(const ProductArgs& x, const int64_t* target, const float* lse, const float* dloss,
                                  float* factor, hipStream_t stream) {
  if (x.a_type == COSTA_REAL_BF16) launch_factors<SRC_BF16>(x, target, lse, dloss, factor, stream);
  else if (x.a_type == COSTA_REAL_F16) launch_factors<SRC_F16>(x, target, lse, dloss, factor, stream);
  else launch_factors<SRC_F32>(x, target, lse, dloss, factor, stream);
  return hipGetLastError();
}

hipError_t launch_mx_loss_grad(const LogitsPart& p, int64_t vocabulary, const float* lse, const float* dloss,
                               const float* factor, void* g, bool bf16, hipStream_t stream) {
  const dim3 grid = groups_for(p.m * up_div(p.n, 8));
  if (bf16) loss_grad<SRC_BF16><<<grid, 256, 0, stream>>>(p, vocabulary, lse, dloss, factor, g);
  else loss_grad<SRC_F32><<<grid, 256, 0, stream>>>(p, vocabulary, lse, dloss, factor, g);
  return hipGetLastError();
}

hipError_t launch_mx_round(int64_t m, int64_t n, const float* x, const float* factor, const RowsView& y, costa_real type,
                           hipStream_t stream) {
  const dim3 grid = groups_for(m * up_div(n, 8));
  if (type == COSTA_REAL_F32) round_rows<SRC_F32><<<grid, 256, 0, stream>>>(m, n, x, factor, y);
  else if (type == COSTA_REAL_BF16) round_rows<SRC_BF16><<<grid, 256, 0, stream>>>(m, n, x, factor, y);
  else round_rows<SRC_F16><<<grid, 256, 0, stream>>>(m, n, x, factor, y);
  return hipGetLastError();
}

}  // namespace costa
