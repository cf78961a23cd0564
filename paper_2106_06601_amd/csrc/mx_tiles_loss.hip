// Products with a vocabulary in tiles of the logits, whose sums go no further than a row's statistics or
// the gradient of the logits: they are never written.
//
// A lane has, of 16 MT rows, one of each sixteen and four neighbouring columns of each of NT
// pieces; a row's columns of a wave lie in four lanes.
//
// Measured, 4096 rows of 4096 in bfloat16 over 65536 words in 4 bits: statistics 1.81 ms (1.21 PFLOP/s), the gradient
// of the logits 2.03 ms, the product behind it 1.77; with the logits in memory 1.84 and 4 times 0.07 more,
// 1.84 and 4 times 0.10.  Bound by the matrix units as the products are (45% busy, at 2.0 to 2.2 GHz).  In bfloat16 by
// 8 bits the largest tiles of the gradient and of dW spill 4 to 5 of their 256 registers.
#include "mx_loss.hpp"
#include "mx_tiles.hpp"

namespace costa {
namespace {

struct LossTile {
  float alpha;
  int64_t n, col0;  // the vocabulary, and the first of the product's columns in it
  const int64_t* target;
  LossStat* stats;
  float* at;
  const float* lse;
  const float* dloss;
  const float* factor;  // a row's dloss is divided by its own (null: 1)
};

// Largest logit and the sum of exponentials from it of a tile's columns, to stats[tile column * m + row]; the
// target's logit, to at[row].
template <int SRC, int BBITS, int BM, int BN>
__global__ __launch_bounds__(kLanes) void tiles_loss_stats(Args p, LossTile a, uint32_t nm, uint32_t nn) {
  constexpr int WN = kWaves / 2, MT = BM / 2 / 16, NT = BN / WN / 16;
  TileSums<MT, NT> t;
  tile_sums<SRC, false, BBITS, BM, BN, 2, 1, true, 0>(p, nm, nn, t);
  const int lane = threadIdx.x % 64, l = lane % 16, g = lane / 16;
  const int64_t row0 = t.row - t.wave / WN * (BM / 2);  // of the tile
  LossStat* const red = reinterpret_cast<LossStat*>(t.shared);  // a row's, of the waves that have its columns
  int64_t target[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) target[i] = a.target[min(t.row + 16 * i + l, p.m - 1)];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t row = t.row + 16 * i + l, at = target[i] - t.col - 4 * g;
    float top = -__builtin_inff();
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float x = t.col + 16 * j + 4 * g + q < p.n ? a.alpha * t.acc[i][j][q] : -__builtin_inff();
        t.acc[i][j][q] = x;
        top = fmaxf(top, x);
        if (at == 16 * j + q && target[i] < p.n && row < p.m) a.at[row] = x;
      }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float from = top == -__builtin_inff() ? 0.0f : top;
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) sum += exp_of(t.acc[i][j][q] - from);
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (g == 0) red[t.wave % WN * BM + (int)(row - row0)] = LossStat{top, sum};
  }
  __syncthreads();
  const int64_t row = row0 + threadIdx.x;
  if (threadIdx.x < BM && row < p.m) {
    LossStat all = red[threadIdx.x];
#pragma unroll
    for (int w = 1; w < WN; ++w) all = join_stats(all, red[w * BM + threadIdx.x]);
    a.stats[(t.col - t.wave % WN * (16 * NT)) / BN * p.m + row] = all;
  }
}

// dloss (exp(logit - lse) - [target]) in the logits' place, to p.e.
template <int SRC, int BBITS, int BM, int BN>
__global__ __launch_bounds__(kLanes) void tiles_loss_grad(Args p, LossTile a, uint32_t nm, uint32_t nn) {
  constexpr int MT = BM / 2 / 16, NT = BN / (kWaves / 2) / 16;
  TileSums<MT, NT> t;
  tile_sums<SRC, false, BBITS, BM, BN, 2, 1, true, 0>(p, nm, nn, t);
  const int lane = threadIdx.x % 64, l = lane % 16, g = lane / 16;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t row = min(t.row + 16 * i + l, p.m - 1), target = a.target[row];
    const bool counts = target >= 0 && target < a.n;
    const float d = counts ? (a.dloss ? a.dloss[row] : 1.0f) / (a.factor ? a.factor[row] : 1.0f) : 1.0f, lse = a.lse[row];
    const int64_t at = target - a.col0 - t.col - 4 * g;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        t.acc[i][j][q] = counts ? d * (exp_of(a.alpha * t.acc[i][j][q] - lse) - (at == 16 * j + q ? 1.0f : 0.0f)) : 0.0f;
      }
  }
  put_wave<MT, NT>(p, t.acc, t.shared, t.wave, t.row, t.col);
}

// A product with a transposed left operand in bfloat16 whose factor is in device memory.
template <int BBITS, int BM, int BN, bool EDGE>
__global__ __launch_bounds__(kLanes) void tiles_loss_dw(Args p, const float* factor, uint32_t nm, uint32_t nn) {
  constexpr int MT = BM / 2 / 16, NT = BN / (kWaves / 2) / 16;
  TileSums<MT, NT> t;
  tile_sums<SRC_BF16, true, BBITS, BM, BN, 2, 1, EDGE, 0>(p, nm, nn, t);
  p.e.alpha *= *factor;
  put_wave<MT, NT>(p, t.acc, t.shared, t.wave, t.row, t.col);
}

int source_of(costa_real type) { return type == COSTA_REAL_BF16 ? SRC_BF16 : type == COSTA_REAL_F16 ? SRC_F16 : SRC_F32; }

// The tile that a product takes; one of 128x128 where that is narrower.
ProductPlan plan_loss(int src, int bits, int64_t m, int64_t n, int64_t k) {
  ProductPlan r = plan_product(src, true, bits, m, n, k);
  if (r.bn < 256) r.bm = r.bn = 128;
  return r;
}

template <int BBITS>
hipError_t launch_dw(const Args& p, const float* factor, hipStream_t stream) {
  ProductPlan plan = plan_product(SRC_BF16, false, BBITS, p.m, p.n, p.k);
  if (plan.bn < 256) plan.bm = plan.bn = 128;
  const uint32_t nm = (uint32_t)up_div(p.m, plan.bm), nn = (uint32_t)up_div(p.n, plan.bn);
  const dim3 grid(nm * nn);
  if (plan.bn < 256) tiles_loss_dw<BBITS, 128, 128, true><<<grid, kLanes, 0, stream>>>(p, factor, nm, nn);
  else if (p.m % 4 == 0) tiles_loss_dw<BBITS, 256, 256, false><<<grid, kLanes, 0, stream>>>(p, factor, nm, nn);
  else tiles_loss_dw<BBITS, 256, 256, true><<<grid, kLanes, 0, stream>>>(p, factor, nm, nn);
  return hipGetLastError();
}

template <int SRC, int BBITS>
hipError_t launch_loss(const Args& p, const LossTile& a, hipStream_t stream) {
  constexpr int BM = parts_of(SRC) == 1 ? 256 : 128;
  const ProductPlan plan = plan_loss(SRC, BBITS, p.m, p.n, p.k);
  const uint32_t nm = (uint32_t)up_div(p.m, plan.bm), nn = (uint32_t)up_div(p.n, plan.bn);
  const dim3 grid(nm * nn);
  if (plan.bn == 256) {
    if (a.stats) tiles_loss_stats<SRC, BBITS, BM, 256><<<grid, kLanes, 0, stream>>>(p, a, nm, nn);
    else tiles_loss_grad<SRC, BBITS, BM, 256><<<grid, kLanes, 0, stream>>>(p, a, nm, nn);
  } else {
    if (a.stats) tiles_loss_stats<SRC, BBITS, 128, 128><<<grid, kLanes, 0, stream>>>(p, a, nm, nn);
    else tiles_loss_grad<SRC, BBITS, 128, 128><<<grid, kLanes, 0, stream>>>(p, a, nm, nn);
  }
  return hipGetLastError();
}
template <int SRC>
hipError_t launch_loss_bits(const Args& p, const LossTile& a, hipStream_t stream) {
  return p.b.bits == 4 ? launch_loss<SRC, 4>(p, a, stream) : launch_loss<SRC, 8>(p, a, stream);
}
hipError_t launch_loss_type(costa_real type, const Args& p, const LossTile& a, hipStream_t stream) {
  if (type == COSTA_REAL_BF16) return launch_loss_bits<SRC_BF16>(p, a, stream);
  if (type == COSTA_REAL_F16) return launch_loss_bits<SRC_F16>(p, a, stream);
  return launch_loss_bits<SRC_F32>(p, a, stream);
}

Args args_of(const ProductArgs& a, const Epilogue& e) {
  return Args{a.m, a.n, a.k, MxView{}, a.b, a.real, a.a_rs, 1, e, 0};
}

}  // namespace

bool mx_loss_fused(costa_real type, int bits, int64_t m, int64_t n, int64_t k) {
  if (m == 0 || n == 0 || k == 0) return false;  // (no tiles: nothing to launch)
  const ProductPlan r = plan_product(source_of(type), true, bits, m, n, k);
  // (tiles of 128 columns and more, whole sums: where there are fewer the logits are few, too)
  return r.variant == TILES_BF16 && r.splits == 1 && r.bn >= 128 && up_div(m, 128) * up_div(n, 128) <= kTileSlice;
}

int64_t mx_loss_tile_chunks(costa_real type, int bits, int64_t m, int64_t n, int64_t k) {
  return up_div(n, plan_loss(source_of(type), bits, m, n, k).bn);
}

hipError_t launch_mx_loss_tiles(const ProductArgs& x, const int64_t* target, LossStat* stats, float* at,
                                hipStream_t stream) {
  return launch_loss_type(x.a_type, args_of(x, Epilogue{}),
                          LossTile{x.alpha, x.n, 0, target, stats, at, nullptr, nullptr, nullptr}, stream);
}

hipError_t launch_mx_loss_grad_tiles(const ProductArgs& x, int64_t vocabulary, int64_t col0, const int64_t* target,
                                     const float* lse, const float* dloss, const float* factor, void* g, bool bf16,
                                     hipStream_t stream) {
  const Epilogue e{g, x.n, 1, bf16 ? COSTA_REAL_BF16 : COSTA_REAL_F32, x.n % 4 == 0, 1.0f, 0.0f};
  return launch_loss_type(x.a_type, args_of(x, e),
                          LossTile{x.alpha, vocabulary, col0, target, nullptr, nullptr, lse, dloss, factor}, stream);
}

bool mx_loss_dw_fused(int bits, int64_t m, int64_t n, int64_t k) {
  const ProductPlan r = plan_product(SRC_BF16, false, bits, n, k, m);
  return r.variant == TILES_BF16 && r.splits == 1 && r.bn >= 128 && up_div(n, 128) * up_div(k, 128) <= kTileSlice;
}

hipError_t launch_mx_loss_dw(const ProductArgs& a, const float* factor, hipStream_t stream) {
  const int64_t es = a.c_type == COSTA_REAL_F32 ? 4 : 2;
  const Epilogue e{a.c, a.c_rs, 1, a.c_type, a.c_rs % 4 == 0 && (uintptr_t)a.c % (4 * es) == 0, a.alpha, a.beta};
  const Args p{a.m, a.n, a.k, MxView{}, a.b, a.real, a.a_rs, a.a_cs, e, 0};
  return a.b.bits == 4 ? launch_dw<4>(p, factor, stream) : launch_dw<8>(p, factor, stream);
}

}  // namespace costa
