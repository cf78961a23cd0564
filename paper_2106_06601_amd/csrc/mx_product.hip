// Products of microscaled matrices: which kernel takes a call, the kernel for
// few rows, and the sum of a split sum's parts.
#include <algorithm>

#include "mx_product.hpp"

namespace costa {
namespace {

constexpr int kCUs = 256;

// ---- few rows ------------------------------------------------------------------
// C has at most 16 MT rows: the time is that of reading B once.  A workgroup
// makes 16 NT columns; its 8 waves take 128-byte pieces of B's rows in turn, so
// that they read whole lines of neighbouring addresses, straight to registers.
// Lane l holds row l % 16 of either operand; of a piece, 16 bytes at 16 (l / 16)
// and 16 at 64 + 16 (l / 16), and the left operand's elements of the same k: any
// order of k will do as long as both sides agree.  The waves' sums are joined
// through shared memory, pairwise, in a fixed order.
constexpr int kFewWaves = 8;

template <int SRC>
__device__ inline void few_left(const Args& p, int64_t row, bool there, int64_t k0, v4u out[parts_of(SRC)]) {
  if (SRC == SRC_MX4 || SRC == SRC_MX8) {
    constexpr int BITS = SRC == SRC_MX4 ? 4 : 8;
    v2u d = {0u, 0u};
    uint32_t s = 0;
    if (there && k0 < p.a.row_scales * kMxBlock) {
      const uint8_t* at = p.a.data + row * p.a.row_bytes;
      if (BITS == 4) d.x = *reinterpret_cast<const uint32_t*>(at + k0 / 2);
      else d = *reinterpret_cast<const v2u*>(at + k0);
      s = p.a.scales[row * p.a.row_scales + k0 / kMxBlock];
    }
    out[0] = mx_decode8_bf16<BITS>(d, s);
  } else {
    const int64_t n = there ? p.k - k0 : 0;
    raw_parts<SRC>(load8<SRC>(static_cast<const char*>(p.real) + (row * p.a_rs + k0) * bytes_of(SRC), n), out);
  }
}

template <int SRC, int BBITS, int MT, int NT>
__global__ __launch_bounds__(64 * kFewWaves) void few_rows(Args p, int splits, int64_t col0) {
  constexpr int UNIT = 1024 / BBITS;  // k of a 128-byte piece
  constexpr int HALF = UNIT / 2, LANE = HALF / 4, STEPS = LANE / 8;
  constexpr int P = parts_of(SRC);
  __shared__ v4f red[kFewWaves / 2][MT * NT][64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, r = lane % 16, g = lane / 16;
  const int64_t j0 = col0 + (int64_t)(blockIdx.x / splits) * (16 * NT);
  const int64_t units = (p.k + UNIT - 1) / UNIT;
  v4f acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = v4f{0, 0, 0, 0};
  const uint8_t* data[NT];
  const uint8_t* scales[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int64_t row = min(j0 + 16 * j + r, p.n - 1);
    data[j] = p.b.data + row * p.b.row_bytes + 16 * g;
    scales[j] = p.b.scales + row * p.b.row_scales + (BBITS == 4 ? g : g / 2);
  }
  const int step = kFewWaves * splits;
  for (int64_t u = (int64_t)(blockIdx.x % splits) * kFewWaves + wave; u < units; u += step) {
    v4u b[NT][2];
    uint32_t s[NT][2];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        b[j][h] = *reinterpret_cast<const v4u*>(data[j] + u * 128 + 64 * h);
        s[j][h] = scales[j][u * (UNIT / kMxBlock) + h * (HALF / kMxBlock)];
      }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t k0 = u * UNIT + h * HALF + g * LANE;
#pragma unroll
      for (int q = 0; q < STEPS; ++q) {
        v4u w[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const v2u d = BBITS == 4 ? v2u{b[j][h][q], 0u} : v2u{b[j][h][2 * q % 4], b[j][h][(2 * q + 1) % 4]};
          w[j] = mx_decode8_bf16<BBITS>(d, s[j][h]);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          v4u a[P];
          few_left<SRC>(p, 16 * i + r, 16 * i + r < p.m, k0 + 8 * q, a);
#pragma unroll
          for (int t = 0; t < P; ++t)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = mfma_bf16(w[j], a[t], acc[i][j]);
        }
      }
    }
  }
#pragma unroll
  for (int half = kFewWaves / 2; half > 0; half /= 2) {
    if (wave >= half && wave < 2 * half)
#pragma unroll
      for (int t = 0; t < MT * NT; ++t) red[wave - half][t][lane] = acc[t / NT][t % NT];
    __syncthreads();
    if (wave < half)
#pragma unroll
      for (int t = 0; t < MT * NT; ++t) acc[t / NT][t % NT] += red[wave][t][lane];
    __syncthreads();
  }
  if (wave != 0) return;
  Epilogue e = p.e;
  if (p.part) e.c = static_cast<float*>(e.c) + (int64_t)(blockIdx.x % splits) * p.part;
  // lane l has row l % 16 of C and columns 4 (l / 16) .. + 3 of each 16 x 16 piece
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int64_t row = 16 * i + r, col = j0 + 16 * j + 4 * g;
      if (row < p.m) put_four(e, row, col, acc[i][j], (int)min((int64_t)4, p.n - col));
    }
}

template <int SRC, int BBITS, int MT>
hipError_t launch_few_nt(const Args& p, const ProductPlan& plan, hipStream_t stream) {
  constexpr int64_t kSlice = (int64_t)1 << 22;  // workgroups of a launch: below 2^32 lanes
  const int64_t groups = (p.n + plan.bn - 1) / plan.bn, per = kSlice / plan.splits;
  for (int64_t at = 0; at < groups; at += per) {
    const dim3 grid((unsigned)(std::min(per, groups - at) * plan.splits)), block(64 * kFewWaves);
    if (plan.bn == 16) few_rows<SRC, BBITS, MT, 1><<<grid, block, 0, stream>>>(p, plan.splits, at * plan.bn);
    else few_rows<SRC, BBITS, MT, 2><<<grid, block, 0, stream>>>(p, plan.splits, at * plan.bn);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <int SRC, int BBITS>
hipError_t launch_few_mt(const Args& p, const ProductPlan& plan, hipStream_t stream) {
  if (plan.bm == 16) return launch_few_nt<SRC, BBITS, 1>(p, plan, stream);
  if (plan.bm == 32) return launch_few_nt<SRC, BBITS, 2>(p, plan, stream);
  return launch_few_nt<SRC, BBITS, 4>(p, plan, stream);
}
template <int SRC>
hipError_t launch_few_src(const Args& p, const ProductPlan& plan, hipStream_t stream) {
  return p.b.bits == 4 ? launch_few_mt<SRC, 4>(p, plan, stream) : launch_few_mt<SRC, 8>(p, plan, stream);
}
hipError_t launch_few(int src, const Args& p, const ProductPlan& plan, hipStream_t stream) {
  switch (src) {
    case SRC_MX4: return launch_few_src<SRC_MX4>(p, plan, stream);
    case SRC_MX8: return launch_few_src<SRC_MX8>(p, plan, stream);
    case SRC_BF16: return launch_few_src<SRC_BF16>(p, plan, stream);
    case SRC_F16: return launch_few_src<SRC_F16>(p, plan, stream);
    default: return launch_few_src<SRC_F32>(p, plan, stream);
  }
}

// ---- the parts of a split sum, in their order -------------------------------------
__global__ __launch_bounds__(256) void join_parts(Epilogue e, const float* parts, int64_t m, int64_t n, int splits) {
  const int64_t upr = (n + 3) / 4, units = m * upr;
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < units; u += (int64_t)gridDim.x * 256) {
    const int64_t i = u / upr, j = (u - i * upr) * 4;
    const int c = (int)min((int64_t)4, n - j);
    v4f acc = {0, 0, 0, 0};
    const float* p = parts + i * n + j;
    if (c == 4 && n % 4 == 0) {
      for (int s = 0; s < splits; ++s) acc += *reinterpret_cast<const v4f*>(p + s * m * n);
    } else {
      for (int s = 0; s < splits; ++s)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[q] += q < c ? p[s * m * n + q] : 0.0f;
    }
    put_four(e, i, j, acc, c);
  }
}

// C <- beta * C: a sum over nothing.
__global__ __launch_bounds__(256) void scale_only(Epilogue e, int64_t m, int64_t n) {
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < m * n; u += (int64_t)gridDim.x * 256)
    put_four(e, u / n, u % n, v4f{0, 0, 0, 0}, 1);
}

// ---- which kernel -------------------------------------------------------------------
constexpr size_t kPartsMax = (size_t)256 << 20;  // bytes of a split sum's parts

// Splits of a sum of `steps` steps over workgroups that fill the device, when
// `groups` of them make the tiles: not below `least` steps each.
int splits_for(int64_t groups, int64_t want, int64_t steps, int64_t least, int64_t m, int64_t n) {
  int64_t s = std::min(want / std::max<int64_t>(groups, 1), steps / least);
  s = std::min<int64_t>(s, (int64_t)(kPartsMax / 4) / std::max<int64_t>(m * n, 1));
  return (int)std::max<int64_t>(s, 1);
}

ProductPlan plan_product(int src, bool k_next, int bbits, int64_t m, int64_t n, int64_t k) {
  ProductPlan r{};
  if (m <= 64 && k_next) {
    r.variant = FEW_ROWS;
    r.bm = m <= 16 ? 16 : m <= 32 ? 32 : 64;
    r.bn = m > 4 && n >= 32 * kCUs ? 32 : 16;
    const int64_t units = (k + 1024 / bbits - 1) / (1024 / bbits);
    r.splits = splits_for((n + r.bn - 1) / r.bn, kCUs, units, 4 * kFewWaves, m, n);
    return r;
  }
  // (the scaled kernel counts a tile's bytes in 32 bits)
  const bool scaled = src == SRC_MX4 && bbits == 4 && k <= 1 << 24;
  r.variant = scaled ? TILES_SCALED : TILES_BF16;
  const int big = scaled || parts_of(src) == 1 ? 256 : 128;
  const auto tiles = [&](int64_t bm, int64_t bn) { return (m + bm - 1) / bm * ((n + bn - 1) / bn); };
  if (tiles(big, 256) >= kCUs / 2) {
    r.bm = big;
    r.bn = 256;
  } else {
    r.bm = 128;
    r.bn = scaled ? 128 : 64;
  }
  const int64_t step = scaled ? 256 : 64;
  r.splits = splits_for(tiles(r.bm, r.bn), kCUs, (k + step - 1) / step, 4, m, n);
  return r;
}

}  // namespace

size_t mx_product_workspace(int64_t m, int64_t n, int64_t k) {
  size_t most = 0;
  for (int src : {SRC_MX4, SRC_MX8, SRC_BF16, SRC_F16, SRC_F32})
    for (int bbits : {4, 8})
      for (bool k_next : {true, false}) {
        const ProductPlan r = plan_product(src, k_next, bbits, m, n, k);
        if (r.splits > 1) most = std::max(most, (size_t)r.splits * m * n * sizeof(float));
      }
  return most;
}

hipError_t launch_mx_product(const ProductArgs& a, hipStream_t stream) {
  const int64_t es = a.c_type == COSTA_REAL_F32 ? 4 : 2;
  const bool vec = a.c_cs == 1 && a.c_rs % 4 == 0 && (uintptr_t)a.c % (4 * es) == 0;
  const Epilogue e{a.c, a.c_rs, a.c_cs, a.c_type, vec, a.alpha, a.beta};
  if (a.k == 0) {
    const int64_t groups = (a.m * a.n + 255) / 256;
    scale_only<<<dim3((unsigned)std::min<int64_t>(groups, 1 << 20)), 256, 0, stream>>>(e, a.m, a.n);
    return hipGetLastError();
  }
  const int src = a.amx.bits == 4                 ? SRC_MX4
                  : a.amx.bits == 8               ? SRC_MX8
                  : a.a_type == COSTA_REAL_BF16   ? SRC_BF16
                  : a.a_type == COSTA_REAL_F16    ? SRC_F16
                                                  : SRC_F32;
  const bool k_next = a.amx.bits != 0 || a.a_cs == 1;
  ProductPlan plan = plan_product(src, k_next, a.b.bits, a.m, a.n, a.k);
  Args p{a.m, a.n, a.k, a.amx, a.b, a.real, a.a_rs, a.a_cs, e, 0};
  const size_t part = (size_t)a.m * a.n * sizeof(float);
  plan.splits = (int)std::min<size_t>(plan.splits, a.workspace_bytes / part);
  if (plan.splits > 1) {
    p.e = Epilogue{a.workspace, a.n, 1, COSTA_REAL_F32, a.n % 4 == 0, 1.0f, 0.0f};
    p.part = a.m * a.n;
  } else {
    plan.splits = 1;
  }
  hipError_t err = plan.variant == FEW_ROWS     ? launch_few(src, p, plan, stream)
                   : plan.variant == TILES_BF16 ? launch_tiles_bf16(src, p, plan, stream)
                                                : launch_tiles_scaled(p, plan, stream);
  if (err != hipSuccess || plan.splits == 1) return err;
  const int64_t groups = (a.m * ((a.n + 3) / 4) + 255) / 256;
  join_parts<<<dim3((unsigned)std::min<int64_t>(groups, 1 << 20)), 256, 0, stream>>>(e, a.workspace, a.m, a.n,
                                                                                    plan.splits);
  return hipGetLastError();
}

}  // namespace costa
