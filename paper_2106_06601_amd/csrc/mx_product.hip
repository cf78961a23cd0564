// Products of microscaled matrices: which kernel takes a call, the kernel for
// few rows, and the sum of a split sum's parts.
#include <algorithm>

#include "mx_product.hpp"

namespace costa {
namespace {

// ---- few rows ------------------------------------------------------------------
// C has at most 16 MT rows: the time is that of reading B once.  A workgroup
// makes 16 NT columns; its waves take 128-byte pieces of B's rows in turn, so
// that they read whole lines of neighbouring addresses, straight to registers.
// Lane l holds row l % 16 of either operand; of a piece, 16 bytes at 16 (l / 16)
// and 16 at 64 + 16 (l / 16), and the left operand's elements of the same k: any
// order of k will do as long as both sides agree.  The left operand goes by slabs
// of 16 rows by 128 of k: a wave reads one as it lies in memory, makes it
// bfloat16 parts once, and turns it to the instruction's order through a piece of
// shared memory of its own.  (Read in that order straight from memory, a load
// touches 64 pieces of 16 bytes, and the left operand costs more than B.)  The next piece of
// B and the next slab are on their way meanwhile.  The waves' sums are joined
// through shared memory, pairwise, in a fixed order.  Measured, B in 4 bits, out of
// memory (32 matrices in turn) and, the same one again and again, out of the last-level
// cache: one row of bfloat16 by 8192x8192 (35.7 MB of B) 15.7 us, 2.3 TB/s, and 12.5
// us, 2.9 TB/s (a launch and the first loads take about 5 us of any call); 13 rows of
// float16 by 20000x4095 26.6 and 24.0 us; 64 rows of bfloat16 by 8192x8192 38 and 35
// us, of float 91 cached (three parts).
constexpr int kSlab = 128;

// A slab: lane l has, of rows l / 16 + 4 q, the eight elements 8 (l % 16) ..
template <int SRC>
struct FewSlab {
  static constexpr bool MX = SRC == SRC_MX4 || SRC == SRC_MX8;
  static constexpr int BITS = SRC == SRC_MX4 ? 4 : 8;
  static constexpr int P = parts_of(SRC);
  Raw8<SRC> raw[MX ? 1 : 4];
  v2u code[MX ? 4 : 1];
  uint32_t scale[MX ? 4 : 1];
  // rows row0 .. of the operand, of which those past its last repeat it (their
  // results are not stored); k0: the slab's first k, `end` elements are there
  __device__ inline void load(const Args& p, int64_t row0, int64_t k0, int64_t end) {
    const int lane = threadIdx.x % 64;
    const int64_t k = k0 + 8 * (lane % 16);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (q > 0 && row0 + 4 * q >= p.m) continue;
      const int64_t row = min(row0 + 4 * q + lane / 16, p.m - 1);
      if constexpr (MX) {  // (padded to whole slabs; past them nothing counts)
        const uint8_t* at = p.a.data + row * p.a.row_bytes;
        code[q] = v2u{0u, 0u};
        scale[q] = 0;
        if (k0 < end) {
          if (BITS == 4) code[q].x = *reinterpret_cast<const uint32_t*>(at + k / 2);
          else code[q] = *reinterpret_cast<const v2u*>(at + k);
          scale[q] = p.a.scales[row * p.a.row_scales + k / kMxBlock];
        }
      } else {
        const char* line = static_cast<const char*>(p.real) + row * p.a_rs * bytes_of(SRC);
        load8<SRC>(raw[q], line, k, end);
      }
    }
  }
  __device__ inline void store(const Args& p, int64_t row0, int64_t k0, int64_t end, v4u* slab) {
    const int lane = threadIdx.x % 64;
    if constexpr (!MX)
      if (k0 + kSlab > end)
#pragma unroll
        for (int q = 0; q < 4; ++q) place8<SRC>(raw[q], k0 + 8 * (lane % 16), end);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (q > 0 && row0 + 4 * q >= p.m) continue;
      v4u out[P];
      if constexpr (MX) out[0] = mx_decode8_bf16<BITS>(code[q], scale[q]);
      else raw_parts<SRC>(raw[q], out);
      const int row = 4 * q + lane / 16;
#pragma unroll
      for (int x = 0; x < P; ++x) slab[x * 256 + row * 16 + (lane % 16 ^ (row & 7))] = out[x];
    }
  }
};

template <int SRC, int BBITS, int MT, int NT>
__global__ __launch_bounds__(64 * kFewWaves) void few_rows(Args p, int splits, int64_t col0) {
  constexpr int UNIT = 1024 / BBITS;  // k of a 128-byte piece
  constexpr int SLABS = UNIT / kSlab, LOADS = 2 / SLABS;  // 16-byte loads of B a slab
  constexpr int STEPS = 128 / 4 / 8 / LOADS;              // instructions a load
  constexpr int P = parts_of(SRC);
  constexpr int SHARED = P * kFewWaves * 256 > kFewWaves / 2 * MT * NT * 64 ? P * kFewWaves * 256
                                                                            : kFewWaves / 2 * MT * NT * 64;
  __shared__ v4u shared[SHARED];  // a slab for each wave; then the sums
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16,
            g = lane / 16;
  v4u* const slab = shared + wave * P * 256;
  const int64_t j0 = col0 + (int64_t)(blockIdx.x / splits) * (16 * NT);
  const uint32_t units = (uint32_t)((p.k + UNIT - 1) / UNIT);
  const int64_t a_end = FewSlab<SRC>::MX ? p.a.row_scales * kMxBlock : p.k;
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
  // this wave's pieces: first, first + step, ..; each workgroup begins at another one of
  // them (rows a power of two apart would all be read at the same distance else)
  const uint32_t step = kFewWaves * splits, first = blockIdx.x % splits * kFewWaves + wave;
  const uint32_t turns = first < units ? (units - first + step - 1) / step : 0;
  uint32_t turn = turns > 0 ? blockIdx.x / splits % turns : 0;
  int64_t u = first + turn * step;
  v4u b[NT][2];
  uint32_t s[NT][2];
  FewSlab<SRC> left;
  auto load = [&](int64_t at) {
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        b[j][h] = *reinterpret_cast<const v4u*>(data[j] + at * 128 + 64 * h);
        s[j][h] = scales[j][at * (UNIT / kMxBlock) + h * (UNIT / 2 / kMxBlock)];
      }
  };
  if (turns > 0) {
    load(u);
    left.load(p, 0, u * UNIT, a_end);
  }
  for (uint32_t to_go = turns; to_go > 0; --to_go) {
    turn = turn + 1 < turns ? turn + 1 : 0;
    // (the last turn loads its own piece again, from the cache: without a branch, the
    // compiler can count the loads on their way and waits for no more than it needs)
    const int64_t next = to_go > 1 ? first + turn * step : u;
    v4u w[NT][2];
    uint32_t t[NT][2];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) w[j][h] = b[j][h], t[j][h] = s[j][h];
    load(next);
#pragma unroll
    for (int h = 0; h < SLABS; ++h) {
      v4u e[NT][LOADS][STEPS];  // the slab's part of B, decoded
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int l = 0; l < LOADS; ++l)
#pragma unroll
          for (int q = 0; q < STEPS; ++q) {
            const v4u& c = w[j][h * LOADS + l];
            e[j][l][q] = mx_decode8_bf16<BBITS>(BBITS == 4 ? v2u{c[q], 0u} : v2u{c[2 * q % 4], c[(2 * q + 1) % 4]},
                                                t[j][h * LOADS + l]);
          }
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        left.store(p, 16 * i, u * UNIT + h * kSlab, a_end, slab);
        if (i + 1 < MT) left.load(p, 16 * (i + 1), u * UNIT + h * kSlab, a_end);
        else if (h + 1 < SLABS) left.load(p, 0, u * UNIT + (h + 1) * kSlab, a_end);
        else left.load(p, 0, next * UNIT, a_end);
        wave_fence();
#pragma unroll
        for (int l = 0; l < LOADS; ++l)
#pragma unroll
          for (int q = 0; q < STEPS; ++q) {
            const int chunk = l * (kSlab / 8 / LOADS) + g * STEPS + q;
#pragma unroll
            for (int x = 0; x < P; ++x) {
              const v4u a = slab[x * 256 + r * 16 + (chunk ^ (r & 7))];
#pragma unroll
              for (int j = 0; j < NT; ++j) acc[i][j] = mfma_bf16(e[j][l][q], a, acc[i][j]);
            }
          }
        wave_fence();
      }
    }
    u = next;
  }
  __syncthreads();
  typedef v4f Sums[MT * NT][64];
  Sums* const red = reinterpret_cast<Sums*>(shared);
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
  // lane l has row l % 16 of C and columns 4 (l / 16) .. + 3 of each 16 x 16 piece; the
  // pieces go through shared memory so that the code that stores them stands there once
#pragma unroll
  for (int t = 0; t < MT * NT; ++t) red[0][t][lane] = acc[t / NT][t % NT];
  wave_fence();
#pragma unroll 1
  for (int t = 0; t < MT * NT; ++t) {
    const int64_t row = 16 * (t / NT) + r, col = j0 + 16 * (t % NT) + 4 * g;
    if (row < p.m) put_four(e, row, col, red[0][t][lane], (int)min((int64_t)4, p.n - col));
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

// ---- what has too little for vector loads --------------------------------------------
// Sums of fewer than 8 elements of a plain operand.  A lane makes one element of C.
template <int SRC, int BBITS>
__global__ __launch_bounds__(256) void thin(Args p) {
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < p.m * p.n; u += (int64_t)gridDim.x * 256) {
    const int64_t i = u / p.n, j = u - i * p.n;
    v2u d = {0u, 0u};
    if (BBITS == 4) d.x = *reinterpret_cast<const uint32_t*>(p.b.data + j * p.b.row_bytes);
    else d = *reinterpret_cast<const v2u*>(p.b.data + j * p.b.row_bytes);
    float b[8], sum = 0.0f;
    mx_decode8<BBITS>(d, p.b.scales[j * p.b.row_scales], b);
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (q < p.k) {
        const int64_t at = i * p.a_rs + q * p.a_cs;
        const float a = SRC == SRC_BF16  ? (float)static_cast<const __bf16*>(p.real)[at]
                        : SRC == SRC_F16 ? (float)static_cast<const _Float16*>(p.real)[at]
                                         : static_cast<const float*>(p.real)[at];
        sum += a * b[q];
      }
    put_four(p.e, i, j, v4f{sum, 0, 0, 0}, 1);
  }
}
template <int SRC>
hipError_t launch_thin_src(const Args& p, hipStream_t stream) {
  const dim3 grid((unsigned)std::min<int64_t>((p.m * p.n + 255) / 256, 1 << 20));
  if (p.b.bits == 4) thin<SRC, 4><<<grid, 256, 0, stream>>>(p);
  else thin<SRC, 8><<<grid, 256, 0, stream>>>(p);
  return hipGetLastError();
}
hipError_t launch_thin(int src, const Args& p, hipStream_t stream) {
  if (src == SRC_BF16) return launch_thin_src<SRC_BF16>(p, stream);
  if (src == SRC_F16) return launch_thin_src<SRC_F16>(p, stream);
  return launch_thin_src<SRC_F32>(p, stream);
}

// ---- the parts of a split sum, in a fixed order -------------------------------------
// LANES lanes share four elements of C, each adding every LANES-th part; their sums
// are then added in turn.
template <int LANES>
__global__ __launch_bounds__(256) void join_parts(Epilogue e, const float* parts, int64_t m, int64_t n, int splits) {
  constexpr int UNITS = 256 / LANES;  // of a workgroup
  __shared__ v4f red[LANES][UNITS];
  const int64_t upr = (n + 3) / 4, units = m * upr;
  const int mine = threadIdx.x / UNITS, at = threadIdx.x % UNITS;
  for (int64_t u0 = (int64_t)blockIdx.x * UNITS; u0 < units; u0 += (int64_t)gridDim.x * UNITS) {
    const int64_t u = u0 + at;
    const int64_t i = ((u | upr) >> 32) == 0 ? (int64_t)((uint32_t)u / (uint32_t)upr) : u / upr, j = (u - i * upr) * 4;
    const int c = u < units ? (int)min((int64_t)4, n - j) : 0;
    v4f acc = {0, 0, 0, 0};
    const float* p = parts + i * n + j;
    if (c == 4 && n % 4 == 0) {
#pragma unroll 8
      for (int s = mine; s < splits; s += LANES) acc += *reinterpret_cast<const v4f*>(p + s * m * n);
    } else {
#pragma unroll 4
      for (int s = mine; s < splits; s += LANES)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[q] += q < c ? p[s * m * n + q] : 0.0f;
    }
    if (LANES > 1) {
      red[mine][at] = acc;
      __syncthreads();
      if (mine == 0)
#pragma unroll
        for (int s = 1; s < LANES; ++s) acc += red[s][at];
    }
    if (mine == 0) put_four(e, i, j, acc, c);
    if (LANES > 1) __syncthreads();
  }
}

// C <- beta * C: a sum over nothing.  (alpha times it would be NaN for an alpha that is
// not finite, and -0 for a negative one.)
__global__ __launch_bounds__(256) void scale_only(Epilogue e, int64_t m, int64_t n) {
  e.alpha = 1.0f;
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < m * n; u += (int64_t)gridDim.x * 256)
    put_four(e, u / n, u % n, v4f{0, 0, 0, 0}, 1);
}

}  // namespace

static size_t split_workspace(int64_t m, int64_t n, int64_t k, bool in_parts) {
  size_t most = 0;
  if (m == 0 || n == 0 || k == 0) return 0;
  for (int src : {SRC_MX4, SRC_MX8, SRC_BF16, SRC_F16, SRC_F32})
    for (int bbits : {4, 8})
      for (bool k_next : {true, false}) {
        const ProductPlan r = plan_product(src, k_next, bbits, m, n, k, in_parts);
        if (r.splits > 1) most = std::max(most, (size_t)r.splits * m * n * sizeof(float));
      }
  return most;
}
size_t mx_product_workspace(int64_t m, int64_t n, int64_t k) { return split_workspace(m, n, k, false); }

namespace {

// Plans a product and launches its sums: split, or where `parts` says so, unscaled to their
// places in the workspace (as many as it holds), else with e to C.
hipError_t launch_sums(const ProductArgs& a, const Epilogue& e, bool parts, ProductPlan& plan, hipStream_t stream) {
  const int src = a.amx.bits == 4                 ? SRC_MX4
                  : a.amx.bits == 8               ? SRC_MX8
                  : a.a_type == COSTA_REAL_BF16   ? SRC_BF16
                  : a.a_type == COSTA_REAL_F16    ? SRC_F16
                                                  : SRC_F32;
  const bool k_next = a.amx.bits != 0 || a.a_cs == 1;
  plan = plan_product(src, k_next, a.b.bits, a.m, a.n, a.k, parts);
  Args p{a.m, a.n, a.k, a.amx, a.b, a.real, a.a_rs, a.a_cs, e, 0};
  const size_t part = (size_t)a.m * a.n * sizeof(float);
  plan.splits = (int)std::min<size_t>(plan.splits, a.workspace_bytes / part);
  if (plan.splits > 1 || parts) {
    p.e = Epilogue{a.workspace, a.n, 1, COSTA_REAL_F32, a.n % 4 == 0, 1.0f, 0.0f};
    p.part = a.m * a.n;
  }
  plan.splits = std::max(plan.splits, 1);
  return plan.variant == THIN         ? launch_thin(src, p, stream)
         : plan.variant == FEW_ROWS   ? launch_few(src, p, plan, stream)
         : plan.variant == TILES_BF16 ? launch_tiles_bf16(src, p, plan, stream)
                                      : launch_tiles_scaled(p, plan, stream);
}

// Splits of a product whose sums go on in parts, in tiles of 64 rows; 0 where other kernels take it.
// (61 rows by 8192x8192 in 4 bits, joined: bfloat16 25 us, with the kernel for few rows 41; float16 31 and 75;
// float 39 and 91.  17 to 32 rows of bfloat16, tiles and the kernel for few rows: 8192x8192 22 and 25 to 28 us,
// 20000 columns of 4096 26 and 28 to 30, 4096x4096 14 both, 1024 columns of 8192 16 and 14.)
int64_t some_rows_splits(int src, int64_t m, int64_t n, int64_t k) {
  const int64_t tiles = up_div(n, 128);
  if (m > 64 || m <= 16 || k < 256 || tiles > 1 << 20) return 0;
  if (src == SRC_BF16 && m <= 32 && tiles < kCUs / 4) return 0;
  // a workgroup for each CU, or two where that leaves sums whole
  const int64_t fill = kCUs / tiles >= 2 ? kCUs / tiles : 2 * kCUs / tiles;
  return std::max<int64_t>(std::min(fill, k / 256), 1);
}

}  // namespace

size_t mx_product_parts_workspace(int64_t m, int64_t n, int64_t k) {
  if (m == 0 || n == 0 || k == 0) return 0;
  const int64_t some = some_rows_splits(SRC_F32, m, n, k);
  return std::max(split_workspace(m, n, k, true), (size_t)std::max<int64_t>(some, 1) * m * n * 4);
}

hipError_t launch_mx_product_parts(const ProductArgs& a, int& splits, hipStream_t stream) {
  const int src = a.a_type == COSTA_REAL_BF16 ? SRC_BF16 : a.a_type == COSTA_REAL_F16 ? SRC_F16 : SRC_F32;
  const int64_t some = a.amx.bits == 0 && a.a_cs == 1 ? some_rows_splits(src, a.m, a.n, a.k) : 0;
  if (some > 0) {
    splits = (int)std::max<int64_t>(std::min<int64_t>(some, a.workspace_bytes / ((size_t)a.m * a.n * 4)), 1);
    const Epilogue e{a.workspace, a.n, 1, COSTA_REAL_F32, a.n % 4 == 0, 1.0f, 0.0f};
    return launch_tiles_few(src, Args{a.m, a.n, a.k, a.amx, a.b, a.real, a.a_rs, a.a_cs, e, a.m * a.n}, splits, stream);
  }
  ProductPlan plan{};
  const hipError_t err = launch_sums(a, Epilogue{}, true, plan, stream);
  splits = plan.splits;
  return err;
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
  ProductPlan plan{};
  hipError_t err = launch_sums(a, e, false, plan, stream);
  if (err != hipSuccess || plan.splits == 1) return err;
  // (with 16 lanes, 256 parts of a 100 x 64 sum are joined in 5 us; with one, in 66)
  const int lanes = plan.splits >= 16 ? 16 : 1;
  const int64_t groups = (a.m * ((a.n + 3) / 4) * lanes + 255) / 256;
  const dim3 grid((unsigned)std::min<int64_t>(groups, 1 << 20));
  if (lanes == 16) join_parts<16><<<grid, 256, 0, stream>>>(e, a.workspace, a.m, a.n, plan.splits);
  else join_parts<1><<<grid, 256, 0, stream>>>(e, a.workspace, a.m, a.n, plan.splits);
  return hipGetLastError();
}

}  // namespace costa
