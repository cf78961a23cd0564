// Root-mean-square norms with the residual's addition and a result in few bits, and
// their gradients.
//
//     h = x + r,  s = 1 / sqrt(mean(h^2) + eps),  y = h s w
//     u = h s,  g = dy w,  dx = s (g - u mean(g u)) + dh,  dw = sum over rows of dy u
//
// Bound by memory: an element is read and written once and costs some ten
// instructions.  A row is held in registers between its sum and what is made of it,
// 8 elements of a lane at a time, so that four neighbouring lanes hold a block of 32.
// Sums of squares in 64 bits: the instructions' rate allows it, and no h is too large
// or too small to be squared.
#include <algorithm>

#include "mx_layer.hpp"
#include "mx_rows.hpp"

namespace costa {
namespace {

// The sum over the LANES lanes that share a row; every lane gets it.
template <int LANES>
__device__ inline double row_sum(double v, double* shared) {
#pragma unroll
  for (int by = 32; by > 0; by /= 2) v += __shfl_xor(v, by);
  if constexpr (LANES > 64) {
    const int wave = threadIdx.x / 64;
    __syncthreads();  // (what was read of the sums before)
    if (threadIdx.x % 64 == 0) shared[wave] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int i = 0; i < LANES / 64; ++i) v += shared[i];
  }
  return v;
}

// 1 / sqrt(v): the instruction's estimate and one step of Newton's, which leaves about
// 46 bits: a float and what it is off by.  0 for an infinity.
struct Factor {
  float s, rest;
};
__device__ inline Factor rsqrt_of(double v) {
  const double r0 = __builtin_amdgcn_rsq(v);
  const double e = fma(-0.5 * v * r0, r0, 0.5);
  const double r = v < __builtin_inf() ? fma(r0, e, r0) : r0;
  const float s = (float)r;
  return Factor{s, (float)(r - (double)s)};
}

// h f w with its roundings made good, so that it is the nearest float (all but where it lies within
// 2^-20 steps of the middle of two): a rounding to few bits then falls on the side that the
// definition's does.  Three instructions of each kind more than two products.
__device__ inline float scaled(float h, Factor f, float w) {
  const float p = h * f.s, e = fmaf(h, f.s, -p) + h * f.rest;
  const float t = p * w, y = t + (fmaf(p, w, -t) + e * w);
  return __builtin_fabsf(t) < __builtin_inff() ? y : t;
}

// y in few bits: a block's scale from four neighbouring lanes.  Lanes past the matrix have
// zeros, up to the end of the padded row.
template <int BITS, typename I>
__device__ inline void quantize8(const MxView& q, int64_t row, I unit, const float y[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, magnitude(y[i]));
  const uint32_t s = mx_scale<BITS>(quad_max(m));
  if (unit >= (I)(q.row_scales * 4)) return;
  const v2u d = mx_encode8<BITS>(y, s);
  if (BITS == 4) *reinterpret_cast<uint32_t*>(q.data + row * q.row_bytes + unit * 4) = d.x;
  else *reinterpret_cast<v2u*>(q.data + row * q.row_bytes + unit * 8) = d;
  if (unit % 4 == 0) q.scales[row * q.row_scales + unit / 4] = (uint8_t)s;
}

// h of a unit; x and r as loaded.
template <int SRC, bool WIDE, typename I>
__device__ inline void unit_h(const NormArgs& a, Raw8<SRC>& x, Raw8<SRC>& r, I c, I cols, float h[8]) {
  floats8<SRC, WIDE>(x, c, cols, h);
  if (a.r.data) {
    float v[8];
    floats8<SRC, WIDE>(r, c, cols, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] += v[i];
  }
}
template <int SRC, int WSRC, bool WIDE, typename I>
__device__ inline void unit_y(const NormArgs& a, int64_t row, I unit, I cols, const float h[8], const Raw8<WSRC>& w,
                              Factor f) {
  const I c = unit * 8;
  if (a.h.data && c < cols) put8<SRC>(line_to<SRC>(a.h, row), c, cols, h);
  if (!a.y.data && !a.q.data) return;
  float y[8], v[8];
  if (a.w) raw_floats<WSRC>(w, v);
  else
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 1.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = scaled(h[i], f, v[i]);
  if (c + 8 > cols)  // (what pads a row is +0, whatever s)
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = c + i < cols ? y[i] : 0.0f;
  if (a.y.data && c < cols) put8<SRC>(line_to<SRC>(a.y, row), c, cols, y);
  if (a.q.data) {
    if (a.q.bits == 4) quantize8<4>(a.q, row, unit, y);
    else quantize8<8>(a.q, row, unit, y);
  }
}

// LANES lanes a row, PER units of each: a wave for rows of up to 2048 elements, so that no barrier
// stands between a row's sum and its results, then four, then sixteen.  PER 0: rows of any length,
// which are read twice.  Measured (h and 8 bits out of x and r): 16384x8192 in bfloat16 191 us, 4.9 TB/s of
// what is read and written (a plain copy reaches 5.1); in 4 bits 175 us, 5.0; 65536x512 41 to 44 us, 5.3 to 5.7;
// 4096x16384 103 us, 4.6; 4096x20000 (twice read) 153 us, 3.8; 8192x8192 floats 175 us, 5.0; one row of 4096 3.8 us.
template <int SRC, int WSRC, int LANES, int PER, bool WIDE>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void norm_rows(NormArgs a) {
  constexpr int ROWS = LANES < 256 ? 256 / LANES : 1, KEPT = PER ? PER : 1;
  typedef typename std::conditional<(PER > 0), int32_t, int64_t>::type I;  // (of columns)
  __shared__ double sums[LANES / 64];
  const I lane = threadIdx.x % LANES, cols = (I)a.cols;
  const I units = (I)(a.q.data ? a.q.row_scales * 4 : (a.cols + 7) / 8);
  Raw8<WSRC> w[KEPT];
  if constexpr (PER > 0)
    if (a.w)
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        get8<WSRC, WIDE>(w[p], a.w, (lane + p * LANES) * 8, cols);
        placed8<WSRC, WIDE>(w[p], (lane + p * LANES) * 8, cols);
      }
  for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < a.rows; row0 += (int64_t)gridDim.x * ROWS) {
    const int64_t mine = row0 + threadIdx.x / LANES, row = min(mine, a.rows - 1);
    const void* const xl = line_of<SRC>(a.x, row);
    const void* const rl = a.r.data ? line_of<SRC>(a.r, row) : nullptr;
    double sum = 0;
    if constexpr (PER > 0) {
      Raw8<SRC> x[PER], r[PER];
      float h[PER][8];
#pragma unroll
      for (int p = 0; p < PER; ++p) get8<SRC, WIDE>(x[p], xl, (lane + p * LANES) * 8, cols);
      if (rl)
#pragma unroll
        for (int p = 0; p < PER; ++p) get8<SRC, WIDE>(r[p], rl, (lane + p * LANES) * 8, cols);
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        unit_h<SRC, WIDE>(a, x[p], r[p], (lane + p * LANES) * 8, cols, h[p]);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fma((double)h[p][i], (double)h[p][i], sum);
      }
      const Factor f = rsqrt_of(row_sum<LANES>(sum, sums) * a.inverse + (double)a.eps);
      if (mine < a.rows) {
        if (a.rstd && lane == 0) a.rstd[row] = f.s;
#pragma unroll
        for (int p = 0; p < PER; ++p) unit_y<SRC, WSRC, WIDE>(a, row, lane + p * LANES, cols, h[p], w[p], f);
      }
    } else {
      Raw8<SRC> x, r;
      float h[8];
      for (I u = lane; u < units; u += LANES) {
        get8<SRC, WIDE>(x, xl, u * 8, cols);
        if (rl) get8<SRC, WIDE>(r, rl, u * 8, cols);
        unit_h<SRC, WIDE>(a, x, r, u * 8, cols, h);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fma((double)h[i], (double)h[i], sum);
      }
      const Factor f = rsqrt_of(row_sum<LANES>(sum, sums) * a.inverse + (double)a.eps);
      if (a.rstd && lane == 0) a.rstd[row] = f.s;
      // (whole rounds of lanes: a block's four lanes stay together)
      for (I u = lane; u < (units + LANES - 1) / LANES * LANES; u += LANES) {
        get8<SRC, WIDE>(x, xl, u * 8, cols);
        if (rl) get8<SRC, WIDE>(r, rl, u * 8, cols);
        if (a.w) {
          get8<WSRC, WIDE>(w[0], a.w, u * 8, cols);
          placed8<WSRC, WIDE>(w[0], u * 8, cols);
        }
        unit_h<SRC, WIDE>(a, x, r, u * 8, cols, h);
        unit_y<SRC, WSRC, WIDE>(a, row, u, cols, h, w[0], f);
      }
    }
  }
}

// ---- gradients ---------------------------------------------------------------
// The sum of eight products, in 32 bits: three roundings of each, its own among them four.
__device__ inline float sum8(const float a[8], const float b[8]) {
  return ((a[0] * b[0] + a[1] * b[1]) + (a[2] * b[2] + a[3] * b[3])) +
         ((a[4] * b[4] + a[5] * b[5]) + (a[6] * b[6] + a[7] * b[7]));
}

// A workgroup's rows share its lanes' part of dw, in registers; the parts are added by
// another kernel.  Measured with dh: 8192x8192 in bfloat16 106 and 5 us, 4.9 TB/s of dy, h, dh and dx (four units
// a lane, with a row's products and its next row in registers, 133 to 137: one wave of a SIMD had room); 8192x8192
// floats 207 us, 5.2; 803x1023 floats without dh 6 and 4 us.  Rows of 8193 to 16384 elements of 16 bits do not
// quite fit 128 registers (11 to 13 are spilled: 4096x16384 131 us, 4.1 TB/s); longer rows (floats: past 8192)
// are read twice and dw is summed in memory: 4096x20000 464 us, 1.4.
template <int SRC, int WSRC, int LANES, int PER, bool WIDE>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES, SRC == SRC_F32 ? 2 : 4) void norm_grad_rows(NormBackArgs a) {
  constexpr int ROWS = LANES < 256 ? 256 / LANES : 1, KEPT = PER ? PER : 1;
  typedef typename std::conditional<(PER > 0), int32_t, int64_t>::type I;  // (of columns)
  __shared__ double sums[LANES / 64];
  const I lane = threadIdx.x % LANES, cols = (I)a.cols, units = (I)((a.cols + 7) / 8);
  float* const part = a.parts + (int64_t)blockIdx.x * a.cols;
  Raw8<WSRC> w[KEPT];
  float dw[KEPT][8];
  if constexpr (PER > 0) {
    if (a.w)
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        get8<WSRC, WIDE>(w[p], a.w, (lane + p * LANES) * 8, cols);
        placed8<WSRC, WIDE>(w[p], (lane + p * LANES) * 8, cols);
      }
#pragma unroll
    for (int p = 0; p < PER; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) dw[p][i] = 0.0f;
  }
  bool first = true;
  // g of a unit, its dy beside it
  auto unit_g = [&](const Raw8<SRC>& raw, const Raw8<WSRC>& wr, float dy[8], float g[8]) {  // (both in place)
    raw_floats<SRC>(raw, dy);
    if (a.w) {
      raw_floats<WSRC>(wr, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] *= dy[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = dy[i];
    }
  };
  auto unit_dx = [&](int64_t row, I c, const float g[8], const float u[8], float s, float mean, Raw8<SRC> d) {
    if (c >= cols) return;
    float dx[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) dx[i] = s * (g[i] - u[i] * mean);
    if (a.dh.data) {
      float v[8];
      floats8<SRC, WIDE>(d, c, cols, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) dx[i] += v[i];
    }
    put8<SRC>(line_to<SRC>(a.dx, row), c, cols, dx);
  };
  for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < a.rows; row0 += (int64_t)gridDim.x * ROWS) {
    const int64_t mine = row0 + threadIdx.x / LANES, row = min(mine, a.rows - 1);
    const void* const dyl = line_of<SRC>(a.dy, row);
    const void* const hl = line_of<SRC>(a.h, row);
    const void* const dhl = a.dh.data ? line_of<SRC>(a.dh, row) : nullptr;
    const float s = a.rstd[row];
    double sum = 0;
    if constexpr (PER > 0) {
      Raw8<SRC> dyr[PER], hr[PER], dhr[PER];
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        get8<SRC, WIDE>(dyr[p], dyl, (lane + p * LANES) * 8, cols);
        get8<SRC, WIDE>(hr[p], hl, (lane + p * LANES) * 8, cols);
      }
      if (dhl)
#pragma unroll
        for (int p = 0; p < PER; ++p) get8<SRC, WIDE>(dhr[p], dhl, (lane + p * LANES) * 8, cols);
      // (g and u are made again after the sum: a row in 16 bits takes half the registers of theirs)
      float dy[8], g[8], u[8];
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        const I c = (lane + p * LANES) * 8;
        placed8<SRC, WIDE>(dyr[p], c, cols);
        placed8<SRC, WIDE>(hr[p], c, cols);
        unit_g(dyr[p], w[p], dy, g);
        raw_floats<SRC>(hr[p], u);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          u[i] *= s;
          if (mine < a.rows) dw[p][i] += dy[i] * u[i];
        }
        sum += (double)sum8(g, u);
      }
      const float mean = (float)(row_sum<LANES>(sum, sums) * a.inverse);
      if (mine < a.rows)
#pragma unroll
        for (int p = 0; p < PER; ++p) {
          unit_g(dyr[p], w[p], dy, g);
          raw_floats<SRC>(hr[p], u);
#pragma unroll
          for (int i = 0; i < 8; ++i) u[i] *= s;
          unit_dx(row, (lane + p * LANES) * 8, g, u, s, mean, dhr[p]);
        }
    } else {
      Raw8<SRC> dyr, hr, dhr;
      float dy[8], g[8], u[8];
      for (I un = lane; un < units; un += LANES) {
        get8<SRC, WIDE>(dyr, dyl, un * 8, cols);
        get8<SRC, WIDE>(hr, hl, un * 8, cols);
        if (a.w) {
          get8<WSRC, WIDE>(w[0], a.w, un * 8, cols);
          placed8<WSRC, WIDE>(w[0], un * 8, cols);
        }
        placed8<SRC, WIDE>(dyr, un * 8, cols);
        unit_g(dyr, w[0], dy, g);
        floats8<SRC, WIDE>(hr, un * 8, cols, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] *= s;
        sum += (double)sum8(g, u);
      }
      const float mean = (float)(row_sum<LANES>(sum, sums) * a.inverse);
      for (I un = lane; un < units; un += LANES) {
        const I c = un * 8;
        get8<SRC, WIDE>(dyr, dyl, c, cols);
        get8<SRC, WIDE>(hr, hl, c, cols);
        if (a.w) {
          get8<WSRC, WIDE>(w[0], a.w, c, cols);
          placed8<WSRC, WIDE>(w[0], c, cols);
        }
        if (dhl) get8<SRC, WIDE>(dhr, dhl, c, cols);
        placed8<SRC, WIDE>(dyr, c, cols);
        unit_g(dyr, w[0], dy, g);
        floats8<SRC, WIDE>(hr, c, cols, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] *= s;
        unit_dx(row, c, g, u, s, mean, dhr);
        if (a.dw)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (c + i < cols) part[c + i] = (first ? 0.0f : part[c + i]) + dy[i] * u[i];
      }
      first = false;
    }
  }
  if constexpr (PER > 0) {
    if (!a.dw) return;
    if constexpr (ROWS > 1) {  // the waves' parts, in a fixed order
      __shared__ float red[ROWS - 1][PER][8][64];
      const int wave = threadIdx.x / 64;
      if (wave > 0)
#pragma unroll
        for (int p = 0; p < PER; ++p)
#pragma unroll
          for (int i = 0; i < 8; ++i) red[wave - 1][p][i][lane] = dw[p][i];
      __syncthreads();
      if (wave > 0) return;
#pragma unroll
      for (int w = 0; w < ROWS - 1; ++w)
#pragma unroll
        for (int p = 0; p < PER; ++p)
#pragma unroll
          for (int i = 0; i < 8; ++i) dw[p][i] += red[w][p][i][lane];
    }
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const I c = (lane + p * LANES) * 8;
      if (c < cols) put8<SRC_F32>(part, c, cols, dw[p]);
    }
  }
}

// dw from its parts, in a fixed order and in 64 bits: a workgroup has 32 columns, 32 lanes
// each add every 32nd part.
template <int DSRC>
__global__ __launch_bounds__(1024) void norm_dw(const float* parts, int64_t n, int64_t cols, void* dw) {
  __shared__ double red[32][33];
  const int col = threadIdx.x % 32, mine = threadIdx.x / 32;
  for (int64_t c0 = (int64_t)blockIdx.x * 32; c0 < cols; c0 += (int64_t)gridDim.x * 32) {
    double sum = 0;
    if (c0 + col < cols)
#pragma unroll 4
      for (int64_t p = mine; p < n; p += 32) sum += (double)parts[p * cols + c0 + col];
    red[mine][col] = sum;
    __syncthreads();
    if (mine == 0 && c0 + col < cols) {
#pragma unroll
      for (int i = 1; i < 32; ++i) sum += red[i][col];
      static_cast<Elem<DSRC>*>(dw)[c0 + col] = (Elem<DSRC>)(float)sum;
    }
    __syncthreads();
  }
}

// How a row of `units` units is taken: lanes, and units of each (0: any number).
struct RowPlan {
  int lanes, per;
};
RowPlan plan_row(int64_t units) {
  for (int per : {1, 2, 4})
    if (units <= 64 * per) return {64, per};
  for (int per : {2, 4})
    if (units <= 256 * per) return {256, per};
  if (units <= 1024 * 2) return {1024, 2};
  return {1024, 0};
}
// Of the gradients, which hold more of a row: two units a lane at most, so that four waves of
// a SIMD fit (16-bit types).
RowPlan plan_grad_row(int64_t units, costa_real type) {
  for (int lanes : {64, 256, 512})
    for (int per : {1, 2})
      if (units <= lanes * per) return {lanes, per};
  return {1024, type != COSTA_REAL_F32 && units <= 2048 ? 2 : 0};
}

constexpr int64_t kNormGroups = 1 << 16;  // workgroups of a launch; they loop over more rows

template <template <int, int, int, int, bool> class Launch, int SRC, int WSRC, typename A>
hipError_t launch_rows(const A& a, RowPlan r, int64_t groups, hipStream_t stream) {
  const int at = r.lanes * 8 + r.per;
  if (a.cols < 8) Launch<SRC, WSRC, 64, 1, false>::go(a, groups, stream);
  else if (at == 64 * 8 + 1) Launch<SRC, WSRC, 64, 1, true>::go(a, groups, stream);
  else if (at == 64 * 8 + 2) Launch<SRC, WSRC, 64, 2, true>::go(a, groups, stream);
  else if (at == 256 * 8 + 1) Launch<SRC, WSRC, 256, 1, true>::go(a, groups, stream);
  else if (at == 256 * 8 + 2) Launch<SRC, WSRC, 256, 2, true>::go(a, groups, stream);
  else if (at == 1024 * 8) Launch<SRC, WSRC, 1024, 0, true>::go(a, groups, stream);
  else if (!Launch<SRC, WSRC, 0, 0, true>::more(a, at, groups, stream)) return hipErrorInvalidValue;
  return hipGetLastError();
}
template <template <int, int, int, int, bool> class Launch, typename A>
hipError_t launch_types(const A& a, RowPlan r, int64_t groups, hipStream_t stream) {
  const bool wide_w = a.w_type == COSTA_REAL_F32;
  switch (a.type) {
    case COSTA_REAL_F32: return launch_rows<Launch, SRC_F32, SRC_F32>(a, r, groups, stream);
    case COSTA_REAL_BF16:
      return wide_w ? launch_rows<Launch, SRC_BF16, SRC_F32>(a, r, groups, stream)
                    : launch_rows<Launch, SRC_BF16, SRC_BF16>(a, r, groups, stream);
    default:
      return wide_w ? launch_rows<Launch, SRC_F16, SRC_F32>(a, r, groups, stream)
                    : launch_rows<Launch, SRC_F16, SRC_F16>(a, r, groups, stream);
  }
}
template <int SRC, int WSRC, int LANES, int PER, bool WIDE>
struct Forward {
  static void go(const NormArgs& a, int64_t groups, hipStream_t stream) {
    norm_rows<SRC, WSRC, LANES, PER, WIDE><<<dim3((unsigned)groups), LANES < 256 ? 256 : LANES, 0, stream>>>(a);
  }
  static bool more(const NormArgs& a, int at, int64_t groups, hipStream_t stream) {
    if (at == 64 * 8 + 4) Forward<SRC, WSRC, 64, 4, true>::go(a, groups, stream);
    else if (at == 256 * 8 + 4) Forward<SRC, WSRC, 256, 4, true>::go(a, groups, stream);
    else if (at == 1024 * 8 + 2) Forward<SRC, WSRC, 1024, 2, true>::go(a, groups, stream);
    else return false;
    return true;
  }
};
template <int SRC, int WSRC, int LANES, int PER, bool WIDE>
struct Backward {
  static void go(const NormBackArgs& a, int64_t groups, hipStream_t stream) {
    norm_grad_rows<SRC, WSRC, LANES, PER, WIDE><<<dim3((unsigned)groups), LANES < 256 ? 256 : LANES, 0, stream>>>(a);
  }
  static bool more(const NormBackArgs& a, int at, int64_t groups, hipStream_t stream) {
    if (at == 512 * 8 + 1) Backward<SRC, WSRC, 512, 1, true>::go(a, groups, stream);
    else if (at == 512 * 8 + 2) Backward<SRC, WSRC, 512, 2, true>::go(a, groups, stream);
    else if (SRC != SRC_F32 && at == 1024 * 8 + 2)
      Backward<SRC, WSRC, 1024, SRC == SRC_F32 ? 0 : 2, true>::go(a, groups, stream);
    else return false;
    return true;
  }
};

int64_t groups_of(RowPlan r, int64_t rows) { return up_div(rows, r.lanes < 256 ? 256 / r.lanes : 1); }

}  // namespace

hipError_t launch_mx_norm(const NormArgs& a, hipStream_t stream) {
  const RowPlan r = plan_row(a.q.data ? a.q.row_scales * 4 : up_div(a.cols, 8));
  // as many workgroups as 2048 lanes for each CU are, which keep w (4096x16384 in bfloat16 103 us, with a
  // workgroup for each row 117; 16384x8192 191 and 196)
  const int64_t most = r.per > 0 ? kCUs * 2048 / std::max(r.lanes, 256) : kNormGroups;
  return launch_types<Forward>(a, r, std::min(groups_of(r, a.rows), most), stream);
}

// A part for each workgroup: as many as 1024 lanes for each CU are (8192x8192 in bfloat16: 512 of them 109 us,
// 1024 of them 115; 4096x2500: 1024 of them 25 us, 256 of them 36).
Parts mx_norm_parts(int64_t rows, int64_t cols) {
  const RowPlan r = plan_grad_row(up_div(cols, 8), COSTA_REAL_BF16);
  return {1, std::max<int64_t>(std::min<int64_t>(groups_of(r, rows), kCUs * 1024 / std::max(r.lanes, 256)), 1)};
}

hipError_t launch_mx_norm_backward(const NormBackArgs& a, hipStream_t stream) {
  const RowPlan r = plan_grad_row(up_div(a.cols, 8), a.type);
  int64_t groups = 0;  // (no rows: dw is a sum over nothing)
  if (a.rows > 0) {
    groups = a.dw ? std::min({mx_norm_parts(a.rows, a.cols).most, a.most, groups_of(r, a.rows)})
                  : std::min(groups_of(r, a.rows), kNormGroups);
    const hipError_t e = launch_types<Backward>(a, r, groups, stream);
    if (e != hipSuccess) return e;
  }
  if (!a.dw) return hipSuccess;
  const dim3 grid((unsigned)std::min<int64_t>(up_div(a.cols, 32), kNormGroups));
  if (a.dw_type == COSTA_REAL_F32) norm_dw<SRC_F32><<<grid, 1024, 0, stream>>>(a.parts, groups, a.cols, a.dw);
  else if (a.dw_type == COSTA_REAL_BF16) norm_dw<SRC_BF16><<<grid, 1024, 0, stream>>>(a.parts, groups, a.cols, a.dw);
  else norm_dw<SRC_F16><<<grid, 1024, 0, stream>>>(a.parts, groups, a.cols, a.dw);
  return hipGetLastError();
}

}  // namespace costa
