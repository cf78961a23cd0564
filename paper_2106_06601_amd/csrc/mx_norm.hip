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
// 46 bits.  0 for an infinity.
__device__ inline float rsqrt_of(double v) {
  const double r = __builtin_amdgcn_rsq(v);
  const double e = fma(-0.5 * v * r, r, 0.5);
  return (float)(v < __builtin_inf() ? fma(r, e, r) : r);
}

// y in few bits: a block's scale from four neighbouring lanes.  Lanes past the matrix have
// zeros, up to the end of the padded row.
template <int BITS>
__device__ inline void quantize8(const MxView& q, int64_t row, int64_t unit, const float y[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, magnitude(y[i]));
  const uint32_t s = mx_scale<BITS>(quad_max(m));
  if (unit >= q.row_scales * 4) return;
  const v2u d = mx_encode8<BITS>(y, s);
  if (BITS == 4) *reinterpret_cast<uint32_t*>(q.data + row * q.row_bytes + unit * 4) = d.x;
  else *reinterpret_cast<v2u*>(q.data + row * q.row_bytes + unit * 8) = d;
  if (unit % 4 == 0) q.scales[row * q.row_scales + unit / 4] = (uint8_t)s;
}

// h of a unit; x and r as loaded.
template <int SRC, bool WIDE>
__device__ inline void unit_h(const NormArgs& a, Raw8<SRC>& x, Raw8<SRC>& r, int64_t c, float h[8]) {
  floats8<SRC, WIDE>(x, c, a.cols, h);
  if (a.r.data) {
    float v[8];
    floats8<SRC, WIDE>(r, c, a.cols, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] += v[i];
  }
}
template <int SRC, int WSRC, bool WIDE>
__device__ inline void unit_y(const NormArgs& a, int64_t row, int64_t unit, const float h[8], const Raw8<WSRC>& w,
                              float s) {
  const int64_t c = unit * 8;
  if (a.h.data && c < a.cols) put8<SRC>(line_to<SRC>(a.h, row), c, a.cols, h);
  if (!a.y.data && !a.q.data) return;
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = h[i] * s;
  if (a.w) {
    float v[8];
    raw_floats<WSRC>(w, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] *= v[i];
  }
  if (c + 8 > a.cols)  // (what pads a row is +0, whatever s)
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = c + i < a.cols ? y[i] : 0.0f;
  if (a.y.data && c < a.cols) put8<SRC>(line_to<SRC>(a.y, row), c, a.cols, y);
  if (a.q.data) {
    if (a.q.bits == 4) quantize8<4>(a.q, row, unit, y);
    else quantize8<8>(a.q, row, unit, y);
  }
}

// LANES lanes a row, PER units of each.  PER 0: rows of any length, which are read twice.
template <int SRC, int WSRC, int LANES, int PER, bool WIDE>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void norm_rows(NormArgs a) {
  constexpr int ROWS = LANES < 256 ? 256 / LANES : 1, KEPT = PER ? PER : 1;
  __shared__ double sums[LANES / 64];
  const int lane = threadIdx.x % LANES;
  const int64_t units = a.q.data ? a.q.row_scales * 4 : (a.cols + 7) / 8;
  Raw8<WSRC> w[KEPT];
  if constexpr (PER > 0)
    if (a.w)
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        get8<WSRC, WIDE>(w[p], a.w, (int64_t)(lane + p * LANES) * 8, a.cols);
        placed8<WSRC, WIDE>(w[p], (int64_t)(lane + p * LANES) * 8, a.cols);
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
      for (int p = 0; p < PER; ++p) get8<SRC, WIDE>(x[p], xl, (int64_t)(lane + p * LANES) * 8, a.cols);
      if (rl)
#pragma unroll
        for (int p = 0; p < PER; ++p) get8<SRC, WIDE>(r[p], rl, (int64_t)(lane + p * LANES) * 8, a.cols);
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        unit_h<SRC, WIDE>(a, x[p], r[p], (int64_t)(lane + p * LANES) * 8, h[p]);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fma((double)h[p][i], (double)h[p][i], sum);
      }
      const float s = rsqrt_of(row_sum<LANES>(sum, sums) * a.inverse + (double)a.eps);
      if (mine < a.rows) {
        if (a.rstd && lane == 0) a.rstd[row] = s;
#pragma unroll
        for (int p = 0; p < PER; ++p) unit_y<SRC, WSRC, WIDE>(a, row, lane + p * LANES, h[p], w[p], s);
      }
    } else {
      Raw8<SRC> x, r;
      float h[8];
      for (int64_t u = lane; u < units; u += LANES) {
        get8<SRC, WIDE>(x, xl, u * 8, a.cols);
        if (rl) get8<SRC, WIDE>(r, rl, u * 8, a.cols);
        unit_h<SRC, WIDE>(a, x, r, u * 8, h);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fma((double)h[i], (double)h[i], sum);
      }
      const float s = rsqrt_of(row_sum<LANES>(sum, sums) * a.inverse + (double)a.eps);
      if (a.rstd && lane == 0) a.rstd[row] = s;
      // (whole rounds of lanes: a block's four lanes stay together)
      for (int64_t u = lane; u < (units + LANES - 1) / LANES * LANES; u += LANES) {
        get8<SRC, WIDE>(x, xl, u * 8, a.cols);
        if (rl) get8<SRC, WIDE>(r, rl, u * 8, a.cols);
        if (a.w) {
          get8<WSRC, WIDE>(w[0], a.w, u * 8, a.cols);
          placed8<WSRC, WIDE>(w[0], u * 8, a.cols);
        }
        unit_h<SRC, WIDE>(a, x, r, u * 8, h);
        unit_y<SRC, WSRC, WIDE>(a, row, u, h, w[0], s);
      }
    }
  }
}

// ---- gradients ---------------------------------------------------------------
// A workgroup's rows share its lanes' part of dw, in registers; the parts are added by
// another kernel.
template <int SRC, int WSRC, int LANES, int PER, bool WIDE>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void norm_grad_rows(NormBackArgs a) {
  constexpr int ROWS = LANES < 256 ? 256 / LANES : 1, KEPT = PER ? PER : 1;
  __shared__ double sums[LANES / 64];
  const int lane = threadIdx.x % LANES;
  const int64_t units = (a.cols + 7) / 8;
  float* const part = a.parts + ((int64_t)blockIdx.x * ROWS + threadIdx.x / LANES) * a.cols;
  Raw8<WSRC> w[KEPT];
  float dw[KEPT][8];
  if constexpr (PER > 0) {
    if (a.w)
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        get8<WSRC, WIDE>(w[p], a.w, (int64_t)(lane + p * LANES) * 8, a.cols);
        placed8<WSRC, WIDE>(w[p], (int64_t)(lane + p * LANES) * 8, a.cols);
      }
#pragma unroll
    for (int p = 0; p < PER; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) dw[p][i] = 0.0f;
  }
  bool first = true;
  // g of a unit, its dy beside it
  auto unit_g = [&](Raw8<SRC>& raw, const Raw8<WSRC>& wr, int64_t c, float dy[8], float g[8]) {
    floats8<SRC, WIDE>(raw, c, a.cols, dy);
    if (a.w) {
      raw_floats<WSRC>(wr, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] *= dy[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = dy[i];
    }
  };
  auto unit_dx = [&](int64_t row, int64_t c, const float g[8], const float u[8], float s, float mean, const Raw8<SRC>* dh) {
    if (c >= a.cols) return;
    float dx[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) dx[i] = s * (g[i] - u[i] * mean);
    if (dh) {
      Raw8<SRC> d = *dh;
      float v[8];
      floats8<SRC, WIDE>(d, c, a.cols, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) dx[i] += v[i];
    }
    put8<SRC>(line_to<SRC>(a.dx, row), c, a.cols, dx);
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
        get8<SRC, WIDE>(dyr[p], dyl, (int64_t)(lane + p * LANES) * 8, a.cols);
        get8<SRC, WIDE>(hr[p], hl, (int64_t)(lane + p * LANES) * 8, a.cols);
      }
      if (dhl)
#pragma unroll
        for (int p = 0; p < PER; ++p) get8<SRC, WIDE>(dhr[p], dhl, (int64_t)(lane + p * LANES) * 8, a.cols);
      float g[PER][8], u[PER][8];
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        const int64_t c = (int64_t)(lane + p * LANES) * 8;
        float dy[8];
        unit_g(dyr[p], w[p], c, dy, g[p]);
        floats8<SRC, WIDE>(hr[p], c, a.cols, u[p]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          u[p][i] *= s;
          sum = fma((double)g[p][i], (double)u[p][i], sum);
          if (mine < a.rows) dw[p][i] += dy[i] * u[p][i];
        }
      }
      const float mean = (float)(row_sum<LANES>(sum, sums) * a.inverse);
      if (mine < a.rows)
#pragma unroll
        for (int p = 0; p < PER; ++p)
          unit_dx(row, (int64_t)(lane + p * LANES) * 8, g[p], u[p], s, mean, dhl ? &dhr[p] : nullptr);
    } else {
      Raw8<SRC> dyr, hr, dhr;
      float dy[8], g[8], u[8];
      for (int64_t un = lane; un < units; un += LANES) {
        get8<SRC, WIDE>(dyr, dyl, un * 8, a.cols);
        get8<SRC, WIDE>(hr, hl, un * 8, a.cols);
        if (a.w) {
          get8<WSRC, WIDE>(w[0], a.w, un * 8, a.cols);
          placed8<WSRC, WIDE>(w[0], un * 8, a.cols);
        }
        unit_g(dyr, w[0], un * 8, dy, g);
        floats8<SRC, WIDE>(hr, un * 8, a.cols, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fma((double)g[i], (double)(u[i] * s), sum);
      }
      const float mean = (float)(row_sum<LANES>(sum, sums) * a.inverse);
      for (int64_t un = lane; un < units; un += LANES) {
        const int64_t c = un * 8;
        get8<SRC, WIDE>(dyr, dyl, c, a.cols);
        get8<SRC, WIDE>(hr, hl, c, a.cols);
        if (a.w) {
          get8<WSRC, WIDE>(w[0], a.w, c, a.cols);
          placed8<WSRC, WIDE>(w[0], c, a.cols);
        }
        if (dhl) get8<SRC, WIDE>(dhr, dhl, c, a.cols);
        unit_g(dyr, w[0], c, dy, g);
        floats8<SRC, WIDE>(hr, c, a.cols, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] *= s;
        unit_dx(row, c, g, u, s, mean, dhl ? &dhr : nullptr);
        if (a.dw)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (c + i < a.cols) part[c + i] = (first ? 0.0f : part[c + i]) + dy[i] * u[i];
      }
      first = false;
    }
  }
  if constexpr (PER > 0)
    if (a.dw)
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        const int64_t c = (int64_t)(lane + p * LANES) * 8;
        if (c < a.cols) put8<SRC_F32>(part, c, a.cols, dw[p]);
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
  for (int per : {2, 4, 8})
    if (units <= 256 * per) return {256, per};
  if (units <= 1024 * 4) return {1024, 4};
  return {1024, 0};
}

constexpr int64_t kNormGroups = 1 << 16;  // workgroups of a launch; they loop over more rows

template <template <int, int, int, int, bool> class Launch, int SRC, int WSRC, typename A>
hipError_t launch_rows(const A& a, RowPlan r, int64_t groups, hipStream_t stream) {
  if (a.cols < 8) Launch<SRC, WSRC, 64, 1, false>::go(a, groups, stream);
  else if (r.lanes == 64 && r.per == 1) Launch<SRC, WSRC, 64, 1, true>::go(a, groups, stream);
  else if (r.lanes == 64 && r.per == 2) Launch<SRC, WSRC, 64, 2, true>::go(a, groups, stream);
  else if (r.lanes == 64) Launch<SRC, WSRC, 64, 4, true>::go(a, groups, stream);
  else if (r.lanes == 256 && r.per == 2) Launch<SRC, WSRC, 256, 2, true>::go(a, groups, stream);
  else if (r.lanes == 256 && r.per == 4) Launch<SRC, WSRC, 256, 4, true>::go(a, groups, stream);
  else if (r.lanes == 256) Launch<SRC, WSRC, 256, 8, true>::go(a, groups, stream);
  else if (r.per == 4) Launch<SRC, WSRC, 1024, 4, true>::go(a, groups, stream);
  else Launch<SRC, WSRC, 1024, 0, true>::go(a, groups, stream);
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
};
template <int SRC, int WSRC, int LANES, int PER, bool WIDE>
struct Backward {
  static void go(const NormBackArgs& a, int64_t groups, hipStream_t stream) {
    norm_grad_rows<SRC, WSRC, LANES, PER, WIDE><<<dim3((unsigned)groups), LANES < 256 ? 256 : LANES, 0, stream>>>(a);
  }
};

int64_t groups_of(RowPlan r, int64_t rows) { return up_div(rows, r.lanes < 256 ? 256 / r.lanes : 1); }

}  // namespace

hipError_t launch_mx_norm(const NormArgs& a, hipStream_t stream) {
  const RowPlan r = plan_row(a.q.data ? a.q.row_scales * 4 : up_div(a.cols, 8));
  return launch_types<Forward>(a, r, std::min(groups_of(r, a.rows), kNormGroups), stream);
}

// (4 workgroups for each CU, 16 rows of each at least)
Parts mx_norm_parts(int64_t rows, int64_t cols) {
  const RowPlan r = plan_row(up_div(cols, 8));
  const int64_t per = r.lanes < 256 ? 256 / r.lanes : 1;
  return {per, std::max<int64_t>(std::min<int64_t>(up_div(groups_of(r, rows), 16), 4 * kCUs), 1) * per};
}

hipError_t launch_mx_norm_backward(const NormBackArgs& a, hipStream_t stream) {
  const RowPlan r = plan_row(up_div(a.cols, 8));
  const int64_t per = r.lanes < 256 ? 256 / r.lanes : 1;
  int64_t groups = 0;  // (no rows: dw is a sum over nothing)
  if (a.rows > 0) {
    groups = a.dw ? std::min(mx_norm_parts(a.rows, a.cols).most, a.most) / per
                  : std::min(groups_of(r, a.rows), kNormGroups);
    const hipError_t e = launch_types<Backward>(a, r, groups, stream);
    if (e != hipSuccess) return e;
  }
  if (!a.dw) return hipSuccess;
  const dim3 grid((unsigned)std::min<int64_t>(up_div(a.cols, 32), kNormGroups));
  if (a.dw_type == COSTA_REAL_F32) norm_dw<SRC_F32><<<grid, 1024, 0, stream>>>(a.parts, groups * per, a.cols, a.dw);
  else if (a.dw_type == COSTA_REAL_BF16) norm_dw<SRC_BF16><<<grid, 1024, 0, stream>>>(a.parts, groups * per, a.cols, a.dw);
  else norm_dw<SRC_F16><<<grid, 1024, 0, stream>>>(a.parts, groups * per, a.cols, a.dw);
  return hipGetLastError();
}

}  // namespace costa
