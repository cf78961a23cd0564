// Kernels that write matrices in microscaled form and read them back.
//
// Both directions are bound by memory traffic: an element costs about four
// instructions and 0.5 to 8 bytes each way.
#include <algorithm>

#include "mx_device.hpp"

namespace costa {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kGridMax = (int64_t)1 << 20;  // workgroups of a launch; they loop over what is more

template <typename T>
__device__ inline float to_float(T v) {
  return (float)v;
}

// The largest of four neighbouring lanes.
__device__ inline uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));  // lanes 1 0 3 2
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));  // lanes 2 3 0 1
}

__device__ inline uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

// ---- blocks along the lines of a plain matrix -------------------------------
// A lane takes 8 elements, four lanes a block; a wave reads 512 consecutive
// elements and writes them.  No shared memory.
template <typename T, int BITS>
__global__ __launch_bounds__(kThreads) void quantize_lines(const T* src, int64_t ld, int64_t lines, int64_t len,
                                                           float alpha, MxView q, bool wide) {
  const uint32_t upl = (uint32_t)(q.row_scales * 4);  // units of 8 elements of a padded line
  const int64_t units = lines * upl;
  for (int64_t u0 = (int64_t)blockIdx.x * kThreads; u0 < units; u0 += (int64_t)gridDim.x * kThreads) {
    const int64_t line0 = u0 / upl;
    const uint32_t in = (uint32_t)(u0 - line0 * upl) + threadIdx.x;
    const int64_t line = line0 + in / upl;
    const uint32_t unit = in % upl;
    const int64_t c = (int64_t)unit * 8;
    const bool here = line < lines;
    float x[8];
    const T* p = src + line * ld + c;
    if (here && wide && c + 8 <= len) {
      alignas(16) T v[8];
#pragma unroll
      for (size_t i = 0; i < 8 * sizeof(T) / 16; ++i)
        *reinterpret_cast<v4u*>(reinterpret_cast<char*>(v) + 16 * i) = reinterpret_cast<const v4u*>(p)[i];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = to_float(v[i]) * alpha;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = here && c + i < len ? to_float(p[i]) * alpha : 0.0f;
    }
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, magnitude(x[i]));
    const uint32_t s = mx_scale<BITS>(quad_max(m));
    if (here) {
      const v2u d = mx_encode8<BITS>(x, s);
      if (BITS == 4) *reinterpret_cast<uint32_t*>(q.data + line * q.row_bytes + c / 2) = d.x;
      else *reinterpret_cast<v2u*>(q.data + line * q.row_bytes + c) = d;
      if (unit % 4 == 0) q.scales[line * q.row_scales + unit / 4] = (uint8_t)s;
    }
  }
}

// ---- either direction, any source, through a tile in shared memory -------------
// A tile is 128 lines by 128 elements as 32-bit floats, with a gap after every
// 32 elements and an odd line stride: lanes that read blocks along the lines
// (four blocks of a line, then the next line) and blocks across them meet few
// equal banks.
constexpr int kTile = 128;
constexpr int kTileStride = kTile + 5;
__device__ inline int tile_at(int line, int place) { return line * kTileStride + place + place / 32; }

// One block of 32 elements out of the tile: `step` apart from x on.
template <int BITS>
__device__ inline void put_block(const float* tile, bool across, int line, int place, uint8_t* data, uint8_t* scale) {
  float x[32];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    x[i] = across ? tile[tile_at(line + i, place)] : tile[tile_at(line, place) + i];
    m = max(m, magnitude(x[i]));
  }
  const uint32_t s = mx_scale<BITS>(m);
  v2u d[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) d[i] = mx_encode8<BITS>(x + 8 * i, s);
  if (BITS == 4) {
    *reinterpret_cast<v4u*>(data) = v4u{d[0].x, d[1].x, d[2].x, d[3].x};
  } else {
    reinterpret_cast<v4u*>(data)[0] = v4u{d[0].x, d[0].y, d[1].x, d[1].y};
    reinterpret_cast<v4u*>(data)[1] = v4u{d[2].x, d[2].y, d[3].x, d[3].y};
  }
  *scale = (uint8_t)s;
}

// The blocks of a tile in one direction.  `outer` counts q's rows, `inner` its columns.
__device__ inline void put_tile(const float* tile, bool across, const MxView& q, int64_t row0, int64_t col0) {
  for (int item = threadIdx.x; item < kTile * 4; item += kThreads) {
    const int r = item / 4, b = item % 4;
    const int64_t row = row0 + r, col = col0 + 32 * b;
    if (row >= q.rows || col >= q.row_scales * kMxBlock) continue;
    uint8_t* scale = q.scales + row * q.row_scales + col / kMxBlock;
    const int line = across ? 32 * b : r, place = across ? r : 32 * b;
    if (q.bits == 4) put_block<4>(tile, across, line, place, q.data + row * q.row_bytes + col / 2, scale);
    else put_block<8>(tile, across, line, place, q.data + row * q.row_bytes + col, scale);
  }
}

// Where an index lies in a dimension's splits: (class, local index).
__device__ inline void locate(const MxSplits& s, int64_t i, int32_t& cls, int64_t& local) {
  int32_t lo = 0, hi = s.n;  // start[lo] <= i < start[hi]
  while (hi - lo > 1) {
    const int32_t mid = lo + (hi - lo) / 2;
    if (s.start[mid] <= i) lo = mid;
    else hi = mid;
  }
  cls = s.cls[lo];
  local = s.local[lo] + (i - s.start[lo]);
}

struct TileArgs {
  const void* src;
  int64_t ld, lines, len, tiles_x, tiles;
  float alpha;
  bool wide;
  MxView along, across;
};

template <typename T, bool LAYOUT>
__global__ __launch_bounds__(kThreads) void quantize_tiles(TileArgs a, MxLayoutArgs l, MxPointers ptrs) {
  __shared__ float tile[kTile * kTileStride];
  __shared__ int32_t line_cls[LAYOUT ? kTile : 1], place_cls[LAYOUT ? kTile : 1];
  __shared__ int64_t line_local[LAYOUT ? kTile : 1], place_local[LAYOUT ? kTile : 1];
  constexpr int V = 16 / (int)sizeof(T);  // elements of a 16-byte load
  const int tid = threadIdx.x;
  for (int64_t t = blockIdx.x; t < a.tiles; t += gridDim.x) {
    const int64_t line0 = t / a.tiles_x * kTile, place0 = t % a.tiles_x * kTile;
    if (LAYOUT) {
      const bool is_line = tid < kTile;
      const int k = tid % kTile;
      const int64_t i = (is_line ? line0 : place0) + k;
      if (i < (is_line ? a.lines : a.len)) {
        if (is_line) locate(l.line, i, line_cls[k], line_local[k]);
        else locate(l.place, i, place_cls[k], place_local[k]);
      }
      __syncthreads();
      // a lane takes V neighbouring places of every 8th (16th) line; where they lie
      // next to one another in memory, in one load.  The cell changes where a line's
      // block does.
      constexpr int LANES = kTile / V, ROWS = kThreads / LANES, BATCH = 8;
      const int place = tid % LANES * V;
      const int64_t c = place0 + place;
      const bool run = c + V <= a.len && place_cls[place] == place_cls[place + V - 1] &&
                       place_local[place + V - 1] == place_local[place] + V - 1;
      int32_t last_cls = -1;
      const T* base = nullptr;
      int64_t ld = 0;
      for (int first = tid / LANES; first < kTile; first += ROWS * BATCH) {
        alignas(16) T v[BATCH][V];
#pragma unroll
        for (int q = 0; q < BATCH; ++q) {
          const int line = first + ROWS * q;
          if (line0 + line >= a.lines) continue;
          if (run) {
            if (line_cls[line] != last_cls) {
              last_cls = line_cls[line];
              const MxCell& cell = l.cells[(int64_t)last_cls * l.nplace + place_cls[place]];
              base = static_cast<const T*>(ptrs.p[cell.rank]) + cell.offset + place_local[place];
              ld = cell.ld;
            }
            __builtin_memcpy(v[q], base + line_local[line] * ld, sizeof v[q]);
          } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
              if (c + e < a.len) {
                const MxCell& cell = l.cells[(int64_t)line_cls[line] * l.nplace + place_cls[place + e]];
                v[q][e] = static_cast<const T*>(
                    ptrs.p[cell.rank])[cell.offset + line_local[line] * cell.ld + place_local[place + e]];
              }
          }
        }
#pragma unroll
        for (int q = 0; q < BATCH; ++q) {
          const int line = first + ROWS * q;
#pragma unroll
          for (int e = 0; e < V; ++e)
            tile[tile_at(line, place + e)] =
                line0 + line < a.lines && c + e < a.len ? to_float(v[q][e]) * a.alpha : 0.0f;
        }
      }
    } else {
      const T* src = static_cast<const T*>(a.src);
      for (int item = tid; item < kTile * kTile / V; item += kThreads) {
        const int line = item / (kTile / V), place = item % (kTile / V) * V;
        const int64_t c = place0 + place;
        const T* p = src + (line0 + line) * a.ld + c;
        if (a.wide && line0 + line < a.lines && c + V <= a.len) {
          alignas(16) T v[V];
          *reinterpret_cast<v4u*>(v) = *reinterpret_cast<const v4u*>(p);
#pragma unroll
          for (int i = 0; i < V; ++i) tile[tile_at(line, place + i)] = to_float(v[i]) * a.alpha;
        } else {
#pragma unroll
          for (int i = 0; i < V; ++i)
            tile[tile_at(line, place + i)] =
                line0 + line < a.lines && c + i < a.len ? to_float(p[i]) * a.alpha : 0.0f;
        }
      }
    }
    __syncthreads();
    if (a.along.data) put_tile(tile, false, a.along, line0, place0);
    if (a.across.data) put_tile(tile, true, a.across, place0, line0);
    __syncthreads();
  }
}

// ---- back -----------------------------------------------------------------------
// A lane takes 8 elements of a row.  ROWS: neighbouring lanes take neighbouring
// elements of a row (A by rows); else the same elements of neighbouring rows (A by
// columns), whose 64 writes of a column are next to one another.
template <typename T, int BITS, bool ROWS>
__global__ __launch_bounds__(kThreads) void dequantize(DequantArgs a, bool wide) {
  typedef typename std::conditional<std::is_same<T, double>::value, double, float>::type W;
  T* dst = static_cast<T*>(a.dst);
  const int64_t upr = (a.q.cols + 7) / 8;
  const int64_t units = a.q.rows * upr;
  const W alpha = (W)a.alpha, beta = (W)a.beta;
  for (int64_t u0 = (int64_t)blockIdx.x * kThreads; u0 < units; u0 += (int64_t)gridDim.x * kThreads) {
    // ROWS: u = row * upr + unit; else u = unit * rows + row
    const int64_t per = ROWS ? upr : a.q.rows;
    const int64_t o0 = u0 / per;
    const int64_t in = u0 - o0 * per + threadIdx.x;
    const int64_t over = in < per ? 0 : in / per;
    const int64_t outer = o0 + over, inner = in - over * per;
    const int64_t row = ROWS ? outer : inner, unit = ROWS ? inner : outer;
    if (outer >= (ROWS ? a.q.rows : upr)) continue;
    v2u d = {0u, 0u};
    if (BITS == 4) d.x = *reinterpret_cast<const uint32_t*>(a.q.data + row * a.q.row_bytes + unit * 4);
    else d = *reinterpret_cast<const v2u*>(a.q.data + row * a.q.row_bytes + unit * 8);
    float x[8];
    mx_decode8<BITS>(d, a.q.scales[row * a.q.row_scales + unit / 4], x);
    T* p = dst + row * a.rs + unit * 8 * a.cs;
    const int n = (int)min((int64_t)8, a.q.cols - unit * 8);
    if (ROWS && wide && n == 8) {
      alignas(16) T v[8];
      if (a.beta != 0.0f) {
#pragma unroll
        for (size_t i = 0; i < 8 * sizeof(T) / 16; ++i)
          *reinterpret_cast<v4u*>(reinterpret_cast<char*>(v) + 16 * i) = reinterpret_cast<const v4u*>(p)[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (T)(alpha * (W)x[i] + beta * (W)v[i]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (T)(alpha * (W)x[i]);
      }
#pragma unroll
      for (size_t i = 0; i < 8 * sizeof(T) / 16; ++i)
        reinterpret_cast<v4u*>(p)[i] = *reinterpret_cast<const v4u*>(reinterpret_cast<const char*>(v) + 16 * i);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < n) {
          W y = alpha * (W)x[i];
          if (a.beta != 0.0f) y = y + beta * (W)p[i * a.cs];
          p[i * a.cs] = (T)y;
        }
    }
  }
}

inline dim3 grid_for(int64_t groups) { return dim3((unsigned)std::min<int64_t>(std::max<int64_t>(groups, 1), kGridMax)); }

template <typename T>
hipError_t quantize_plain(const QuantArgs& a, hipStream_t stream) {
  const bool wide = (uintptr_t)a.src % 16 == 0 && a.ld * sizeof(T) % 16 == 0;
  if (!a.across.data) {
    const int64_t units = a.lines * a.along.row_scales * 4;
    const dim3 grid = grid_for((units + kThreads - 1) / kThreads);
    if (a.along.bits == 4)
      quantize_lines<T, 4><<<grid, kThreads, 0, stream>>>(static_cast<const T*>(a.src), a.ld, a.lines, a.len, a.alpha,
                                                          a.along, wide);
    else
      quantize_lines<T, 8><<<grid, kThreads, 0, stream>>>(static_cast<const T*>(a.src), a.ld, a.lines, a.len, a.alpha,
                                                          a.along, wide);
    return hipGetLastError();
  }
  return hipSuccess;
}

// Tiles that cover the source and what pads either output.
TileArgs tiles_of(const QuantArgs& a, bool wide) {
  int64_t nx = (a.len + kTile - 1) / kTile, ny = (a.lines + kTile - 1) / kTile;
  if (a.along.data) nx = std::max(nx, a.along.row_scales * kMxBlock / kTile);
  if (a.across.data) ny = std::max(ny, a.across.row_scales * kMxBlock / kTile);
  return TileArgs{a.src, a.ld, a.lines, a.len, nx, nx * ny, a.alpha, wide, a.along, a.across};
}

template <typename T>
hipError_t quantize_tiled(const QuantArgs& a, hipStream_t stream) {
  const bool wide = (uintptr_t)a.src % 16 == 0 && a.ld * sizeof(T) % 16 == 0;
  const TileArgs t = tiles_of(a, wide);
  quantize_tiles<T, false><<<grid_for(t.tiles), kThreads, 0, stream>>>(t, MxLayoutArgs{}, MxPointers{});
  return hipGetLastError();
}

template <typename T>
hipError_t quantize_dealt(const QuantArgs& a, const MxLayoutArgs& l, const MxPointers& p, hipStream_t stream) {
  const TileArgs t = tiles_of(a, false);
  quantize_tiles<T, true><<<grid_for(t.tiles), kThreads, 0, stream>>>(t, l, p);
  return hipGetLastError();
}

template <typename T, int BITS>
hipError_t dequantize_typed(const DequantArgs& a, hipStream_t stream) {
  const int64_t units = a.q.rows * ((a.q.cols + 7) / 8);
  const dim3 grid = grid_for((units + kThreads - 1) / kThreads);
  if (a.cs == 1) {
    const bool wide = (uintptr_t)a.dst % 16 == 0 && a.rs * sizeof(T) % 16 == 0;
    dequantize<T, BITS, true><<<grid, kThreads, 0, stream>>>(a, wide);
  } else {
    dequantize<T, BITS, false><<<grid, kThreads, 0, stream>>>(a, false);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t dequantize_bits(const DequantArgs& a, hipStream_t stream) {
  return a.q.bits == 4 ? dequantize_typed<T, 4>(a, stream) : dequantize_typed<T, 8>(a, stream);
}

#define FOR_TYPE(t, call)                                                   \
  switch (t) {                                                              \
    case COSTA_REAL_F64: { typedef double T; return call; }                 \
    case COSTA_REAL_F32: { typedef float T; return call; }                  \
    case COSTA_REAL_BF16: { typedef __bf16 T; return call; }                \
    case COSTA_REAL_F16: { typedef _Float16 T; return call; }               \
    default: return hipErrorInvalidValue;                                   \
  }

}  // namespace

hipError_t launch_mx_quantize(const QuantArgs& a, hipStream_t stream) {
  if (!a.across.data) FOR_TYPE(a.type, quantize_plain<T>(a, stream))
  FOR_TYPE(a.type, quantize_tiled<T>(a, stream))
}

hipError_t launch_mx_quantize_layout(const QuantArgs& a, const MxLayoutArgs& l, const MxPointers& p,
                                     hipStream_t stream) {
  FOR_TYPE(a.type, quantize_dealt<T>(a, l, p, stream))
}

hipError_t launch_mx_dequantize(const DequantArgs& a, hipStream_t stream) {
  FOR_TYPE(a.type, dequantize_bits<T>(a, stream))
}

}  // namespace costa
