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

// a / b of a non-negative a; in 32 bits where they do (64-bit divisions take several
// times as long).
__device__ inline int64_t quotient(int64_t a, int64_t b) {
  if (((a | b) >> 32) == 0) return (int64_t)((uint32_t)a / (uint32_t)b);
  return a / b;
}

// ---- blocks along the lines of a plain matrix -------------------------------
// A lane takes 8 elements, four lanes a block; a wave reads 512 consecutive
// elements and writes them.  No shared memory.  Bound by memory: 16384^2 floats to 4
// bits 213 us, 5.7 TB/s of what is read and written (a plain copy reaches 5.1);
// 8192^2 of bfloat16 28 us, 6.0; a row of 1023 floats 2.0 us.
template <typename T, int BITS>
__global__ __launch_bounds__(kThreads) void quantize_lines(const T* src, int64_t ld, int64_t lines, int64_t len,
                                                           float alpha, MxView q) {
  const uint32_t upl = (uint32_t)(q.row_scales * 4);  // units of 8 elements of a padded line
  const int64_t units = lines * upl;
  for (int64_t u0 = (int64_t)blockIdx.x * kThreads; u0 < units; u0 += (int64_t)gridDim.x * kThreads) {
    const int64_t line0 = quotient(u0, upl);
    const uint32_t in = (uint32_t)(u0 - line0 * upl) + threadIdx.x;
    const int64_t line = line0 + in / upl;
    const uint32_t unit = in % upl;
    const int64_t c = (int64_t)unit * 8;
    const bool here = line < lines;
    float x[8];
    const T* p = src + line * ld + c;
    if (here && c + 8 <= len) {
      alignas(16) T v[8];
      __builtin_memcpy(v, p, sizeof v);  // (vector loads need no alignment)
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
// A tile is 128 lines by 128 (16-bit types, held as they are) or 64 places (held as
// 32-bit floats): 34 KiB, so that four workgroups of a CU overlap their loads with
// the others' arithmetic.  A gap of 4 bytes after every 32 elements and an odd number
// of words a line let lanes that read blocks along the lines (the blocks of a line,
// then the next line) and across them meet few equal banks.
constexpr int kLines = 128;
template <typename T>
struct Tile {
  static constexpr bool HALF = sizeof(T) == 2;
  typedef typename std::conditional<HALF, T, float>::type S;
  static constexpr int PLACES = HALF ? 128 : 64;
  static constexpr int GAP = 4 / (int)sizeof(S);
  static constexpr int STRIDE = HALF ? 138 : 67;
  static __device__ inline int at(int line, int place) { return line * STRIDE + place + place / 32 * GAP; }
};

// One block of 32 elements out of the tile, of which n are the matrix's.
template <typename T, int BITS>
__device__ inline void put_block(const typename Tile<T>::S* tile, bool across, int line, int place, int64_t n,
                                 float alpha, uint8_t* data, uint8_t* scale) {
  float x[32];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const float v = (float)(across ? tile[Tile<T>::at(line + i, place)] : tile[Tile<T>::at(line, place) + i]);
    x[i] = v * alpha;
  }
  if (n < 32)  // what pads a row is +0, whatever alpha
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = i < n ? x[i] : 0.0f;
#pragma unroll
  for (int i = 0; i < 32; ++i) m = max(m, magnitude(x[i]));
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

// The blocks of a tile in one direction: ROWS of q, BLOCKS of each.
template <typename T, bool ACROSS>
__device__ inline void put_tile(const typename Tile<T>::S* tile, const MxView& q, int64_t row0, int64_t col0,
                                float alpha) {
  constexpr int ROWS = ACROSS ? Tile<T>::PLACES : kLines, BLOCKS = (ACROSS ? kLines : Tile<T>::PLACES) / 32;
  for (int item = threadIdx.x; item < ROWS * BLOCKS; item += kThreads) {
    const int r = item / BLOCKS, b = item % BLOCKS;
    const int64_t row = row0 + r, col = col0 + 32 * b;
    if (row >= q.rows || col >= q.row_scales * kMxBlock) continue;
    uint8_t* scale = q.scales + row * q.row_scales + col / kMxBlock;
    const int line = ACROSS ? 32 * b : r, place = ACROSS ? r : 32 * b;
    const int64_t n = q.cols - col;
    if (q.bits == 4) put_block<T, 4>(tile, ACROSS, line, place, n, alpha, q.data + row * q.row_bytes + col / 2, scale);
    else put_block<T, 8>(tile, ACROSS, line, place, n, alpha, q.data + row * q.row_bytes + col, scale);
  }
}

// Where an index lies in a dimension: (class, local index).
__device__ inline void locate(const MxSplits& s, int64_t i, int32_t& cls, int64_t& local) {
  if (s.blk > 0 && s.narrow) {  // (64-bit divisions take several times as long)
    const uint32_t at = (uint32_t)(s.off + i), blk = (uint32_t)min(s.blk, (int64_t)0xffffffff), np = (uint32_t)s.np;
    const uint32_t block = at / blk, round = block / np;
    cls = (int32_t)((block - round * np + (uint32_t)s.src) % np);
    local = (int64_t)round * blk + (at - block * blk);
    return;
  }
  if (s.blk > 0) {
    const int64_t at = s.off + i, block = at / s.blk, round = block / s.np;
    cls = (int32_t)((block - round * s.np + s.src) % s.np);
    local = round * s.blk + (at - block * s.blk);
    return;
  }
  int32_t lo = 0, hi = s.n;  // start[lo] <= i < start[hi]
  while (hi - lo > 1) {
    const int32_t mid = lo + (hi - lo) / 2;
    if (s.start[mid] <= i) lo = mid;
    else hi = mid;
  }
  cls = lo;
  local = i - s.start[lo];
}

struct TileArgs {
  const void* src;
  int64_t ld, lines, len, tiles_x, tiles;
  float alpha;
  MxView along, across;
};

// A lane takes V neighbouring places of every LINES-th line, BATCH loads at a time;
// those that are next to one another in memory in one load, of any alignment.  Bound by
// memory and the way there: 16384x4096 of bfloat16 both ways in 8 bits 72 us (4.3
// TB/s; two calls, each way by itself, 34 + 38 us and two reads), 16384^2 floats out of 128x128 blocks of
// 16 ranks to 4 bits 300 to 330 us (4.0; the plain matrix by columns 275), 2501x1999 doubles out of
// 64x100 blocks 17 us (the plain matrix 12).  Tiles of 128 by 128 floats (68 KiB, two
// workgroups a CU) took 600 us on the second.
struct Dealt {
  MxLayoutArgs l;
  MxPointers ptrs;
};
struct Plain {};
template <typename T, typename Where>
__global__ __launch_bounds__(kThreads) void quantize_tiles(TileArgs a, Where where) {
  constexpr bool LAYOUT = std::is_same<Where, Dealt>::value;
  typedef Tile<T> Ti;
  typedef typename Ti::S S;
  constexpr int V = 16 / (int)sizeof(T), LANES = Ti::PLACES / V, LINES = kThreads / LANES;
  constexpr int PASSES = kLines / LINES, BATCH = PASSES < 8 ? PASSES : 8;
  __shared__ S tile[kLines * Ti::STRIDE];
  __shared__ int32_t line_cls[LAYOUT ? kLines : 1], place_cls[LAYOUT ? Ti::PLACES : 1];
  __shared__ int64_t line_local[LAYOUT ? kLines : 1], place_local[LAYOUT ? Ti::PLACES : 1];
  const int tid = threadIdx.x;
  const int place = tid % LANES * V;
  for (int64_t t = blockIdx.x; t < a.tiles; t += gridDim.x) {
    const int64_t ty = quotient(t, a.tiles_x), line0 = ty * kLines, place0 = (t - ty * a.tiles_x) * Ti::PLACES;
    const int64_t c = place0 + place;
    bool run = c + V <= a.len;
    if constexpr (LAYOUT) {
      const MxLayoutArgs& l = where.l;
      if (tid < kLines) {
        if (line0 + tid < a.lines) locate(l.line, line0 + tid, line_cls[tid], line_local[tid]);
      } else if (tid < kLines + Ti::PLACES) {
        const int k = tid - kLines;
        if (place0 + k < a.len) locate(l.place, place0 + k, place_cls[k], place_local[k]);
      }
      __syncthreads();
      run = run && place_cls[place] == place_cls[place + V - 1] &&
            place_local[place + V - 1] == place_local[place] + V - 1;
    }
    const T* base = static_cast<const T*>(a.src) + c;
    const int last = (int)min((int64_t)kLines, a.lines - line0) - 1;  // (may be below 0: padding only)
#pragma unroll 1
    for (int first = tid / LANES; first < kLines; first += LINES * BATCH) {
      alignas(16) T v[BATCH][V];
      if (run && last >= 0) {
        // all addresses, then all loads: none waits for another (lines past the last
        // repeat it and are dropped below)
        const T* from[BATCH];
#pragma unroll
        for (int q = 0; q < BATCH; ++q) {
          const int line = min(first + LINES * q, last);
          if constexpr (LAYOUT) {
            const int64_t at_cell = (int64_t)line_cls[line] * where.l.nplace + place_cls[place];
            const MxCell& cell = where.l.cells[at_cell];
            from[q] = static_cast<const T*>(where.ptrs.p[where.l.dealt ? at_cell : cell.pointer]) + cell.offset +
                      place_local[place] + line_local[line] * cell.ld;
          } else {
            from[q] = base + (line0 + line) * a.ld;
          }
        }
#pragma unroll
        for (int q = 0; q < BATCH; ++q) __builtin_memcpy(v[q], from[q], sizeof v[q]);
      } else if (last >= 0) {  // across an edge of a block or of the matrix: place by place
#pragma unroll
        for (int e = 0; e < V; ++e) {
          if (c + e >= a.len) continue;
          const T* from[BATCH];
#pragma unroll
          for (int q = 0; q < BATCH; ++q) {
            const int line = min(first + LINES * q, last);
            if constexpr (LAYOUT) {
              const int64_t at_cell = (int64_t)line_cls[line] * where.l.nplace + place_cls[place + e];
              const MxCell& cell = where.l.cells[at_cell];
              from[q] = static_cast<const T*>(where.ptrs.p[where.l.dealt ? at_cell : cell.pointer]) + cell.offset +
                        place_local[place + e] + line_local[line] * cell.ld;
            } else {
              from[q] = base + (line0 + line) * a.ld + e;
            }
          }
#pragma unroll
          for (int q = 0; q < BATCH; ++q) v[q][e] = *from[q];
        }
      }
#pragma unroll
      for (int q = 0; q < BATCH; ++q) {
        const int line = first + LINES * q;
        const bool there = line0 + line < a.lines;
#pragma unroll
        for (int e = 0; e < V; ++e) tile[Ti::at(line, place + e)] = there && c + e < a.len ? (S)v[q][e] : (S)0.0f;
      }
    }
    __syncthreads();
    if (a.along.data) put_tile<T, false>(tile, a.along, line0, place0, a.alpha);
    if (a.across.data) put_tile<T, true>(tile, a.across, place0, line0, a.alpha);
    __syncthreads();
  }
}

// ---- back -----------------------------------------------------------------------
// A lane takes 8 elements of a row.  ROWS: neighbouring lanes take neighbouring
// elements of a row (A by rows); else the same elements of neighbouring rows (A by
// columns), whose 64 writes of a column are next to one another.  Bound by memory:
// 16384^2 from 4 bits to floats 250 us (4.9 TB/s), 16384x4096 from 8 bits to bfloat16 32 to 41 us (5.0 to 6.4).
template <typename T, int BITS, bool ROWS>
__global__ __launch_bounds__(kThreads) void dequantize(DequantArgs a) {
  typedef typename std::conditional<std::is_same<T, double>::value, double, float>::type W;
  T* dst = static_cast<T*>(a.dst);
  const int64_t upr = (a.q.cols + 7) / 8;
  const int64_t units = a.q.rows * upr;
  const W alpha = (W)a.alpha, beta = (W)a.beta;
  for (int64_t u0 = (int64_t)blockIdx.x * kThreads; u0 < units; u0 += (int64_t)gridDim.x * kThreads) {
    // ROWS: u = row * upr + unit; else u = unit * rows + row
    const int64_t per = ROWS ? upr : a.q.rows;
    const int64_t o0 = quotient(u0, per);
    const uint32_t in = (uint32_t)(u0 - o0 * per) + threadIdx.x;  // (per is below 2^31)
    const uint32_t over = in / (uint32_t)per;
    const int64_t outer = o0 + over, inner = in - over * (uint32_t)per;
    const int64_t row = ROWS ? outer : inner, unit = ROWS ? inner : outer;
    if (outer >= (ROWS ? a.q.rows : upr)) continue;
    v2u d = {0u, 0u};
    if (BITS == 4) d.x = *reinterpret_cast<const uint32_t*>(a.q.data + row * a.q.row_bytes + unit * 4);
    else d = *reinterpret_cast<const v2u*>(a.q.data + row * a.q.row_bytes + unit * 8);
    float x[8];
    mx_decode8<BITS>(d, a.q.scales[row * a.q.row_scales + unit / 4], x);
    T* p = dst + row * a.rs + unit * 8 * a.cs;
    const int n = (int)min((int64_t)8, a.q.cols - unit * 8);
    if (ROWS && n == 8) {  // (vector accesses need no alignment)
      alignas(16) T v[8];
      if (a.beta != 0.0f) {
        __builtin_memcpy(v, p, sizeof v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (T)(alpha * (W)x[i] + beta * (W)v[i]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (T)(alpha * (W)x[i]);
      }
      __builtin_memcpy(p, v, sizeof v);
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
  const int64_t units = a.lines * a.along.row_scales * 4;
  const dim3 grid = grid_for((units + kThreads - 1) / kThreads);
  const T* src = static_cast<const T*>(a.src);
  if (a.along.bits == 4)
    quantize_lines<T, 4><<<grid, kThreads, 0, stream>>>(src, a.ld, a.lines, a.len, a.alpha, a.along);
  else
    quantize_lines<T, 8><<<grid, kThreads, 0, stream>>>(src, a.ld, a.lines, a.len, a.alpha, a.along);
  return hipGetLastError();
}

// Tiles that cover the source and what pads either output.
template <typename T>
TileArgs tiles_of(const QuantArgs& a) {
  constexpr int PLACES = Tile<T>::PLACES;
  int64_t nx = (a.len + PLACES - 1) / PLACES, ny = (a.lines + kLines - 1) / kLines;
  if (a.along.data) nx = std::max(nx, a.along.row_scales * kMxBlock / PLACES);
  if (a.across.data) ny = std::max(ny, a.across.row_scales * kMxBlock / kLines);
  return TileArgs{a.src, a.ld, a.lines, a.len, nx, nx * ny, a.alpha, a.along, a.across};
}

template <typename T>
hipError_t quantize_tiled(const QuantArgs& a, hipStream_t stream) {
  const TileArgs t = tiles_of<T>(a);
  quantize_tiles<T, Plain><<<grid_for(t.tiles), kThreads, 0, stream>>>(t, Plain{});
  return hipGetLastError();
}

template <typename T>
hipError_t quantize_dealt(const QuantArgs& a, const MxLayoutArgs& l, const MxPointers& p, hipStream_t stream) {
  const TileArgs t = tiles_of<T>(a);
  quantize_tiles<T, Dealt><<<grid_for(t.tiles), kThreads, 0, stream>>>(t, Dealt{l, p});
  return hipGetLastError();
}

template <typename T, int BITS>
hipError_t dequantize_typed(const DequantArgs& a, hipStream_t stream) {
  const int64_t units = a.q.rows * ((a.q.cols + 7) / 8);
  const dim3 grid = grid_for((units + kThreads - 1) / kThreads);
  if (a.cs == 1) dequantize<T, BITS, true><<<grid, kThreads, 0, stream>>>(a);
  else dequantize<T, BITS, false><<<grid, kThreads, 0, stream>>>(a);
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
