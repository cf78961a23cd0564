// Low-rank adapters, another one for each row, beside a product:
//
//     v_i = x_i A_a^T,   c_i = alpha p_i + s_a v_i B_a + beta c_i,   a = index[i]
//     g_a = s_a sum over the rows i of a of v_i^T z_i
//
// A and B are kept rank by rank, so that one kernel makes the products of rows with an
// adapter's rows (A; B in the backward pass), one adds combinations of an adapter's
// rows (B; A), and one sums either gradient.
//
// Bound by memory: x, the product's sums and c go by once, and of an adapter 2 rank
// operations come to an element of them.  v is kept in 32 bits; it enters a matrix
// instruction as three bfloat16 parts, which hold it, and an adapter's elements as one
// (bfloat16), two (float16) or three (float): products of parts whose places add up to
// less than 2^-24 are left out.
//
// Rows go by sixteen, the width of a matrix instruction, and each distinct adapter among
// them (mostly one: a prompt's rows have the same) by turns: the instruction makes all
// sixteen rows' results with it, and those that are its own are taken.  (Rows of other
// adapters are not set to zero before: an infinity of one request's adapter times a
// zero would be a NaN in another's rows.)
#include <algorithm>

#include "mx_layer.hpp"
#include "mx_rows.hpp"

namespace costa {
namespace {

__device__ inline int32_t adapter_of(const AdapterIndex& at, int64_t row) {
  const int32_t a = at.index[row];
  return a >= 0 && a < at.count ? a : -1;
}
__device__ inline int rank_of(const AdapterIndex& at, int32_t a) {
  if (a < 0) return 0;
  return at.ranks ? min(max(at.ranks[a], 0), at.rank) : at.rank;
}
__device__ inline float scale_of(const AdapterIndex& at, int32_t a) { return at.scales ? at.scales[a] : 1.0f; }

// ---- few rows: a row at a time, on the vector units ----------------------------
// A workgroup makes RANKS of a row's products; its lanes go along the row.  The time is that
// of reading the adapters' rows, all of them on their way at once.
constexpr int kDotRanks = 4;
template <int SRC, bool WIDE>
__global__ __launch_bounds__(256) void adapter_dots_row(AdapterDotsArgs p, int64_t row0) {
  __shared__ float red[4][kDotRanks];
  const int64_t row = row0 + blockIdx.x;
  const int r0 = blockIdx.y * kDotRanks;
  const int32_t a = adapter_of(p.at, row);
  const int rank = rank_of(p.at, a);
  float sum[kDotRanks] = {};
  if (r0 < rank) {
    const void* const xl = line_of<SRC>(p.x, row);
    const void* al[kDotRanks];
#pragma unroll
    for (int j = 0; j < kDotRanks; ++j)  // (past the last row: that again, and its product is not taken)
      al[j] = line_of<SRC>(p.low, (int64_t)a * p.at.rank + min(r0 + j, rank - 1));
#pragma unroll 4
    for (int64_t k = threadIdx.x * 8; k < p.k; k += 2048) {
      Raw8<SRC> xr, ar[kDotRanks];
      get8<SRC, WIDE>(xr, xl, k, p.k);
#pragma unroll
      for (int j = 0; j < kDotRanks; ++j) get8<SRC, WIDE>(ar[j], al[j], k, p.k);
      float x[8], y[8];
      floats8<SRC, WIDE>(xr, k, p.k, x);
#pragma unroll
      for (int j = 0; j < kDotRanks; ++j) {
        floats8<SRC, WIDE>(ar[j], k, p.k, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[j] = fmaf(x[i], y[i], sum[j]);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < kDotRanks; ++j) {
#pragma unroll
    for (int by = 32; by > 0; by /= 2) sum[j] += __shfl_xor(sum[j], by);
    if (threadIdx.x % 64 == 0) red[threadIdx.x / 64][j] = sum[j];
  }
  __syncthreads();
  const int j = threadIdx.x, r = r0 + j;
  if (j < kDotRanks && r < p.at.rank)
    p.v[row * p.v_ld + r] = r < rank ? (red[0][j] + red[1][j]) + (red[2][j] + red[3][j]) : 0.0f;
}

// c's elements c .. c + 7 of a row: the product's parts, what the adapter adds, c.
template <int CSRC>
__device__ inline void put_sums(const AdapterAddArgs& p, int64_t row, int64_t c, const float add[8]) {
  float v[8] = {};
  const bool all = c + 8 <= p.n;
  const float* part = p.parts + row * p.n + c;
  for (int s = 0; s < p.splits; ++s, part += p.m * p.n) {
    if (all) {
      float w[8];
      __builtin_memcpy(w, part, sizeof w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += w[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < p.n) v[i] += part[i];
    }
  }
  if (p.splits > 0)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= p.alpha;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] += add[i];
  if (p.beta != 0.0f) {
    const Elem<CSRC>* old = static_cast<const Elem<CSRC>*>(p.c.data) + row * p.c.ld + c;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < p.n) v[i] += p.beta * (float)old[i];
  }
  put8<CSRC>(line_to<CSRC>(p.c, row), c, p.n, v);
}
__device__ inline void put_sums_typed(const AdapterAddArgs& p, int64_t row, int64_t c, const float add[8]) {
  if (p.c_type == COSTA_REAL_F32) put_sums<SRC_F32>(p, row, c, add);
  else if (p.c_type == COSTA_REAL_BF16) put_sums<SRC_BF16>(p, row, c, add);
  else put_sums<SRC_F16>(p, row, c, add);
}

// A workgroup has 2048 columns of a row, eight a lane.
template <int SRC, bool WIDE>
__global__ __launch_bounds__(256) void adapter_add_row(AdapterAddArgs p, int64_t row0, int64_t col0) {
  const int64_t row = row0 + blockIdx.x, c = col0 + ((int64_t)blockIdx.y * 256 + threadIdx.x) * 8;
  const int32_t a = adapter_of(p.at, row);
  const int rank = rank_of(p.at, a);
  float add[8] = {};
  if (rank > 0) {
    const float* const v = p.v + row * p.v_ld;
#pragma unroll 8
    for (int r = 0; r < rank; ++r) {
      Raw8<SRC> raw;
      float b[8];
      get8<SRC, WIDE>(raw, line_of<SRC>(p.low, (int64_t)a * p.at.rank + r), c, p.n);
      floats8<SRC, WIDE>(raw, c, p.n, b);
      const float x = v[r];
#pragma unroll
      for (int i = 0; i < 8; ++i) add[i] = fmaf(x, b[i], add[i]);
    }
    const float s = scale_of(p.at, a);
#pragma unroll
    for (int i = 0; i < 8; ++i) add[i] *= s;
  }
  if (c < p.n) put_sums_typed(p, row, c, add);
}

// ---- many rows: sixteen at a time, on the matrix units --------------------------
// The distinct adapters of the lanes l < 16 whose rows are there: by turns, each with the lanes
// that have it.  `left` holds the lanes to come; -1 (no adapter) is one of them.
struct Turn {
  int32_t a;
  bool mine;  // this lane's row (l % 16) has it
};
__device__ inline bool next_turn(uint64_t& left, int32_t idx, Turn& t) {
  if (left == 0) return false;
  t.a = __builtin_amdgcn_readlane(idx, (int)__builtin_ctzll(left));
  const uint64_t same = __ballot(idx == t.a);
  t.mine = idx == t.a;
  left &= ~same;
  return true;
}

// Sums of products of parts, those of 2^-24 and less left out.
template <int PA, int PB>
__device__ inline v4f mfma_parts(const v4u* a, const v4u* b, v4f c) {
#pragma unroll
  for (int i = 0; i < PA; ++i)
#pragma unroll
    for (int j = 0; j < PB; ++j)
      if (i + j < 3) c = mfma_bf16(a[i], b[j], c);
  return c;
}

// A workgroup has sixteen rows and 16 RT ranks; its eight waves take 128 elements of the rows
// in turn, straight to registers in the instruction's order (lane l: row l % 16, eight
// elements from 8 (l / 16) of each 32), and their sums are joined through shared memory.
constexpr int kDotWaves = 8, kDotSpan = 128;
template <int SRC, int RT, bool WIDE>
__global__ __launch_bounds__(64 * kDotWaves) void adapter_dots_tile(AdapterDotsArgs p, int64_t row0) {
  constexpr int P = parts_of(SRC), STEPS = kDotSpan / 32;
  __shared__ v4f red[kDotWaves][RT][64];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = lane % 16,
            g = lane / 16;
  const int64_t i0 = row0 + (int64_t)blockIdx.x * 16, row = min(i0 + l, p.m - 1);
  const int r0 = blockIdx.y * 16 * RT;
  const int32_t idx = i0 + l < p.m ? adapter_of(p.at, row) : -1;
  const void* const xl = line_of<SRC>(p.x, row);
  v4f all[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) all[t] = v4f{0, 0, 0, 0};
  uint64_t left = __ballot(idx >= 0);
  Turn turn;
  while (next_turn(left, idx, turn)) {
    const int rank = rank_of(p.at, turn.a);
    if (r0 >= rank) continue;
    const void* al[RT];
    v4f acc[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {  // (past the last row: that again, and its product is not taken)
      al[t] = line_of<SRC>(p.low, (int64_t)turn.a * p.at.rank + min(r0 + 16 * t + l, rank - 1));
      acc[t] = v4f{0, 0, 0, 0};
    }
    for (int64_t k0 = wave * kDotSpan; k0 < p.k; k0 += kDotWaves * kDotSpan) {
      Raw8<SRC> x[STEPS], a[STEPS][RT];
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        const int64_t k = k0 + 32 * s + 8 * g;
        get8<SRC, WIDE>(x[s], xl, k, p.k);
#pragma unroll
        for (int t = 0; t < RT; ++t) get8<SRC, WIDE>(a[s][t], al[t], k, p.k);
      }
      if (k0 + kDotSpan > p.k)
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
          const int64_t k = k0 + 32 * s + 8 * g;
          placed8<SRC, WIDE>(x[s], k, p.k);
#pragma unroll
          for (int t = 0; t < RT; ++t) placed8<SRC, WIDE>(a[s][t], k, p.k);
        }
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        v4u xp[P], ap[P];
        raw_parts<SRC>(x[s], xp);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          raw_parts<SRC>(a[s][t], ap);
          acc[t] = mfma_parts<P, P>(ap, xp, acc[t]);
        }
      }
    }
    // lane: row l, ranks r0 + 16 t + 4 g .. + 3
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (turn.mine && r0 + 16 * t + 4 * g + q < rank) all[t][q] = acc[t][q];
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) red[wave][t][lane] = all[t];
  __syncthreads();
  for (int u = threadIdx.x; u < RT * 64; u += 64 * kDotWaves) {
    const int t = u / 64, at = u % 64;
    v4f sum = red[0][t][at];
#pragma unroll
    for (int w = 1; w < kDotWaves; ++w) sum += red[w][t][at];
    const int64_t i = i0 + at % 16;
    const int r = r0 + 16 * t + at / 16 * 4;
    if (i < p.m)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (r + q < p.at.rank) p.v[i * p.v_ld + r + q] = sum[q];
  }
}

// Zeros in place of what is not there.
template <int SRC>
__device__ inline void keep8(Raw8<SRC>& r, bool there) {
#pragma unroll
  for (int i = 0; i < (int)(sizeof r.w / 4); ++i) r.w[i] = there ? r.w[i] : 0u;
}

// Eight rows of eight neighbouring columns, as lane l of a wave loads them (rows 8 (l / 16) ..
// + 7, columns 8 (l % 16) .. + 7): column e of each lane is an operand of the matrix
// instruction whose sixteen columns are e, 8 + e, 16 + e ..  No shared memory.
template <int SRC>
__device__ inline void column_parts(const Raw8<SRC> z[8], int e, v4u out[parts_of(SRC)]) {
  Raw8<SRC> r;
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    if constexpr (bytes_of(SRC) == 4) r.w[q] = z[q].w[e];
    else if (q % 2 == 0)
      r.w[q / 2] = __builtin_amdgcn_perm(z[q + 1].w[e / 2], z[q].w[e / 2], e % 2 ? 0x07060302u : 0x05040100u);
  }
  raw_parts<SRC>(r, out);
}

// A wave has 16 S rows and 128 columns; four waves of a workgroup have the same columns of
// rows that follow one another.  The results lie so that a lane has four runs of eight columns
// of a row.
template <int SRC, int S, bool WIDE>
__global__ __launch_bounds__(256) void adapter_add_tile(AdapterAddArgs p, int64_t row0, int64_t col0) {
  constexpr int P = parts_of(SRC);
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = lane % 16,
            g = lane / 16;
  const int64_t i0 = row0 + ((int64_t)blockIdx.x * 4 + wave) * 16 * S,
                j0 = col0 + (int64_t)blockIdx.y * 128;
  if (i0 >= p.m) return;
  int32_t idx[S];
  uint64_t left[S], any = 0;
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int64_t row = i0 + 16 * s + l;
    idx[s] = row < p.m ? adapter_of(p.at, row) : -2;
    left[s] = __ballot(idx[s] != -2);
    any |= left[s];
  }
  while (any) {
    // the first strip's next adapter, and the strips that have it
    int32_t a = -2;
#pragma unroll
    for (int s = S - 1; s >= 0; --s)
      if (left[s]) a = __builtin_amdgcn_readlane(idx[s], (int)__builtin_ctzll(left[s]));
    uint64_t has[S];
    any = 0;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      has[s] = __ballot(idx[s] == a);
      left[s] &= ~has[s];
      any |= left[s];
    }
    const int rank = rank_of(p.at, a);
    const float scale = a < 0 ? 0.0f : scale_of(p.at, a);
    v4f acc[S][8];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[s][e] = v4f{0, 0, 0, 0};
    for (int r0 = 0; r0 < rank; r0 += 32) {
      Raw8<SRC> b[8];
#pragma unroll
      for (int q = 0; q < 8; ++q)
        get8<SRC, WIDE>(b[q], line_of<SRC>(p.low, (int64_t)a * p.at.rank + min(r0 + 8 * g + q, rank - 1)), j0 + 8 * l, p.n);
      if (j0 + 128 > p.n)
#pragma unroll
        for (int q = 0; q < 8; ++q) placed8<SRC, WIDE>(b[q], j0 + 8 * l, p.n);
      if (r0 + 32 > rank)
#pragma unroll
        for (int q = 0; q < 8; ++q) keep8<SRC>(b[q], r0 + 8 * g + q < rank);
      v4u v[S][3];
#pragma unroll
      for (int s = 0; s < S; ++s) {
        if (!has[s]) continue;
        const float* at = p.v + min(i0 + 16 * s + l, p.m - 1) * p.v_ld + r0 + 8 * g;
        Raw8<SRC_F32> raw;
#pragma unroll
        for (int q = 0; q < 8; ++q)
          raw.w[q] = r0 + 8 * g + q < rank ? __builtin_bit_cast(uint32_t, scale * at[q]) : 0u;
        raw_parts<SRC_F32>(raw, v[s]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v4u bp[P];
        column_parts<SRC>(b, e, bp);
#pragma unroll
        for (int s = 0; s < S; ++s)
          if (has[s]) acc[s][e] = mfma_parts<P, 3>(bp, v[s], acc[s][e]);
      }
    }
#pragma unroll
    for (int s = 0; s < S; ++s) {
      if (idx[s] != a) continue;
      const int64_t row = i0 + 16 * s + l;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float add[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) add[e] = acc[s][e][q];
        const int64_t c = j0 + 8 * (4 * g + q);
        if (c < p.n) put_sums_typed(p, row, c, add);
      }
    }
  }
}

// ---- gradients --------------------------------------------------------------------
// A workgroup's four waves have 128 columns each of 16 RT ranks of an adapter, and a part of the
// rows, of which those of the adapter are listed in shared memory, 2048 rows at a time, and
// taken by 32.
constexpr int kListed = 2048;
template <int SRC, int RT, bool WIDE>
__global__ __launch_bounds__(256) void adapter_grad_tile(AdapterGradArgs p, int64_t col0, int64_t pair0,
                                                         int64_t per) {
  constexpr int P = parts_of(SRC);
  __shared__ int32_t list[kListed + 32];
  __shared__ int32_t counts[4];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = lane % 16,
            g = lane / 16;
  const int chunks = (p.at.rank + 16 * RT - 1) / (16 * RT);
  const int32_t pair = (int32_t)(pair0 + blockIdx.y), a = pair / chunks;
  const int r0 = pair % chunks * 16 * RT, rank = rank_of(p.at, a);
  const int64_t j0 = col0 + ((int64_t)blockIdx.x * 4 + wave) * 128, j = j0 + 8 * l;
  const int64_t first = (int64_t)blockIdx.z * per, last = min(first + per, p.m);
  v4f acc[RT][8];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[t][e] = v4f{0, 0, 0, 0};
  for (int64_t from = first; r0 < rank && from < last; from += kListed) {
    int n = 0;
    for (int64_t at = from; at < min(from + kListed, last); at += 256) {
      const int64_t row = at + threadIdx.x;
      const bool mine = row < last && p.at.index[row] == a;
      const uint64_t who = __ballot(mine);
      if (lane == 0) counts[wave] = __popcll(who);
      __syncthreads();
      int before = n + __popcll(who & (((uint64_t)1 << lane) - 1));
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if (w < wave) before += counts[w];
        n += counts[w];
      }
      if (mine) list[before] = (int32_t)(row - first);
      __syncthreads();
    }
    if (n == 0) continue;
    if (threadIdx.x < 32) list[n + threadIdx.x] = list[n - 1];
    __syncthreads();
    if (j0 < p.len)
      for (int at = 0; at < n; at += 32) {
        Raw8<SRC> z[8];
        uint32_t v[RT][8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int64_t row = first + list[at + 8 * g + q];
          get8<SRC, WIDE>(z[q], line_of<SRC>(p.z, row), j, p.len);
#pragma unroll
          for (int t = 0; t < RT; ++t)
            v[t][q] = __builtin_bit_cast(uint32_t, p.v[row * p.v_ld + min(r0 + 16 * t + l, rank - 1)]);
        }
        if (at + 32 > n)  // (past the list's end is its last row again)
#pragma unroll
          for (int q = 0; q < 8; ++q) keep8<SRC>(z[q], at + 8 * g + q < n);
        if (j0 + 128 > p.len)
#pragma unroll
          for (int q = 0; q < 8; ++q) placed8<SRC, WIDE>(z[q], j, p.len);
        v4u vp[RT][3];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          Raw8<SRC_F32> raw;
#pragma unroll
          for (int q = 0; q < 8; ++q) raw.w[q] = at + 8 * g + q < n ? v[t][q] : 0u;
          raw_parts<SRC_F32>(raw, vp[t]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v4u zp[P];
          column_parts<SRC>(z, e, zp);
#pragma unroll
          for (int t = 0; t < RT; ++t) acc[t][e] = mfma_parts<P, 3>(zp, vp[t], acc[t][e]);
        }
      }
    __syncthreads();  // (the list is read)
  }
  if (j0 >= p.len) return;
  const float scale = scale_of(p.at, a);
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int r = r0 + 16 * t + l;
    if (r >= p.at.rank) continue;
    const int64_t row = (int64_t)a * p.at.rank + r;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t c = j0 + 8 * (4 * g + q);
      if (c >= p.len) continue;
      float out[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) out[e] = r < rank ? scale * acc[t][e][q] : 0.0f;
      put8<SRC_F32>(p.parts + ((int64_t)blockIdx.z * p.at.count * p.at.rank + row) * p.len, c, p.len, out);
    }
  }
}

// The parts in a fixed order, with what g holds.
template <int GSRC>
__global__ __launch_bounds__(256) void adapter_grad_join(AdapterGradArgs p, int64_t splits) {
  const int64_t rows = (int64_t)p.at.count * p.at.rank, upr = (p.len + 7) / 8;
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < rows * upr; u += (int64_t)gridDim.x * 256) {
    const int64_t row = u / upr, c = (u - row * upr) * 8;
    const bool all = c + 8 <= p.len;
    float v[8] = {};
    for (int64_t s = 0; s < splits; ++s) {
      const float* part = p.parts + (s * rows + row) * p.len + c;
      float w[8] = {};
      if (all) __builtin_memcpy(w, part, sizeof w);
      else
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i < p.len) w[i] = part[i];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += w[i];
    }
    if (p.beta != 0.0f) {
      const Elem<GSRC>* old = static_cast<const Elem<GSRC>*>(p.g.data) + row * p.g.ld + c;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < p.len) v[i] += p.beta * (float)old[i];
    }
    put8<GSRC>(line_to<GSRC>(p.g, row), c, p.len, v);
  }
}

// ---- launches ----------------------------------------------------------------------
// Workgroups of a launch, along x and along y: together, and with the parts of a gradient, below
// 2^32 lanes.
constexpr int64_t kRowGrid = 1 << 9, kColGrid = 1 << 12;

// Calls f<SRC, WIDE>
template <typename F>
hipError_t by_type(costa_real type, bool wide, F f) {
  auto go = [&](auto src) {
    if (wide) f(src, std::true_type{});
    else f(src, std::false_type{});
  };
  if (type == COSTA_REAL_BF16) go(std::integral_constant<int, SRC_BF16>{});
  else if (type == COSTA_REAL_F16) go(std::integral_constant<int, SRC_F16>{});
  else go(std::integral_constant<int, SRC_F32>{});
  return hipGetLastError();
}

constexpr int64_t kFewRows = 64;

// Ranks of a workgroup of the gradients' kernel, in sixteens, and workgroups along the columns.
struct GradPlan {
  int rt;
  int64_t across, pairs;
};
GradPlan plan_grad(int64_t len, int32_t count, int32_t rank) {
  const int rt = rank <= 16 ? 1 : rank <= 32 ? 2 : 4;
  return {rt, up_div(len, 512), (int64_t)count * up_div(rank, 16 * rt)};
}

}  // namespace

hipError_t launch_mx_adapter_dots(const AdapterDotsArgs& a, hipStream_t stream) {
  const bool few = a.m <= kFewRows;
  const int64_t groups = few ? a.m : up_div(a.m, 16);
  const int rt = a.at.rank <= 16 ? 1 : a.at.rank <= 32 ? 2 : 4;
  constexpr int64_t kDotGrid = 1 << 16;
  for (int64_t at = 0; at < groups; at += kDotGrid) {
    const unsigned x = (unsigned)std::min(kDotGrid, groups - at);
    const hipError_t e = by_type(a.type, a.k >= 8, [&](auto src, auto wide) {
      constexpr int SRC = decltype(src)::value;
      constexpr bool WIDE = decltype(wide)::value;
      const dim3 tiles(x, (unsigned)up_div(a.at.rank, 16 * rt));
      if (few) adapter_dots_row<SRC, WIDE><<<dim3(x, (unsigned)up_div(a.at.rank, kDotRanks)), 256, 0, stream>>>(a, at);
      else if (rt == 1) adapter_dots_tile<SRC, 1, WIDE><<<tiles, 64 * kDotWaves, 0, stream>>>(a, at * 16);
      else if (rt == 2) adapter_dots_tile<SRC, 2, WIDE><<<tiles, 64 * kDotWaves, 0, stream>>>(a, at * 16);
      else adapter_dots_tile<SRC, 4, WIDE><<<tiles, 64 * kDotWaves, 0, stream>>>(a, at * 16);
    });
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_mx_adapter_add(const AdapterAddArgs& a, hipStream_t stream) {
  const bool few = a.m <= kFewRows;
  const int64_t rows = few ? 1 : 128, cols = few ? 2048 : 128, down = up_div(a.m, rows), across = up_div(a.n, cols);
  for (int64_t j = 0; j < across; j += kColGrid)
    for (int64_t i = 0; i < down; i += kRowGrid) {
      const dim3 grid((unsigned)std::min(kRowGrid, down - i), (unsigned)std::min(kColGrid, across - j));
      const hipError_t e = by_type(a.type, a.n >= 8, [&](auto src, auto wide) {
        constexpr int SRC = decltype(src)::value;
        constexpr bool WIDE = decltype(wide)::value;
        if (few) adapter_add_row<SRC, WIDE><<<grid, 256, 0, stream>>>(a, i * rows, j * cols);
        else adapter_add_tile<SRC, 2, WIDE><<<grid, 256, 0, stream>>>(a, i * rows, j * cols);
      });
      if (e != hipSuccess) return e;
    }
  return hipSuccess;
}

// (so that the workgroups are two for each CU, with 128 rows of each at least)
int64_t mx_adapter_grad_parts(int64_t m, int64_t len, int32_t count, int32_t rank) {
  const GradPlan g = plan_grad(len, count, rank);
  return std::max<int64_t>(std::min(2 * kCUs / std::max<int64_t>(g.across * g.pairs, 1), m / 128), 1);
}

hipError_t launch_mx_adapter_grad(const AdapterGradArgs& a, hipStream_t stream) {
  const GradPlan g = plan_grad(a.len, a.at.count, a.at.rank);
  const int64_t splits = std::min(mx_adapter_grad_parts(a.m, a.len, a.at.count, a.at.rank), a.most);
  const int64_t per = up_div(a.m, splits);
  for (int64_t j = 0; j < g.across; j += kRowGrid)
    for (int64_t i = 0; i < g.pairs; i += kColGrid) {
      const dim3 grid((unsigned)std::min(kRowGrid, g.across - j), (unsigned)std::min(kColGrid, g.pairs - i),
                      (unsigned)splits);
      const hipError_t e = by_type(a.type, a.len >= 8, [&](auto src, auto wide) {
        constexpr int SRC = decltype(src)::value;
        constexpr bool WIDE = decltype(wide)::value;
        if (g.rt == 1) adapter_grad_tile<SRC, 1, WIDE><<<grid, 256, 0, stream>>>(a, j * 512, i, per);
        else if (g.rt == 2) adapter_grad_tile<SRC, 2, WIDE><<<grid, 256, 0, stream>>>(a, j * 512, i, per);
        else adapter_grad_tile<SRC, 4, WIDE><<<grid, 256, 0, stream>>>(a, j * 512, i, per);
      });
      if (e != hipSuccess) return e;
    }
  const int64_t units = (int64_t)a.at.count * a.at.rank * up_div(a.len, 8);
  const dim3 grid((unsigned)std::min<int64_t>(up_div(units, 256), 1 << 20));
  if (a.g_type == COSTA_REAL_F32) adapter_grad_join<SRC_F32><<<grid, 256, 0, stream>>>(a, splits);
  else if (a.g_type == COSTA_REAL_BF16) adapter_grad_join<SRC_BF16><<<grid, 256, 0, stream>>>(a, splits);
  else adapter_grad_join<SRC_F16><<<grid, 256, 0, stream>>>(a, splits);
  return hipGetLastError();
}

}  // namespace costa
