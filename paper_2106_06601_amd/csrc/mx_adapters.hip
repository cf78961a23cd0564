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

#include "mx_adapters.hpp"
#include "mx_tiles.hpp"

namespace costa {
namespace {

// ---- few rows: a row at a time, on the vector units ----------------------------
// A workgroup makes four of a row's products; its lanes go along the row.  The time is that
// of reading the adapters' rows, all of them on their way at once: 61 rows of 32 adapters of rank 16 over 8192
// in bfloat16 5.3 us (16.8 MB would take 3.3 at the rate of a copy).
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

// v, with what c holds there, to c's elements c .. c + 7 of a row.
template <int CSRC>
__device__ inline void put_scaled(const AdapterAddArgs& p, int64_t row, int64_t c, float v[8]) {
  if (p.beta != 0.0f) {
    const Elem<CSRC>* old = static_cast<const Elem<CSRC>*>(p.c.data) + row * p.c.ld + c;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < p.n) v[i] += p.beta * (float)old[i];
  }
  put8<CSRC>(line_to<CSRC>(p.c, row), c, p.n, v);
}

constexpr int kAddRanks = 8;  // rows of an adapter that are on their way at once
// A workgroup has 2048 columns of a row, eight a lane: the product's parts, what the adapter
// adds, c.  (Of the adapter all rows are read, those past its rank for nothing: how many there are
// is known later than where they are.)  61 rows of 32 adapters of rank 16, 8192 columns, four parts: 6.5 us; 333 rows
// of float16, rank 24, 1999 columns 11.4 us (with the parts after the ranks, one after another, 15.5).
template <int SRC, bool WIDE>
__global__ __launch_bounds__(256) void adapter_add_row(AdapterAddArgs p, int64_t row0, int64_t col0) {
  const int64_t row = row0 + blockIdx.x, c = col0 + ((int64_t)blockIdx.y * 256 + threadIdx.x) * 8;
  const bool all = c + 8 <= p.n;
  const int32_t a = adapter_of(p.at, row);
  float v[8] = {};
  const float* part = p.parts + row * p.n + c;
#pragma unroll 4
  for (int s = 0; s < p.splits; ++s, part += p.m * p.n) {
    float w[8] = {};
    if (all) __builtin_memcpy(w, part, sizeof w);
    else
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < p.n) w[i] = part[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += w[i];
  }
  if (p.splits > 0)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= p.alpha;
  if (a >= 0) {
    const int rank = rank_of(p.at, a);
    const float s = scale_of(p.at, a);
    const float* const x = p.v + row * p.v_ld;
    const void* const low = line_of<SRC>(p.low, (int64_t)a * p.at.rank);
    float add[8] = {};
    for (int r0 = 0; r0 < p.at.rank; r0 += kAddRanks) {
      Raw8<SRC> raw[kAddRanks];
      float xr[kAddRanks];
#pragma unroll
      for (int j = 0; j < kAddRanks; ++j) {
        const int r = min(r0 + j, p.at.rank - 1);
        get8<SRC, WIDE>(raw[j], static_cast<const char*>(low) + r * p.low.ld * bytes_of(SRC), c, p.n);
        xr[j] = x[r];
      }
#pragma unroll
      for (int j = 0; j < kAddRanks; ++j) {
        if (r0 + j >= rank) break;
        float b[8];
        floats8<SRC, WIDE>(raw[j], c, p.n, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) add[i] = fmaf(xr[j], b[i], add[i]);
      }
    }
    if (rank > 0)  // (a sum over nothing is 0, whatever s)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += s * add[i];
  }
  if (c >= p.n) return;
  if (p.c_type == COSTA_REAL_F32) put_scaled<SRC_F32>(p, row, c, v);
  else if (p.c_type == COSTA_REAL_BF16) put_scaled<SRC_BF16>(p, row, c, v);
  else put_scaled<SRC_F16>(p, row, c, v);
}

// ---- many rows, on the matrix units ---------------------------------------------
// A workgroup has BM rows and RN ranks of a part of the sum, which goes by 64: both operands' steps
// go through shared memory (read straight to registers in the instruction's order, sixteen
// neighbouring lanes touch sixteen lines: 4096 rows by 64 ranks over 8192 took 73 us so), two of them
// on their way while one is worked on.  That takes 36 us, of rank 16 20 us, against 13 for reading x: 63% of the
// waves' time is waiting, for the steps that follow one another.  128 rows a workgroup (38 us), four steps ahead (34 to
// 36; of rank 16 32) and steps in another order for every workgroup (36) brought nothing.  Eight waves of sixteen rows by 16 NT ranks.
constexpr int kDotAhead = 2;
template <int SRC, int BM, int RN>
__global__ __launch_bounds__(kLanes, parts_of(SRC) == 1 ? 4 : 2) void adapter_dots_tile(AdapterDotsArgs p, int64_t row0, int64_t per) {
  constexpr int P = parts_of(SRC), STRIPS = BM / 16, NT = RN / 16 / (kWaves / STRIPS), HALVES = BM / 64;
  __shared__ v4u xs[2][P * BM * 8];
  __shared__ v4u as[2][P * RN * 8];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = lane % 16,
            g = lane / 16;
  const int64_t i0 = row0 + (int64_t)blockIdx.x * BM;
  const int r0 = blockIdx.y * RN, strip = wave % STRIPS * 16, rn = wave / STRIPS * 16 * NT;
  const int64_t first = blockIdx.z * per, last = min(first + per, (p.k + kStepBf16 - 1) / kStepBf16);  // steps
  const int32_t mine = i0 + strip + l < p.m ? adapter_of(p.at, i0 + strip + l) : -1;
  int32_t idx[HALVES];  // of the tile's rows, the same in every wave
  uint64_t left[HALVES], any = 0;
#pragma unroll
  for (int h = 0; h < HALVES; ++h) {
    idx[h] = i0 + 64 * h + lane < p.m ? adapter_of(p.at, i0 + 64 * h + lane) : -1;
    left[h] = __ballot(idx[h] >= 0);
    any |= left[h];
  }
  const Args x{p.m, 0, p.k, MxView{}, MxView{}, p.x.data, p.x.ld, 1, Epilogue{}, 0};
  v4f all[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) all[t] = v4f{0, 0, 0, 0};
  while (any) {
    int32_t a = -1;
#pragma unroll
    for (int h = HALVES - 1; h >= 0; --h)
      if (left[h]) a = __builtin_amdgcn_readlane(idx[h], (int)__builtin_ctzll(left[h]));
    any = 0;
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
      left[h] &= ~__ballot(idx[h] == a);
      any |= left[h];
    }
    const int rank = rank_of(p.at, a);
    if (r0 >= rank || first >= last) continue;
    // (past the last rank: that again, and its products are not taken)
    const char* const low = static_cast<const char*>(line_of<SRC>(p.low, (int64_t)a * p.at.rank + min(r0 + (int)threadIdx.x / 8, rank - 1)));
    v4f acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = v4f{0, 0, 0, 0};
    LeftStage<SRC, false, BM, false> xl[kDotAhead];
    Raw8<SRC> al[kDotAhead];
    const int c = threadIdx.x % 8, ar = threadIdx.x / 8;
    auto load = [&](int set, int64_t t) {
      if (t >= last) return;
      const int64_t k0 = t * kStepBf16;
      xl[set].load(x, i0, k0);
      if (ar < RN) load8<SRC>(al[set], low, k0 + 8 * c, p.k);
    };
    auto store = [&](int set, int64_t t, int s) {
      xl[set].store(x, i0, xs[s]);
      if (ar < RN) {
        const int64_t k0 = t * kStepBf16;
        if (k0 + kStepBf16 > p.k) place8<SRC>(al[set], k0 + 8 * c, p.k);
        v4u out[P];
        raw_parts<SRC>(al[set], out);
#pragma unroll
        for (int q = 0; q < P; ++q) as[s][q * RN * 8 + chunk_at(ar, c)] = out[q];
      }
    };
#pragma unroll
    for (int s = 0; s < kDotAhead; ++s) load(s, first + s);
    __syncthreads();  // (the adapter's before: its last step is read)
    store(0, first, 0);
    load(0, first + kDotAhead);
    __syncthreads();
    for (int64_t t0 = first; t0 < last; t0 += kDotAhead) {
#pragma unroll
      for (int s = 0; s < kDotAhead; ++s) {
        const int64_t t = t0 + s;
        if (t >= last) break;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          v4u xp[P];
#pragma unroll
          for (int q = 0; q < P; ++q) xp[q] = xs[s % 2][q * BM * 8 + chunk_at(strip + l, 2 * g + h)];
#pragma unroll
          for (int u = 0; u < NT; ++u) {
            v4u ap[P];
#pragma unroll
            for (int q = 0; q < P; ++q) ap[q] = as[s % 2][q * RN * 8 + chunk_at(rn + 16 * u + l, 2 * g + h)];
            acc[u] = mfma_parts<P, P>(ap, xp, acc[u]);
          }
        }
        if (t + 1 < last) {
          store((s + 1) % kDotAhead, t + 1, (s + 1) % 2);
          load((s + 1) % kDotAhead, t + 1 + kDotAhead);
        }
        __syncthreads();
      }
    }
    // lane: row l of the strip, ranks r0 + rn + 16 u + 4 g .. + 3
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (mine == a && r0 + rn + 16 * u + 4 * g + q < rank) all[u][q] = acc[u][q];
  }
  const int64_t row = i0 + strip + l;
  if (row >= p.m) return;
  float* const v = p.parts ? p.parts + ((int64_t)blockIdx.z * p.m + row) * p.at.rank : p.v + row * p.v_ld;
#pragma unroll
  for (int u = 0; u < NT; ++u)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int r = r0 + rn + 16 * u + 4 * g + q;
      if (r < p.at.rank) v[r] = all[u][q];
    }
}

// The parts of v, in a fixed order.
__global__ __launch_bounds__(256) void adapter_dots_join(AdapterDotsArgs p, int64_t splits) {
  const int64_t all = p.m * p.at.rank;
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < all; u += (int64_t)gridDim.x * 256) {
    float sum = 0.0f;
#pragma unroll 4
    for (int64_t s = 0; s < splits; ++s) sum += p.parts[s * all + u];
    p.v[u / p.at.rank * p.v_ld + u % p.at.rank] = sum;
  }
}

// v from its parts (or as it is) to v and, spread, to the operands that the products' tiles add.
__global__ __launch_bounds__(256) void adapter_spread(AdapterDotsArgs p, int64_t splits, v4u* spread) {
  const int64_t steps = (p.at.rank + 31) / 32, units = (p.m + 15) / 16 * steps * 64, all = p.m * p.at.rank;
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < units; u += (int64_t)gridDim.x * 256) {
    const int lane = (int)(u % 64);
    const int64_t unit = u / 64, tile = unit / steps, row = tile * 16 + lane % 16;
    const int r0 = (int)(unit - tile * steps) * 32 + lane / 16 * 8;
    Raw8<SRC_F32> raw;
    const int32_t a = row < p.m ? adapter_of(p.at, row) : -1;
    const float scale = a < 0 ? 0.0f : scale_of(p.at, a);
    float x[8] = {};
    if (row < p.m && r0 + 8 <= p.at.rank) {
      const float* at = splits > 0 ? p.parts + row * p.at.rank + r0 : p.v + row * p.v_ld + r0;
#pragma unroll 4
      for (int64_t s = 0; s < max(splits, (int64_t)1); ++s) {
        float w[8];
        __builtin_memcpy(w, at + s * all, sizeof w);
#pragma unroll
        for (int q = 0; q < 8; ++q) x[q] += w[q];
      }
      if (splits > 0) __builtin_memcpy(p.v + row * p.v_ld + r0, x, sizeof x);
    } else if (row < p.m) {
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        if (r0 + q >= p.at.rank) continue;
        if (splits > 0) {
          for (int64_t s = 0; s < splits; ++s) x[q] += p.parts[s * all + row * p.at.rank + r0 + q];
          p.v[row * p.v_ld + r0 + q] = x[q];
        } else {
          x[q] = p.v[row * p.v_ld + r0 + q];
        }
      }
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) raw.w[q] = a < 0 ? 0u : __builtin_bit_cast(uint32_t, scale * x[q]);
    v4u out[3];
    raw_parts<SRC_F32>(raw, out);
#pragma unroll
    for (int x = 0; x < 3; ++x) spread[(unit * 3 + x) * 64 + lane] = out[x];
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

// ---- gradients --------------------------------------------------------------------
// v, with what g holds there, to g's elements c .. c + 7 of a row.
template <int GSRC>
__device__ inline void put_grad(const AdapterGradArgs& p, int64_t row, int64_t c, float v[8]) {
  if (p.beta != 0.0f) {
    const Elem<GSRC>* old = static_cast<const Elem<GSRC>*>(p.g.data) + row * p.g.ld + c;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < p.len) v[i] += p.beta * (float)old[i];
  }
  put8<GSRC>(line_to<GSRC>(p.g, row), c, p.len, v);
}
__device__ inline void put_grad_typed(const AdapterGradArgs& p, int64_t row, int64_t c, float v[8]) {
  if (p.g_type == COSTA_REAL_F32) put_grad<SRC_F32>(p, row, c, v);
  else if (p.g_type == COSTA_REAL_BF16) put_grad<SRC_BF16>(p, row, c, v);
  else put_grad<SRC_F16>(p, row, c, v);
}

// A workgroup has 128 columns of 16 RT ranks of an adapter, and a part of the rows, of which those
// of the adapter are listed in shared memory, 2048 rows at a time.  Its four waves take 32 of them by
// turns, straight to registers (the next ones are on their way while some are worked on), and
// their sums are joined through shared memory.  8192 rows of two adapters of rank 32, 4096 columns of
// bfloat16: 22 us, 3.1 TB/s of z, and 5 joining 8 parts (with the waves beside one another along the columns
// 34 and 13, for 32 parts).
constexpr int kListed = 2048;
template <int SRC, int RT, bool WIDE>
__global__ __launch_bounds__(256) void adapter_grad_tile(AdapterGradArgs p, int64_t col0, int64_t pair0,
                                                         int64_t per) {
  constexpr int P = parts_of(SRC);
  __shared__ union {
    struct {
      int32_t list[kListed + 128];
      int32_t counts[4];
    } rows;
    v4f sums[2][RT * 8][64];
  } shared;
  int32_t* const list = shared.rows.list;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = lane % 16,
            g = lane / 16;
  const int chunks = (p.at.rank + 16 * RT - 1) / (16 * RT);
  const int32_t pair = (int32_t)(pair0 + blockIdx.y), a = pair / chunks;
  const int r0 = pair % chunks * 16 * RT, rank = rank_of(p.at, a);
  const int64_t j0 = col0 + (int64_t)blockIdx.x * 128, j = j0 + 8 * l;
  const int64_t first = (int64_t)blockIdx.z * per, last = min(first + per, p.m);
  v4f acc[RT][8];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[t][e] = v4f{0, 0, 0, 0};
  bool some = false;  // rows of the adapter
  for (int64_t from = first; r0 < rank && from < last; from += kListed) {
    int n = 0;
    for (int64_t at = from; at < min(from + kListed, last); at += 256) {
      const int64_t row = at + threadIdx.x;
      const bool mine = row < last && p.at.index[row] == a;
      const uint64_t who = __ballot(mine);
      if (lane == 0) shared.rows.counts[wave] = __popcll(who);
      __syncthreads();
      int before = n + __popcll(who & (((uint64_t)1 << lane) - 1));
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if (w < wave) before += shared.rows.counts[w];
        n += shared.rows.counts[w];
      }
      if (mine) list[before] = (int32_t)(row - first);
      __syncthreads();
    }
    if (n == 0) continue;
    some = true;
    if (threadIdx.x < 128) list[n + threadIdx.x] = list[n - 1];
    __syncthreads();
    Raw8<SRC> z[8];
    uint32_t v[RT][8];
    auto load = [&](int at) {
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int64_t row = first + list[min(at, n) + 8 * g + q];
        get8<SRC, WIDE>(z[q], line_of<SRC>(p.z, row), j, p.len);
#pragma unroll
        for (int t = 0; t < RT; ++t)
          v[t][q] = __builtin_bit_cast(uint32_t, p.v[row * p.v_ld + min(r0 + 16 * t + l, rank - 1)]);
      }
    };
    load(wave * 32);
    for (int at = wave * 32; at < n; at += 128) {
      Raw8<SRC> zs[8];
      v4u vp[RT][3];
#pragma unroll
      for (int q = 0; q < 8; ++q) zs[q] = z[q];
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        Raw8<SRC_F32> raw;
#pragma unroll
        for (int q = 0; q < 8; ++q) raw.w[q] = at + 8 * g + q < n ? v[t][q] : 0u;
        raw_parts<SRC_F32>(raw, vp[t]);
      }
      load(at + 128);
      if (at + 32 > n)  // (past the list's end is its last row again)
#pragma unroll
        for (int q = 0; q < 8; ++q) keep8<SRC>(zs[q], at + 8 * g + q < n);
      if (j0 + 128 > p.len)
#pragma unroll
        for (int q = 0; q < 8; ++q) placed8<SRC, WIDE>(zs[q], j, p.len);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v4u zp[P];
        column_parts<SRC>(zs, e, zp);
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[t][e] = mfma_parts<P, 3>(zp, vp[t], acc[t][e]);
      }
    }
    __syncthreads();  // (the list is read)
  }
#pragma unroll
  for (int half = 2; half > 0; half /= 2) {
    if (wave >= half && wave < 2 * half)
#pragma unroll
      for (int t = 0; t < RT * 8; ++t) shared.sums[wave - half][t][lane] = acc[t / 8][t % 8];
    __syncthreads();
    if (wave < half)
#pragma unroll
      for (int t = 0; t < RT * 8; ++t) acc[t / 8][t % 8] += shared.sums[wave][t][lane];
    __syncthreads();
  }
  if (wave != 0) return;
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
      for (int e = 0; e < 8; ++e) out[e] = some && r < rank ? scale * acc[t][e][q] : 0.0f;  // (0, whatever the scale)
      if (p.parts) put8<SRC_F32>(p.parts + ((int64_t)blockIdx.z * p.at.count * p.at.rank + row) * p.len, c, p.len, out);
      else put_grad_typed(p, row, c, out);
    }
  }
}

// The parts in a fixed order, with what g holds.
__global__ __launch_bounds__(256) void adapter_grad_join(AdapterGradArgs p, int64_t splits) {
  const int64_t rows = (int64_t)p.at.count * p.at.rank, upr = (p.len + 7) / 8;
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < rows * upr; u += (int64_t)gridDim.x * 256) {
    const int64_t row = u / upr, c = (u - row * upr) * 8;
    const bool all = c + 8 <= p.len;
    float v[8] = {};
#pragma unroll 4
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
    put_grad_typed(p, row, c, v);
  }
}

// ---- launches ----------------------------------------------------------------------
// Workgroups of a launch, along x and along y: together, and with the parts of a gradient, below
// 2^32 lanes.
constexpr int64_t kRowGrid = 1 << 12, kColGrid = 1 << 9;

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

// Whether products are made row by row, each reading its adapter's rows out of the cache, where the
// tiles' kernel reads them once for its rows that share them: 300 rows of 32 to 64 adapters of 16
// ranks over 8192 cost 20 us by rows and 209 in tiles, 4096 rows in runs of 8 adapters 65 us by rows and
// 22 in tiles.  (Whether rows share is in device memory: many rows of many adapters mixed go in tiles all the
// same, 4096 of 64 adapters 800 us.)
constexpr int64_t kByRowsBytes = (int64_t)256 << 20;
bool dots_by_rows(int64_t m, int rank, int64_t k, costa_real type) {
  return m <= 64 || k < 8 || m * rank * k * (type == COSTA_REAL_F32 ? 4 : 2) <= kByRowsBytes;
}
// Rows and ranks of a workgroup of the tiles' kernel.
void dots_tile(int rank, int& bm, int& rn) {
  rn = rank <= 16 ? 16 : rank <= 32 ? 32 : 64;
  bm = rn == 16 ? 128 : 64;
}

// Ranks of a workgroup of the gradients' kernel, in sixteens, and workgroups along the columns.
struct GradPlan {
  int rt;
  int64_t across, pairs;
};
GradPlan plan_grad(int64_t len, int32_t count, int32_t rank) {
  const int rt = rank <= 16 ? 1 : rank <= 32 ? 2 : 4;
  return {rt, up_div(len, 128), (int64_t)count * up_div(rank, 16 * rt)};
}

}  // namespace

// (so that the workgroups are two for each CU, with 512 elements of the sum at least)
int64_t mx_adapter_dots_parts(int64_t m, int64_t k, int rank) {
  int bm, rn;
  dots_tile(rank, bm, rn);
  const int64_t tiles = up_div(m, bm) * up_div(std::max(rank, 1), rn);
  return std::max<int64_t>(std::min(2 * kCUs / std::max<int64_t>(tiles, 1), k / 512), 1);
}

hipError_t launch_mx_adapter_dots(const AdapterDotsArgs& a, int64_t& left, hipStream_t stream) {
  left = 0;
  constexpr int64_t kGrid = 1 << 16;
  if (dots_by_rows(a.m, a.at.rank, a.k, a.type)) {
    for (int64_t at = 0; at < a.m; at += kGrid) {
      const dim3 grid((unsigned)std::min(kGrid, a.m - at), (unsigned)up_div(a.at.rank, kDotRanks));
      const hipError_t e = by_type(a.type, a.k >= 8, [&](auto src, auto wide) {
        adapter_dots_row<decltype(src)::value, decltype(wide)::value><<<grid, 256, 0, stream>>>(a, at);
      });
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
  AdapterDotsArgs b = a;
  const int64_t splits = std::min(mx_adapter_dots_parts(a.m, a.k, a.at.rank), std::max<int64_t>(a.most, 1));
  if (splits == 1) b.parts = nullptr;
  int bm, rn;
  dots_tile(a.at.rank, bm, rn);
  const int64_t steps = up_div(a.k, kStepBf16), per = up_div(steps, splits), tiles = up_div(a.m, bm);
  for (int64_t at = 0; at < tiles; at += kGrid) {
    const dim3 grid((unsigned)std::min(kGrid, tiles - at), (unsigned)up_div(a.at.rank, rn), (unsigned)splits);
    const hipError_t e = by_type(a.type, true, [&](auto src, auto wide) {
      constexpr int SRC = decltype(src)::value;
      if (!decltype(wide)::value) return;
      if (rn == 16) adapter_dots_tile<SRC, 128, 16><<<grid, kLanes, 0, stream>>>(b, at * bm, per);
      else if (rn == 32) adapter_dots_tile<SRC, 64, 32><<<grid, kLanes, 0, stream>>>(b, at * bm, per);
      else adapter_dots_tile<SRC, 64, 64><<<grid, kLanes, 0, stream>>>(b, at * bm, per);
    });
    if (e != hipSuccess) return e;
  }
  left = splits > 1 ? splits : 0;
  return hipSuccess;
}

hipError_t launch_mx_adapter_dots_join(const AdapterDotsArgs& a, int64_t splits, hipStream_t stream) {
  adapter_dots_join<<<dim3((unsigned)std::min<int64_t>(up_div(a.m * a.at.rank, 256), 1 << 20)), 256, 0, stream>>>(a, splits);
  return hipGetLastError();
}

hipError_t launch_mx_adapter_spread(const AdapterDotsArgs& a, int64_t splits, void* spread, hipStream_t stream) {
  const int64_t units = up_div(a.m, 16) * up_div(a.at.rank, 32) * 64;
  adapter_spread<<<dim3((unsigned)std::min<int64_t>(up_div(units, 256), 1 << 20)), 256, 0, stream>>>(
      a, splits, static_cast<v4u*>(spread));
  return hipGetLastError();
}

hipError_t launch_mx_adapter_add(const AdapterAddArgs& a, hipStream_t stream) {
  const int64_t across = up_div(a.n, 2048);
  for (int64_t j = 0; j < across; j += kColGrid)
    for (int64_t i = 0; i < a.m; i += kRowGrid) {
      const dim3 grid((unsigned)std::min(kRowGrid, a.m - i), (unsigned)std::min(kColGrid, across - j));
      const hipError_t e = by_type(a.type, a.n >= 8, [&](auto src, auto wide) {
        adapter_add_row<decltype(src)::value, decltype(wide)::value><<<grid, 256, 0, stream>>>(a, i, j * 2048);
      });
      if (e != hipSuccess) return e;
    }
  return hipSuccess;
}

// (so that the workgroups are two for each CU, with 512 rows of each at least)
int64_t mx_adapter_grad_parts(int64_t m, int64_t len, int32_t count, int32_t rank) {
  const GradPlan g = plan_grad(len, count, rank);
  return std::max<int64_t>(std::min(2 * kCUs / std::max<int64_t>(g.across * g.pairs, 1), m / 512), 1);
}

hipError_t launch_mx_adapter_grad(const AdapterGradArgs& a, hipStream_t stream) {
  const GradPlan g = plan_grad(a.len, a.at.count, a.at.rank);
  AdapterGradArgs b = a;
  const int64_t splits = std::max<int64_t>(std::min(mx_adapter_grad_parts(a.m, a.len, a.at.count, a.at.rank), a.most), 1);
  const int64_t per = up_div(a.m, splits);
  if (splits == 1) b.parts = nullptr;  // straight to g
  for (int64_t j = 0; j < g.across; j += kColGrid)
    for (int64_t i = 0; i < g.pairs; i += kRowGrid) {
      const dim3 grid((unsigned)std::min(kColGrid, g.across - j), (unsigned)std::min(kRowGrid, g.pairs - i),
                      (unsigned)splits);
      const hipError_t e = by_type(a.type, a.len >= 8, [&](auto src, auto wide) {
        constexpr int SRC = decltype(src)::value;
        constexpr bool WIDE = decltype(wide)::value;
        if (g.rt == 1) adapter_grad_tile<SRC, 1, WIDE><<<grid, 256, 0, stream>>>(b, j * 128, i, per);
        else if (g.rt == 2) adapter_grad_tile<SRC, 2, WIDE><<<grid, 256, 0, stream>>>(b, j * 128, i, per);
        else adapter_grad_tile<SRC, 4, WIDE><<<grid, 256, 0, stream>>>(b, j * 128, i, per);
      });
      if (e != hipSuccess) return e;
    }
  if (splits == 1) return hipSuccess;
  const int64_t units = (int64_t)a.at.count * a.at.rank * up_div(a.len, 8);
  adapter_grad_join<<<dim3((unsigned)std::min<int64_t>(up_div(units, 256), 1 << 20)), 256, 0, stream>>>(b, splits);
  return hipGetLastError();
}

}  // namespace costa
