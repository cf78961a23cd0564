// Products of some tens of rows, whose sums go on in parts: tiles of 64 rows and 128 columns.
//
// Between the kernel for few rows, whose every workgroup converts all of the rows for 16 or 32 columns, and the
// larger tiles, which would be half empty.  The time is that of reading B and, in the caches, of reading the rows
// once for every 128 columns, so k goes by 128 (rows of B are padded to as much): neighbouring lanes read 64 or
// 128 bytes of a row of B and 256 of a row of bfloat16.  Two stages in shared memory, one
// barrier a step, two steps' loads on their way in registers; eight waves of 32 rows and 32 columns.  B's
// elements are decoded on the way to the matrix instruction: lane l has, of row l % 16, the block of 32
// elements l / 16 of the step, for four instructions.
// (61 rows by 8192x8192 in 4 bits, joined, against steps of 64 with eight waves of 64 rows and 16 columns: bfloat16
// 25 us and 32, float16 31 and 36, float 39 and 45; by 20000 columns of 4096 30 and 38, 43 and 42, 53 and 52.)
#include "mx_tiles.hpp"

namespace costa {
namespace {

constexpr int kStepFew = 128, kFewRowsMax = 64, kFewCols = 128;
constexpr int kChunksA = kStepFew / 8;  // 16-byte chunks of a row's parts
__device__ inline int few_chunk(int row, int chunk) { return row * kChunksA + (chunk ^ (row & 15)); }

template <int SRC, int BBITS>
struct FewStage {
  static constexpr int P = parts_of(SRC), CHUNKS = kStepFew * BBITS / 128;  // of a row of B
  static constexpr int PASSES = kFewCols * CHUNKS / kLanes;
  Raw8<SRC> a[2];
  v4u b[PASSES];
  uint32_t scale;
  static __device__ inline int place(int row, int chunk) {  // (8 bits: neighbouring rows meet different banks)
    return row * CHUNKS + (BBITS == 8 ? chunk ^ (row & 7) : chunk);
  }
  __device__ inline void load(const Args& p, int64_t j0, int64_t k0) {
    const int t = threadIdx.x;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int64_t i = min((int64_t)(t / kChunksA + 32 * q), p.m - 1);
      load8<SRC>(a[q], static_cast<const char*>(p.real) + i * p.a_rs * bytes_of(SRC), k0 + t % kChunksA * 8, p.k);
    }
#pragma unroll
    for (int q = 0; q < PASSES; ++q) {
      const int at = t + q * kLanes;
      const int64_t j = min(j0 + at / CHUNKS, p.n - 1);
      b[q] = *reinterpret_cast<const v4u*>(p.b.data + j * p.b.row_bytes + k0 * BBITS / 8 + at % CHUNKS * 16);
    }
    const int64_t j = min(j0 + t % kFewCols, p.n - 1);
    scale = *reinterpret_cast<const uint32_t*>(p.b.scales + j * p.b.row_scales + k0 / kMxBlock);
  }
  __device__ inline void store(const Args& p, int64_t k0, v4u* left, v4u* right, uint32_t* scales) {
    const int t = threadIdx.x;
    if (k0 + kStepFew > p.k)
#pragma unroll
      for (int q = 0; q < 2; ++q) place8<SRC>(a[q], k0 + t % kChunksA * 8, p.k);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      v4u out[P];
      raw_parts<SRC>(a[q], out);
#pragma unroll
      for (int x = 0; x < P; ++x) left[x * kFewRowsMax * kChunksA + few_chunk(t / kChunksA + 32 * q, t % kChunksA)] = out[x];
    }
#pragma unroll
    for (int q = 0; q < PASSES; ++q) {
      const int at = t + q * kLanes;
      right[place(at / CHUNKS, at % CHUNKS)] = b[q];
    }
    if (t < kFewCols) scales[t] = scale;
  }
};

template <int SRC, int BBITS>
__global__ __launch_bounds__(kLanes) void tiles_few(Args p) {
  typedef FewStage<SRC, BBITS> Stage;
  constexpr int P = Stage::P;
  __shared__ v4u left[2][P * kFewRowsMax * kChunksA];
  __shared__ v4u right[2][kFewCols * Stage::CHUNKS];
  __shared__ uint32_t scales[2][kFewCols];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16, g = lane / 16;
  const int wm = wave / 4 * 32, wn = wave % 4 * 32;
  const int64_t j0 = (int64_t)blockIdx.x * kFewCols;
  int64_t first, last;
  steps_of((uint32_t)((p.k + kStepFew - 1) / kStepFew), blockIdx.y, gridDim.y, first, last);
  v4f acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = v4f{0, 0, 0, 0};
  Stage st[2];
  auto load = [&](int set, int64_t t) {
    if (t < last) st[set].load(p, j0, t * kStepFew);
  };
  load(0, first);
  load(1, first + 1);
  st[0].store(p, first * kStepFew, left[0], right[0], scales[0]);
  load(0, first + 2);
  __syncthreads();
  for (int64_t t0 = first; t0 < last; t0 += 2) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int64_t t = t0 + s;
      if (t >= last) break;
      v4u b[2][BBITS == 4 ? 1 : 2];
      uint32_t sc[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int row = wn + 16 * j + r;
        if (BBITS == 4) {
          b[j][0] = right[s][Stage::place(row, g)];
        } else {
          b[j][0] = right[s][Stage::place(row, 2 * g)];
          b[j][1 % (BBITS / 4)] = right[s][Stage::place(row, 2 * g + 1)];
        }
        sc[j] = reinterpret_cast<const uint8_t*>(scales[s])[row * 4 + g];
      }
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        v4u w[2];
#pragma unroll
        for (int j = 0; j < 2; ++j)
          w[j] = mx_decode8_bf16<BBITS>(BBITS == 4 ? v2u{b[j][0][h], 0u}
                                                   : v2u{b[j][h / 2 % (BBITS / 4)][2 * h % 4], b[j][h / 2 % (BBITS / 4)][(2 * h + 1) % 4]},
                                        sc[j]);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int x = 0; x < P; ++x) {
            const v4u a = left[s][x * kFewRowsMax * kChunksA + few_chunk(wm + 16 * i + r, 4 * g + h)];
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = mfma_bf16(w[j], a, acc[i][j]);
          }
      }
      if (t + 1 < last) {
        st[1 - s].store(p, (t + 1) * kStepFew, left[1 - s], right[1 - s], scales[1 - s]);
        load(1 - s, t + 3);
      }
      __syncthreads();
    }
  }
  put_wave<2, 2>(p, acc, &left[0][0], wave, wm, j0 + wn);
}

template <int SRC>
hipError_t launch(const Args& p, int splits, hipStream_t stream) {
  const dim3 grid((unsigned)up_div(p.n, kFewCols), splits);
  if (p.b.bits == 4) tiles_few<SRC, 4><<<grid, kLanes, 0, stream>>>(p);
  else tiles_few<SRC, 8><<<grid, kLanes, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tiles_few(int src, const Args& p, int splits, hipStream_t stream) {
  if (p.m > kFewRowsMax || p.k < 8) return hipErrorInvalidValue;  // not a product of this kernel
  if (src == SRC_BF16) return launch<SRC_BF16>(p, splits, stream);
  if (src == SRC_F16) return launch<SRC_F16>(p, splits, stream);
  return launch<SRC_F32>(p, splits, stream);
}

}  // namespace costa
