// Products of microscaled matrices in tiles of C, with both operands staged in
// shared memory.
//
// Both kernels run 8 waves on a tile and keep two stages of k, one barrier a step:
// while the matrix instructions work on one stage, the next one's loads are on
// their way, to registers (and are then written to the other stage) or, where both
// operands are in 4 bits, straight to the other stage.  The operands
// of a matrix instruction are passed with B first: lane l then ends up with row
// l % 16 of C and four neighbouring columns, which makes wide stores.
#include <algorithm>

#include "mx_tiles.hpp"

namespace costa {
namespace {

template <int SRC, bool TRANS, int BBITS, int BM, int BN, int WM, int AHEAD, bool EDGE>
__global__ __launch_bounds__(kLanes) void tiles_bf16(Args p, uint32_t nm, uint32_t nn) {
  constexpr int MT = BM / WM / 16, NT = BN / (kWaves / WM) / 16;
  TileSums<MT, NT> t;
  tile_sums<SRC, TRANS, BBITS, BM, BN, WM, AHEAD, EDGE, 0>(p, nm, nn, t);
  put_wave<MT, NT>(p, t.acc, t.shared, t.wave, t.row, t.col);
}

// ---- both operands in 4 bits: the scaled instructions -----------------------------------
// An instruction sums 128 products, each block of 32 with its scales: exactly, then
// rounded into a 32-bit sum.  (The same instruction on 8-bit elements drops what is
// some 2^-13 of its largest product: 1.5e-5 of a product of normal matrices, more
// where a few columns stand out; those products take the bfloat16 kernel.)  k goes
// by 256, so that a step's row is 128 bytes.  Measured at 8192^3: 296 to 333 us, 3.3 to 3.7
// PFLOP/s (the library's 8-bit product reaches 2.7); the matrix units are busy 41% of the time at
// 2.0 GHz, and the waves wait a third of theirs, mostly for the next stage.  With the stage
// loaded to registers first the tile's registers did not suffice (1914 us).
constexpr int kStep4 = 256;
constexpr int kRowChunks = 8;  // 16-byte chunks of a step's row
__device__ inline int code_at(int row, int chunk) { return row * kRowChunks + (chunk ^ (row & 7)); }

// A stage of BR rows goes from memory to shared memory without registers: a lane
// names 16 bytes, the wave's 1024 bytes land next to one another.  The permutation
// of a row's chunks is in the lanes' addresses.  The compiler does not see these
// loads: wait_stage() waits for them.
template <int BR>
struct CodeStage {
  static constexpr int PASSES = BR * kRowChunks / kLanes;
  uint32_t offset[PASSES];  // of the lane's bytes from the tile's first row
  const uint8_t* base;
  __device__ inline CodeStage(const MxView& q, int64_t row0) : base(q.data + row0 * q.row_bytes) {
#pragma unroll
    for (int c = 0; c < PASSES; ++c) {
      const int at = threadIdx.x + c * kLanes, row = at / kRowChunks;
      const uint32_t there = (uint32_t)min((int64_t)row, q.rows - 1 - row0);
      offset[c] = there * (uint32_t)q.row_bytes + (at % kRowChunks ^ (row & 7)) * 16;
    }
  }
  __device__ inline void load(int64_t t, v4u* stage) const {
    const uint8_t* from = base + t * (kRowChunks * 16);
#pragma unroll
    for (int c = 0; c < PASSES; ++c) {
      const uint32_t to = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(
          __attribute__((address_space(3))) v4u*)(stage + c * kLanes + threadIdx.x / 64 * 64));
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                   :
                   : "s"(to), "v"(offset[c]), "s"(from)
                   : "m0", "memory");
    }
  }
};
__device__ inline void wait_stage() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ inline v8i operand4(v4u d) {  // the instruction reads four of the eight registers
  const v4i c = __builtin_bit_cast(v4i, d);
  return __builtin_shufflevector(c, c, 0, 1, 2, 3, -1, -1, -1, -1);
}

template <int BM, int BN, int WM>
__global__ __launch_bounds__(kLanes) void tiles_scaled(Args p, uint32_t nm, uint32_t nn) {
  constexpr int WN = kWaves / WM, MT = BM / WM / 16, NT = BN / WN / 16;
  __shared__ v4u left[2][BM * kRowChunks];
  __shared__ v4u right[2][BN * kRowChunks];
  __shared__ v2u scales[2][BM + BN];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16, g = lane / 16;
  const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
  int64_t tm, tn;
  tile_of(blockIdx.x, nm, nn, tm, tn);
  const int64_t i0 = tm * BM, j0 = tn * BN;
  int64_t first, last;
  steps_of((uint32_t)((p.k + kStep4 - 1) / kStep4), blockIdx.y, gridDim.y, first, last);

  v4f acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = v4f{0, 0, 0, 0};

  // a lane stages the scales of one row of either operand
  static_assert(BM + BN <= kLanes, "a lane a row");
  const bool mine = threadIdx.x < BM + BN, of_a = threadIdx.x < BM;
  const MxView& sv = of_a ? p.a : p.b;
  const int64_t srow = of_a ? min(i0 + threadIdx.x, p.m - 1) : min(j0 + threadIdx.x - BM, p.n - 1);
  const uint8_t* sp = sv.scales + srow * sv.row_scales;
  v2u sreg;
  const CodeStage<BM> as(p.a, i0);
  const CodeStage<BN> bs(p.b, j0);
  auto load = [&](int64_t t, int s) {
    if (mine) sreg = *reinterpret_cast<const v2u*>(sp + t * (kStep4 / kMxBlock));
    as.load(t, left[s]);
    bs.load(t, right[s]);
  };
  auto arrive = [&](int s) {
    wait_stage();
    if (mine) scales[s][threadIdx.x] = sreg;
    __syncthreads();
  };
  load(first, 0);
  arrive(0);
  for (int64_t t = first; t < last; ++t) {
    const int s = (int)(t - first) & 1;
    if (t + 1 < last) load(t + 1, 1 - s);
    const uint8_t* sc = reinterpret_cast<const uint8_t*>(scales[s]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      v8i b[NT];
      int sb[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int row = wn + 16 * j + r;
        b[j] = operand4(right[s][code_at(row, 4 * h + g)]);
        sb[j] = sc[(BM + row) * 8 + 4 * h + g];
      }
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int row = wm + 16 * i + r;
        const v8i a = operand4(left[s][code_at(row, 4 * h + g)]);
        const int sa = sc[row * 8 + 4 * h + g];
#pragma unroll
        for (int j = 0; j < NT; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[j], a, acc[i][j], 4, 4, 0, sb[j], 0, sa);
      }
      // the first three rows' operands are read ahead, then one for every half row of
      // instructions (8192^3: 341 us in the compiler's own order, 333 so)
      __builtin_amdgcn_sched_group_barrier(0x100, 2 * NT + 6, 0);  // reads of shared memory
#pragma unroll
      for (int i = 0; i < 2 * MT; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, NT / 2, 0);  // matrix instructions
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
    }
    if (t + 1 < last) arrive(1 - s);
  }
  __syncthreads();
  put_wave<MT, NT>(p, acc, &left[0][0], wave, i0 + wm, j0 + wn);
}

template <int SRC, bool TRANS, int BBITS>
hipError_t launch_bf16(const Args& p, const ProductPlan& plan, hipStream_t stream) {
  constexpr int BM = parts_of(SRC) == 1 ? 256 : 128;
  const bool wide = plan.bm == BM && plan.bn == 256;
  if (!wide && (plan.bm != 128 || (plan.bn != 128 && plan.bn != 64)))
    return hipErrorInvalidValue;  // not a tile of this kernel
  return launch_slices(p, plan, bytes_of(SRC), [&](dim3 grid, const Args& q, uint32_t nm, uint32_t nn) {
    if (wide) {
      // (transposed operands: a kernel of its own where every lane has all of its rows or none.
      // 4096x4096 over 16384 in bfloat16 takes 470 us, with the other kernel 511; 803x236 over 66454 takes 77 us with
      // the other one, with its last lane's rows one by one 96)
      if constexpr (TRANS) {
        if (q.m % (BM / 64) == 0) {
          tiles_bf16<SRC, TRANS, BBITS, BM, 256, 2, 1, false><<<grid, kLanes, 0, stream>>>(q, nm, nn);
          return;
        }
      }
      tiles_bf16<SRC, TRANS, BBITS, BM, 256, 2, 1, true><<<grid, kLanes, 0, stream>>>(q, nm, nn);
    } else if (plan.bn == 128) {
      tiles_bf16<SRC, TRANS, BBITS, 128, 128, 2, 1, true><<<grid, kLanes, 0, stream>>>(q, nm, nn);
    } else {
      tiles_bf16<SRC, TRANS, BBITS, 128, 64, 4, 2, true><<<grid, kLanes, 0, stream>>>(q, nm, nn);
    }
  });
}
template <int SRC, bool TRANS>
hipError_t launch_bf16_bits(const Args& p, const ProductPlan& plan, hipStream_t stream) {
  return p.b.bits == 4 ? launch_bf16<SRC, TRANS, 4>(p, plan, stream) : launch_bf16<SRC, TRANS, 8>(p, plan, stream);
}
template <int SRC>
hipError_t launch_bf16_op(const Args& p, const ProductPlan& plan, hipStream_t stream) {
  return p.a_cs == 1 ? launch_bf16_bits<SRC, false>(p, plan, stream) : launch_bf16_bits<SRC, true>(p, plan, stream);
}

}  // namespace

hipError_t launch_tiles_bf16(int src, const Args& p, const ProductPlan& plan, hipStream_t stream) {
  switch (src) {
    case SRC_MX4: return launch_bf16_bits<SRC_MX4, false>(p, plan, stream);
    case SRC_MX8: return launch_bf16_bits<SRC_MX8, false>(p, plan, stream);
    case SRC_BF16: return launch_bf16_op<SRC_BF16>(p, plan, stream);
    case SRC_F16: return launch_bf16_op<SRC_F16>(p, plan, stream);
    default: return launch_bf16_op<SRC_F32>(p, plan, stream);
  }
}

hipError_t launch_tiles_scaled(const Args& p, const ProductPlan& plan, hipStream_t stream) {
  const bool wide = plan.bm == 256 && plan.bn == 256;
  if (!wide && (plan.bm != 128 || plan.bn != 128)) return hipErrorInvalidValue;  // not a tile of this kernel
  return launch_slices(p, plan, 0, [&](dim3 grid, const Args& q, uint32_t nm, uint32_t nn) {
    if (wide) tiles_scaled<256, 256, 2><<<grid, kLanes, 0, stream>>>(q, nm, nn);
    else tiles_scaled<128, 128, 2><<<grid, kLanes, 0, stream>>>(q, nm, nn);
  });
}

}  // namespace costa
