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

#include "mx_product.hpp"

namespace costa {
namespace {

constexpr int kWaves = 8;
constexpr int kLanes = 64 * kWaves;

// Tile (tm, tn) of workgroup b of a launch over nm x nn tiles.  Workgroups go
// round the 8 XCDs in turn; each XCD gets a run of neighbouring tiles (8 tile
// rows wide, by columns), whose operands its L2 holds.
__device__ inline void tile_of(uint32_t b, uint32_t nm, uint32_t nn, int64_t& tm, int64_t& tn) {
  const uint32_t total = nm * nn, per = total / 8, more = total % 8, x = b % 8;
  const uint32_t t = x * per + min(x, more) + b / 8;
  const uint32_t group = t / (8 * nn), rows = min(8u, nm - group * 8), in = t - group * 8 * nn;
  // (the division runs on vector registers: both are the wave's, not a lane's)
  tm = __builtin_amdgcn_readfirstlane(group * 8 + in % rows);
  tn = __builtin_amdgcn_readfirstlane(in / rows);
}

// Part y of `parts` of a sum's steps.
__device__ inline void steps_of(uint32_t steps, uint32_t y, uint32_t parts, int64_t& first, int64_t& last) {
  const uint32_t per = steps / parts, more = steps % parts;
  first = __builtin_amdgcn_readfirstlane(y * per + min(y, more));
  last = __builtin_amdgcn_readfirstlane((y + 1) * per + min(y + 1, more));
}

// A wave's part of C, rows i0 .. and columns j0 .., through a piece of shared memory
// (the operands are done with): whole rows are written at a time, and the code that
// rounds and stores stands there twice and not for each of the MT x NT pieces, where
// fetching it cost small products more than running it.
template <int MT, int NT>
__device__ inline void put_wave(const Args& p, const v4f (&acc)[MT][NT], v4u* shared, int wave, int64_t i0,
                                int64_t j0) {
  constexpr int ROWS = 16, COLS = NT * 16, STRIDE = COLS / 4 + 1;  // 16-byte units: neighbouring rows, other banks
  constexpr int LANES = COLS / 4, PER = 64 / LANES;               // lanes a row, rows at a time
  v4f* const mine = reinterpret_cast<v4f*>(shared) + wave * ROWS * STRIDE;
  const int lane = threadIdx.x % 64, r = lane % 16, g = lane / 16;
  Epilogue e = p.e;
  if (p.part) e.c = static_cast<float*>(e.c) + blockIdx.y * p.part;
  const int64_t col = j0 + lane % LANES * 4;
  const int n = (int)max((int64_t)0, min((int64_t)4, p.n - col));
#pragma unroll
  for (int i = 0; i < MT; ++i) {
#pragma unroll
    for (int j = 0; j < NT; ++j) mine[r * STRIDE + 4 * j + g] = acc[i][j];
    wave_fence();
#pragma unroll 1
    for (int q = 0; q < ROWS; q += PER) {
      const int64_t row = i0 + 16 * i + q + lane / LANES;
      if (row < p.m) put_four(e, row, col, mine[(q + lane / LANES) * STRIDE + lane % LANES], n);
    }
    wave_fence();
  }
}

// ---- plain (or decoded) left operand: bfloat16 instructions --------------------------
// k goes by 64.  The left tile is held as bfloat16 parts, 128 bytes a row, its 16-byte
// chunks (8 elements) permuted within a row so that lanes on neighbouring rows meet
// different banks; the right tile as stored, decoded on the way to the matrix
// instruction (16 elements of a row a lane and step, 8 for each of two
// instructions; the left operand is read in the same order of k).  A few-bit tile in
// shared memory is a quarter or half of what it is decoded, and decoding costs 8
// conversions for 4 * MT matrix instructions.
//
// Measured: 2048x8192x8192 of bfloat16 by 4 bits 217 to 235 us (1.17 to 1.27 PFLOP/s; the
// library's product of two bfloat16 matrices reaches 1.47 at 8192^3), 4096x4096 over 16384
// transposed by 8 bits 470 to 515 us (1.07 to 1.17).  The matrix units are busy half of the
// time, at 2.0 to 2.1 GHz; a third stage, reading further ahead and wave priorities changed
// nothing.  256x256 tiles for one bfloat16 part (8 waves of 128x64: 128 registers of sums), 128x256
// for two and three, whose parts fill the shared memory; smaller tiles where those are few.
constexpr int kStepBf16 = 64;
__device__ inline int chunk_at(int row, int chunk) { return row * 8 + (chunk ^ ((row ^ row >> 3) & 7)); }

// EDGE: a transposed operand's last lane may have fewer rows than MPT.
template <int SRC, bool TRANS, int BM, bool EDGE>
struct LeftStage {
  static constexpr bool MX = SRC == SRC_MX4 || SRC == SRC_MX8;
  static constexpr int BITS = SRC == SRC_MX4 ? 4 : 8;
  static constexpr int P = parts_of(SRC);
  static constexpr int ES = bytes_of(SRC);
  static constexpr int PASSES = BM / 64;  // chunks of a lane (k next to one another)
  static constexpr int MPT = BM / 64;     // rows of a lane (rows next to one another)
  static constexpr int TW = (MPT * ES + 3) / 4;

  Raw8<SRC> raw[TRANS || MX ? 1 : PASSES];
  // few-bit operands: sixteen elements of a lane at a time, half a block
  static constexpr int HALVES = BM / 128;
  v4u code[MX ? HALVES : 1];
  uint32_t scale[MX ? HALVES : 1];
  uint32_t line[TRANS ? 8 : 1][TW];
  bool moved;  // (transposed) the last lane's rows are not in place yet

  // (Where a whole step is there, all of its loads stand behind one branch: none
  // waits for another.)
  __device__ inline void load(const Args& p, int64_t i0, int64_t k0) {
    const int t = threadIdx.x;
    if constexpr (TRANS) {
      // wave w has k = k0 + 8 w .. + 7, lane l rows MPT l .. of each
      const int wave = __builtin_amdgcn_readfirstlane(t / 64);
      const char* base = static_cast<const char*>(p.real) + ((k0 + 8 * wave) * p.a_cs + i0) * ES;
      moved = false;
      if (!EDGE && k0 + kStepBf16 <= p.k) {
        if (MPT * (t % 64) < p.m - i0)
#pragma unroll
          for (int q = 0; q < 8; ++q) __builtin_memcpy(line[q], base + q * p.a_cs * ES + MPT * ES * (t % 64), MPT * ES);
      } else if (EDGE && p.m >= MPT && k0 + kStepBf16 <= p.k) {
        // the last lane with rows reads the matrix's last MPT, as do those past it
        // (whose results are not stored); store() moves what it read into place.
        // (803x236 over 66454 in float: 211 us row by row, 142 so)
        moved = true;
        const char* at = base + min((int64_t)MPT * (t % 64), p.m - i0 - MPT) * ES;
#pragma unroll
        for (int q = 0; q < 8; ++q) __builtin_memcpy(line[q], at + q * p.a_cs * ES, MPT * ES);
      } else {  // the last of k, or fewer rows than a lane takes: one by one
        const int64_t left = p.m - i0 - MPT * (t % 64);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
#pragma unroll
          for (int w = 0; w < TW; ++w) line[q][w] = 0;
          if (k0 + 8 * wave + q < p.k) {
            const char* from = base + (q * p.a_cs + MPT * (t % 64)) * ES;
#pragma unroll
            for (int e = 0; e < MPT; ++e)
              if (e < left) {
                if (ES == 4) line[q][e % TW] = reinterpret_cast<const uint32_t*>(from)[e];
                else line[q][e / 2 % TW] |= (uint32_t) reinterpret_cast<const uint16_t*>(from)[e] << (e % 2 * 16);
              }
          }
        }
      }
    } else {
      const int c = t % 8;
      const int64_t k = k0 + 8 * c;
      if constexpr (MX) {
#pragma unroll
        for (int q = 0; q < HALVES; ++q) {  // (a row is padded to whole steps)
          const int64_t i = min(i0 + t / 4 + 128 * q, p.m - 1), k16 = k0 + 16 * (t % 4);
          const uint8_t* at = p.a.data + i * p.a.row_bytes + k16 * BITS / 8;
          if constexpr (BITS == 4) {
            const v2u d = *reinterpret_cast<const v2u*>(at);
            code[q] = v4u{d.x, 0u, d.y, 0u};
          } else {
            code[q] = *reinterpret_cast<const v4u*>(at);
          }
          scale[q] = p.a.scales[i * p.a.row_scales + k16 / kMxBlock];
        }
      } else if (k0 + kStepBf16 <= p.k) {
#pragma unroll
        for (int q = 0; q < PASSES; ++q) {
          const int64_t i = min(i0 + t / 8 + 64 * q, p.m - 1);
          __builtin_memcpy(raw[q].w, static_cast<const char*>(p.real) + (i * p.a_rs + k) * ES, sizeof raw[q].w);
        }
      } else {
#pragma unroll
        for (int q = 0; q < PASSES; ++q) {
          const int64_t i = min(i0 + t / 8 + 64 * q, p.m - 1);
          load8<SRC>(raw[q], static_cast<const char*>(p.real) + i * p.a_rs * ES, k, p.k);
          place8<SRC>(raw[q], k, p.k);
        }
      }
    }
  }

  // stage: P planes of BM x 8 chunks
  __device__ inline void store(const Args& p, int64_t i0, v4u* stage) {
    const int t = threadIdx.x;
    if constexpr (TRANS) {
      if (EDGE && moved) {
        const uint32_t drop = (uint32_t)max((int64_t)0, MPT * (t % 64) - (p.m - i0 - MPT));
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          if constexpr (TW == 1) {
            line[q][0] >>= 16 * (drop & 1);
          } else {
            const uint64_t v = (line[q][0] | (uint64_t)line[q][1] << 32) >> (8 * ES * (drop % MPT));
            line[q][0] = (uint32_t)v;
            line[q][1] = (uint32_t)(v >> 32);
          }
        }
      }
#pragma unroll
      for (int e = 0; e < MPT; ++e) {
        v4u out[P];
        if constexpr (SRC == SRC_BF16) {
#pragma unroll
          for (int q = 0; q < 4; ++q)  // halves of two k side by side
            out[0][q] = __builtin_amdgcn_perm(line[2 * q + 1][e / 2], line[2 * q][e / 2],
                                              e % 2 ? 0x07060302u : 0x05040100u);
        } else {
          Raw8<SRC> r;
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            if constexpr (ES == 4) r.w[q] = line[q][e];
            else if (q % 2 == 0) r.w[q / 2] = __builtin_amdgcn_perm(line[q + 1][e / 2], line[q][e / 2],
                                                                    e % 2 ? 0x07060302u : 0x05040100u);
          }
          raw_parts<SRC>(r, out);
        }
#pragma unroll
        for (int x = 0; x < P; ++x) stage[x * BM * 8 + chunk_at(MPT * (t % 64) + e, t / 64)] = out[x];
      }
    } else if constexpr (MX) {
#pragma unroll
      for (int q = 0; q < HALVES; ++q)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          stage[chunk_at(t / 4 + 128 * q, 2 * (t % 4) + h)] =
              mx_decode8_bf16<BITS>(v2u{code[q][2 * h], code[q][2 * h + 1]}, scale[q]);
    } else {
#pragma unroll
      for (int q = 0; q < PASSES; ++q) {
        v4u out[P];
        raw_parts<SRC>(raw[q], out);
#pragma unroll
        for (int x = 0; x < P; ++x) stage[x * BM * 8 + chunk_at(t / 8 + 64 * q, t % 8)] = out[x];
      }
    }
  }
};

template <int BBITS, int BN>
struct RightStage {
  static constexpr int BYTES = kStepBf16 * BBITS / 8;         // of a row
  static constexpr int CHUNKS = BYTES / 16;                   // 2 or 4 of them
  static constexpr int PASSES = (BN * CHUNKS + kLanes - 1) / kLanes;
  v4u data[PASSES];
  uint32_t scale;
  __device__ inline void load(const Args& p, int64_t j0, int64_t k0) {
    const int t = threadIdx.x;
#pragma unroll
    for (int q = 0; q < PASSES; ++q) {
      const int at = (t + q * kLanes) % (BN * CHUNKS);  // (lanes past the tile repeat others' loads)
      const int64_t j = min(j0 + at / CHUNKS, p.n - 1);
      data[q] = *reinterpret_cast<const v4u*>(p.b.data + j * p.b.row_bytes + k0 * BBITS / 8 + at % CHUNKS * 16);
    }
    // (every lane in the small tiles, where a branch costs a wait for all loads: 1041x1999x2501 of 8 by 4 bits
    // 43 us with, 37 without; in the large ones the loads cost more than the branch: 470 and 478 us)
    if (BN < 256 || t < BN) {
      const int64_t j = min(j0 + t % BN, p.n - 1);
      scale = *reinterpret_cast<const uint16_t*>(p.b.scales + j * p.b.row_scales + k0 / kMxBlock);
    }
  }
  __device__ inline void store(v4u* stage, uint16_t* scales) const {
    const int t = threadIdx.x;
#pragma unroll
    for (int q = 0; q < PASSES; ++q) {
      const int at = t + q * kLanes;
      if (BN * CHUNKS % kLanes == 0 || at < BN * CHUNKS) stage[at] = data[q];
    }
    if (t < BN) scales[t] = (uint16_t)scale;
  }
};

// AHEAD: steps whose loads are on their way at once.
template <int SRC, bool TRANS, int BBITS, int BM, int BN, int WM, int AHEAD, bool EDGE>
__global__ __launch_bounds__(kLanes) void tiles_bf16(Args p, uint32_t nm, uint32_t nn) {
  constexpr int WN = kWaves / WM, MT = BM / WM / 16, NT = BN / WN / 16, P = parts_of(SRC);
  constexpr int BROW = kStepBf16 * BBITS / 8;
  __shared__ v4u left[2][P * BM * 8];
  __shared__ v4u right[2][BN * BROW / 16];
  __shared__ uint16_t scales[2][BN];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16, g = lane / 16;
  const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
  int64_t tm, tn;
  tile_of(blockIdx.x, nm, nn, tm, tn);
  const int64_t i0 = tm * BM, j0 = tn * BN;
  int64_t first, last;
  steps_of((uint32_t)((p.k + kStepBf16 - 1) / kStepBf16), blockIdx.y, gridDim.y, first, last);

  v4f acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = v4f{0, 0, 0, 0};

  LeftStage<SRC, TRANS, BM, EDGE> ls[AHEAD];
  RightStage<BBITS, BN> rs[AHEAD];
  auto load = [&](int set, int64_t t) {
    if (t < last) {
      ls[set].load(p, i0, t * kStepBf16);
      rs[set].load(p, j0, t * kStepBf16);
    }
  };
  load(0, first);
  ls[0].store(p, i0, left[0]);
  rs[0].store(right[0], scales[0]);
#pragma unroll
  for (int a = 1; a <= AHEAD; ++a) load(a % AHEAD, first + a);
  __syncthreads();
  for (int64_t t0 = first; t0 < last; t0 += 2) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int64_t t = t0 + s;
      if (t >= last) break;
      v4u b[NT];
      uint32_t sc[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int row = wn + 16 * j + r;
        if (BBITS == 4) {
          const v2u d = reinterpret_cast<const v2u*>(right[s])[row * 4 + g];
          b[j] = v4u{d.x, d.y, 0u, 0u};
        } else {
          b[j] = right[s][row * 4 + g];
        }
        sc[j] = reinterpret_cast<const uint8_t*>(scales[s])[row * 2 + g / 2];
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        v4u w[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j)
          w[j] = mx_decode8_bf16<BBITS>(BBITS == 4 ? v2u{b[j][h], 0u} : v2u{b[j][2 * h], b[j][2 * h + 1]}, sc[j]);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int x = 0; x < P; ++x) {
            const v4u a = left[s][x * BM * 8 + chunk_at(wm + 16 * i + r, 2 * g + h)];
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = mfma_bf16(w[j], a, acc[i][j]);
          }
      }
      if (t + 1 < last) {
        const int set = (s + 1) % AHEAD;  // (AHEAD is 1 or 2: a step's parity is its set)
        ls[set].store(p, i0, left[1 - s]);
        rs[set].store(right[1 - s], scales[1 - s]);
        load(set, t + 1 + AHEAD);
      }
      __syncthreads();
    }
  }
  put_wave<MT, NT>(p, acc, &left[0][0], wave, i0 + wm, j0 + wn);
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

constexpr int64_t kTilesMax = INT32_MAX;
constexpr int64_t kTileSlice = (int64_t)1 << 22;  // workgroups of a launch: below 2^32 lanes

// Launches the tiles of C, in slices of whole rows or columns of tiles where a grid does
// not hold them all: each a product of its own.  (The kernels take no part in this: an
// offset among their arguments changed how the compiler ordered one of them, 1041x1999x2501
// of 8 by 4 bits 43.0 us without, 45.3 with.)
template <typename F>
hipError_t launch_slices(const Args& p, const ProductPlan& plan, int elem_bytes, F launch) {
  const int64_t nm = (p.m + plan.bm - 1) / plan.bm, nn = (p.n + plan.bn - 1) / plan.bn;
  // (a C of 16 TiB and more: either dimension is below 2^31)
  if (nm * nn > kTilesMax) throw LimitExceeded("a product of more than 2^31 - 1 tiles");
  const int64_t cols = std::min(nn, kTileSlice), rows = std::min(nm, kTileSlice / cols);
  for (int64_t tm = 0; tm < nm; tm += rows)
    for (int64_t tn = 0; tn < nn; tn += cols) {
      const int64_t i = tm * plan.bm, j = tn * plan.bn;
      Args q = p;
      q.m = q.a.rows = std::min(rows * plan.bm, p.m - i);
      q.n = q.b.rows = std::min(cols * plan.bn, p.n - j);
      if (p.real) q.real = static_cast<const char*>(p.real) + i * p.a_rs * elem_bytes;
      q.a.data += i * p.a.row_bytes;
      q.a.scales += i * p.a.row_scales;
      q.b.data += j * p.b.row_bytes;
      q.b.scales += j * p.b.row_scales;
      q.e.c = static_cast<char*>(p.e.c) + (i * p.e.rs + j * p.e.cs) * (p.e.type == COSTA_REAL_F32 ? 4 : 2);
      const uint32_t tall = (uint32_t)std::min(rows, nm - tm), wide = (uint32_t)std::min(cols, nn - tn);
      launch(dim3(tall * wide, plan.splits), q, tall, wide);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  return hipSuccess;
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
