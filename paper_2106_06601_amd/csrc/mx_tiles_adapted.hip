// Products in tiles of C with the adapters' part added to a tile's sums before they are
// rounded and stored:  c_i = alpha p_i + s_a v_i B_a + beta c_i.
//
// A wave has 16 MT rows and 16 NT columns.  It takes the distinct adapters of its rows by turns:
// an adapter's ranks go by 32, straight from memory to registers, eight ranks of NT neighbouring
// columns a lane, which are operands of the matrix instruction for the NT pieces (the tile's
// columns are dealt to them so).  Of a piece's sixteen rows those that have the adapter take
// what comes out.
//
// Measured: 4096 rows in runs of 8 adapters of rank 64 by 8192x8192 in 4 bits about 10 us over the product's 441
// (added to sums in memory by another kernel: 223 and 20 more for the sums); making v's parts here, 32 times
// over, cost 70.  Rows of many adapters mixed cost more, each adapter's ranks being loaded for a few rows:
// 4096 rows of 8 adapters of rank 16 100 us, of 64 adapters 350.  Bound by the matrix units as the products are
// (51% busy at 2.0 GHz).  In bfloat16 by 8 bits the largest tile spills 4 of its 256 registers.
#include "mx_adapters.hpp"
#include "mx_tiles.hpp"

namespace costa {
namespace {

template <int SRC, int MT, int NT>
__device__ inline void add_adapters(const AdapterAddArgs& a, TileSums<MT, NT>& t) {
  constexpr int P = parts_of(SRC), ES = bytes_of(SRC), WORDS = NT * ES / 4;
  const int lane = threadIdx.x % 64, l = lane % 16, g = lane / 16;
  const int64_t col = t.col + NT * l;
  const bool edge = t.col + 16 * NT > a.n;
  const int64_t steps = (a.at.rank + 31) / 32, last = (a.m - 1) / 16 - t.row / 16;  // (the last piece with rows)
  int32_t idx[MT];
  uint32_t left[MT], any = 0;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t row = t.row + 16 * i + l;
    idx[i] = row < a.m ? adapter_of(a.at, row) : -1;
    left[i] = (uint32_t)__ballot(idx[i] >= 0) & 0xffff;
    any |= left[i];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) t.acc[i][j][q] *= a.alpha;
  }
  while (any) {
    // the first piece's next adapter, and the pieces that have it
    int32_t id = -1;
#pragma unroll
    for (int i = MT - 1; i >= 0; --i)
      if (left[i]) id = __builtin_amdgcn_readlane(idx[i], __builtin_ctz(left[i]));
    uint32_t has = 0, full = 0;
    any = 0;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const uint32_t mine = (uint32_t)__ballot(idx[i] == id) & 0xffff;
      has |= mine ? 1u << i : 0u;
      full |= mine == 0xffff ? 1u << i : 0u;
      left[i] &= ~mine;
      any |= left[i];
    }
    const int rank = rank_of(a.at, id);
    for (int r0 = 0; r0 < rank; r0 += 32) {
      uint32_t b[8][WORDS];
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int r = r0 + 8 * g + q;
        const char* at = static_cast<const char*>(a.low.data) + (((int64_t)id * a.at.rank + min(r, rank - 1)) * a.low.ld + col) * ES;
        if (!edge) {
          __builtin_memcpy(b[q], at, sizeof b[q]);
        } else {
#pragma unroll
          for (int w = 0; w < WORDS; ++w) b[q][w] = 0;
#pragma unroll
          for (int e = 0; e < NT; ++e)
            if (col + e < a.n) {
              if constexpr (ES == 4) b[q][e] = reinterpret_cast<const uint32_t*>(at)[e];
              else b[q][e / 2] |= (uint32_t) reinterpret_cast<const uint16_t*>(at)[e] << (e % 2 * 16);
            }
        }
      }
      // s v of a piece's rows, as operands (the next piece's are on their way while one is worked on)
      const v4u* const spread = a.spread + ((t.row / 16 * steps + r0 / 32) * 3) * 64 + lane;
      v4u next[3];
      auto load_v = [&](int i) {  // (a wave past the last row has nothing to do here)
#pragma unroll
        for (int x = 0; x < 3; ++x) next[x] = spread[(min((int64_t)i, last) * steps * 3 + x) * 64];
      };
      if (has & 1) load_v(0);
      if (r0 + 32 > rank)  // (past the last rank was that again)
#pragma unroll
        for (int q = 0; q < 8; ++q)
#pragma unroll
          for (int w = 0; w < WORDS; ++w) b[q][w] = r0 + 8 * g + q < rank ? b[q][w] : 0u;
      v4u bp[NT][P];
#pragma unroll
      for (int e = 0; e < NT; ++e) {
        Raw8<SRC> raw;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          if constexpr (ES == 4) raw.w[q] = b[q][e];
          else if (q % 2 == 0) raw.w[q / 2] = __builtin_amdgcn_perm(b[q + 1][e / 2], b[q][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
        }
        raw_parts<SRC>(raw, bp[e]);
      }
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        v4u v[3];
#pragma unroll
        for (int x = 0; x < 3; ++x) v[x] = next[x];
        if (i + 1 < MT && (has >> (i + 1) & 1)) load_v(i + 1);
        if (!(has >> i & 1)) continue;
        if (full >> i & 1) {  // all of the piece's rows
#pragma unroll
          for (int e = 0; e < NT; ++e) t.acc[i][e] = mfma_parts<P, 3>(bp[e], v, t.acc[i][e]);
        } else {
#pragma unroll
          for (int e = 0; e < NT; ++e) {
            const v4f d = mfma_parts<P, 3>(bp[e], v, v4f{0, 0, 0, 0});
#pragma unroll
            for (int q = 0; q < 4; ++q) t.acc[i][e][q] += idx[i] == id ? d[q] : 0.0f;
          }
        }
      }
    }
  }
}

template <int SRC, int BBITS, int BM, int BN>
__global__ __launch_bounds__(kLanes) void tiles_adapted(Args p, AdapterAddArgs a, uint32_t nm, uint32_t nn) {
  constexpr int MT = BM / 2 / 16, NT = BN / (kWaves / 2) / 16;
  TileSums<MT, NT> t;
  tile_sums<SRC, false, BBITS, BM, BN, 2, 1, true, NT>(p, nm, nn, t);
  add_adapters<SRC, MT, NT>(a, t);
  put_wave<MT, NT, NT>(p, t.acc, t.shared, t.wave, t.row, t.col);
}

template <int SRC, int BBITS>
hipError_t launch_adapted(const Args& p, const AdapterAddArgs& a, const ProductPlan& plan, hipStream_t stream) {
  constexpr int BM = parts_of(SRC) == 1 ? 256 : 128;
  const uint32_t nm = (uint32_t)up_div(p.m, plan.bm), nn = (uint32_t)up_div(p.n, plan.bn);
  if (plan.bm == BM && plan.bn == 256) tiles_adapted<SRC, BBITS, BM, 256><<<dim3(nm * nn), kLanes, 0, stream>>>(p, a, nm, nn);
  else if (plan.bm == 128 && plan.bn == 128) tiles_adapted<SRC, BBITS, 128, 128><<<dim3(nm * nn), kLanes, 0, stream>>>(p, a, nm, nn);
  else return hipErrorInvalidValue;  // not a tile of this kernel
  return hipGetLastError();
}
template <int SRC>
hipError_t launch_adapted_bits(const Args& p, const AdapterAddArgs& a, const ProductPlan& plan, hipStream_t stream) {
  return p.b.bits == 4 ? launch_adapted<SRC, 4>(p, a, plan, stream) : launch_adapted<SRC, 8>(p, a, plan, stream);
}

int source_of(costa_real type) { return type == COSTA_REAL_BF16 ? SRC_BF16 : type == COSTA_REAL_F16 ? SRC_F16 : SRC_F32; }

}  // namespace

bool mx_adapted_fused(costa_real type, int bits, int64_t m, int64_t n, int64_t k) {
  if (n == 0 || k == 0 || m < 1024) return false;
  const ProductPlan r = plan_product(source_of(type), true, bits, m, n, k);
  return r.variant == TILES_BF16 && r.splits == 1 && r.bn >= 128 && up_div(m, r.bm) * up_div(n, r.bn) <= kTileSlice;
}

hipError_t launch_mx_adapted_product(const AdapterAddArgs& a, const RowsView& x, int64_t k, const MxView& w,
                                     hipStream_t stream) {
  const int src = source_of(a.type);
  const ProductPlan plan = plan_product(src, true, w.bits, a.m, a.n, k);
  const int64_t es = a.c_type == COSTA_REAL_F32 ? 4 : 2;
  const Epilogue e{a.c.data, a.c.ld, 1, a.c_type, a.c.ld % 4 == 0 && (uintptr_t)a.c.data % (4 * es) == 0, 1.0f, a.beta};
  const Args p{a.m, a.n, k, MxView{}, w, x.data, x.ld, 1, e, 0};
  if (src == SRC_BF16) return launch_adapted_bits<SRC_BF16>(p, a, plan, stream);
  if (src == SRC_F16) return launch_adapted_bits<SRC_F16>(p, a, plan, stream);
  return launch_adapted_bits<SRC_F32>(p, a, plan, stream);
}

}  // namespace costa
