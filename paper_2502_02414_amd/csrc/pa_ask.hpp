// Attention of query points over the states of their request (gfx950): what the
// kernels of pa_ask_fwd.hip and pa_ask_bwd.hip have in common.
//
// Rows of a request and of a head of k and v: its queries times the G = Hq / Hkv
// query heads that share the head ("virtual" row v: query v / G, head v % G of the
// group), so that states are read once for all of them.  A block takes a tile of
// such rows; requests' tiles lie one behind the other in the grid at slots
//   first(r) = floor(q_off[r] G / tile) + r,
// which leaves each request at least as many slots as it has tiles, needs no sum
// over the requests before it, and so no pass over the offsets on the host.
//
// Products (v_mfma_f32_16x16x32_bf16; fp32: 16x16x4) are laid out so that the scores
// leave the matrix cores where the next product reads them: with states as rows and
// queries as columns a lane holds states 4g .. 4g+3 of its query, which is an operand
// of the product over the states (and with the two exchanged, over the queries).
#pragma once

#include <type_traits>

#include "pa_ops_internal.h"
#include "pa_stream.hpp"

namespace pa {
namespace ask {

constexpr int kTile = 64;  // rows of a tile in LDS

// Operands over the width: K32 of 32 elements for bf16; for fp32, whose products take 16
// times as long, K16 of 16, so that less of a width is padding.
template <typename T> struct Wide;
template <> struct Wide<bf16> {
  typedef K32<bf16> F;
  static constexpr int W = 32, L = 8;  // elements of a step, and of a lane
};
template <> struct Wide<float> {
  typedef K16<float> F;
  static constexpr int W = 16, L = 4;
};
template <typename T> using WideF = typename Wide<T>::F;
__device__ __forceinline__ f32x4 mma(const K32<bf16>& a, const K32<bf16>& b, f32x4 c) {
  return mma32(a, b, c);
}
__device__ __forceinline__ f32x4 mma(const K16<float>& a, const K16<float>& b, f32x4 c) {
  return mma16(a, b, c);
}
__device__ __forceinline__ void set_wide(K32<bf16>& f, const uint4& x) {
  f.v = __builtin_bit_cast(bf16x8, x);
}
__device__ __forceinline__ void set_wide(K16<float>& f, const uint4& x) {
  f.v = __builtin_bit_cast(f32x4, x);
}
__device__ __forceinline__ float wide_elem(const K32<bf16>& f, int e) { return (float)f.v[e]; }
__device__ __forceinline__ float wide_elem(const K16<float>& f, int e) { return f.v[e]; }

// DP: the width, rounded up to a multiple of 16.
template <typename T, int DP> struct AskGeo {
  static constexpr int SZ = (int)sizeof(T), E = 16 / SZ;  // E: elements of 16 bytes
  static constexpr int NK = (DP + Wide<T>::W - 1) / Wide<T>::W, ND = DP / 16;  // steps; tiles
  static constexpr int ROW = NK * Wide<T>::W * SZ;        // bytes of a row
  static constexpr int RB = ROW + 32;                     // in LDS (lds_off)
  static constexpr int CPR = ROW / 16;                    // 16-byte chunks of a row
  static constexpr int NCH = kTile * CPR / 256;           // chunks of a tile per thread
  static constexpr int TB = kTile * RB;                   // bytes of a tile
};

__device__ __forceinline__ int64_t clamp64(int64_t v, int64_t lo, int64_t hi) {
  return v < lo ? lo : v > hi ? hi : v;
}

// A request's rows [b, e); offsets outside of the tensor are moved to its ends.
struct Range {
  int64_t b, e;
};
__device__ __forceinline__ Range range_of(const int64_t* off, int r, int64_t N) {
  if (!off) return {0, N};
  const int64_t b = clamp64(off[r], 0, N);
  return {b, clamp64(off[r + 1], b, N)};
}

// The request whose slots hold `slot` (-1: none), by 64 lanes at once.
__device__ __forceinline__ int request_of(const int64_t* off, int R, int64_t N, int G, int shift,
                                          int64_t slot) {
  if (!off) return 0;
  int lo = 0, hi = R;
  bool first = true;
  while (first || hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, r = lo + lane_id() * step;
    const bool below =
        r < hi && ((clamp64(off[r < R ? r : R - 1], 0, N) * G) >> shift) + r <= slot;
    const int n = __popcll(__ballot(below));
    if (n == 0) {
      if (first) return -1;
      break;
    }
    first = false;
    lo += (n - 1) * step;
    if (lo + step < hi) hi = lo + step;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// A piece of [b, e): the s-th of S, in whole tiles.
__device__ __forceinline__ Range piece(Range k, int s, int S) {
  if (S == 1) return k;
  const int64_t per = ((k.e - k.b + S - 1) / S + kTile - 1) / kTile * kTile;
  const int64_t b = k.b + per * s;
  return {b < k.e ? b : k.e, b + per < k.e ? b + per : k.e};
}

__device__ __forceinline__ uint4 zero16() { return uint4{0, 0, 0, 0}; }

// Memory that loads are checked against: an offset past its end reads zeros, so that
// no load stands behind a branch.
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_of(const void* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00027000);
}
__device__ __forceinline__ uint4 load16(Buffer b, int at) {
  return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(b, at, 0, 0));
}
constexpr int kNowhere = 0x7fffff00;

// A tile of up to 64 rows on its way to LDS: 256 threads, 16 bytes each, zeros where
// rows or columns end.  Offsets within a tile stay below 2^31: rows are at most 2^25
// bytes apart.
template <typename T, int DP> struct TileLoad {
  using G_ = AskGeo<T, DP>;
  uint4 c[G_::NCH];
  int off[G_::NCH];

  static __device__ __forceinline__ int row(int j) { return (threadIdx.x + 256 * j) / G_::CPR; }
  static __device__ __forceinline__ int col(int j) {
    return (threadIdx.x + 256 * j) % G_::CPR * G_::E;
  }
  // rows of states, ld elements apart
  __device__ __forceinline__ void states(int64_t ld, int D) {
#pragma unroll
    for (int j = 0; j < G_::NCH; ++j)
      off[j] = col(j) < D ? (row(j) * (int)ld + col(j)) * G_::SZ : kNowhere;
  }
  // virtual rows of a request from row `rem` of a query's group on
  __device__ __forceinline__ void queries(int64_t ld, int G, int rem, int D) {
#pragma unroll
    for (int j = 0; j < G_::NCH; ++j) {
      const uint32_t v = rem + row(j), i = G == 1 ? v : v / (uint32_t)G, g = v - i * G;
      off[j] = col(j) < D ? (int)(i * (uint32_t)ld + g * D + col(j)) * G_::SZ : kNowhere;
    }
  }
  __device__ __forceinline__ void load(Buffer b, int rows) {
#pragma unroll
    for (int j = 0; j < G_::NCH; ++j) c[j] = load16(b, row(j) < rows ? off[j] : kNowhere);
  }
  __device__ __forceinline__ void put(char* tile) const {
#pragma unroll
    for (int j = 0; j < G_::NCH; ++j)
      *reinterpret_cast<uint4*>(tile + lds_off(row(j), col(j) * G_::SZ, G_::RB)) = c[j];
  }
};

// Tiles of a request's states: k and v, and which of them count, two of each in LDS.
template <typename T, int DP> struct StateTiles {
  using Gm = AskGeo<T, DP>;
  TileLoad<T, DP> k, v;
  const T *K, *V;
  const uint8_t* mask;
  int64_t ldk, ldv, e;
  int D;
  uint8_t keep[Gm::NCH];
  uint8_t counts;
  __device__ __forceinline__ void init(const AskArgs& a, int h, Range r) {
    K = reinterpret_cast<const T*>(a.k) + (int64_t)h * a.D;
    V = reinterpret_cast<const T*>(a.v) + (int64_t)h * a.D;
    mask = a.mask; ldk = a.ldk; ldv = a.ldv; e = r.e; D = a.D;
    k.states(ldk, D);
    v.states(ldv, D);
  }
  __device__ __forceinline__ void load(int64_t p0) {
    const int rows = e - p0 < kTile ? (int)(e - p0) : kTile;
    k.load(buffer_of(K + p0 * ldk, ((rows - 1) * ldk + D) * Gm::SZ), rows);
    v.load(buffer_of(V + p0 * ldv, ((rows - 1) * ldv + D) * Gm::SZ), rows);
    counts = (int)threadIdx.x < rows;
    if (mask) {
      const Buffer m = buffer_of(mask + p0, rows);
      counts = __builtin_amdgcn_raw_buffer_load_b8(m, threadIdx.x & 63, 0, 0);
#pragma unroll
      for (int j = 0; j < Gm::NCH; ++j)
        keep[j] = __builtin_amdgcn_raw_buffer_load_b8(m, k.row(j), 0, 0);
    }
  }
  // into LDS: k's tile, v's behind it; live: 0, or -infinity where a state is left out
  __device__ __forceinline__ void put(char* tiles, float* live) {
    if (mask) {  // (zeros for what may hold anything)
#pragma unroll
      for (int j = 0; j < Gm::NCH; ++j) {
        k.c[j] = keep[j] ? k.c[j] : zero16();
        v.c[j] = keep[j] ? v.c[j] : zero16();
      }
    }
    k.put(tiles);
    v.put(tiles + Gm::TB);
    if (threadIdx.x < kTile) live[threadIdx.x] = counts ? 0.f : -INFINITY;
  }
};

// Operand of lane (r, g)'s row straight from memory, zeros past D or where the row is
// none (its address has to be one that may be read all the same).
template <typename T, int DP>
__device__ __forceinline__ void row_frags(WideF<T>* f, const T* row, int D, bool on) {
  const int g = lane_id() >> 4;
#pragma unroll
  for (int k = 0; k < AskGeo<T, DP>::NK; ++k) {
    const int c = Wide<T>::W * k + Wide<T>::L * g;
    const uint4 x = ld_global16<false>(row + (c < D ? c : 0));
    set_wide(f[k], on && c < D ? x : zero16());
  }
}
// The same from LDS: row r of the 16 that begin at byte `at`, step k.
template <typename T>
__device__ __forceinline__ void ld_wide(WideF<T>& f, const char* tile, int base, int at) {
  set_wide(f, *reinterpret_cast<const uint4*>(tile + base + at));
}
template <typename T, int DP> __device__ __forceinline__ int wide_base() {
  return lds_off(lane_id() & 15, 16 * (lane_id() >> 4), AskGeo<T, DP>::RB);
}
constexpr int kStep = 64;  // bytes from one step over the width to the next

// The larger one, NaN where either is (one instruction of three operands; the score of
// a NaN makes its row NaN in any case).
__device__ __forceinline__ float largest(float a, float b) {
  return __builtin_elementwise_maximum(a, b);
}
// Of an accumulator's four.
__device__ __forceinline__ float largest(float a, const f32x4& x) {
  return largest(largest(a, largest(x[0], x[1])), largest(x[2], x[3]));
}

// Four consecutive elements of a row.
template <typename T> __device__ __forceinline__ void store4(T* p, const f32x4& v) {
  if constexpr (sizeof(T) == 2) {
    bf16x4 o;
    o[0] = (bf16)v[0]; o[1] = (bf16)v[1]; o[2] = (bf16)v[2]; o[3] = (bf16)v[3];
    *reinterpret_cast<bf16x4*>(p) = o;
  } else {
    *reinterpret_cast<f32x4*>(p) = v;
  }
}

// f(type, std::integral_constant of the width rounded up): fp32 is padded to multiples
// of 16, bf16, whose steps are 32 wide, too (the tiles of its results are 16 wide).
template <typename F> hipError_t by_width(int D, int dtype, F f) {
  const auto go = [&](auto type) {
    using std::integral_constant;
    if constexpr (sizeof(type) == 4)
      if (D <= 16) return f(type, integral_constant<int, 16>{});
    if (D <= 32) return f(type, integral_constant<int, 32>{});
    if (D <= 48) return f(type, integral_constant<int, 48>{});
    if (D <= 64) return f(type, integral_constant<int, 64>{});
    if (D <= 80) return f(type, integral_constant<int, 80>{});
    if (D <= 96) return f(type, integral_constant<int, 96>{});
    return f(type, integral_constant<int, 128>{});
  };
  return dtype == 1 ? go(bf16{}) : go(float{});
}

}  // namespace ask
}  // namespace pa
