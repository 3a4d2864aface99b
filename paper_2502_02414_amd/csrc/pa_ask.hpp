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

#include "pa_ops_internal.h"
#include "pa_stream.hpp"

namespace pa {
namespace ask {

constexpr int kTile = 64;  // rows of a tile in LDS

template <typename T, int DP> struct AskGeo {
  static constexpr int SZ = (int)sizeof(T), E = 16 / SZ;  // E: elements of 16 bytes
  static constexpr int RB = DP * SZ + 32;                 // bytes of a row in LDS (lds_off)
  static constexpr int CPR = DP * SZ / 16;                // 16-byte chunks of a row
  static constexpr int NCH = kTile * CPR / 256;           // chunks of a tile per thread
  static constexpr int NK = DP / 32, ND = DP / 16;        // steps over the width; tiles of it
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

// A tile of up to 64 rows on its way to LDS: 256 threads, 16 bytes each.  Loads have
// no branch around them: rows past the end read the last one, columns past D the
// first chunk, and both become zeros, as do the rows of states that are left out
// (which may hold anything).
template <typename T, int DP> struct TileLoad {
  using G_ = AskGeo<T, DP>;
  uint4 c[G_::NCH];

  // states [p0, p0 + 64) below e
  __device__ __forceinline__ void states(const T* base, int64_t ld, int64_t p0, int64_t e, int D,
                                         const uint8_t* mask) {
#pragma unroll
    for (int j = 0; j < G_::NCH; ++j) {
      const int q = threadIdx.x + 256 * j, row = q / G_::CPR, col = (q % G_::CPR) * G_::E;
      const int64_t p = p0 + row < e ? p0 + row : e - 1;
      uint8_t counts = 1;
      if (mask) counts = mask[p];
      const bool in = p0 + row < e && col < D && counts;
      const uint4 x = ld_global16<false>(base + p * ld + (col < D ? col : 0));
      c[j] = in ? x : zero16();
    }
  }
  // virtual rows [v0, v0 + 64) below n of a request that begins at query b
  __device__ __forceinline__ void queries(const T* base, int64_t ld, int64_t b, int G, int v0, int n,
                                          int D) {
#pragma unroll
    for (int j = 0; j < G_::NCH; ++j) {
      const int q = threadIdx.x + 256 * j, row = q / G_::CPR, col = (q % G_::CPR) * G_::E;
      const uint32_t v = v0 + row < n ? v0 + row : n - 1;
      const uint32_t i = G == 1 ? v : v / (uint32_t)G, g = v - i * G;
      const uint4 x = ld_global16<false>(base + (b + i) * ld + g * D + (col < D ? col : 0));
      c[j] = v0 + row < n && col < D ? x : zero16();
    }
  }
  __device__ __forceinline__ void put(char* tile) const {
#pragma unroll
    for (int j = 0; j < G_::NCH; ++j) {
      const int q = threadIdx.x + 256 * j;
      *reinterpret_cast<uint4*>(tile + lds_off(q / G_::CPR, (q % G_::CPR) * 16, G_::RB)) = c[j];
    }
  }
};

// A row's K32 fragments straight from memory: lane (r, g) elements 32 k + 8 g .. + 8
// of its row, zeros past D or where the row is none.
template <typename T, int DP>
__device__ __forceinline__ void row_frags(K32<T> (&f)[DP / 32], const T* row, int D, bool on) {
  const int g = lane_id() >> 4;
#pragma unroll
  for (int k = 0; k < DP / 32; ++k) {
    const int c = 32 * k + 8 * g;
    const bool in = on && c < D;
    const T* p = row + (c < D ? c : 0);
    if constexpr (sizeof(T) == 2) {
      const uint4 x = ld_global16<false>(p);
      f[k].v = __builtin_bit_cast(bf16x8, in ? x : zero16());
    } else {
      const uint4 x = ld_global16<false>(p), y = ld_global16<false>(p + 4);
      f[k].lo = __builtin_bit_cast(f32x4, in ? x : zero16());
      f[k].hi = __builtin_bit_cast(f32x4, in ? y : zero16());
    }
  }
}

template <typename T> __device__ __forceinline__ float k32_elem(const K32<T>& f, int e) {
  if constexpr (sizeof(T) == 2) return (float)f.v[e];
  else return e < 4 ? f.lo[e & 3] : f.hi[e & 3];
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

}  // namespace ask
}  // namespace pa
