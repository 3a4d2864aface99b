// Attention of query points over the states of their request (gfx950): what the
// kernels of pa_ask_fwd.hip, pa_ask_bwd.hip and pa_ask_few.hip have in common.
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

// DP: the width, rounded up to a multiple of 16.  A tile in LDS has rows of a power of
// two of 16-byte chunks, the chunk c of row i in place c ^ key(i).  A product reads rows
// (16 bytes a lane: in one cycle rows 0-3 and 12-15 of one chunk and 4-11 of its
// neighbour) and, bf16, columns (ds_read_b64_tr_b16: in one cycle two chunks of rows 0-7
// or of 8-15); with these keys both meet every bank once: 4.2 and 2.2 cycles for 1 KB and
// 512 B, with keys that make the 16 rows' places differ 4.2 and 4.1, or 8.1 and 2.2.
// W: waves of a block; ROWS: of a tile.
template <typename T, int DP, int W = 4, int ROWS = kTile> struct AskGeo {
  static constexpr int SZ = (int)sizeof(T), E = 16 / SZ;  // E: elements of 16 bytes
  static constexpr int NK = (DP + Wide<T>::W - 1) / Wide<T>::W, ND = DP / 16;  // steps; tiles
  static constexpr int CP = NK <= 1 ? 4 : NK <= 2 ? 8 : NK <= 4 ? 16 : 32;     // chunks of a row
  static constexpr int RB = 16 * CP, TB = ROWS * RB;      // bytes of a row, of a tile
  static constexpr int NP = (TB + 1024 * W - 1) / (1024 * W);  // loads of a tile per wave
  static __device__ __forceinline__ int key(int row) {
    if constexpr (SZ == 4) return CP == 4 ? row >> 2 & 3 : CP == 8 ? row >> 1 & 7 : row & 15;
    return CP == 4 ? 2 * (row >> 2 & 1) : CP == 8 ? 2 * (row >> 1 & 3) : 2 * (row & 7);
  }
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

// The request whose slots hold `slot`, its rows of the side that the slots are of (N of them,
// G times) and of the other one (M); false: none.  Up to 63 requests all offsets come in
// one load of a lane each: a block's start is a chain of loads (offsets, mask, tile), of
// which this leaves out one (20,003 queries of 7 requests over 1,777 states, fp32: 19.0 us for
// the call where it takes 19.3 with the search and what it finds read again).
struct Place {
  int r;
  Range mine, theirs;
};
__device__ __forceinline__ int64_t of_lane(int64_t v, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)v, lane);
  const int hi = __builtin_amdgcn_readlane((int)(v >> 32), lane);
  return (int64_t)((uint64_t)(uint32_t)hi << 32 | lo);
}
__device__ __forceinline__ bool place_of(Place& p, const int64_t* off, int64_t N, const int64_t* other,
                                         int64_t M, int R, int G, int shift, int64_t slot) {
  if (off && R < 64) {
    const int at = lane_id() < R ? lane_id() : R;
    const int64_t x = clamp64(off[at], 0, N), y = clamp64(other[at], 0, M);
    const int n = __popcll(__ballot(lane_id() < R && ((x * G) >> shift) + lane_id() <= slot));
    if (n == 0) return false;
    p.r = n - 1;
    p.mine.b = of_lane(x, n - 1);
    p.mine.e = clamp64(of_lane(x, n), p.mine.b, N);
    p.theirs.b = of_lane(y, n - 1);
    p.theirs.e = clamp64(of_lane(y, n), p.theirs.b, M);
    return true;
  }
  p.r = request_of(off, R, N, G, shift, slot);
  if (p.r < 0) return false;
  p.mine = range_of(off, p.r, N);
  p.theirs = range_of(other, p.r, M);
  return true;
}

// A grid of any number of blocks (HIP takes 2^32 threads of a dimension), and a block's number
// in it: there may be more blocks than were asked for.
constexpr int kGridX = 22;
inline dim3 grid_of(int64_t blocks, int pieces) {
  const int64_t x = (int64_t)1 << kGridX;
  return dim3((uint32_t)(blocks < x ? blocks : x), pieces, (uint32_t)((blocks + x - 1) / x));
}
__device__ __forceinline__ uint32_t block_of() { return (blockIdx.z << kGridX) + blockIdx.x; }

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
// 16 bytes a lane to LDS, one behind the other from dst on (the same in all lanes).
__device__ __forceinline__ void load_lds16(Buffer b, char* dst, int at) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (__attribute__((address_space(3))) void*)dst, 16, at,
                                           0, 0, 0);
}
constexpr int kNowhere = 0x7fffff00;

// Loads of a tile of up to 64 rows into LDS by W waves, 16 bytes a lane, without a
// register between, zeros where rows or columns end.  Offsets within a tile stay below
// 2^31: rows are at most 2^25 bytes apart.
template <typename T, int DP, int W, int ROWS = kTile> struct TileLoad {
  using Gm = AskGeo<T, DP, W, ROWS>;
  int off[Gm::NP];

  // this lane's row and column in load j of its wave
  static __device__ __forceinline__ int row(int j) { return (64 * W * j + (int)threadIdx.x) / Gm::CP; }
  static __device__ __forceinline__ int col(int j) {
    return ((64 * W * j + (int)threadIdx.x) % Gm::CP ^ Gm::key(row(j))) * Gm::E;
  }
  // rows of states, ld elements apart
  __device__ __forceinline__ void states(int64_t ld, int D) {
#pragma unroll
    for (int j = 0; j < Gm::NP; ++j)
      off[j] = col(j) < D ? (row(j) * (int)ld + col(j)) * Gm::SZ : kNowhere;
  }
  // `rows` virtual rows of a request from row `rem` of a query's group on, the last one again
  // behind it
  __device__ __forceinline__ void queries(int64_t ld, int G, int rem, int D, int rows) {
#pragma unroll
    for (int j = 0; j < Gm::NP; ++j) {
      const uint32_t v = rem + (row(j) < rows ? row(j) : rows - 1), i = G == 1 ? v : v / (uint32_t)G, g = v - i * G;
      off[j] = col(j) < D ? (int)(i * (uint32_t)ld + g * D + col(j)) * Gm::SZ : kNowhere;
    }
  }
  __device__ __forceinline__ void load(Buffer b, int j, bool in, char* tile) const {
    const int at = 1024 * (W * j + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    if (Gm::TB % (1024 * W) == 0 || at < Gm::TB) load_lds16(b, tile + at, in ? off[j] : kNowhere);
  }
};

// Tiles of a request's states in LDS: k's, v's behind it, and which of them count (0, or
// -infinity where one is left out, whose rows are zeros: they may hold anything).  Which
// rows are left out is asked for a tile ahead, before its loads are.
template <typename T, int DP, int W> struct StateTiles {
  using Gm = AskGeo<T, DP, W>;
  TileLoad<T, DP, W> k, v;
  const T *K, *V;
  const uint8_t* mask;
  int64_t ldk, ldv, e;
  int D;
  uint8_t keep[Gm::NP], counts;
  float alive;
  __device__ __forceinline__ void init(const AskArgs& a, int h, Range r) {
    K = reinterpret_cast<const T*>(a.k) + (int64_t)h * a.D;
    V = reinterpret_cast<const T*>(a.v) + (int64_t)h * a.D;
    mask = a.mask; ldk = a.ldk; ldv = a.ldv; e = r.e; D = a.D;
    k.states(ldk, D);
    v.states(ldv, D);
    if (mask && r.b < r.e) ask(r.b);
  }
  __device__ __forceinline__ void ask(int64_t p0) {
    const Buffer m = buffer_of(mask + p0, e - p0 < kTile ? e - p0 : kTile);
    counts = __builtin_amdgcn_raw_buffer_load_b8(m, threadIdx.x & 63, 0, 0);
#pragma unroll
    for (int j = 0; j < Gm::NP; ++j) keep[j] = __builtin_amdgcn_raw_buffer_load_b8(m, k.row(j), 0, 0);
  }
  __device__ __forceinline__ void load(int64_t p0, char* tiles) {
    const int rows = e - p0 < kTile ? (int)(e - p0) : kTile;
    const Buffer bk = buffer_of(K + p0 * ldk, ((rows - 1) * ldk + D) * Gm::SZ);
    const Buffer bv = buffer_of(V + p0 * ldv, ((rows - 1) * ldv + D) * Gm::SZ);
    if (!mask) {  // (rows past the end lie past the buffers')
      alive = (int)threadIdx.x < rows ? 0.f : -INFINITY;
#pragma unroll
      for (int j = 0; j < Gm::NP; ++j) {
        k.load(bk, j, true, tiles);
        v.load(bv, j, true, tiles + Gm::TB);
      }
      return;
    }
    alive = counts ? 0.f : -INFINITY;
    bool in[Gm::NP];
#pragma unroll
    for (int j = 0; j < Gm::NP; ++j) in[j] = keep[j];
    if (p0 + kTile < e) ask(p0 + kTile);
#pragma unroll
    for (int j = 0; j < Gm::NP; ++j) {
      k.load(bk, j, in[j], tiles);
      v.load(bv, j, in[j], tiles + Gm::TB);
    }
  }
  __device__ __forceinline__ void put(float* live) {
    if (threadIdx.x < kTile) live[threadIdx.x] = alive;
  }
  // One of a tile's states counts (a tile of none is no work; nor does a query that is NaN
  // make its row NaN where nothing counts).
  __device__ __forceinline__ bool some(const float* live) const {
    return !mask || __any(live[threadIdx.x & 63] == 0.f);
  }
};

// Tiles of ROWS of a request's virtual rows: q's, do's behind it, and their lse (base 2) and
// delta, [2][64] floats, with which rows past the end have weights of 0: they are the last row
// again, whose scores are none that are NaN, where zeros' would be with a state's infinity.
template <typename T, int DP, int W, int ROWS> struct QueryTiles {
  using Gm = AskGeo<T, DP, W, ROWS>;
  TileLoad<T, DP, W, ROWS> q, d;
  const T *Q, *DO;
  const float *lse, *delta;
  int64_t ldq, lddo, Nq;
  int G, D, n;
  float l, de;
  // up to virtual row n of a request that begins at query b
  __device__ __forceinline__ void init(const AskArgs& a, int h, int64_t b, int n_) {
    G = a.Hq / a.Hkv; D = a.D; n = n_; Nq = a.Nq; ldq = a.ldq; lddo = a.lddo;
    Q = reinterpret_cast<const T*>(a.q) + (int64_t)h * G * D + b * ldq;
    DO = reinterpret_cast<const T*>(a.d_o) + (int64_t)h * G * D + b * lddo;
    lse = a.lse + (int64_t)h * G * Nq + b;
    delta = a.delta + (int64_t)h * G * Nq + b;
    if (ROWS % G == 0) places(0, ROWS);
  }
  __device__ __forceinline__ void places(int rem, int rows) {
    q.queries(ldq, G, rem, D, rows);
    d.queries(lddo, G, rem, D, rows);
  }
  __device__ __forceinline__ void load(int v0, char* tiles) {
    const int rows = n - v0 < ROWS ? n - v0 : ROWS;
    const int i0 = G == 1 ? v0 : v0 / G, i1 = G == 1 ? v0 + rows - 1 : (v0 + rows - 1) / G;
    // (tiles do not begin at a query; the last one ends inside)
    if (ROWS % G || rows < ROWS) places(v0 - i0 * G, rows);
    const Buffer bq = buffer_of(Q + i0 * ldq, ((i1 - i0) * ldq + G * D) * Gm::SZ);
    const Buffer bd = buffer_of(DO + i0 * lddo, ((i1 - i0) * lddo + G * D) * Gm::SZ);
#pragma unroll
    for (int j = 0; j < Gm::NP; ++j) {
      q.load(bq, j, true, tiles);
      d.load(bd, j, true, tiles + Gm::TB);
    }
    if (threadIdx.x < kTile) {
      const bool ok = (int)threadIdx.x < rows;
      const uint32_t v = ok ? v0 + threadIdx.x : v0 + rows - 1;
      const uint32_t i = G == 1 ? v : v / (uint32_t)G;
      const int64_t at = (v - i * G) * Nq + i;
      l = lse[at] * kLog2e;
      de = delta[at];
      if (!ok || l == -INFINITY) l = INFINITY;
      if (!ok) de = 0.f;
    }
  }
  __device__ __forceinline__ void put(float* stat) {
    if (threadIdx.x < kTile) {
      stat[threadIdx.x] = l;
      stat[kTile + threadIdx.x] = de;
    }
  }
};

// Every wave's loads into LDS and writes to it have arrived.
__device__ __forceinline__ void tiles_ready() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Reads of a tile's operands: a wide one, lane (r, g) elements of row 16 t + r; and
// columns, lane (r, g) element 16 d + r of rows 16 t + 4 g .. + 3.
template <typename T, int DP> struct TileRead {
  using Gm = AskGeo<T, DP>;
  int wide[Gm::NK], cols[Gm::ND], more[sizeof(T) == 2 ? 1 : 4];
  __device__ __forceinline__ TileRead() {
    const int r = lane_id() & 15, g = lane_id() >> 4;
#pragma unroll
    for (int k = 0; k < Gm::NK; ++k) wide[k] = r * Gm::RB + ((4 * k + g) ^ Gm::key(r)) * 16;
    if constexpr (sizeof(T) == 2) {
      const int row = 4 * g + (r >> 2);
#pragma unroll
      for (int d = 0; d < Gm::ND; ++d)
        cols[d] = row * Gm::RB + ((2 * d + (r >> 1 & 1)) ^ Gm::key(row)) * 16 + 8 * (r & 1);
    } else {  // (a key's upper part is the same for the four rows)
#pragma unroll
      for (int d = 0; d < Gm::ND; ++d) cols[d] = ((d ^ (Gm::key(4 * g) >> 2)) * 4) * 16 + 4 * (r & 3);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        more[i] = (4 * g + i) * Gm::RB + (((r >> 2) ^ Gm::key(4 * g + i)) & 3) * 16;
    }
  }
  __device__ __forceinline__ void rows(WideF<T>& f, const char* tile, int t, int k) const {
    set_wide(f, *reinterpret_cast<const uint4*>(tile + wide[k] + t * 16 * Gm::RB));
  }
  __device__ __forceinline__ void columns(K16<T>& f, const char* tile, int t, int d) const {
    if constexpr (sizeof(T) == 2) {
      ld_tr<T>(f, tile, cols[d], t * 16 * Gm::RB, 0);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        f.v[i] = *reinterpret_cast<const float*>(tile + cols[d] + more[i] + t * 16 * Gm::RB);
    }
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
// Operands that are read together, ahead of their products (pipelined()): as the compiler
// orders them, it reads, waits and multiplies.
template <typename T> struct WidePair {
  WideF<T> a, b;
};
template <typename T> struct ColumnPair {
  K16<T> a, b;
};

// The larger one, NaN where either is (one instruction of three operands; the score of
// a NaN makes its row NaN in any case).
__device__ __forceinline__ float largest(float a, float b) {
  return __builtin_elementwise_maximum(a, b);
}
// Of the four lane groups.
__device__ __forceinline__ float groups_largest(float v) {
  float a = v, b = v;
  lane_swap16(a, b);
  float c = largest(a, b), d = c;
  lane_swap32(c, d);
  return largest(c, d);
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

// Sums over pieces by a block of 256: U groups of threads take every U-th piece and are
// added in a tree (so in the same order every time).  v: this thread's; the first group's
// threads, of P each, get the totals.
template <typename V> __device__ __forceinline__ V add_groups(V v, V* lds, int u, int U, int at, int P) {
  for (int half = U >> 1; half > 0; half >>= 1) {
    __syncthreads();
    if (u >= half && u < 2 * half) lds[(u - half) * P + at] = v;
    __syncthreads();
    if (u < half) v += lds[u * P + at];
  }
  return v;
}

// Of a block's 256 threads; lds: four floats of the call's own.
__device__ __forceinline__ float block_largest(float v, float* lds) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) v = fmaxf(v, __shfl_xor(v, m));
  if (lane_id() == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
}
__device__ __forceinline__ float block_sum(float v, float* lds) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
  if (lane_id() == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}
// Is a row one of a request's?
__device__ __forceinline__ bool asked_for(const AskArgs& a, int64_t row) {
  return !a.q_off || (row >= a.q_off[0] && row < a.q_off[a.R]);
}

// How pieces are joined: up to 8 one behind the other by a thread, many rows to a block
// (U = 0); more by a block for P fours of a row's elements, whose U groups of threads take
// every U-th piece, all loads of a thread on their way together.  us, of calls with 256
// pieces, with a thread for a row's four, a block for a row, and so: 62 queries of 4 heads over
// 181,477 states 160, 41, 39; 4 queries over 60,000 states, 128 wide, fp32: -, 48, 33; one of 8
// heads over 20,000 -, 19, 12.5.
struct Join {
  int P, U;
  dim3 grid;
};
inline Join join_of(const AskArgs& a) {
  const int per = a.D / 4;
  const int64_t rows = a.Nq * a.Hq;
  if (a.S <= 8) return {256 / per, 0, dim3((uint32_t)((rows + 256 / per - 1) / (256 / per)))};
  const int blocks = (per + 7) / 8, P = (per + blocks - 1) / blocks;
  int U = 1;
  while (2 * U * P <= 256 && 2 * U <= a.S) U *= 2;
  return {P, U, dim3((uint32_t)rows, blocks)};
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
