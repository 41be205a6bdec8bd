// LDS tiles and packed-sequence lookup shared by the sequence mixers
// (packed attention and linear attention).
//
// A tile is ROWS rows of one head, [ROWS][DH] in its natural layout, filled by
// direct global->LDS loads of 16-byte chunks.  Chunk c of row r lies at chunk
// c ^ swz(r) of its row.  The 64 LDS banks hold 256 bytes, and 16 lanes of a
// 16-byte read, or 32 lanes of a transposing 8-byte read, are served at once:
//   - a row read (16 lanes, 16 consecutive rows, one chunk) needs the 16 rows
//     on 16 distinct 16-byte bank groups;
//   - a transposing read (8 consecutive rows from a multiple of 8, two
//     adjacent chunks) needs them on 8 distinct pairs of groups.
// With NCH chunks per row, 16 / NCH rows fill the banks once (none left to
// permute for NCH >= 16), so swz orders the remaining row bits such that the
// next row bit goes to the highest chunk bit.
#pragma once

#include <utility>

#include "common.h"

namespace bcmt {

// Results of the inline-assembly LDS reads below, in the pieces in which the
// reads return them.  Nothing may touch a piece before lds_tr_wait(); take()
// ties every piece to that wait and only then joins them, so that no register
// copy can come before the data.
template <typename T> struct RowRaw;
template <> struct RowRaw<bf16> { bf16x8 v; };
template <> struct RowRaw<float> { f32x4 a, b; };
template <typename T> struct ColRaw;
template <> struct ColRaw<bf16> { bf16x4 a, b; };
template <> struct ColRaw<float> { float e[8]; };

__device__ __forceinline__ bf16x8 take(RowRaw<bf16>& r) {
  lds_tr_bind(r.v);
  return r.v;
}
__device__ __forceinline__ f32x8 take(RowRaw<float>& r) {
  lds_tr_bind(r.a);
  lds_tr_bind(r.b);
  return f32x8{r.a[0], r.a[1], r.a[2], r.a[3], r.b[0], r.b[1], r.b[2], r.b[3]};
}
__device__ __forceinline__ bf16x8 take(ColRaw<bf16>& r) {
  lds_tr_bind(r.a);
  lds_tr_bind(r.b);
  return bf16x8{r.a[0], r.a[1], r.a[2], r.a[3], r.b[0], r.b[1], r.b[2], r.b[3]};
}
__device__ __forceinline__ f32x8 take(ColRaw<float>& r) {
#pragma unroll
  for (int i = 0; i < 8; ++i) lds_tr_bind(r.e[i]);
  return f32x8{r.e[0], r.e[1], r.e[2], r.e[3], r.e[4], r.e[5], r.e[6], r.e[7]};
}

// The addresses of a lane's column operands: one with the transposing reads,
// one for each of four rows otherwise.
template <typename T> struct ColBase { unsigned a[sizeof(T) == 2 ? 1 : 4]; };

template <class P>
__device__ __forceinline__ unsigned lds_addr(const P* p) {
  return (unsigned)(uintptr_t)((__attribute__((address_space(3))) P*)(p));
}

// f(0), ..., f(N - 1) with the index as a constant.
template <class Fn, int... I>
__device__ __forceinline__ void each_(Fn& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class Fn>
__device__ __forceinline__ void each(Fn f) {
  each_(f, std::make_integer_sequence<int, N>{});
}

constexpr int64_t kNearLd = 1 << 24;

template <typename T, int DH>
struct Tile {
  static constexpr int CH = 16 / (int)sizeof(T);  // elements of a chunk
  static constexpr int NCH = DH / CH;             // chunks of a row: 2 .. 32
  __device__ static __forceinline__ int swz(int r) {
    if constexpr (NCH >= 16) return ((r & 7) << 1) | ((r >> 3) & 1);
    else if constexpr (NCH == 8) return ((r >> 3) & 1) | (r & 2) | ((r ^ (r >> 1)) & 4);
    else if constexpr (NCH == 4) return ((r >> 1) & 2) | ((r >> 3) & 1);
    else return (r >> 3) & 1;
  }
  __device__ static __forceinline__ int off(int r, int c) {
    return r * DH + (((c / CH) ^ swz(r)) * CH) + c % CH;
  }
  // One wave's instruction i of the loads of a tile: 64 chunks.  Row r of the
  // tile is row min(r0 + r, rlast) of src: a clamped row is never used
  // unmasked.
  __device__ static __forceinline__ void issue(const T* src, int64_t ld, int r0, int rlast, T* t,
                                               int i, int lane) {
    const int id = i * 64 + lane;
    const int row = id / NCH, pos = id % NCH;
    const int grow = min(r0 + row, rlast);
    __builtin_amdgcn_global_load_lds(src + (int64_t)grow * ld + ((pos ^ swz(row)) * CH),
                                     (lds_void_t*)(t + i * 64 * CH), 16, 0, 0);
  }
  // The same loads of whole tiles with the lane's part of the address formed once
  // (lane_off: bytes from the tile's lowest row, whose address is the wave's): one
  // vector instruction a load instead of ten.  Row strides up to kNearLd, so that a
  // tile's rows are within 2^32 bytes.
  __device__ static __forceinline__ unsigned lane_off(int64_t ld, int i, int lane) {
    const int id = i * 64 + lane, row = id / NCH, pos = id % NCH;
    return (unsigned)(row * (unsigned)ld + (pos ^ swz(row)) * CH) * (unsigned)sizeof(T);
  }
  __device__ static __forceinline__ void issue_near(const T* lowest, unsigned off, T* t, int i) {
    __builtin_amdgcn_global_load_lds((const char*)lowest + off, (lds_void_t*)(t + i * 64 * CH), 16, 0,
                                     0);
  }
  // The reads of a tile go by a byte address of the lane, formed once, an
  // exclusive or for the columns (a row begins at a multiple of its size, so
  // that the or only permutes its chunks) and a constant offset for the rows.
  //
  // Row operand: elements 32 DS + 8g .. + 7, g = lane / 16, of row r + R; zero
  // where a row is narrower than a product's 32 columns.  Float32 rows of 16 take
  // elements 4g .. + 3 instead, and half of the product's instructions (mma).
  static constexpr bool SHORT = sizeof(T) == 4 && DH == 16;
  __device__ static __forceinline__ int row_col(int lane) { return (lane >> 4) * (SHORT ? 4 : 8); }
  __device__ static __forceinline__ unsigned row_base(const T* t, int r, int lane) {
    const int c = row_col(lane);
    return lds_addr(t + off(r, c < DH ? c : 0));
  }
  // The same of a row in global memory (zero if !ok).
  __device__ static __forceinline__ typename Frag<T>::type row_global(const T* p, int ds, int lane,
                                                                      bool ok) {
    typedef typename Frag<T>::type F;
    const int c = ds * 32 + row_col(lane);
    if (!ok || c >= DH) return F{};
    if constexpr (SHORT) {
      const f32x4 x = load4f(p + c);
      return F{x[0], x[1], x[2], x[3], 0.f, 0.f, 0.f, 0.f};
    } else {
      return load_frag(p + c);
    }
  }
  // Product of two row operands.
  __device__ static __forceinline__ f32x4 mma(const typename Frag<T>::type& a,
                                              const typename Frag<T>::type& b, f32x4 c) {
    if constexpr (SHORT) {
#pragma unroll
      for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
      return c;
    } else {
      return mma16(a, b, c);
    }
  }
  template <int DS, int R>
  __device__ static __forceinline__ RowRaw<T> row_at(unsigned a) {
    constexpr int O = R * DH * (int)sizeof(T);
    if constexpr (sizeof(T) == 2) return {lds_read_b128_at<O>(a ^ (DS * 64))};
    else if constexpr (SHORT) return {lds_read_f32x4_at<O>(a), f32x4{0.f, 0.f, 0.f, 0.f}};
    else return {lds_read_f32x4_at<O>(a ^ (DS * 128)), lds_read_f32x4_at<O>(a ^ (DS * 128 + 16))};
  }
  __device__ static __forceinline__ typename Frag<T>::type take_row(RowRaw<T>& r, int lane) {
    typedef typename Frag<T>::type F;
    const F f = take(r);
    return DH >= 32 || SHORT || (lane >> 4) * 8 < DH ? f : F{};
  }
  // Column operand: column 16 JJ + lane % 16 of rows B0 + 4g .. + 3 and
  // B1 + 4g .. + 3: the order in which two 16-row result tiles hold their rows.
  __device__ static __forceinline__ ColBase<T> col_base(const T* t, int lane) {
    const int g = lane >> 4, i = lane & 15;
    if constexpr (sizeof(T) == 2) {
      return {{lds_addr(t + off(4 * g + (i >> 2), (i & 3) << 2))}};
    } else {
      ColBase<T> r;
#pragma unroll
      for (int e = 0; e < 4; ++e) r.a[e] = lds_addr(t + off(4 * g + e, i));
      return r;
    }
  }
  template <int JJ, int B0, int B1>
  __device__ static __forceinline__ ColRaw<T> col_at(const ColBase<T>& b, unsigned add) {
    constexpr int O0 = B0 * DH * (int)sizeof(T), O1 = B1 * DH * (int)sizeof(T);
    if constexpr (sizeof(T) == 2) {
      const unsigned a = (b.a[0] ^ (JJ * 32)) + add;
      return {lds_read_tr_at<O0>(a), lds_read_tr_at<O1>(a)};
    } else {
      ColRaw<T> r;
      each<4>([&](auto e) {
        const unsigned a = (b.a[e] ^ (JJ * 64)) + add;
        r.e[e] = lds_read_f32_at<O0>(a);
        r.e[4 + e] = lds_read_f32_at<O1>(a);
      });
      return r;
    }
  }
};

// The wave's index as a scalar.  Branches on it must be scalar branches: a
// matrix instruction ignores the lane mask, so in a block that is skipped by
// masking every lane off it would still write its result.
__device__ __forceinline__ int wave_index() {
  return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
}
// Waits here for a value loaded from global memory.  The compiler does not see
// the waits of vm_wait(): a value still in flight where a loop begins would be
// waited for inside the loop, together with every tile requested since.
template <class V>
__device__ __forceinline__ void settle(V& v) {
  asm volatile("" : "+v"(v));
}

// Workgroup barrier without the vmcnt drain of __syncthreads(): direct loads
// stay in flight, and no memory access moves across it.
__device__ __forceinline__ void wg_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
template <int N>
__device__ __forceinline__ void vm_wait() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Sequences are rows [cu[s], cu[s + 1]) of the packed arrays, cut into tiles of
// TILE rows from their own start.  Slot x of total / TILE + nseq slots stands
// for tile x - first(s) of the last sequence s with first(s) <= x, where
// first(s) = cu[s] / TILE + s: sequence s has cu[s+1] / TILE - cu[s] / TILE + 1
// >= ceil(length / TILE) slots, and a slot behind the sequence's end is empty.
// No host copy of cu and no table is needed.  Offsets outside [0, total] or out
// of order are clamped, so that no row outside the arrays is ever addressed.
// Called by whole waves; 64 sequences per search step.
struct SeqTile {
  int seq, begin, end, tile;  // rows [begin, end) of the sequence; tile index
};
__device__ __forceinline__ SeqTile find_tile(const int* __restrict__ cu, int nseq, int total,
                                             int TILE, int slot) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = nseq;
  while (n > 1) {
    const int st = (n + 63) / 64;
    const int s = lo + lane * st;
    const bool le = lane * st < n && min(max(cu[s < lo + n ? s : lo], 0), total) / TILE + s <= slot;
    const int c = max((int)__popcll(__ballot(le)), 1) - 1;
    lo += c * st;
    n = min(st, n - c * st);
  }
  SeqTile r;
  r.seq = __builtin_amdgcn_readfirstlane(lo);
  r.begin = __builtin_amdgcn_readfirstlane(min(max(cu[r.seq], 0), total));
  r.end = __builtin_amdgcn_readfirstlane(min(max(cu[r.seq + 1], r.begin), total));
  r.tile = slot - (r.begin / TILE + r.seq);
  return r;
}

// Item x of all tiles of all sequences, the ones with the most work first: in
// descending order of their index (LAST: of the tiles behind them in their
// sequence), so that no long tile starts when the chip is nearly done.  f(t) = sum
// over sequences of max(0, tiles - t) items have index >= t; the largest t with
// f(t) > x is the item's, and among the sequences that have it, x - f(t + 1) counts.
// Up to 64 sequences, one a lane; more are walked slot by slot, which costs most
// where one is long: sequences of 4096 and 63 times 128, 16 heads of 128 on 2, forward
// 121 us and with an empty 65th 170 (12 heads of 64 on 4: 94 and 114); 64 of 16 to
// 1024, gradients 844 and 1122 (312 and 376).  Items from f(0) on are empty (tile < 0).
template <bool LAST>
__device__ __forceinline__ SeqTile find_item(const int* __restrict__ cu, int nseq, int total,
                                             int TILE, int x) {
  if (nseq > 64) return find_tile(cu, nseq, total, TILE, LAST ? x : total / TILE + nseq - 1 - x);
  const int lane = threadIdx.x & 63;
  int begin = 0, end = 0;
  if (lane < nseq) {
    begin = min(max(cu[lane], 0), total);
    end = min(max(cu[lane + 1], begin), total);
  }
  const int n = (end - begin + TILE - 1) / TILE;
  auto f = [&](int t) {  // (at most total / TILE + 64 tiles, below 2^24: exact in float32)
    return (int)wave_sum((float)max(0, n - t));
  };
  int lo = 0, hi = (total + TILE - 1) / TILE;  // f(hi) = 0
  int flo = f(0);
  SeqTile r{0, 0, 0, -1};
  if (x >= flo) return r;
  int fhi = 0;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2, fm = f(mid);
    if (fm > x) {
      lo = mid;
    } else {
      hi = mid;
      fhi = fm;
    }
  }
  const unsigned long long has = __ballot(n > lo);
  const bool mine = n > lo && (int)__popcll(has & ((1ull << lane) - 1)) == x - fhi;
  const int s = __builtin_ctzll(__ballot(mine) | 1ull << 63);  // (none: offsets out of order)
  r.seq = s;
  r.begin = __builtin_amdgcn_readlane(begin, s);
  r.end = __builtin_amdgcn_readlane(end, s);
  r.tile = LAST ? __builtin_amdgcn_readlane(n, s) - 1 - lo : lo;
  return r;
}

// Nonzero if an element is infinite or NaN (its exponent bits are all ones).
__device__ __forceinline__ unsigned nonfinite_bits(const bf16x8& v) {
  typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
  const u32x4 x = __builtin_bit_cast(u32x4, v);
  unsigned b = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) b |= ((x[i] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
  return b;
}
__device__ __forceinline__ unsigned nonfinite_bits(const f32x8& v) {
  typedef unsigned u32x8 __attribute__((ext_vector_type(8)));
  const u32x8 x = __builtin_bit_cast(u32x8, v);
  unsigned b = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) b |= ((x[i] & 0x7f800000u) + 0x00800000u) & 0x80000000u;
  return b;
}
}  // namespace bcmt

// Dispatch of a launcher template over the types and head widths.
#define BY_TYPE_AND_WIDTH(fn, dt, dh, ...)                   \
  do {                                                       \
    if ((dt) == DType::BF16) {                               \
      switch (dh) {                                          \
        case 16: return fn<bf16, 16>(__VA_ARGS__);           \
        case 32: return fn<bf16, 32>(__VA_ARGS__);           \
        case 64: return fn<bf16, 64>(__VA_ARGS__);           \
        default: return fn<bf16, 128>(__VA_ARGS__);          \
      }                                                      \
    }                                                        \
    switch (dh) {                                            \
      case 16: return fn<float, 16>(__VA_ARGS__);            \
      case 32: return fn<float, 32>(__VA_ARGS__);            \
      case 64: return fn<float, 64>(__VA_ARGS__);            \
      default: return fn<float, 128>(__VA_ARGS__);           \
    }                                                        \
  } while (0)

