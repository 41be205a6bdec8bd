// Linear attention with one decay per head over packed sequences.
//
//   S_t = g S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t
// Chunked form, for a chunk of C rows with local index i = 0 .. C-1 and the
// state S before it:
//   o_i = scale (sum_{j <= i} g^(i-j) (q_i . k_j) v_j  +  g^(i+1) S^T q_i)
//   S' = g^C S + sum_j g^(C-1-j) k_j v_j^T
// The gradients are the same operator.  With R the gradient of the state
// after a chunk (R' the one of the state before it):
//   dq_i = scale (sum_{j <= i} g^(i-j) (do_i . v_j) k_j + g^(i+1) S do_i)
//   dk_j = scale sum_{i >= j} g^(i-j) (v_j . do_i) q_i + g^(C-1-j) R v_j
//   dv_j = scale sum_{i >= j} g^(i-j) (k_j . q_i) do_i + g^(C-1-j) R^T k_j
//   R' = g^C R + scale sum_i g^(i+1) q_i do_i^T
// so one kernel takes rows a (queries), b (keys), c (values) of any of the
// three and a direction: in reverse, the local index i' = C-1-i makes the state
// terms g^i' and g^(C-i') instead of g^(i+1) and g^(C-1-j).
//
// A workgroup owns one head of one segment of a sequence and walks its chunks
// of 64 rows in order.  Wave w owns columns 16w .. 16w+15 of the value width
// and keeps its part of the state, [DH][16] in float32, in registers in the
// layout of a product's result, which is also the layout of a product's first
// operand: the state never leaves the registers between chunks.  The masked,
// decayed scores of a chunk are shared through LDS.
//
// The sum of a state takes its weighted rows g^n c_j in three bf16 parts
// (24 bits) where the float32 state can be an output, so that it loses nothing to
// bf16 products, and in two (16 bits) where only bf16 outputs read it.  Decayed
// scores and the state as operands of a bf16 output are rounded to bf16 once, since
// the matrix instructions take no other: each at most 2^-8 of the sum of magnitudes
// of the output, which where terms cancel is more than the output's own rounding.
// With that an error of 2.3e-3 in the 2-norm, 1.7e-3 by the output's rounding alone.
//
// Long sequences are cut into segments of `seg` rows that run side by side:
// their own sums first (lin_kernel<..., STATE>), then a scan over a sequence's
// segments, which leaves the state at every boundary between two segments.
// Boundary k >= 1 of a sequence that begins at row b is entry b / seg + k of the
// array: distinct for all boundaries, at most total / seg, and sequences of one
// segment have none.
#include "kernels.h"
#include "mixer_tile.h"

namespace bcmt {
namespace {

constexpr int kC = 64;  // rows of a chunk

__device__ __forceinline__ float powg(float lg2, int e) {  // g^e; 0^0 = 1
  return e == 0 ? 1.f : exp2_fast(lg2 * (float)e);
}

// x as a sum of operands of the type: one in float32, three in bf16 (24 bits; the
// third only if `fine`).
template <typename T> struct Parts;
template <> struct Parts<float> { static constexpr int N = 1; };
template <> struct Parts<bf16> { static constexpr int N = 3; };

__device__ __forceinline__ void split(const float (&x)[8], f32x8 (&p)[1], bool) {
  p[0] = f32x8{x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ void split(const float (&x)[8], bf16x8 (&p)[3], bool fine) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    p[0][e] = (bf16)x[e];
    r[e] = x[e] - (float)p[0][e];
    p[1][e] = (bf16)r[e];
  }
  if (fine) {
#pragma unroll
    for (int e = 0; e < 8; ++e) p[2][e] = (bf16)(r[e] - (float)p[1][e]);
  }
}

// Elements 4g .. + 3 and 16 + 4g .. + 3 of the 32 from c0 of a row (one half if
// the row has 16): the order in which two state tiles hold them.
template <typename T> struct HalfRaw;
template <> struct HalfRaw<bf16> { bf16x4 a, b; };
template <> struct HalfRaw<float> { f32x4 a, b; };
template <typename T, int DH>
__device__ __forceinline__ unsigned half_base(const T* t, int r, int lane) {
  return lds_addr(t + Tile<T, DH>::off(r, 4 * (lane >> 4)));
}
template <typename T, int DH, int KS, int R>
__device__ __forceinline__ HalfRaw<T> half_at(unsigned a) {
  constexpr int O = R * DH * (int)sizeof(T), C = 32 * KS * (int)sizeof(T);
  constexpr int D = DH >= 32 ? 16 * (int)sizeof(T) : 0;
  if constexpr (sizeof(T) == 2) return {lds_read_b64_at<O>(a ^ C), lds_read_b64_at<O>(a ^ (C + D))};
  else return {lds_read_f32x4_at<O>(a ^ C), lds_read_f32x4_at<O>(a ^ (C + D))};
}
template <typename T, int DH>
__device__ __forceinline__ typename Frag<T>::type take_row8p(HalfRaw<T>& r) {
  lds_tr_bind(r.a);
  lds_tr_bind(r.b);
  const auto b = DH >= 32 ? r.b : decltype(r.b){};
  return {r.a[0], r.a[1], r.a[2], r.a[3], b[0], b[1], b[2], b[3]};
}

// state += (rows a)^T (weighted rows c): this wave's 16 columns, the 64 rows
// of a chunk.  w: weights of the 8 rows lane / 16 holds in each half chunk.
template <typename T, int DH, int TB_ = DH / 16>
__device__ __forceinline__ void add_outer(f32x4 (&S)[DH / 16], const ColBase<T>& abase, unsigned add,
                                          const typename Frag<T>::type (&cf)[2],
                                          const float (&w)[2][8], bool fine) {
  typedef typename Frag<T>::type F;
  constexpr int NP = Parts<T>::N, NT = DH / 16, TB = sizeof(T) == 2 || NT < 2 ? (TB_ < NT ? TB_ : NT) : 2;
  each<2>([&](auto us) __attribute__((always_inline)) {
    each<NT / TB>([&](auto tb) __attribute__((always_inline)) {
      ColRaw<T> ar[TB];
      each<TB>([&](auto t) {
        ar[t] = Tile<T, DH>::template col_at<tb * TB + t, us * 32, us * 32 + 16>(abase, add);
      });
      F p[NP];
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = w[us][e] * to_f32(cf[us][e]);
      split(x, p, fine);
      lds_tr_wait();
      F a[TB];
#pragma unroll
      for (int t = 0; t < TB; ++t) a[t] = take(ar[t]);
      if (NP == 3 && fine) {
#pragma unroll
        for (int t = 0; t < TB; ++t) S[tb * TB + t] = mma16(a[t], p[NP - 1], S[tb * TB + t]);
      }
#pragma unroll
      for (int n = NP == 3 ? 1 : 0; n >= 0; --n)
#pragma unroll
        for (int t = 0; t < TB; ++t) S[tb * TB + t] = mma16(a[t], p[n], S[tb * TB + t]);
    });
  });
}

// The wave's part of a [DH][DH] state in memory: rows 16t + 4g + r, column col.
template <int NT>
__device__ __forceinline__ void load_state(f32x4 (&S)[NT], const float* p, int sr, int sc, int col,
                                           int lg) {
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) S[t][r] = p[(16 * t + 4 * lg + r) * sr + col * sc];
}
template <int NT>
__device__ __forceinline__ void store_state(const f32x4 (&S)[NT], float* p, int sr, int sc, int col,
                                            int lg) {
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) p[(16 * t + 4 * lg + r) * sr + col * sc] = S[t][r];
}

struct LinSeg {
  int seq, n, t0, len, row0;  // sequence; its length; segment [t0, t0 + len); first row
  int bound;                  // entry of the boundary before it; the one after it follows
  int first;                  // entry of the sequence's first boundary
  bool last;                  // the sequence's last segment
};
// Segment of slot x (segments are tiles of `seg` rows from the sequence's
// start); len < 0: an empty slot.  An empty sequence has one segment of no rows.
__device__ __forceinline__ LinSeg lin_segment(const int* cu, int nseq, int total, int seg, int slot) {
  const SeqTile st = find_tile(cu, nseq, total, seg, slot);
  LinSeg r;
  r.seq = st.seq;
  r.n = st.end - st.begin;
  r.t0 = st.tile * seg;
  r.len = min(seg, r.n - r.t0);
  if (st.tile < 0 || (st.tile > 0 && r.len <= 0)) r.len = -1;
  r.row0 = st.begin + r.t0;
  r.bound = st.begin / seg + st.tile;
  r.first = st.begin / seg + 1;
  r.last = r.t0 + seg >= r.n;
  return r;
}

// A workgroup takes as many heads side by side as make 256 bytes of a row, so that
// memory sees that much of a row at once: 131072 rows of 16 heads of 64 take 362 us
// with two heads to a workgroup, 431 with one (whose passes run at 3.9 TB/s; the same
// data as rows of one or two heads at 4.9).
template <typename T, int DH> constexpr int lin_heads = DH * sizeof(T) < 256 ? 256 / (DH * sizeof(T)) : 1;

// Buffers of the chunks' tiles: what the LDS of a CU holds besides the scores, up to
// three (two and three measured alike where both fit), and two for the sums, of which
// a CU then holds two workgroups.
template <typename T, int DH>
constexpr int lin_buffers(int tiles, bool state) {
  const int set = tiles * kC * DH * (int)sizeof(T) * lin_heads<T, DH>;
  const int scores = state ? 0 : kC * kC * (int)sizeof(T) * lin_heads<T, DH>;
  const int n = (163840 - scores) / set;
  return state ? 2 : n > 3 ? 3 : n < 1 ? 1 : n;
}

// ------------------------------------------------------------------ the operator
// REV: rows in reverse.  STATE: only the segment's own sum of states.  SUM: the
// gradient's dq pass, which also leaves the segment's own sum of R, scale sum_i
// g^(i+1) q_i do_i^T, for the reverse pass (its rows a are do; q is a fourth tile):
// the local index runs forward, so the sum needs no decay, only falling weights.

template <typename T, int DH, bool REV, bool STATE, bool SUM>
__global__ __launch_bounds__((DH * 4 * lin_heads<T, DH>), sizeof(T) == 2 ? (STATE && DH < 128 ? 4 : 2) : 1)
void lin_kernel(LinPass a) {
  typedef typename Frag<T>::type F;
  typedef Tile<T, DH> TL;
  typedef Tile<T, kC> TP;
  constexpr int NW = DH / 16, NT = DH / 16, KS = DH >= 32 ? DH / 32 : 1;
  constexpr int FIRST = STATE ? 1 : 0;  // tiles a, b, c: the sum needs b and c
  constexpr int TILES = SUM ? 4 : 3 - FIRST;
  constexpr int HP = lin_heads<T, DH>, NB = lin_buffers<T, DH>(TILES, STATE);
  constexpr int NI = TL::NCH / NW;  // loads of a tile by each wave
  __shared__ __attribute__((aligned(1024))) T lds_all[HP][NB][TILES][kC * DH];
  __shared__ __attribute__((aligned(1024))) T P_all[HP][STATE ? 16 : kC * kC];
  // NW waves a head; a head behind the last one repeats it and writes nothing
  const int lane = threadIdx.x & 63, wave = wave_index() % NW, hw = wave_index() / NW;
  const int lr = lane & 15, lg = lane >> 4;
  const int HG = (a.H + HP - 1) / HP, hx = (int)(blockIdx.x % HG) * HP + hw;
  const bool alive = hx < a.H;
  const int h = alive ? hx : a.H - 1;
  T(*lds)[TILES][kC * DH] = lds_all[hw];
  T* P = P_all[hw];
  const LinSeg sg = lin_segment(a.cu, a.nseq, a.total, a.seg, blockIdx.x / HG);
  if (sg.len < 0) return;
  // the sum of a segment that no other follows is not needed
  if (STATE && (REV ? sg.t0 == 0 : sg.last)) return;
  const float lg2 = log2f(a.gamma[h]);
  const int col = wave * 16 + lr;

  f32x4 S[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) S[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int64_t sq = ((int64_t)sg.seq * a.H + h) * DH * DH;
  const int64_t dd = (int64_t)a.H * DH * DH;
  float* bs = a.seg_state + sg.bound * dd + (int64_t)h * DH * DH;  // the boundary before; + dd: after
  if (!STATE) {
    if (REV ? !sg.last : sg.t0 > 0) load_state<NT>(S, REV ? bs + dd : bs, a.sr, a.sc, col, lg);
    else if (a.given && !(REV ? sg.t0 == 0 : sg.last))
      load_state<NT>(S, a.given + sg.first * dd + (int64_t)h * DH * DH, a.sr, a.sc, col, lg);
    else if (a.s_in) load_state<NT>(S, a.s_in + sq, a.sr, a.sc, col, lg);
  }
  const int nc = (sg.len + kC - 1) / kC;
  const int64_t r0 = REV ? sg.row0 + sg.len - 1 : sg.row0;
  const int64_t la = REV ? -a.lda : a.lda, lb = REV ? -a.ldb : a.ldb, lc = REV ? -a.ldc : a.ldc;
  const T* A = STATE ? nullptr : (const T*)a.a + r0 * a.lda + h * DH;
  const T* B = (const T*)a.b + r0 * a.ldb + h * DH;
  const T* Cc = (const T*)a.c + r0 * a.ldc + h * DH;
  const T* Q = SUM ? (const T*)a.q + r0 * a.ldq + h * DH : nullptr;
  auto issue = [=](int c, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int ti = wave * NI + i;
      if (!STATE) TL::issue(A, la, c * kC, sg.len - 1, lds[buf][0], ti, lane);
      TL::issue(B, lb, c * kC, sg.len - 1, lds[buf][1 - FIRST], ti, lane);
      TL::issue(Cc, lc, c * kC, sg.len - 1, lds[buf][2 - FIRST], ti, lane);
      if (SUM) TL::issue(Q, a.ldq, c * kC, sg.len - 1, lds[buf][TILES - 1], ti, lane);
    }
  };
  // g^(64 - 1 - j) (forward) or g^(64 - j) (reverse) for the rows this lane
  // holds in each half chunk; the row factors of the state's term
  constexpr int EI = REV ? 0 : 1, EU = REV ? 1 : 0;
  float w[2][8], fi[4];
  auto weights = [&](int len) __attribute__((always_inline)) {
#pragma unroll
    for (int us = 0; us < 2; ++us)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int j = us * 32 + (e < 4 ? 4 * lg + e : 12 + 4 * lg + e);
        w[us][e] = j < len ? a.s_upd * powg(lg2, len - 1 - j + EU) : 0.f;
      }
  };
  weights(kC);
#pragma unroll
  for (int ib = 0; ib < 4; ++ib) fi[ib] = a.s_inter * powg(lg2, ib * 16 + lr + EI);
  const float gC = powg(lg2, kC);

  // The scores of a chunk: 16 x 16 blocks (ib, jb), jb <= ib, and the zero blocks
  // (0, 1) and (2, 3) that complete the half chunks beside the diagonal, dealt to
  // the waves by diagonals, so that a lane's decay factors stay in registers.  Row
  // i of P holds the keys of a half chunk in the order of Tile::col_at.
  constexpr int NR = STATE ? 1 : (12 + NW - 1) / NW;
  float fac[NR][4];
  unsigned ra[NR], rb[NR];
  int at[NR];
  if constexpr (!STATE) {
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int b = n * NW + wave;
      // diagonals 0 (4 blocks), 1 (3), 3 (1), 2 (2), then the zeros
      const int d = b < 4 ? 0 : b < 7 ? 1 : b < 8 ? 3 : 2;
      const int ib = b < 4 ? b : b < 7 ? b - 3 : b < 8 ? 3 : b < 10 ? b - 6 : (b - 10) * 2;
      const int jb = b < 10 ? ib - d : ib + 1;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int lag = 16 * d + lr - 4 * lg - r;
        fac[n][r] = lag >= 0 ? a.s_intra * powg(lg2, lag) : 0.f;
      }
      ra[n] = TL::row_base(lds[0][0], (ib & 3) * 16 + lr, lane);
      rb[n] = TL::row_base(lds[0][1], (jb & 3) * 16 + lr, lane);
      at[n] = TP::off((ib & 3) * 16 + lr, ((jb >> 1) & 1) * 32 + 8 * lg + 4 * (jb & 1));
    }
  }
  const ColBase<T> bcol = TL::col_base(lds[0][1 - FIRST], lane);
  ColBase<T> ccol = TL::col_base(lds[0][2 - FIRST], lane);  // this wave's columns
  for (auto& x : ccol.a) x ^= wave * 16 * (int)sizeof(T);
  const unsigned half = half_base<T, DH>(lds[0][0], lr, lane);
  const unsigned prow = TP::row_base(P, lr, lane);
  constexpr unsigned BUF = TILES * kC * DH * sizeof(T);
  // SUM: q's columns, do's columns of this wave; R's part, its weights, g^(64 c)
  const ColBase<T> qcol = TL::col_base(lds[0][TILES - 1], lane);
  ColBase<T> dcol = TL::col_base(lds[0][0], lane);
  for (auto& x : dcol.a) x ^= wave * 16 * (int)sizeof(T);
  f32x4 R[SUM ? NT : 1];
  float wr[2][8], gc = 1.f;
  if constexpr (SUM) {
#pragma unroll
    for (int t = 0; t < NT; ++t) R[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int us = 0; us < 2; ++us)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        wr[us][e] = a.s_sum * powg(lg2, us * 32 + (e < 4 ? 4 * lg + e : 12 + 4 * lg + e) + 1);
  }
#pragma unroll
  for (int i = 0; i < NB - 1; ++i)
    if (i < nc) issue(i, i);
#pragma unroll
  for (int t = 0; t < NT; ++t) settle(S[t]);
  constexpr int AHEAD = NB > 2 ? (NB - 2) * TILES * NI : 0;  // loads behind the next chunk's
  if (NB - 1 <= nc) vm_wait<AHEAD>();
  else vm_wait<0>();
  int buf = 0, next = NB - 1;
  for (int c = 0; c < nc; ++c) {
    wg_barrier();  // this chunk's tiles are there; every wave is done with the last chunk
    if (NB > 1) {
      if (c + NB - 1 < nc) issue(c + NB - 1, next);
    } else {
      issue(c, 0);
      vm_wait<0>();
      wg_barrier();
    }
    const unsigned ba = buf * BUF;
    const int len = min(kC, sg.len - c * kC);
    f32x4 oa[4];
    F cf[2];
    if constexpr (!STATE) {
      each<NR>([&](auto n) __attribute__((always_inline)) {
        if (n * NW + wave >= 12) return;
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
        if (n * NW + wave < 10) {
          RowRaw<T> br[KS], ar[KS];
          each<KS>([&](auto ds) {
            br[ds] = TL::template row_at<ds, 0>(rb[n] + ba);
            ar[ds] = TL::template row_at<ds, 0>(ra[n] + ba);
          });
          lds_tr_wait();
#pragma unroll
          for (int ds = 0; ds < KS; ++ds) {
            const F bf = TL::take_row(br[ds], lane);
            s = TL::mma(bf, TL::take_row(ar[ds], lane), s);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) s[r] = fac[n][r] == 0.f ? 0.f : s[r] * fac[n][r];
        }
        store4(P + at[n], s[0], s[1], s[2], s[3]);
      });
      // the state's term, while the scores arrive
#pragma unroll
      for (int ib = 0; ib < 4; ++ib) oa[ib] = f32x4{0.f, 0.f, 0.f, 0.f};
      const unsigned ha = half + ba;
      each<KS>([&](auto ks) __attribute__((always_inline)) {
        const F sf = frag_from<T>(S[2 * ks], DH >= 32 ? S[2 * ks + (DH >= 32)] : f32x4{});
        HalfRaw<T> qr[4];
        each<4>([&](auto ib) { qr[ib] = half_at<T, DH, ks, ib * 16>(ha); });
        lds_tr_wait();
#pragma unroll
        for (int ib = 0; ib < 4; ++ib) oa[ib] = mma16(sf, take_row8p<T, DH>(qr[ib]), oa[ib]);
      });
#pragma unroll
      for (int ib = 0; ib < 4; ++ib) oa[ib] *= fi[ib];
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the scores are written
      wg_barrier();
    }
    ColRaw<T> cr[2];
    each<2>([&](auto us) { cr[us] = TL::template col_at<0, us * 32, us * 32 + 16>(ccol, ba); });
    lds_tr_wait();
#pragma unroll
    for (int us = 0; us < 2; ++us) cf[us] = take(cr[us]);
    if constexpr (!STATE) {
      // A value that is not finite must not reach the rows before it through
      // 0 * inf: such columns are summed row by row.
      if (__ballot((nonfinite_bits(cf[0]) | nonfinite_bits(cf[1])) != 0) == 0) {
        each<4>([&](auto ib) __attribute__((always_inline)) {
          constexpr int NU = ib / 2 + 1;
          RowRaw<T> pr[NU];
          each<NU>([&](auto us) { pr[us] = TP::template row_at<us, ib * 16>(prow); });
          lds_tr_wait();
#pragma unroll
          for (int us = 0; us < NU; ++us) oa[ib] = mma16(cf[us], take(pr[us]), oa[ib]);
        });
      } else {
#pragma unroll
        for (int ib = 0; ib < 4; ++ib) {
          const int i = ib * 16 + lr;
#pragma unroll 1
          for (int j = 0; j <= min(i, len - 1); ++j) {
            const int pos = (j & 32) + 8 * ((j >> 2) & 3) + ((j >> 4) & 1) * 4 + (j & 3);
            const float p = to_f32(P[TP::off(i, pos)]);
            const f32x4 vv = load4f(lds[buf][2 - FIRST] + TL::off(j, wave * 16 + lg * 4));
#pragma unroll
            for (int e = 0; e < 4; ++e) oa[ib][e] = fmaf(p, vv[e], oa[ib][e]);
          }
        }
      }
    }
    // the state after the chunk, unless nothing reads it
    if (STATE || c + 1 < nc || a.s_out) {
      float g = gC;
      if (len < kC) {
        weights(len);
        g = powg(lg2, len);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) S[t] *= g;
      add_outer<T, DH, STATE ? 2 : SUM ? 4 : DH / 16>(S, bcol, ba, cf, w, a.fine);
    }
    if constexpr (SUM) {
      if (sg.t0 > 0) {  // (the sequence's first segment has no boundary before it)
        ColRaw<T> dr[2];
        each<2>([&](auto us) { dr[us] = TL::template col_at<0, us * 32, us * 32 + 16>(dcol, ba); });
        lds_tr_wait();
        F df[2];
        float wc[2][8];
#pragma unroll
        for (int us = 0; us < 2; ++us) {
          df[us] = take(dr[us]);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            wc[us][e] = us * 32 + (e < 4 ? 4 * lg + e : 12 + 4 * lg + e) < len ? wr[us][e] * gc : 0.f;
        }
        add_outer<T, DH, 4>(R, qcol, ba, df, wc, true);
        gc *= gC;
      }
    }
    if (NB > 1) {  // the next chunk's tiles, before the stores
      if (c + NB - 1 < nc) vm_wait<AHEAD>();
      else vm_wait<0>();
    }
    if constexpr (!STATE) {
#pragma unroll
      for (int ib = 0; ib < 4; ++ib) {
        const int i = ib * 16 + lr;
        if (alive && i < len)
          store4((T*)a.out + (r0 + (REV ? -1 : 1) * (int64_t)(c * kC + i)) * a.ldo + h * DH +
                     wave * 16 + lg * 4,
                 oa[ib][0], oa[ib][1], oa[ib][2], oa[ib][3]);
      }
    }
    buf = buf + 1 == NB ? 0 : buf + 1;
    next = next + 1 == NB ? 0 : next + 1;
  }
  if (!alive) return;
  if constexpr (SUM) {
    if (sg.t0 > 0)
      store_state<NT>(R, a.sum_state + sg.bound * dd + (int64_t)h * DH * DH, DH, 1, col, lg);
  }
  if (STATE) store_state<NT>(S, REV ? bs : bs + dd, DH, 1, col, lg);
  else if (a.s_out && (REV ? sg.t0 == 0 : sg.last))
    store_state<NT>(S, a.s_out + sq, a.sr, a.sc, col, lg);
}

// dk and dv in one reverse pass (bf16, up to 64 columns): two roles of the operator over the same
// four tiles,
//   role 0: a, b, c = k, q, do -> dv, the state R [q][do];
//   role 1: a, b, c = v, do, q -> dk, its transpose;
// the rows are read once for both, and a chunk's two barriers are shared.  8192
// rows, 12 heads of 64: 28 us against 20 + 20 us.  With 128 columns a pass is bound
// by what its eight waves read from LDS and issue, not by its rows (32768 rows, 16
// heads: 356 us against 161 + 161 us, and 243 us for dq with the sum of R against
// 161 + 87 us), so those stay apart.
template <int DH>
__global__ __launch_bounds__(DH * 4, 2) void lin_dkdv_kernel(LinPair a) {
  typedef bf16 T;
  typedef bf16x8 F;
  typedef Tile<T, DH> TL;
  typedef Tile<T, kC> TP;
  constexpr int NW = DH / 16, NT = DH / 16, KS = DH >= 32 ? DH / 32 : 1, NI = TL::NCH / NW;
  constexpr unsigned TILE = kC * DH * sizeof(T), BUF = 4 * TILE, PB = kC * kC * sizeof(T);
  __shared__ __attribute__((aligned(1024))) T lds[2][4][kC * DH];  // k, v, q, do
  __shared__ __attribute__((aligned(1024))) T P[2][kC * kC];
  const int lane = threadIdx.x & 63, wave = wave_index();
  const int lr = lane & 15, lg = lane >> 4;
  const int h = blockIdx.x % a.H;
  const LinSeg sg = lin_segment(a.cu, a.nseq, a.total, a.seg, blockIdx.x / a.H);
  if (sg.len < 0) return;
  const float lg2 = log2f(a.gamma[h]);
  const int col = wave * 16 + lr;

  f32x4 S[2][NT];
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int t = 0; t < NT; ++t) S[p][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int64_t dd = (int64_t)a.H * DH * DH, hs = (int64_t)h * DH * DH, sq = sg.seq * dd + hs;
  const float* from = !sg.last              ? a.seg_state + (sg.bound + 1) * dd + hs
                      : a.given && sg.t0 > 0 ? a.given + sg.first * dd + hs
                      : a.ds_out            ? a.ds_out + sq
                                            : nullptr;
  if (from) {
    load_state<NT>(S[0], from, DH, 1, col, lg);
    load_state<NT>(S[1], from, 1, DH, col, lg);
  }
  const int nc = (sg.len + kC - 1) / kC;
  const int64_t r0 = sg.row0 + sg.len - 1;
  const T* K = (const T*)a.k + r0 * a.ldk + h * DH;
  const T* V = (const T*)a.v + r0 * a.ldv + h * DH;
  const T* Q = (const T*)a.q + r0 * a.ldq + h * DH;
  const T* O = (const T*)a.dout + r0 * a.ldo + h * DH;
  auto issue = [=](int c, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int ti = wave * NI + i;
      TL::issue(K, -a.ldk, c * kC, sg.len - 1, lds[buf][0], ti, lane);
      TL::issue(V, -a.ldv, c * kC, sg.len - 1, lds[buf][1], ti, lane);
      TL::issue(Q, -a.ldq, c * kC, sg.len - 1, lds[buf][2], ti, lane);
      TL::issue(O, -a.ldo, c * kC, sg.len - 1, lds[buf][3], ti, lane);
    }
  };
  float w[2][8], fi[4];
  auto weights = [&](int len) __attribute__((always_inline)) {
#pragma unroll
    for (int us = 0; us < 2; ++us)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int j = us * 32 + (e < 4 ? 4 * lg + e : 12 + 4 * lg + e);
        w[us][e] = j < len ? a.scale * powg(lg2, len - j) : 0.f;
      }
  };
  weights(kC);
#pragma unroll
  for (int ib = 0; ib < 4; ++ib) fi[ib] = powg(lg2, ib * 16 + lr);
  const float gC = powg(lg2, kC);
  // the blocks of the scores, as above
  constexpr int NR = (12 + NW - 1) / NW;
  float fac[NR][4];
  unsigned ra[NR], rb[NR];
  int at[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int b = n * NW + wave;
    const int d = b < 4 ? 0 : b < 7 ? 1 : b < 8 ? 3 : 2;
    const int ib = b < 4 ? b : b < 7 ? b - 3 : b < 8 ? 3 : b < 10 ? b - 6 : (b - 10) * 2;
    const int jb = b < 10 ? ib - d : ib + 1;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int lag = 16 * d + lr - 4 * lg - r;
      fac[n][r] = lag >= 0 ? a.scale * powg(lg2, lag) : 0.f;
    }
    ra[n] = TL::row_base(lds[0][0], (ib & 3) * 16 + lr, lane);
    rb[n] = TL::row_base(lds[0][2], (jb & 3) * 16 + lr, lane);
    at[n] = TP::off((ib & 3) * 16 + lr, ((jb >> 1) & 1) * 32 + 8 * lg + 4 * (jb & 1));
  }
  const ColBase<T> bcol = TL::col_base(lds[0][2], lane);
  ColBase<T> ccol = TL::col_base(lds[0][2], lane);  // this wave's columns (of role 1)
  ccol.a[0] ^= wave * 16 * (int)sizeof(T);
  const unsigned half = half_base<T, DH>(lds[0][0], lr, lane);
  const unsigned prow = TP::row_base(P[0], lr, lane);

  if (nc > 0) issue(0, 0);
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int t = 0; t < NT; ++t) settle(S[p][t]);
  vm_wait<0>();
  for (int c = 0; c < nc; ++c) {
    wg_barrier();  // this chunk's tiles are there; every wave is done with the last chunk
    if (c + 1 < nc) issue(c + 1, (c + 1) & 1);
    const int buf = c & 1, len = min(kC, sg.len - c * kC);
    const unsigned ba = buf * BUF;
    f32x4 oa[2][4];
    each<2>([&](auto p) __attribute__((always_inline)) {
      each<NR>([&](auto n) __attribute__((always_inline)) {
        if (n * NW + wave >= 12) return;
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
        if (n * NW + wave < 10) {
          RowRaw<T> br[KS], ar[KS];
          each<KS>([&](auto ds) {
            br[ds] = TL::template row_at<ds, 0>(rb[n] + (ba + p * TILE));
            ar[ds] = TL::template row_at<ds, 0>(ra[n] + (ba + p * TILE));
          });
          lds_tr_wait();
#pragma unroll
          for (int ds = 0; ds < KS; ++ds) {
            const F bf = TL::take_row(br[ds], lane);
            s = TL::mma(bf, TL::take_row(ar[ds], lane), s);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) s[r] = fac[n][r] == 0.f ? 0.f : s[r] * fac[n][r];
        }
        store4(P[p] + at[n], s[0], s[1], s[2], s[3]);
      });
#pragma unroll
      for (int ib = 0; ib < 4; ++ib) oa[p][ib] = f32x4{0.f, 0.f, 0.f, 0.f};
      each<KS>([&](auto ks) __attribute__((always_inline)) {
        const F sf = frag_from<T>(S[p][2 * ks], DH >= 32 ? S[p][2 * ks + (DH >= 32)] : f32x4{});
        HalfRaw<T> qr[4];
        each<4>([&](auto ib) { qr[ib] = half_at<T, DH, ks, ib * 16>(half + (ba + p * TILE)); });
        lds_tr_wait();
#pragma unroll
        for (int ib = 0; ib < 4; ++ib) oa[p][ib] = mma16(sf, take_row8p<T, DH>(qr[ib]), oa[p][ib]);
      });
#pragma unroll
      for (int ib = 0; ib < 4; ++ib) oa[p][ib] *= fi[ib];
    });
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the scores are written
    wg_barrier();
    const bool more = c + 1 < nc || a.ds_in;
    float g = gC;
    if (len < kC && more) {
      weights(len);
      g = powg(lg2, len);
    }
    each<2>([&](auto p) __attribute__((always_inline)) {
      ColRaw<T> cr[2];
      F cf[2];
      const unsigned ca = ba + (1 - p) * TILE;  // c is q for role 1, do for role 0
      each<2>([&](auto us) { cr[us] = TL::template col_at<0, us * 32, us * 32 + 16>(ccol, ca); });
      lds_tr_wait();
#pragma unroll
      for (int us = 0; us < 2; ++us) cf[us] = take(cr[us]);
      each<4>([&](auto ib) __attribute__((always_inline)) {
        constexpr int NU = ib / 2 + 1;
        RowRaw<T> pr[NU];
        each<NU>([&](auto us) { pr[us] = TP::template row_at<us, ib * 16>(prow + p * PB); });
        lds_tr_wait();
#pragma unroll
        for (int us = 0; us < NU; ++us) oa[p][ib] = mma16(cf[us], take(pr[us]), oa[p][ib]);
      });
      if (more) {
#pragma unroll
        for (int t = 0; t < NT; ++t) S[p][t] *= g;
        add_outer<T, DH, 4>(S[p], bcol, ba + p * TILE, cf, w, p == 0);
      }
    });
    vm_wait<0>();  // the next chunk's tiles, before the stores
#pragma unroll
    for (int ib = 0; ib < 4; ++ib) {
      const int i = ib * 16 + lr;
      if (i < len) {
        const int64_t r = r0 - (c * kC + i);
        store4((T*)a.dv + r * a.ldv + h * DH + wave * 16 + lg * 4, oa[0][ib][0], oa[0][ib][1],
               oa[0][ib][2], oa[0][ib][3]);
        store4((T*)a.dk + r * a.ldk + h * DH + wave * 16 + lg * 4, oa[1][ib][0], oa[1][ib][1],
               oa[1][ib][2], oa[1][ib][3]);
      }
    }
  }
  if (a.ds_in && sg.t0 == 0) store_state<NT>(S[0], a.ds_in + sq, DH, 1, col, lg);
}

// The segments' own sums -> the states at the boundaries, in place, from the
// sequence's given state.  `given`, if the operator writes its last state over the
// given one (by another workgroup than the one that reads it), keeps a copy at the
// sequence's first boundary.  Forward: the sum of segment i lies at the boundary
// after it; reverse: at the one before it.  One thread per four elements.
template <bool REV>
__global__ __launch_bounds__(256) void lin_scan_kernel(const int* __restrict__ cu, int nseq,
                                                       int total, int seg, int H, int dd,
                                                       const float* __restrict__ gamma,
                                                       const float* __restrict__ s_in,
                                                       float* __restrict__ seg_state,
                                                       float* __restrict__ given) {
  const int h = blockIdx.y;
  const int e = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (e >= dd) return;
  const float lg2 = log2f(gamma[h]);
  for (int seq = blockIdx.z; seq < nseq; seq += gridDim.z) {
    const int begin = min(max(cu[seq], 0), total), end = min(max(cu[seq + 1], begin), total);
    const int n = end - begin, ns = (n + seg - 1) / seg;
    if (ns < 2) continue;
    f32x4 u = {0.f, 0.f, 0.f, 0.f};
    if (s_in) u = *(const f32x4*)(s_in + ((int64_t)seq * H + h) * dd + e);
    if (given) *(f32x4*)(given + ((int64_t)(begin / seg + 1) * H + h) * dd + e) = u;
    // boundary k: n - (the rows behind it), in reverse; eight sums at a time
    float* p0 = seg_state + ((int64_t)(begin / seg) * H + h) * dd + e;
    const int64_t step = (int64_t)H * dd;
    const float gs = powg(lg2, seg);
    for (int i = 1; i < ns; i += 8) {
      f32x4 own[8];
#pragma unroll
      for (int x = 0; x < 8; ++x)
        if (i + x < ns) own[x] = *(const f32x4*)(p0 + (REV ? ns - i - x : i + x) * step);
#pragma unroll
      for (int x = 0; x < 8; ++x)
        if (i + x < ns) {
          const int k = REV ? ns - i - x : i + x;
          // the segment just passed: whole, but for the last of the sequence
          u = u * (REV && k == ns - 1 ? powg(lg2, n - k * seg) : gs) + own[x];
          *(f32x4*)(p0 + k * step) = u;
        }
    }
  }
}

// ------------------------------------------------------------------ decay gradient
// dg = sum_t <R_t, S_{t-1}>, per segment from the state S before it and the
// gradient R of the state after it: with D = dS / dg from 0 at the segment's
// start,
//   dg_seg = sum_t scale do_t . (D_t^T q_t) + <R, D_end>
// chunk by chunk:
//   sum_{j < i} (i-j) g^(i-j-1) scale (q_i . k_j) (do_i . v_j)
//   + <S, scale sum_i (i+1) g^i q_i do_i^T> + <D, scale sum_i g^(i+1) q_i do_i^T>
//   D' = g^C D + C g^(C-1) S + sum_j (C-1-j) g^(C-2-j) k_j v_j^T
// Both inner products take the states from float32 registers and the sums in
// parts.  One partial sum per wave, added in a fixed order at the end.

template <typename T, int DH>
__global__ __launch_bounds__(DH * 4) void lin_dgamma_kernel(LinDecay a) {
  typedef typename Frag<T>::type F;
  typedef Tile<T, DH> TL;
  constexpr int NW = DH / 16, NT = DH / 16, KS = DH >= 32 ? DH / 32 : 1;
  constexpr int NI = TL::NCH / NW, NB = sizeof(T) * DH > 256 ? 1 : 2;
  __shared__ __attribute__((aligned(1024))) T ring[NB][4][kC * DH];  // q, k, v, do
  __shared__ __attribute__((aligned(16))) float tab[2][3][kC];
  const int lane = threadIdx.x & 63, wave = wave_index();
  const int lr = lane & 15, lg = lane >> 4;
  const int h = blockIdx.x % a.H, slot = blockIdx.x / a.H;
  const LinSeg sg = lin_segment(a.cu, a.nseq, a.total, a.seg, slot);
  float* out = a.part + ((int64_t)h * a.nslot + slot) * NW + wave;
  if (sg.len <= 0) {
    // an empty slot, or an empty sequence: the state passes through unchanged
    if (lane == 0) *out = 0.f;
    return;
  }
  const float lg2h = log2f(a.gamma[h]);
  const int col = wave * 16 + lr;
  f32x4 S[NT], D[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    S[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    D[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int64_t sq = ((int64_t)sg.seq * a.H + h) * DH * DH;
  const int64_t dd = (int64_t)a.H * DH * DH, bd = sg.bound * dd + (int64_t)h * DH * DH;
  if (sg.t0 > 0) load_state<NT>(S, a.seg_s + bd, DH, 1, col, lg);
  else if (a.s_in) load_state<NT>(S, a.s_in + sq, DH, 1, col, lg);

  const T* qs = (const T*)a.q + sg.row0 * a.ldq + h * DH;
  const T* ks_ = (const T*)a.k + sg.row0 * a.ldk + h * DH;
  const T* vs = (const T*)a.v + sg.row0 * a.ldv + h * DH;
  const T* ds_ = (const T*)a.dout + sg.row0 * a.ldo + h * DH;
  float sum = 0.f;
  const int nc = (sg.len + kC - 1) / kC;
  auto issue = [=](int c) __attribute__((always_inline)) {
    T(*t)[kC * DH] = ring[NB == 2 ? c & 1 : 0];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int ti = wave * NI + i;
      TL::issue(qs, a.ldq, c * kC, sg.len - 1, t[0], ti, lane);
      TL::issue(ks_, a.ldk, c * kC, sg.len - 1, t[1], ti, lane);
      TL::issue(vs, a.ldv, c * kC, sg.len - 1, t[2], ti, lane);
      TL::issue(ds_, a.ldo, c * kC, sg.len - 1, t[3], ti, lane);
    }
  };
  // The weights of a chunk's rows j, for a whole chunk and for the last one: g^j,
  // g^(len-1-j) and (len-1-j) g^(len-2-j); and each lane's factors (i-j) g^(i-j-1) of
  // the scores.  (Powers formed anew for every use took half of this kernel.)
  if (threadIdx.x < kC) {
    const int j = threadIdx.x;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int len = x ? sg.len - (nc - 1) * kC : kC;
      tab[x][0][j] = j < len ? powg(lg2h, j) : 0.f;
      tab[x][1][j] = j < len ? powg(lg2h, len - 1 - j) : 0.f;
      tab[x][2][j] = j < len - 1 ? (float)(len - 1 - j) * powg(lg2h, len - 2 - j) : 0.f;
    }
  }
  constexpr int NR = (10 + NW - 1) / NW;
  float fac[NR][4];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int blk = n * NW + wave;
    const int ib = blk >= 6 ? 3 : blk >= 3 ? 2 : blk >= 1 ? 1 : 0, jb = blk - ib * (ib + 1) / 2;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int lag = (ib - jb) * 16 + lr - lg * 4 - r;
      fac[n][r] = lag > 0 ? a.scale * (float)lag * powg(lg2h, lag - 1) : 0.f;
    }
  }
  const float gh = a.gamma[h], gC = powg(lg2h, kC), gC1 = powg(lg2h, kC - 1);
  __syncthreads();
  if (NB == 2) issue(0);
#pragma unroll
  for (int t = 0; t < NT; ++t) settle(S[t]);
  for (int c = 0; c < nc; ++c) {
    if (NB == 2) vm_wait<0>();
    wg_barrier();  // (two buffers: this chunk's tiles are there,) the last chunk's are read
    if (NB == 1) {
      issue(c);
      vm_wait<0>();
      wg_barrier();
    } else if (c + 1 < nc) {
      issue(c + 1);
    }
    const T(*lds)[kC * DH] = ring[NB == 2 ? c & 1 : 0];
    const int len = min(kC, sg.len - c * kC);
    const unsigned tb = lds_addr(&tab[len < kC][0][4 * lg]);
    each<NR>([&](auto n) __attribute__((always_inline)) {
      const int blk = n * NW + wave;
      if (blk >= 10) return;
      const int ib = blk >= 6 ? 3 : blk >= 3 ? 2 : blk >= 1 ? 1 : 0, jb = blk - ib * (ib + 1) / 2;
      f32x4 s = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
      each<KS>([&](auto ds) __attribute__((always_inline)) {
        RowRaw<T> qr = TL::template row_at<ds, 0>(TL::row_base(lds[0], ib * 16 + lr, lane));
        RowRaw<T> kr = TL::template row_at<ds, 0>(TL::row_base(lds[1], jb * 16 + lr, lane));
        RowRaw<T> vr = TL::template row_at<ds, 0>(TL::row_base(lds[2], jb * 16 + lr, lane));
        RowRaw<T> dr = TL::template row_at<ds, 0>(TL::row_base(lds[3], ib * 16 + lr, lane));
        lds_tr_wait();
        const F kf = TL::take_row(kr, lane), vf = TL::take_row(vr, lane);
        s = TL::mma(kf, TL::take_row(qr, lane), s);
        dp = TL::mma(vf, TL::take_row(dr, lane), dp);
      });
      if (ib * 16 + lr < len) {
#pragma unroll
        for (int r = 0; r < 4; ++r) sum += s[r] * dp[r] * fac[n][r];
      }
    });
    ColRaw<T> dr[2], vr[2];
    F df[2], vf[2];
    ColBase<T> db = TL::col_base(lds[3], lane), vb = TL::col_base(lds[2], lane);
    for (auto& x : db.a) x ^= wave * 16 * (int)sizeof(T);
    for (auto& x : vb.a) x ^= wave * 16 * (int)sizeof(T);
    each<2>([&](auto us) {
      dr[us] = TL::template col_at<0, us * 32, us * 32 + 16>(db, 0);
      vr[us] = TL::template col_at<0, us * 32, us * 32 + 16>(vb, 0);
    });
    lds_tr_wait();
#pragma unroll
    for (int us = 0; us < 2; ++us) {
      df[us] = take(dr[us]);
      vf[us] = take(vr[us]);
    }
    // the weights of the rows this lane holds, from table x
    float w[2][8];
    auto weights = [&](auto x) __attribute__((always_inline)) {
      f32x4 t[2][2];
      each<2>([&](auto us) {
        t[us][0] = lds_read_f32x4_at<(x * kC + us * 32) * 4>(tb);
        t[us][1] = lds_read_f32x4_at<(x * kC + us * 32 + 16) * 4>(tb);
      });
      lds_tr_wait();
#pragma unroll
      for (int us = 0; us < 2; ++us)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          lds_tr_bind(t[us][hf]);
#pragma unroll
          for (int e = 0; e < 4; ++e) w[us][hf * 4 + e] = t[us][hf][e];
        }
    };
    f32x4 W[NT];
    auto inner = [&](const f32x4(&x)[NT]) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) sum += W[t][r] * x[t][r];
    };
    // scale g^(i+1), then scale (i+1) g^i
    const ColBase<T> qb = TL::col_base(lds[0], lane), kb = TL::col_base(lds[1], lane);
    weights(std::integral_constant<int, 0>{});
#pragma unroll
    for (int us = 0; us < 2; ++us)
#pragma unroll
      for (int e = 0; e < 8; ++e) w[us][e] *= a.scale * gh;
#pragma unroll
    for (int t = 0; t < NT; ++t) W[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    add_outer<T, DH, 4>(W, qb, 0, df, w, true);
    inner(D);
    weights(std::integral_constant<int, 0>{});
#pragma unroll
    for (int us = 0; us < 2; ++us)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        w[us][e] *= a.scale * (float)(us * 32 + (e < 4 ? e : 12 + e) + 1 + 4 * lg);
#pragma unroll
    for (int t = 0; t < NT; ++t) W[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    add_outer<T, DH, 4>(W, qb, 0, df, w, true);
    inner(S);
    const float g = len == kC ? gC : powg(lg2h, len);
    const float g1 = (float)len * (len == kC ? gC1 : powg(lg2h, len - 1));
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      D[t] = D[t] * g + S[t] * g1;
      S[t] *= g;
    }
    weights(std::integral_constant<int, 2>{});
    add_outer<T, DH, 4>(D, kb, 0, vf, w, true);
    weights(std::integral_constant<int, 1>{});
    add_outer<T, DH, 4>(S, kb, 0, vf, w, true);
  }
  const float* R = !sg.last ? a.seg_r + bd + dd : a.ds_out ? a.ds_out + sq : nullptr;
  if (R) {
    load_state<NT>(S, R, DH, 1, col, lg);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) sum += S[t][r] * D[t][r];
  }
  sum = wave_sum(sum);
  if (lane == 0) *out = sum;
}

// dgamma[h] = sum of its partials, in a fixed order.
__global__ __launch_bounds__(256) void lin_dgamma_sum_kernel(const float* __restrict__ part, int n,
                                                             float* __restrict__ dgamma) {
  __shared__ float red[4];
  const float* p = part + (int64_t)blockIdx.x * n;
  float s = 0.f;
  for (int i = threadIdx.x; i < n; i += 256) s += p[i];
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) dgamma[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// ------------------------------------------------------------------ single tokens
// S' = g S + k v^T, o = scale S'^T q: each state is read and written once, in
// 16-byte vectors along its columns; the rows of a head are spread over the
// workgroup and their products with q joined in LDS.

template <typename T, int DH>
__global__ __launch_bounds__(256) void lin_step_kernel(LinStep a) {
  constexpr int CV = DH / 4, NR = 256 / CV;  // vectors of a row; rows at a time
  __shared__ __attribute__((aligned(16))) float red[NR][DH];
  const int h = blockIdx.x % a.H, b = blockIdx.x / a.H;
  const int c = (threadIdx.x % CV) * 4, r0 = threadIdx.x / CV;
  const int slot = a.slot ? a.slot[b] : b;
  T* o = (T*)a.o + (int64_t)b * a.ldo + h * DH;
  if (slot < 0 || slot >= a.slots) {
    if (r0 == 0) store4(o + c, 0.f, 0.f, 0.f, 0.f);
    return;
  }
  const T* q = (const T*)a.q + (int64_t)b * a.ldq + h * DH;
  const T* k = (const T*)a.k + (int64_t)b * a.ldk + h * DH;
  const f32x4 v = load4f((const T*)a.v + (int64_t)b * a.ldv + h * DH + c);
  const int64_t base = ((int64_t)slot * a.H + h) * DH * DH + c;
  const float g = a.gamma[h];
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < (DH + NR - 1) / NR; ++i) {
    const int r = i * NR + r0;
    if (NR <= DH || r < DH) {
      f32x4 s = *(const f32x4*)(a.s_in + base + r * DH);
      const float kr = to_f32(k[r]), qr = to_f32(q[r]);
      s = s * g + v * kr;
      *(f32x4*)(a.s_out + base + r * DH) = s;
      acc += s * qr;
    }
  }
  *(f32x4*)&red[r0][c] = acc;
  __syncthreads();
  for (int x = threadIdx.x; x < DH; x += 256) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NR; ++i) s += red[i][x];
    o[x] = from_f32<T>(s * a.scale);
  }
}

template <typename T, int DH> constexpr bool lin_joined = sizeof(T) == 2 && DH <= 64;

template <typename T, int DH>
hipError_t pass_t(const LinPass& a, bool rev, bool state, hipStream_t s) {
  constexpr int HP = lin_heads<T, DH>, BS = DH * 4 * HP;
  const dim3 grid((unsigned)((int64_t)(a.total / a.seg + a.nseq) * ((a.H + HP - 1) / HP)));
  if constexpr (!lin_joined<T, DH>) {
    if (rev && state) lin_kernel<T, DH, true, true, false><<<grid, BS, 0, s>>>(a);
    else if (rev) lin_kernel<T, DH, true, false, false><<<grid, BS, 0, s>>>(a);
  }
  if (!rev && state) lin_kernel<T, DH, false, true, false><<<grid, BS, 0, s>>>(a);
  else if (!rev && a.sum_state) {
    if constexpr (lin_joined<T, DH>) lin_kernel<T, DH, false, false, true><<<grid, BS, 0, s>>>(a);
  } else if (!rev) {
    lin_kernel<T, DH, false, false, false><<<grid, BS, 0, s>>>(a);
  }
  return hipGetLastError();
}
template <int DH>
hipError_t dkdv_t(const LinPair& a, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)(a.total / a.seg + a.nseq) * a.H));
  lin_dkdv_kernel<DH><<<grid, DH * 4, 0, s>>>(a);
  return hipGetLastError();
}
template <typename T, int DH>
hipError_t dgamma_t(const LinDecay& a, hipStream_t s) {
  lin_dgamma_kernel<T, DH><<<dim3((unsigned)((int64_t)a.nslot * a.H)), DH * 4, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  lin_dgamma_sum_kernel<<<dim3(a.H), 256, 0, s>>>(a.part, a.nslot * (DH / 16), a.dgamma);
  return hipGetLastError();
}
template <typename T, int DH>
hipError_t step_t(const LinStep& a, hipStream_t s) {
  lin_step_kernel<T, DH><<<dim3((unsigned)((int64_t)a.B * a.H)), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t lin_pass(DType dt, int dh, const LinPass& a, bool rev, bool state, hipStream_t s) {
  BY_TYPE_AND_WIDTH(pass_t, dt, dh, a, rev, state, s);
}
hipError_t lin_scan(int dh, const LinPass& a, bool rev, hipStream_t s) {
  const dim3 grid((dh * dh / 4 + 255) / 256, a.H, a.nseq < 64 ? a.nseq : 64);
  if (rev)
    lin_scan_kernel<true><<<grid, 256, 0, s>>>(a.cu, a.nseq, a.total, a.seg, a.H, dh * dh, a.gamma,
                                               a.s_in, a.seg_state, a.given);
  else
    lin_scan_kernel<false><<<grid, 256, 0, s>>>(a.cu, a.nseq, a.total, a.seg, a.H, dh * dh, a.gamma,
                                                a.s_in, a.seg_state, a.given);
  return hipGetLastError();
}
hipError_t lin_dkdv(int dh, const LinPair& a, hipStream_t s) {
  switch (dh) {
    case 16: return dkdv_t<16>(a, s);
    case 32: return dkdv_t<32>(a, s);
    default: return dkdv_t<64>(a, s);
  }
}
bool lin_joined_backward(DType dt, int dh) { return dt == DType::BF16 && dh <= 64; }
hipError_t lin_dgamma(DType dt, int dh, const LinDecay& a, hipStream_t s) {
  BY_TYPE_AND_WIDTH(dgamma_t, dt, dh, a, s);
}
hipError_t lin_step(DType dt, int dh, const LinStep& a, hipStream_t s) {
  BY_TYPE_AND_WIDTH(step_t, dt, dh, a, s);
}

// Rows of a segment: such that the workgroups, at most total / seg + nseq of a group
// of heads, are one round of those that the chip holds at once (one of eight waves
// to a CU), or, with many sequences, a quarter of it more than these (131072 rows, 16
// heads of 64, by segments of 1024, 4544 and 8192 rows: sums 117, 131, 173 us, operator
// 270, 266, 373, scan 22, 7, 5).  Down to one chunk: where that leaves CUs idle, the
// chunks of a segment one after another are the time (1024 rows of 12 heads of 64,
// forward and gradients, at least 64, 128 or 256 rows: 62, 67, 93 us; of 8 float32
// heads of 128: 176, 246, 405).
int lin_segment_rows(DType dt, int total, int nseq, int H, int dh) {
  const int row = dh * (dt == DType::BF16 ? 2 : 4), hp = row < 256 ? 256 / row : 1;
  const int round = 256 / ((H + hp - 1) / hp);  // segments of a group of heads
  int n = round - nseq;
  if (n < round / 4) n = round / 4;
  if (n < 1) n = 1;
  const int64_t want = ((int64_t)total + n - 1) / n;
  return (int)((want + kC - 1) / kC * kC);
}

}  // namespace bcmt
