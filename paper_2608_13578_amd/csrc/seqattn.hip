// Causal softmax attention over packed sequences with grouped heads.
//
// Rows [cu[s], cu[s+1]) of the packed arrays are sequence s.  Query head h
// reads key/value head j = h / G.  For a row t and the rows u <= t of its
// sequence:
//   z_tu = scale q_t . k_u,  p_tu = exp(z_tu - lse_t),  lse_t = log sum_u exp z_tu
//   o_t = sum_u p_tu v_u
//   delta_t = do_t . o_t,  dz_tu = p_tu (do_t . v_u - delta_t)
//   dq_t = scale sum_u dz_tu k_u
//   dk_u = scale sum_h sum_t dz_tu q_t,  dv_u = sum_h sum_t p_tu do_t
// with the sums over h taken over the group of query heads.  No score matrix
// leaves registers.
//
// Register layouts (common.h): a matrix instruction returns lane l the column
// l % 16 and rows 4 (l / 16) + r.  The forward and dQ compute transposed
// scores, so a lane holds one query and a set of keys, and those registers are
// the second operand of the next product as they are (Tile::col_at reads the
// first operand in the same key order).  dK/dV computes them untransposed,
// one key per lane, to the same end.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "kernels.h"
#include "mixer_tile.h"

namespace bcmt {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// The two tiles (K, V or Q, dO) of one step, 2 NCH wave instructions shared by
// NW waves (the first 2 NCH of them where there are more waves).
template <typename T, int DH, int NW>
constexpr int kPairLoads = 2 * Tile<T, DH>::NCH / NW > 1 ? 2 * Tile<T, DH>::NCH / NW : 1;
// NEAR: with the lane's part of the addresses in registers (kept where a kernel has
// some left; with a single spill in its loop it would wait for memory there).
template <typename T, int DH, int NW, bool NEAR>
struct PairLoads {
  typedef Tile<T, DH> TL;
  static constexpr int NI = kPairLoads<T, DH, NW>;
  static_assert(NI * NW == 2 * TL::NCH || NI == 1, "loads of two tiles");
  unsigned off[NI];
  int64_t lda, ldb;
  int wave, lane;
  bool near;
  __device__ __forceinline__ PairLoads(int64_t lda_, int64_t ldb_, int wave_, int lane_)
      : lda(lda_), ldb(ldb_), wave(wave_), lane(lane_) {
    near = NEAR && lda <= kNearLd && ldb <= kNearLd;
    if (!NEAR) return;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int gi = wave * NI + i;
      off[i] = TL::lane_off(gi < TL::NCH ? lda : ldb, gi % TL::NCH, lane);
    }
  }
  // Rows r0 .. r0 + 63 of a and b (those behind rlast: rlast's) into ta and tb.
  __device__ __forceinline__ void operator()(const T* a, const T* b, int r0, int rlast, T* ta,
                                             T* tb) const {
    const bool whole = near && r0 + 63 <= rlast;
    int ln = lane;
    if (!NEAR) settle(ln);  // (opaque: the addresses are formed anew, not kept)
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int gi = wave * NI + i;
      if (gi >= 2 * TL::NCH) break;
      const bool first = gi < TL::NCH;
      const T* src = first ? a : b;
      T* t = first ? ta : tb;
      const int64_t ld = first ? lda : ldb;
      if (NEAR && whole) TL::issue_near(src + r0 * ld, off[i], t, gi % TL::NCH);
      else TL::issue(src, ld, r0, rlast, t, gi % TL::NCH, ln);
    }
  }
};

// ------------------------------------------------------------------ forward
// One workgroup of NW waves, NQ groups of 16 queries each, over NW / wph heads of
// one group (wph waves a head): every tile of 64 keys is fetched once for all of
// them.  The tiles go through a ring of NS buffers, one barrier a tile.  Four
// waves over 128 queries, two workgroups per CU and double buffers left a CU
// waiting for its keys more than half of the time (16384 rows, 16 heads of 128:
// 866 us, 471 us with the loads left out); eight waves halve the traffic, and
// three tiles ahead hide the rest (462 us, 0.86 PFLOP/s).  Where few workgroups
// make a launch, NG = 2 teams of NW waves take the tiles in turn, each through its own
// ring, and are joined in LDS at the end.
//
// The maximum is raised only when a score passes it by more than kRaise (both in
// base-2 logarithms): the weights then stay below 2^kRaise (their relative rounding
// is the same at any scale, and float32 sums have the room), and the outputs are
// rescaled, and the lanes of a row agree on its maximum, in a few tiles of a
// sequence instead of in all.  Tiles that every query of a wave sees whole take no
// mask.
//
// In bfloat16 the weights are rounded to the type as operands of the product with
// V, since the matrix instructions take no other; their sum l is of the float32
// weights.  With the output's own rounding: an error of 1.8e-3 to 2.0e-3 in the
// 2-norm, 1.6e-3 by the output's rounding alone.

constexpr float kRaise = 8.f;

template <typename T, int DH, int NW_, int NG_> struct QueryShape {
  static constexpr int NW = NW_, NG = NG_, NQ = sizeof(T) == 2 ? 2 : 1;
  // buffers of a team's ring: 128 KB of LDS a workgroup, or 64 KB for two of four waves
  static constexpr int NS = sizeof(T) == 2 ? (DH == 128 && NW == 4 ? 2 : 4)
                            : DH == 128 || (DH == 64 && NG == 2) ? 2 : 3;
  static constexpr int WAVES = sizeof(T) == 4 && NG == 1 ? 1 : 2;  // of a SIMD
};

// The second team's part of a row joins the first's: what a wave leaves in LDS.
template <int NQ, int NJ> struct TeamPart {
  f32x4 a[NQ][NJ][64];
  float m[NQ][64], l[NQ][64];
  int dropped;
};

template <typename T, int DH, int NW, int NG>
__global__ __launch_bounds__(NW * NG * 64, (QueryShape<T, DH, NW, NG>::WAVES)) void seq_fwd_kernel(
    const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v,
    const int* __restrict__ cu, T* __restrict__ o, float* __restrict__ lse, int total, int nseq,
    int H, int G, int wph, int64_t ldq, int64_t ldk, int64_t ldv, int64_t ldo, float sl2) {
  typedef typename Frag<T>::type F;
  typedef Tile<T, DH> TL;
  constexpr int NQ = QueryShape<T, DH, NW, NG>::NQ, NS = QueryShape<T, DH, NW, NG>::NS;
  constexpr int KS = DH >= 32 ? DH / 32 : 1, NJ = DH / 16;
  constexpr int NI = kPairLoads<T, DH, NW>;
  constexpr int KUS = sizeof(T) == 2 ? 2 : 1;  // key groups read at once
  __shared__ __attribute__((aligned(1024))) T ring[NG][NS][2][64 * DH];
  const int lane = threadIdx.x & 63, wave = wave_index() % NW, team = wave_index() / NW;
  T(*lds)[2][64 * DH] = ring[team];
  const int lr = lane & 15, lg = lane >> 4;
  const int QT = wph * 16 * NQ, hp = NW / wph, HG = H / hp;
  const int wq = wave % wph;
  const int h = (int)(blockIdx.x % HG) * hp + wave / wph;
  const SeqTile st = find_item<false>(cu, nseq, total, QT, (int)(blockIdx.x / HG));
  const int bs = st.begin, be = st.end, q0 = bs + st.tile * QT;
  if (st.tile < 0 || q0 >= be) return;
  const int j = h / G;
  const T* kb = k + j * DH;
  const T* vb = v + j * DH;
  // A head's groups of 16 queries are dealt w, 2 wph - 1 - w: a causal group's work
  // grows with its position.
  int tq[NQ];
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) tq[nq] = q0 + 16 * (nq & 1 ? 2 * wph - 1 - wq : wq);
  const int kend = min(be, q0 + QT);
  const int nt = (kend - bs + 63) / 64, own = (nt - team + NG - 1) / NG;  // tiles; the team's

  F qf[NQ][KS];
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
    for (int ds = 0; ds < KS; ++ds) {
      const int t = tq[nq] + lr;
      qf[nq][ds] = TL::row_global(q + (int64_t)t * ldq + h * DH, ds, lane, t < be);
    }
  f32x4 oa[NQ][NJ];
  float m[NQ], l[NQ];
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) {
    m[nq] = -INFINITY;
    l[nq] = 0.f;
#pragma unroll
    for (int jj = 0; jj < NJ; ++jj) oa[nq][jj] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  int dropped = INT_MAX;  // first tile of which a value was left out
  constexpr unsigned BUF = 2 * 64 * DH * sizeof(T);
  const unsigned krow = TL::row_base(lds[0][0], lr, lane);
  const ColBase<T> vcol = TL::col_base(lds[0][1], lane);
  auto tile = [&](auto masked, int kt, int buf) __attribute__((always_inline)) {
    constexpr bool MASK = decltype(masked)::value;
    const unsigned ba = buf * BUF, ka = krow + ba;
    bool live[NQ];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq)
      live[nq] = !MASK || !(tq[nq] >= be || tq[nq] + 15 < kt);  // wave-uniform
    f32x4 s[NQ][4];
    each<4 / KUS>([&](auto kk) __attribute__((always_inline)) {
      constexpr int k0 = kk * KUS;
      RowRaw<T> kr[KUS][KS];
      each<KUS>([&](auto ku) {
        each<KS>([&](auto ds) { kr[ku][ds] = TL::template row_at<ds, (k0 + ku) * 16>(ka); });
      });
      lds_tr_wait();
#pragma unroll
      for (int ku = 0; ku < KUS; ++ku) {
        F kf[KS];
#pragma unroll
        for (int ds = 0; ds < KS; ++ds) kf[ds] = TL::take_row(kr[ku][ds], lane);
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
          s[nq][k0 + ku] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ds = 0; ds < KS; ++ds)
            s[nq][k0 + ku] = TL::mma(kf[ds], qf[nq][ds], s[nq][k0 + ku]);
        }
      }
    });
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      if (MASK) {
        const int t_eff = live[nq] ? min(tq[nq] + lr, be - 1) : -1;
#pragma unroll
        for (int ku = 0; ku < 4; ++ku)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (kt + ku * 16 + lg * 4 + r > t_eff) s[nq][ku][r] = -INFINITY;
      }
      float mx = s[nq][0][0];
#pragma unroll
      for (int ku = 0; ku < 4; ++ku)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[nq][ku][r]);
      mx *= sl2;
      if (__ballot(mx > m[nq] + kRaise) != 0) {  // (m = -inf: any finite score)
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float mnew = fmaxf(m[nq], mx);
        const float alpha = exp2_fast(m[nq] - (mnew == -INFINITY ? 0.f : mnew));
        l[nq] *= alpha;
        m[nq] = mnew;
#pragma unroll
        for (int jj = 0; jj < NJ; ++jj) oa[nq][jj] *= alpha;
      }
      // all scores so far -inf: subtract 0, so that the weights are 0 and later
      // finite scores still count
      const float neg = m[nq] == -INFINITY ? 0.f : -m[nq];
      float ps = 0.f;
#pragma unroll
      for (int ku = 0; ku < 4; ++ku)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float p = exp2_fast(fmaf(s[nq][ku][r], sl2, neg));
          s[nq][ku][r] = p;
          ps += p;
        }
      l[nq] += ps;
    }
    each<2>([&](auto us) __attribute__((always_inline)) {
      ColRaw<T> vr[NJ];
      each<NJ>([&](auto jj) { vr[jj] = TL::template col_at<jj, us * 32, us * 32 + 16>(vcol, ba); });
      lds_tr_wait();
      F vf[NJ];
#pragma unroll
      for (int jj = 0; jj < NJ; ++jj) vf[jj] = take(vr[jj]);
      // 0 * inf would reach the queries that do not see an infinite or NaN value:
      // such values count as 0 here and are added at the end, to the rows that
      // see them.
      if (MASK) {
        unsigned bad = 0;
#pragma unroll
        for (int jj = 0; jj < NJ; ++jj) bad |= nonfinite_bits(vf[jj]);
        if (__ballot(bad != 0) != 0) {
          dropped = min(dropped, kt);
#pragma unroll
          for (int jj = 0; jj < NJ; ++jj)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (!(fabsf(to_f32(vf[jj][e])) < INFINITY)) vf[jj][e] = from_f32<T>(0.f);
        }
      }
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) {
        if (!live[nq]) continue;
        const F pf = frag_from<T>(s[nq][2 * us], s[nq][2 * us + 1]);
#pragma unroll
        for (int jj = 0; jj < NJ; ++jj) oa[nq][jj] = mma16(vf[jj], pf, oa[nq][jj]);
      }
    });
  };

  const PairLoads<T, DH, NW, (DH <= 64)> load(ldk, ldv, wave, lane);
  auto issue = [&](int it, int buf) __attribute__((always_inline)) {
    load(kb, vb, bs + (it * NG + team) * 64, kend - 1, lds[buf][0], lds[buf][1]);
  };
#pragma unroll
  for (int i = 0; i < NS - 1; ++i)
    if (i < own) issue(i, i);
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
    for (int ds = 0; ds < KS; ++ds) settle(qf[nq][ds]);
  int buf = 0, next = NS - 1;
  for (int it = 0; it * NG < nt; ++it) {
    if (it + NS - 2 < own) vm_wait<(NS - 2) * NI>();
    else vm_wait<0>();
    wg_barrier();  // tile it is there, and every wave is done with the one before
    if (it + NS - 1 < own) issue(it + NS - 1, next);
    const int kt = bs + (it * NG + team) * 64;
    if (kt + 63 <= tq[0]) tile(std::false_type{}, kt, buf);
    else if (kt <= min(tq[NQ - 1] + 15, be - 1)) tile(std::true_type{}, kt, buf);
    buf = buf + 1 == NS ? 0 : buf + 1;
    next = next + 1 == NS ? 0 : next + 1;
  }

  if constexpr (NG == 2) {
    typedef TeamPart<NQ, NJ> Part;
    static_assert(sizeof(Part) * NW <= sizeof(ring), "the parts lie in the ring");
    Part* part = (Part*)&ring[0][0][0][0] + wave;
    wg_barrier();  // every wave is done with its last tile
    if (team == 1) {
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) {
#pragma unroll
        for (int jj = 0; jj < NJ; ++jj) part->a[nq][jj][lane] = oa[nq][jj];
        part->m[nq][lane] = m[nq];
        part->l[nq][lane] = l[nq];
      }
      if (lane == 0) part->dropped = dropped;
    }
    __syncthreads();
    if (team == 1) return;
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      const float mo = part->m[nq][lane], mn = fmaxf(m[nq], mo);
      const float ms = mn == -INFINITY ? 0.f : mn;
      const float w0 = exp2_fast(m[nq] - ms), w1 = exp2_fast(mo - ms);
      l[nq] = l[nq] * w0 + part->l[nq][lane] * w1;
      m[nq] = mn;
#pragma unroll
      for (int jj = 0; jj < NJ; ++jj) oa[nq][jj] = oa[nq][jj] * w0 + part->a[nq][jj][lane] * w1;
    }
    dropped = min(dropped, part->dropped);
  }
  for (int u = dropped; u < min(be, tq[NQ - 1] + 16); ++u)  // (none, as a rule)
#pragma unroll
    for (int jj = 0; jj < NJ; ++jj) {
      const f32x4 x = load4f(vb + (int64_t)u * ldv + jj * 16 + lg * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
          if (u <= tq[nq] + lr && !(fabsf(x[e]) < INFINITY)) oa[nq][jj][e] += x[e];
    }
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) {
    float lt = l[nq];
    lt += __shfl_xor(lt, 16, 64);
    lt += __shfl_xor(lt, 32, 64);
    const int t = tq[nq] + lr;
    if (t < be) {
      const float inv = 1.0f / lt;
      T* op = o + (int64_t)t * ldo + h * DH + lg * 4;
#pragma unroll
      for (int jj = 0; jj < NJ; ++jj)
        store4(op + jj * 16, oa[nq][jj][0] * inv, oa[nq][jj][1] * inv, oa[nq][jj][2] * inv,
               oa[nq][jj][3] * inv);
      if (lse && lg == 0) lse[(int64_t)h * total + t] = m[nq] * kLn2 + logf(lt);
    }
  }
}

// ------------------------------------------------------------------ backward: dQ
// The forward's walk again, with delta_t = do_t . o_t formed (and stored for
// dK/dV) first: s and dp per key tile, dz in place, dQ^T += K^T dZ^T.  The teams'
// parts are added.  dz is rounded to the type as an operand: with the rounding of dq
// itself an error of 2.5e-3 in the 2-norm in bfloat16 against 1.7e-3 of the output's
// rounding alone; a second part of dz would add a third to the products.

// Four waves a workgroup and one a SIMD for 128-wide heads: two would spill.
template <typename T, int DH, int NW, int NG> struct DqShape {
  static constexpr bool WIDE = sizeof(T) == 2 && DH == 128;
  static constexpr int NS = WIDE ? 4 : QueryShape<T, DH, NW, NG>::NS;
  static constexpr int WAVES = WIDE ? 1 : QueryShape<T, DH, NW, NG>::WAVES;
};

template <typename T, int DH, int NW, int NG>
__global__ __launch_bounds__(NW * NG * 64, (DqShape<T, DH, NW, NG>::WAVES)) void seq_dq_kernel(
    const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v,
    const int* __restrict__ cu, const T* __restrict__ o, const float* __restrict__ lse,
    const T* __restrict__ dout, T* __restrict__ dq, float* __restrict__ delta, int total, int nseq,
    int H, int G, int wph, int64_t ldq, int64_t ldk, int64_t ldv, int64_t ldo, float sl2,
    float scale) {
  typedef typename Frag<T>::type F;
  typedef Tile<T, DH> TL;
  constexpr int NQ = QueryShape<T, DH, NW, NG>::NQ, NS = DqShape<T, DH, NW, NG>::NS;
  constexpr int KS = DH >= 32 ? DH / 32 : 1, NJ = DH / 16;
  constexpr int NI = kPairLoads<T, DH, NW>;
  constexpr int JB = NJ > 4 ? 4 : NJ;  // column operands read at once
  __shared__ __attribute__((aligned(1024))) T ring[NG][NS][2][64 * DH];
  const int lane = threadIdx.x & 63, wave = wave_index() % NW, team = wave_index() / NW;
  T(*lds)[2][64 * DH] = ring[team];
  const int lr = lane & 15, lg = lane >> 4;
  const int QT = wph * 16 * NQ, hp = NW / wph, HG = H / hp;
  const int wq = wave % wph;
  const int h = (int)(blockIdx.x % HG) * hp + wave / wph;
  const SeqTile st = find_item<false>(cu, nseq, total, QT, (int)(blockIdx.x / HG));
  const int bs = st.begin, be = st.end, q0 = bs + st.tile * QT;
  if (st.tile < 0 || q0 >= be) return;
  const int j = h / G;
  const T* kb = k + j * DH;
  const T* vb = v + j * DH;
  int tq[NQ];
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) tq[nq] = q0 + 16 * (nq & 1 ? 2 * wph - 1 - wq : wq);
  const int kend = min(be, q0 + QT);
  const int nt = (kend - bs + 63) / 64, own = (nt - team + NG - 1) / NG;  // tiles; the team's
  const PairLoads<T, DH, NW, true> load(ldk, ldv, wave, lane);
  auto issue = [&](int it, int buf) __attribute__((always_inline)) {
    load(kb, vb, bs + (it * NG + team) * 64, kend - 1, lds[buf][0], lds[buf][1]);
  };

  F qf[NQ][KS], df[NQ][KS];
  float dl[NQ], ls[NQ];
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) {
    const int t = tq[nq] + lr;
    float part = 0.f;
#pragma unroll
    for (int ds = 0; ds < KS; ++ds) {
      qf[nq][ds] = TL::row_global(q + (int64_t)t * ldq + h * DH, ds, lane, t < be);
      df[nq][ds] = TL::row_global(dout + (int64_t)t * ldo + h * DH, ds, lane, t < be);
      const F of = TL::row_global(o + (int64_t)t * ldo + h * DH, ds, lane, t < be);
#pragma unroll
      for (int e = 0; e < 8; ++e) part += to_f32(df[nq][ds][e]) * to_f32(of[e]);
    }
    part += __shfl_xor(part, 16, 64);
    part += __shfl_xor(part, 32, 64);
    dl[nq] = part;
    ls[nq] = t < be ? lse[(int64_t)h * total + t] * kLog2e : 0.f;
    if (team == 0 && t < be && lg == 0) delta[(int64_t)h * total + t] = part;
  }
  f32x4 da[NQ][NJ];
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
    for (int jj = 0; jj < NJ; ++jj) da[nq][jj] = f32x4{0.f, 0.f, 0.f, 0.f};

  constexpr unsigned BUF = 2 * 64 * DH * sizeof(T);
  const unsigned krow = TL::row_base(lds[0][0], lr, lane), vrow = TL::row_base(lds[0][1], lr, lane);
  const ColBase<T> kcol = TL::col_base(lds[0][0], lane);
  auto tile = [&](auto masked, int kt, int buf) __attribute__((always_inline)) {
    constexpr bool MASK = decltype(masked)::value;
    const unsigned ba = buf * BUF;
    bool live[NQ];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq)
      live[nq] = !MASK || !(tq[nq] >= be || tq[nq] + 15 < kt);  // wave-uniform
    // 32 keys at a time: scores and dp of two key groups, then their part of dQ
    each<2>([&](auto us) __attribute__((always_inline)) {
      f32x4 s[NQ][2];
      each<2>([&](auto k2) __attribute__((always_inline)) {
        constexpr int ku = us * 2 + k2;
        RowRaw<T> kr[KS], vr[KS];
        each<KS>([&](auto ds) {
          kr[ds] = TL::template row_at<ds, ku * 16>(krow + ba);
          vr[ds] = TL::template row_at<ds, ku * 16>(vrow + ba);
        });
        lds_tr_wait();
        F kf[KS], vf[KS];
#pragma unroll
        for (int ds = 0; ds < KS; ++ds) {
          kf[ds] = TL::take_row(kr[ds], lane);
          vf[ds] = TL::take_row(vr[ds], lane);
        }
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
          f32x4 sv = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ds = 0; ds < KS; ++ds) {
            sv = TL::mma(kf[ds], qf[nq][ds], sv);
            dp = TL::mma(vf[ds], df[nq][ds], dp);
          }
          const int t_eff = min(tq[nq] + lr, be - 1);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float z = exp2_fast(fmaf(sv[r], sl2, -ls[nq])) * (dp[r] - dl[nq]);
            s[nq][k2][r] = !MASK || kt + ku * 16 + lg * 4 + r <= t_eff ? z : 0.f;
          }
        }
      });
      F zf[NQ];
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) zf[nq] = frag_from<T>(s[nq][0], s[nq][1]);
      each<NJ / JB>([&](auto jb) __attribute__((always_inline)) {
        ColRaw<T> kr[JB];
        each<JB>([&](auto jj) {
          kr[jj] = TL::template col_at<jb * JB + jj, us * 32, us * 32 + 16>(kcol, ba);
        });
        lds_tr_wait();
#pragma unroll
        for (int jj = 0; jj < JB; ++jj) {
          const F kc = take(kr[jj]);
#pragma unroll
          for (int nq = 0; nq < NQ; ++nq)
            if (live[nq]) da[nq][jb * JB + jj] = mma16(kc, zf[nq], da[nq][jb * JB + jj]);
        }
      });
    });
  };

#pragma unroll
  for (int i = 0; i < NS - 1; ++i)
    if (i < own) issue(i, i);
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) {
    settle(ls[nq]);
#pragma unroll
    for (int ds = 0; ds < KS; ++ds) {
      settle(qf[nq][ds]);
      settle(df[nq][ds]);
    }
  }
  int buf = 0, next = NS - 1;
  for (int it = 0; it * NG < nt; ++it) {
    if (it + NS - 2 < own) vm_wait<(NS - 2) * NI>();
    else vm_wait<0>();
    wg_barrier();  // tile it is there, and every wave is done with the one before
    if (it + NS - 1 < own) issue(it + NS - 1, next);
    const int kt = bs + (it * NG + team) * 64;
    if (kt + 63 <= tq[0]) tile(std::false_type{}, kt, buf);
    else if (kt <= min(tq[NQ - 1] + 15, be - 1)) tile(std::true_type{}, kt, buf);
    buf = buf + 1 == NS ? 0 : buf + 1;
    next = next + 1 == NS ? 0 : next + 1;
  }
  if constexpr (NG == 2) {
    typedef f32x4 Part[NQ][NJ][64];
    static_assert(sizeof(Part) * NW <= sizeof(ring), "the parts lie in the ring");
    Part* part = (Part*)&ring[0][0][0][0] + wave;
    wg_barrier();  // every wave is done with its last tile
    if (team == 1) {
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
        for (int jj = 0; jj < NJ; ++jj) (*part)[nq][jj][lane] = da[nq][jj];
    }
    __syncthreads();
    if (team == 1) return;
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
      for (int jj = 0; jj < NJ; ++jj) da[nq][jj] += (*part)[nq][jj][lane];
  }
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) {
    const int t = tq[nq] + lr;
    if (t < be) {
      T* p = dq + (int64_t)t * ldq + h * DH + lg * 4;
#pragma unroll
      for (int jj = 0; jj < NJ; ++jj)
        store4(p + jj * 16, da[nq][jj][0] * scale, da[nq][jj][1] * scale, da[nq][jj][2] * scale,
               da[nq][jj][3] * scale);
    }
  }
}

// ------------------------------------------------------------------ backward: dK, dV
// A workgroup owns 64 NK keys of one key/value head and walks the steps (query
// head of the group, tile of 64 queries at or after its keys).  NH teams of four
// waves take the steps in turn and are joined at the end, so that a SIMD has
// two waves and the keys with the most queries behind them are done sooner.
// Shared heads are summed in registers, in a fixed order; where there are too
// few workgroups for the chip, several take the steps of the same keys in turn
// and leave float32 sums that a second kernel adds.  In bfloat16 the weights and dz
// are rounded to the type as operands, as in the other two passes.

template <typename T, int DH> struct KeyShape {
  static constexpr int NK = sizeof(T) == 2 ? 2 : 1;  // groups of 16 keys of a wave
  static constexpr int NH = sizeof(T) * DH > 128 ? 1 : 2;
  static constexpr int NS = sizeof(T) * DH >= 512 ? 2 : 3;  // buffers of the ring
};

template <typename T, int DH>
__global__ __launch_bounds__((KeyShape<T, DH>::NH * 256)) void seq_dkdv_kernel(
    const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v,
    const int* __restrict__ cu, const float* __restrict__ lse, const float* __restrict__ delta,
    const T* __restrict__ dout, T* __restrict__ dk, T* __restrict__ dv, float* __restrict__ part,
    int parts, int total, int nseq, int H, int G, int64_t ldq, int64_t ldk, int64_t ldv,
    int64_t ldo, float sl2, float scale) {
  typedef typename Frag<T>::type F;
  typedef Tile<T, DH> TL;
  constexpr int NK = KeyShape<T, DH>::NK, NH = KeyShape<T, DH>::NH, NS = KeyShape<T, DH>::NS;
  constexpr int NW = 4, KT = NW * 16 * NK, KS = DH >= 32 ? DH / 32 : 1, NJ = DH / 16;
  constexpr int NI = kPairLoads<T, DH, NW> + 1;
  constexpr int JB = sizeof(T) == 2 ? NJ : NJ > 2 ? 2 : NJ;  // column operands read at once
  constexpr int RING = NS * NH * 2 * 64 * DH, JOIN = NH > 1 ? 2 * NW * NK * NJ * 64 * 4 : 0;
  constexpr int LDS = RING * (int)sizeof(T) > JOIN * 4 ? RING : JOIN * 4 / (int)sizeof(T);
  __shared__ __attribute__((aligned(1024))) T lds[LDS];
  __shared__ __attribute__((aligned(16))) float rows[NS][NH][NW][64];  // lse, delta: waves 0, 1
  const int lane = threadIdx.x & 63, wave = wave_index() % NW, team = wave_index() / NW;
  const int lr = lane & 15, lg = lane >> 4;
  const int Hkv = H / G;
  const int j = blockIdx.x % Hkv, pt = blockIdx.x / Hkv % parts;
  const SeqTile st = find_item<true>(cu, nseq, total, KT, (int)(blockIdx.x / (Hkv * parts)));
  const int be = st.end, k0 = st.begin + st.tile * KT;
  if (st.tile < 0 || k0 >= be) return;
  const int nt1 = (be - k0 + 63) / 64, nstep = nt1 * G;  // query tiles of a head, of all
  const int nt = (nstep + NH * (parts - pt) - 1) / (NH * parts);  // rounds of this part's teams

  int uk[NK];
  F kf[NK][KS], vf[NK][KS];
  f32x4 ka[NK][NJ], va[NK][NJ];
#pragma unroll
  for (int nk = 0; nk < NK; ++nk) {
    uk[nk] = k0 + 16 * (nk & 1 ? 2 * NW - 1 - wave : wave);
    const int u = uk[nk] + lr;
#pragma unroll
    for (int ds = 0; ds < KS; ++ds) {
      kf[nk][ds] = TL::row_global(k + (int64_t)u * ldk + j * DH, ds, lane, u < be);
      vf[nk][ds] = TL::row_global(v + (int64_t)u * ldv + j * DH, ds, lane, u < be);
    }
#pragma unroll
    for (int jj = 0; jj < NJ; ++jj) {
      ka[nk][jj] = f32x4{0.f, 0.f, 0.f, 0.f};
      va[nk][jj] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  constexpr int TILE = 64 * DH;
  const PairLoads<T, DH, NW, (DH <= 32)> load(ldq, ldo, wave, lane);
  // the team's step of a round into a buffer (beyond the last step: the last one again)
  auto issue = [&](int it, int buf) __attribute__((always_inline)) {
    const int step = min((it * parts + pt) * NH + team, nstep - 1);
    const int h = j * G + step / nt1, tt = k0 + (step % nt1) * 64;
    T* t = lds + (buf * NH + team) * 2 * TILE;
    load(q + h * DH, dout + h * DH, tt, be - 1, t, t + TILE);
    const float* src = (wave & 1 ? delta : lse) + (int64_t)h * total + min(tt + lane, be - 1);
    __builtin_amdgcn_global_load_lds(src, (lds_void_t*)rows[buf][team][wave], 4, 0, 0);
  };
  constexpr unsigned BUF = NH * 2 * TILE * sizeof(T);
  T* mine = lds + team * 2 * TILE;
  const unsigned qrow = TL::row_base(mine, lr, lane), drow = TL::row_base(mine + TILE, lr, lane);
  const ColBase<T> qcol = TL::col_base(mine, lane), dcol = TL::col_base(mine + TILE, lane);
  const unsigned lrow = lds_addr(&rows[0][team][0][lg * 4]);
  const unsigned dlrow = lds_addr(&rows[0][team][1][lg * 4]);

  auto tile = [&](auto masked, int tt, int buf) __attribute__((always_inline)) {
    constexpr bool MASK = decltype(masked)::value;
    const unsigned ba = buf * BUF, br = buf * (NH * NW * 64 * 4);
    bool live[NK];
#pragma unroll
    for (int nk = 0; nk < NK; ++nk)
      live[nk] = !MASK || !(uk[nk] >= be || tt + 63 < uk[nk]);  // wave-uniform
    // 32 queries at a time
    each<2>([&](auto us) __attribute__((always_inline)) {
      f32x4 p[NK][2], z[NK][2];
      each<2>([&](auto t2) __attribute__((always_inline)) {
        constexpr int ts = us * 2 + t2;
        RowRaw<T> qr[KS], dr[KS];
        each<KS>([&](auto ds) {
          qr[ds] = TL::template row_at<ds, ts * 16>(qrow + ba);
          dr[ds] = TL::template row_at<ds, ts * 16>(drow + ba);
        });
        f32x4 ls = lds_read_f32x4_at<ts * 64>(lrow + br);
        f32x4 dl = lds_read_f32x4_at<ts * 64>(dlrow + br);
        lds_tr_wait();
        F qf[KS], df[KS];
#pragma unroll
        for (int ds = 0; ds < KS; ++ds) {
          qf[ds] = TL::take_row(qr[ds], lane);
          df[ds] = TL::take_row(dr[ds], lane);
        }
        lds_tr_bind(ls);
        lds_tr_bind(dl);
        ls *= -kLog2e;
#pragma unroll
        for (int nk = 0; nk < NK; ++nk) {
          f32x4 sv = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ds = 0; ds < KS; ++ds) {
            sv = TL::mma(qf[ds], kf[nk][ds], sv);
            dp = TL::mma(df[ds], vf[nk][ds], dp);
          }
          const int u = uk[nk] + lr;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float pv = exp2_fast(fmaf(sv[r], sl2, ls[r])), zv = pv * (dp[r] - dl[r]);
            const int t = tt + ts * 16 + lg * 4 + r;
            const bool ok = !MASK || (t >= u && t < be);
            p[nk][t2][r] = ok ? pv : 0.f;
            z[nk][t2][r] = ok ? zv : 0.f;
          }
        }
      });
      F pf[NK], zf[NK];
#pragma unroll
      for (int nk = 0; nk < NK; ++nk) {
        pf[nk] = frag_from<T>(p[nk][0], p[nk][1]);
        zf[nk] = frag_from<T>(z[nk][0], z[nk][1]);
      }
      each<NJ / JB>([&](auto jb) __attribute__((always_inline)) {
        ColRaw<T> dr[JB], qr[JB];
        each<JB>([&](auto jj) {
          dr[jj] = TL::template col_at<jb * JB + jj, us * 32, us * 32 + 16>(dcol, ba);
          qr[jj] = TL::template col_at<jb * JB + jj, us * 32, us * 32 + 16>(qcol, ba);
        });
        lds_tr_wait();
#pragma unroll
        for (int jj = 0; jj < JB; ++jj) {
          const F dc = take(dr[jj]), qc = take(qr[jj]);
#pragma unroll
          for (int nk = 0; nk < NK; ++nk)
            if (live[nk]) {
              va[nk][jb * JB + jj] = mma16(dc, pf[nk], va[nk][jb * JB + jj]);
              ka[nk][jb * JB + jj] = mma16(qc, zf[nk], ka[nk][jb * JB + jj]);
            }
        }
      });
    });
  };

#pragma unroll
  for (int i = 0; i < NS - 1; ++i)
    if (i < nt) issue(i, i);
#pragma unroll
  for (int nk = 0; nk < NK; ++nk)
#pragma unroll
    for (int ds = 0; ds < KS; ++ds) {
      settle(kf[nk][ds]);
      settle(vf[nk][ds]);
    }
  int buf = 0, next = NS - 1;
  for (int it = 0; it < nt; ++it) {
    if (it + NS - 2 < nt) vm_wait<(NS - 2) * NI>();
    else vm_wait<0>();
    wg_barrier();  // the round's steps are there, and every wave is done with those before
    if (it + NS - 1 < nt) issue(it + NS - 1, next);
    const int step = (it * parts + pt) * NH + team, tt = k0 + (step % nt1) * 64;
    if (step < nstep && uk[0] < be) {
      if (tt >= uk[NK - 1] + 15 && tt + 64 <= be) tile(std::false_type{}, tt, buf);
      else if (tt + 63 >= uk[0]) tile(std::true_type{}, tt, buf);
    }
    buf = buf + 1 == NS ? 0 : buf + 1;
    next = next + 1 == NS ? 0 : next + 1;
  }
  if constexpr (NH > 1) {
    wg_barrier();  // every wave is done with the ring
    f32x4* join = (f32x4*)lds;
    if (team == 1) {
#pragma unroll
      for (int nk = 0; nk < NK; ++nk)
#pragma unroll
        for (int jj = 0; jj < NJ; ++jj) {
          join[((wave * NK + nk) * NJ + jj) * 64 + lane] = ka[nk][jj];
          join[(((NW + wave) * NK + nk) * NJ + jj) * 64 + lane] = va[nk][jj];
        }
    }
    __syncthreads();
    if (team == 1) return;
#pragma unroll
    for (int nk = 0; nk < NK; ++nk)
#pragma unroll
      for (int jj = 0; jj < NJ; ++jj) {
        ka[nk][jj] += join[((wave * NK + nk) * NJ + jj) * 64 + lane];
        va[nk][jj] += join[(((NW + wave) * NK + nk) * NJ + jj) * 64 + lane];
      }
  }
#pragma unroll
  for (int nk = 0; nk < NK; ++nk) {
    const int u = uk[nk] + lr;
    if (u < be) {
      if (parts > 1) {
        float* p = part + (((int64_t)pt * total + u) * Hkv + j) * 2 * DH + lg * 4;
#pragma unroll
        for (int jj = 0; jj < NJ; ++jj) {
          *(f32x4*)(p + jj * 16) = ka[nk][jj] * scale;
          *(f32x4*)(p + DH + jj * 16) = va[nk][jj];
        }
        continue;
      }
      T* pk = dk + (int64_t)u * ldk + j * DH + lg * 4;
      T* pv = dv + (int64_t)u * ldv + j * DH + lg * 4;
#pragma unroll
      for (int jj = 0; jj < NJ; ++jj) {
        store4(pk + jj * 16, ka[nk][jj][0] * scale, ka[nk][jj][1] * scale, ka[nk][jj][2] * scale,
               ka[nk][jj][3] * scale);
        store4(pv + jj * 16, va[nk][jj][0], va[nk][jj][1], va[nk][jj][2], va[nk][jj][3]);
      }
    }
  }
}

// dK and dV of the rows of all sequences from the parts of their heads: DH / 2
// threads a row and head, four values each.
template <typename T, int DH>
__global__ __launch_bounds__(256) void seq_dkdv_sum_kernel(const int* __restrict__ cu,
                                                           const float* __restrict__ part,
                                                           int parts, T* __restrict__ dk,
                                                           T* __restrict__ dv, int total, int nseq,
                                                           int Hkv, int64_t ldk, int64_t ldv) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n = (int64_t)total * Hkv * (DH / 2);
  if (i >= n) return;
  const int c = (int)(i % (DH / 2)) * 4;
  const int64_t r = i / (DH / 2);
  const int j = (int)(r % Hkv), u = (int)(r / Hkv);
  if (u < cu[0] || u >= cu[nseq]) return;
  f32x4 s = *(const f32x4*)(part + r * 2 * DH + c);
  for (int p = 1; p < parts; ++p)
    s += *(const f32x4*)(part + ((int64_t)p * total * Hkv + r) * 2 * DH + c);
  if (c < DH) store4(dk + (int64_t)u * ldk + j * DH + c, s[0], s[1], s[2], s[3]);
  else store4(dv + (int64_t)u * ldv + j * DH + c - DH, s[0], s[1], s[2], s[3]);
}

// Waves per head of a workgroup of NW: as many heads of a group share it as
// divide the group, since their queries see the same keys; a power of two of them,
// so that a group of 3 heads shares nothing.  Four sequences of 2048, 12 heads of 64
// on 12, 4 and 3 (groups of 1, 3 and 4): forward 52, 51 and 51 us, gradients 149,
// 150 and 158: the keys' traffic does not bound these.
int waves_per_head(int NW, int G) {
  int hp = NW;
  while (G % hp) hp /= 2;
  return NW / hp;
}
int64_t query_grid(int NW, int NQ, const SeqAttn& a) {
  const int wph = waves_per_head(NW, a.H / a.Hkv);
  return (int64_t)(a.total / (wph * 16 * NQ) + a.nseq) * (a.H * wph / NW);
}
// Eight waves a workgroup (less traffic per query) once they make four rounds
// over the CUs, else four (16 heads of 128 on 2, forward, 8 against 4 waves: 4096
// rows 145 and 121 us, 16384 rows 624 and 685, 32768 rows 4.74 and 5.38 ms).
bool wide_queries(DType dt, const SeqAttn& a) {
  return dt == DType::BF16 && query_grid(8, 2, a) >= 1024;
}

template <typename T, int DH, int NW, int NG = 1>
hipError_t fwd_nw(const SeqAttn& a, hipStream_t s) {
  const int64_t grid = query_grid(NW, QueryShape<T, DH, NW, NG>::NQ, a);
  const int G = a.H / a.Hkv;
  seq_fwd_kernel<T, DH, NW, NG><<<dim3((unsigned)grid), NW * NG * 64, 0, s>>>(
      (const T*)a.q, (const T*)a.k, (const T*)a.v, a.cu, (T*)a.o, a.lse, a.total, a.nseq, a.H, G,
      waves_per_head(NW, G), a.ldq, a.ldk, a.ldv, a.ldo, a.scale * kLog2e);
  return hipGetLastError();
}
template <typename T, int DH, int NW, int NG = 1>
hipError_t dq_nw(const SeqAttn& a, hipStream_t s) {
  const int64_t grid = query_grid(NW, QueryShape<T, DH, NW, NG>::NQ, a);
  const int G = a.H / a.Hkv;
  seq_dq_kernel<T, DH, NW, NG><<<dim3((unsigned)grid), NW * NG * 64, 0, s>>>(
      (const T*)a.q, (const T*)a.k, (const T*)a.v, a.cu, (const T*)a.o, a.lse, (const T*)a.dout,
      (T*)a.dq, a.delta, a.total, a.nseq, a.H, G, waves_per_head(NW, G), a.ldq, a.ldk, a.ldv, a.ldo,
      a.scale * kLog2e, a.scale);
  return hipGetLastError();
}

// Two teams of waves, which take the tiles of keys in turn and are joined at the end,
// where the workgroups of one team are no more than two for a CU: half as many tiles
// one after another, no fewer waves on a CU.  One sequence of 4096, 8 heads of 64 in
// bfloat16 (256 workgroups): forward 55 us, 73 with one team, the whole gradient 148
// and 170; 16 heads of 128 on 2 (512): forward 99 and 122; two of 3000, 12 heads of 64
// (552): 65 and 58, 180 and 169.  Float32 heads of 64, whose tiles leave a CU room for
// one workgroup only, take them always: eight sequences of 2048, 12 heads: 544 and 621
// us, 1853 and 1912 (of 32: 629 and 512).  Sequences of one tile have nothing to share.
template <typename T, int DH>
bool two_teams(const SeqAttn& a) {
  constexpr int NQ = sizeof(T) == 2 ? 2 : 1;
  const int wph = waves_per_head(4, a.H / a.Hkv);
  const int64_t grid = (int64_t)(a.total / (wph * 16 * NQ)) * (a.H * wph / 4);
  return a.total > 64 * (int64_t)a.nseq && (grid <= 512 || (sizeof(T) == 4 && DH == 64));
}

template <typename T, int DH>
hipError_t fwd_t(const SeqAttn& a, hipStream_t s) {
  if constexpr (sizeof(T) == 2)
    if (wide_queries(DType::BF16, a)) return fwd_nw<T, DH, 8>(a, s);
  if constexpr (sizeof(T) * DH <= 256)  // (float32 heads of 128: their LDS is full)
    if (two_teams<T, DH>(a)) return fwd_nw<T, DH, 4, 2>(a, s);
  return fwd_nw<T, DH, 4>(a, s);
}

template <typename T, int DH>
hipError_t dq_t(const SeqAttn& a, hipStream_t s) {
  if constexpr (DH <= 64) {
    if constexpr (sizeof(T) == 2)
      if (wide_queries(DType::BF16, a)) return dq_nw<T, DH, 8>(a, s);
    if (two_teams<T, DH>(a)) return dq_nw<T, DH, 4, 2>(a, s);
  }
  return dq_nw<T, DH, 4>(a, s);
}

// Parts of the steps for dK and dV, until there are two workgroups for every CU (the
// whole gradient of four sequences of 2048, 16 heads of 64 on 4: 179 us, 200 with
// four, 244 with no parts; of one of 4096, 16 heads of 128 on 2: 405, the same, 1747).
// As many as the group has heads; more, up to 16, while a part has 8 rounds of its
// teams (float32: 4, which take longer): a part costs the traffic of its float32 sums
// (one sequence of 4096, 8 heads of 64 in bfloat16: 131 us with two parts, 146 with
// one; two of 1024: 55 with four and 48 with one).  The rounds are those of a sequence
// of the mean length, since the host does not see the lengths: a long sequence among
// short ones gets as few parts as they do.
template <typename T, int DH>
int parts_t(int total, int nseq, int Hkv, int G) {
  typedef KeyShape<T, DH> KS;
  const int64_t wgs = ((int64_t)total / (64 * KS::NK) + nseq) * Hkv;
  const int64_t rounds = (int64_t)total * G / ((int64_t)64 * nseq * KS::NH);
  const int64_t most = std::max<int64_t>(G, std::min<int64_t>(rounds / (sizeof(T) == 2 ? 8 : 4), 16));
  return (int)std::min((512 + wgs - 1) / wgs, most);
}

template <typename T, int DH>
hipError_t bwd_t(const SeqAttn& a, hipStream_t s) {
  const int G = a.H / a.Hkv;
  hipError_t e = dq_t<T, DH>(a, s);
  if (e != hipSuccess) return e;
  constexpr int KT = 64 * KeyShape<T, DH>::NK;
  const int parts = parts_t<T, DH>(a.total, a.nseq, a.Hkv, G);
  const int64_t grid = (int64_t)(a.total / KT + a.nseq) * a.Hkv * parts;
  seq_dkdv_kernel<T, DH><<<dim3((unsigned)grid), KeyShape<T, DH>::NH * 256, 0, s>>>(
      (const T*)a.q, (const T*)a.k, (const T*)a.v, a.cu, a.lse, a.delta, (const T*)a.dout,
      (T*)a.dk, (T*)a.dv, a.part, parts, a.total, a.nseq, a.H, G, a.ldq, a.ldk, a.ldv, a.ldo,
      a.scale * kLog2e, a.scale);
  e = hipGetLastError();
  if (e != hipSuccess || parts == 1) return e;
  const int64_t n = (int64_t)a.total * a.Hkv * (DH / 2);
  seq_dkdv_sum_kernel<T, DH><<<dim3((unsigned)((n + 255) / 256)), 256, 0, s>>>(
      a.cu, a.part, parts, (T*)a.dk, (T*)a.dv, a.total, a.nseq, a.Hkv, a.ldk, a.ldv);
  return hipGetLastError();
}

// ------------------------------------------------------------------ single tokens
// One workgroup per (sequence, key/value head, 16 query heads of its group,
// part of the cache).  The heads of the group are the columns of the score
// product, so each cache row is read once for all of them.  Every wave walks
// its own tiles of KT keys through its own LDS (no barriers), and the waves'
// maxima, sums and outputs are joined at the end.  The token's own key and
// value are put into the tile that holds its position, whose later rows are
// cleared (the cache may hold anything there); the wave that owns the tile
// also writes them to the cache.  Weights are rounded to bfloat16 as in the prompt's
// pass, with the same error (2.0e-3 to 2.1e-3 in the 2-norm).

template <typename T, int DH> struct DecShape {
  // LDS of two buffers of K and V tiles per wave
  static constexpr int KT = 32;
  static constexpr int NW = (int)sizeof(T) * DH >= 512 ? 2 : 4;
};

template <typename T, int DH>
__global__ __launch_bounds__((DecShape<T, DH>::NW * 64)) void dec_part_kernel(DecAttn a) {
  typedef typename Frag<T>::type F;
  typedef Tile<T, DH> TL;
  constexpr int KT = DecShape<T, DH>::KT, NW = DecShape<T, DH>::NW;
  constexpr int KS = DH >= 32 ? DH / 32 : 1, NJ = DH / 16;
  constexpr int NI = KT * TL::NCH / 64;  // loads of a tile
  static_assert(NI >= 1 && NI * 64 == KT * TL::NCH, "tile loads");
  __shared__ __attribute__((aligned(1024))) T lds[NW][2][2][KT * DH];
  __shared__ float red_m[NW][16], red_l[NW][16];
  const int lane = threadIdx.x & 63, wave = wave_index();
  const int lr = lane & 15, lg = lane >> 4;
  const int G = a.H / a.Hkv, NH = (G + 15) / 16;
  const int part = blockIdx.x, y = blockIdx.y;
  const int hg = y % NH, j = (y / NH) % a.Hkv, b = y / NH / a.Hkv;
  const int slot = a.slot ? a.slot[b] : b, n = a.length[b];
  const int h = j * G + hg * 16 + lr;      // this lane's query head
  const bool hok = hg * 16 + lr < G;
  if (slot < 0 || slot >= a.slots || n < 0 || n >= a.cap) {
    if (part == 0 && a.nsplit == 1 && wave == 0 && hok)
      for (int jj = 0; jj < NJ; ++jj)
        store4((T*)a.o + (int64_t)b * a.ldo + h * DH + jj * 16 + lg * 4, 0.f, 0.f, 0.f, 0.f);
    return;
  }
  const int ntile = n / KT + 1;  // rows 0 .. n
  const int per = (ntile + a.nsplit - 1) / a.nsplit;
  const int t0 = part * per, t1 = min(t0 + per, ntile);
  if (t0 >= t1) return;
  T* kc = (T*)a.kcache + slot * a.cs + j * a.ch;
  T* vc = (T*)a.vcache + slot * a.cs + j * a.ch;
  const T* kn = (const T*)a.k + (int64_t)b * a.ldk + j * DH;
  const T* vn = (const T*)a.v + (int64_t)b * a.ldv + j * DH;

  F qf[KS];
#pragma unroll
  for (int ds = 0; ds < KS; ++ds)
    qf[ds] = TL::row_global((const T*)a.q + (int64_t)b * a.ldq + h * DH, ds, lane, hok);
  float m = -INFINITY, l = 0.f;
  f32x4 oa[NJ];
#pragma unroll
  for (int jj = 0; jj < NJ; ++jj) oa[jj] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto issue = [&](int t, int buf) {
#pragma unroll
    for (int i = 0; i < NI; ++i) TL::issue(kc, a.ct, t * KT, n, lds[wave][buf][0], i, lane);
#pragma unroll
    for (int i = 0; i < NI; ++i) TL::issue(vc, a.ct, t * KT, n, lds[wave][buf][1], i, lane);
  };
  const unsigned krow = TL::row_base(lds[wave][0][0], lr, lane);
  const ColBase<T> vcol = TL::col_base(lds[wave][0][1], lane);
  int t = t0 + wave, buf = 0;
  if (t < t1) issue(t, 0);
  if (t + NW < t1) issue(t + NW, 1);
#pragma unroll
  for (int ds = 0; ds < KS; ++ds) settle(qf[ds]);
  for (; t < t1; t += NW, buf ^= 1) {
    if (t + NW < t1) vm_wait<2 * NI>();
    else vm_wait<0>();
    T* Kt = lds[wave][buf][0];
    T* Vt = lds[wave][buf][1];
    if (t * KT + KT > n) {  // the tile of position n
      for (int id = lane; id < KT * TL::NCH; id += 64) {
        const int r = id / TL::NCH, c = (id % TL::NCH) * TL::CH, u = t * KT + r;
        if (u < n) continue;
        typename Vec16<T>::type kv = {}, vv = {};
        if (u == n) {
          kv = load16(kn + c);
          vv = load16(vn + c);
          if (hg == 0) {
            store16(kc + (int64_t)n * a.ct + c, kv);
            store16(vc + (int64_t)n * a.ct + c, vv);
          }
        }
        store16(Kt + TL::off(r, c), kv);
        store16(Vt + TL::off(r, c), vv);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    f32x4 s[2];
    const unsigned ba = buf * 2 * KT * DH * sizeof(T);
    ColRaw<T> vr[NJ];
    each<2>([&](auto ku) {
      RowRaw<T> kr[KS];
      each<KS>([&](auto ds) { kr[ds] = TL::template row_at<ds, ku * 16>(krow + ba); });
      lds_tr_wait();
      s[ku] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ds = 0; ds < KS; ++ds) s[ku] = TL::mma(TL::take_row(kr[ds], lane), qf[ds], s[ku]);
    });
    each<NJ>([&](auto jj) { vr[jj] = TL::template col_at<jj, 0, 16>(vcol, ba); });
    float mx = -INFINITY;
#pragma unroll
    for (int ku = 0; ku < 2; ++ku)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int u = t * KT + ku * 16 + lg * 4 + r;
        s[ku][r] = u <= n ? s[ku][r] * a.sl2 : -INFINITY;
        mx = fmaxf(mx, s[ku][r]);
      }
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float mnew = fmaxf(m, mx);
    const float ms = mnew == -INFINITY ? 0.f : mnew;
    const float alpha = exp2_fast(m - ms);
    float ps = 0.f;
#pragma unroll
    for (int ku = 0; ku < 2; ++ku)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[ku][r] = exp2_fast(s[ku][r] - ms);
        ps += s[ku][r];
      }
    l = l * alpha + ps;
    m = mnew;
    const F pf = frag_from<T>(s[0], s[1]);
    lds_tr_wait();
#pragma unroll
    for (int jj = 0; jj < NJ; ++jj) oa[jj] = mma16(take(vr[jj]), pf, oa[jj] * alpha);
    if (t + 2 * NW < t1) issue(t + 2 * NW, buf);
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);

  // join the waves: the weights of each wave's maximum, then the outputs
  // through the first wave's own tiles (every wave is past its loop)
  if (lg == 0) {
    red_m[wave][lr] = m;
    red_l[wave][lr] = l;
  }
  __syncthreads();
  float mm = -INFINITY, lt = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) mm = fmaxf(mm, red_m[w][lr]);
  const float msafe = mm == -INFINITY ? 0.f : mm;
#pragma unroll
  for (int w = 0; w < NW; ++w) lt += red_l[w][lr] * exp2_fast(red_m[w][lr] - msafe);
  const float wgt = exp2_fast(m - msafe);
  float* acc = (float*)&lds[0][0][0][0];  // [NW][16][DH] floats
  static_assert((size_t)NW * 16 * DH * 4 <= sizeof(T) * NW * 4 * KT * DH, "join buffer");
#pragma unroll
  for (int jj = 0; jj < NJ; ++jj)
    store4(acc + (wave * 16 + lr) * DH + jj * 16 + lg * 4, oa[jj][0] * wgt, oa[jj][1] * wgt,
           oa[jj][2] * wgt, oa[jj][3] * wgt);
  __syncthreads();
  if (wave == 0 && lg == 0) {
    red_m[0][lr] = mm;
    red_l[0][lr] = lt;
  }
  __syncthreads();
  const int heads = min(16, G - hg * 16);
  for (int i = threadIdx.x; i < heads * (DH / 4); i += NW * 64) {
    const int hh = i / (DH / 4), c = (i % (DH / 4)) * 4;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) v += *(const f32x4*)(acc + (w * 16 + hh) * DH + c);
    const int head = j * G + hg * 16 + hh;
    if (a.nsplit == 1) {
      const float inv = 1.0f / red_l[0][hh];
      store4((T*)a.o + (int64_t)b * a.ldo + head * DH + c, v[0] * inv, v[1] * inv, v[2] * inv,
             v[3] * inv);
    } else {
      const int64_t row = ((int64_t)b * a.H + head) * a.nsplit + part;
      *(f32x4*)(a.part_o + row * DH + c) = v;
      if (c == 0) {
        a.part_ml[row * 2] = red_m[0][hh];
        a.part_ml[row * 2 + 1] = red_l[0][hh];
      }
    }
  }
}

// Joins the parts of one (sequence, head): DH / 4 lanes for the columns, as many
// groups of them as a workgroup has take the parts in turn, eight loads at a time
// (one sequence of 32768 positions, 4 heads of 64, 128 parts: 13 us for the step,
// 52 with the parts one after another).
template <typename T, int DH>
__global__ __launch_bounds__(256) void dec_join_kernel(DecAttn a) {
  constexpr int KT = DecShape<T, DH>::KT, L = DH / 4, AT = 8;
  __shared__ __attribute__((aligned(16))) float acc_of[256 / L][DH];
  __shared__ float m_of[256 / L], l_of[256 / L];
  const int row = blockIdx.x, b = row / a.H, h = row % a.H;
  const int ng = blockDim.x / L, gi = threadIdx.x / L, c = (threadIdx.x % L) * 4;
  const int slot = a.slot ? a.slot[b] : b, n = a.length[b];
  T* o = (T*)a.o + (int64_t)b * a.ldo + h * DH + c;
  if (slot < 0 || slot >= a.slots || n < 0 || n >= a.cap) {
    if (gi == 0) store4(o, 0.f, 0.f, 0.f, 0.f);
    return;
  }
  const int ntile = n / KT + 1, per = (ntile + a.nsplit - 1) / a.nsplit;
  const int np = (ntile + per - 1) / per;
  const float* ml = a.part_ml + (int64_t)row * a.nsplit * 2;
  const float* po = a.part_o + (int64_t)row * a.nsplit * DH + c;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  for (int p0 = gi; p0 < np; p0 += ng * AT) {
    f32x4 x[AT];
    float mx[AT], lx[AT], mn = m;
#pragma unroll
    for (int i = 0; i < AT; ++i) {
      const int p = min(p0 + i * ng, np - 1);  // one behind the last has no weight
      mx[i] = ml[2 * p];
      lx[i] = ml[2 * p + 1];
      x[i] = *(const f32x4*)(po + (int64_t)p * DH);
    }
#pragma unroll
    for (int i = 0; i < AT; ++i) mn = fmaxf(mn, mx[i]);
    const float ms = mn == -INFINITY ? 0.f : mn, old = exp2_fast(m - ms);
    l *= old;
    acc *= old;
#pragma unroll
    for (int i = 0; i < AT; ++i)
      if (p0 + i * ng < np) {
        const float w = exp2_fast(mx[i] - ms);
        l += w * lx[i];
        acc += w * x[i];
      }
    m = mn;
  }
  *(f32x4*)&acc_of[gi][c] = acc;
  if (c == 0) {
    m_of[gi] = m;
    l_of[gi] = l;
  }
  __syncthreads();
  if (gi != 0) return;
  m = -INFINITY;
  for (int i = 0; i < ng; ++i) m = fmaxf(m, m_of[i]);
  const float ms = m == -INFINITY ? 0.f : m;
  acc = f32x4{0.f, 0.f, 0.f, 0.f};
  l = 0.f;
  for (int i = 0; i < ng; ++i) {
    const float w = exp2_fast(m_of[i] - ms);
    l += w * l_of[i];
    acc += w * *(const f32x4*)&acc_of[i][c];
  }
  const float inv = 1.0f / l;
  store4(o, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
}

template <typename T, int DH>
hipError_t dec_t(const DecAttn& a, hipStream_t s) {
  constexpr int NW = DecShape<T, DH>::NW;
  const int G = a.H / a.Hkv, NH = (G + 15) / 16;
  dec_part_kernel<T, DH><<<dim3(a.nsplit, a.B * a.Hkv * NH), NW * 64, 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.nsplit == 1) return e;
  // a wave for each row, or four where it has many parts
  dec_join_kernel<T, DH><<<dim3((unsigned)(a.B * a.H)), a.nsplit > 16 ? 256 : 64, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t seq_attn_fwd(DType dt, int dh, const SeqAttn& a, hipStream_t s) {
  BY_TYPE_AND_WIDTH(fwd_t, dt, dh, a, s);
}
hipError_t seq_attn_bwd(DType dt, int dh, const SeqAttn& a, hipStream_t s) {
  BY_TYPE_AND_WIDTH(bwd_t, dt, dh, a, s);
}
int seq_attn_bwd_parts(DType dt, int dh, int total, int nseq, int Hkv, int G) {
  BY_TYPE_AND_WIDTH(parts_t, dt, dh, total, nseq, Hkv, G);
}
hipError_t seq_attn_decode(DType dt, int dh, const DecAttn& a, hipStream_t s) {
  BY_TYPE_AND_WIDTH(dec_t, dt, dh, a, s);
}

// Parts of the cache: enough workgroups for four per CU, so that sequences of
// different lengths even out (32 of up to 8192 positions, 8 heads of 128: 111 us,
// 119 with two or eight per CU; 32 of 4096 each: 106, 105 and 119), at least two
// tiles of every wave in a part, and no more parts than CUs, since the join reads
// them all (one sequence of 131072, one head: 23 us with 256, 32 with 512).  Caches of
// at most eight tiles a wave stay whole and need no second launch: a conversation fills
// its cache, and over its course one part costs a captured graph as much as several,
// and a host that makes the calls one by one less.  In us, one sequence whose cache is
// a quarter, half, three quarters and all full, in one part | in four or more:
//   12 heads of 64,      1024: 5.5  6.9  8.2  9.5 |  7.5  7.6  8.3  8.3, from a host 8.5 to 9.5 | 11.5
//                        2048: 6.9  9.5 12.1 14.9 |  7.7  7.8  8.5  8.6,            8.4 to 14.9 | 11.5
//   32 heads of 128 on 8, 1024: 7.1  9.2 11.2 13.2 |  8.8  9.0  9.9 10.2,            8.3 to 13.1 | 11.4
//                        2048: 9.2 13.1 17.3 21.2 |  8.9  9.0 10.1 10.2,            9.3 to 21.1 | 11.4
// 32 sequences of up to 1024, 8 heads of 128: 18 us in one part and 29 in four.
int seq_attn_decode_splits(DType dt, int dh, int B, int H, int Hkv, int cap) {
  const int G = H / Hkv, NH = (G + 15) / 16;
  const int nw = (dt == DType::BF16 ? 2 : 4) * dh >= 512 ? 2 : 4;
  if (cap <= nw * 256) return 1;
  const int64_t wgs = (int64_t)B * Hkv * NH;
  const int64_t want = wgs < 4 ? 256 : (1024 + wgs - 1) / wgs, most = (cap + nw * 64 - 1) / (nw * 64);
  const int64_t n = want < most ? want : most;
  return n < 1 ? 1 : (int)n;
}

}  // namespace bcmt
