// C ABI of the sequence mixers over packed sequences: argument checks, the
// scratch plan and the launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/bcmt.h"
#include "kernels.h"

namespace bcmt {
namespace {

constexpr int kMaxTotal = 1 << 30, kMaxSeq = 65535;

size_t up256(size_t x) { return (x + 255) / 256 * 256; }
bool is16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
bool is4(const void* p) { return ((uintptr_t)p & 3u) == 0; }
DType dtype_of(int dt) { return dt == BCMT_BF16 ? DType::BF16 : DType::F32; }
int esize(int dt) { return dt == BCMT_BF16 ? 2 : 4; }

// A launch holds fewer than 2^32 threads; no kernel has more than 512 in a
// workgroup.
bool grid_ok(int64_t workgroups) { return workgroups <= (1LL << 23) - 1; }

int check_heads(int dh, int dtype, float scale) {
  if (dtype != BCMT_F32 && dtype != BCMT_BF16) return BCMT_ERR_INVALID;
  if (!std::isfinite(scale) || dh < 1) return BCMT_ERR_INVALID;
  return dh == 16 || dh == 32 || dh == 64 || dh == 128 ? BCMT_OK : BCMT_ERR_UNSUPPORTED;
}
// A row stride: 0, or at least the row and a multiple of 16 bytes.
bool stride_ok(int64_t ld, int64_t width, int es) {
  return ld == 0 || (ld >= width && ld % (16 / es) == 0 && ld <= (1LL << 28));
}

// Rows of a packed array: total rows of `width` elements, `ld` apart.
struct Rows {
  const void* p;
  int64_t ld, width;
};
bool rows_meet(const Rows& a, const Rows& b, int64_t n, int es) {
  const int64_t x = (int64_t)(uintptr_t)a.p, y = (int64_t)(uintptr_t)b.p;
  const int64_t ea = ((n - 1) * a.ld + a.width) * es, eb = ((n - 1) * b.ld + b.width) * es;
  if (x + ea <= y || y + eb <= x) return false;
  if (a.ld != b.ld) return true;
  // columns of one array: where b's row begins within a's
  const int64_t pitch = a.ld * es;
  const int64_t d = ((y - x) % pitch + pitch) % pitch;
  return d < a.width * es || d + b.width * es > pitch;
}
bool bytes_meet(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a && b && x < y + nb && y < x + na;
}
// Any of the first nout arrays meets any other.
bool any_meet(const Rows* r, int nout, int n, int64_t rows, int es) {
  for (int i = 0; i < nout; ++i)
    for (int j = i + 1; j < n; ++j)
      if (rows_meet(r[i], r[j], rows, es)) return true;
  return false;
}
// A plain array meets any of the packed ones.
bool meets_any(const void* p, size_t bytes, const Rows* r, int n, int64_t rows, int es) {
  for (int i = 0; i < n; ++i)
    if (bytes_meet(p, bytes, r[i].p, (size_t)((rows - 1) * r[i].ld + r[i].width) * es)) return true;
  return false;
}

int check_attn(const bcmt_attn_config* c) {
  if (!c || c->total < 1 || c->nseq < 1 || c->H < 1 || c->Hkv < 1 || c->H % c->Hkv != 0)
    return BCMT_ERR_INVALID;
  const int st = check_heads(c->dh, c->dtype, c->scale);
  if (st == BCMT_ERR_INVALID || !(c->scale > 0.f)) return BCMT_ERR_INVALID;
  const int es = esize(c->dtype);
  const int64_t wq = (int64_t)c->H * c->dh, wk = (int64_t)c->Hkv * c->dh;
  if (!stride_ok(c->ldq, wq, es) || !stride_ok(c->ldo, wq, es) || !stride_ok(c->ldk, wk, es) ||
      !stride_ok(c->ldv, wk, es))
    return BCMT_ERR_INVALID;
  if (st != BCMT_OK) return st;
  if (c->total > kMaxTotal || c->nseq > kMaxSeq || c->H > 65535) return BCMT_ERR_UNSUPPORTED;
  return grid_ok(((int64_t)c->total / 64 + c->nseq) * c->H) ? BCMT_OK : BCMT_ERR_UNSUPPORTED;
}

int check_decode(const bcmt_attn_decode_config* c) {
  if (!c || c->B < 1 || c->slots < 1 || c->cap < 1 || c->H < 1 || c->Hkv < 1 || c->H % c->Hkv != 0)
    return BCMT_ERR_INVALID;
  const int st = check_heads(c->dh, c->dtype, c->scale);
  if (st == BCMT_ERR_INVALID || !(c->scale > 0.f)) return BCMT_ERR_INVALID;
  const int es = esize(c->dtype);
  const int64_t wq = (int64_t)c->H * c->dh, wk = (int64_t)c->Hkv * c->dh;
  if (!stride_ok(c->ldq, wq, es) || !stride_ok(c->ldo, wq, es) || !stride_ok(c->ldk, wk, es) ||
      !stride_ok(c->ldv, wk, es))
    return BCMT_ERR_INVALID;
  if (c->cs || c->ct || c->ch) {
    for (int64_t s : {c->cs, c->ct, c->ch})
      if (s < c->dh || s % (16 / es) != 0) return BCMT_ERR_INVALID;
  }
  // the caches' extent in bytes fits 62 bits
  const double cs = c->cs ? (double)c->cs : (double)c->cap * wk;
  if (c->slots * cs + (double)c->cap * c->ct + (double)c->Hkv * c->ch > 1e18)
    return BCMT_ERR_INVALID;
  if (st != BCMT_OK) return st;
  const int nh = (c->H / c->Hkv + 15) / 16;
  if (c->cap > kMaxTotal || c->slots > kMaxTotal || (int64_t)c->B * c->Hkv * nh > 65535 || c->H > 65535)
    return BCMT_ERR_UNSUPPORTED;
  return BCMT_OK;
}

int check_lin(const bcmt_linattn_config* c) {
  if (!c || c->total < 1 || c->nseq < 1 || c->H < 1) return BCMT_ERR_INVALID;
  const int st = check_heads(c->dh, c->dtype, c->scale);
  if (st == BCMT_ERR_INVALID) return st;
  const int es = esize(c->dtype);
  const int64_t w = (int64_t)c->H * c->dh;
  for (int64_t ld : {c->ldq, c->ldk, c->ldv, c->ldo})
    if (!stride_ok(ld, w, es)) return BCMT_ERR_INVALID;
  if (st != BCMT_OK) return st;
  if (c->total > kMaxTotal || c->nseq > kMaxSeq || c->H > 65535) return BCMT_ERR_UNSUPPORTED;
  return grid_ok(((int64_t)c->total / 64 + c->nseq) * c->H) ? BCMT_OK : BCMT_ERR_UNSUPPORTED;
}

int check_step(const bcmt_linattn_step_config* c) {
  if (!c || c->B < 1 || c->slots < 1 || c->H < 1) return BCMT_ERR_INVALID;
  const int st = check_heads(c->dh, c->dtype, c->scale);
  if (st == BCMT_ERR_INVALID) return st;
  const int es = esize(c->dtype);
  const int64_t w = (int64_t)c->H * c->dh;
  for (int64_t ld : {c->ldq, c->ldk, c->ldv, c->ldo})
    if (!stride_ok(ld, w, es)) return BCMT_ERR_INVALID;
  if (st != BCMT_OK) return st;
  if (c->slots > kMaxTotal || c->H > 65535) return BCMT_ERR_UNSUPPORTED;
  return grid_ok((int64_t)c->B * c->H) ? BCMT_OK : BCMT_ERR_UNSUPPORTED;
}

// Scratch of linear attention: the states between segments (of the forward
// order, of the reverse order) and the decay gradient's partial sums.
struct LinPlan {
  int seg, nslot;
  bool cut;  // whether a sequence can have more than one segment
  size_t fwd, rev, given, part, fwd_bytes, bwd_bytes;
  explicit LinPlan(const bcmt_linattn_config& c) {
    seg = lin_segment_rows(dtype_of(c.dtype), c.total, c.nseq, c.H, c.dh);
    cut = seg < c.total;
    if (!cut) seg = (c.total + 63) / 64 * 64;
    nslot = c.total / seg + c.nseq;
    const size_t states =
        cut ? up256((size_t)(c.total / seg + 1) * c.H * c.dh * c.dh * 4) : 0;
    fwd = 0;
    given = states;
    rev = 2 * states;
    part = 3 * states;
    fwd_bytes = 2 * states;
    bwd_bytes = part + up256((size_t)c.H * nslot * (c.dh / 16) * 4);
  }
};

}  // namespace
}  // namespace bcmt

using namespace bcmt;

extern "C" {

int bcmt_attn_validate(const bcmt_attn_config* cfg) { return check_attn(cfg); }

size_t bcmt_attn_workspace_bytes(const bcmt_attn_config* cfg) {
  if (check_attn(cfg) != BCMT_OK) return 0;
  const bcmt_attn_config& c = *cfg;
  const int parts =
      seq_attn_bwd_parts(dtype_of(c.dtype), c.dh, c.total, c.nseq, c.Hkv, c.H / c.Hkv);
  return up256((size_t)c.H * c.total * 4) +
         (parts > 1 ? up256((size_t)parts * c.total * c.Hkv * 2 * c.dh * 4) : 0);
}

int bcmt_attn_forward(const bcmt_attn_config* cfg, const void* q, const void* k, const void* v,
                      const int32_t* cu, void* o, float* lse, void* stream) {
  const int st = check_attn(cfg);
  if (st != BCMT_OK) return st;
  if (!q || !k || !v || !cu || !o) return BCMT_ERR_INVALID;
  if (!is16(q) || !is16(k) || !is16(v) || !is16(o) || !is4(cu) || !is4(lse)) return BCMT_ERR_INVALID;
  const bcmt_attn_config& c = *cfg;
  const int es = esize(c.dtype);
  const int64_t wq = (int64_t)c.H * c.dh, wk = (int64_t)c.Hkv * c.dh;
  SeqAttn a{};
  a.ldq = c.ldq ? c.ldq : wq;
  a.ldk = c.ldk ? c.ldk : wk;
  a.ldv = c.ldv ? c.ldv : wk;
  a.ldo = c.ldo ? c.ldo : wq;
  const Rows r[4] = {{o, a.ldo, wq}, {q, a.ldq, wq}, {k, a.ldk, wk}, {v, a.ldv, wk}};
  const size_t nl = (size_t)c.H * c.total * 4, nc = (size_t)(c.nseq + 1) * 4;
  if (any_meet(r, 1, 4, c.total, es) || meets_any(lse, nl, r, 4, c.total, es) ||
      meets_any(cu, nc, r, 1, c.total, es) || bytes_meet(lse, nl, cu, nc))
    return BCMT_ERR_INVALID;
  a.q = q;
  a.k = k;
  a.v = v;
  a.cu = cu;
  a.o = o;
  a.lse = lse;
  a.total = c.total;
  a.nseq = c.nseq;
  a.H = c.H;
  a.Hkv = c.Hkv;
  a.scale = c.scale;
  return seq_attn_fwd(dtype_of(c.dtype), c.dh, a, (hipStream_t)stream) == hipSuccess ? BCMT_OK
                                                                                    : BCMT_ERR_HIP;
}

int bcmt_attn_backward(const bcmt_attn_config* cfg, const void* q, const void* k, const void* v,
                       const int32_t* cu, const void* o, const float* lse, const void* dO,
                       void* dq, void* dk, void* dv, void* ws, size_t ws_bytes, void* stream) {
  const int st = check_attn(cfg);
  if (st != BCMT_OK) return st;
  if (!q || !k || !v || !cu || !o || !lse || !dO || !dq || !dk || !dv || !ws)
    return BCMT_ERR_INVALID;
  for (const void* p : {q, k, v, o, dO, (const void*)dq, (const void*)dk, (const void*)dv,
                        (const void*)ws})
    if (!is16(p)) return BCMT_ERR_INVALID;
  if (!is4(cu) || !is4(lse)) return BCMT_ERR_INVALID;
  const bcmt_attn_config& c = *cfg;
  const int es = esize(c.dtype);
  const int64_t wq = (int64_t)c.H * c.dh, wk = (int64_t)c.Hkv * c.dh;
  SeqAttn a{};
  a.ldq = c.ldq ? c.ldq : wq;
  a.ldk = c.ldk ? c.ldk : wk;
  a.ldv = c.ldv ? c.ldv : wk;
  a.ldo = c.ldo ? c.ldo : wq;
  const Rows r[8] = {{dq, a.ldq, wq}, {dk, a.ldk, wk}, {dv, a.ldv, wk}, {q, a.ldq, wq},
                     {k, a.ldk, wk},  {v, a.ldv, wk},  {o, a.ldo, wq},  {dO, a.ldo, wq}};
  const size_t need = bcmt_attn_workspace_bytes(cfg), nl = (size_t)c.H * c.total * 4;
  const size_t nc = (size_t)(c.nseq + 1) * 4;
  if (any_meet(r, 3, 8, c.total, es) || meets_any(ws, need, r, 8, c.total, es) ||
      meets_any(lse, nl, r, 3, c.total, es) || meets_any(cu, nc, r, 3, c.total, es) ||
      bytes_meet(ws, need, lse, nl) || bytes_meet(ws, need, cu, nc))
    return BCMT_ERR_INVALID;
  if (ws_bytes < need) return BCMT_ERR_WORKSPACE;
  a.q = q;
  a.k = k;
  a.v = v;
  a.cu = cu;
  a.o = const_cast<void*>(o);
  a.lse = const_cast<float*>(lse);
  a.dout = dO;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  a.delta = (float*)ws;
  a.part = (float*)((char*)ws + up256((size_t)c.H * c.total * 4));
  a.total = c.total;
  a.nseq = c.nseq;
  a.H = c.H;
  a.Hkv = c.Hkv;
  a.scale = c.scale;
  return seq_attn_bwd(dtype_of(c.dtype), c.dh, a, (hipStream_t)stream) == hipSuccess ? BCMT_OK
                                                                                    : BCMT_ERR_HIP;
}

int bcmt_attn_decode_validate(const bcmt_attn_decode_config* cfg) { return check_decode(cfg); }

size_t bcmt_attn_decode_workspace_bytes(const bcmt_attn_decode_config* cfg) {
  if (check_decode(cfg) != BCMT_OK) return 0;
  const int n = seq_attn_decode_splits(dtype_of(cfg->dtype), cfg->dh, cfg->B, cfg->H, cfg->Hkv,
                                       cfg->cap);
  // (room for one part also where the outputs are written at once)
  return up256((size_t)cfg->B * cfg->H * n * (cfg->dh + 2) * 4);
}

int bcmt_attn_decode(const bcmt_attn_decode_config* cfg, const void* q, const void* k,
                     const void* v, const int32_t* slot, const int32_t* length, void* kcache,
                     void* vcache, void* o, void* ws, size_t ws_bytes, void* stream) {
  const int st = check_decode(cfg);
  if (st != BCMT_OK) return st;
  if (!q || !k || !v || !length || !kcache || !vcache || !o || !ws) return BCMT_ERR_INVALID;
  for (const void* p : {q, k, v, (const void*)kcache, (const void*)vcache, (const void*)o,
                        (const void*)ws})
    if (!is16(p)) return BCMT_ERR_INVALID;
  if (!is4(slot) || !is4(length)) return BCMT_ERR_INVALID;
  const bcmt_attn_decode_config& c = *cfg;
  const int es = esize(c.dtype);
  const int64_t wq = (int64_t)c.H * c.dh, wk = (int64_t)c.Hkv * c.dh;
  DecAttn a{};
  a.ldq = c.ldq ? c.ldq : wq;
  a.ldk = c.ldk ? c.ldk : wk;
  a.ldv = c.ldv ? c.ldv : wk;
  a.ldo = c.ldo ? c.ldo : wq;
  const bool dense = !(c.cs || c.ct || c.ch);
  a.ch = dense ? c.dh : c.ch;
  a.ct = dense ? wk : c.ct;
  a.cs = dense ? (int64_t)c.cap * wk : c.cs;
  const size_t need = bcmt_attn_decode_workspace_bytes(cfg);
  const Rows r[4] = {{o, a.ldo, wq}, {q, a.ldq, wq}, {k, a.ldk, wk}, {v, a.ldv, wk}};
  const size_t cache = (size_t)((c.slots - 1) * a.cs + (c.cap - 1) * a.ct + (c.Hkv - 1) * a.ch +
                                c.dh) * es;
  const size_t ni = (size_t)c.B * 4;
  if (any_meet(r, 1, 4, c.B, es) || meets_any(ws, need, r, 4, c.B, es) ||
      meets_any(kcache, cache, r, 4, c.B, es) || meets_any(vcache, cache, r, 4, c.B, es) ||
      bytes_meet(ws, need, kcache, cache) || bytes_meet(ws, need, vcache, cache))
    return BCMT_ERR_INVALID;
  // the two caches may interleave in one allocation, but not be the same rows
  if (dense ? bytes_meet(kcache, cache, vcache, cache) : kcache == vcache) return BCMT_ERR_INVALID;
  for (const void* p : {(const void*)slot, (const void*)length})
    if (meets_any(p, ni, r, 1, c.B, es) || bytes_meet(p, ni, ws, need) ||
        bytes_meet(p, ni, kcache, cache) || bytes_meet(p, ni, vcache, cache))
      return BCMT_ERR_INVALID;
  if (ws_bytes < need) return BCMT_ERR_WORKSPACE;
  a.q = q;
  a.k = k;
  a.v = v;
  a.slot = slot;
  a.length = length;
  a.kcache = kcache;
  a.vcache = vcache;
  a.o = o;
  a.B = c.B;
  a.slots = c.slots;
  a.cap = c.cap;
  a.H = c.H;
  a.Hkv = c.Hkv;
  a.sl2 = c.scale * 1.4426950408889634f;
  a.nsplit = seq_attn_decode_splits(dtype_of(c.dtype), c.dh, c.B, c.H, c.Hkv, c.cap);
  a.part_o = (float*)ws;
  a.part_ml = a.part_o + (size_t)c.B * c.H * a.nsplit * c.dh;
  return seq_attn_decode(dtype_of(c.dtype), c.dh, a, (hipStream_t)stream) == hipSuccess
             ? BCMT_OK
             : BCMT_ERR_HIP;
}

int bcmt_linattn_validate(const bcmt_linattn_config* cfg) { return check_lin(cfg); }

size_t bcmt_linattn_workspace_bytes(const bcmt_linattn_config* cfg, int pass) {
  if (check_lin(cfg) != BCMT_OK) return 0;
  const LinPlan p(*cfg);
  return pass == BCMT_PASS_FORWARD ? p.fwd_bytes : pass == BCMT_PASS_BACKWARD ? p.bwd_bytes : 0;
}

int bcmt_linattn_forward(const bcmt_linattn_config* cfg, const void* q, const void* k,
                         const void* v, const float* gamma, const int32_t* cu, const float* S_in,
                         void* o, float* S_out, void* ws, size_t ws_bytes, void* stream) {
  const int st = check_lin(cfg);
  if (st != BCMT_OK) return st;
  if (!q || !k || !v || !gamma || !cu || !o) return BCMT_ERR_INVALID;
  for (const void* p : {q, k, v, (const void*)o, (const void*)S_in, (const void*)S_out,
                        (const void*)ws})
    if (!is16(p)) return BCMT_ERR_INVALID;
  if (!is4(gamma) || !is4(cu)) return BCMT_ERR_INVALID;
  const bcmt_linattn_config& c = *cfg;
  const LinPlan pl(c);
  if (pl.fwd_bytes && !ws) return BCMT_ERR_INVALID;
  const int es = esize(c.dtype);
  const int64_t w = (int64_t)c.H * c.dh;
  const int64_t ldq = c.ldq ? c.ldq : w, ldk = c.ldk ? c.ldk : w, ldv = c.ldv ? c.ldv : w,
                ldo = c.ldo ? c.ldo : w;
  const Rows r[4] = {{o, ldo, w}, {q, ldq, w}, {k, ldk, w}, {v, ldv, w}};
  const size_t ns = (size_t)c.nseq * c.H * c.dh * c.dh * 4, nc = (size_t)(c.nseq + 1) * 4;
  const size_t ng = (size_t)c.H * 4, nw = pl.fwd_bytes;
  if (any_meet(r, 1, 4, c.total, es) || meets_any(S_out, ns, r, 4, c.total, es) ||
      meets_any(S_in, ns, r, 1, c.total, es) || meets_any(cu, nc, r, 1, c.total, es) ||
      meets_any(gamma, ng, r, 1, c.total, es) || bytes_meet(S_out, ns, cu, nc) ||
      bytes_meet(S_out, ns, gamma, ng) || (S_in != S_out && bytes_meet(S_in, ns, S_out, ns)))
    return BCMT_ERR_INVALID;
  if (nw && (meets_any(ws, nw, r, 4, c.total, es) || bytes_meet(ws, nw, S_in, ns) ||
             bytes_meet(ws, nw, S_out, ns) || bytes_meet(ws, nw, cu, nc) ||
             bytes_meet(ws, nw, gamma, ng)))
    return BCMT_ERR_INVALID;
  if (ws_bytes < nw) return BCMT_ERR_WORKSPACE;
  LinPass a{};
  a.a = q;
  a.b = k;
  a.c = v;
  a.lda = ldq;
  a.ldb = ldk;
  a.ldc = ldv;
  a.ldo = ldo;
  a.out = o;
  a.cu = cu;
  a.gamma = gamma;
  a.s_in = S_in;
  a.s_out = S_out;
  a.seg_state = (float*)((char*)ws + pl.fwd);
  a.given = pl.cut && S_in && S_in == S_out ? (float*)((char*)ws + pl.given) : nullptr;
  a.sr = c.dh;
  a.sc = 1;
  a.total = c.total;
  a.nseq = c.nseq;
  a.H = c.H;
  a.seg = pl.seg;
  a.s_intra = a.s_inter = c.scale;
  a.s_upd = 1.f;
  a.fine = true;
  const DType dt = dtype_of(c.dtype);
  const hipStream_t s = (hipStream_t)stream;
  if (pl.cut) {
    if (lin_pass(dt, c.dh, a, false, true, s) != hipSuccess) return BCMT_ERR_HIP;
    if (lin_scan(c.dh, a, false, s) != hipSuccess) return BCMT_ERR_HIP;
  }
  return lin_pass(dt, c.dh, a, false, false, s) == hipSuccess ? BCMT_OK : BCMT_ERR_HIP;
}

int bcmt_linattn_backward(const bcmt_linattn_config* cfg, const void* q, const void* k,
                          const void* v, const float* gamma, const int32_t* cu,
                          const float* S_in, const void* dO, const float* dS_out, void* dq,
                          void* dk, void* dv, float* dS_in, float* dgamma, void* ws,
                          size_t ws_bytes, void* stream) {
  const int st = check_lin(cfg);
  if (st != BCMT_OK) return st;
  if (!q || !k || !v || !gamma || !cu || !dO || !dq || !dk || !dv || !ws) return BCMT_ERR_INVALID;
  for (const void* p : {q, k, v, dO, (const void*)dq, (const void*)dk, (const void*)dv,
                        (const void*)S_in, (const void*)dS_out, (const void*)dS_in,
                        (const void*)ws})
    if (!is16(p)) return BCMT_ERR_INVALID;
  if (!is4(gamma) || !is4(cu) || !is4(dgamma)) return BCMT_ERR_INVALID;
  const bcmt_linattn_config& c = *cfg;
  const LinPlan pl(c);
  const int es = esize(c.dtype);
  const int64_t w = (int64_t)c.H * c.dh;
  const int64_t ldq = c.ldq ? c.ldq : w, ldk = c.ldk ? c.ldk : w, ldv = c.ldv ? c.ldv : w,
                ldo = c.ldo ? c.ldo : w;
  const Rows r[7] = {{dq, ldq, w}, {dk, ldk, w}, {dv, ldv, w}, {q, ldq, w},
                     {k, ldk, w},  {v, ldv, w},  {dO, ldo, w}};
  const size_t ns = (size_t)c.nseq * c.H * c.dh * c.dh * 4, nc = (size_t)(c.nseq + 1) * 4;
  const size_t ng = (size_t)c.H * 4, nw = pl.bwd_bytes;
  if (any_meet(r, 3, 7, c.total, es) || meets_any(dS_in, ns, r, 7, c.total, es) ||
      meets_any(dgamma, ng, r, 7, c.total, es) || meets_any(ws, nw, r, 7, c.total, es) ||
      meets_any(S_in, ns, r, 3, c.total, es) || meets_any(dS_out, ns, r, 3, c.total, es) ||
      meets_any(cu, nc, r, 3, c.total, es) || meets_any(gamma, ng, r, 3, c.total, es))
    return BCMT_ERR_INVALID;
  const struct {
    const void* p;
    size_t n;
  } small[6] = {{dS_in, ns}, {dgamma, ng}, {ws, nw}, {S_in, ns}, {cu, nc}, {gamma, ng}};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 6; ++j)
      if (bytes_meet(small[i].p, small[i].n, small[j].p, small[j].n)) return BCMT_ERR_INVALID;
  if ((dS_in != dS_out && bytes_meet(dS_in, ns, dS_out, ns)) || bytes_meet(dgamma, ng, dS_out, ns) ||
      bytes_meet(ws, nw, dS_out, ns))
    return BCMT_ERR_INVALID;
  if (ws_bytes < nw) return BCMT_ERR_WORKSPACE;

  char* W = (char*)ws;
  float *seg_s = (float*)(W + pl.fwd), *seg_r = (float*)(W + pl.rev);
  float* given = pl.cut && dS_in && dS_in == dS_out ? (float*)(W + pl.given) : nullptr;
  const DType dt = dtype_of(c.dtype);
  const hipStream_t s = (hipStream_t)stream;
  LinPass a{};
  a.cu = cu;
  a.gamma = gamma;
  a.total = c.total;
  a.nseq = c.nseq;
  a.H = c.H;
  a.seg = pl.seg;
  a.fine = true;  // (the same bits whatever outputs are wanted)
  auto rows = [&](const void* x, int64_t lx, const void* y, int64_t ly, const void* z, int64_t lz,
                  void* out, int64_t lo) {
    a.a = x;
    a.lda = lx;
    a.b = y;
    a.ldb = ly;
    a.c = z;
    a.ldc = lz;
    a.out = out;
    a.ldo = lo;
  };
  // The states between segments: S of k, v in order; R of q, dO in reverse
  // (joined: its sums come with dq).
  const bool joined = lin_joined_backward(dt, c.dh);
  if (pl.cut) {
    rows(nullptr, 0, k, ldk, v, ldv, nullptr, 0);
    a.s_in = S_in;
    a.seg_state = seg_s;
    a.s_upd = 1.f;
    if (lin_pass(dt, c.dh, a, false, true, s) != hipSuccess) return BCMT_ERR_HIP;
    if (lin_scan(c.dh, a, false, s) != hipSuccess) return BCMT_ERR_HIP;
  }
  // dq: rows dO, v, k in order, the state transposed.
  rows(dO, ldo, v, ldv, k, ldk, dq, ldq);
  a.s_in = S_in;
  a.seg_state = seg_s;
  a.sr = 1;
  a.sc = c.dh;
  a.s_intra = a.s_inter = c.scale;
  a.s_upd = 1.f;
  a.fine = false;
  if (joined && pl.cut) {
    a.q = q;
    a.ldq = ldq;
    a.sum_state = seg_r;
    a.s_sum = c.scale;
  }
  if (lin_pass(dt, c.dh, a, false, false, s) != hipSuccess) return BCMT_ERR_HIP;
  if (pl.cut) {
    rows(nullptr, 0, q, ldq, dO, ldo, nullptr, 0);
    a.s_in = dS_out;
    a.seg_state = seg_r;
    a.given = given;
    a.s_upd = c.scale;
    a.sr = c.dh;
    a.sc = 1;
    a.fine = true;
    if (!joined && lin_pass(dt, c.dh, a, true, true, s) != hipSuccess) return BCMT_ERR_HIP;
    if (lin_scan(c.dh, a, true, s) != hipSuccess) return BCMT_ERR_HIP;
  }
  if (dgamma) {
    LinDecay g{};
    g.q = q;
    g.k = k;
    g.v = v;
    g.dout = dO;
    g.cu = cu;
    g.gamma = gamma;
    g.s_in = S_in;
    g.ds_out = dS_out;
    g.seg_s = seg_s;
    g.seg_r = seg_r;
    g.part = (float*)(W + pl.part);
    g.dgamma = dgamma;
    g.total = c.total;
    g.nseq = c.nseq;
    g.H = c.H;
    g.seg = pl.seg;
    g.nslot = pl.nslot;
    g.ldq = ldq;
    g.ldk = ldk;
    g.ldv = ldv;
    g.ldo = ldo;
    g.scale = c.scale;
    if (lin_dgamma(dt, c.dh, g, s) != hipSuccess) return BCMT_ERR_HIP;
  }
  if (joined) {
    LinPair g{};
    g.k = k;
    g.v = v;
    g.q = q;
    g.dout = dO;
    g.dk = dk;
    g.dv = dv;
    g.cu = cu;
    g.gamma = gamma;
    g.ds_out = dS_out;
    g.ds_in = dS_in;
    g.seg_state = seg_r;
    g.given = given;
    g.total = c.total;
    g.nseq = c.nseq;
    g.H = c.H;
    g.seg = pl.seg;
    g.ldk = ldk;
    g.ldv = ldv;
    g.ldq = ldq;
    g.ldo = ldo;
    g.scale = c.scale;
    return lin_dkdv(c.dh, g, s) == hipSuccess ? BCMT_OK : BCMT_ERR_HIP;
  }
  // dk: rows v, dO, q in reverse, the state transposed.
  rows(v, ldv, dO, ldo, q, ldq, dk, ldk);
  a.s_in = dS_out;
  a.seg_state = seg_r;
  a.given = nullptr;
  a.sr = 1;
  a.sc = c.dh;
  a.s_intra = c.scale;
  a.s_inter = 1.f;
  a.s_upd = c.scale;
  a.fine = false;
  if (lin_pass(dt, c.dh, a, true, false, s) != hipSuccess) return BCMT_ERR_HIP;
  // dv: rows k, q, dO in reverse; last, since dS_in may be dS_out.
  rows(k, ldk, q, ldq, dO, ldo, dv, ldv);
  a.s_out = dS_in;
  a.given = given;
  a.fine = true;
  a.sr = c.dh;
  a.sc = 1;
  return lin_pass(dt, c.dh, a, true, false, s) == hipSuccess ? BCMT_OK : BCMT_ERR_HIP;
}

int bcmt_linattn_step_validate(const bcmt_linattn_step_config* cfg) { return check_step(cfg); }

int bcmt_linattn_step(const bcmt_linattn_step_config* cfg, const void* q, const void* k,
                      const void* v, const float* gamma, const int32_t* slot, const float* S_in,
                      float* S_out, void* o, void* stream) {
  const int st = check_step(cfg);
  if (st != BCMT_OK) return st;
  if (!q || !k || !v || !gamma || !S_in || !S_out || !o) return BCMT_ERR_INVALID;
  for (const void* p : {q, k, v, (const void*)S_in, (const void*)S_out, (const void*)o})
    if (!is16(p)) return BCMT_ERR_INVALID;
  if (!is4(gamma) || !is4(slot)) return BCMT_ERR_INVALID;
  const bcmt_linattn_step_config& c = *cfg;
  const int es = esize(c.dtype);
  const int64_t w = (int64_t)c.H * c.dh;
  LinStep a{};
  a.ldq = c.ldq ? c.ldq : w;
  a.ldk = c.ldk ? c.ldk : w;
  a.ldv = c.ldv ? c.ldv : w;
  a.ldo = c.ldo ? c.ldo : w;
  const Rows r[4] = {{o, a.ldo, w}, {q, a.ldq, w}, {k, a.ldk, w}, {v, a.ldv, w}};
  const size_t ns = (size_t)c.slots * c.H * c.dh * c.dh * 4;
  if (any_meet(r, 1, 4, c.B, es) || meets_any(S_out, ns, r, 4, c.B, es) ||
      meets_any(S_in, ns, r, 1, c.B, es) || (S_in != S_out && bytes_meet(S_in, ns, S_out, ns)) ||
      meets_any(gamma, (size_t)c.H * 4, r, 1, c.B, es) ||
      meets_any(slot, (size_t)c.B * 4, r, 1, c.B, es) ||
      bytes_meet(gamma, (size_t)c.H * 4, S_out, ns) || bytes_meet(slot, (size_t)c.B * 4, S_out, ns))
    return BCMT_ERR_INVALID;
  a.q = q;
  a.k = k;
  a.v = v;
  a.gamma = gamma;
  a.s_in = S_in;
  a.s_out = S_out;
  a.slot = slot;
  a.o = o;
  a.B = c.B;
  a.slots = c.slots;
  a.H = c.H;
  a.scale = c.scale;
  return lin_step(dtype_of(c.dtype), c.dh, a, (hipStream_t)stream) == hipSuccess ? BCMT_OK
                                                                                : BCMT_ERR_HIP;
}

}  // extern "C"
