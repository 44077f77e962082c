// kdn_layer_abi.cu -- the extern "C" entry points of the hybrid layer's operators
// (declared in include/kdn.h): sliding-window attention with sinks, the residual RMS
// norm, rotary positions and the gated feed-forward block.  Argument validation, workspace
// carve-up and dispatch; nothing here allocates memory.
#include <math.h>

#include <initializer_list>

#include "kdn_ffn.cuh"
#include "kdn_rmsnorm.cuh"
#include "kdn_rope.cuh"
#include "kdn_swa.cuh"

namespace kdn {
namespace {

constexpr size_t kAlign = 256;

size_t round_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

bool ptrs_ok(std::initializer_list<const void *> required, std::initializer_list<const void *> optional = {}) {
  for (const void *p : required)
    if (!p || !aligned(p, 16)) return false;
  for (const void *p : optional)
    if (p && !aligned(p, 16)) return false;
  return true;
}

// Memory of a tensor (p null or n 0: there is none).
struct Span {
  const void *p;
  size_t n;
};
// No output shares memory with another one or with an input.
bool apart(std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
  const auto meet = [](const Span &a, const Span &b) {
    return a.p && b.p && a.n && b.n && (uintptr_t)a.p < (uintptr_t)b.p + b.n && (uintptr_t)b.p < (uintptr_t)a.p + a.n;
  };
  for (const Span *a = outs.begin(); a != outs.end(); ++a) {
    for (const Span *b = outs.begin(); b != a; ++b)
      if (meet(*a, *b)) return false;
    for (const Span &b : ins)
      if (meet(*a, b)) return false;
  }
  return true;
}

// Fills `a` from the descriptor; tokens = false for the decode step (no T axis).
kdn_status_t fill_swa(const kdn_swa_desc_t *d, bool tokens, SwaArgs *a) {
  if (!d) return KDN_ERR_INVALID_ARG;
  if (d->B < 0 || d->H < 0 || d->Hk < 0 || (tokens && d->T < 0)) return KDN_ERR_INVALID_ARG;
  if (d->d <= 0 || d->window < 1 || d->sinks < 0) return KDN_ERR_INVALID_ARG;
  if (d->dtype != KDN_F32 && d->dtype != KDN_BF16) return KDN_ERR_INVALID_ARG;
  if (!isnan(d->scale) && !(d->scale > 0.f && d->scale < INFINITY)) return KDN_ERR_INVALID_ARG;
  // (kv heads that no query head reads would leave their gradients and cache unwritten)
  if ((d->H == 0) != (d->Hk == 0) || (d->H && d->H % d->Hk)) return KDN_ERR_INVALID_ARG;
  if (d->d != 32 && d->d != 64 && d->d != 128) return KDN_ERR_UNSUPPORTED;
  if (d->B > 65535 || d->H > 65535) return KDN_ERR_UNSUPPORTED;
  const int T = tokens ? d->T : 1;
  if (T > (1 << 21) || (long long)d->B * d->H * T > (1LL << 31) - 1) return KDN_ERR_UNSUPPORTED;
  if ((long long)d->window + d->sinks > (1LL << 30)) return KDN_ERR_UNSUPPORTED;
  *a = SwaArgs{};
  a->B = d->B;
  a->T = T;
  a->H = d->H;
  a->Hk = d->Hk;
  a->G = d->Hk ? d->H / d->Hk : 1;
  a->d = d->d;
  a->W = d->window;
  a->ns = d->sinks;
  a->dtype = d->dtype;
  a->scale = isnan(d->scale) ? 1.f / sqrtf((float)d->d) : d->scale;
  return KDN_OK;
}

bool has_work(const SwaArgs &a) { return (size_t)a.B * a.H * a.T > 0; }

size_t swa_fwd_bytes(const SwaArgs &) { return kAlign; }

// Backward workspace: status word, delta, nlse, partial sums of split key tiles.
size_t swa_bwd_layout(SwaArgs *a, const SwaSplits &sp, int BN, char *base) {
  const size_t rows = round_up((size_t)a->B * a->H * a->T * sizeof(float));
  if (base) {
    a->status = reinterpret_cast<unsigned *>(base);
    a->nlse = reinterpret_cast<float *>(base + kAlign);
    a->delta = reinterpret_cast<float *>(base + kAlign + rows);
    a->part = reinterpret_cast<float *>(base + kAlign + 2 * rows);
  }
  return kAlign + 2 * rows + (size_t)a->B * a->Hk * sp.part_blocks * 2 * BN * a->d * sizeof(float);
}

kdn_status_t fill_norm(const kdn_norm_desc_t *d, NormArgs *a) {
  if (!d) return KDN_ERR_INVALID_ARG;
  if (d->rows < 0 || d->D <= 0) return KDN_ERR_INVALID_ARG;
  if (d->dtype != KDN_F32 && d->dtype != KDN_BF16) return KDN_ERR_INVALID_ARG;
  if (d->out_dtype != d->dtype && d->out_dtype != KDN_F8E4M3) return KDN_ERR_INVALID_ARG;
  if (d->block != 0 && (d->block != 128 || d->out_dtype != KDN_F8E4M3)) return KDN_ERR_INVALID_ARG;
  if (!(d->eps >= 0.f && d->eps < INFINITY)) return KDN_ERR_INVALID_ARG;
  if (d->D % 8 || d->D > 16384 || d->rows > (1LL << 31) - 1) return KDN_ERR_UNSUPPORTED;
  *a = NormArgs{};
  a->rows = d->rows;
  a->D = d->D;
  a->dtype = d->dtype;
  a->f8 = d->out_dtype == KDN_F8E4M3;
  a->block = d->block;
  a->eps = d->eps;
  return KDN_OK;
}

// Fills `a` from the descriptor but for the tensors.
kdn_status_t fill_rope(const kdn_rope_desc_t *d, const unsigned long long *turns, RopeArgs *a) {
  if (!d) return KDN_ERR_INVALID_ARG;
  if (d->B < 0 || d->T < 0 || d->H < 0 || d->Hk < 0 || d->d <= 0) return KDN_ERR_INVALID_ARG;
  if (d->rot < 2 || d->rot % 2 || d->rot > d->d || !isfinite(d->mscale)) return KDN_ERR_INVALID_ARG;
  if (d->dtype != KDN_F32 && d->dtype != KDN_BF16) return KDN_ERR_INVALID_ARG;
  if (d->interleaved != 0 && d->interleaved != 1) return KDN_ERR_INVALID_ARG;
  if (d->pos_per_token != 0 && d->pos_per_token != 1) return KDN_ERR_INVALID_ARG;
  if (d->d % 8 || d->d > 2 * kRopeMaxPairs || d->T > (1 << 21)) return KDN_ERR_UNSUPPORTED;
  if (d->H > 65535 || d->Hk > 65535 || (long long)d->B * d->T > (1LL << 31) - 1) return KDN_ERR_UNSUPPORTED;
  // rows that overlap one another; rows more than 2^31 elements apart
  const long long lds[4] = {d->ldq, d->ldqo, d->ldk, d->ldko};
  for (int i = 0; i < 4; ++i) {
    const long long dense = (long long)(i < 2 ? d->H : d->Hk) * d->d;
    if (lds[i] != 0 && lds[i] < dense) return KDN_ERR_INVALID_ARG;
    if (lds[i] > (1LL << 31)) return KDN_ERR_UNSUPPORTED;
  }
  *a = RopeArgs{};
  a->B = d->B;
  a->T = d->T;
  a->H = d->H;
  a->Hk = d->Hk;
  a->d = d->d;
  a->rot = d->rot;
  a->inter = d->interleaved;
  a->per_token = d->pos_per_token;
  a->dtype = d->dtype;
  a->mscale = d->mscale;
  if (turns)
    for (int i = 0; i < d->rot / 2; ++i) a->turns[i] = turns[i];
  return KDN_OK;
}

// Whether two tensors of `rows` rows share memory: `w` bytes a row, `ld` bytes from one to the next.
struct Rows {
  const void *p;
  long long ld, w;
};
bool rows_meet(const Rows &a, const Rows &b, long long rows) {
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  if (a.w == 0 || b.w == 0 || x >= y + (rows - 1) * b.ld + b.w || y >= x + (rows - 1) * a.ld + a.w) return false;
  if (rows == 1 || a.ld != b.ld) return true;
  const long long d = ((long long)(y - x) % a.ld + a.ld) % a.ld;  // heads of one projection lie beside one another
  return d < a.w || d + b.w > a.ld;
}

// One direction: `back` reads the outputs' gradients and writes the inputs'.
kdn_status_t rope(const kdn_rope_desc_t *desc, const unsigned long long *turns, bool back, const void *q,
                  const void *k, const int *pos, const int *lens, void *qo, void *ko, void *stream) {
  RopeArgs a;
  const kdn_status_t st = fill_rope(desc, turns, &a);
  if (st != KDN_OK) return st;
  if ((long long)a.B * a.T * (a.H + a.Hk) == 0) return KDN_OK;
  if (!turns || (a.per_token && !pos)) return KDN_ERR_INVALID_ARG;
  if (!ptrs_ok({}, {pos, lens})) return KDN_ERR_INVALID_ARG;
  if ((a.H && !ptrs_ok({q, qo})) || (a.Hk && !ptrs_ok({k, ko}))) return KDN_ERR_INVALID_ARG;
  const long long dense[2] = {(long long)a.H * a.d, (long long)a.Hk * a.d};
  const long long in[2] = {back ? desc->ldqo : desc->ldq, back ? desc->ldko : desc->ldk};
  const long long out[2] = {back ? desc->ldq : desc->ldqo, back ? desc->ldk : desc->ldko};
  for (int i = 0; i < 2; ++i) {
    a.in[i] = i ? k : q;
    a.out[i] = i ? ko : qo;
    a.ldi[i] = in[i] ? in[i] : dense[i];
    a.ldo[i] = out[i] ? out[i] : dense[i];
    // a row would be written where another one is still to be read
    if (dense[i] && a.in[i] == a.out[i] && a.ldi[i] != a.ldo[i]) return KDN_ERR_INVALID_ARG;
  }
  const long long es = a.dtype == KDN_F32 ? 4 : 2, rows = (long long)a.B * a.T;
  for (int i = 0; i < 2; ++i) {
    const Rows out{a.out[i], a.ldo[i] * es, dense[i] * es};
    if (i && rows_meet(out, {a.out[0], a.ldo[0] * es, dense[0] * es}, rows)) return KDN_ERR_INVALID_ARG;
    for (int j = 0; j < 2; ++j)
      if (!(i == j && a.in[i] == a.out[i]) && rows_meet(out, {a.in[j], a.ldi[j] * es, dense[j] * es}, rows))
        return KDN_ERR_INVALID_ARG;
  }
  a.pos = pos;
  a.lens = lens;
  a.sign = back ? -1.f : 1.f;
  return launch_rope(a, static_cast<cudaStream_t>(stream));
}

kdn_status_t fill_ffn(const kdn_ffn_desc_t *d, FfnArgs *a) {
  if (!d) return KDN_ERR_INVALID_ARG;
  if (d->rows < 0 || d->D <= 0 || d->F <= 0) return KDN_ERR_INVALID_ARG;
  if (d->dtype != KDN_F32 && d->dtype != KDN_BF16) return KDN_ERR_INVALID_ARG;
  if (d->act != KDN_ACT_SILU && d->act != KDN_ACT_GELU) return KDN_ERR_INVALID_ARG;
  if (d->dw_dtype != d->dtype && d->dw_dtype != KDN_F32) return KDN_ERR_INVALID_ARG;
  if (d->D % 8 || d->F % 8 || d->D > (1 << 20) || d->F > (1 << 20)) return KDN_ERR_UNSUPPORTED;
  if (d->rows > (1LL << 31) - 1) return KDN_ERR_UNSUPPORTED;
  *a = FfnArgs{};
  a->rows = d->rows;
  a->D = d->D;
  a->F = d->F;
  a->dtype = d->dtype;
  a->act = d->act;
  a->dw_dtype = d->dw_dtype;
  return KDN_OK;
}

// Workspace: status word; the backward's dg and du, or in float32 the operands' planes; partial sums.
size_t ffn_layout(FfnArgs *a, bool back, char *base) {
  const bool f32 = a->dtype == KDN_F32;
  const size_t rows = back && !f32 ? round_up((size_t)a->rows * a->F * 2) : 0;
  const size_t planes = f32 && a->rows > 0 ? ffn_planes_bytes_f32(*a, back) : 0;
  if (base) {
    a->status = reinterpret_cast<unsigned *>(base);
    a->dg = base + kAlign;
    a->du = base + kAlign + rows;
    a->planes = base + kAlign;
    a->part = reinterpret_cast<float *>(base + kAlign + 2 * rows + planes);
  }
  const size_t part = a->rows == 0 ? 0 : f32 ? ffn_part_floats_f32(*a, back) : ffn_part_floats_tc(*a, back);
  return kAlign + 2 * rows + planes + round_up(part * sizeof(float));
}

}  // namespace
}  // namespace kdn

using namespace kdn;

extern "C" {

size_t kdn_swa_fwd_workspace_bytes(const kdn_swa_desc_t *desc) {
  SwaArgs a;
  return fill_swa(desc, true, &a) == KDN_OK ? swa_fwd_bytes(a) : 0;
}

size_t kdn_swa_bwd_workspace_bytes(const kdn_swa_desc_t *desc) {
  SwaArgs a;
  if (fill_swa(desc, true, &a) != KDN_OK) return 0;
  if (!has_work(a)) return kAlign;
  const int BN = swa_tc_supported(a) ? kSwaTcTile : kSwaGenTile;
  return swa_bwd_layout(&a, swa_splits(a, BN, BN), BN, nullptr);
}

kdn_status_t kdn_swa_fwd(const kdn_swa_desc_t *desc, const void *q, const void *k, const void *v, const int *lens,
                         void *o, float *lse, void *workspace, size_t workspace_bytes, void *stream) {
  SwaArgs a;
  const kdn_status_t st = fill_swa(desc, true, &a);
  if (st != KDN_OK) return st;
  if (!has_work(a)) return KDN_OK;
  if (!ptrs_ok({q, k, v, o}, {lens, lse})) return KDN_ERR_INVALID_ARG;
  if (!workspace || !aligned(workspace, kAlign) || workspace_bytes < swa_fwd_bytes(a)) return KDN_ERR_WORKSPACE;
  a.q = q; a.k = k; a.v = v; a.lens = lens; a.o = o; a.lse = lse;
  a.status = static_cast<unsigned *>(workspace);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (swa_tc_supported(a)) return launch_swa_fwd_tc(a, s);
  if (cudaMemsetAsync(a.status, 0, sizeof(unsigned), s) != cudaSuccess) return KDN_ERR_CUDA;
  return launch_swa_fwd_general(a, s);
}

kdn_status_t kdn_swa_bwd(const kdn_swa_desc_t *desc, const void *q, const void *k, const void *v, const int *lens,
                         const void *o, const float *lse, const void *dO, void *dq, void *dk, void *dv,
                         void *workspace, size_t workspace_bytes, void *stream) {
  SwaArgs a;
  kdn_status_t st = fill_swa(desc, true, &a);
  if (st != KDN_OK) return st;
  if (!has_work(a)) return KDN_OK;
  if (!ptrs_ok({q, k, v, o, lse, dO, dq, dk, dv}, {lens})) return KDN_ERR_INVALID_ARG;
  const bool tc = swa_tc_supported(a);
  const int BN = tc ? kSwaTcTile : kSwaGenTile;
  const SwaSplits sp = swa_splits(a, BN, BN);
  if (!workspace || !aligned(workspace, kAlign) || workspace_bytes < swa_bwd_layout(&a, sp, BN, nullptr))
    return KDN_ERR_WORKSPACE;
  swa_bwd_layout(&a, sp, BN, static_cast<char *>(workspace));
  a.q = q; a.k = k; a.v = v; a.lens = lens; a.o = const_cast<void *>(o); a.lse = const_cast<float *>(lse);
  a.dO = dO; a.dq = dq; a.dk = dk; a.dv = dv;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((st = launch_swa_prep(a, s)) != KDN_OK) return st;
  if ((st = tc ? launch_swa_bwd_tc(a, sp, s) : launch_swa_bwd_general(a, sp, s)) != KDN_OK) return st;
  return launch_swa_join(a, sp, BN, s);
}

kdn_status_t kdn_swa_cache_fill(const kdn_swa_desc_t *desc, const void *k, const void *v, const int *lens, void *kc,
                                void *vc, void *stream) {
  SwaArgs a;
  const kdn_status_t st = fill_swa(desc, true, &a);
  if (st != KDN_OK) return st;
  if (!has_work(a)) return KDN_OK;
  if (!ptrs_ok({k, v, kc, vc}, {lens})) return KDN_ERR_INVALID_ARG;
  a.k = k; a.v = v; a.lens = lens;
  return launch_swa_cache_fill(a, kc, vc, static_cast<cudaStream_t>(stream));
}

kdn_status_t kdn_swa_decode_step(const kdn_swa_desc_t *desc, const void *q, const void *k, const void *v, void *kc,
                                 void *vc, const int *pos, void *o, void *stream) {
  SwaArgs a;
  const kdn_status_t st = fill_swa(desc, false, &a);
  if (st != KDN_OK) return st;
  if (!has_work(a)) return KDN_OK;
  if (!ptrs_ok({q, k, v, kc, vc, pos, o})) return KDN_ERR_INVALID_ARG;
  a.q = q; a.k = k; a.v = v; a.o = o;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return swa_tc_supported(a) ? launch_swa_decode_tc(a, kc, vc, pos, s) : launch_swa_decode_general(a, kc, vc, pos, s);
}

kdn_status_t kdn_add_rmsnorm_fwd(const kdn_norm_desc_t *desc, const void *x, const void *res, const void *w, void *y,
                                 void *h, float *rstd, float *scales, void *stream) {
  NormArgs a;
  const kdn_status_t st = fill_norm(desc, &a);
  if (st != KDN_OK) return st;
  if (a.rows == 0) return KDN_OK;
  if (!ptrs_ok({x, w, y}, {res, h, rstd, scales})) return KDN_ERR_INVALID_ARG;
  if (a.f8 && !scales) return KDN_ERR_INVALID_ARG;
  a.x = x; a.res = res; a.w = w; a.y = y; a.h = h; a.rstd = rstd; a.scales = scales;
  return launch_add_rmsnorm(a, static_cast<cudaStream_t>(stream));
}

size_t kdn_add_rmsnorm_bwd_workspace_bytes(const kdn_norm_desc_t *desc) {
  NormArgs a;
  if (fill_norm(desc, &a) != KDN_OK) return 0;
  return round_up((size_t)rmsnorm_bwd_blocks(a.rows, a.D) * a.D * sizeof(float)) + kAlign;
}

kdn_status_t kdn_add_rmsnorm_bwd(const kdn_norm_desc_t *desc, const void *h, const void *w, const float *rstd,
                                 const void *dy, const void *dh, void *dx, float *dw, void *workspace,
                                 size_t workspace_bytes, void *stream) {
  NormArgs a;
  const kdn_status_t st = fill_norm(desc, &a);
  if (st != KDN_OK) return st;
  if (a.f8) return KDN_ERR_INVALID_ARG;
  if (!ptrs_ok({dw})) return KDN_ERR_INVALID_ARG;
  if (a.rows > 0 && !ptrs_ok({h, w, rstd, dy, dx}, {dh})) return KDN_ERR_INVALID_ARG;
  if (!workspace || !aligned(workspace, kAlign) || workspace_bytes < kdn_add_rmsnorm_bwd_workspace_bytes(desc))
    return KDN_ERR_WORKSPACE;
  a.hin = h; a.w = w; a.rstd_in = rstd; a.dy = dy; a.dh = dh; a.dx = dx; a.dw = dw;
  a.part = static_cast<float *>(workspace);
  return launch_add_rmsnorm_bwd(a, static_cast<cudaStream_t>(stream));
}

kdn_status_t kdn_rope_freqs(const kdn_rope_freqs_t *f, unsigned long long *turns, float *mscale) {
  if (!f || !turns) return KDN_ERR_INVALID_ARG;
  if (f->rot < 2 || f->rot % 2 || !(f->base > 1 && isfinite(f->base))) return KDN_ERR_INVALID_ARG;
  if (!(f->factor >= 1 && isfinite(f->factor)) || !(f->trained >= 0 && isfinite(f->trained)))
    return KDN_ERR_INVALID_ARG;
  if (!(f->beta_slow >= 0 && f->beta_fast > f->beta_slow && isfinite(f->beta_fast))) return KDN_ERR_INVALID_ARG;
  if (f->rot > 2 * kRopeMaxPairs) return KDN_ERR_UNSUPPORTED;
  const double two_pi = 6.283185307179586476925;
  for (int i = 0; i < f->rot / 2; ++i) {
    double w = 0, x = pow(f->base, -2.0 * i / f->rot);
    if (f->trained > 0) w = (f->trained * x / two_pi - f->beta_slow) / (f->beta_fast - f->beta_slow);
    w = w < 0 ? 0 : w > 1 ? 1 : w;
    if (f->factor > 1) x *= (1 - w) / f->factor + w;
    turns[i] = (unsigned long long)rint(ldexp(x / two_pi, 64));  // x <= 1: at most 0.16 turns
  }
  if (mscale) *mscale = f->factor > 1 && f->trained > 0 ? (float)(0.1 * log(f->factor) + 1) : 1.f;
  return KDN_OK;
}

kdn_status_t kdn_rope_fwd(const kdn_rope_desc_t *desc, const unsigned long long *turns, const void *q, const void *k,
                          const int *pos, const int *lens, void *qo, void *ko, void *stream) {
  return rope(desc, turns, false, q, k, pos, lens, qo, ko, stream);
}

kdn_status_t kdn_rope_bwd(const kdn_rope_desc_t *desc, const unsigned long long *turns, const void *dqo,
                          const void *dko, const int *pos, const int *lens, void *dq, void *dk, void *stream) {
  return rope(desc, turns, true, dqo, dko, pos, lens, dq, dk, stream);
}

size_t kdn_ffn_fwd_workspace_bytes(const kdn_ffn_desc_t *desc) {
  FfnArgs a;
  return fill_ffn(desc, &a) == KDN_OK ? ffn_layout(&a, false, nullptr) : 0;
}

size_t kdn_ffn_bwd_workspace_bytes(const kdn_ffn_desc_t *desc) {
  FfnArgs a;
  return fill_ffn(desc, &a) == KDN_OK ? ffn_layout(&a, true, nullptr) : 0;
}

kdn_status_t kdn_ffn_fwd(const kdn_ffn_desc_t *desc, const void *x, const void *wg, const void *wu, const void *wd,
                         void *g, void *u, void *h, void *y, void *workspace, size_t workspace_bytes, void *stream) {
  FfnArgs a;
  const kdn_status_t st = fill_ffn(desc, &a);
  if (st != KDN_OK) return st;
  if (a.rows == 0) return KDN_OK;
  if (!ptrs_ok({x, wg, wu, wd, h, y}, {g, u}) || !g != !u) return KDN_ERR_INVALID_ARG;
  const size_t need = ffn_layout(&a, false, static_cast<char *>(workspace));
  if (!workspace || !aligned(workspace, kAlign) || workspace_bytes < need) return KDN_ERR_WORKSPACE;
  // (h, g and u are written while x and the weights are still read, y while h and Wd are)
  const size_t es = a.dtype == KDN_F32 ? 4 : 2, xs = es * a.rows * a.D, hs = es * a.rows * a.F, ws = es * a.D * a.F;
  if (!apart({{g, hs}, {u, hs}, {h, hs}, {y, xs}, {workspace, need}},
             {{x, xs}, {wg, ws}, {wu, ws}, {wd, ws}}))
    return KDN_ERR_INVALID_ARG;
  a.x = x; a.wg = wg; a.wu = wu; a.wd = wd; a.g = g; a.u = u; a.h = h; a.y = y;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return a.dtype == KDN_BF16 ? launch_ffn_fwd_tc(a, s) : launch_ffn_fwd_f32(a, s);
}

kdn_status_t kdn_ffn_bwd(const kdn_ffn_desc_t *desc, const void *x, const void *wg, const void *wu, const void *wd,
                         const void *g, const void *u, const void *h, const void *dy, void *dx, void *dwg, void *dwu,
                         void *dwd, void *workspace, size_t workspace_bytes, void *stream) {
  FfnArgs a;
  const kdn_status_t st = fill_ffn(desc, &a);
  if (st != KDN_OK) return st;
  // (without rows the weights' gradients are sums over nothing, and are written)
  if (!ptrs_ok({dwg, dwu, dwd})) return KDN_ERR_INVALID_ARG;
  if (a.rows > 0 && !ptrs_ok({x, wg, wu, wd, g, u, h, dy, dx})) return KDN_ERR_INVALID_ARG;
  const size_t need = ffn_layout(&a, true, static_cast<char *>(workspace));
  if (!workspace || !aligned(workspace, kAlign) || workspace_bytes < need) return KDN_ERR_WORKSPACE;
  // (dx is written before the weights' gradients read x and dy)
  const size_t es = a.dtype == KDN_F32 ? 4 : 2, xs = es * a.rows * a.D, hs = es * a.rows * a.F, ws = es * a.D * a.F;
  const size_t dws = (size_t)(a.dw_dtype == KDN_F32 ? 4 : 2) * a.D * a.F;
  if (!apart({{dx, xs}, {dwg, dws}, {dwu, dws}, {dwd, dws}, {workspace, need}},
             {{x, xs}, {wg, ws}, {wu, ws}, {wd, ws}, {g, hs}, {u, hs}, {h, hs}, {dy, xs}}))
    return KDN_ERR_INVALID_ARG;
  a.x = x; a.wg = wg; a.wu = wu; a.wd = wd; a.dy = dy;
  a.g = const_cast<void *>(g); a.u = const_cast<void *>(u); a.h = const_cast<void *>(h);
  a.dx = dx; a.dwg = dwg; a.dwu = dwu; a.dwd = dwd;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (a.rows == 0) {
    const size_t n = (size_t)a.D * a.F * (a.dw_dtype == KDN_F32 ? 4 : 2);
    bool ok = cudaMemsetAsync(a.status, 0, sizeof(unsigned), s) == cudaSuccess;
    for (void *p : {dwg, dwu, dwd}) ok = ok && cudaMemsetAsync(p, 0, n, s) == cudaSuccess;
    return ok ? KDN_OK : KDN_ERR_CUDA;
  }
  return a.dtype == KDN_BF16 ? launch_ffn_bwd_tc(a, s) : launch_ffn_bwd_f32(a, s);
}

}  // extern "C"
