// kdn_layer_abi.cu -- the extern "C" entry points of the hybrid layer's operators
// (declared in include/kdn.h): sliding-window attention with sinks and the residual
// RMS norm.  Argument validation, workspace carve-up and dispatch; nothing here
// allocates memory.
#include <math.h>

#include <initializer_list>

#include "kdn_rmsnorm.cuh"
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

}  // extern "C"
