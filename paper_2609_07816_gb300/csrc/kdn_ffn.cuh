// kdn_ffn.cuh -- internal types of the gated feed-forward block (kdn_ffn_* of
// include/kdn.h), shared by its translation units.
//
//   g = x Wg^T, u = x Wu^T, h = act(g) u, y = h Wd^T
//   dh = dy Wd, dg = dh u act'(g), du = dh act(g), dx = dg Wg + du Wu,
//   dWg = dg^T x, dWu = du^T x, dWd = dy^T h
//
// In bfloat16, what is rounded to 2^-9 before the end: h, dg and du, since the tensor cores take operands of the
// weights' type; g and u, which the forward leaves for the backward in the activations' type.  So y is 2.3e-3 of its
// norm off and dx, dWg and dWu 3.1e-3, where one rounding of an exact result is 1.7e-3.  Two bfloat16s for h, dg and du
// would take twice the products that read them; g and u in float32 0.7 GB more each way for 32768 tokens of F = 5632,
// and formed again in the backward 2.3 of the pass' 6.8 TFLOP.
#pragma once

#include "kdn_beside.cuh"
#include "kdn_internal.cuh"

namespace kdn {

struct FfnArgs {
  long long rows;
  int D, F, dtype, act, dw_dtype;
  const void *x, *wg, *wu, *wd, *dy;
  void *g, *u, *h, *y;             // forward's outputs; read by the backward
  void *dg, *du;                   // [rows][F] in the workspace (bfloat16; float32 uses `planes`)
  void *dx, *dwg, *dwu, *dwd;
  unsigned *status;
  void *planes;                    // float32: operands cut into bfloat16s, dg and du among them; few rows: dg and du
  float *part;                     // partial sums of a product whose K axis is cut
};

// act(g) and its derivative; s = 1 / (1 + e^-z) goes to 0 and 1 where e^-z leaves float32's range.
//   silu: a = g s(g), a' = s (1 + g (1 - s))
//   gelu: a = g s(z), z = 2 sqrt(2/pi) (g + 0.044715 g^3), a' = s (1 + g (1 - s) dz/dg)
constexpr float kGelu = 1.5957691216057308f, kGelu3 = 0.044715f;

// Near float32's own precision, 2^-20.5 of act(g) (ex2 2^-22 and six roundings).  An error of the exponential's
// argument is multiplied by the argument, so -|z| log2(e) is a sum of two float32s: a product's rest is exact by a
// fused multiply-add, a sum's by Dekker's Fast2Sum (the larger term first).  A Newton step behind the reciprocal, and
// neither s nor 1 - s by cancellation.  Where e^-|z| is below 2^-126 it is 0.
//   silu: |z| log2(e) = L |g|;  gelu: |g| (A + B g^2), A = log2(e) kGelu, B = A kGelu3
// (gelu with z rounded once was 2^-16.4 off at g = -8; 2048 tokens of 1024 x 4096, forward with g and u 217.6 us then
// and 219.0 now, gradients 473 and 477.)
template <int ACT> __device__ __forceinline__ void ffn_act_near(float g, float *a, float *da) {
  constexpr float kL = 1.44269502f, kLRest = 1.92596299e-8f, kLn2 = 0.69314718f;
  constexpr float kA = 2.30220819f, kARest = 1.29484024e-08f, kB = 0.102943242f, kBRest = -2.01619854e-09f;
  // |g| ends where e^-|z| has long been 0 and nothing overflows
  const float m = fminf(fabsf(g), ACT == KDN_ACT_SILU ? 200.f : 20.f), g2 = m * m;
  float f = kL, rest = kLRest;
  if (ACT == KDN_ACT_GELU) {
    const float p = kB * g2, big = fmaxf(p, kA), least = fminf(p, kA);
    f = big + least;
    rest = (least - (f - big)) + (fmaf(kB, g2, -p) + fmaf(kB, fmaf(m, m, -g2), fmaf(kBRest, g2, kARest)));
  }
  const float hi = -m * f, lo = fmaf(-m, f, -hi) - m * rest;
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(hi));
  e = fmaf(e, lo * kLn2, e);
  const float y = 1.f + e;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
  r = fmaf(r, fmaf(-y, r, 1.f), r);
  const float er = e * r, s = g < 0.f ? er : r, t = g < 0.f ? r : er;  // s(z) and 1 - s(z)
  *a = g * s;
  *da = ACT == KDN_ACT_SILU ? fmaf(*a, t, s) : fmaf(*a * t, fmaf(g2, 3.f * kGelu * kGelu3, kGelu), s);
}

// For values that are stored in bfloat16: a fast exponential (2^-22 and 2^-24 of its exponent) and reciprocal, and
// 1 - s by cancellation, 2^-24 beside a' near 1.  A third of the instructions, which bound the gradient's epilogue.
template <int ACT> __device__ __forceinline__ void ffn_act_fast(float g, float *a, float *da) {
  constexpr float kLog2e = 1.4426950408889634f;
  // g^2 of gelu ends at 1e6: s is 0 or 1 long before, and dz stays finite
  const float g2 = ACT == KDN_ACT_SILU ? 0.f : fminf(g * g, 1e6f);
  const float z = ACT == KDN_ACT_SILU ? g * -kLog2e : g * fmaf(g2, -kLog2e * kGelu * kGelu3, -kLog2e * kGelu);
  float e, s;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.f + e));
  const float y = g * s, q = fmaf(-s, y, y);  // q = g s (1 - s)
  *a = y;
  *da = ACT == KDN_ACT_SILU ? s + q : fmaf(q, fmaf(g2, 3.f * kGelu * kGelu3, kGelu), s);
}

// Floats of partial sums that a call needs.  Neither form is called without rows.
size_t ffn_part_floats_tc(const FfnArgs &a, bool back);  // bfloat16 (kdn_ffn_tc.cu)
kdn_status_t launch_ffn_fwd_tc(const FfnArgs &a, cudaStream_t s);
kdn_status_t launch_ffn_bwd_tc(const FfnArgs &a, cudaStream_t s);
// Few rows (kdn_ffn_rows.cu): the forward, and the backward but for the weights' gradients.
bool ffn_few_rows(const FfnArgs &a, bool back);
kdn_status_t launch_ffn_fwd_rows(const FfnArgs &a, cudaStream_t s);
kdn_status_t launch_ffn_bwd_rows(const FfnArgs &a, cudaStream_t s);
size_t ffn_part_floats_f32(const FfnArgs &a, bool back);  // float32 (kdn_ffn_f32.cu)
size_t ffn_planes_bytes_f32(const FfnArgs &a, bool back);
kdn_status_t launch_ffn_fwd_f32(const FfnArgs &a, cudaStream_t s);
kdn_status_t launch_ffn_bwd_f32(const FfnArgs &a, cudaStream_t s);
// Few rows in float32 (kdn_ffn_rows_f32.cu); in place of planes its workspace has dg and du.
bool ffn_few_rows_f32(const FfnArgs &a);
size_t ffn_part_floats_rows_f32(const FfnArgs &a, bool back);
size_t ffn_gradients_bytes_rows_f32(const FfnArgs &a, bool back);
kdn_status_t launch_ffn_fwd_rows_f32(const FfnArgs &a, cudaStream_t s);
kdn_status_t launch_ffn_bwd_rows_f32(const FfnArgs &a, cudaStream_t s);

}  // namespace kdn
