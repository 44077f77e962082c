// kdn_rmsnorm.cu -- the residual's addition with the RMS norm behind it, its output in
// the activations' type or in 8 bits with scales, and its gradients.
//
//   h = x + res,  rstd = (mean h^2 + eps)^-1/2,  y = h rstd w
//   8 bits: scale = max |y| / 448 over a row or over 128 columns, q = e4m3(y (1 / scale))
//   backward, g = w dy, xh = h rstd: dx = dh + rstd (g - xh mean(g xh)), dw = sum_rows dy xh
//
// A row is read once: TPR threads hold it in registers (EPT elements each, 16-byte
// vectors, vector number i TPR + thread), so the statistics, the scales and the output
// come from one pass over memory.  Sums are float32 and their order is fixed.
// HBM traffic bounds both directions.
#include <cuda_fp8.h>

#include "kdn_beside.cuh"
#include "kdn_internal.cuh"
#include "kdn_rmsnorm.cuh"

namespace kdn {
namespace {

constexpr float kF8Max = 448.f;           // largest finite e4m3 value
constexpr float kMinNormal = 0x1p-126f;  // of float32

template <typename DT> constexpr int EV = 16 / (int)sizeof(DT);  // elements of a 16-byte vector

template <typename DT> __device__ __forceinline__ void unpack(uint4 u, float *x) {
  if constexpr (sizeof(DT) == 4) {
    x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y);
    x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
  } else {
    const __nv_bfloat162 *p = reinterpret_cast<const __nv_bfloat162 *>(&u);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __bfloat1622float2(p[i]);
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
}
template <typename DT> __device__ __forceinline__ uint4 pack(const float *x) {
  uint4 u;
  if constexpr (sizeof(DT) == 4) {
    u = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  } else {
    __nv_bfloat162 *p = reinterpret_cast<__nv_bfloat162 *>(&u);
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
  }
  return u;
}

// Sum (or maximum) over the TPR threads of a row.  `red` holds one float a warp and is
// double-buffered by the caller, so one barrier a reduction is enough.
template <int TPR, bool MAX> __device__ __forceinline__ float row_reduce(float x, float *red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float y = __shfl_xor_sync(0xffffffffu, x, o);
    x = MAX ? fmaxf(x, y) : x + y;
  }
  if constexpr (TPR > 32) {
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = x;
    __syncthreads();
    x = red[0];
#pragma unroll
    for (int w = 1; w < TPR / 32; ++w) x = MAX ? fmaxf(x, red[w]) : x + red[w];
  }
  return x;
}

// threads of a CTA: eight rows of 32 threads, or one row
template <int TPR> constexpr int CTA = TPR == 32 ? 256 : TPR;

template <typename DT, int F8, int TPR, int EPT>
__global__ void __launch_bounds__(CTA<TPR>) k_add_rmsnorm(const NormArgs a) {
  constexpr int V = EV<DT>, NV = EPT / V;
  __shared__ float red[2][32];
  const long long row = (long long)blockIdx.x * (CTA<TPR> / TPR) + threadIdx.x / TPR;
  const int ln = threadIdx.x % TPR;
  if (row >= a.rows) return;  // whole warps; with TPR > 32 a CTA is one row
  const int nv = a.D / V;
  const uint4 *x = static_cast<const uint4 *>(a.x) + row * nv, *w = static_cast<const uint4 *>(a.w);
  const uint4 *r = a.res ? static_cast<const uint4 *>(a.res) + row * nv : nullptr;
  float h[NV][V];
  uint4 ux[NV], ur[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = i * TPR + ln;
    ux[i] = c < nv ? x[c] : make_uint4(0, 0, 0, 0);
    ur[i] = r && c < nv ? r[c] : make_uint4(0, 0, 0, 0);
  }
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float t[V];
    unpack<DT>(ux[i], h[i]);
    unpack<DT>(ur[i], t);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      h[i][e] += t[e];
      ss = fmaf(h[i][e], h[i][e], ss);
    }
  }
  if (a.h) {
    uint4 *o = static_cast<uint4 *>(a.h) + row * nv;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i * TPR + ln < nv) o[i * TPR + ln] = pack<DT>(h[i]);
  }
  ss = row_reduce<TPR, false>(ss, red[0]);
  const float rstd = 1.f / sqrtf(ss / (float)a.D + a.eps);
  if (a.rstd && ln == 0) a.rstd[row] = rstd;
  float big = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float t[V];
    const int c = i * TPR + ln;
    unpack<DT>(c < nv ? w[c] : make_uint4(0, 0, 0, 0), t);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      h[i][e] *= rstd * t[e];
      big = fmaxf(big, fabsf(h[i][e]));
    }
  }
  if constexpr (!F8) {
    uint4 *o = static_cast<uint4 *>(a.y) + row * nv;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i * TPR + ln < nv) o[i * TPR + ln] = pack<DT>(h[i]);
  } else {
    // a block of 128 columns is 128 / V consecutive lanes of one warp
    const int nb = a.block ? (a.D + 127) / 128 : 1;
    if (!a.block) big = row_reduce<TPR, true>(big, red[1]);
    unsigned char *o = static_cast<unsigned char *>(a.y) + row * a.D;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = i * TPR + ln;
      if (a.block) {
        big = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) big = fmaxf(big, fabsf(h[i][e]));
#pragma unroll
        for (int s = 64 / V; s > 0; s >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, s));
      }
      // an all-zero block has scale 1; so has one whose magnitudes are not finite (its
      // elements are NaN: a row with an infinity or a NaN has no finite norm)
      const bool ok = big > 0.f && big < INFINITY;
      float scale = ok ? big / kF8Max : 1.f, up = 1.f;
      if (scale < kMinNormal) {
        // its reciprocal may be infinite and itself zero: rounded up, so that no element
        // passes 448, and divided by with both moved up by an (exact) power of two
        scale = __fdiv_ru(big, kF8Max);
        up = 0x1p100f;
#pragma unroll
        for (int e = 0; e < V; ++e) h[i][e] *= up;
      }
      const float inv = 1.f / (scale * up);
      if (c < nv) {
        unsigned char q[V];
#pragma unroll
        for (int e = 0; e < V; e += 2) {
          const __nv_fp8x2_storage_t p = __nv_cvt_float2_to_fp8x2(
              make_float2(h[i][e] * inv, h[i][e + 1] * inv), __NV_SATFINITE, __NV_E4M3);
          q[e] = (unsigned char)(p & 0xff);
          q[e + 1] = (unsigned char)(p >> 8);
        }
        if constexpr (V == 8) *reinterpret_cast<uint2 *>(o + c * V) = *reinterpret_cast<const uint2 *>(q);
        else *reinterpret_cast<uint32_t *>(o + c * V) = *reinterpret_cast<const uint32_t *>(q);
        if (a.block ? (c * V) % 128 == 0 : c == 0) a.scales[row * nb + (a.block ? c * V / 128 : 0)] = scale;
      }
    }
  }
}

// Rows are dealt out to the CTAs in turn; dw stays in registers across a CTA's rows
// and leaves as one float32 row of partial sums a CTA.  A row is kept as it was loaded
// (unpacked twice) so that the next one's loads can be in flight from the start of it.
//
// WARP: a row a warp, four of them a CTA (up to 512 columns, EPT 8 or 16).  Otherwise a
// CTA a row, with as many threads as it has groups of EPT = 8 elements (16 beyond
// 8192, without the early loads, for which 64 registers do not suffice): no registers
// idle, and 1024 threads an SM whatever the width.  5.6 TB/s at 32768 x 2048 (96 us, the
// join of dw included); 128 threads of 16 elements each, without early loads: 3.4 TB/s.
template <typename DT, int EPT, bool WARP>
__global__ void __launch_bounds__(WARP ? 128 : 1024, WARP ? 4 : 1) k_add_rmsnorm_bwd(const NormArgs a) {
  constexpr int V = EV<DT>, NV = EPT / V;
  constexpr bool AHEAD = WARP || EPT == 8;
  let_next_start();
  __shared__ float red[2][32];
  __shared__ __align__(16) float s_dw[WARP ? 4 * 32 * EPT : 1];
  const int TPR = WARP ? 32 : blockDim.x, RPC = WARP ? 4 : 1;
  const int ln = WARP ? threadIdx.x % 32 : threadIdx.x, sub = WARP ? threadIdx.x / 32 : 0, nv = a.D / V;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  float dw[NV][V] = {};
  uint4 w[NV];
  struct Row {
    uint4 h[NV], y[NV], d[NV];
    float rstd;
  };
  Row cur, next;
#pragma unroll
  for (int i = 0; i < NV; ++i) w[i] = i * TPR + ln < nv ? static_cast<const uint4 *>(a.w)[i * TPR + ln] : zero;
  auto load = [&](Row &r, long long row) {
    const bool in = row < a.rows;
    r.rstd = in ? a.rstd_in[row] : 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = i * TPR + ln;
      const bool ok = in && c < nv;
      r.h[i] = ok ? static_cast<const uint4 *>(a.hin)[row * nv + c] : zero;
      r.y[i] = ok ? static_cast<const uint4 *>(a.dy)[row * nv + c] : zero;
      r.d[i] = ok && a.dh ? static_cast<const uint4 *>(a.dh)[row * nv + c] : zero;
    }
  };
  const long long step = (long long)gridDim.x * RPC;
  long long row = (long long)blockIdx.x * RPC + sub;
  load(cur, row);
  for (int par = 0; row < a.rows; row += step, par ^= 1) {
    if (AHEAD) load(next, row + step);
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float xh[V], g[V], t[V];
      unpack<DT>(cur.h[i], xh);
      unpack<DT>(cur.y[i], g);
      unpack<DT>(w[i], t);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        xh[e] *= cur.rstd;
        dw[i][e] = fmaf(g[e], xh[e], dw[i][e]);
        dot = fmaf(g[e] * t[e], xh[e], dot);
      }
    }
    dot = warp_sum(dot);
    if constexpr (!WARP) {  // two rows' sums have their own places: one barrier a row
      if (threadIdx.x % 32 == 0) red[par][threadIdx.x / 32] = dot;
      __syncthreads();
      dot = warp_sum(threadIdx.x % 32 < blockDim.x / 32 ? red[par][threadIdx.x % 32] : 0.f);
    }
    dot = dot / (float)a.D * cur.rstd;
    uint4 *o = static_cast<uint4 *>(a.dx) + row * nv;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float h[V], g[V], t[V], d[V];
      unpack<DT>(cur.h[i], h);
      unpack<DT>(cur.y[i], g);
      unpack<DT>(w[i], t);
      unpack<DT>(cur.d[i], d);
#pragma unroll
      for (int e = 0; e < V; ++e) d[e] = fmaf(cur.rstd, fmaf(-dot, h[e], g[e] * t[e]), d[e]);
      if (i * TPR + ln < nv) o[i * TPR + ln] = pack<DT>(d);
    }
    if (AHEAD) cur = next;
    else load(cur, row + step);
  }
  float *part = a.part + (size_t)blockIdx.x * a.D;
  if constexpr (!WARP) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = i * TPR + ln;
      if (c < nv)
#pragma unroll
        for (int e = 0; e < V; ++e) part[c * V + e] = dw[i][e];
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) s_dw[sub * 32 * EPT + (i * 32 + ln) * V + e] = dw[i][e];
    __syncthreads();
    for (int c = threadIdx.x; c < a.D; c += 128) {
      float x = 0.f;
#pragma unroll
      for (int r = 0; r < 4; ++r) x += s_dw[r * 32 * EPT + c];
      part[c] = x;
    }
  }
}

// dw: the CTAs' partial rows added in order, 32 columns a CTA.
__global__ void __launch_bounds__(1024) k_rmsnorm_dw(const float *part, int n, int D, float *dw) {
  __shared__ float s[32][33];
  const int cx = threadIdx.x % 32, ry = threadIdx.x / 32, c = blockIdx.x * 32 + cx;
  wait_for_previous();
  float x = 0.f;
  if (c < D)
    for (int r = ry; r < n; r += 32) x += part[(size_t)r * D + c];
  s[ry][cx] = x;
  __syncthreads();
  if (ry == 0 && c < D) {
    float y = 0.f;
#pragma unroll
    for (int r = 0; r < 32; ++r) y += s[r][cx];
    dw[c] = y;
  }
}

kdn_status_t launched() { return cudaGetLastError() == cudaSuccess ? KDN_OK : KDN_ERR_CUDA; }

// Threads a row and elements a thread: a warp a row up to 1024 columns (no barrier),
// else 128 threads (up to 4096) or 512.  Elements past a row are idle registers, so
// the steps are small: 2304 columns with 32 elements a thread in place of 24 took half
// as long again with an 8-bit output.
template <int TPR, int EPT> struct Shape { static constexpr int tpr = TPR, ept = EPT; };
template <typename F> kdn_status_t by_shape(int D, F f) {
  if (D <= 256) return f(Shape<32, 8>{});
  if (D <= 512) return f(Shape<32, 16>{});
  if (D <= 1024) return f(Shape<32, 32>{});
  if (D <= 128 * 16) return f(Shape<128, 16>{});
  if (D <= 128 * 24) return f(Shape<128, 24>{});
  if (D <= 4096) return f(Shape<128, 32>{});
  if (D <= 8192) return f(Shape<512, 16>{});
  return f(Shape<512, 32>{});
}

template <typename DT, int F8> kdn_status_t fwd_t(const NormArgs &a, cudaStream_t s) {
  return by_shape(a.D, [&](auto sh) {
    constexpr int TPR = decltype(sh)::tpr, EPT = decltype(sh)::ept, RPC = CTA<TPR> / TPR;
    k_add_rmsnorm<DT, F8, TPR, EPT><<<(unsigned)((a.rows + RPC - 1) / RPC), CTA<TPR>, 0, s>>>(a);
    return launched();
  });
}

// Threads of the backward's CTA: four rows of a warp, or a row with EPT elements a thread.
int bwd_threads(int D) {
  if (D <= 512) return 128;
  const int ept = D <= 8192 ? 8 : 16;
  return ((D + ept - 1) / ept + 31) / 32 * 32;
}

template <typename DT> kdn_status_t bwd_t(const NormArgs &a, cudaStream_t s) {
  const int n = rmsnorm_bwd_blocks(a.rows, a.D), nt = bwd_threads(a.D);
  if (n) {
    if (a.D <= 256) k_add_rmsnorm_bwd<DT, 8, true><<<n, nt, 0, s>>>(a);
    else if (a.D <= 512) k_add_rmsnorm_bwd<DT, 16, true><<<n, nt, 0, s>>>(a);
    else if (a.D <= 8192) k_add_rmsnorm_bwd<DT, 8, false><<<n, nt, 0, s>>>(a);
    else k_add_rmsnorm_bwd<DT, 16, false><<<n, nt, 0, s>>>(a);
  }
  if (launched() != KDN_OK) return KDN_ERR_CUDA;
  return launch_beside(k_rmsnorm_dw, dim3((a.D + 31) / 32), 1024, 0, s, (const float *)a.part, n, a.D, a.dw);
}

}  // namespace

// CTAs of the backward: those that are resident at once, each with its own row of partial sums.
int rmsnorm_bwd_blocks(long long rows, int D) {
  const long long rpc = D <= 512 ? 4 : 1, full = 152LL * (D <= 512 ? 4 : 1024 / bwd_threads(D));
  const long long n = (rows + rpc - 1) / rpc;
  return (int)(n < full ? n : full);
}

kdn_status_t launch_add_rmsnorm(const NormArgs &a, cudaStream_t s) {
  if (a.dtype == KDN_BF16) return a.f8 ? fwd_t<__nv_bfloat16, 1>(a, s) : fwd_t<__nv_bfloat16, 0>(a, s);
  return a.f8 ? fwd_t<float, 1>(a, s) : fwd_t<float, 0>(a, s);
}

kdn_status_t launch_add_rmsnorm_bwd(const NormArgs &a, cudaStream_t s) {
  return a.dtype == KDN_BF16 ? bwd_t<__nv_bfloat16>(a, s) : bwd_t<float>(a, s);
}

}  // namespace kdn
