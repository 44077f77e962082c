// kdn_ffn_rows_f32.cu -- the feed-forward block of up to 16 tokens in float32, on the CUDA cores.
//
// The weights are read once and every value meets each token in a multiply-add; nothing has to be cut into bfloat16s
// first, which takes longer than all of this.
//   dot    C[t, m] = sum_k X(t, k) W(m, k): a warp takes four rows of the weights (of the gate two of Wg and two of
//          Wu), a lane four values of k at a time, tokens pass through shared memory: g, u, h; y
//   column C[t, c] = sum_r X(t, r) W(r, c): a lane takes four columns, the warps of a CTA rows in turn, CTAs parts of
//          the rows; a second kernel adds the parts in order: dh, and with g and u dg and du; dx
//   outer  C[m, n] = sum_t A(t, m) B(t, n): the weights' gradients
// Weights of 3272 x 8192 (322 MB): 1 token 61 us forward (5.3 TB/s) and 120 of gradients, which write as much as they
// read (writes alone reach 4 TB/s); 16 tokens 112 and 171, where dot waits for shared memory and for itself (two CTAs an
// SM of four warps, a 16-byte read of a token for eight double multiply-adds; FMA pipe 19 %).  The tensor cores' form
// takes 290 and 396, and 17 tokens of 520 x 1400 25 and 43 us where 12 take 12 and 23 here.  Above 16 the sums do not
// fit a thread's registers; a second pass over the weights for 17 to 32 tokens has not been tried.
#include "kdn_ffn.cuh"

namespace kdn {
namespace {

constexpr int NT = 256, WARPS = NT / 32, CHUNK = 512, COLS = 128;

// Two multiply-adds in one instruction.
using Pair = unsigned long long;
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ Pair pair(float lo, float hi) {
  Pair d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ float sum_of(Pair p) {
  float lo, hi;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p));
  return lo + hi;
}

struct Dot {
  const float *x, *w[2];
  float *out[3];  // y; the gate: h, g, u (null: not written)
  int rows, K, M, act;
  unsigned *status;  // cleared by the gate
};

__device__ __forceinline__ float act_of(int act, float g) {
  float a, da;
  if (act == KDN_ACT_SILU) ffn_act_near<KDN_ACT_SILU>(g, &a, &da);
  else ffn_act_near<KDN_ACT_GELU>(g, &a, &da);
  return a;
}

// How dot goes through K: threads of a CTA, and values of K a pass.  A lane holds one pass's weights and fetches the
// next one's, as many as its registers take beside the sums (3272 x 8192, 8 tokens: 512 of K 77 us, 256 92).  Small
// CTAs come to an end evenly; more tokens share their copies among more warps (16 tokens: CTAs of 256 134 us, 128 117;
// 4 tokens: 128 68, 64 65).
template <int R> struct Pass {
  static constexpr int T = R <= 4 ? 64 : 128, N = R <= 8 ? 512 : 256, SMEM = 2 * R * N * (int)sizeof(float);
};
template <int R> struct Weights {
  static constexpr int S = Pass<R>::N / 128;
  ulonglong2 v[S][4];  // four values of k as two pairs
  __device__ __forceinline__ void load(const float *const (&w)[4], int k0, int K) {
#pragma unroll
    for (int i = 0; i < S; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = k0 + 128 * i + 4 * (threadIdx.x & 31);
        v[i][j] = k < K ? __ldcs(reinterpret_cast<const ulonglong2 *>(w[j] + k)) : make_ulonglong2(0, 0);
      }
  }
};
template <int R> __device__ __forceinline__ void tokens(float *xs, const float *x, int rows, int k0, int K) {
  constexpr int N = Pass<R>::N;
  for (int e = threadIdx.x * 4; e < R * N; e += Pass<R>::T * 4) {
    const int t = e / N, k = k0 + e % N;
    const bool in = t < rows && k < K;
    // (nothing is read where the source size is zero; zeros are written)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((unsigned)__cvta_generic_to_shared(xs + e)),
                 "l"(x + (in ? (size_t)t * K + k : 0)), "r"(in ? 16 : 0)
                 : "memory");
  }
  asm volatile("cp.async.commit_group;" ::: "memory");
}

// Sums over a warp of R values a lane: lane l is left with value l % R (R = 12 is filled up to 16).  In each step a lane
// hands half of its values on and adds the other half of its partner's.
template <int R> __device__ __forceinline__ float sum_across(const Pair (&acc)[R]) {
  constexpr int M = R == 12 ? 16 : R;
  const int lane = threadIdx.x & 31;
  float v[M];
#pragma unroll
  for (int t = 0; t < M; ++t) v[t] = t < R ? sum_of(acc[t < R ? t : 0]) : 0.f;
#pragma unroll
  for (int h = M / 2; h > 0; h /= 2) {
    const bool up = lane & h;
#pragma unroll
    for (int t = 0; t < h; ++t) {
      const float give = up ? v[t] : v[t + h], keep = up ? v[t + h] : v[t];
      v[t] = keep + __shfl_xor_sync(0xffffffffu, give, h);
    }
  }
#pragma unroll
  for (int h = M; h < 32; h *= 2) v[0] += __shfl_xor_sync(0xffffffffu, v[0], h);
  return v[0];
}

template <int R, bool GATE> __global__ void __launch_bounds__(Pass<R>::T) k_ffn_dot(const Dot P) {
  extern __shared__ float xs[];  // [2][R][N]
  constexpr int N = Pass<R>::N, PER = GATE ? 2 : 4;  // PER: of C's columns a warp
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int m0 = (blockIdx.x * (Pass<R>::T / 32) + warp) * PER;
  const float *w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = P.w[GATE ? j >> 1 : 0] + (size_t)min(m0 + (GATE ? j & 1 : j), P.M - 1) * P.K;
  Weights<R> v;
  // the gate is a call's first kernel and lets the next one start once all before the call is done: Wd is there
  if (GATE) wait_for_previous();
  let_next_start();
  v.load(w, 0, P.K);
  if (!GATE) wait_for_previous();
  if (GATE && blockIdx.x == 0 && threadIdx.x == 0) *P.status = 0;
  Pair acc[4][R];  // sums over even and odd k
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int t = 0; t < R; ++t) acc[j][t] = 0;
  tokens<R>(xs, P.x, P.rows, 0, P.K);
  for (int k0 = 0, odd = 0; k0 < P.K; k0 += N, odd ^= 1) {
    Weights<R> next;
    next.load(w, k0 + N, P.K);  // (zeros behind K)
    if (k0 + N < P.K) tokens<R>(xs + (odd ^ 1) * R * N, P.x, P.rows, k0 + N, P.K);
    if (k0 + N < P.K) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    const float *xc = xs + odd * R * N + 4 * lane;
#pragma unroll
    for (int i = 0; i < N / 128; ++i)
#pragma unroll
      for (int t = 0; t < R; ++t) {
        const ulonglong2 x = *reinterpret_cast<const ulonglong2 *>(xc + t * N + 128 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j][t] = fma2(v.v[i][j].y, x.y, fma2(v.v[i][j].x, x.x, acc[j][t]));
      }
    __syncthreads();  // the other half of xs is written again
    v = next;
  }
  float mine[4];  // lane t: token t's
#pragma unroll
  for (int j = 0; j < 4; ++j) mine[j] = sum_across<R>(acc[j]);
  if (lane >= P.rows) return;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    if (m0 + j >= P.M) continue;
    const size_t at = (size_t)lane * P.M + m0 + j;
    if (GATE) {
      const float g = mine[j], u = mine[j + 2];
      if (P.out[1]) {
        P.out[1][at] = g;
        P.out[2][at] = u;
      }
      P.out[0][at] = act_of(P.act, g) * u;
    } else {
      P.out[0][at] = mine[j];
    }
  }
}

// A token's values behind one another become a value's tokens behind one another.
template <int R> __device__ __forceinline__ void across_tokens(float *to, const float *x, int stride, int n, int rows) {
  for (int i = threadIdx.x; i < n; i += NT) {
    float f[R];
#pragma unroll
    for (int t = 0; t < R; ++t) f[t] = t < rows ? x[(size_t)t * stride + i] : 0.f;
#pragma unroll
    for (int t = 0; t < R; ++t) to[i * R + t] = f[t];
  }
}

struct Column {
  const float *x[2], *w[2];  // two sums, one behind the other (the second null: one)
  float *part;               // [parts][rows][C]
  int rows, N, C, parts;     // N: rows of a weight matrix
  unsigned *status;
};
template <int R> __global__ void __launch_bounds__(NT) k_ffn_column(const Column P) {
  extern __shared__ float sm[];  // x [rows of this part][R], then sums [WARPS][R][COLS]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = blockIdx.x * COLS + 4 * lane;
  const int halves = P.w[1] ? 2 : 1, per = P.parts / halves, half = blockIdx.y / per, i = blockIdx.y - half * per;
  const int r0 = (int)((long long)P.N * i / per), r1 = (int)((long long)P.N * (i + 1) / per);
  const float *w = half ? P.w[1] : P.w[0], *x = half ? P.x[1] : P.x[0];
  wait_for_previous();
  let_next_start();
  if (P.status && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *P.status = 0;
  ulonglong2 acc[R];  // four columns as two pairs
#pragma unroll
  for (int t = 0; t < R; ++t) acc[t] = make_ulonglong2(0, 0);
  for (int b = r0; b < r1; b += CHUNK) {
    const int n = min(CHUNK, r1 - b);
    __syncthreads();
    across_tokens<R>(sm, x + b, P.N, n, P.rows);
    __syncthreads();
    constexpr int AHEAD = 8;
    for (int r = warp; r < n; r += WARPS * AHEAD) {
      ulonglong2 v[AHEAD];
#pragma unroll
      for (int a = 0; a < AHEAD; ++a)
        v[a] = r + a * WARPS < n && c < P.C
                   ? __ldcs(reinterpret_cast<const ulonglong2 *>(w + (size_t)(b + r + a * WARPS) * P.C + c))
                   : make_ulonglong2(0, 0);
#pragma unroll
      for (int a = 0; a < AHEAD; ++a) {
        if (r + a * WARPS >= n) continue;
        const float *xr = sm + (r + a * WARPS) * R;
#pragma unroll
        for (int t = 0; t < R; ++t) {
          const Pair f = pair(xr[t], xr[t]);
          acc[t].x = fma2(f, v[a].x, acc[t].x);
          acc[t].y = fma2(f, v[a].y, acc[t].y);
        }
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < R; ++t) *reinterpret_cast<ulonglong2 *>(sm + (warp * R + t) * COLS + 4 * lane) = acc[t];
  __syncthreads();
  for (int e = threadIdx.x; e < P.rows * COLS; e += NT) {
    const int t = e / COLS, k = e % COLS;
    if (blockIdx.x * COLS + k >= P.C) continue;
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < WARPS; ++j) s += sm[(j * R + t) * COLS + k];
    P.part[((size_t)blockIdx.y * P.rows + t) * P.C + blockIdx.x * COLS + k] = s;
  }
}

// Parts added in order: dx, or dh and with g and u what follows from it.
struct Finish {
  const float *part, *g, *u;
  float *out[2];
  size_t n;
  int parts, act;
};
template <bool DGATE> __global__ void __launch_bounds__(NT) k_ffn_finish(const Finish P) {
  wait_for_previous();
  let_next_start();
  for (size_t i = (size_t)blockIdx.x * NT + threadIdx.x; i < P.n; i += (size_t)gridDim.x * NT) {
    float s = 0.f;
    for (int j = 0; j < P.parts; ++j) s += P.part[j * P.n + i];
    if (DGATE) {
      float a, da;
      if (P.act == KDN_ACT_SILU) ffn_act_near<KDN_ACT_SILU>(P.g[i], &a, &da);
      else ffn_act_near<KDN_ACT_GELU>(P.g[i], &a, &da);
      P.out[0][i] = s * P.u[i] * da;
      P.out[1][i] = s * a;
    } else {
      P.out[0][i] = s;
    }
  }
}

struct Outer {
  const float *a[3], *b[3];
  float *out[3];
  int M[3], N[3], first[3], rows, side;  // first: of a problem's CTAs; side: rows of C a CTA
};
template <int R> __global__ void __launch_bounds__(NT) k_ffn_outer(const Outer P) {
  extern __shared__ float as[];  // [side][R]
  const int p = (blockIdx.x >= P.first[1]) + (blockIdx.x >= P.first[2]), warp = threadIdx.x >> 5;
  const int M = P.M[p], N = P.N[p], i = blockIdx.x - P.first[p], across = (N + COLS - 1) / COLS;
  const int m0 = i / across * P.side, n = i % across * COLS + 4 * (threadIdx.x & 31);
  wait_for_previous();
  let_next_start();
  const int side = min(P.side, M - m0);
  across_tokens<R>(as, P.a[p] + m0, M, side, P.rows);
  ulonglong2 b[R];
#pragma unroll
  for (int t = 0; t < R; ++t)
    b[t] = t < P.rows && n < N ? *reinterpret_cast<const ulonglong2 *>(P.b[p] + (size_t)t * N + n)
                               : make_ulonglong2(0, 0);
  __syncthreads();
  for (int m = warp; m < side; m += WARPS) {
    ulonglong2 s = make_ulonglong2(0, 0);
#pragma unroll
    for (int t = 0; t < R; ++t) {
      const Pair f = pair(as[m * R + t], as[m * R + t]);
      s.x = fma2(f, b[t].x, s.x);
      s.y = fma2(f, b[t].y, s.y);
    }
    if (n < N) *reinterpret_cast<ulonglong2 *>(P.out[p] + (size_t)(m0 + m) * N + n) = s;
  }
}

template <int R, bool GATE> kdn_status_t dot(const Dot &P, cudaStream_t s) {
  const int per = Pass<R>::T / 32 * (GATE ? 2 : 4);
  return launch_beside(k_ffn_dot<R, GATE>, dim3((P.M + per - 1) / per), Pass<R>::T, Pass<R>::SMEM, s, P);
}

// Parts of a column sum: four CTAs an SM (one token of 3272 x 8192: 55 us for both sums, with two an SM 63), 64 rows
// each at least.
int parts_of(int N, int C, int halves) {
  const int blocks = (C + COLS - 1) / COLS * halves;
  int per = 608 / blocks;
  if (per > N / 64) per = N / 64;
  return halves * (per < 1 ? 1 : per);
}
template <int R> kdn_status_t column(const Column &P, cudaStream_t s) {
  constexpr int bytes = (CHUNK > WARPS * COLS ? CHUNK : WARPS * COLS) * R * (int)sizeof(float);
  if (bytes > 48 * 1024 && cudaFuncSetAttribute(k_ffn_column<R>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) !=
                               cudaSuccess)
    return KDN_ERR_CUDA;
  return launch_beside(k_ffn_column<R>, dim3((P.C + COLS - 1) / COLS, P.parts), NT, bytes, s, P);
}
template <bool DGATE> kdn_status_t finish(const Finish &P, cudaStream_t s) {
  const size_t blocks = (P.n + NT - 1) / NT;
  return launch_beside(k_ffn_finish<DGATE>, dim3((unsigned)(blocks < 1216 ? blocks : 1216)), NT, 0, s, P);
}

template <int R> kdn_status_t forward(const FfnArgs &a, cudaStream_t s) {
  const auto f = [](const void *p) { return static_cast<const float *>(p); };
  const auto o = [](void *p) { return static_cast<float *>(p); };
  const Dot up{f(a.x), {f(a.wg), f(a.wu)}, {o(a.h), o(a.g), o(a.u)}, (int)a.rows, a.D, a.F, a.act, a.status};
  const kdn_status_t st = dot<R, true>(up, s);
  if (st != KDN_OK) return st;
  const Dot down{f(a.h), {f(a.wd), nullptr}, {o(a.y), nullptr, nullptr}, (int)a.rows, a.F, a.D, a.act, nullptr};
  return dot<R, false>(down, s);
}

template <int R> kdn_status_t backward(const FfnArgs &a, cudaStream_t s) {
  const auto f = [](const void *p) { return static_cast<const float *>(p); };
  const auto o = [](void *p) { return static_cast<float *>(p); };
  const int rows = (int)a.rows;
  float *const dg = o(a.planes), *const du = dg + (size_t)rows * a.F;  // (F is a multiple of 8: 16 bytes)
  const Column dh{{f(a.dy), nullptr}, {f(a.wd), nullptr}, a.part, rows, a.D, a.F, parts_of(a.D, a.F, 1), a.status};
  kdn_status_t st = column<R>(dh, s);
  if (st != KDN_OK) return st;
  const Finish gate{a.part, f(a.g), f(a.u), {dg, du}, (size_t)rows * a.F, dh.parts, a.act};
  if ((st = finish<true>(gate, s)) != KDN_OK) return st;
  const Column dx{{dg, du}, {f(a.wg), f(a.wu)}, a.part, rows, a.F, a.D, parts_of(a.F, a.D, 2), nullptr};
  if ((st = column<R>(dx, s)) != KDN_OK) return st;
  const Finish sum{a.part, nullptr, nullptr, {o(a.dx), nullptr}, (size_t)rows * a.D, dx.parts, a.act};
  if ((st = finish<false>(sum, s)) != KDN_OK) return st;
  Outer w{{dg, du, f(a.dy)}, {f(a.x), f(a.x), f(a.h)}, {o(a.dwg), o(a.dwu), o(a.dwd)},
          {a.F, a.F, a.D}, {a.D, a.D, a.F}, {}, rows};
  // A CTA reads its tokens' values once for all of its side, so a long one (2 tokens of 3272 x 8192: 256 rows 60 us, 64
  // rows 72); four CTAs an SM if there is that much.
  const auto blocks = [&w](int side) {
    long long n = 0;
    for (int p = 0; p < 3; ++p) {
      w.first[p] = (int)n;
      n += (long long)((w.M[p] + side - 1) / side) * ((w.N[p] + COLS - 1) / COLS);
    }
    return n;
  };
  w.side = 256;
  while (w.side > 32 && blocks(w.side) < 608) w.side /= 2;
  const unsigned grid = (unsigned)blocks(w.side);
  return launch_beside(k_ffn_outer<R>, dim3(grid), NT, w.side * R * (int)sizeof(float), s, w);
}

}  // namespace

bool ffn_few_rows_f32(const FfnArgs &a) { return a.rows <= 16; }

size_t ffn_gradients_bytes_rows_f32(const FfnArgs &a, bool back) {
  return back ? ((size_t)2 * a.rows * a.F * sizeof(float) + 255) / 256 * 256 : 0;
}

size_t ffn_part_floats_rows_f32(const FfnArgs &a, bool back) {
  if (!back) return 0;
  const size_t dh = (size_t)parts_of(a.D, a.F, 1) * a.rows * a.F, dx = (size_t)parts_of(a.F, a.D, 2) * a.rows * a.D;
  return dh > dx ? dh : dx;
}

kdn_status_t launch_ffn_fwd_rows_f32(const FfnArgs &a, cudaStream_t s) {
  return a.rows <= 2   ? forward<2>(a, s)
         : a.rows <= 4 ? forward<4>(a, s)
         : a.rows <= 8 ? forward<8>(a, s)
         : a.rows <= 12 ? forward<12>(a, s)
                       : forward<16>(a, s);
}
kdn_status_t launch_ffn_bwd_rows_f32(const FfnArgs &a, cudaStream_t s) {
  return a.rows <= 2   ? backward<2>(a, s)
         : a.rows <= 4 ? backward<4>(a, s)
         : a.rows <= 8 ? backward<8>(a, s)
         : a.rows <= 12 ? backward<12>(a, s)
                       : backward<16>(a, s);
}

}  // namespace kdn
