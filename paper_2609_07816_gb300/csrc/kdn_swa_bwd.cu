// kdn_swa_bwd.cu -- gradients of the sliding-window attention with sinks on the tensor
// cores (bfloat16; d = 32 runs as 64 with the upper half of every row loaded as zeros),
// from the forward's o and lse.
//
//   P = exp2(c2 S - nlse), dP = dO V^T, dS = P (dP - delta),
//   dV = P^T dO, dK = c dS^T Q, dQ = c dS K
//
// Two kernels, each the owner of what it sums, so that no sum depends on timing and no
// float32 dQ goes through memory: seven products of 128 x 128 x d a tile pair in place of
// the five of a single kernel that adds dQ with atomics.
//   k_swa_dkv  a CTA owns 128 keys of a kv head and goes over the query tiles that see
//              them, for every query head of the group.  S^T and dP^T have keys as rows:
//              P^T and dS^T go back to TMEM as bf16 A operands of dV and dK, both in the
//              place of dP^T, so that the next S^T is formed while P and dS are.
//   k_swa_dq   a CTA owns 128 queries and goes over the keys that they see.  Its CTAs start
//              on the SMs that k_swa_dkv's last ones leave idle.
// 256 threads do the pointwise part, each a row and 64 of its 128 columns (two threads
// share a row), one warp loads, one thread issues the products.
#include "kdn_swa_tc.cuh"

namespace kdn {
namespace {

using namespace swa;

// Barrier of the 128 (or 256) threads that share `id`.
__device__ __forceinline__ void named_sync(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
constexpr int THREADS = 384, SOFT = 256;
template <int D> constexpr int TILE_BYTES = D / 64 * SLAB;

// acc (TMEM) += A B over K = d: both tiles along their 64-element rows
template <int D> __device__ __forceinline__ void mma_d(uint32_t acc, uint64_t a, uint64_t b, uint32_t id) {
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) umma_bf16(acc, a + step_k(kk), b + step_k(kk), id, kk > 0);
}
// acc += A B over the 128 columns of A in TMEM, which lie as bf16 in 32 columns of each
// 64-column half of their region; B along its rows
__device__ __forceinline__ void mma_t(uint32_t acc, uint32_t a, uint64_t b, uint32_t id, uint32_t accumulate) {
#pragma unroll
  for (int kk = 0; kk < TILE / 16; ++kk)
    umma_ts(acc, a + (kk >> 2) * 64 + (kk & 3) * 8, b + step_mn(kk), id, kk ? 1u : accumulate);
}

// 64 values as bf16 in 32 registers, and those into 32 columns
__device__ __forceinline__ void pack64(uint32_t *u, const float *x) {
#pragma unroll
  for (int e = 0; e < 32; ++e) u[e] = pack_bf2(x[2 * e], x[2 * e + 1]);
}
__device__ __forceinline__ void store32(uint32_t taddr, const uint32_t *u) {
  tmem_st16u(taddr, u);
  tmem_st16u(taddr + 16, u + 16);
}

// Columns [c0, c0 + n) of a 128-row accumulator times f as bf16 into a swizzled tile
template <int N>
__device__ __forceinline__ void acc_to_tile(uint32_t taddr, unsigned char *tile, int r, int c0, float f, bool live,
                                            bool written) {
#pragma unroll
  for (int c = c0; c < c0 + N; c += 32) {
    float o[32];
    if (written) {
      tmem_ld32(taddr + c, o);
      tmem_ld_wait<32>(o);
    }
#pragma unroll
    for (int e = 0; e < 32; e += 8) {
      uint32_t u[4];
#pragma unroll
      for (int p = 0; p < 4; ++p) u[p] = live ? pack_bf2(o[e + 2 * p] * f, o[e + 2 * p + 1] * f) : 0u;
      sm16(tile + (c >> 6) * SLAB, chunk_off(r, ((c & 63) + e) >> 3)) = make_uint4(u[0], u[1], u[2], u[3]);
    }
  }
}

// ------------------------------------------------------------------ dK, dV

constexpr int KV_STAGES = 2;  // stages of (Q, dO)
constexpr int ROW_STAGES = 4;  // stages of the row sums, which come by plain loads
template <int D> constexpr int KV_SMEM = (2 + 2 * KV_STAGES) * TILE_BYTES<D> + ROW_STAGES * 2 * TILE * 4 + 256 + 1024;

template <int D>
__global__ void __launch_bounds__(THREADS, 1)
    k_swa_dkv(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
              const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mg,
              const __grid_constant__ CUtensorMap mdk, const __grid_constant__ CUtensorMap mdv, const SwaArgs a,
              const SwaSplits sp) {
  constexpr int NS = KV_STAGES, NR = ROW_STAGES, TB = TILE_BYTES<D>, SL = D / 64;
  extern __shared__ unsigned char smraw[];
  unsigned char *sm =
      reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smraw) + 1023) & ~uintptr_t(1023));
  unsigned char *sk = sm, *sv = sk + TB, *sq = sv + TB, *sg = sq + NS * TB;
  float *srow = reinterpret_cast<float *>(sg + NS * TB);  // [stage][nlse, delta][128]
  uint64_t *bars = reinterpret_cast<uint64_t *>(srow + NR * 2 * TILE);
  uint64_t *q_full = bars, *q_empty = q_full + NS, *g_full = q_empty + NS, *g_empty = g_full + NS;
  uint64_t *clean = g_empty + NS, *l_full = clean + NS, *l_empty = l_full + NR;
  uint64_t *kv_full = l_empty + NR, *s_full = kv_full + 2, *s_read = s_full + 1, *dp_full = s_read + 1;
  uint64_t *p_full = dp_full + 1, *ds_full = p_full + 1, *done = ds_full + 1;
  uint32_t *s_tmem = reinterpret_cast<uint32_t *>(done + 1);
  int *s_fail = reinterpret_cast<int *>(s_tmem + 1);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = blockIdx.z, hk = blockIdx.y, x = blockIdx.x;
  const int nsx = sp.sink_tiles * sp.splits_sink;
  const int t = x < nsx ? x / sp.splits_sink : sp.sink_tiles + (x - nsx) / sp.splits;
  const int split = x < nsx ? x % sp.splits_sink : (x - nsx) % sp.splits;
  const int per = x < nsx ? sp.per_sink : sp.per;
  const int len = swa_len(a, b), j0 = t * TILE;
  int first = 0, last = -1;
  if (j0 < len) swa_query_tiles(t, TILE, TILE, a.W, a.ns, len, &first, &last);
  const int nq = last - first + 1, it0 = split * per, N = max(0, min(per, a.G * nq - it0));

  // the loading thread: K, V and the first stages are on their way before the CTA meets
  int loads = 0, load_h = hk * a.G, load_q = 0;
  auto load_q_tile = [&](int n) {
    const int st = n % NS;
    mbar_expect_tx(q_full + st, TB);
    for (int s = 0; s < SL; ++s)
      tma_load_4d(sq + st * TB + s * SLAB, &mq, q_full + st, 64 * s, load_h, (first + load_q) * TILE, b);
  };
  auto load_g_tile = [&](int n) {
    const int st = n % NS;
    mbar_expect_tx(g_full + st, TB);
    for (int s = 0; s < SL; ++s)
      tma_load_4d(sg + st * TB + s * SLAB, &mg, g_full + st, 64 * s, load_h, (first + load_q) * TILE, b);
    if (++load_q == nq) { load_q = 0; ++load_h; }
  };
  if (tid == SOFT) {
    for (int i = 0; i < NS; ++i) {
      mbar_init(q_full + i, 1);
      mbar_init(q_empty + i, 1);
      mbar_init(g_full + i, 1);
      mbar_init(g_empty + i, 1);
      mbar_init(clean + i, 1);
    }
    for (int i = 0; i < NR; ++i) {
      mbar_init(l_full + i, 1);
      mbar_init(l_empty + i, SOFT);
    }
    mbar_init(kv_full, 1);
    mbar_init(kv_full + 1, 1);
    mbar_init(s_full, 1);
    mbar_init(s_read, SOFT);
    mbar_init(dp_full, 1);
    mbar_init(p_full, SOFT);
    mbar_init(ds_full, SOFT);
    mbar_init(done, 1);
    *s_fail = 0;
    fence_mbar_init();
    fence_proxy_async();
    if (N > 0) {
      load_h += it0 / nq;
      load_q = it0 % nq;
      mbar_expect_tx(kv_full, TB);
      for (int s = 0; s < SL; ++s) tma_load_4d(sk + s * SLAB, &mk, kv_full, 64 * s, hk, j0, b);
      load_q_tile(0);
      mbar_expect_tx(kv_full + 1, TB);
      for (int s = 0; s < SL; ++s) tma_load_4d(sv + s * SLAB, &mv, kv_full + 1, 64 * s, hk, j0, b);
      load_g_tile(0);
      for (loads = 1; loads < min(NS, N); ++loads) {
        load_q_tile(loads);
        load_g_tile(loads);
      }
    }
  }
  if (warp == 0) {
    tmem_alloc(s_tmem, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tb = *s_tmem, TS = tb, TP = tb + 128, TV = tb + 256, TK = tb + 384;
  const Waiter wait{s_fail, a.status};

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 8 && N > 0) {
      if (lane == 0) {  // ------------------------------------------------ loads
        int n = loads;
        for (; n < N; ++n) {
          const int st = n % NS, par = (n / NS - 1) & 1;
          if (!wait.lazy(q_empty + st, par)) break;
          load_q_tile(n);
          if (!wait.lazy(g_empty + st, par)) break;
          load_g_tile(n);
        }
        if (*wait.fail) {  // copies in flight land before the CTA leaves
          mbar_wait(kv_full, 0, kWait >> 6);
          mbar_wait(kv_full + 1, 0, kWait >> 6);
          for (int m = max(0, n - NS); m <= min(n, N - 1); ++m) mbar_wait(q_full + m % NS, (m / NS) & 1, kWait >> 6);
          for (int m = max(0, n - NS); m < n; ++m) mbar_wait(g_full + m % NS, (m / NS) & 1, kWait >> 6);
        }
      }
    } else if (warp == 9 && N > 0) {  // ---------------------------------- products
      if (elect_one()) {
        const uint32_t id_s = idesc_bf16(TILE, TILE, 0, 0), id_o = idesc_bf16(TILE, D, 0, 1);
        const uint64_t dk = desc_k(sk), dv = desc_k(sv), dq = desc_k(sq), dg = desc_k(sg);
        const uint64_t mq_ = desc_mn(sq), mg_ = desc_mn(sg);
        auto off = [](int st) { return (uint64_t)(st * (TB >> 4)); };
        bool ok = wait(kv_full, 0);
        // S^T of query tile n
        auto s_mma = [&](int n) {
          const int st = n % NS, par = (n / NS) & 1;
          if (!wait(q_full + st, par)) return false;
          if (len < a.T && !wait(clean + st, par)) return false;
          mma_d<D>(TS, dk, dq + off(st), id_s);
          umma_commit(s_full);
          return true;
        };
        auto dp_mma = [&](int n) {
          if (!wait(g_full + n % NS, (n / NS) & 1)) return false;
          mma_d<D>(TP, dv, dg + off(n % NS), id_s);
          umma_commit(dp_full);
          return true;
        };
        ok = ok && s_mma(0) && wait(kv_full + 1, 0) && dp_mma(0);
        for (int n = 0; ok && n < N; ++n) {
          const int st = n % NS;
          if (n + 1 < N) {
            if (!(ok = wait(s_read, n & 1))) break;
            tc_fence_after();
            if (!(ok = s_mma(n + 1))) break;
          }
          if (!(ok = wait(p_full, n & 1))) break;
          tc_fence_after();
          mma_t(TV, TP, mg_ + off(st), id_o, n > 0);
          umma_commit(g_empty + st);
          if (!(ok = wait(ds_full, n & 1))) break;
          tc_fence_after();
          mma_t(TK, TP + 32, mq_ + off(st), id_o, n > 0);
          umma_commit(n + 1 < N ? q_empty + st : done);
          if (n + 1 < N) ok = dp_mma(n + 1);
        }
      }
    } else if (warp == 10) {  // --------------------------------------- row sums
      // everything else may start before the row sums are there; k_swa_dq, which reads them
      // too, after this
      wait_for_previous();
      let_next_start();
      int g = it0 / max(nq, 1), qt = it0 % max(nq, 1);
      for (int n = 0; n < N; ++n) {
        const int st = n % NR, h = hk * a.G + g, i0 = (first + qt) * TILE;
        const float *nl = a.nlse + ((size_t)b * a.H + h) * a.T + i0, *de = a.delta + (nl - a.nlse);
        float x[4], y[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int i = 32 * c + lane;
          x[c] = i0 + i < len ? nl[i] : INFINITY;
          y[c] = i0 + i < len ? de[i] : 0.f;
        }
        if (n >= NR) wait.warp(l_empty + st, (n / NR - 1) & 1);
        float *d = srow + st * 2 * TILE;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          d[32 * c + lane] = x[c];
          d[TILE + 32 * c + lane] = y[c];
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(l_full + st);
        if (++qt == nq) { qt = 0; ++g; }
      }
    } else if (warp == 11 && len < a.T) {  // ------ a ragged last tile's Q and dO
      int qt = it0 % max(nq, 1);
      for (int n = 0; n < N; ++n) {
        const int st = n % NS, par = (n / NS) & 1, i0 = (first + qt) * TILE;
        wait.warp(q_full + st, par);
        wait.warp(g_full + st, par);
        if (i0 + TILE > len) {
          zero_rows(sq + st * TB, SL, len - i0, lane);
          zero_rows(sg + st * TB, SL, len - i0, lane);
          fence_proxy_async();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(clean + st);
        if (++qt == nq) qt = 0;
      }
    }
  } else {  // ----------------------------------------------------------- pointwise
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    const int wg = warp >> 2, r = tid & 127, j = j0 + r, q0 = 64 * wg;
    const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
    const uint32_t ts = TS + lanes + q0, tp = TP + lanes + q0;
    const float c2 = a.scale * kLog2e;
    const float2 cc = make_float2(c2, c2);
    int qt = it0 % max(nq, 1);
    for (int n = 0; n < N; ++n) {
      const int st = n % NR, i0 = (first + qt) * TILE;
      if (++qt == nq) qt = 0;
      const float *nl = srow + st * 2 * TILE + q0, *de = nl + TILE;
      wait.warp(l_full + st, (n / NR) & 1);
      wait.warp(s_full, n & 1);
      tc_fence_after();
      float p[64];
      tmem_ld32(ts, p);
      tmem_ld32(ts + 32, p + 32);
      tmem_ld_wait<64>(p);
      tc_fence_before();
      mbar_arrive(s_read);
#pragma unroll
      for (int c = 0; c < 64; c += 4) {
        const float4 l4 = *reinterpret_cast<const float4 *>(nl + c);
        const float2 y = fma2(make_float2(p[c], p[c + 1]), cc, make_float2(-l4.x, -l4.y));
        const float2 z = fma2(make_float2(p[c + 2], p[c + 3]), cc, make_float2(-l4.z, -l4.w));
        p[c] = ex2(y.x);
        p[c + 1] = ex2(y.y);
        p[c + 2] = ex2(z.x);
        p[c + 3] = ex2(z.y);
      }
      if (i0 == j0 || j0 + a.W <= i0 + TILE - 1) {  // some key is not seen by some query
#pragma unroll
        for (int c = 0; c < 64; c += 32) {
          const int d = j - i0 - q0 - c;  // the first of the 32 queries that is not before the key
          const uint32_t see = ~low_bits(d) & (j < a.ns ? ~0u : low_bits(d + a.W));
#pragma unroll
          for (int e = 0; e < 32; ++e) p[c + e] = (see >> e & 1u) ? p[c + e] : 0.f;
        }
      }
      uint32_t u[32];
      pack64(u, p);
      wait.warp(dp_full, n & 1);
      tc_fence_after();
      float g[64];
      tmem_ld32(tp, g);
      tmem_ld32(tp + 32, g + 32);
      tmem_ld_wait<64>(g);
      store32(tp, u);  // P^T and dS^T take the place of this thread's part of dP^T
      tmem_st_wait();
      tc_fence_before();
      mbar_arrive(p_full);
#pragma unroll
      for (int c = 0; c < 64; c += 4) {
        const float4 d4 = *reinterpret_cast<const float4 *>(de + c);
        const float2 y = mul2(make_float2(p[c], p[c + 1]),
                              add2(make_float2(g[c], g[c + 1]), make_float2(-d4.x, -d4.y)));
        const float2 z = mul2(make_float2(p[c + 2], p[c + 3]),
                              add2(make_float2(g[c + 2], g[c + 3]), make_float2(-d4.z, -d4.w)));
        g[c] = y.x;
        g[c + 1] = y.y;
        g[c + 2] = z.x;
        g[c + 3] = z.y;
      }
      pack64(u, g);
      store32(tp + 32, u);
      tmem_st_wait();
      tc_fence_before();
      mbar_arrive(ds_full);
      mbar_arrive(l_empty + st);
    }
    if (N > 0) wait.warp(done, 0);
    tc_fence_after();
    // threads of the first half store dV, those of the second dK
    const bool part = x < sp.part_blocks;
    const uint32_t acc = (wg ? TK : TV) + lanes;
    unsigned char *so = wg ? sk : sv;
    const int rows = part ? swa_split_rows(t, split, per, TILE, a.W, a.ns, a.G, len) : TILE;
    if (part && 32 * (warp & 3) < rows) {
      float *dst = a.part + (((size_t)b * a.Hk + hk) * sp.part_blocks + x) * (2 * TILE * a.d) +
                   (wg ? 0 : TILE * a.d) + (size_t)r * a.d;
#pragma unroll 1
      for (int c = 0; c < a.d; c += 32) {
        float o[32];
        tmem_ld32(acc + c, o);  // rows > 0: the split has iterations
        tmem_ld_wait<32>(o);
        if (r < rows)
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            *reinterpret_cast<float4 *>(dst + c + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
      }
    } else if (!part) {
      acc_to_tile<D>(acc, so, r, 0, wg ? a.scale : 1.f, j < len && N > 0, N > 0);
      fence_proxy_async();
    }
    named_sync(1 + wg, TILE);
    if (r == 0 && !part) {  // rows past T are not written
      for (int s = 0; s < SL; ++s) tma_store_4d(wg ? &mdk : &mdv, so + s * SLAB, 64 * s, hk, j0, b);
      bulk_commit();
      bulk_wait_read();
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tb, 512);
}

// ------------------------------------------------------------------ dQ

constexpr int DQ_K = 3, DQ_V = 2;  // stages of K and of V
template <int D> constexpr int DQ_SMEM = (2 + DQ_K + DQ_V) * TILE_BYTES<D> + 256 + 1024;

template <int D>
__global__ void __launch_bounds__(THREADS, 1)
    k_swa_dq(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
             const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mg,
             const __grid_constant__ CUtensorMap mdq, const SwaArgs a) {
  constexpr int NK = DQ_K, NV = DQ_V, TB = TILE_BYTES<D>, SL = D / 64;
  extern __shared__ unsigned char smraw[];
  unsigned char *sm =
      reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smraw) + 1023) & ~uintptr_t(1023));
  unsigned char *sq = sm, *sg = sq + TB, *sk = sg + TB, *sv = sk + NK * TB;
  uint64_t *bars = reinterpret_cast<uint64_t *>(sv + NV * TB);
  uint64_t *k_full = bars, *k_empty = k_full + NK, *v_full = k_empty + NK, *v_empty = v_full + NV;
  uint64_t *s_full = v_empty + NV, *q_full = s_full + 2, *g_full = q_full + 1, *dp_full = g_full + 1, *dp_read = dp_full + 1;
  uint64_t *ds_full = dp_read + 1, *clean = ds_full + 2, *done = clean + 1;
  uint32_t *s_tmem = reinterpret_cast<uint32_t *>(done + 1);
  int *s_fail = reinterpret_cast<int *>(s_tmem + 1);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = blockIdx.z, h = blockIdx.y, hk = h / a.G;
  // the last queries see the most keys: their CTAs start first
  const int i0 = (int)(gridDim.x - 1 - blockIdx.x) * TILE;
  const int len = swa_len(a, b);
  const SwaKeyTiles kt(i0, max(min(i0 + TILE, len), i0 + 1), a.W, a.ns, TILE);
  const int N = i0 < len ? kt.count : 0;

  // the loading thread: the first stages are on their way before the CTA meets
  int loads = 0;
  auto load_k_tile = [&](int n) {
    const int st = n % NK;
    mbar_expect_tx(k_full + st, TB);
    for (int s = 0; s < SL; ++s)
      tma_load_4d(sk + st * TB + s * SLAB, &mk, k_full + st, 64 * s, hk, kt.at(n) * TILE, b);
  };
  auto load_v_tile = [&](int n) {
    const int st = n % NV;
    mbar_expect_tx(v_full + st, TB);
    for (int s = 0; s < SL; ++s)
      tma_load_4d(sv + st * TB + s * SLAB, &mv, v_full + st, 64 * s, hk, kt.at(n) * TILE, b);
  };
  if (tid == SOFT) {
    for (int i = 0; i < NK; ++i) {
      mbar_init(k_full + i, 1);
      mbar_init(k_empty + i, 1);
    }
    for (int i = 0; i < NV; ++i) {
      mbar_init(v_full + i, 1);
      mbar_init(v_empty + i, 1);
    }
    mbar_init(s_full, 1);
    mbar_init(s_full + 1, 1);
    mbar_init(q_full, 1);
    mbar_init(g_full, 1);
    mbar_init(dp_full, 1);
    mbar_init(dp_read, SOFT);
    mbar_init(ds_full, SOFT);
    mbar_init(ds_full + 1, SOFT);
    mbar_init(clean, 1);
    mbar_init(done, 1);
    *s_fail = 0;
    fence_mbar_init();
    fence_proxy_async();
    if (N > 0) {
      mbar_expect_tx(q_full, TB);
      for (int s = 0; s < SL; ++s) tma_load_4d(sq + s * SLAB, &mq, q_full, 64 * s, h, i0, b);
      load_k_tile(0);
      mbar_expect_tx(g_full, TB);
      for (int s = 0; s < SL; ++s) tma_load_4d(sg + s * SLAB, &mg, g_full, 64 * s, h, i0, b);
      load_v_tile(0);
      for (loads = 1; loads < min(NV, N); ++loads) {
        load_k_tile(loads);
        load_v_tile(loads);
      }
    }
  }
  if (warp == 0) {
    tmem_alloc(s_tmem, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tb = *s_tmem, TP = tb + 256, TQ = tb + 384;
  const Waiter wait{s_fail, a.status};
  const bool ragged = len < a.T && N > 0 && kt.at(N - 1) * TILE + TILE > len;

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 8 && N > 0) {
      if (lane == 0) {  // ------------------------------------------------ loads
        int kl = loads, vl = loads;
        for (int n = loads; n < N; ++n) {
          if (n >= NK && !wait.lazy(k_empty + n % NK, (n / NK - 1) & 1)) break;
          load_k_tile(n);
          ++kl;
          if (n >= NV && !wait.lazy(v_empty + n % NV, (n / NV - 1) & 1)) break;
          load_v_tile(n);
          ++vl;
        }
        if (*wait.fail) {  // copies in flight land before the CTA leaves
          mbar_wait(q_full, 0, kWait >> 6);
          mbar_wait(g_full, 0, kWait >> 6);
          for (int m = max(0, kl - NK); m < kl; ++m) mbar_wait(k_full + m % NK, (m / NK) & 1, kWait >> 6);
          for (int m = max(0, vl - NV); m < vl; ++m) mbar_wait(v_full + m % NV, (m / NV) & 1, kWait >> 6);
        }
      }
      __syncwarp();
      if (ragged) {  // the last tile's keys past the length
        const int m = N - 1;
        wait.warp(k_full + m % NK, (m / NK) & 1);
        wait.warp(v_full + m % NV, (m / NV) & 1);
        zero_rows(sk + m % NK * TB, SL, len % TILE, lane);
        zero_rows(sv + m % NV * TB, SL, len % TILE, lane);
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(clean);
      }
    } else if (warp == 9 && N > 0) {  // ---------------------------------- products
      if (elect_one()) {
        const uint32_t id_s = idesc_bf16(TILE, TILE, 0, 0), id_o = idesc_bf16(TILE, D, 0, 1);
        const uint64_t dq = desc_k(sq), dg = desc_k(sg), dk = desc_k(sk), dv = desc_k(sv), mk_ = desc_mn(sk);
        auto off = [](int st) { return (uint64_t)(st * (TB >> 4)); };
        bool ok = wait(q_full, 0);
        auto s_mma = [&](int n) {
          if (!wait(k_full + n % NK, (n / NK) & 1)) return false;
          if (ragged && n == N - 1 && !wait(clean, 0)) return false;
          mma_d<D>(tb + (n & 1) * 128, dq, dk + off(n % NK), id_s);
          umma_commit(s_full + (n & 1));
          return true;
        };
        auto dp_mma = [&](int n) {
          if (!wait(v_full + n % NV, (n / NV) & 1)) return false;
          mma_d<D>(TP, dg, dv + off(n % NV), id_s);
          umma_commit(dp_full);
          umma_commit(v_empty + n % NV);
          return true;
        };
        ok = ok && s_mma(0) && wait(g_full, 0) && dp_mma(0);
        for (int n = 0; ok && n < N; ++n) {
          if (n + 1 < N) {
            if (!(ok = s_mma(n + 1))) break;
            if (!(ok = wait(dp_read, n & 1))) break;
            tc_fence_after();
            if (!(ok = dp_mma(n + 1))) break;
          }
          if (!(ok = wait(ds_full + (n & 1), (n >> 1) & 1))) break;
          tc_fence_after();
          mma_t(TQ, tb + (n & 1) * 128, mk_ + off(n % NK), id_o, n > 0);
          umma_commit(n + 1 < N ? k_empty + n % NK : done);
        }
      }
    }
  } else {  // ----------------------------------------------------------- pointwise
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    const int wg = warp >> 2, r = tid & 127, i = i0 + r, k0 = 64 * wg;
    const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
    const uint32_t tp = TP + lanes + k0;
    const float c2 = a.scale * kLog2e;
    const size_t row = ((size_t)b * a.H + h) * a.T + i;
    const float nl = i < len ? -__ldcg(a.nlse + row) : -INFINITY, de = i < len ? -__ldcg(a.delta + row) : 0.f;
    const float2 cc = make_float2(c2, c2), nn = make_float2(nl, nl), dd = make_float2(de, de);
    for (int n = 0; n < N; ++n) {
      const int j0 = kt.at(n) * TILE;
      const uint32_t ts = tb + (n & 1) * 128 + lanes + k0;
      wait.warp(s_full + (n & 1), (n >> 1) & 1);
      tc_fence_after();
      float p[64];
      tmem_ld32(ts, p);
      tmem_ld32(ts + 32, p + 32);
      tmem_ld_wait<64>(p);
#pragma unroll
      for (int c = 0; c < 64; c += 2) {
        const float2 y = fma2(make_float2(p[c], p[c + 1]), cc, nn);
        p[c] = ex2(y.x);
        p[c + 1] = ex2(y.y);
      }
      if (n == N - 1 || j0 + a.W <= i0 + TILE - 1) {  // some query does not see some key
#pragma unroll
        for (int c = 0; c < 64; c += 32) {
          const uint32_t see = key_bits(i - j0 - k0 - c, a.W, a.ns - j0 - k0 - c);
#pragma unroll
          for (int e = 0; e < 32; ++e) p[c + e] = (see >> e & 1u) ? p[c + e] : 0.f;
        }
      }
      wait.warp(dp_full, n & 1);
      tc_fence_after();
      float g[64];
      tmem_ld32(tp, g);
      tmem_ld32(tp + 32, g + 32);
      tmem_ld_wait<64>(g);
      tc_fence_before();
      mbar_arrive(dp_read);
#pragma unroll
      for (int c = 0; c < 64; c += 2) {
        const float2 y = mul2(make_float2(p[c], p[c + 1]), add2(make_float2(g[c], g[c + 1]), dd));
        g[c] = y.x;
        g[c + 1] = y.y;
      }
      uint32_t u[32];
      pack64(u, g);
      store32(ts, u);
      tmem_st_wait();
      tc_fence_before();
      // Two barriers in turn: dP of tile n + 1 does not wait for dS of tile n, so threads of one
      // half may come here with it before the other half's have with n.  (Nobody comes with
      // n + 2 so early: its dP is issued behind the wait for dS of n.)
      mbar_arrive(ds_full + (n & 1));
    }
    if (N > 0) wait.warp(done, 0);
    tc_fence_after();
    // two threads a query, half of the channels each, through the queries' place in shared memory
    acc_to_tile<D / 2>(TQ + lanes, sq, r, wg * (D / 2), a.scale, i < len, N > 0);
    fence_proxy_async();
    named_sync(1, SOFT);
    if (tid == 0) {  // rows past T are not written
      for (int s = 0; s < SL; ++s) tma_store_4d(&mdq, sq + s * SLAB, 64 * s, h, i0, b);
      bulk_commit();
      bulk_wait_read();
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tb, 512);
  __syncwarp();
  end_after_previous();
}

template <int D> kdn_status_t launch(const SwaArgs &a, const SwaSplits &sp, cudaStream_t s) {
  CUtensorMap mq, mk, mv, mg, mdq, mdk, mdv;
  if (!token_map(&mq, a.q, a.B, a.T, a.H, a.d) || !token_map(&mk, a.k, a.B, a.T, a.Hk, a.d) ||
      !token_map(&mv, a.v, a.B, a.T, a.Hk, a.d) || !token_map(&mg, a.dO, a.B, a.T, a.H, a.d) ||
      !token_map(&mdq, a.dq, a.B, a.T, a.H, a.d) || !token_map(&mdk, a.dk, a.B, a.T, a.Hk, a.d) ||
      !token_map(&mdv, a.dv, a.B, a.T, a.Hk, a.d))
    return KDN_ERR_CUDA;
  if (cudaFuncSetAttribute(k_swa_dkv<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, KV_SMEM<D>) != cudaSuccess ||
      cudaFuncSetAttribute(k_swa_dq<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, DQ_SMEM<D>) != cudaSuccess)
    return KDN_ERR_CUDA;
  const kdn_status_t st = launch_beside(k_swa_dkv<D>, dim3(sp.blocks, a.Hk, a.B), THREADS, KV_SMEM<D>, s, mq, mk, mv,
                                        mg, mdk, mdv, a, sp);
  if (st != KDN_OK) return st;
  return launch_beside(k_swa_dq<D>, dim3((a.T + TILE - 1) / TILE, a.H, a.B), THREADS, DQ_SMEM<D>, s, mq, mk, mv, mg,
                       mdq, a);
}

}  // namespace

kdn_status_t launch_swa_bwd_tc(const SwaArgs &a, const SwaSplits &sp, cudaStream_t s) {
  return a.d == 128 ? launch<128>(a, sp, s) : launch<64>(a, sp, s);
}

}  // namespace kdn
