// kdn_swa_fwd.cu -- sliding-window attention with sinks, forward, on the tensor cores
// (bfloat16, d = 64 or 128).
//
// One CTA owns 256 queries of one head as two accumulators A and B of 128, and goes once
// over the keys they see, 128 at a time, with the running maximum and sum of a softmax:
//   S = Q K^T (TMEM), P = exp2(c S - m) (registers, back to TMEM as bf16), O += P V (TMEM).
// Roles: warps 0-3 and 4-7 the softmax of A and of B (a thread a query), warp 8 the TMA
// loads, warp 9 the products.  While one accumulator's softmax runs, the tensor cores work
// on the other's products.  P takes the place of S: the next S of the same accumulator is
// issued behind the product that reads P.
//
// The running maximum is only followed when it grows by more than 2^8 (O and l are then
// rescaled, by the softmax threads: S being complete says that every earlier product into
// O is); until then P is at most 2^8 and the sums keep float32's relative precision.
#include "kdn_swa_tc.cuh"

namespace kdn {

bool swa_tc_supported(const SwaArgs &a) { return a.dtype == KDN_BF16 && a.d >= 64; }

namespace {

using namespace swa;

constexpr int THREADS = 384;
template <int D> constexpr int STAGES = D == 128 ? 2 : 4;
template <int D> constexpr int TILE_BYTES = D / 64 * SLAB;
template <int D> constexpr int SMEM = (2 + 2 * STAGES<D>) * TILE_BYTES<D> + 1024 + 256;

struct Half {  // the key tiles that one accumulator's live queries see
  int first, last, ns;
  __device__ __forceinline__ Half(int i0, int len, int W, int sinks) : ns(sinks) {
    first = max(0, i0 - W + 1) / TILE;
    last = i0 < len ? i0 / TILE : -1;
  }
  __device__ __forceinline__ bool needs(int t) const { return t <= last && (t >= first || t * TILE < ns); }
};

template <int D>
__global__ void __launch_bounds__(THREADS, 1)
    k_swa_fwd_tc(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                 const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mo, const SwaArgs a) {
  constexpr int NS = STAGES<D>, TB = TILE_BYTES<D>, SL = D / 64;
  extern __shared__ unsigned char smraw[];
  unsigned char *sm =
      reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smraw) + 1023) & ~uintptr_t(1023));
  unsigned char *sq = sm, *sk = sm + 2 * TB, *sv = sk + NS * TB;
  uint64_t *bars = reinterpret_cast<uint64_t *>(sv + NS * TB);
  uint64_t *k_full = bars, *k_empty = k_full + NS, *v_full = k_empty + NS, *v_empty = v_full + NS;
  uint64_t *s_full = v_empty + NS, *p_full = s_full + 2, *o_full = p_full + 2, *q_full = o_full + 2, *v_clean = q_full + 1;
  uint32_t *s_tmem = reinterpret_cast<uint32_t *>(v_clean + 1);
  int *s_fail = reinterpret_cast<int *>(s_tmem + 1);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = blockIdx.z, h = blockIdx.y, hk = h / a.G;
  // the last queries see the most keys: their CTAs start first
  const int i0 = (int)(gridDim.x - 1 - blockIdx.x) * 2 * TILE;
  const int len = swa_len(a, b);
  const Half half[2] = {Half(i0, len, a.W, a.ns), Half(i0 + TILE, len, a.W, a.ns)};
  const SwaKeyTiles kt(i0, max(min(i0 + 2 * TILE, len), i0 + 1), a.W, a.ns, TILE);
  const int N = i0 < len ? kt.count : 0;

  if (tid == 0) {
    for (int i = 0; i < NS; ++i) {
      mbar_init(k_full + i, 1);
      mbar_init(v_full + i, 1);
      mbar_init(k_empty + i, 1);
      mbar_init(v_empty + i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + i, 1);
      mbar_init(p_full + i, TILE);
      mbar_init(o_full + i, 1);
    }
    mbar_init(q_full, 1);
    mbar_init(v_clean, 1);
    *s_fail = 0;
    fence_mbar_init();
    prefetch_tmap(&mq);
    prefetch_tmap(&mk);
    prefetch_tmap(&mv);
    prefetch_tmap(&mo);
  }
  if (warp == 0) {
    tmem_alloc(s_tmem, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tb = *s_tmem;
  const Waiter wait{s_fail, a.status};

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 8 && N > 0) {
      if (lane == 0) {  // ------------------------------------------------ loads
        mbar_expect_tx(q_full, (half[1].last >= 0 ? 2 : 1) * TB);
        for (int x = 0; x < 2; ++x)
          if (half[x].last >= 0)
            for (int s = 0; s < SL; ++s) tma_load_4d(sq + x * TB + s * SLAB, &mq, q_full, 64 * s, h, i0 + x * TILE, b);
        int n = 0;
        for (; n < N; ++n) {
          const int st = n % NS, par = (n / NS - 1) & 1, j0 = kt.at(n) * TILE;
          if (n >= NS && !wait(k_empty + st, par)) break;
          mbar_expect_tx(k_full + st, TB);
          for (int s = 0; s < SL; ++s) tma_load_4d(sk + st * TB + s * SLAB, &mk, k_full + st, 64 * s, hk, j0, b);
          if (n >= NS && !wait(v_empty + st, par)) break;
          mbar_expect_tx(v_full + st, TB);
          for (int s = 0; s < SL; ++s) tma_load_4d(sv + st * TB + s * SLAB, &mv, v_full + st, 64 * s, hk, j0, b);
        }
        if (*wait.fail) {  // copies in flight land before the CTA leaves
          mbar_wait(q_full, 0, kWait);
          for (int m = max(0, n - NS); m <= min(n, N - 1); ++m) mbar_wait(k_full + m % NS, (m / NS) & 1, kWait >> 6);
          for (int m = max(0, n - NS); m < n; ++m) mbar_wait(v_full + m % NS, (m / NS) & 1, kWait >> 6);
        }
      }
      __syncwarp();
      if (len < a.T && kt.at(N - 1) * TILE + TILE > len) {  // the last tile's V past the length
        const int st = (N - 1) % NS;
        wait.warp(v_full + st, ((N - 1) / NS) & 1);
        zero_rows(sv + st * TB, SL, len % TILE, lane);
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(v_clean);
      }
    } else if (warp == 9 && N > 0) {  // ---------------------------------- products
      if (elect_one()) {
        const uint32_t id_s = idesc_bf16(TILE, TILE, 0, 0), id_o = idesc_bf16(TILE, D, 0, 1);
        const uint64_t dq = desc_k(sq), dk = desc_k(sk), dv = desc_mn(sv);
        int pending[2] = {-1, -1}, done[2] = {0, 0};
        uint32_t used = 0;  // stages whose V one of two accumulators has used
        bool ok = wait(q_full, 0);
        // O_x += P_x V of tile number m of the list; the P is the accumulator's done[x]-th
        auto pv = [&](int x, int m) {
          const int st = m % NS, t = kt.at(m);
          // V is free when the last accumulator that needs it has used it
          const bool both = half[0].needs(t) && half[1].needs(t);
          const bool last_use = !both || (used >> st & 1);
          if (both) used ^= 1u << st;
          if (!wait(v_full + st, (m / NS) & 1)) return false;
          if (t * TILE + TILE > len && len < a.T && !wait(v_clean, 0)) return false;
          if (!wait(p_full + x, done[x] & 1)) return false;
          tc_fence_after();
          const uint64_t d = dv + st * (TB >> 4);
          const uint32_t acc = done[x] > 0;
#pragma unroll
          for (int kk = 0; kk < TILE / 16; ++kk)
            umma_ts(tb + 256 + x * 128, tb + x * 128 + kk * 8, d + step_mn(kk), id_o, kk ? 1u : acc);
          if (last_use) umma_commit(v_empty + st);
          ++done[x];
          return true;
        };
        for (int n = 0; ok && n < N; ++n) {
          const int st = n % NS, t = kt.at(n);
          if (!(ok = wait(k_full + st, (n / NS) & 1))) break;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            if (!half[x].needs(t)) continue;
            if (pending[x] >= 0 && !(ok = pv(x, pending[x]))) break;
            const uint64_t d = dk + st * (TB >> 4), e = dq + x * (TB >> 4);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
              umma_bf16(tb + x * 128, e + step_k(kk), d + step_k(kk), id_s, kk > 0);
            umma_commit(s_full + x);
            if (x == 1 || !half[1].needs(t)) umma_commit(k_empty + st);
            pending[x] = n;
          }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x)
          if (ok && pending[x] >= 0) {
            ok = pv(x, pending[x]);
            umma_commit(o_full + x);
          }
      }
    }
  } else {  // ------------------------------------------------------------- softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int x = warp >> 2, r = tid & 127, r0 = i0 + x * TILE, i = r0 + r;
    const uint32_t ts = tb + x * 128 + ((uint32_t)(32 * (warp & 3)) << 16), to = ts + 256;
    const float c2 = a.scale * kLog2e;
    const Half hx = x ? half[1] : half[0];
    float ref = -INFINITY, l = 0.f;
    int k = 0;
    for (int n = 0; n < N; ++n) {
      const int t = kt.at(n), j0 = t * TILE;
      if (!hx.needs(t)) continue;
      wait.warp(s_full + x, k & 1);
      tc_fence_after();
      float s[TILE];
#pragma unroll
      for (int c = 0; c < TILE; c += 32) tmem_ld32(ts + c, s + c);
      tmem_ld_wait<TILE>(s);
      if (t == hx.last || j0 + a.W <= r0 + TILE - 1) {  // some query does not see some key
#pragma unroll
        for (int c = 0; c < TILE; c += 32) {
          const uint32_t see = key_bits(i - j0 - c, a.W, a.ns - j0 - c);
#pragma unroll
          for (int e = 0; e < 32; ++e) s[c + e] = (see >> e & 1u) ? s[c + e] : -INFINITY;
        }
      }
      float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
      for (int c = 4; c < TILE; c += 4)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx[e] = fmaxf(mx[e], s[c + e]);
      const float m = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * c2;
      float f = 1.f;
      if (m > ref + 8.f) {  // also a row's first keys: O and l are still zero then
        f = ref == -INFINITY ? 1.f : ex2(ref - m);
        ref = m;
        l *= f;
      }
      if (__any_sync(0xffffffffu, f != 1.f)) {
        const float2 ff = make_float2(f, f);
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          float o[32];
          tmem_ld32(to + c, o);
          tmem_ld_wait<32>(o);
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float2 y = mul2(make_float2(o[e], o[e + 1]), ff);
            o[e] = y.x;
            o[e + 1] = y.y;
          }
          tmem_st32(to + c, o);
        }
      }
      const float nr = ref == -INFINITY ? 0.f : -ref;  // a row that has seen nothing yet
      const float2 cc = make_float2(c2, c2), nn = make_float2(nr, nr);
      float2 ls[2] = {make_float2(l, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
      for (int c = 0; c < TILE; c += 32) {
        uint32_t u[16];
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          float2 y = fma2(make_float2(s[c + e], s[c + e + 1]), cc, nn);
          y.x = ex2(y.x);
          y.y = ex2(y.y);
          ls[(e >> 1) & 1] = add2(ls[(e >> 1) & 1], y);
          u[e / 2] = pack_bf2(y.x, y.y);
        }
        tmem_st16u(ts + c / 2, u);
      }
      l = (ls[0].x + ls[0].y) + (ls[1].x + ls[1].y);
      tmem_st_wait();
      tc_fence_before();
      mbar_arrive(p_full + x);
      ++k;
    }
    if (k > 0) wait.warp(o_full + x, 0);
    // o through shared memory (this accumulator's queries are no longer needed there)
    unsigned char *so = sq + x * TB;
    if (r0 < a.T) {
      const bool live = i < len;
      const float inv = live ? 1.f / l : 0.f;
      tc_fence_after();
#pragma unroll 1
      for (int c = 0; c < D; c += 32) {
        float o[32];
        if (k > 0) {
          tmem_ld32(to + c, o);
          tmem_ld_wait<32>(o);
        }
#pragma unroll
        for (int e = 0; e < 32; e += 8) {
          uint32_t u[4];
#pragma unroll
          for (int p = 0; p < 4; ++p)
            u[p] = live ? pack_bf2(o[e + 2 * p] * inv, o[e + 2 * p + 1] * inv) : 0u;
          sm16(so + (c >> 6) * SLAB, chunk_off(r, ((c & 63) + e) >> 3)) = make_uint4(u[0], u[1], u[2], u[3]);
        }
      }
      if (a.lse && i < a.T)
        a.lse[((size_t)b * a.H + h) * a.T + i] = live ? (ref + log2f(l)) * kLn2 : -INFINITY;
      fence_proxy_async();
    }
    named_sync(1 + x, TILE);
    if (r == 0 && r0 < a.T) {  // rows past T are not written
      for (int s = 0; s < SL; ++s) tma_store_4d(&mo, so + s * SLAB, 64 * s, h, r0, b);
      bulk_commit();
      bulk_wait_all();
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tb, 512);
}

template <int D> kdn_status_t launch(const SwaArgs &a, cudaStream_t s) {
  CUtensorMap mq, mk, mv, mo;
  if (!token_map(&mq, a.q, a.B, a.T, a.H, D) || !token_map(&mk, a.k, a.B, a.T, a.Hk, D) ||
      !token_map(&mv, a.v, a.B, a.T, a.Hk, D) || !token_map(&mo, a.o, a.B, a.T, a.H, D))
    return KDN_ERR_CUDA;
  if (cudaFuncSetAttribute(k_swa_fwd_tc<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM<D>) != cudaSuccess)
    return KDN_ERR_CUDA;
  k_swa_fwd_tc<D><<<dim3((a.T + 2 * TILE - 1) / (2 * TILE), a.H, a.B), THREADS, SMEM<D>, s>>>(mq, mk, mv, mo, a);
  return cudaGetLastError() == cudaSuccess ? KDN_OK : KDN_ERR_CUDA;
}

}  // namespace

kdn_status_t launch_swa_fwd_tc(const SwaArgs &a, cudaStream_t s) {
  return a.d == 128 ? launch<128>(a, s) : launch<64>(a, s);
}

}  // namespace kdn
