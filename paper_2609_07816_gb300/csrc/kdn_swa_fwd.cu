// kdn_swa_fwd.cu -- sliding-window attention with sinks, forward, on the tensor cores
// (bfloat16; d = 32 runs as 64 with the upper half of every row loaded as zeros).
//
// A work item is 256 queries of one head, as two accumulators A and B of 128.  It goes once
// over the keys they see, 128 at a time, with the running maximum and sum of a softmax:
//   S = Q K^T (TMEM), P = exp2(c S - m) (registers, back to TMEM as bf16), O += P V (TMEM).
// Roles: warps 0-3 and 4-7 the softmax of A and of B (a thread a query), warp 8 the TMA
// loads, one thread of warp 9 the products.  While one accumulator's softmax runs, the
// tensor cores work on the other's products.  P takes the place of S: the next S of the
// same accumulator is issued behind the product that reads P.
//
// CTAs are persistent, one an SM, and the roles run ahead of one another across items: an
// item's first loads and products are under way while the one before it is written out.
// (With a CTA an item, start and end cost 10 us of an item's 29 at window 2048.)
//
// The running maximum is only followed when it grows by more than 2^8 (O and l are then
// rescaled, by the softmax threads: S being complete says that every earlier product into
// O is); until then P is at most 2^8 and the sums keep float32's relative precision.
#include "kdn_swa_tc.cuh"

namespace kdn {

bool swa_tc_supported(const SwaArgs &a) { return a.dtype == KDN_BF16; }

namespace {

using namespace swa;

constexpr int THREADS = 384;
template <int D> constexpr int STAGES = D == 128 ? 2 : 4;
template <int D> constexpr int TILE_BYTES = D / 64 * SLAB;
template <int D> constexpr int SMEM = (2 + 2 * STAGES<D>) * TILE_BYTES<D> + 1024 + 512;

struct Half {  // the key tiles that one accumulator's live queries see
  int first, last, ns;
  __device__ __forceinline__ Half(int i0, int len, int W, int sinks) : ns(sinks) {
    first = max(0, i0 - W + 1) / TILE;
    last = i0 < len ? i0 / TILE : -1;
  }
  __device__ __forceinline__ bool needs(int t) const { return t <= last && (t >= first || t * TILE < ns); }
};

struct Shape {  // of the work: items, 256-query blocks of a head
  int items, blocks;
  FastDiv by_blocks, by_heads, by_group;
};

// One work item: 256 queries of a head.
struct Item {
  int b, h, hk, i0, len, N;
  Half half[2];
  SwaKeyTiles kt;
  bool ragged;  // the last tile holds keys past the length
  __device__ __forceinline__ Item(const SwaArgs &a, const Shape &S, int item, int bh)
      : b(S.by_heads.div(bh)), h(bh - b * a.H), hk(S.by_group.div(h)),
        i0((S.blocks - 1 - (item - bh * S.blocks)) * 2 * TILE), len(swa_len(a, b)),
        half{Half(i0, len, a.W, a.ns), Half(i0 + TILE, len, a.W, a.ns)},
        kt(i0, max(min(i0 + 2 * TILE, len), i0 + 1), a.W, a.ns, TILE) {
    N = i0 < len ? kt.count : 0;
    ragged = N > 0 && len < a.T && kt.at(N - 1) * TILE + TILE > len;
  }
  __device__ __forceinline__ Item(const SwaArgs &a, const Shape &S, int item)
      : Item(a, S, item, S.by_blocks.div(item)) {}
  // whether tile number n of the list is the first that accumulator x needs: the list's
  // first, or for B, which may see less far back, the second
  __device__ __forceinline__ bool first(int x, int n) const {
    return n == 0 || (x == 1 && n == 1 && !half[1].needs(kt.at(0)));
  }
};

// What a tile is to the products, from the loading to the issuing thread: bits of A, those
// of B eight higher, and of the tile itself.
constexpr uint32_t kNeeds = 1, kFirst = 2, kLast = 4, kFrees = 8;  // (kFrees: set by the issuing thread)
constexpr uint32_t kRagged = 1u << 16, kEnd = 1u << 17;

// The status word and the counter of work items.
__global__ void k_swa_clear(unsigned *status) {
  let_next_start();
  if (threadIdx.x < 2) status[threadIdx.x] = 0;
}

template <int D>
__global__ void __launch_bounds__(THREADS, 1)
    k_swa_fwd_tc(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                 const __grid_constant__ CUtensorMap mv, const SwaArgs a, const Shape S) {
  constexpr int NS = STAGES<D>, TB = TILE_BYTES<D>, SL = D / 64;
  extern __shared__ unsigned char smraw[];
  unsigned char *sm =
      reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smraw) + 1023) & ~uintptr_t(1023));
  unsigned char *sq = sm, *sk = sm + 2 * TB, *sv = sk + NS * TB;
  uint64_t *bars = reinterpret_cast<uint64_t *>(sv + NS * TB);
  uint64_t *k_full = bars, *k_empty = k_full + NS, *v_full = k_empty + NS, *v_empty = v_full + NS;
  uint64_t *s_full = v_empty + NS, *p_full = s_full + 2, *o_full = p_full + 2, *q_full = o_full + 2;
  uint64_t *q_empty = q_full + 2, *v_clean = q_empty + 2;
  uint32_t *s_tmem = reinterpret_cast<uint32_t *>(v_clean + NS + 2 * kRing);
  int *s_fail = reinterpret_cast<int *>(s_tmem + 1);
  volatile uint32_t *s_info = s_tmem + 2;  // [stage] what K's tile is to the products
  const ItemRing ring{v_clean + NS, v_clean + NS + kRing, reinterpret_cast<int *>(s_tmem + 2 + NS)};

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < NS; ++i) {
      mbar_init(k_full + i, 1);
      mbar_init(v_full + i, 1);
      mbar_init(k_empty + i, 1);
      mbar_init(v_empty + i, 1);
      mbar_init(v_clean + i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + i, 1);
      mbar_init(p_full + i, TILE);
      mbar_init(o_full + i, 1);
      mbar_init(q_full + i, 1);
      mbar_init(q_empty + i, 1);
    }
    for (int i = 0; i < kRing; ++i) {
      mbar_init(ring.full + i, 1);
      mbar_init(ring.empty + i, 8);  // the softmax warps
    }
    *s_fail = 0;
    fence_mbar_init();
    prefetch_tmap(&mq);
    prefetch_tmap(&mk);
    prefetch_tmap(&mv);
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
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 8) {  // --------------------------------------------------- loads
      int kn = 0, vn = 0, qa = 0, qb = 0;  // loads issued (K and V: tiles, Q: items)
      bool ok = true;
      wait_for_previous();  // the counter is clear
      ItemSource work(ring, wait, a.status + 1, S.items);
      for (int item; (item = work.next()) >= 0;) {
        const Item I(a, S, item);
        if (I.N == 0) continue;
        if (lane == 0) {
          auto load_q = [&](int x, int &n) {
            if (n > 0 && !wait.lazy(q_empty + x, (n - 1) & 1)) return false;
            mbar_expect_tx(q_full + x, TB);
            for (int s = 0; s < SL; ++s)
              tma_load_4d(sq + x * TB + s * SLAB, &mq, q_full + x, 64 * s, I.h, I.i0 + x * TILE, I.b);
            ++n;
            return true;
          };
          ok = load_q(0, qa) && (I.half[1].last < 0 || load_q(1, qb));
          for (int n = 0; ok && n < I.N; ++n) {
            const int st = kn % NS, par = (kn / NS - 1) & 1, t = I.kt.at(n);
            if (kn >= NS && !(ok = wait.lazy(k_empty + st, par))) break;
            uint32_t f = I.ragged && n == I.N - 1 ? kRagged : 0u;
            for (int x = 0; x < 2; ++x)
              if (I.half[x].needs(t))
                f |= (kNeeds | (I.half[x].last == t ? kLast : 0u) | (I.first(x, n) ? kFirst : 0u)) << (8 * x);
            s_info[st] = f;
            mbar_expect_tx(k_full + st, TB);
            for (int s = 0; s < SL; ++s)
              tma_load_4d(sk + st * TB + s * SLAB, &mk, k_full + st, 64 * s, I.hk, t * TILE, I.b);
            ++kn;
            if (vn >= NS && !(ok = wait.lazy(v_empty + st, par))) break;
            mbar_expect_tx(v_full + st, TB);
            for (int s = 0; s < SL; ++s)
              tma_load_4d(sv + st * TB + s * SLAB, &mv, v_full + st, 64 * s, I.hk, t * TILE, I.b);
            ++vn;
          }
        }
        __syncwarp();
        if (I.ragged) {  // the last tile's V past the length
          const int m = __shfl_sync(0xffffffffu, vn, 0) - 1, st = max(m, 0) % NS;
          if (m >= 0) wait.warp(v_full + st, (m / NS) & 1);
          if (m >= 0) zero_rows(sv + st * TB, SL, I.len % TILE, lane);
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) mbar_arrive(v_clean + st);
        }
      }
      if (lane == 0) {
        if (ok && (kn < NS || wait(k_empty + kn % NS, (kn / NS - 1) & 1))) {  // no more tiles
          s_info[kn % NS] = kEnd;
          mbar_arrive(k_full + kn % NS);
        } else {  // copies in flight land before the CTA leaves
          if (qa > 0) mbar_wait(q_full, (qa - 1) & 1, kWait >> 6);
          if (qb > 0) mbar_wait(q_full + 1, (qb - 1) & 1, kWait >> 6);
          for (int m = max(0, kn - NS); m < kn; ++m) mbar_wait(k_full + m % NS, (m / NS) & 1, kWait >> 6);
          for (int m = max(0, vn - NS); m < vn; ++m) mbar_wait(v_full + m % NS, (m / NS) & 1, kWait >> 6);
        }
      }
    } else if (warp == 9) {  // ------------------------------------------ products
      if (elect_one()) {
        const uint32_t id_s = idesc_bf16(TILE, TILE, 0, 0), id_o = idesc_bf16(TILE, D, 0, 1);
        const uint64_t dq = desc_k(sq), dk = desc_k(sk), dv = desc_mn(sv);
        // of each accumulator: the tile whose P it is making (-1: none) and what that tile is
        // to it, its products P V and its items so far
        int pending[2] = {-1, -1}, np[2] = {0, 0}, nq[2] = {0, 0};
        uint32_t what[2] = {0, 0}, clean = 0;  // (clean: a stage's number of clearings, odd or even)
        auto pv = [&](int x) {  // O_x (+)= P_x V of its pending tile
          const int m = pending[x], st = m % NS;
          pending[x] = -1;
          if (!wait(v_full + st, (m / NS) & 1)) return false;
          if (what[x] & kRagged) {
            // of this stage: the loading warp may have cleared the tile of a later item too
            if (!wait(v_clean + st, clean >> st & 1)) return false;
            clean ^= 1u << st;
          }
          if (!wait(p_full + x, np[x]++ & 1)) return false;
          tc_fence_after();
          const uint64_t d = dv + st * (TB >> 4);
          const uint32_t acc = !(what[x] & kFirst);
#pragma unroll
          for (int kk = 0; kk < TILE / 16; ++kk)
            umma_ts(tb + 256 + x * 128, tb + x * 128 + kk * 8, d + step_mn(kk), id_o, kk ? 1u : acc);
          if (what[x] & kFrees) umma_commit(v_empty + st);
          if (what[x] & kLast) umma_commit(o_full + x);
          return true;
        };
        bool ok = true;
        for (int m = 0; ok; ++m) {
          const int st = m % NS;
          if (!mbar_try_wait(k_full + st, (m / NS) & 1)) {
            // The next tile may only come once the softmax warps have taken up later items,
            // which they do after this one's last products.
#pragma unroll
            for (int x = 0; x < 2; ++x)
              if (ok && pending[x] >= 0 && (what[x] & kLast)) ok = pv(x);
            if (!ok || !(ok = wait(k_full + st, (m / NS) & 1))) break;
          }
          const uint32_t info = s_info[st];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint32_t f = (info >> (8 * x) & 255u) | (info & kRagged);
            // (an item's last product into O does not wait for the accumulator's next tile)
            if (pending[x] >= 0 && ((f & kNeeds) || (what[x] & kLast)) && !(ok = pv(x))) break;
            if (!(f & kNeeds)) continue;
            if ((f & kFirst) && !(ok = wait(q_full + x, nq[x]++ & 1))) break;
            const uint64_t d = dk + st * (TB >> 4), e = dq + x * (TB >> 4);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
              umma_bf16(tb + x * 128, e + step_k(kk), d + step_k(kk), id_s, kk > 0);
            umma_commit(s_full + x);
            const bool alone = x == 0 && !(info >> 8 & kNeeds);
            if (x == 1 || alone) umma_commit(k_empty + st);
            if (f & kLast) umma_commit(q_empty + x);
            pending[x] = m;
            what[x] = f | (x == 1 || alone ? kFrees : 0u);  // A comes to a tile's V before B does
          }
          if (info & kEnd) break;
        }
      }
    }
  } else {  // ------------------------------------------------------------- softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    const int x = warp >> 2, r = tid & 127;
    const uint32_t ts = tb + x * 128 + ((uint32_t)(32 * (warp & 3)) << 16), to = ts + 256;
    const float c2 = a.scale * kLog2e;
    const bool wide = aligned32(a.o);
    int k = 0, done = 0;  // tiles and items of this accumulator so far
    ItemSink work(ring, wait);
    for (int item; (item = work.next()) >= 0;) {
      const Item I(a, S, item);
      const Half hx = x ? I.half[1] : I.half[0];
      const int r0 = I.i0 + x * TILE, i = r0 + r;
      if (r0 >= a.T) continue;
      float ref = -INFINITY, l = 0.f;
      for (int n = 0; n < I.N; ++n) {
        const int t = I.kt.at(n), j0 = t * TILE;
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
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(p_full + x);
        l = (ls[0].x + ls[0].y) + (ls[1].x + ls[1].y);
        ++k;
      }
      const bool live = i < I.len;
      if (a.lse && i < a.T)
        a.lse[((size_t)I.b * a.H + I.h) * a.T + i] = live ? (ref + log2f(l)) * kLn2 : -INFINITY;
      const float inv = live ? 1.f / l : 0.f;
      __nv_bfloat16 *dst = static_cast<__nv_bfloat16 *>(a.o) + (((size_t)I.b * a.T + i) * a.H + I.h) * a.d;
      const bool any = hx.last >= 0;  // the accumulator has been written
      if (any) {
        wait.warp(o_full + x, done & 1);
        tc_fence_after();
        ++done;
      }
#pragma unroll 1
      for (int c = 0; c < D; c += 32) {
        float o[32];
        if (any) {
          tmem_ld32(to + c, o);
          tmem_ld_wait<32>(o);
        }
        if (i < a.T && (D == 128 || c < a.d)) store_row32(dst + c, o, inv, live, wide);
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tb, 512);
}

template <int D> kdn_status_t launch(const SwaArgs &a, cudaStream_t s) {
  CUtensorMap mq, mk, mv;
  if (!token_map(&mq, a.q, a.B, a.T, a.H, a.d) || !token_map(&mk, a.k, a.B, a.T, a.Hk, a.d) ||
      !token_map(&mv, a.v, a.B, a.T, a.Hk, a.d))
    return KDN_ERR_CUDA;
  if (cudaFuncSetAttribute(k_swa_fwd_tc<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM<D>) != cudaSuccess)
    return KDN_ERR_CUDA;
  const int blocks = (a.T + 2 * TILE - 1) / (2 * TILE);
  const Shape S{blocks * a.H * a.B, blocks, FastDiv(blocks), FastDiv(a.H), FastDiv(a.G)};
  k_swa_clear<<<1, 32, 0, s>>>(a.status);
  if (cudaGetLastError() != cudaSuccess) return KDN_ERR_CUDA;
  return launch_beside(k_swa_fwd_tc<D>, dim3(S.items < kCtas ? S.items : kCtas), THREADS, SMEM<D>, s, mq, mk, mv, a, S);
}

}  // namespace

kdn_status_t launch_swa_fwd_tc(const SwaArgs &a, cudaStream_t s) {
  return a.d == 128 ? launch<128>(a, s) : launch<64>(a, s);
}

}  // namespace kdn
