// kdn_ffn_f32.cu -- the gated feed-forward block in float32, on the tensor cores.
//
// A float32 is the sum of three bfloat16s, x = x0 + x1 + x2 with |x1| <= 2^-9 |x| and |x2| <= 2^-18 |x|, exact to
// 2^-27, so a product of two is six products of bfloat16s,
//   x y = x0 y0 + (x0 y1 + x1 y0 + x1 y1 + x0 y2 + x2 y0),
// and what is left out is below 2^-26 of it.  Six times 1/16 of the bfloat16 time is a third of what the CUDA
// cores need.  Operands are cut into their three planes once, in the workspace (a kernel for what the call
// is given; the hidden axis' values in the epilogue that makes them).
//
// Sums.  The tensor cores truncate when they add into an accumulator, always towards 0: of positive terms 4e-6 of the
// sum over K = 2048, 1.6e-4 over 32768 (kdn_ffn_tc.cu).  So x0 y0 has an accumulator of its own, the
// five small products another, and after 128 along K (8 additions) both are added in float32, rounded to
// nearest, to sums in the epilogue's registers, while the products go on with a second pair of accumulators.
//
// Tiles of 256 x 128 by pairs of CTAs as in kdn_ffn_tc.cu: a step of 64 along K is 72 KB of planes a CTA and 24
// products, so that the operands' way into the SM (47 bytes a cycle) does not bound it.  The tensor cores do: 2048
// tokens of 1024 x 4096 take 66 us in y (pipe 84 % active), 138 in the gate (69 %, cutting what it makes into planes).
#include "kdn_ffn_tc.cuh"

namespace kdn {
namespace {

using namespace ffn;

constexpr int THREADS = 384, BN = 128, EPI_WARPS = 8, CHUNK = 2;  // steps between two additions
constexpr int A_PLANES = 3 * 128 * BK * 2, STAGE = A_PLANES + 3 * 64 * BK * 2, STAGES = 3;
constexpr int SMEM = STAGES * STAGE + 1024 + 512;

struct Work {
  CUtensorMap maps[6];  // of planes: A and B of each problem or sum (GATE: A, B of g, B of u)
  Problem p[3];
  int np, tiles;
  int am, bm;           // A and B are stored along their own axes
  int act;
  float *out[3];        // PLAIN: of each problem, or its partial sums; GATE: g, u (null: not written), h
  bf *planes[2];        // GATE: h; DGATE: dg, du
  const float *in[2];   // DGATE: g, u
  size_t plane;         // elements of a plane of those
  int wide, wide_planes;  // rows (of planes) start on 32 bytes
  unsigned *status;
};

struct Planes {
  bf v[3];
};
__device__ __forceinline__ Planes split(float x) {
  Planes p;
  p.v[0] = __float2bfloat16_rn(fminf(fmaxf(x, -3.3895313892515355e38f), 3.3895313892515355e38f));
  x -= __bfloat162float(p.v[0]);
  p.v[1] = __float2bfloat16_rn(x);
  p.v[2] = __float2bfloat16_rn(x - __bfloat162float(p.v[1]));
  return p;
}
// eight values to their places in the three planes
__device__ __forceinline__ void split8(const float *x, bf *to, size_t plane) {
  uint4 v[3];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const Planes p = split(x[i]);
#pragma unroll
    for (int j = 0; j < 3; ++j) reinterpret_cast<bf *>(v + j)[i] = p.v[j];
  }
#pragma unroll
  for (int j = 0; j < 3; ++j) *reinterpret_cast<uint4 *>(to + j * plane) = v[j];
}

struct Cuts {  // tensors that a call is given
  const float *from[6];
  bf *to[6];
  size_t n[6];  // elements, a multiple of 8
  unsigned *status;
};
__global__ void __launch_bounds__(256) k_ffn_split(const __grid_constant__ Cuts c) {
  let_next_start();
  wait_for_previous();
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *c.status = 0;
  const int t = blockIdx.y;
  for (size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 8; i < c.n[t]; i += (size_t)gridDim.x * 2048) {
    float x[8];
    *reinterpret_cast<float4 *>(x) = *reinterpret_cast<const float4 *>(c.from[t] + i);
    *reinterpret_cast<float4 *>(x + 4) = *reinterpret_cast<const float4 *>(c.from[t] + i + 4);
    split8(x, c.to[t] + i, c.n[t]);
  }
}

// 32 columns of a thread's own row, the first `n` of them (a multiple of 8), in whole sectors of 32 bytes where rows
// are aligned to them.  In dh a tile's end is bound by them: 196 KB a CTA in 8 us, 3.7 TB/s for all, what writes reach;
// exchanged between lanes into pieces of 128 bytes they take no less (gradients 470 and 476 us).  (There is no room
// to pass blocks through shared memory on their way to whole lines: with two stages in place of three the products
// wait, 241 us in place of 201 for the gradients of 4096 x 1024's weights.)
struct Row {
  int n;
  bool wide;
  __device__ __forceinline__ void store(float *p, const float *x) const {
#pragma unroll
    for (int c = 0; c < 32; c += 8) {
      if (c >= n) continue;
      if (wide) {
        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p + c), "f"(x[c]), "f"(x[c + 1]),
                     "f"(x[c + 2]), "f"(x[c + 3]), "f"(x[c + 4]), "f"(x[c + 5]), "f"(x[c + 6]), "f"(x[c + 7])
                     : "memory");
      } else {
        *reinterpret_cast<float4 *>(p + c) = *reinterpret_cast<const float4 *>(x + c);
        *reinterpret_cast<float4 *>(p + c + 4) = *reinterpret_cast<const float4 *>(x + c + 4);
      }
    }
  }
  __device__ __forceinline__ void load(const float *p, float *x) const {
#pragma unroll
    for (int c = 0; c < 32; c += 8) {
      if (c >= n) {
#pragma unroll
        for (int l = 0; l < 8; ++l) x[c + l] = 0.f;
      } else if (wide) {
        asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(x[c]), "=f"(x[c + 1]), "=f"(x[c + 2]), "=f"(x[c + 3]), "=f"(x[c + 4]), "=f"(x[c + 5]),
                       "=f"(x[c + 6]), "=f"(x[c + 7])
                     : "l"(p + c)
                     : "memory");
      } else {
        *reinterpret_cast<float4 *>(x + c) = *reinterpret_cast<const float4 *>(p + c);
        *reinterpret_cast<float4 *>(x + c + 4) = *reinterpret_cast<const float4 *>(p + c + 4);
      }
    }
  }
  __device__ __forceinline__ void store_planes(bf *to, size_t plane, const float *x, bool wide_planes) const {
#pragma unroll
    for (int c = 0; c < 32; c += 16) {
      uint4 v[3][2];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const Planes p = split(x[c + i]);
#pragma unroll
        for (int j = 0; j < 3; ++j) reinterpret_cast<bf *>(v[j])[i] = p.v[j];
      }
#pragma unroll
      for (int j = 0; j < 3; ++j) {
        bf *q = to + j * plane + c;
        if (wide_planes && c + 16 <= n) {
          asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(q), "r"(v[j][0].x), "r"(v[j][0].y),
                       "r"(v[j][0].z), "r"(v[j][0].w), "r"(v[j][1].x), "r"(v[j][1].y), "r"(v[j][1].z), "r"(v[j][1].w)
                       : "memory");
        } else {
          if (c < n) *reinterpret_cast<uint4 *>(q) = v[j][0];
          if (c + 8 < n) *reinterpret_cast<uint4 *>(q + 8) = v[j][1];
        }
      }
    }
  }
};
template <int ACT> __device__ __forceinline__ void gate32(float *g, const float *u) {
#pragma unroll
  for (int l = 0; l < 32; ++l) {
    float a, da;
    ffn_act_near<ACT>(g[l], &a, &da);
    g[l] = a * u[l];
  }
}
template <int ACT> __device__ __forceinline__ void gradients32(const float *dh, float *g, float *u) {
#pragma unroll
  for (int l = 0; l < 32; ++l) {
    float a, da;
    ffn_act_near<ACT>(g[l], &a, &da);
    g[l] = dh[l] * u[l] * da;
    u[l] = dh[l] * a;
  }
}

// a box of all three planes, into this CTA's shared memory, counted at a barrier of the pair
__device__ __forceinline__ void load_planes(void *dst, const CUtensorMap *map, uint32_t bar, int c0, int c1) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2"
      " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(0), "r"(bar)
      : "memory");
}

template <int EPI>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1) k_ffn_f32(const __grid_constant__ Work w) {
  extern __shared__ unsigned char smraw[];
  unsigned char *sm =
      reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smraw) + 1023) & ~uintptr_t(1023));
  uint64_t *full = reinterpret_cast<uint64_t *>(sm + STAGES * STAGE);
  uint64_t *empty = full + STAGES, *acc_full = empty + STAGES, *acc_empty = acc_full + 2;
  uint32_t *s_tmem = reinterpret_cast<uint32_t *>(acc_empty + 2);
  int *s_fail = reinterpret_cast<int *>(s_tmem + 1);
  constexpr int COLS = EPI == GATE ? BN / 2 : BN;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  if (tid == 0) {
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(full + i, 1);
      mbar_init(empty + i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(acc_full + i, 1);
      mbar_init(acc_empty + i, 2 * EPI_WARPS);
    }
    *s_fail = 0;
    fence_mbar_init();
  }
  if (warp == 2) tmem_alloc_pair(s_tmem, 512);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  let_next_start();
  const uint32_t tb = *s_tmem;
  const Waiter wait{s_fail, w.status};
  wait_for_previous();

  if (warp == 0) {  // ------------------------------------------------------- loads
    if (elect_one()) {
      int n = 0;  // steps so far
      bool ok = true;
      for (int t = pair; ok && t < w.tiles; t += pairs) {
        const Tile T = tile_at(w.p, w.np, COLS, t);
        for (int k = T.k0; k < T.k1; ++k, ++n) {
          const int st = n % STAGES, seg = k >= T.p->steps[0], kk = (k - (seg ? T.p->steps[0] : 0)) * BK;
          if (n >= STAGES && !(ok = wait(empty + st, (n / STAGES - 1) & 1))) break;
          unsigned char *sa = sm + st * STAGE;
          if (rank == 0) mbar_expect_tx(full + st, 2 * STAGE);
          const uint32_t bar = in_cta(full + st, 0);
          const CUtensorMap *ma = w.maps + T.p->a[seg], *mb = w.maps + T.p->b[EPI == GATE ? rank : seg];
          const int m = T.m + 128 * (int)rank, c = EPI == GATE ? T.n : T.n + 64 * (int)rank;
          if (w.am) {
            load_planes(sa, ma, bar, m, kk);
            load_planes(sa + A_PLANES / 2, ma, bar, m + 64, kk);
          } else {
            load_planes(sa, ma, bar, kk, m);
          }
          if (w.bm) load_planes(sa + A_PLANES, mb, bar, c, kk);
          else load_planes(sa + A_PLANES, mb, bar, kk, c);
        }
      }
      // what the pair still copies and signals arrives before its CTAs leave
      for (int m = max(0, n - STAGES); m < n; ++m) {
        if (!ok && rank == 0) mbar_wait(full + m % STAGES, (m / STAGES) & 1, kWait >> 6);
        if (ok) ok = wait.lazy(empty + m % STAGES, (m / STAGES) & 1);
      }
    }
  } else if (warp == 1) {  // ------------------------------------------------ products
    if (rank == 0 && elect_one()) {
      const uint32_t id = idesc_bf16(256, BN, w.am, w.bm), base = smem_u32(sm);
      const uint64_t da = sw128_desc(base, w.am ? A_PLANES / 2 : 16, 1024);
      const uint64_t db = sw128_desc(base + A_PLANES, 16, 1024);
      const uint64_t ka = (w.am ? 2048 : 32) >> 4, kb = (w.bm ? 2048 : 32) >> 4;
      const uint64_t pa = (w.am ? 8192 : 16384) >> 4, pb = 8192 >> 4;  // from plane to plane
      int n = 0, i = 0;  // steps and additions so far
      bool ok = true;
      for (int t = pair; ok && t < w.tiles; t += pairs) {
        const Tile T = tile_at(w.p, w.np, COLS, t);
        if (!(ok = wait(full + n % STAGES, (n / STAGES) & 1))) break;
        for (int k = T.k0; k < T.k1; ++k, ++n) {
          const int st = n % STAGES, at = (k - T.k0) % CHUNK;
          const uint32_t big = tb + (i & 1) * 256, small = big + BN;
          if (at == 0) {
            if (i >= 2 && !(ok = wait(acc_empty + (i & 1), (i / 2 - 1) & 1))) break;
            tc_fence_after();
          }
          const uint64_t a = da + st * (STAGE >> 4), b = db + st * (STAGE >> 4);
#pragma unroll
          for (int kk = 0; kk < BK / 16; ++kk) {
            const uint64_t x = a + kk * ka, y = b + kk * kb;
            const uint32_t more = at > 0 || kk > 0;
            umma_pair(small, x, y + pb, id, more);
            umma_pair(small, x + pa, y, id, 1);
            umma_pair(small, x + pa, y + pb, id, 1);
            umma_pair(small, x, y + 2 * pb, id, 1);
            umma_pair(small, x + 2 * pa, y, id, 1);
            // the next step's operands are waited for while this step's products still run
            if (kk == BK / 16 - 1 && k + 1 < T.k1) ok = wait(full + (n + 1) % STAGES, ((n + 1) / STAGES) & 1);
            umma_pair(big, x, y, id, more);
          }
          commit_pair(empty + st);
          if (at == CHUNK - 1 || k + 1 == T.k1) commit_pair(acc_full + (i++ & 1));
          if (!ok) break;
        }
      }
    }
  } else if (warp >= 4) {  // ------------------------------------------------ sums and epilogue
    const int q = warp & 3, half = (warp - 4) >> 2;
    const uint32_t lanes = (uint32_t)(32 * q) << 16;
    // this thread's 2 x 32 columns of the accumulator: of GATE 32 of g and the same of u
    const int first = EPI == GATE ? 32 * half : 64 * half, other = EPI == GATE ? 64 : 32;
    int i = 0;
    for (int t = pair; t < w.tiles; t += pairs) {
      const Tile T = tile_at(w.p, w.np, COLS, t);
      const int m = T.m + 128 * (int)rank + 32 * q + lane, M = T.p->M, N = T.p->N;
      if (EPI == DGATE && m < M) {  // g and u are on their way to L2 while the products run
        const int n = T.n + 64 * half;
#pragma unroll
        for (int c = 0; c < 64; c += 32)
          if (n + c < N)
            for (const float *in : {w.in[0], w.in[1]})
              asm volatile("prefetch.global.L2 [%0];" ::"l"(in + (size_t)m * N + n + c));
      }
      float x[64];
#pragma unroll
      for (int j = 0; j < 64; ++j) x[j] = 0.f;
      for (int k = T.k0; k < T.k1; k += CHUNK, ++i) {
        wait_quietly(wait, acc_full + (i & 1), (i / 2) & 1);
        tc_fence_after();
        const uint32_t ta = tb + (i & 1) * 256 + first + lanes;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float big[32], small[32];
          tmem_ld32(ta + h * other, big);
          tmem_ld32(ta + h * other + BN, small);
          tmem_ld_wait<32>(big);
          pin32(small);
#pragma unroll
          for (int j = 0; j < 32; ++j) x[32 * h + j] += big[j] + small[j];
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_at(in_cta(acc_empty + (i & 1), 0));
      }
#pragma unroll
      for (int h = 0; h < (EPI == GATE ? 1 : 2); ++h) {
        const int n = T.n + (EPI == GATE ? 32 : 64) * half + 32 * h;
        const Row R{m < M ? N - n : 0, w.wide != 0};
        const size_t at = (size_t)m * N + n;
        if (R.n <= 0) continue;
        if (EPI == PLAIN) {
          R.store(w.out[T.p - w.p] + (size_t)T.split * M * N + at, x + 32 * h);
        } else if (EPI == GATE) {
          if (w.out[0]) {
            R.store(w.out[0] + at, x);
            R.store(w.out[1] + at, x + 32);
          }
          if (w.act == KDN_ACT_SILU) gate32<KDN_ACT_SILU>(x, x + 32);
          else gate32<KDN_ACT_GELU>(x, x + 32);
          R.store(w.out[2] + at, x);
          R.store_planes(w.planes[0] + at, w.plane, x, w.wide_planes);
        } else {
          float g[32], u[32];
          R.load(w.in[0] + at, g);
          R.load(w.in[1] + at, u);
          if (w.act == KDN_ACT_SILU) gradients32<KDN_ACT_SILU>(x + 32 * h, g, u);
          else gradients32<KDN_ACT_GELU>(x + 32 * h, g, u);
          R.store_planes(w.planes[0] + at, w.plane, g, w.wide_planes);
          R.store_planes(w.planes[1] + at, w.plane, u, w.wide_planes);
        }
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // neither CTA leaves while the other may reach into it
  tc_fence_after();
  if (warp == 2) tmem_dealloc_pair(tb, 512);
}

// ----------------------------------------------------------------------- host

// Parts of the K axis: in us, a step takes 0.85, a tile's start and end 3, partial sums 4 and their traffic.
int splits_of(const Spec &S) {
  const int steps = S.sums * cut(S.K, BK);
  const double tiles = (double)cut(S.M[0], 256) * cut(S.N[0], BN) * S.problems;
  int best = 1;
  double least = 1e30;
  for (int s = 1; s <= 32 && (s == 1 || steps >= 2 * s); ++s) {
    const double waves = (double)(long long)((tiles * s + PAIRS - 1) / PAIRS);
    const double c = waves * ((steps + s - 1) / s * 0.85 + 3) +
                     (s > 1 ? 4 + (double)S.M[0] * S.N[0] * S.problems * (8 * s + 4) / 4e6 : 0);
    if (c < 0.97 * least) {
      least = c;
      best = s;
    }
  }
  return best;
}
size_t part_of(const Spec &S) {
  const int n = splits_of(S);
  return n > 1 ? (size_t)n * S.M[0] * S.N[0] * S.problems : 0;
}

template <int EPI> kdn_status_t launch(Work &w, cudaStream_t s) {
  w.wide = 1;  // (columns are a multiple of 8)
  for (const float *p : {(const float *)w.out[0], (const float *)w.out[1], (const float *)w.out[2], w.in[0], w.in[1]})
    if ((uintptr_t)p % 32) w.wide = 0;
  w.wide_planes = w.p[0].N % 16 == 0 && w.plane % 16 == 0;
  static std::atomic<unsigned long long> done{0};
  const kdn_status_t st = once_a_device(done, [] {
    return cudaFuncSetAttribute(k_ffn_f32<EPI>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM) == cudaSuccess;
  });
  if (st != KDN_OK) return st;
  return launch_beside(k_ffn_f32<EPI>, dim3(2 * (w.tiles < PAIRS ? w.tiles : PAIRS)), THREADS, SMEM, s, w);
}

// planes of a matrix: A's rows a CTA are 128, B's 64
bool map_planes(CUtensorMap *m, const Operand &x, long long rows, long long K, int box) {
  return x.own ? map_of(m, x.p, false, rows, K, 3, 64, 64, true, 3) : map_of(m, x.p, false, K, rows, 3, 64, box, true, 3);
}

kdn_status_t plain(const Spec &S, float *part, unsigned *status, cudaStream_t s) {
  Work w{};
  const int splits = splits_of(S);
  w.am = S.a[0].own;
  w.bm = S.b[0].own;
  w.np = S.problems;
  w.status = status;
  size_t at = 0;
  for (int i = 0; i < S.problems; ++i) {
    Problem &p = w.p[i];
    p.M = (int)S.M[i];
    p.N = (int)S.N[i];
    p.tm = cut(S.M[i], 256);
    p.tn = cut(S.N[i], BN);
    p.splits = splits;
    p.tiles = p.tm * p.tn * splits;
    w.tiles += p.tiles;
    w.out[i] = splits > 1 ? part + at : static_cast<float *>(S.out[i]);
    at += (size_t)splits * S.M[i] * S.N[i];
    for (int j = 0; j < S.sums; ++j) {
      p.steps[j] = cut(S.K, BK);
      p.a[j] = 2 * (i + j);
      p.b[j] = 2 * (i + j) + 1;
      if (!map_planes(w.maps + p.a[j], S.a[i + j], S.M[i], S.K, 128) ||
          !map_planes(w.maps + p.b[j], S.b[i + j], S.N[i], S.K, 64))
        return KDN_ERR_CUDA;
    }
  }
  const kdn_status_t st = launch<PLAIN>(w, s);
  if (st != KDN_OK || splits == 1) return st;
  Spec R = S;
  R.out_f32 = true;
  return join_parts(R, splits, part, s);
}

// p: planes in the places of the tensors; a: the call's own
kdn_status_t gate(const FfnArgs &p, const FfnArgs &a, bool back, cudaStream_t s) {
  Work w{};
  w.act = a.act;
  w.status = a.status;
  w.bm = back;
  w.np = 1;
  Problem &P = w.p[0];
  P.M = (int)a.rows;
  P.N = a.F;
  P.tm = cut(a.rows, 256);
  P.tn = cut(a.F, back ? BN : BN / 2);
  P.splits = 1;
  w.tiles = P.tiles = P.tm * P.tn;
  P.steps[0] = cut(a.D, BK);
  P.b[0] = 1;
  P.b[1] = 2;
  w.plane = (size_t)a.rows * a.F;
  bool ok = map_planes(w.maps, {back ? p.dy : p.x, false}, a.rows, a.D, 128);
  if (back) {
    w.in[0] = static_cast<const float *>(a.g);
    w.in[1] = static_cast<const float *>(a.u);
    w.planes[0] = static_cast<bf *>(p.dg);
    w.planes[1] = static_cast<bf *>(p.du);
    ok = ok && map_planes(w.maps + 1, {p.wd, true}, a.F, a.D, 64);
  } else {
    w.out[0] = static_cast<float *>(a.g);
    w.out[1] = static_cast<float *>(a.u);
    w.out[2] = static_cast<float *>(a.h);
    w.planes[0] = static_cast<bf *>(p.h);
    ok = ok && map_planes(w.maps + 1, {p.wg, false}, a.F, a.D, 64) && map_planes(w.maps + 2, {p.wu, false}, a.F, a.D, 64);
  }
  if (!ok) return KDN_ERR_CUDA;
  return back ? launch<DGATE>(w, s) : launch<GATE>(w, s);
}

size_t round_up(size_t x) { return (x + 255) / 256 * 256; }

// The planes' places in the workspace; returns their bytes.
size_t planes_of(const FfnArgs &a, bool back, char *base, FfnArgs *p, Cuts *c) {
  size_t at = 0;
  int n = 0;
  auto room = [&](size_t elements, const void *from) {
    char *to = base ? base + at : nullptr;
    at += round_up(elements * 6);
    if (from && c) {
      c->from[n] = static_cast<const float *>(from);
      c->to[n] = reinterpret_cast<bf *>(to);
      c->n[n++] = elements;
    }
    return to;
  };
  const size_t xs = (size_t)a.rows * a.D, hs = (size_t)a.rows * a.F, ws = (size_t)a.D * a.F;
  FfnArgs r = a;
  r.x = room(xs, a.x);
  r.wg = room(ws, a.wg);
  r.wu = room(ws, a.wu);
  r.wd = room(ws, a.wd);
  r.h = room(hs, back ? a.h : nullptr);
  if (back) {
    r.dy = room(xs, a.dy);
    r.dg = room(hs, nullptr);
    r.du = room(hs, nullptr);
  }
  if (p) *p = r;
  return at;
}

kdn_status_t cut_planes(const FfnArgs &a, bool back, FfnArgs *p, cudaStream_t s) {
  Cuts c{};
  planes_of(a, back, static_cast<char *>(a.planes), p, &c);
  c.status = a.status;
  size_t most = 0;
  const int n = back ? 6 : 4;
  for (int i = 0; i < n; ++i) most = c.n[i] > most ? c.n[i] : most;
  const size_t blocks = (most + 2047) / 2048;
  return launch_beside(k_ffn_split, dim3((unsigned)(blocks < 1216 ? blocks : 1216), n), 256, 0, s, c);
}

}  // namespace

size_t ffn_planes_bytes_f32(const FfnArgs &a, bool back) {
  return ffn_few_rows_f32(a) ? ffn_gradients_bytes_rows_f32(a, back) : planes_of(a, back, nullptr, nullptr, nullptr);
}

size_t ffn_part_floats_f32(const FfnArgs &a, bool back) {
  if (ffn_few_rows_f32(a)) return ffn_part_floats_rows_f32(a, back);
  if (!back) return part_of(down(a));
  const size_t x = part_of(back_x(a)), y = part_of(back_w(a));
  return x > y ? x : y;
}

kdn_status_t launch_ffn_fwd_f32(const FfnArgs &a, cudaStream_t s) {
  if (ffn_few_rows_f32(a)) return launch_ffn_fwd_rows_f32(a, s);
  FfnArgs p;
  kdn_status_t st = cut_planes(a, false, &p, s);
  if (st != KDN_OK || (st = gate(p, a, false, s)) != KDN_OK) return st;
  return plain(down(p), a.part, a.status, s);
}

kdn_status_t launch_ffn_bwd_f32(const FfnArgs &a, cudaStream_t s) {
  if (ffn_few_rows_f32(a)) return launch_ffn_bwd_rows_f32(a, s);
  FfnArgs p;
  kdn_status_t st = cut_planes(a, true, &p, s);
  if (st != KDN_OK || (st = gate(p, a, true, s)) != KDN_OK) return st;
  if ((st = plain(back_x(p), a.part, a.status, s)) != KDN_OK) return st;
  return plain(back_w(p), a.part, a.status, s);
}

}  // namespace kdn
