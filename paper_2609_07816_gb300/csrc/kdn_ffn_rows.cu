// kdn_ffn_rows.cu -- the feed-forward block of few tokens (bfloat16): single tokens of a
// serving batch, where reading the weights once is all that there is to do.
//
// The weights take the side of 128 of the tensor cores' tile and the tokens the other (16 .. 128
// of them), so that a CTA streams its rows of a weight matrix once, for all tokens:
//   GATE   `per` rows of Wg and as many of Wu (K = D): g, u and act(g) u
//   PLAIN  rows of Wd (K = F): y;  columns of Wg, then of Wu (K = 2F): dx
//   DGATE  columns of Wd (K = D): dh, and with g and u: dg and du
// Rows are dealt out evenly, in any number up to the tile's: idle rows of a tile cost nothing that
// bounds here.  Where that leaves SMs idle a cluster's CTAs share a tile, each with a part of the K axis, and
// add up their sums through distributed shared memory in the order of their ranks.
//
// What one thread does for a step of 64 along K (a wait of 90 cycles, copies at 100 each; a wait, a commit of 45
// and four products at 40 each) takes longer than the step's share of HBM.  So up to four pipelines stand side by
// side in a CTA, each with a loading and a multiplying thread, stages and an accumulator of its own; pipeline
// number p takes steps p, p + P, ...
//
// A call's second kernel starts beside the first (both fit an SM at once) and loads its weights
// while the tokens' side is still being computed.  The start of a stream of weights and what lies between the two
// kernels bound it: 61 tokens of 2048 x 5632 take 11 us in the gate from first to last byte (4.2 TB/s), 10 more in y.
#include "kdn_ffn_tc.cuh"

namespace kdn {
namespace {

using namespace ffn;

constexpr int THREADS = 256, MAX_PIPES = 4, MAX_STAGES = 16;

struct Work {
  CUtensorMap a[2], b[2];
  int mode, own;        // own: the weights' rows of the tile lie along their matrix' rows (K is its other axis)
  int M, per, second;   // rows of the tile's side; of a CTA; where u's begin in the tile
  int rows, nb;         // tokens; padded to 16 (places that hold none hold anything, and give sums that nobody reads)
  int steps0, steps;    // K steps of the first operands, and of both
  int parts;            // CTAs of a cluster
  int pipes;            // pipelines of a CTA
  int a_bytes, stage, stages;  // bytes of the weights' part of a stage, of a stage; stages of a pipeline
  int act, first, back;
  const __nv_bfloat16 *in[2];  // DGATE: g, u
  __nv_bfloat16 *out[3];       // h (GATE: then g, u), dg and du, or y and dx
  unsigned *status;
};

__device__ __forceinline__ void load_2d(void *dst, const CUtensorMap *map, uint64_t *bar, int c0, int c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
          smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ void prefetch_2d(const CUtensorMap *map, int c0, int c1) {
  asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(reinterpret_cast<uint64_t>(map)),
               "r"(c0), "r"(c1)
               : "memory");
}
__device__ __forceinline__ float4 at_cluster(uint32_t addr) {
  float4 x;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w)
               : "r"(addr)
               : "memory");
  return x;
}

__global__ void __launch_bounds__(THREADS) k_ffn_rows(const __grid_constant__ Work w) {
  extern __shared__ unsigned char smraw[];
  unsigned char *sm =
      reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smraw) + 1023) & ~uintptr_t(1023));
  __shared__ uint64_t full[MAX_STAGES], empty[MAX_STAGES], done[MAX_PIPES];
  __shared__ uint32_t s_tmem;
  __shared__ int s_fail;

  const int tid = threadIdx.x, warp = tid >> 5;
  const int rank = w.parts > 1 ? (int)cluster_rank() : 0, m0 = (int)blockIdx.x / w.parts * w.per;
  const int k0 = w.steps * rank / w.parts, nk = w.steps * (rank + 1) / w.parts - k0;
  const int pipes = min(w.pipes, nk), NS = w.stages;
  const uint32_t need = w.pipes * w.nb, cols = need <= 64 ? 64 : need <= 128 ? 128 : need <= 256 ? 256 : 512;
  if (w.mode == DGATE) {  // g and u are on their way to L2 while the products run
    const int chunks = (min(w.per, w.M - m0) * 2 + 127) >> 7, mine = (w.rows - rank + w.parts - 1) / w.parts;
    for (int e = tid; e < mine * chunks; e += THREADS) {
      const size_t at = (size_t)(rank + e / chunks * w.parts) * w.M + m0 + e % chunks * 64;
      asm volatile("prefetch.global.L2 [%0];" ::"l"(w.in[0] + at));
      asm volatile("prefetch.global.L2 [%0];" ::"l"(w.in[1] + at));
    }
  }
  const int pipe = warp & 3;
  const bool loads = warp < 4 && pipe < pipes;
  uint64_t *const pf = full + pipe * NS, *const pe = empty + pipe * NS;
  unsigned char *const ps = sm + pipe * NS * w.stage;
  const Waiter wait{&s_fail, w.status};
  const bool two = w.mode == GATE, own = w.own, wide = w.per > 64;
  const uint32_t bytes = ((two ? 2 : 1) * w.per + w.rows) * 128;
  const int steps0 = w.steps0, stage = w.stage, second = w.second * 128, behind = w.a_bytes;
  const int end = k0 + nk, first = k0 + pipe;
  const CUtensorMap *const ma = w.a, *const mb = w.b;
  auto weights = [&](int k, int st) {
    const int seg = k >= steps0, kk = (k - (seg ? steps0 : 0)) * BK;
    unsigned char *sa = ps + st * stage;
    mbar_expect_tx(pf + st, bytes);
    if (own) {
      load_2d(sa, ma, pf + st, kk, m0);
      if (two) load_2d(sa + second, ma + 1, pf + st, kk, m0);
    } else {
      load_2d(sa, ma + seg, pf + st, m0, kk);
      if (wide) load_2d(sa + 8192, ma + seg, pf + st, m0 + 64, kk);
    }
  };
  auto tokens = [&](int k, int st) {
    const int seg = k >= steps0;
    load_2d(ps + st * stage + behind, mb + seg, pf + st, (k - (seg ? steps0 : 0)) * BK, 0);
  };
  if (loads) {
    // A loading thread makes its pipeline's barriers and has the first weights on their way before the CTA's
    // other threads are ready; they do not wait for the kernel before either.
    if (elect_one()) {
      for (int i = 0; i < NS; ++i) {
        mbar_init(pf + i, 1);
        mbar_init(pe + i, 1);
      }
      mbar_init(done + pipe, 1);
      fence_mbar_init();
      fence_proxy_async();
      if (w.first) wait_for_previous();  // (which may write the weights; the second kernel starts behind that)
      int st = 0, k = first;
      for (; k < end && st < NS; k += pipes) weights(k, st++);
      // the second kernel's other weights come as far as L2 meanwhile
      if (!w.first)
        for (; k < end; k += pipes) {
          const int seg = k >= steps0, kk = (k - (seg ? steps0 : 0)) * BK;
          if (own) {
            prefetch_2d(ma, kk, m0);
          } else {
            prefetch_2d(ma + seg, m0, kk);
            if (wide) prefetch_2d(ma + seg, m0 + 64, kk);
          }
        }
    }
    __syncwarp();
  }
  if (tid == 32 * 7) {
    s_fail = 0;
    // (a wait runs out seconds after the launch, whose first block this is)
    if (w.first && blockIdx.x == 0) {
      wait_for_previous();
      *w.status = 0;
    }
  }
  if (warp == 5) {
    tmem_alloc(&s_tmem, cols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // The next kernel starts behind this one's allocation (whoever waits for TMEM waits for nobody that starts
  // later), and the second one, which reads weights at once, behind whatever came before the call.
  if (w.first) wait_for_previous();
  let_next_start();
  const uint32_t tb = s_tmem;

  if (loads) {  // ------------------------------------------------------------- loads
    if (elect_one()) {
      wait_for_previous();
      int st = 0, k = first;
      for (; k < end && st < NS; k += pipes) tokens(k, st++);
      bool ok = true;
      st = 0;
      for (int turn = 0; k < end; k += pipes) {
        if (!(ok = wait(pe + st, turn))) break;
        weights(k, st);
        tokens(k, st);
        if (++st == NS) st = 0, turn ^= 1;
      }
      if (!ok) {  // copies in flight land before the CTA leaves
        const int n = (k - first) / pipes;  // issued
        for (int m = max(0, n - NS); m < n; ++m) mbar_wait(pf + m % NS, (m / NS) & 1, kWait >> 6);
      }
    }
  } else if (warp >= 4 && pipe < pipes) {  // -------------------------------------- products
    if (elect_one()) {
      const uint32_t id = idesc_bf16(128, w.nb, !w.own, 0), base = smem_u32(ps), acc = tb + pipe * w.nb;
      const uint64_t da = sw128_desc(base, w.own ? 16 : 8192, 1024), db = sw128_desc(base + w.a_bytes, 16, 1024);
      const uint64_t ka = (w.own ? 32 : 2048) >> 4;
      bool ok = true;
      uint32_t some = 0;
      for (int k = pipe, st = 0, turn = 0; k < nk; k += pipes) {
        if (!(ok = wait(pf + st, turn))) break;
        const uint64_t off = (uint64_t)(st * (stage >> 4));
#pragma unroll
        for (int kk = 0; kk < BK / 16; ++kk) umma_bf16(acc, da + off + kk * ka, db + off + kk * 2, id, kk ? 1u : some);
        umma_commit(pe + st);
        some = 1;
        if (++st == NS) st = 0, turn ^= 1;
      }
      if (ok) {
        umma_commit(done + pipe);
        wait(done + pipe, 0);
      }
    }
  }
  // (the others wait here: threads that poll a barrier take issue slots from those that work)
  __syncwarp();
  __syncthreads();
  tc_fence_after();
  wait_for_previous();  // it may still read what is written here, or write what is read
  // Every copy has been consumed: the stages' memory holds the sums [token][128].  Half of the warps
  // take the even blocks of 16 tokens each, half the odd ones.
  float *sums = reinterpret_cast<float *>(sm);
  const int m = tid & 127;
  for (int c = 16 * (warp >> 2); c < w.nb; c += 32) {
    float x[16], y[16];
    const uint32_t at = tb + c + ((uint32_t)(32 * (warp & 3)) << 16);
    tmem_ld16(at, x);
    for (int p = 1; p < pipes; ++p) {
      tmem_ld16(at + p * w.nb, y);
#pragma unroll
      for (int j = 0; j < 16; ++j) x[j] += y[j];
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) sums[(c + j) * 128 + m] = x[j];
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 5) {  // before the CTAs of a cluster wait for one another, which may wait for TMEM
    tc_fence_after();
    tmem_dealloc(tb, cols);
  }
  if (w.parts > 1) cluster_sync_all();

  // eight rows of a token a thread; a cluster's CTAs take the tokens in turn
  const int chunks = min(w.per, w.M - m0) >> 3, mine = (w.rows - rank + w.parts - 1) / w.parts;
  for (int e = tid; e < mine * chunks; e += THREADS) {
    const int j = e / chunks, i = (e - j * chunks) * 8, t = rank + j * w.parts;
    const size_t at = (size_t)t * w.M + m0 + i;
    auto sum = [&](int i, float *x) {
      const float *p = sums + t * 128 + i;
      if (w.parts == 1) {
        *reinterpret_cast<float4 *>(x) = *reinterpret_cast<const float4 *>(p);
        *reinterpret_cast<float4 *>(x + 4) = *reinterpret_cast<const float4 *>(p + 4);
        return;
      }
#pragma unroll
      for (int l = 0; l < 8; ++l) x[l] = 0.f;
      for (int r = 0; r < w.parts; ++r) {
        const float4 a = at_cluster(in_cta(p, r)), b = at_cluster(in_cta(p + 4, r));
        x[0] += a.x; x[1] += a.y; x[2] += a.z; x[3] += a.w;
        x[4] += b.x; x[5] += b.y; x[6] += b.z; x[7] += b.w;
      }
    };
    float x[8], g[8], u[8];
    if (w.mode == DGATE) {
      const uint4 pg = *reinterpret_cast<const uint4 *>(w.in[0] + at), pu = *reinterpret_cast<const uint4 *>(w.in[1] + at);
      sum(i, x);
      fused::unpack_bf8(pg, g);
      fused::unpack_bf8(pu, u);
      hidden_gradients<8>(w.act, x, g, u);
      *reinterpret_cast<uint4 *>(w.out[0] + at) = fused::pack_bf8(g);
      *reinterpret_cast<uint4 *>(w.out[1] + at) = fused::pack_bf8(u);
    } else {
      sum(i, x);
      if (w.mode == GATE) {
        sum(w.second + i, u);
        if (w.out[2]) {
          *reinterpret_cast<uint4 *>(w.out[1] + at) = fused::pack_bf8(x);
          *reinterpret_cast<uint4 *>(w.out[2] + at) = fused::pack_bf8(u);
        }
        gate_values<8>(w.act, x, u);
      }
      *reinterpret_cast<uint4 *>(w.out[0] + at) = fused::pack_bf8(x);
    }
  }
  if (w.parts > 1) {
    __syncwarp();
    cluster_sync_all();  // the others may still read this CTA's sums
  }
}

// How many rows a CTA takes and how many share a tile: the time of a CTA's loads at its share of HBM
// (weights) and of L2 (tokens), in us, a tenth at least, and 1.5 for a sum over a cluster.
struct Deal {
  int per, parts;
};
Deal deal(int M, int steps, int nb, int matrices, bool own) {
  Deal best{64, 1};
  double least = 1e30;
  for (int parts = 1; parts <= 4 && parts <= steps; parts *= 2) {
    const int tiles = 152 / parts, most = matrices == 2 ? 64 : 128;
    for (int waves = 1; waves < 1 << 20; ++waves) {
      int per = cut(M, tiles * waves);
      per = own ? (per + 7) / 8 * 8 : (per + 63) / 64 * 64;
      if (per > most) continue;
      const double ctas = (double)cut(M, per) * parts, rounds = cut((long long)ctas, 152);
      const double step = matrices * per * 128 / 45e3 + nb * 128 / 130e3;
      const double c = rounds * ((steps + parts - 1) / parts) * (step > 0.1 ? step : 0.1) + (parts > 1 ? 1.5 : 0);
      if (c < least) {
        least = c;
        best = {per, parts};
      }
      break;
    }
  }
  return best;
}

kdn_status_t launch(Work &w, cudaStream_t s) {
  // A call's two kernels share an SM and its TMEM, so that the second's start beside the first.  Not in the
  // backward of more than 64 tokens, whose second kernel is the longer one and would have too few stages (96 tokens,
  // 2048 x 5632: 61 us shared, 54 us alone; the forward 29 and 33 us).
  const bool share = w.nb <= 64 || !w.back;
  const int room = (!share ? 220 : w.first ? (w.nb <= 64 ? 120 : 140) : w.nb <= 64 ? 102 : 82) * 1024;
  w.stage = w.a_bytes + w.nb * 128;
  const int behind = w.stage < 16384 ? 16384 - w.stage : 0;  // (a product reads 128 rows from a stage's start)
  int stages = (room - behind) / w.stage;
  if (stages > MAX_STAGES) stages = MAX_STAGES;
  const int most = (w.steps + w.parts - 1) / w.parts;
  if (stages > most) stages = most;
  w.pipes = stages >= 2 * MAX_PIPES ? MAX_PIPES : stages > 1 ? stages / 2 : 1;
  const int columns = share ? 256 : 512;
  if (w.pipes * w.nb > columns) w.pipes = columns / w.nb;
  w.stages = stages / w.pipes;
  int bytes = w.pipes * w.stages * w.stage + behind;
  if (bytes < w.nb * 512) bytes = w.nb * 512;
  bytes += 1024;
  // (all of an SM's memory as shared memory: the size that fits the first kernel alone would keep the second out)
  static std::atomic<unsigned long long> done{0};
  const kdn_status_t st = once_a_device(done, [] {
    return cudaFuncSetAttribute(k_ffn_rows, cudaFuncAttributeMaxDynamicSharedMemorySize, 226 * 1024) == cudaSuccess &&
           cudaFuncSetAttribute(k_ffn_rows, cudaFuncAttributePreferredSharedMemoryCarveout, 100) == cudaSuccess;
  });
  if (st != KDN_OK) return st;
  cudaLaunchAttribute at[2]{};
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = w.parts;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t c{};
  c.gridDim = dim3((unsigned)(cut(w.M, w.per) * w.parts));
  c.blockDim = dim3(THREADS);
  c.dynamicSmemBytes = bytes;
  c.stream = s;
  c.attrs = at;
  c.numAttrs = 2;
  return cudaLaunchKernelEx(&c, k_ffn_rows, (const Work)w) == cudaSuccess ? KDN_OK : KDN_ERR_CUDA;
}

struct Side {  // a weight matrix, and the tokens' rows that it is multiplied with
  const void *weight, *tokens;
};
// n pairs of a sum over K columns of the tokens each (GATE: two matrices, one side of tokens)
kdn_status_t run(Work &w, const FfnArgs &a, int M, int K, const Side *p, int n, cudaStream_t s) {
  const int matrices = w.mode == GATE ? 2 : 1;
  w.M = M;
  w.rows = (int)a.rows;
  w.nb = (w.rows + 15) / 16 * 16;
  w.act = a.act;
  w.status = a.status;
  w.steps0 = cut(K, BK);
  w.steps = w.steps0 * (w.mode == GATE ? 1 : n);
  const Deal d = deal(M, w.steps, w.nb, matrices, w.own);
  w.per = d.per;
  w.parts = d.parts;
  w.second = (w.per + 7) / 8 * 8;
  w.a_bytes = matrices * w.second * 128;
  for (int i = 0; i < n; ++i) {
    const bool ok = w.own ? map_of(w.a + i, p[i].weight, false, K, M, 1, 64, w.per, false)
                          : map_of(w.a + i, p[i].weight, false, M, K, 1, 64, 64, false);
    if (!ok) return KDN_ERR_CUDA;
    if (p[i].tokens && !map_of(w.b + i, p[i].tokens, false, K, w.rows, 1, 64, w.rows, false)) return KDN_ERR_CUDA;
  }
  return launch(w, s);
}

}  // namespace

// (2048 x 5632: forward of 96 tokens 29 us here and 30 by tiles of 256, of 128 33 and 31; gradients of 128 57 and 62.
// At other sizes the two forms differ little there, but for the forward of small weights: 520 x 1400, forward of 96 here
// 12 and of 97 there 19, gradients of 128 here and 129 there 27; 4096 x 8192, 57 and 52, 121 and 125.)
// A hidden axis beyond 65536 would take more than that along K into one accumulator (dx 2 F into two or more).
bool ffn_few_rows(const FfnArgs &a, bool back) { return a.rows <= (back ? 128 : 96) && a.F <= 65536; }

kdn_status_t launch_ffn_fwd_rows(const FfnArgs &a, cudaStream_t s) {
  Work w{};
  w.mode = GATE;
  w.own = w.first = 1;
  w.out[0] = static_cast<bf *>(a.h);
  w.out[1] = static_cast<bf *>(a.g);
  w.out[2] = static_cast<bf *>(a.u);
  const Side up[2] = {{a.wg, a.x}, {a.wu, nullptr}};
  const kdn_status_t st = run(w, a, a.F, a.D, up, 2, s);
  if (st != KDN_OK) return st;
  w.mode = PLAIN;
  w.first = 0;
  w.out[0] = static_cast<bf *>(a.y);
  const Side down[1] = {{a.wd, a.h}};
  return run(w, a, a.D, a.F, down, 1, s);
}

kdn_status_t launch_ffn_bwd_rows(const FfnArgs &a, cudaStream_t s) {
  Work w{};
  w.mode = DGATE;
  w.first = w.back = 1;
  w.in[0] = static_cast<const bf *>(a.g);
  w.in[1] = static_cast<const bf *>(a.u);
  w.out[0] = static_cast<bf *>(a.dg);
  w.out[1] = static_cast<bf *>(a.du);
  const Side up[1] = {{a.wd, a.dy}};
  const kdn_status_t st = run(w, a, a.F, a.D, up, 1, s);
  if (st != KDN_OK) return st;
  w.mode = PLAIN;
  w.first = 0;
  w.out[0] = static_cast<bf *>(a.dx);
  const Side back[2] = {{a.wg, a.dg}, {a.wu, a.du}};
  return run(w, a, a.D, a.F, back, 2, s);
}

}  // namespace kdn
