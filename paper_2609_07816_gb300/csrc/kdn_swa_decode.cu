// kdn_swa_decode.cu -- one token of every sequence over the bounded cache of the
// sliding-window attention (bfloat16).
//
// The cache's filled slots are a prefix, and attention does not care for their order, so a
// step is o = softmax(c q K^T) V over the first n slots: every byte of K and V is read once
// and HBM traffic bounds it.  A CTA serves up to 16 query heads that share a kv head
// (the rows of an m16n8k16 product, so that grouped heads read the cache once), and each
// of its 4 warps goes over its own chunks of 8 KB of K and V with a pipeline of its own: 16-byte
// asynchronous copies into 128-byte-swizzled rows, S = Q K^T and O += P V on the legacy
// tensor path (a chunk's products take a third of its copy's time), a running softmax.
// Two CTAs of 96 KB an SM keep about 128 KB of loads in flight.
//
// When there are few (sequence, kv head) pairs a cluster of CTAs splits the slots and joins
// the partial softmaxes through distributed shared memory: one launch, no workspace.
//
// The new token's row is taken from the inputs wherever it is needed and written into
// its slot by one CTA of the group: no CTA reads the slot that another one writes.
#include <cooperative_groups.h>
#include <math.h>

#include "kdn_swa.cuh"

namespace kdn {
namespace {

namespace cg = cooperative_groups;

constexpr int NT = 128, WARPS = 4, STAGES = 3, HEADS = 16;
template <int D> constexpr int KEYS = 2048 / D;  // a chunk: 4 KB of K and 4 KB of V
constexpr int CHUNK = 4096;
constexpr int SMEM = WARPS * STAGES * 2 * CHUNK;

__device__ __forceinline__ uint32_t smem_at(const void *p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
// 16 bytes, or zeros where `bytes` is 0
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t *r, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t *r, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
// 16 x 8 += 16 x 16 (rows) times 16 x 8
__device__ __forceinline__ void mma(float *c, const uint32_t *a, const uint32_t *b) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&p);
}
__device__ __forceinline__ float factor(float m, float ref) { return m == -INFINITY ? 0.f : exp2f(m - ref); }

// 16-byte column of a row of D bf16 in shared memory: rows that are read together lie in
// different banks.
template <int D> __device__ __forceinline__ int swz(int c, int r) {
  return D >= 64 ? c ^ (r & 7) : c ^ (r >> 1 & 3);
}

template <int D>
__global__ void __launch_bounds__(NT, 2)
    k_swa_decode_tc(const SwaArgs a, __nv_bfloat16 *kc, __nv_bfloat16 *vc, const int *pos, const int head_blocks) {
  constexpr int KN = KEYS<D>, ROW = D * 2, VPR = ROW / 16, KT = D / 16, NTL = KN / 8;
  extern __shared__ __align__(128) unsigned char sm[];
  __shared__ float s_m[HEADS], s_l[HEADS];  // this CTA's part, for the cluster
  cg::cluster_group cluster = cg::this_cluster();
  const int C = gridDim.x, rank = blockIdx.x;  // the cluster is the x axis of the grid
  const int hk = blockIdx.y / head_blocks, h0 = hk * a.G + blockIdx.y % head_blocks * HEADS, b = blockIdx.z;
  const int heads = min(HEADS, (hk + 1) * a.G - h0);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int p = pos[b];
  __nv_bfloat16 *o = static_cast<__nv_bfloat16 *>(a.o) + ((size_t)b * a.H + h0) * D;
  if (p < 0) {  // an idle sequence (the whole cluster leaves)
    for (int e = rank * NT + tid; e < heads * D; e += C * NT) o[e] = __float2bfloat16_rn(0.f);
    return;
  }
  const size_t slots = (size_t)a.W + a.ns;
  const int slot = p < a.ns ? p : a.ns + (p - a.ns) % a.W;
  const int n = (int)min((long long)p + 1, (long long)slots);
  const size_t base = ((size_t)b * a.Hk + hk) * slots * D;
  const __nv_bfloat16 *kn = static_cast<const __nv_bfloat16 *>(a.k) + ((size_t)b * a.Hk + hk) * D;
  const __nv_bfloat16 *vn = static_cast<const __nv_bfloat16 *>(a.v) + ((size_t)b * a.Hk + hk) * D;

  // this warp's chunks: every (4 C)-th
  const int chunks = (n + KN - 1) / KN, step = C * WARPS;
  const uint32_t buf = smem_at(sm) + warp * STAGES * 2 * CHUNK;
  auto load = [&](int ch, int st) {
    if (ch < chunks) {
      const uint32_t dst = buf + st * 2 * CHUNK;
#pragma unroll
      for (int i = 0; i < CHUNK / 16 / 32; ++i) {
        const int e = i * 32 + lane, r = e / VPR, c = e % VPR, j = ch * KN + r;
        const bool live = j < n;  // rows past n are zeros, whatever the cache holds
        const size_t at = base + (size_t)(live ? j : 0) * D + c * 8;
        const uint32_t to = dst + r * ROW + (swz<D>(c, r) << 4);
        copy16(to, j == slot ? kn + c * 8 : kc + at, live ? 16 : 0);
        copy16(to + CHUNK, j == slot ? vn + c * 8 : vc + at, live ? 16 : 0);
      }
    }
    copies_commit();
  };
  int ch = rank * WARPS + warp;
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) load(ch + s * step, s);

  if (rank == 0 && blockIdx.y % head_blocks == 0 && tid < 2 * VPR) {  // the new token's slot
    const int c = tid % VPR;
    const __nv_bfloat16 *src = tid < VPR ? kn : vn;
    __nv_bfloat16 *dst = (tid < VPR ? kc : vc) + base + (size_t)slot * D;
    reinterpret_cast<uint4 *>(dst)[c] = reinterpret_cast<const uint4 *>(src)[c];
  }

  // queries: rows of the products, zeros past the group's heads
  const int r0 = lane >> 2, cq = (lane & 3) * 2;
  uint32_t q[KT][4];
#pragma unroll
  for (int k = 0; k < KT; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = r0 + (e & 1) * 8, c = k * 16 + cq + (e >> 1) * 8;
      q[k][e] = r < heads ? *reinterpret_cast<const uint32_t *>(static_cast<const __nv_bfloat16 *>(a.q) +
                                                                ((size_t)b * a.H + h0 + r) * D + c)
                          : 0u;
    }
  const float c2 = a.scale * kLog2e;
  float acc[D / 8][4] = {}, m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  const int mi = lane >> 3, mr = lane & 7;
  int st = 0;
  for (; ch < chunks; ch += step) {
    copies_wait<STAGES - 2>();
    __syncwarp();  // the other lanes' copies too, and their reads of the stage loaded next
    load(ch + (STAGES - 1) * step, st == 0 ? STAGES - 1 : st - 1);
    const uint32_t sk = buf + st * 2 * CHUNK, sv = sk + CHUNK;
    st = st + 1 == STAGES ? 0 : st + 1;
    float s[NTL][4] = {};
#pragma unroll
    for (int t = 0; t < NTL; t += 2) {
      const int key = t * 8 + (mi >> 1) * 8 + mr;
#pragma unroll
      for (int k = 0; k < KT; ++k) {
        uint32_t f[4];
        ldsm4(f, sk + key * ROW + (swz<D>(k * 2 + (mi & 1), key) << 4));
        mma(s[t], q[k], f);
        mma(s[t + 1], q[k], f + 2);
      }
    }
    float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int t = 0; t < NTL; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool live = ch * KN + t * 8 + cq + (e & 1) < n;
        s[t][e] = live ? s[t][e] * c2 : -INFINITY;
        mx[e >> 1] = fmaxf(mx[e >> 1], s[t][e]);
      }
    float f[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 1));
      mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 2));
      mx[i] = fmaxf(mx[i], m[i]);  // a chunk has at least one key: finite unless the scores are not
      f[i] = exp2f(m[i] - mx[i]);
      m[i] = mx[i];
      l[i] *= f[i];
    }
    if (__any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f))
#pragma unroll
      for (int t = 0; t < D / 8; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[t][e] *= f[e >> 1];
#pragma unroll
    for (int t = 0; t < NTL; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[t][e] = exp2f(s[t][e] - m[e >> 1]);
        l[e >> 1] += s[t][e];
      }
#pragma unroll
    for (int t = 0; t < NTL; t += 2) {
      const uint32_t w[4] = {pack2(s[t][0], s[t][1]), pack2(s[t][2], s[t][3]), pack2(s[t + 1][0], s[t + 1][1]),
                             pack2(s[t + 1][2], s[t + 1][3])};
      const int key = t * 8 + (mi & 1) * 8 + mr;
#pragma unroll
      for (int d = 0; d < D / 8; d += 2) {
        uint32_t g[4];
        ldsm4t(g, sv + key * ROW + (swz<D>(d + (mi >> 1), key) << 4));
        mma(acc[d], w, g);
        mma(acc[d + 1], w, g + 2);
      }
    }
  }
  copies_wait<0>();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
  }

  // join: the warps' partial results, then those of the cluster's CTAs
  __syncthreads();  // the stages are free
  float *so = reinterpret_cast<float *>(sm);           // [WARPS][heads][D], then [heads][D]
  float *sw = so + WARPS * HEADS * D;                  // [WARPS][2][HEADS]: m, l
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = r0 + i * 8;
    if (r < heads) {
#pragma unroll
      for (int t = 0; t < D / 8; ++t)
        *reinterpret_cast<float2 *>(so + (warp * heads + r) * D + t * 8 + cq) =
            make_float2(acc[t][2 * i], acc[t][2 * i + 1]);
      if ((lane & 3) == 0) {
        sw[warp * 2 * HEADS + r] = m[i];
        sw[warp * 2 * HEADS + HEADS + r] = l[i];
      }
    }
  }
  __syncthreads();
  for (int e = tid; e < heads * D; e += NT) {
    const int r = e / D;
    float mm = -INFINITY, ll = 0.f, x = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) mm = fmaxf(mm, sw[w * 2 * HEADS + r]);
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float g = factor(sw[w * 2 * HEADS + r], mm);
      ll = fmaf(sw[w * 2 * HEADS + HEADS + r], g, ll);
      x = fmaf(so[w * heads * D + e], g, x);
    }
    if (C == 1) {
      o[e] = __float2bfloat16_rn(x / ll);
    } else {
      so[e] = x;  // warp 0's place: only this thread reads and writes element e of it
      if (e % D == 0) {
        s_m[r] = mm;
        s_l[r] = ll;
      }
    }
  }
  if (C == 1) return;
  cluster.sync();
  for (int e = rank * NT + tid; e < heads * D; e += C * NT) {
    const int r = e / D;
    float mm = -INFINITY, ll = 0.f, x = 0.f;
    for (int k = 0; k < C; ++k) mm = fmaxf(mm, *cluster.map_shared_rank(s_m + r, k));
#pragma unroll 4
    for (int k = 0; k < C; ++k) {
      const float g = factor(*cluster.map_shared_rank(s_m + r, k), mm);
      ll = fmaf(*cluster.map_shared_rank(s_l + r, k), g, ll);
      x = fmaf(*cluster.map_shared_rank(so + e, k), g, x);
    }
    o[e] = __float2bfloat16_rn(x / ll);
  }
  cluster.sync();  // no CTA leaves while another reads its part
}

template <int D>
kdn_status_t launch(const SwaArgs &a, void *kc, void *vc, const int *pos, cudaStream_t s) {
  const int head_blocks = (a.G + HEADS - 1) / HEADS;
  // CTAs of a cluster, by what a step costs with C of them: each wave of 304 CTAs (two an
  // SM) about 8 us of start and end, 10.5 in a cluster, 17 in one of more than 8; and the
  // bytes, at 68 GB/s a CTA or 6.8 TB/s together.  Measured at d = 128, 2052 slots: one
  // sequence of 16 heads 22.5, 16.4, 14.3, 12.3, 18.4 us with C = 1, 2, 4, 8, 16; 64 x 4
  // pairs 58, 64, 68, 78, 140 us; 1 pair of 32768 slots 248, 131, 72, 41, 27 us.
  const double pairs = (double)a.B * a.Hk * head_blocks, bytes = 4.0 * D * ((double)a.W + a.ns);
  int C = 1;
  double best = 0;
  for (int c = 1; c <= 16; c *= 2) {
    const double rate = bytes / c / 68e3, all = pairs * bytes / 6.8e6;
    const double cost = ceil(pairs * c / 304) * (c == 1 ? 8 : c <= 8 ? 10.5 : 17) + (rate > all ? rate : all);
    if (c == 1 || cost < best) {
      best = cost;
      C = c;
    }
  }
  auto kernel = k_swa_decode_tc<D>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM) != cudaSuccess ||
      cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
    return KDN_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(C, a.Hk * head_blocks, a.B);
  cfg.blockDim = dim3(NT);
  cfg.dynamicSmemBytes = SMEM;
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = C;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, a, static_cast<__nv_bfloat16 *>(kc), static_cast<__nv_bfloat16 *>(vc), pos,
                            head_blocks) == cudaSuccess
             ? KDN_OK
             : KDN_ERR_CUDA;
}

}  // namespace

kdn_status_t launch_swa_decode_tc(const SwaArgs &a, void *kc, void *vc, const int *pos, cudaStream_t s) {
  return a.d == 128  ? launch<128>(a, kc, vc, pos, s)
         : a.d == 64 ? launch<64>(a, kc, vc, pos, s)
                     : launch<32>(a, kc, vc, pos, s);
}

}  // namespace kdn
