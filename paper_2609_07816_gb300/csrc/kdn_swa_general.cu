// kdn_swa_general.cu -- sliding-window attention with sinks on the CUDA cores:
// float32 activations, float32 arithmetic throughout; and the parts that every path shares (the backward's
// row sums, the join of split key tiles, the copy of a prompt into the cache).
//
//   s_ij = c q_i.k_j,  o_i = sum_j exp(s_ij - lse_i) v_j   over the keys that i sees
//   dS = P (dO V^T - delta), dQ = c dS K, dK = c dS^T Q, dV = P^T dO
//
// Tiles are 64 queries x 64 keys, 256 threads; thread (ty, tx) owns rows ty + 16 i
// and columns tx + 16 j of a 64 x 64 product (i, j < 4), so that with rows of d + 4
// floats both operands' 16-byte reads are free of bank conflicts, and eight such
// reads feed 64 multiply-adds.  Shared memory bounds these kernels: at T4096 H16 d128 W1024
// it is at 82 % of its throughput in the forward (73 and 74 % in the gradients), the
// multiply-add pipe at 54 (50) %.  37 TFLOP/s forward, 25 of the five products that the
// gradients need (35 of the seven done), B2 T4096 H16 d128 W1024.
#include <cooperative_groups.h>
#include <math.h>

#include "kdn_swa.cuh"

namespace kdn {

namespace cg = cooperative_groups;

SwaSplits swa_splits(const SwaArgs &a, int BM, int BN) {
  SwaSplits p{};
  auto cdiv = [](long long x, long long y) { return (int)((x + y - 1) / y); };
  p.tiles = cdiv(a.T, BN);
  const int qtiles = cdiv(a.T, BM);
  p.sink_tiles = cdiv(a.ns < a.T ? a.ns : a.T, BN);
  const long long reach = (long long)a.W + BN - 2;  // last query of a window tile, from its first key
  const int nq = (int)(reach / BM + 1 < qtiles ? reach / BM + 1 : qtiles);
  const int iters = a.G * nq, iters_sink = a.G * qtiles;
  // Iterations of a split, where whole tiles would be less than two waves of one CTA an
  // SM: the length that ends soonest, each wave taking its longest split and a fixed part
  // (first loads, last stores; about two iterations, and two more where partial sums are
  // written and joined).  Many more splits than SMs would be bound by those sums.
  // Otherwise only a sink tile may be split, where its list is more than twice the others':
  // into k parts that are no shorter than those, for the least of what the splits add to
  // every SM, 4 k iterations a tile, and the list's k-th part, by which the last tile's may
  // outlast the rest.  Gradients at H16 d128 window 128, with splits of the others' length and
  // so: B1 T8192 4 sinks 194 and 172 us, B1 T65536 4 sinks 1321 and 1068 us (537 and 67 MB of
  // partial sums), B8 T8192 1024 sinks 4300 and 1887 us (4.3 GB and none).
  // Either way a call has at most 8 partial sums an SM: 160 MB.
  const long long heads = (long long)a.B * a.Hk, sinks = heads * p.sink_tiles, most = 8 * 152;
  int sink_whole = iters_sink;
  if (sinks && iters_sink > 2LL * iters) {
    const long long k = (long long)sqrt(iters_sink * 152.0 / (4.0 * sinks)), part = k < most / sinks ? k : most / sinks;
    if (part > 1) sink_whole = cdiv(iters_sink, part) > iters ? cdiv(iters_sink, part) : iters;
  }
  long long whole = 0;
  double best = 0;
  for (int n = 1; n <= 8 && (n == 1 || iters / n >= 2); ++n) {
    const int per = cdiv(iters, n), per_sink = n == 1 ? sink_whole : per;
    const long long blocks = (long long)p.sink_tiles * cdiv(iters_sink, per_sink) +
                             (long long)(p.tiles - p.sink_tiles) * cdiv(iters, per);
    const int longest = p.sink_tiles && per_sink > per ? per_sink : per;
    if (n == 1) whole = heads * blocks;
    else if (whole >= 2 * 152 || heads * blocks > most) break;
    const double cost = (double)((heads * blocks + 151) / 152) * (longest + (n == 1 ? 2 : 4));
    if (n == 1 || cost < 0.95 * best) {
      best = cost;
      p.per = per;
      p.per_sink = per_sink;
    }
  }
  p.splits = cdiv(iters, p.per);
  p.splits_sink = cdiv(iters_sink, p.per_sink);
  p.blocks = p.sink_tiles * p.splits_sink + (p.tiles - p.sink_tiles) * p.splits;
  p.part_blocks = p.splits > 1 ? p.blocks : p.splits_sink > 1 ? p.sink_tiles * p.splits_sink : 0;
  return p;
}

namespace {

constexpr int BT = kSwaGenTile, NT = 256, LP = BT + 4;  // LP: row stride of a 64 x 64 tile

template <int D> constexpr int LD = D + 4;

// acc[i][j] += sum_d A[ty + 16 i][d] B[tx + 16 j][d]
template <int D>
__device__ __forceinline__ void mm_nt(float (&acc)[4][4], const float *A, const float *B, int ty, int tx) {
#pragma unroll 4
  for (int d = 0; d < D; d += 4) {
    float4 x[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = *reinterpret_cast<const float4 *>(A + (ty + 16 * i) * LD<D> + d);
      y[i] = *reinterpret_cast<const float4 *>(B + (tx + 16 * i) * LD<D> + d);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        acc[i][j] = fmaf(x[i].x, y[j].x, acc[i][j]);
        acc[i][j] = fmaf(x[i].y, y[j].y, acc[i][j]);
        acc[i][j] = fmaf(x[i].z, y[j].z, acc[i][j]);
        acc[i][j] = fmaf(x[i].w, y[j].w, acc[i][j]);
      }
  }
}

// Column of entry c (of d / 16) that thread tx owns in a [64][d] product: groups of
// four (two for d = 32) consecutive columns.
template <int D> constexpr int VW = D >= 64 ? 4 : 2;
template <int D> __device__ __forceinline__ int col_of(int tx, int c) {
  return (c / VW<D>) * 16 * VW<D> + tx * VW<D> + c % VW<D>;
}

// acc[i][c] += sum_k P[ty + 16 i][k] X[k][col(c)]
template <int D>
__device__ __forceinline__ void mm_nn(float (&acc)[4][D / 16], const float *P, const float *X, int ty, int tx) {
  constexpr int NC = D / 16;
#pragma unroll 4
  for (int k = 0; k < BT; k += 4) {
    float p[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 t = *reinterpret_cast<const float4 *>(P + (ty + 16 * i) * LP + k);
      p[i][0] = t.x; p[i][1] = t.y; p[i][2] = t.z; p[i][3] = t.w;
    }
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      float x[NC];
#pragma unroll
      for (int c = 0; c < NC; c += VW<D>) {
        const float *src = X + (k + kk) * LD<D> + col_of<D>(tx, c);
        if constexpr (VW<D> == 4) {
          const float4 t = *reinterpret_cast<const float4 *>(src);
          x[c] = t.x; x[c + 1] = t.y; x[c + 2] = t.z; x[c + 3] = t.w;
        } else {
          const float2 t = *reinterpret_cast<const float2 *>(src);
          x[c] = t.x; x[c + 1] = t.y;
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < NC; ++c) acc[i][c] = fmaf(p[i][kk], x[c], acc[i][c]);
    }
  }
}

// Rows [r0, r0 + 64) of head h of a [B, T, heads, D] tensor on their way into a tile, in
// registers while the tile before them is worked on; rows at and past `len` are zeros
// (whatever memory holds there).
template <int D> struct Fetch {
  static constexpr int V4 = D / 4, N = BT * V4 / NT;
  float4 x[N];
  __device__ __forceinline__ void load(const void *src, int b, int h, int heads, int T, int r0, int len) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = i * NT + threadIdx.x, t = r0 + e / V4;
      x[i] = t < len ? static_cast<const float4 *>(src)[(((size_t)b * T + t) * heads + h) * V4 + e % V4]
                     : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
  __device__ __forceinline__ void store(float *dst) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = i * NT + threadIdx.x;
      *reinterpret_cast<float4 *>(dst + (e / V4) * LD<D> + 4 * (e % V4)) = x[i];
    }
  }
};
template <int D>
__device__ __forceinline__ void load_tile(float *dst, const void *src, int b, int h, int heads, int T, int r0,
                                          int len) {
  Fetch<D> f;
  f.load(src, b, h, heads, T, r0, len);
  f.store(dst);
}

// sum / max over the 16 threads of a row (tx = 0..15 of a half-warp)
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
__device__ __forceinline__ float row_max(float x) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}

template <int D> constexpr int FWD_SMEM = (2 * BT * LD<D> + (BT * LD<D> > BT * LP ? BT * LD<D> : BT * LP)) * 4;

template <int D> __global__ void __launch_bounds__(NT) k_swa_fwd(const SwaArgs a) {
  extern __shared__ __align__(16) float sm[];
  float *sq = sm, *sv = sq + BT * LD<D>, *sk = sv + BT * LD<D>, *sp = sk;  // P takes K's place
  constexpr int NC = D / 16;
  const int tid = threadIdx.x, ty = tid / 16, tx = tid % 16;
  const int b = blockIdx.z, h = blockIdx.y, hk = h / a.G, i0 = blockIdx.x * BT;
  const int len = swa_len(a, b), i1 = min(i0 + BT, len);
  float o[4][NC] = {}, m[4], l[4] = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) m[i] = -INFINITY;
  if (i0 < len) {
    load_tile<D>(sq, a.q, b, h, a.H, a.T, i0, len);
    const SwaKeyTiles kt(i0, i1, a.W, a.ns, BT);
    const float c2 = a.scale * kLog2e;
    for (int n = 0; n < kt.count; ++n) {
      const int j0 = kt.at(n) * BT;
      __syncthreads();
      // (the next tile on its way would take the second CTA of an SM: 2.0 for 1.75 ms at d = 128)
      load_tile<D>(sk, a.k, b, hk, a.Hk, a.T, j0, len);
      load_tile<D>(sv, a.v, b, hk, a.Hk, a.T, j0, len);
      __syncthreads();
      float s[4][4] = {};
      mm_nt<D>(s, sq, sk, ty, tx);
      __syncthreads();  // K has been read: P may take its place
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int qi = i0 + ty + 16 * i;
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int kj = j0 + tx + 16 * j;
          s[i][j] = (qi < len && swa_sees(qi, kj, a.W, a.ns)) ? s[i][j] * c2 : -INFINITY;
          mx = fmaxf(mx, s[i][j]);
        }
        const float mn = fmaxf(m[i], row_max(mx));
        const float ref = mn == -INFINITY ? 0.f : mn;  // a row that has seen nothing yet
        const float f = exp2f(m[i] - ref);
        m[i] = mn;
        l[i] *= f;
#pragma unroll
        for (int c = 0; c < NC; ++c) o[i][c] *= f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p = exp2f(s[i][j] - ref);
          l[i] += p;
          sp[(ty + 16 * i) * LP + tx + 16 * j] = p;
        }
      }
      __syncthreads();
      mm_nn<D>(o, sp, sv, ty, tx);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int qi = i0 + ty + 16 * i;
    const float ls = row_sum(l[i]);
    if (qi >= a.T) continue;
    const bool live = qi < len;
    const float inv = live ? 1.f / ls : 0.f;
    const size_t at = (((size_t)b * a.T + qi) * a.H + h) * D;
#pragma unroll
    for (int c = 0; c < NC; ++c) st<float>(a.o, at + col_of<D>(tx, c), live ? o[i][c] * inv : 0.f);
    if (a.lse && tx == 0)
      a.lse[((size_t)b * a.H + h) * a.T + qi] = live ? (m[i] + log2f(ls)) * kLn2 : -INFINITY;
  }
}

template <int D> constexpr int BWD_SMEM = (4 * BT * LD<D> + BT * LP + 2 * BT) * 4;

// dQ of a query tile: one pass over the keys that it sees.
template <int D> __global__ void __launch_bounds__(NT) k_swa_bwd_dq(const SwaArgs a) {
  extern __shared__ __align__(16) float sm[];
  float *sq = sm, *sg = sq + BT * LD<D>, *sk = sg + BT * LD<D>, *sv = sk + BT * LD<D>, *sd = sv + BT * LD<D>;
  constexpr int NC = D / 16;
  const int tid = threadIdx.x, ty = tid / 16, tx = tid % 16;
  const int b = blockIdx.z, h = blockIdx.y, hk = h / a.G, i0 = blockIdx.x * BT;
  const int len = swa_len(a, b), i1 = min(i0 + BT, len);
  float acc[4][NC] = {};
  if (i0 < len) {
    load_tile<D>(sq, a.q, b, h, a.H, a.T, i0, len);
    load_tile<D>(sg, a.dO, b, h, a.H, a.T, i0, len);
    const size_t row0 = ((size_t)b * a.H + h) * a.T;
    float nl[4], de[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int qi = i0 + ty + 16 * i;
      nl[i] = qi < len ? a.nlse[row0 + qi] : INFINITY;
      de[i] = qi < len ? a.delta[row0 + qi] : 0.f;
    }
    const SwaKeyTiles kt(i0, i1, a.W, a.ns, BT);
    const float c2 = a.scale * kLog2e;
    Fetch<D> fk, fv;
    fk.load(a.k, b, hk, a.Hk, a.T, kt.at(0) * BT, len);
    fv.load(a.v, b, hk, a.Hk, a.T, kt.at(0) * BT, len);
    for (int n = 0; n < kt.count; ++n) {
      const int j0 = kt.at(n) * BT;
      __syncthreads();
      fk.store(sk);
      fv.store(sv);
      __syncthreads();
      if (n + 1 < kt.count) {
        fk.load(a.k, b, hk, a.Hk, a.T, kt.at(n + 1) * BT, len);
        fv.load(a.v, b, hk, a.Hk, a.T, kt.at(n + 1) * BT, len);
      }
      float s[4][4] = {}, dp[4][4] = {};
      mm_nt<D>(s, sq, sk, ty, tx);
      mm_nt<D>(dp, sg, sv, ty, tx);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int qi = i0 + ty + 16 * i, kj = j0 + tx + 16 * j;
          const bool see = qi < len && swa_sees(qi, kj, a.W, a.ns);
          const float p = see ? exp2f(fmaf(s[i][j], c2, -nl[i])) : 0.f;
          sd[(ty + 16 * i) * LP + tx + 16 * j] = see ? p * (dp[i][j] - de[i]) : 0.f;
        }
      __syncthreads();
      mm_nn<D>(acc, sd, sk, ty, tx);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int qi = i0 + ty + 16 * i;
    if (qi >= a.T) continue;
    const size_t at = (((size_t)b * a.T + qi) * a.H + h) * D;
#pragma unroll
    for (int c = 0; c < NC; ++c) st<float>(a.dq, at + col_of<D>(tx, c), acc[i][c] * a.scale);
  }
}

// dK and dV of a split of a key tile: one pass over (query head of the group, query
// tile) pairs.  Thread (ty, tx) holds P^T and dS^T of keys ty + 16 i, queries tx + 16 j.
template <int D>
__global__ void __launch_bounds__(NT) k_swa_bwd_dkv(const SwaArgs a, const SwaSplits sp) {
  extern __shared__ __align__(16) float sm[];
  float *sk = sm, *sv = sk + BT * LD<D>, *sq = sv + BT * LD<D>, *sg = sq + BT * LD<D>, *st_ = sg + BT * LD<D>;
  float *snl = st_ + BT * LP, *sde = snl + BT;
  constexpr int NC = D / 16;
  const int tid = threadIdx.x, ty = tid / 16, tx = tid % 16;
  const int b = blockIdx.z, hk = blockIdx.y, x = blockIdx.x;
  const int nsx = sp.sink_tiles * sp.splits_sink;
  const int t = x < nsx ? x / sp.splits_sink : sp.sink_tiles + (x - nsx) / sp.splits;
  const int split = x < nsx ? x % sp.splits_sink : (x - nsx) % sp.splits;
  const int per = x < nsx ? sp.per_sink : sp.per;
  const int len = swa_len(a, b), j0 = t * BT;
  float dk[4][NC] = {}, dv[4][NC] = {};
  if (j0 < len) {
    int first, last;
    swa_query_tiles(t, BT, BT, a.W, a.ns, len, &first, &last);
    const int nq = last - first + 1;
    const int it1 = min((split + 1) * per, a.G * nq);
    const float c2 = a.scale * kLog2e;
    load_tile<D>(sk, a.k, b, hk, a.Hk, a.T, j0, len);
    load_tile<D>(sv, a.v, b, hk, a.Hk, a.T, j0, len);
    Fetch<D> fq, fg;
    float row_nl, row_de;
    auto fetch = [&](int it) {
      const int h = hk * a.G + it / nq, i0 = (first + it % nq) * BT;
      fq.load(a.q, b, h, a.H, a.T, i0, len);
      fg.load(a.dO, b, h, a.H, a.T, i0, len);
      const size_t row0 = ((size_t)b * a.H + h) * a.T;
      row_nl = tid < BT && i0 + tid < len ? a.nlse[row0 + i0 + tid] : INFINITY;
      row_de = tid < BT && i0 + tid < len ? a.delta[row0 + i0 + tid] : 0.f;
    };
    if (split * per < it1) fetch(split * per);
    for (int it = split * per; it < it1; ++it) {
      const int i0 = (first + it % nq) * BT;
      __syncthreads();
      fq.store(sq);
      fg.store(sg);
      if (tid < BT) {
        snl[tid] = row_nl;
        sde[tid] = row_de;
      }
      __syncthreads();
      if (it + 1 < it1) fetch(it + 1);
      float s[4][4] = {}, dp[4][4] = {};
      mm_nt<D>(s, sk, sq, ty, tx);
      mm_nt<D>(dp, sv, sg, ty, tx);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int kj = j0 + ty + 16 * i, qc = tx + 16 * j, qi = i0 + qc;
          const bool see = qi < len && swa_sees(qi, kj, a.W, a.ns);
          s[i][j] = see ? exp2f(fmaf(s[i][j], c2, -snl[qc])) : 0.f;
          dp[i][j] = see ? s[i][j] * (dp[i][j] - sde[qc]) : 0.f;
          st_[(ty + 16 * i) * LP + qc] = s[i][j];
        }
      __syncthreads();
      mm_nn<D>(dv, st_, sg, ty, tx);
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) st_[(ty + 16 * i) * LP + tx + 16 * j] = dp[i][j];
      __syncthreads();
      mm_nn<D>(dk, st_, sq, ty, tx);
    }
  }
  if (x < sp.part_blocks) {
    float *part = a.part + (((size_t)b * a.Hk + hk) * sp.part_blocks + x) * (2 * BT * D);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int e = (ty + 16 * i) * D + col_of<D>(tx, c);
        part[e] = dk[i][c];
        part[BT * D + e] = dv[i][c];
      }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int kj = j0 + ty + 16 * i;
    if (kj >= a.T) continue;
    const size_t at = (((size_t)b * a.T + kj) * a.Hk + hk) * D;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      st<float>(a.dk, at + col_of<D>(tx, c), dk[i][c] * a.scale);
      st<float>(a.dv, at + col_of<D>(tx, c), dv[i][c]);
    }
  }
}

// A query that sees at most kNear keys; bfloat16 forms its delta from them.
constexpr int kNear = 64;
__device__ __forceinline__ bool near(int i, const SwaArgs &a) {
  return min(i + 1, a.W) + min(max(i + 1 - a.W, 0), a.ns) <= kNear;
}

// delta_i = sum_d o_id dO_id, and lse in log2 units.  Rows past the length get +inf, so
// that their weights are exp2(-inf) = 0.  LPR lanes share a row, 16 bytes each; a CTA
// takes 4 NT / LPR tokens of a head, so that its row sums leave in one run of memory.
// Reads 2 d elements a row: bandwidth.
template <typename DT, int LPR> __global__ void __launch_bounds__(NT) k_swa_prep(const SwaArgs a) {
  let_next_start();
  constexpr int V = 16 / (int)sizeof(DT), RPP = NT / LPR, PASSES = 4;
  const int b = blockIdx.z, h = blockIdx.y, len = swa_len(a, b);
  const int ln = threadIdx.x % LPR, t0 = blockIdx.x * RPP * PASSES + threadIdx.x / LPR;
  if (blockIdx.x + blockIdx.y + blockIdx.z == 0 && threadIdx.x == 0) *a.status = 0;
  uint4 x[PASSES], y[PASSES];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int t = t0 + p * RPP;
    const size_t at = (((size_t)b * a.T + t) * a.H + h) * LPR + ln;
    x[p] = t < len ? static_cast<const uint4 *>(a.o)[at] : make_uint4(0, 0, 0, 0);
    y[p] = t < len ? static_cast<const uint4 *>(a.dO)[at] : make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int t = t0 + p * RPP;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < V; ++e) s = fmaf(ld<DT>(&x[p], e), ld<DT>(&y[p], e), s);
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (ln == 0 && t < a.T) {
      const size_t out = ((size_t)b * a.H + h) * a.T + t;
      a.nlse[out] = t < len ? a.lse[out] * kLog2e : INFINITY;
      if (sizeof(DT) == 4 || t >= len || !near(t, a)) a.delta[out] = s;
    }
  }
  if (sizeof(DT) == 2) end_after_previous();  // k_swa_near
}

// delta of queries that see at most kNear keys (k_swa_prep, beside it, leaves them out), from the keys: sum_j P_ij dP_ij.  The
// stored o is rounded to bfloat16, and where it averages few values that rounding weighs
// as much as the gradients' own (two tokens of d = 64: dk 5.1e-3 off, against 1.7e-3).
// Far rows keep sum_d o dO: there it is 3 % of the error.  Only the first 64 queries of a
// sequence are near, unless the window itself is.
//
// A CTA takes 16 queries, its four warps every fourth group of eight keys; S and dP are
// m16n8k16 products of rows as they lie in memory (exact products, float32 sums).  Lane
// c = lane % 4 of a row holds channels 32 m + 8 c .. + 7: the products sum over the
// channels in that order, the same for both operands, so that every load is 16 bytes.
__device__ __forceinline__ void mma_near(float *c, const uint32_t *a, const uint32_t *b) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}

template <int D> __global__ void __launch_bounds__(128) k_swa_near(const SwaArgs a) {
  constexpr int M = D / 32;  // 16-byte loads of a lane for a row
  let_next_start();
  __shared__ float part[4][16];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, b = blockIdx.z, h = blockIdx.y, hk = h / a.G;
  const int i0 = blockIdx.x * 16, len = swa_len(a, b);
  if (i0 >= len || !near(i0, a)) return;
  const int r = lane >> 2, c = lane & 3, last = min(i0 + 15, len - 1);
  uint4 q[M][2], g[M][2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const size_t at = (((size_t)b * a.T + min(i0 + r + 8 * e, last)) * a.H + h) * (D / 8) + c;
#pragma unroll
    for (int m = 0; m < M; ++m) {
      q[m][e] = static_cast<const uint4 *>(a.q)[at + 4 * m];
      g[m][e] = static_cast<const uint4 *>(a.dO)[at + 4 * m];
    }
  }
  const size_t row0 = ((size_t)b * a.H + h) * a.T;
  const float nl[2] = {a.lse[row0 + min(i0 + r, last)] * kLog2e, a.lse[row0 + min(i0 + r + 8, last)] * kLog2e};
  const float c2 = a.scale * kLog2e;
  const SwaKeyTiles kt(i0, last + 1, a.W, a.ns, 8);
  float de[2] = {0.f, 0.f};
#pragma unroll 2
  for (int n = warp; n < kt.count; n += 4) {
    const int j0 = kt.at(n) * 8;
    const size_t at = (((size_t)b * a.T + min(j0 + r, len - 1)) * a.Hk + hk) * (D / 8) + c;
    uint4 kf[M], vf[M];
#pragma unroll
    for (int m = 0; m < M; ++m) {
      kf[m] = static_cast<const uint4 *>(a.k)[at + 4 * m];
      vf[m] = static_cast<const uint4 *>(a.v)[at + 4 * m];
    }
    float s[4] = {}, dp[4] = {};
#pragma unroll
    for (int m = 0; m < M; ++m) {  // the two 8-byte halves of a load: a product each
      const uint32_t q0[4] = {q[m][0].x, q[m][1].x, q[m][0].y, q[m][1].y};
      const uint32_t q1[4] = {q[m][0].z, q[m][1].z, q[m][0].w, q[m][1].w};
      const uint32_t g0[4] = {g[m][0].x, g[m][1].x, g[m][0].y, g[m][1].y};
      const uint32_t g1[4] = {g[m][0].z, g[m][1].z, g[m][0].w, g[m][1].w};
      const uint32_t k0[2] = {kf[m].x, kf[m].y}, k1[2] = {kf[m].z, kf[m].w};
      const uint32_t v0[2] = {vf[m].x, vf[m].y}, v1[2] = {vf[m].z, vf[m].w};
      mma_near(s, q0, k0);
      mma_near(s, q1, k1);
      mma_near(dp, g0, v0);
      mma_near(dp, g1, v1);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = i0 + r + (e >> 1) * 8, j = j0 + 2 * c + (e & 1);
      if (i <= last && swa_sees(i, j, a.W, a.ns))
        de[e >> 1] = fmaf(exp2f(fmaf(s[e], c2, -nl[e >> 1])), dp[e], de[e >> 1]);
    }
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    de[e] += __shfl_xor_sync(0xffffffffu, de[e], 1);
    de[e] += __shfl_xor_sync(0xffffffffu, de[e], 2);
    if (c == 0) part[warp][r + 8 * e] = de[e];
  }
  __syncthreads();
  const int i = i0 + threadIdx.x;
  if (threadIdx.x < 16 && i <= last && near(i, a))
    a.delta[row0 + i] = (part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x]);
}

// dk, dv of split key tiles: their partial sums added in split order, four channels a
// thread.  Bound by reading the partial sums.
template <typename DT> __global__ void __launch_bounds__(NT) k_swa_join(const SwaArgs a, const SwaSplits sp, int BN) {
  const int d4 = a.d / 4, chunks = BN * d4 / NT;  // NT divides BN d / 4
  const int b = blockIdx.z, hk = blockIdx.y, t = blockIdx.x / chunks;
  const int e = (blockIdx.x % chunks) * NT + threadIdx.x, row = e / d4, j = t * BN + row;
  const bool sink = t < sp.sink_tiles;
  const int n = sink ? sp.splits_sink : sp.splits, per = sink ? sp.per_sink : sp.per;
  const int x0 = sink ? t * n : sp.sink_tiles * sp.splits_sink + (t - sp.sink_tiles) * n;
  const int len = swa_len(a, b);
  const size_t half = (size_t)BN * d4;
  const float4 *part = reinterpret_cast<const float4 *>(a.part) +
                       (((size_t)b * a.Hk + hk) * sp.part_blocks + x0) * 2 * half + e;
  if (j >= a.T) return;
  float4 k = make_float4(0.f, 0.f, 0.f, 0.f), v = k;
  if (j < len)
#pragma unroll 4
    for (int s = 0; s < n; ++s) {
      if (row >= swa_split_rows(t, s, per, BN, a.W, a.ns, a.G, len)) continue;
      const float4 x = part[2 * s * half], y = part[(2 * s + 1) * half];
      k.x += x.x; k.y += x.y; k.z += x.z; k.w += x.w;
      v.x += y.x; v.y += y.y; v.z += y.z; v.w += y.w;
    }
  const size_t at = (((size_t)b * a.T + j) * a.Hk + hk) * a.d + 4 * (e % d4);
  const float kk[4] = {k.x, k.y, k.z, k.w}, vv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    st<DT>(a.dk, at + c, kk[c] * a.scale);
    st<DT>(a.dv, at + c, vv[c]);
  }
}

// Copies the tokens of a prompt that decode still sees into the cache's slots:
// token t < s to slot t, later ones to slot s + (t - s) mod W, the newest W of them.
// Slots that no token of the prompt belongs to are left as they are.
__global__ void __launch_bounds__(NT) k_swa_cache_fill(const SwaArgs a, uint4 *kc, uint4 *vc, int v16) {
  const int b = blockIdx.z, hk = blockIdx.y, len = swa_len(a, b);
  const size_t S = (size_t)a.W + a.ns;
  const size_t n = (size_t)min((long long)len, (long long)S) * v16;  // filled slots come first
  for (size_t e = (size_t)blockIdx.x * NT + threadIdx.x; e < n; e += (size_t)gridDim.x * NT) {
    const int slot = (int)(e / v16), c = (int)(e % v16);
    // the newest token of the slot: the last t < len with (t - s) mod W = slot - s
    const int t = slot < a.ns ? slot : slot + (len - 1 - slot) / a.W * a.W;
    const size_t from = (((size_t)b * a.T + t) * a.Hk + hk) * v16 + c;
    const size_t to = (((size_t)b * a.Hk + hk) * S + slot) * v16 + c;
    kc[to] = static_cast<const uint4 *>(a.k)[from];
    vc[to] = static_cast<const uint4 *>(a.v)[from];
  }
}

// One token over the cache: 8 lanes a key (d / 8 channels each), 32 keys at a time in
// the CTA's 8 warps and two of them under way, a running softmax per group of lanes,
// joined through shared memory.  A CTA, or a cluster of them that splits the slots,
// serves one query head; the group's first head writes the new token into its slot, and
// every head takes that slot's row from the inputs.
template <int D>
__global__ void __launch_bounds__(NT) k_swa_decode(const SwaArgs a, void *kc, void *vc, const int *pos) {
  constexpr int E = D / 8, GR = NT / 8, U = 2;
  __shared__ float s_m[GR], s_l[GR], s_o[GR][D], s_part[D + 2];
  cg::cluster_group cluster = cg::this_cluster();
  const int C = gridDim.x, rank = blockIdx.x;  // the cluster is the x axis of the grid
  const int tid = threadIdx.x, gr = tid / 8, ln = tid % 8;
  const int h = blockIdx.y, b = blockIdx.z, hk = h / a.G;
  const int p = pos[b];
  const size_t out = ((size_t)b * a.H + h) * D;
  if (p < 0) {  // an idle sequence (the whole cluster leaves)
    if (rank == 0 && tid < D) st<float>(a.o, out + tid, 0.f);
    return;
  }
  const size_t S = (size_t)a.W + a.ns;
  const int slot = p < a.ns ? p : a.ns + (p - a.ns) % a.W;
  const int n = (int)min((long long)p + 1, (long long)S);
  const size_t base = ((size_t)b * a.Hk + hk) * S * D, in = ((size_t)b * a.Hk + hk) * D;
  if (h % a.G == 0 && rank == 0 && tid < D) {
    static_cast<float *>(kc)[base + (size_t)slot * D + tid] = static_cast<const float *>(a.k)[in + tid];
    static_cast<float *>(vc)[base + (size_t)slot * D + tid] = static_cast<const float *>(a.v)[in + tid];
  }
  // lane's channels: E / 4 runs of four, 32 apart
  const float c2 = a.scale * kLog2e;
  float q[E], o[E], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    q[e] = ld<float>(a.q, out + 32 * (e / 4) + 4 * ln + e % 4) * c2;
    o[e] = 0.f;
  }
  for (int j0 = rank * U * GR; j0 < n; j0 += C * U * GR) {  // the same trip count for every lane
    float s[U], v[U][E];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * GR + gr;
      const bool live = j < n;
      const void *kp = j == slot ? a.k : kc, *vp = j == slot ? a.v : vc;
      const size_t at = j == slot ? in : base + (size_t)(live ? j : 0) * D;
      s[u] = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const size_t x = at + 32 * (e / 4) + 4 * ln + e % 4;
        s[u] = fmaf(q[e], live ? ld<float>(kp, x) : 0.f, s[u]);
        v[u][e] = live ? ld<float>(vp, x) : 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int w = 4; w > 0; w >>= 1) s[u] += __shfl_xor_sync(0xffffffffu, s[u], w);
      if (j0 + u * GR + gr >= n) continue;
      const float mn = fmaxf(m, s[u]), f = exp2f(m - mn), pr = exp2f(s[u] - mn);
      m = mn;
      l = fmaf(l, f, pr);
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = fmaf(o[e], f, pr * v[u][e]);
    }
  }
  if (ln == 0) { s_m[gr] = m; s_l[gr] = l; }
#pragma unroll
  for (int e = 0; e < E; ++e) s_o[gr][32 * (e / 4) + 4 * ln + e % 4] = o[e];
  __syncthreads();
  // a group (or a CTA) without keys has m = -inf and l = 0
  auto factor = [](float x, float ref) { return x == -INFINITY ? 0.f : exp2f(x - ref); };
  if (tid < D) {
    float mm = -INFINITY, ls = 0.f, x = 0.f;
    for (int g = 0; g < GR; ++g) mm = fmaxf(mm, s_m[g]);
    for (int g = 0; g < GR; ++g) {
      const float f = factor(s_m[g], mm);
      ls = fmaf(s_l[g], f, ls);
      x = fmaf(s_o[g][tid], f, x);
    }
    if (C == 1) st<float>(a.o, out + tid, x / ls);
    s_part[tid] = x;
    if (tid == 0) { s_part[D] = mm; s_part[D + 1] = ls; }
  }
  if (C == 1) return;
  cluster.sync();
  if (rank == 0 && tid < D) {
    float mm = -INFINITY, ls = 0.f, x = 0.f;
    for (int k = 0; k < C; ++k) mm = fmaxf(mm, cluster.map_shared_rank(s_part, k)[D]);
    for (int k = 0; k < C; ++k) {
      const float *r = cluster.map_shared_rank(s_part, k);
      const float f = factor(r[D], mm);
      ls = fmaf(r[D + 1], f, ls);
      x = fmaf(r[tid], f, x);
    }
    st<float>(a.o, out + tid, x / ls);
  }
  cluster.sync();  // no CTA leaves while another reads its part
}

kdn_status_t launched() { return cudaGetLastError() == cudaSuccess ? KDN_OK : KDN_ERR_CUDA; }

template <typename K> bool smem_ok(K kernel, int bytes) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess;
}

template <int D> kdn_status_t fwd_t(const SwaArgs &a, cudaStream_t s) {
  if (!smem_ok(k_swa_fwd<D>, FWD_SMEM<D>)) return KDN_ERR_CUDA;
  k_swa_fwd<D><<<dim3((a.T + BT - 1) / BT, a.H, a.B), NT, FWD_SMEM<D>, s>>>(a);
  return launched();
}

template <int D> kdn_status_t bwd_t(const SwaArgs &a, const SwaSplits &sp, cudaStream_t s) {
  if (!smem_ok(k_swa_bwd_dq<D>, BWD_SMEM<D>) || !smem_ok(k_swa_bwd_dkv<D>, BWD_SMEM<D>)) return KDN_ERR_CUDA;
  k_swa_bwd_dkv<D><<<dim3(sp.blocks, a.Hk, a.B), NT, BWD_SMEM<D>, s>>>(a, sp);
  k_swa_bwd_dq<D><<<dim3((a.T + BT - 1) / BT, a.H, a.B), NT, BWD_SMEM<D>, s>>>(a);
  return launched();
}

template <int D>
kdn_status_t dec_t(const SwaArgs &a, void *kc, void *vc, const int *pos, cudaStream_t s) {
  // CTAs of a cluster: enough for two an SM, with four rounds of 64 keys each at least
  int C = 1;
  while (C < 8 && (long long)a.B * a.H * C < 2 * 152 && (long long)a.W + a.ns > C * 256LL) C *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(C, a.H, a.B);
  cfg.blockDim = dim3(NT);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = C;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_swa_decode<D>, a, kc, vc, pos) == cudaSuccess ? KDN_OK : KDN_ERR_CUDA;
}

}  // namespace

kdn_status_t launch_swa_fwd_general(const SwaArgs &a, cudaStream_t s) {
  return a.d == 128 ? fwd_t<128>(a, s) : a.d == 64 ? fwd_t<64>(a, s) : fwd_t<32>(a, s);
}

kdn_status_t launch_swa_bwd_general(const SwaArgs &a, const SwaSplits &sp, cudaStream_t s) {
  return a.d == 128 ? bwd_t<128>(a, sp, s) : a.d == 64 ? bwd_t<64>(a, sp, s) : bwd_t<32>(a, sp, s);
}

kdn_status_t launch_swa_decode_general(const SwaArgs &a, void *kc, void *vc, const int *pos, cudaStream_t s) {
  return a.d == 128  ? dec_t<128>(a, kc, vc, pos, s)
         : a.d == 64 ? dec_t<64>(a, kc, vc, pos, s)
                     : dec_t<32>(a, kc, vc, pos, s);
}

template <int D> static kdn_status_t near_t(const SwaArgs &a, cudaStream_t s) {
  const int rows = (long long)a.W + a.ns <= kNear || a.T < kNear ? a.T : kNear;
  k_swa_near<D><<<dim3((rows + 15) / 16, a.H, a.B), 128, 0, s>>>(a);
  return launched();
}

kdn_status_t launch_swa_prep(const SwaArgs &a, cudaStream_t s) {
  const int lpr = a.d * (a.dtype == KDN_BF16 ? 2 : 4) / 16, rows = 4 * NT / lpr;
  const dim3 grid((a.T + rows - 1) / rows, a.H, a.B);
  if (a.dtype == KDN_BF16) {
    const kdn_status_t st = a.d == 128 ? near_t<128>(a, s) : a.d == 64 ? near_t<64>(a, s) : near_t<32>(a, s);
    if (st != KDN_OK) return st;
    return launch_beside(lpr == 16  ? k_swa_prep<__nv_bfloat16, 16>
                         : lpr == 8 ? k_swa_prep<__nv_bfloat16, 8>
                                    : k_swa_prep<__nv_bfloat16, 4>,
                         grid, NT, 0, s, a);
  }
  if (lpr == 32) k_swa_prep<float, 32><<<grid, NT, 0, s>>>(a);
  else if (lpr == 16) k_swa_prep<float, 16><<<grid, NT, 0, s>>>(a);
  else k_swa_prep<float, 8><<<grid, NT, 0, s>>>(a);
  return launched();
}

kdn_status_t launch_swa_join(const SwaArgs &a, const SwaSplits &sp, int BN, cudaStream_t s) {
  if (!sp.part_blocks) return KDN_OK;
  const dim3 grid((sp.splits > 1 ? sp.tiles : sp.sink_tiles) * (BN * a.d / 4 / NT), a.Hk, a.B);
  if (a.dtype == KDN_BF16) k_swa_join<__nv_bfloat16><<<grid, NT, 0, s>>>(a, sp, BN);
  else k_swa_join<float><<<grid, NT, 0, s>>>(a, sp, BN);
  return launched();
}

kdn_status_t launch_swa_cache_fill(const SwaArgs &a, void *kc, void *vc, cudaStream_t s) {
  const int v16 = a.d * (a.dtype == KDN_BF16 ? 2 : 4) / 16;
  const long long most = ((long long)a.W + a.ns < a.T ? (long long)a.W + a.ns : a.T) * v16;
  const unsigned gx = (unsigned)((most + 4 * NT - 1) / (4 * NT));
  k_swa_cache_fill<<<dim3(gx, a.Hk, a.B), NT, 0, s>>>(a, static_cast<uint4 *>(kc), static_cast<uint4 *>(vc), v16);
  return launched();
}

}  // namespace kdn
