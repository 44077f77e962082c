// kdn_ffn_tc.cu -- the products of the gated feed-forward block on the tensor cores (bfloat16).
//
// All products are C[m, n] = sum_k A(m, k) B(n, k), with either operand stored along k or along
// its own axis (a flag of the shared-memory descriptor).  Two CTAs of a cluster form a tile of
// 256 x BN: each loads its 128 rows of A and half of B's BN rows by TMA, one thread of the first
// issues the products of both (cta_group::2), and each keeps its 128 rows of the accumulator in
// its own TMEM.  Operand bytes a product are so a third less than with one CTA's 128 x 256.
//   GATE   B's halves are rows of Wg and of Wu: g and u of an element lie in one TMEM lane, and the
//          epilogue writes act(g) u (and g and u for the gradients).
//   DGATE  the accumulator is dh; the epilogue reads g and u and writes dg and du.
//   PLAIN  a sum over up to two pairs of operands (dx = dg Wg + du Wu), or up to three problems of one
//          launch (the weights' gradients), or parts of a K axis that leave float32 partial sums.
//
// Sums.  The tensor cores truncate what they add into an accumulator, always towards 0: of positive terms 7e-7 of the
// sum is lost after 512 along K, 4e-6 after 2048, 3e-5 after 8192, 1.6e-4 after 32768 (2^-25.4 to 2^-23.6 for every
// 16).  A float32 output's sum leaves the accumulator every 512 along K and is added, rounded to nearest, in the
// epilogue's registers, while the products go on in the second accumulator; so do partial sums of a bfloat16 output,
// every 4096.  A bfloat16 output that would take more than 65536 along K into one accumulator (3e-4, a sixth of half
// a step) goes through a float32 one.
//
// CTAs are persistent, one an SM; the accumulator is doubled, so that a tile's epilogue runs beside
// the next one's products.  Roles: warp 0 the loads, warp 1 the products, warps 4-11 the epilogue
// (32 rows each, columns halved); PLAIN's results go out through shared memory by TMA.
//
// The tensor cores bound it: 8192 tokens of 2048 x 5632 take 211 us in the gate (1.79 PFLOP/s, pipe 92 % active), 115
// in y, 148 in dh (61 %: g, u, dg and du pass beside the operands), 223 in dx and 303 in the weights' gradients (1.87).
#include "kdn_ffn_tc.cuh"

namespace kdn {
namespace {

using namespace ffn;

constexpr int THREADS = 384;
constexpr int A_BYTES = 128 * BK * 2, OUT_BYTES = 4096, EPI_WARPS = 8;
template <int BN> constexpr int STAGE = A_BYTES + BN / 2 * BK * 2;
// Shared memory of an epilogue warp: two blocks on their way out (PLAIN); three blocks of g and u, one at work
// and two on their way in (DGATE).
template <int EPI> constexpr int OUT = EPI_WARPS * OUT_BYTES * (EPI == PLAIN ? 2 : EPI == DGATE ? 3 : 0);
template <int BN, int EPI> constexpr int STAGES = (224 * 1024 - OUT<EPI>) / STAGE<BN>;
template <int BN, int EPI> constexpr int SMEM = STAGES<BN, EPI> * STAGE<BN> + OUT<EPI> + 1024 + 512;

struct Work {
  CUtensorMap maps[9];  // PLAIN: of each problem C, A, B; else A, B, and B of u
  Problem p[3];
  int nmaps, np, tiles;
  int am, bm;           // A and B are stored along their own axes
  int keep;             // B is a weight matrix that L2 has room for
  int ks;               // 16s along K that a step loads and multiplies: 4, fewer where K ends before (both own)
  int chunk;            // SUMS: steps of a sum between two additions into registers
  int act;
  bf *out[3];           // GATE: g, u (null: not written), h; DGATE: dg, du
  const bf *in[2];      // DGATE: g, u
  int wide;             // GATE: the outputs' rows start on 32 bytes
  int first;            // the call's first kernel: it clears the status word
  unsigned *status;
};

template <int BN, int EPI> __device__ __forceinline__ Tile tile_of(const Work &w, int t) {
  return tile_at(w.p, w.np, EPI == GATE ? BN / 2 : BN, t);
}

// What is read once (or by CTAs that run together) leaves L2 first; weights, which every row block reads, stay.
__device__ __forceinline__ uint64_t leaves_first() {
  uint64_t policy;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  return policy;
}
__device__ __forceinline__ uint64_t stays() {
  uint64_t policy;
  asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(policy));
  return policy;
}
__device__ __forceinline__ uint64_t no_preference() {
  uint64_t policy;
  asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
  return policy;
}
// into this CTA's shared memory, counted at a barrier of the pair
__device__ __forceinline__ void load_2d(void *dst, const CUtensorMap *map, uint32_t bar, int c0, int c1,
                                        uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2.L2::cache_hint"
      " [%0], [%1, {%2, %3}], [%4], %5;" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(bar), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void store_3d(const CUtensorMap *map, const void *src, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(
                   reinterpret_cast<uint64_t>(map)),
               "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(src))
               : "memory");
}
// 32 columns of one row of a staged block (rows of 128 bytes, swizzled as TMA takes them), from chunk `first` on
__device__ __forceinline__ void stage32(unsigned char *buf, int row, int first, const float *x) {
#pragma unroll
  for (int c = 0; c < 4; ++c) sm16(buf, chunk_off(row, first + c)) = fused::pack_bf8(x + 8 * c);
}
__device__ __forceinline__ void stage_f32(unsigned char *buf, int row, const float *x) {
#pragma unroll
  for (int c = 0; c < 8; ++c)
    *reinterpret_cast<float4 *>(buf + chunk_off(row, c)) = *reinterpret_cast<const float4 *>(x + 4 * c);
}

// 32 consecutive columns of a thread's own row, the first `n` of them (a multiple of 8): whole 32-byte sectors
// where rows are aligned to them.  (By TMA they would stand in the way of the operands' copies: it takes
// about two cycles for a row of a box, and the products waited another tenth of the time.)
__device__ __forceinline__ void store_row(__nv_bfloat16 *p, const float *x, int n, bool wide) {
  uint4 v[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) v[c] = fused::pack_bf8(x + 8 * c);
#pragma unroll
  for (int c = 0; c < 4; c += 2) {
    if (wide && 8 * c + 16 <= n) {
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p + 8 * c), "r"(v[c].x), "r"(v[c].y),
                   "r"(v[c].z), "r"(v[c].w), "r"(v[c + 1].x), "r"(v[c + 1].y), "r"(v[c + 1].z), "r"(v[c + 1].w)
                   : "memory");
    } else {
      if (8 * c < n) *reinterpret_cast<uint4 *>(p + 8 * c) = v[c];
      if (8 * c + 8 < n) *reinterpret_cast<uint4 *>(p + 8 * c + 8) = v[c + 1];
    }
  }
}

// A block of 32 rows x 32 columns of bfloat16 in shared memory: chunk c of 16 bytes of a row, so that 8 rows of
// one chunk and 2 rows of all four lie in different banks.
__device__ __forceinline__ uint32_t block_off(int row, int c) { return row * 64 + ((c ^ (row >> 1 & 3)) << 4); }
__device__ __forceinline__ void copy_async(void *dst, const void *src, bool live, uint64_t policy) {  // 16 bytes, or zeros
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(smem_u32(dst)), "l"(src),
               "r"(live ? 16 : 0), "l"(policy)
               : "memory");
}

// SUMS: a tile's sum is longer than a chunk.  (A form of its own: its registers leave less room to the kernel that
// starts beside it, 256 tokens of 2048 x 5632 30.5 us with it and 30.0 without.)
template <int BN, int EPI, bool F32, bool SUMS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1) k_ffn_tc(const __grid_constant__ Work w) {
  constexpr int NS = STAGES<BN, EPI>, SB = STAGE<BN>;
  extern __shared__ unsigned char smraw[];
  unsigned char *sm =
      reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smraw) + 1023) & ~uintptr_t(1023));
  unsigned char *stage_out = sm + NS * SB;
  uint64_t *full = reinterpret_cast<uint64_t *>(stage_out + OUT<EPI>);
  uint64_t *empty = full + NS, *acc_full = empty + NS, *acc_empty = acc_full + 2;
  uint32_t *s_tmem = reinterpret_cast<uint32_t *>(acc_empty + 2);
  int *s_fail = reinterpret_cast<int *>(s_tmem + 1);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  if (tid == 0) {
    for (int i = 0; i < NS; ++i) {
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
  if (warp == 2) tmem_alloc_pair(s_tmem, 2 * BN);
  if (warp == 3 && lane < w.nmaps) prefetch_tmap(w.maps + lane);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  let_next_start();
  const uint32_t tb = *s_tmem;
  const Waiter wait{s_fail, w.status};
  wait_for_previous();
  // (a wait runs out seconds after the launch, whose first block this is)
  if (w.first && blockIdx.x == 0 && tid == 0) *w.status = 0;

  // The loops of the two threads below are what a step takes at least: whatever does not change from step to step
  // stays in registers, and the next barrier is looked at ahead.  (With the tile's numbers read from the parameters and
  // stages counted by division the loading thread took 500 cycles a step, as long as its products.)
  if (warp == 0) {  // ------------------------------------------------------- loads
    if (elect_one()) {
      // (rows whose tiles all run at once are read once)
      const uint64_t pa = w.keep && w.p[0].tn * 8 <= PAIRS ? leaves_first() : no_preference();
      const uint64_t pb = w.keep ? stays() : no_preference();
      const bool am = w.am, bm = w.bm;
      const uint32_t bytes = 2 * SB / 4 * w.ks;
      const uint32_t bars = in_cta(full, 0);
      int st = 0, n = 0;      // stage, steps so far
      uint32_t turn = 1;      // (a barrier's phase before its first counts as complete)
      bool ok = true, ready = true;
      for (int t = pair; ok && t < w.tiles; t += pairs) {
        const Tile T = tile_of<BN, EPI>(w, t);
        const int m = T.m + 128 * (int)rank, c = EPI == GATE ? T.n : T.n + BN / 2 * (int)rank, s0 = T.p->steps[0];
        for (int k = T.k0; ok && k < T.k1;) {
          const int seg = k >= s0, end = seg ? T.k1 : min(s0, T.k1);
          const CUtensorMap *ma = w.maps + T.p->a[seg], *mb = w.maps + T.p->b[EPI == GATE ? rank : seg];
          for (int kk = (k - (seg ? s0 : 0)) * BK; k < end; ++k, ++n, kk += BK) {
            if (!ready && !(ok = wait(empty + st, turn))) break;
            unsigned char *sa = sm + st * SB, *sb = sa + A_BYTES;
            const uint32_t bar = bars + 8 * st;
            if (rank == 0) mbar_expect_tx(full + st, bytes);
            if (++st == NS) {
              st = 0;
              turn ^= 1;
            }
            ready = mbar_try_wait(empty + st, turn);
            if (am) {
              load_2d(sa, ma, bar, m, kk, pa);
              load_2d(sa + 8192, ma, bar, m + 64, kk, pa);
            } else {
              load_2d(sa, ma, bar, kk, m, pa);
            }
            if (bm) {
#pragma unroll
              for (int s = 0; s < BN / 128; ++s) load_2d(sb + s * 8192, mb, bar, c + 64 * s, kk, pb);
            } else {
              load_2d(sb, mb, bar, kk, c, pb);
            }
          }
        }
      }
      // what the pair still copies and signals arrives before its CTAs leave
      for (int m = max(0, n - NS); m < n; ++m) {
        if (!ok && rank == 0) mbar_wait(full + m % NS, (m / NS) & 1, kWait >> 6);
        if (ok) ok = wait.lazy(empty + m % NS, (m / NS) & 1);
      }
    }
  } else if (warp == 1) {  // ------------------------------------------------ products
    if (rank == 0 && elect_one()) {
      const uint32_t id = idesc_bf16(256, BN, w.am, w.bm);
      const uint32_t base = smem_u32(sm);
      const uint64_t da = sw128_desc(base, w.am ? 8192 : 16, 1024);
      const uint64_t db = sw128_desc(base + A_BYTES, w.bm ? 8192 : 16, 1024);
      const uint64_t ka = (w.am ? 2048 : 32) >> 4, kb = (w.bm ? 2048 : 32) >> 4;
      const int ks = w.ks;
      int st = 0;
      uint32_t turn = 0, acc = 0, acc_turn = 1;
      bool ok = true;
      for (int t = pair; ok && t < w.tiles; t += pairs) {
        const Tile T = tile_of<BN, EPI>(w, t);
        for (int left = T.k1 - T.k0; left > 0;) {
          const int some = SUMS ? min(left, w.chunk) : left;
          left -= some;
          if (!(ok = wait(acc_empty + acc, acc_turn))) break;
          tc_fence_after();
          const uint32_t d = tb + acc * BN;
          uint32_t more = 0;
          bool ready = false;
          for (int k = some; k > 0; --k) {
            if (!ready && !(ok = wait(full + st, turn))) break;
            uint64_t *const bar = empty + st;
            const uint64_t a = da + st * (SB >> 4), b = db + st * (SB >> 4);
            if (++st == NS) {
              st = 0;
              turn ^= 1;
            }
            umma_pair(d, a, b, id, more);
            if (ks > 1) umma_pair(d, a + ka, b + kb, id, 1);
            ready = k > 1 && mbar_try_wait(full + st, turn);
            if (ks > 2) umma_pair(d, a + 2 * ka, b + 2 * kb, id, 1);
            if (ks > 3) umma_pair(d, a + 3 * ka, b + 3 * kb, id, 1);
            commit_pair(bar);
            more = 1;
          }
          if (!ok) break;
          commit_pair(acc_full + acc);
          if (acc ^= 1, acc == 0) acc_turn ^= 1;
        }
      }
    }
  } else if (warp >= 4) {  // ------------------------------------------------ epilogue
    constexpr int COLS = F32 ? 32 : 64;                  // of a staged block
    constexpr int HALF = EPI == GATE ? BN / 4 : BN / 2;  // columns of a warp
    const int e = warp - 4, q = warp & 3, half = e >> 2;
    unsigned char *const bufs = stage_out + e * (OUT<EPI> / EPI_WARPS);
    const uint32_t lanes = (uint32_t)(32 * q) << 16;
    // DGATE: block c of tile number t, where four lanes hold a row's 64 bytes and a warp eight rows at a time:
    // f(place in the block, place in the matrix, whether it is one)
    constexpr int BLOCKS = HALF / 32;
    auto each = [&](int t, int c, auto f) {
      const Tile T = tile_of<BN, EPI>(w, t);
      const int m = T.m + 128 * (int)rank + 32 * q + (lane >> 2), n = T.n + half * HALF + 32 * c + 8 * (lane & 3);
      const size_t at = (size_t)m * T.p->N + n;
#pragma unroll
      for (int r = 0; r < 32; r += 8)
        f(block_off((lane >> 2) + r, lane & 3), at + (size_t)r * T.p->N, m + r < T.p->M && n < T.p->N);
    };
    const uint64_t policy = leaves_first();
    auto fetch = [&](int t, int c, int set) {  // g and u of a block, as a group of copies (of nothing behind the end)
      if (t < w.tiles)
        each(t, c, [&](uint32_t to, size_t at, bool live) {
          unsigned char *b = bufs + set * OUT_BYTES + to;
          copy_async(b, live ? w.in[0] + at : w.in[0], live, policy);
          copy_async(b + OUT_BYTES / 2, live ? w.in[1] + at : w.in[1], live, policy);
        });
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int block = 0;
    if (EPI == DGATE)
      for (int c = 0; c < 2; ++c) fetch(pair, c, c);
    int i = 0, sent = 0;  // accumulators read, blocks sent
    for (int t = pair; t < w.tiles; t += pairs) {
      const Tile T = tile_of<BN, EPI>(w, t);
      const int acc = i & 1;
      const uint32_t ta = tb + acc * BN + half * HALF + lanes;
      // PLAIN: a block of COLS columns from c on, which `write` puts into a buffer, goes out
      auto send = [&](int c, auto write) {
        unsigned char *b = bufs + (sent++ & 1) * OUT_BYTES;  // whose last store but one has left it
        if (lane == 0) bulk_wait_read_but1();
        __syncwarp();
        write(b);
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          const int m = T.m + 128 * (int)rank + 32 * q, n = T.n + half * HALF + c;
          if (m < T.p->M && n < T.p->N) store_3d(w.maps + T.p->out, b, n, m, T.split);
          bulk_commit();  // (a group of nothing too: they are counted)
        }
      };
      if constexpr (SUMS) {
        float x[HALF];
#pragma unroll
        for (int j = 0; j < HALF; ++j) x[j] = 0.f;
#pragma unroll 1
        for (int k = T.k0; k < T.k1; k += w.chunk, ++i) {
          const int acc = i & 1;
          const bool last = k + w.chunk >= T.k1;
          wait_quietly(wait, acc_full + acc, (i / 2) & 1);
          tc_fence_after();
#pragma unroll
          for (int c = 0; c < HALF; c += 32) {
#pragma unroll
            for (int h = c; h < c + 32; h += 16) {
              float y[16];
              tmem_ld16(tb + acc * BN + half * HALF + lanes + h, y);
#pragma unroll
              for (int j = 0; j < 16; ++j) x[h + j] += y[j];
            }
            if (last) send(c, [&](unsigned char *b) { stage_f32(b, lane, x + c); });
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_at(in_cta(acc_empty + acc, 0));
        }
        continue;
      }
      wait_quietly(wait, acc_full + acc, (i++ / 2) & 1);
      tc_fence_after();
      if (EPI == PLAIN) {
#pragma unroll 1
        for (int c = 0; c < HALF; c += COLS) {
          float x[COLS];
#pragma unroll
          for (int j = 0; j < COLS; j += 32) tmem_ld32(ta + c + j, x + j);
          send(c, [&](unsigned char *b) {
            tmem_ld_wait<COLS>(x);
            if (F32) {
              stage_f32(b, lane, x);
            } else {
#pragma unroll
              for (int j = 0; j < COLS; j += 32) stage32(b, lane, j / 8, x + j);
            }
          });
        }
      } else if (EPI == GATE) {
#pragma unroll 1
        for (int c = 0; c < HALF / 32; ++c) {
          float g[32], u[32];
          tmem_ld32(ta + c * 32, g);
          tmem_ld32(ta + BN / 2 + c * 32, u);
          const int m = T.m + 128 * (int)rank + 32 * q + lane, n = T.n + half * HALF + 32 * c;
          const int cols = m < T.p->M ? T.p->N - n : 0;
          const size_t at = (size_t)m * T.p->N + n;
          tmem_ld_wait<32>(g);
          pin32(u);
          if (w.out[0]) {
            store_row(w.out[0] + at, g, cols, w.wide);
            store_row(w.out[1] + at, u, cols, w.wide);
          }
          gate_values<32>(w.act, g, u);
          store_row(w.out[2] + at, g, cols, w.wide);
        }
      } else {  // DGATE: a block is worked on in place; two more are on their way
#pragma unroll 1
        for (int c = 0; c < BLOCKS; ++c, ++block) {
          float x[32];
          tmem_ld32(ta + c * 32, x);
          unsigned char *const bg = bufs + block % 3 * OUT_BYTES, *const bu = bg + OUT_BYTES / 2;
          asm volatile("cp.async.wait_group 1;" ::: "memory");
          __syncwarp();
          // (into the set of the block before, which every lane has left)
          fetch(c + 2 < BLOCKS ? t : t + pairs, c + 2 < BLOCKS ? c + 2 : c + 2 - BLOCKS, (block + 2) % 3);
          tmem_ld_wait<32>(x);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint4 &pg = sm16(bg, block_off(lane, k)), &pu = sm16(bu, block_off(lane, k));
            float g[8], u[8];
            fused::unpack_bf8(pg, g);
            fused::unpack_bf8(pu, u);
            hidden_gradients<8>(w.act, x + 8 * k, g, u);
            pg = fused::pack_bf8(g);
            pu = fused::pack_bf8(u);
          }
          __syncwarp();
          each(t, c, [&](uint32_t from, size_t at, bool live) {
            if (!live) return;
            *reinterpret_cast<uint4 *>(w.out[0] + at) = sm16(bg, from);
            *reinterpret_cast<uint4 *>(w.out[1] + at) = sm16(bu, from);
          });
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_at(in_cta(acc_empty + acc, 0));
    }
    if (EPI == PLAIN && lane == 0) bulk_wait_all();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // neither CTA leaves while the other may reach into it
  tc_fence_after();
  if (warp == 2) tmem_dealloc_pair(tb, 2 * BN);
}

// ----------------------------------------------------------------------- host

// How a product is cut: columns of a tile, and parts of its K axis.  In units of a K step of a 256 x 256 tile
// (0.27 us at 1.9 GHz): a step of 256 x 128 takes 0.75 of it (its operands' way into the SM bounds it: 256 rows of
// 2048 x 5632, y by whole K axes 29 and 23 us), a tile's start and end 3 and 2, partial sums 14 and their traffic.
struct Cut {
  int BN, splits;
};
double cost(long long M, long long N, int steps, int problems, int BN, int splits, bool gate) {
  const double tiles = (double)cut(M, 256) * cut(N, gate ? BN / 2 : BN) * problems * splits;
  const double waves = (double)(long long)((tiles + PAIRS - 1) / PAIRS);
  double c = waves * (((steps + splits - 1) / splits) * (BN == 256 ? 1 : 0.75) + (BN == 256 ? 3 : 2)) + 5;
  if (splits > 1) c += 14 + (double)M * N * problems * (splits * 8 + 2) / 1.4e6;
  return c;
}
Cut choose(long long M, long long N, int steps, int problems, bool may_split, bool gate) {
  Cut best{256, 1};
  double least = cost(M, N, steps, problems, 256, 1, gate);
  for (int BN = 256; BN >= 128; BN /= 2)
    for (int s = 1; s <= (may_split ? 16 : 1) && steps >= 4 * s; ++s) {
      const double c = cost(M, N, steps, problems, BN, s, gate);
      if (c < 0.97 * least) {
        least = c;
        best = {BN, s};
      }
    }
  return best;
}

// Steps of a sum that one accumulator takes: of a float32 output, of a float32 part of a bfloat16 one, of a bfloat16
// one.  (Of the first every 4, 8 and 16: the backward pass of 32768 tokens of 2048 x 5632 3190, 2620 and 2620 us, where
// bfloat16 gradients of weights take 2500; 3e-7, 7e-7 and 1.7e-6 of a sum of positive terms lost.)
constexpr int OUT_CHUNK = 8, PART_CHUNK = 64, LONGEST = 1024;
// Steps of a part, at most.
int steps_of(const Spec &S, const Cut c) { return cut(S.sums * (long long)cut(S.K, BK), c.splits); }
// Whether a product goes through float32 parts (a single one where a bfloat16 output's sum is too long).
bool in_parts(const Spec &S, const Cut c) { return c.splits > 1 || (!S.out_f32 && steps_of(S, c) > LONGEST); }

// Half of L2, of which each of two dies may hold a copy.
bool keeps(long long weights) { return weights * 2 <= 63LL << 20; }

template <int BN, int EPI, bool F32 = false, bool SUMS = false> kdn_status_t launch(const Work &w, cudaStream_t s) {
  auto kernel = k_ffn_tc<BN, EPI, F32, SUMS>;
  static std::atomic<unsigned long long> done{0};
  const kdn_status_t st = once_a_device(done, [&] {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM<BN, EPI>) == cudaSuccess;
  });
  if (st != KDN_OK) return st;
  const int grid = 2 * (w.tiles < PAIRS ? w.tiles : PAIRS);
  return launch_beside(kernel, dim3(grid), THREADS, SMEM<BN, EPI>, s, w);
}

template <int BN> kdn_status_t launch_plain(const Work &w, bool f32, bool sums, cudaStream_t s) {
  if (sums) return launch<BN, PLAIN, true, true>(w, s);
  return f32 ? launch<BN, PLAIN, true>(w, s) : launch<BN, PLAIN>(w, s);
}

kdn_status_t plain(const Spec &S, const Cut c, float *part, unsigned *status, bool first, cudaStream_t s) {
  Work w{};
  w.am = S.a[0].own;
  w.bm = S.b[0].own;
  w.keep = S.problems == 1 && keeps(S.N[0] * S.K * S.sums);
  w.np = S.problems;
  // (rows of a box that lie past the tensor take longer than others: 1 row's gradients of 2304 x 6144, 36 us with 64)
  w.ks = w.am && w.bm && S.K < BK ? cut(S.K, 16) : 4;
  w.nmaps = 3 * (S.problems > S.sums ? S.problems : S.sums);
  w.status = status;
  w.first = first;
  const bool parts = in_parts(S, c), f32 = S.out_f32 || parts;
  w.chunk = S.out_f32 ? OUT_CHUNK : PART_CHUNK;
  size_t at = 0;
  for (int i = 0; i < S.problems; ++i) {
    Problem &p = w.p[i];
    p.M = (int)S.M[i];
    p.N = (int)S.N[i];
    p.tm = cut(S.M[i], 256);
    p.tn = cut(S.N[i], c.BN);
    p.splits = c.splits;
    p.tiles = p.tm * p.tn * c.splits;
    w.tiles += p.tiles;
    p.out = 3 * i;
    void *out = S.out[i];
    if (parts) {
      out = part + at;
      at += (size_t)c.splits * S.M[i] * S.N[i];
    }
    if (!map_of(w.maps + 3 * i, out, f32, S.N[i], S.M[i], c.splits, f32 ? 32 : 64, 32, true)) return KDN_ERR_CUDA;
    for (int j = 0; j < S.sums; ++j) {  // (two sums: problem 1's places are free)
      p.steps[j] = cut(S.K, BK);
      p.a[j] = 3 * (i + j) + 1;
      p.b[j] = 3 * (i + j) + 2;
      const Operand &a = S.a[i + j], &b = S.b[i + j];
      if (!(a.own ? map_of(w.maps + p.a[j], a.p, false, S.M[i], S.K, 1, 64, 16 * w.ks, false)
                  : map_of(w.maps + p.a[j], a.p, false, S.K, S.M[i], 1, 64, 128, false)))
        return KDN_ERR_CUDA;
      if (!(b.own ? map_of(w.maps + p.b[j], b.p, false, S.N[i], S.K, 1, 64, 16 * w.ks, false)
                  : map_of(w.maps + p.b[j], b.p, false, S.K, S.N[i], 1, 64, c.BN / 2, false)))
        return KDN_ERR_CUDA;
    }
  }
  if (S.sums == 2) w.maps[3] = w.maps[0];  // (a place that nothing else takes; descriptors are fetched ahead)
  const bool sums = f32 && steps_of(S, c) > w.chunk;
  const kdn_status_t st = c.BN == 256 ? launch_plain<256>(w, f32, sums, s) : launch_plain<128>(w, f32, sums, s);
  if (st != KDN_OK || !parts) return st;
  return join_parts(S, c.splits, part, s);
}

Cut cut_of(const Spec &S) {
  return choose(S.M[0], S.N[0], S.sums * cut(S.K, BK), S.problems, true, false);
}
size_t part_of(const Spec &S) {
  const Cut c = cut_of(S);
  return in_parts(S, c) ? (size_t)c.splits * S.M[0] * S.N[0] * S.problems : 0;
}

// h (and g and u), or dg and du: the two kernels with an epilogue of their own
kdn_status_t gate(const FfnArgs &a, bool back, bool first, cudaStream_t s) {
  Work w{};
  const int steps = cut(a.D, BK);
  const Cut c = choose(a.rows, a.F, steps, 1, false, !back);
  w.act = a.act;
  w.status = a.status;
  w.first = first;
  w.bm = back;
  w.keep = keeps((back ? 1LL : 2LL) * a.D * a.F);
  w.np = 1;
  w.ks = 4;
  w.nmaps = back ? 2 : 3;
  Problem &p = w.p[0];
  p.M = (int)a.rows;
  p.N = a.F;
  p.tm = cut(a.rows, 256);
  p.tn = cut(a.F, back ? c.BN : c.BN / 2);
  p.splits = 1;
  w.tiles = p.tiles = p.tm * p.tn;
  p.steps[0] = steps;
  p.b[0] = 1;
  p.b[1] = 2;
  w.wide = !back && a.F % 16 == 0;
  void *const t[3] = {back ? a.dg : a.g, back ? a.du : a.u, back ? nullptr : a.h};
  for (int i = 0; i < 3; ++i) {
    w.out[i] = static_cast<bf *>(t[i]);
    if (t[i] && (uintptr_t)t[i] % 32) w.wide = 0;
  }
  bool ok = map_of(w.maps, back ? a.dy : a.x, false, a.D, a.rows, 1, 64, 128, false);
  if (back) {
    w.in[0] = static_cast<const bf *>(a.g);
    w.in[1] = static_cast<const bf *>(a.u);
    ok = ok && map_of(w.maps + 1, a.wd, false, a.F, a.D, 1, 64, 64, false);
  } else {
    ok = ok && map_of(w.maps + 1, a.wg, false, a.D, a.F, 1, 64, c.BN / 2, false);
    ok = ok && map_of(w.maps + 2, a.wu, false, a.D, a.F, 1, 64, c.BN / 2, false);
  }
  if (!ok) return KDN_ERR_CUDA;
  if (back) return c.BN == 256 ? launch<256, DGATE>(w, s) : launch<128, DGATE>(w, s);
  return c.BN == 256 ? launch<256, GATE>(w, s) : launch<128, GATE>(w, s);
}

}  // namespace

size_t ffn_part_floats_tc(const FfnArgs &a, bool back) {
  const bool few = ffn_few_rows(a, back);
  if (!back) return few ? 0 : part_of(down(a));
  const size_t x = few ? 0 : part_of(back_x(a)), y = part_of(back_w(a));
  return x > y ? x : y;
}

kdn_status_t launch_ffn_fwd_tc(const FfnArgs &a, cudaStream_t s) {
  if (ffn_few_rows(a, false)) return launch_ffn_fwd_rows(a, s);
  const kdn_status_t st = gate(a, false, true, s);
  if (st != KDN_OK) return st;
  const Spec S = down(a);
  return plain(S, cut_of(S), a.part, a.status, false, s);
}

kdn_status_t launch_ffn_bwd_tc(const FfnArgs &a, cudaStream_t s) {
  kdn_status_t st;
  if (ffn_few_rows(a, true)) {
    if ((st = launch_ffn_bwd_rows(a, s)) != KDN_OK) return st;
  } else {
    if ((st = gate(a, true, true, s)) != KDN_OK) return st;
    const Spec X = back_x(a);
    if ((st = plain(X, cut_of(X), a.part, a.status, false, s)) != KDN_OK) return st;
  }
  const Spec W = back_w(a);
  return plain(W, cut_of(W), a.part, a.status, false, s);
}

}  // namespace kdn
