// kdn_swa.cuh -- internal types of the sliding-window attention with sinks
// (kdn_swa_* of include/kdn.h), shared by its translation units.
//
// Query i of a sequence of `len` tokens sees key j when j <= i and
// (j > i - W or j < s): the last W tokens up to itself, and the first s.
#pragma once

#include "kdn_beside.cuh"
#include "kdn_internal.cuh"

namespace kdn {

// log2(e): the kernels take exp as exp2 with the factor folded into the scale
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct SwaArgs {
  int B, T, H, Hk, G, d;  // G = H / Hk query heads share one kv head
  int W, ns;              // window, sinks
  int dtype;
  float scale;
  const void *q, *k, *v;
  const int *lens;  // [B] or null (every sequence has T tokens)
  void *o;
  float *lse;       // [B][H][T], null: not written
  // backward
  const void *dO;
  void *dq, *dk, *dv;
  float *nlse;      // [B][H][T] lse in log2 units (+inf for rows that see nothing)
  float *delta;     // [B][H][T] sum_d o dO
  float *part;      // split key tiles: float32 partial dk, dv
  unsigned *status;
};

__device__ __forceinline__ int swa_len(const SwaArgs &a, int b) {
  return a.lens ? min(max(a.lens[b], 0), a.T) : a.T;
}

__device__ __forceinline__ bool swa_sees(int i, int j, int W, int ns) {
  return j <= i && (j > i - W || j < ns);
}

// Key tiles (of BN keys) that queries [i0, i1) see, i0 < i1: first the tiles of
// the sinks that lie before the window, then the window's tiles up to the
// diagonal.  Tile number n of the list is `at(n)`.
struct SwaKeyTiles {
  int nsink, first, count;
  __device__ __forceinline__ SwaKeyTiles(int i0, int i1, int W, int ns, int BN) {
    first = max(0, i0 - W + 1) / BN;
    nsink = min((min(ns, i1) + BN - 1) / BN, first);
    count = nsink + (i1 - 1) / BN - first + 1;
  }
  __device__ __forceinline__ int at(int n) const { return n < nsink ? n : first + n - nsink; }
};

// The backward over key tiles: each tile's list of (query head of the group,
// query tile) iterations is cut into splits of equal length.  Tiles that
// hold sinks are seen by every later query and get `splits_sink` splits, the
// others `splits`; tiles with more than one split leave float32 partial sums,
// added in split order by a second kernel (the result does not depend on timing).
struct SwaSplits {
  int tiles, sink_tiles;     // key tiles of a sequence; those that hold sinks
  int per_sink, per;         // iterations of one split
  int splits_sink, splits;
  int blocks;                // splits of one (batch, kv head)
  int part_blocks;           // the first so many of them write partial sums
};

// Query tiles [first, last] that see key tile t (keys [t*BN, ..)), len > t*BN.
__host__ __device__ inline void swa_query_tiles(int t, int BN, int BM, int W, int ns, int len,
                                                int *first, int *last) {
  const int j0 = t * BN;
  const long long end = j0 < ns ? (long long)len : (long long)j0 + BN - 1 + W;  // exclusive
  *first = j0 / BM;
  *last = (int)(((end < len ? end : (long long)len) - 1) / BM);
}

SwaSplits swa_splits(const SwaArgs &a, int BM, int BN);

// Rows of key tile t (tiles of BN queries and keys) that split number `split` adds to: a
// split of a sink tile whose queries all lie past the tile's window only has the sinks'.
__device__ __forceinline__ int swa_split_rows(int t, int split, int per, int BN, int W, int ns, int G, int len) {
  const int j0 = t * BN;
  if (j0 >= len) return 0;
  int first, last;
  swa_query_tiles(t, BN, BN, W, ns, len, &first, &last);
  const int nq = last - first + 1, it0 = split * per, it1 = min(it0 + per, G * nq);
  if (it0 >= it1) return 0;
  const int q = it0 / nq == (it1 - 1) / nq ? first + it0 % nq : first;  // its first query tile
  return j0 < ns && q * BN - W >= j0 + BN - 1 ? min(BN, ns - j0) : BN;
}

// bfloat16 runs on the tensor cores, float32 on the general kernels
bool swa_tc_supported(const SwaArgs &a);
kdn_status_t launch_swa_fwd_tc(const SwaArgs &a, cudaStream_t s);
kdn_status_t launch_swa_bwd_tc(const SwaArgs &a, const SwaSplits &sp, cudaStream_t s);
kdn_status_t launch_swa_decode_tc(const SwaArgs &a, void *kc, void *vc, const int *pos, cudaStream_t s);
constexpr int kSwaTcTile = 128;  // query and key tile of the tensor-core kernels
kdn_status_t launch_swa_fwd_general(const SwaArgs &a, cudaStream_t s);
kdn_status_t launch_swa_bwd_general(const SwaArgs &a, const SwaSplits &sp, cudaStream_t s);
// delta, nlse and a cleared status word: the first launches of every backward
kdn_status_t launch_swa_prep(const SwaArgs &a, cudaStream_t s);
// adds the partial sums of split key tiles into dk, dv
kdn_status_t launch_swa_join(const SwaArgs &a, const SwaSplits &sp, int BN, cudaStream_t s);
kdn_status_t launch_swa_cache_fill(const SwaArgs &a, void *kc, void *vc, cudaStream_t s);
kdn_status_t launch_swa_decode_general(const SwaArgs &a, void *kc, void *vc, const int *pos, cudaStream_t s);

constexpr int kSwaGenTile = 64;  // query and key tile of the general kernels

}  // namespace kdn
