// kdn_swa_tc.cuh -- what the tensor-core kernels of the sliding-window attention share:
// TMEM accesses of 32 columns, products with the A operand in TMEM, packed float32
// arithmetic, and the TMA descriptor of 128 tokens of one head.
#pragma once

#include "kdn_fused_common.cuh"
#include "kdn_swa.cuh"

namespace kdn {
namespace swa {

using namespace sm103;
using fused::chunk_off;
using fused::sm16;

constexpr uint32_t kWait = 1u << 25;  // polls of a bounded wait (seconds), as in the other fused kernels
constexpr int TILE = 128;             // queries of an accumulator, keys of a tile
constexpr int SLAB = TILE * 128;      // 128 rows of 64 bf16: one 128-byte-swizzled slab

// 32 lanes x 32 columns; the registers are valid after tmem_ld_wait(r).
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float *v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
      "%15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]),
        "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]),
        "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(taddr)
      : "memory");
}
// Ties 32 registers to this point of the program: what a load wrote into them is not
// used before it.
__device__ __forceinline__ void pin32(float *v) {
  asm volatile(""
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                 "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]),
                 "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]),
                 "+f"(v[22]), "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]),
                 "+f"(v[29]), "+f"(v[30]), "+f"(v[31])::"memory");
}
template <int N> __device__ __forceinline__ void tmem_ld_wait(float *v) {  // N registers, a multiple of 32
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; i += 32) pin32(v + i);
}
__device__ __forceinline__ void tmem_st16u(uint32_t taddr, const uint32_t *v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
      "%15, %16};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
      "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const float *v) {
  tmem_st16(taddr, v);
  tmem_st16(taddr + 16, v + 16);
}

// D(tmem) (+)= A(tmem) * B(smem desc): A holds 128 rows (lanes), two 16-bit elements of
// the K axis a column.
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc,
                                        uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// One lane of a converged warp, the same one every time.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
  return p != 0;
}
// A value that is the same in every lane, in a form the compiler knows to be.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __shfl_sync(0xffffffffu, x, 0); }

// Descriptors of a [128][64 n] tile in 128-byte-swizzled slabs, as a sum of a part that is
// formed once and the offset of a K step, so that a product issues with one addition:
// K along the 64-element rows (its step kk of 16 elements) ...
__device__ __forceinline__ uint64_t desc_k(const void *tile) { return sw128_desc(smem_u32(tile), 16, 1024); }
__device__ __forceinline__ constexpr uint64_t step_k(int kk) { return ((kk >> 2) * SLAB + (kk & 3) * 32) >> 4; }
// ... or along the 128 rows (the M or N axis along the 64-element rows).
__device__ __forceinline__ uint64_t desc_mn(const void *tile) { return sw128_desc(smem_u32(tile), SLAB, 1024); }
__device__ __forceinline__ constexpr uint64_t step_mn(int kk) { return (kk * 2048) >> 4; }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// two float32 multiply-adds (additions) in one instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<unsigned long long &>(d))
      : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)),
        "l"(reinterpret_cast<unsigned long long &>(c)));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<unsigned long long &>(d))
      : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<unsigned long long &>(d))
      : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)));
  return d;
}
__device__ __forceinline__ uint32_t pack_bf2(float lo, float hi) {
  uint32_t u;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(hi), "f"(lo));
  return u;
}

// The first n bits of a word (n of any size).
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : n > 0 ? (1u << n) - 1u : 0u; }
// Bits of 32 consecutive keys that a query sees; key 0 of them lies `hi` before it
// (hi < 0: behind it), and `sinks` of them are sinks.
__device__ __forceinline__ uint32_t key_bits(int hi, int W, int sinks) {
  return low_bits(hi + 1) & (~low_bits(hi - W + 1) | low_bits(sinks));
}

// A bounded wait that gives up for the whole CTA: the first thread whose wait runs out
// raises `fail` (shared memory) and records the timeout; from then on no wait of the CTA
// lasts.  Threads that must stay together go on regardless (what they compute is invalid
// and the status says so); the loading and the issuing thread leave their loops.
struct Waiter {
  volatile int *fail;
  unsigned *status;
  __device__ __forceinline__ bool operator()(uint64_t *bar, uint32_t parity) const {
    if (mbar_try_wait(bar, parity)) return true;
    for (uint32_t i = 0; i < kWait; ++i) {
      if (mbar_try_wait(bar, parity)) return true;
      if (*fail) return false;
      if (i > 256) __nanosleep(64);
    }
    *fail = 1;
    atomicExch(status, (unsigned)KDN_ERR_TIMEOUT);
    return false;
  }
  // by the loading thread and others that run ahead: they poll less often, since polls
  // take issue slots from the warps that everything waits for
  __device__ __forceinline__ bool lazy(uint64_t *bar, uint32_t parity) const {
    if (mbar_try_wait(bar, parity)) return true;
    for (uint32_t i = 0; i < kWait; ++i) {
      __nanosleep(64);
      if (mbar_try_wait(bar, parity)) return true;
      if ((i & 15) == 15 && *fail) return false;
    }
    *fail = 1;
    atomicExch(status, (unsigned)KDN_ERR_TIMEOUT);
    return false;
  }
  // by all lanes of a warp, which go on together
  __device__ __forceinline__ void warp(uint64_t *bar, uint32_t parity) const {
    (*this)(bar, parity);
    __syncwarp();
  }
};

// 32 consecutive columns of a row times f as bf16 (zeros where the row is not live).
// wide: the row is 32-byte aligned, which takes half as many stores.
__device__ __forceinline__ void store_row32(__nv_bfloat16 *dst, const float *x, float f, bool live, bool wide) {
  uint32_t u[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) u[e] = live ? pack_bf2(x[2 * e] * f, x[2 * e + 1] * f) : 0u;
  if (wide) {
#pragma unroll
    for (int e = 0; e < 16; e += 8)
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst + 2 * e), "r"(u[e]),
                   "r"(u[e + 1]), "r"(u[e + 2]), "r"(u[e + 3]), "r"(u[e + 4]), "r"(u[e + 5]), "r"(u[e + 6]),
                   "r"(u[e + 7])
                   : "memory");
  } else {
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      *reinterpret_cast<uint4 *>(dst + 2 * e) = make_uint4(u[e], u[e + 1], u[e + 2], u[e + 3]);
  }
}
__device__ __forceinline__ bool aligned32(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 31) == 0; }

// n / d for 0 <= n < 2^31 by a multiplication: with 2^s < d <= 2^(s+1) and
// m = ceil(2^(32+s) / d), the excess m d - 2^(32+s) is below d, and n times it below 2^(32+s).
struct FastDiv {
  uint32_t m, s;  // m = 0: d = 1
  explicit FastDiv(uint32_t d) : m(0), s(0) {
    if (d == 1) return;
    while ((2ull << s) < d) ++s;
    m = (uint32_t)(((1ull << (32 + s)) + d - 1) / d);
  }
  __device__ __forceinline__ int div(int n) const { return m ? (int)(__umulhi((uint32_t)n, m) >> s) : n; }
};

// The work items of a persistent CTA.  Its first is blockIdx.x; the loading warp takes
// the others from a counter in global memory (zero at launch), in order, as it comes to
// them, and hands each to the CTA's other warps through a ring in shared memory.
constexpr int kRing = 4;
struct ItemRing {
  uint64_t *full, *empty;  // [kRing]; empty: one arrival a consuming warp
  volatile int *slot;      // [kRing]
};
struct ItemSource {  // the loading warp
  const ItemRing &ring;
  const Waiter &wait;
  unsigned *counter;
  int total, n = 0, ahead = 0;
  __device__ __forceinline__ ItemSource(const ItemRing &r, const Waiter &w, unsigned *c, int items)
      : ring(r), wait(w), counter(c), total(items) {}
  __device__ __forceinline__ int next() {  // by all lanes; -1: no more
    int item = 0;
    if (threadIdx.x % 32 == 0) {
      item = n == 0 ? (int)blockIdx.x : ahead;
      if (item >= total) item = -1;
      // the next one's number arrives while this one is loaded
      else if ((ahead = (int)(gridDim.x + atomicAdd(counter, 1u))) < 0) ahead = total;
      const int s = n % kRing;
      if (n >= kRing && !wait(ring.empty + s, (n / kRing - 1) & 1)) item = -1;
      ring.slot[s] = item;
      mbar_arrive(ring.full + s);
    }
    ++n;
    return __shfl_sync(0xffffffffu, item, 0);
  }
};
struct ItemSink {  // a warp that works on them
  const ItemRing &ring;
  const Waiter &wait;
  int n = 0;
  __device__ __forceinline__ ItemSink(const ItemRing &r, const Waiter &w) : ring(r), wait(w) {}
  __device__ __forceinline__ int next() {  // by all lanes; -1: no more
    const int s = n % kRing;
    const bool ok = wait(ring.full + s, (n / kRing) & 1);
    const int item = __shfl_sync(0xffffffffu, ok ? ring.slot[s] : -1, 0);
    __syncwarp();
    if (threadIdx.x % 32 == 0) mbar_arrive(ring.empty + s);
    ++n;
    return item;
  }
};
constexpr int kCtas = 152;  // one persistent CTA an SM

// Rows [first, 128) of a tile of `slabs` slabs set to zero by one warp: tokens past a
// sequence's length hold anything, and a weight of zero does not hide a NaN.
__device__ __forceinline__ void zero_rows(unsigned char *tile, int slabs, int first, int lane) {
  for (int s = 0; s < slabs; ++s)
    for (int c = first * 8 + lane; c < TILE * 8; c += 32)
      *reinterpret_cast<uint4 *>(tile + s * SLAB + c * 16) = make_uint4(0, 0, 0, 0);
}

// TMA descriptor of a [B, T, heads, d] bf16 tensor; box: 64 channels of one head, 128 tokens.
inline bool token_map(CUtensorMap *m, const void *p, int B, int T, int heads, int d) {
  auto enc = fused::encoder();
  if (!enc) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)T, (cuuint64_t)B};
  const cuuint64_t strides[3] = {(cuuint64_t)d * 2, (cuuint64_t)heads * d * 2, (cuuint64_t)T * heads * d * 2};
  const cuuint32_t box[4] = {64, 1, TILE, 1}, es[4] = {1, 1, 1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(p), dims, strides, box, es,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace swa
}  // namespace kdn
