// kdn_rope.cu -- rotary positions of queries and keys, both directions.
//
//   pair (x1, x2) of a token at position p, angle a = p f:  y1 = m (x1 cos a - x2 sin a),
//   y2 = m (x1 sin a + x2 cos a);  backward: the same with -a.
//
// Angles.  f is kept as a fraction of a turn in units of 2^-64, so p f modulo one turn is one
// integer product whose overflow is the modulus: the angle is as exact at position 2^31 as at 1
// (a float32 product is off by 2^-24 of the whole angle: 0.03 turns after 500 000 of them).
//
// A CTA takes TT tokens.  Its threads first issue the loads of their units (a unit is what one
// thread turns: a 16-byte vector of either half, or one vector of neighbouring pairs), then form the
// tokens' cosines and sines once for all heads into shared memory while the loads fly.
// HBM traffic bounds it where whole heads are turned: 86 us a direction for 8 x 4096 tokens of 16 + 16 heads of 128 in
// bfloat16, 6.2 TB/s of the 6.8 of a copy.  Instructions do where most vectors are only copied or cleared: 8 x 1777 tokens
// of 18 + 3 heads, 32 of 128 channels turned, padded, 29 us with 75 % of the issue slots taken (a vector's place is
// formed twice, and its token's length looked up).
#include "kdn_beside.cuh"
#include "kdn_fastdiv.cuh"
#include "kdn_rope.cuh"

namespace kdn {
namespace {

constexpr int NT = 256;

enum { HALF = 0, NEIGHBOURS = 1, SINGLE = 2 };  // units: two vectors, one vector, a pair of elements

struct Shape {
  int TT;               // tokens a CTA
  int turned, units;    // units of a head that are turned; all of them (the others are copied)
  FastDiv by_token, by_head;  // units of a token, of a head
};

template <typename DT, int N> struct Vec;  // N elements as they are stored
template <> struct Vec<__nv_bfloat16, 8> { uint4 v; };
template <> struct Vec<float, 4> { uint4 v; };
template <> struct Vec<__nv_bfloat16, 1> { __nv_bfloat16 v; };
template <> struct Vec<float, 1> { float v; };

template <typename DT, int N> __device__ __forceinline__ void unpack(const Vec<DT, N> &u, float *x) {
  const DT *p = reinterpret_cast<const DT *>(&u);
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = (float)p[i];
}
template <typename DT, int N> __device__ __forceinline__ Vec<DT, N> pack(const float *x) {
  Vec<DT, N> u;
  DT *p = reinterpret_cast<DT *>(&u);
#pragma unroll
  for (int i = 0; i < N; ++i) p[i] = (DT)x[i];
  return u;
}

template <typename DT, int KIND, int NU>
__global__ void __launch_bounds__(NT) k_rope(const __grid_constant__ RopeArgs a, const Shape S) {
  constexpr int V = KIND == SINGLE ? 1 : 16 / (int)sizeof(DT);
  constexpr int PER = KIND == NEIGHBOURS ? V / 2 : V;  // pairs of a unit
  using Vc = Vec<DT, V>;
  extern __shared__ float2 s_cs[];  // [TT][rot / 2]: m cos, m sin
  const int pairs = a.rot / 2, total = a.B * a.T, n0 = blockIdx.x * S.TT, nt = min(S.TT, total - n0);
  const int heads = a.H + a.Hk, all = nt * heads * S.units;

  // where a unit's one or two vectors lie; second < 0: there is only one
  struct Place {
    int token, which, first, second, pair;
    long long row;
  };
  auto place = [&](int unit) {
    Place p;
    p.token = S.by_token.div(unit);
    unit -= p.token * heads * S.units;
    int head = S.by_head.div(unit);
    const int i = unit - head * S.units;
    p.which = head >= a.H;
    head -= p.which ? a.H : 0;
    p.row = n0 + p.token;
    const int c = head * a.d;
    p.pair = i < S.turned ? i * PER : -1;
    if (KIND == HALF) {
      p.first = c + (i < S.turned ? i * V : a.rot + (i - S.turned) * V);
      p.second = i < S.turned ? p.first + pairs : -1;
    } else if (KIND == NEIGHBOURS) {
      p.first = c + i * V;
      p.second = -1;
    } else {
      p.first = c + (i >= S.turned ? a.rot + (i - S.turned) : a.inter ? 2 * i : i);
      p.second = i >= S.turned ? -1 : p.first + (a.inter ? 1 : pairs);
    }
    return p;
  };
  auto live = [&](int token) {
    if (!a.lens) return true;
    const int n = n0 + token, b = n / a.T;
    return n - b * a.T < a.lens[b];
  };
  constexpr bool TWO = KIND != NEIGHBOURS;
  Vc x[NU], y[TWO ? NU : 1];
  auto load = [&](int unit0) {
#pragma unroll
    for (int j = 0; j < NU; ++j) {
      const int unit = unit0 + j * NT;
      if (unit >= all) continue;
      const Place p = place(unit);
      const bool on = live(p.token);
      const DT *src = static_cast<const DT *>(a.in[p.which]) + p.row * a.ldi[p.which];
      x[j] = on ? *reinterpret_cast<const Vc *>(src + p.first) : Vc{};
      if (TWO) y[TWO ? j : 0] = on && p.second >= 0 ? *reinterpret_cast<const Vc *>(src + p.second) : Vc{};
    }
  };
  let_next_start();
  wait_for_previous();
  load(threadIdx.x);

  for (int e = threadIdx.x; e < nt * pairs; e += NT) {
    const int token = e / pairs, i = e - token * pairs, n = n0 + token, b = n / a.T, t = n - b * a.T;
    const long long p = a.per_token ? a.pos[n] : (a.pos ? (long long)a.pos[b] : 0) + t;
    const unsigned long long at = a.turns[i] * (unsigned long long)p;  // modulo one turn
    // the nearest quarter turn, exactly, and the rest of it: within 1/8 turn the rest's rounding to
    // float32 is at most 2^-25 of 0.8 radians
    const unsigned hi = (unsigned)(at >> 32), quarter = (hi + (1u << 29)) >> 30;
    float sn, cs;
    sincospif((float)(int)(hi - (quarter << 30)) * 0x1p-31f, &sn, &cs);
    if (quarter & 1) {
      const float x = sn;
      sn = cs;
      cs = -x;
    }
    if (quarter & 2) {
      sn = -sn;
      cs = -cs;
    }
    s_cs[e] = make_float2(a.mscale * cs, a.sign * a.mscale * sn);
  }
  __syncthreads();

  for (int unit0 = threadIdx.x; unit0 < all;) {
#pragma unroll
    for (int j = 0; j < NU; ++j) {
      const int unit = unit0 + j * NT;
      if (unit >= all) continue;
      const Place p = place(unit);
      DT *dst = static_cast<DT *>(a.out[p.which]) + p.row * a.ldo[p.which];
      if (p.pair < 0) {
        *reinterpret_cast<Vc *>(dst + p.first) = x[j];
        continue;
      }
      const float2 *cs = s_cs + p.token * pairs + p.pair;
      float f[V], g[V];
      unpack(x[j], f);
      if (KIND == NEIGHBOURS) {
#pragma unroll
        for (int e = 0; e < V; e += 2) {
          const float2 c = cs[e / 2];
          const float x1 = f[e], x2 = f[e + 1];
          f[e] = x1 * c.x - x2 * c.y;
          f[e + 1] = x1 * c.y + x2 * c.x;
        }
      } else {
        unpack(y[TWO ? j : 0], g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float2 c = cs[e];
          const float x1 = f[e], x2 = g[e];
          f[e] = x1 * c.x - x2 * c.y;
          g[e] = x1 * c.y + x2 * c.x;
        }
        *reinterpret_cast<Vc *>(dst + p.second) = pack<DT, V>(g);
      }
      *reinterpret_cast<Vc *>(dst + p.first) = pack<DT, V>(f);
    }
    unit0 += NU * NT;
    if (unit0 < all) load(unit0);
  }
}

template <typename DT, int KIND> kdn_status_t launch(const RopeArgs &a, cudaStream_t s) {
  constexpr int V = KIND == SINGLE ? 1 : 16 / (int)sizeof(DT), NU = KIND == HALF ? 4 : 8;
  const bool in_place = a.in[0] == a.out[0] && (!a.Hk || a.in[1] == a.out[1]);
  const int turned = KIND == NEIGHBOURS ? a.rot / V : a.rot / 2 / V;
  // channels that are not turned are not touched in place, but for padding, which is set to 0
  const int units = turned + (in_place && !a.lens ? 0 : (a.d - a.rot) / V), heads = a.H + a.Hk;
  const long long total = (long long)a.B * a.T;
  // as many tokens as fill a CTA's threads once, while that leaves two CTAs an SM
  long long TT = NU * NT / (heads * units);
  if (TT > total / 304) TT = total / 304;
  TT = TT < 1 ? 1 : TT > 16 ? 16 : TT;
  const Shape S{(int)TT, turned, units, FastDiv((uint32_t)(heads * units)), FastDiv((uint32_t)units)};
  return launch_beside(k_rope<DT, KIND, NU>, dim3((unsigned)((total + TT - 1) / TT)), NT,
                       (int)TT * a.rot / 2 * (int)sizeof(float2), s, a, S);
}

template <typename DT> kdn_status_t by_kind(const RopeArgs &a, cudaStream_t s) {
  constexpr int V = 16 / (int)sizeof(DT);
  bool wide = true;  // rows that start on 16 bytes
  for (int i = 0; i < (a.Hk ? 2 : 1); ++i) wide = wide && a.ldi[i] % V == 0 && a.ldo[i] % V == 0;
  if (wide && a.inter && a.rot % V == 0) return launch<DT, NEIGHBOURS>(a, s);
  if (wide && !a.inter && a.rot % (2 * V) == 0) return launch<DT, HALF>(a, s);
  return launch<DT, SINGLE>(a, s);
}

}  // namespace

kdn_status_t launch_rope(const RopeArgs &a, cudaStream_t s) {
  return a.dtype == KDN_BF16 ? by_kind<__nv_bfloat16>(a, s) : by_kind<float>(a, s);
}

}  // namespace kdn
