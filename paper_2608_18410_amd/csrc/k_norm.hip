// Queries and keys divided by their heads' root mean square, weighted, and turned by
// their positions:
//   n = x w / sqrt(mean x^2 + eps),  y_i = n_i cos a_i - n_j sin a_i,  y_j = n_i sin a_i + n_j cos a_i,
// and the same on the way into the paged cache, with the values taken into the routing
// space, z = R^T v, and their kept groups packed.
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "launch.hpp"
#include "rotary.hpp"

namespace rolesub {
namespace {

// Where a call's new token goes in the cache: first its place in the sequence, then (a
// load later, which other work can cover) its page.
struct Spot {
  int page, row;  // -1: nowhere
};
struct Place {
  unsigned b;
  int64_t t;  // -1: nowhere
};
__device__ __forceinline__ Place place_of(const TurnParams& p, int64_t tok) {
  const PagedCache& c = p.c;
  const unsigned b = static_cast<unsigned>(tok) / static_cast<unsigned>(p.T);  // fewer than 2^31 tokens
  const int j = static_cast<int>(static_cast<unsigned>(tok) - b * static_cast<unsigned>(p.T));
  const int64_t cap = static_cast<int64_t>(p.max_pages) << c.shift;
  const int n = p.n_new ? p.n_new[b] : p.T;
  const int64_t t = min(static_cast<int64_t>(max(p.lens[b], 0)), cap) + j;
  return Place{b, t < cap && j < n ? t : -1};
}
__device__ __forceinline__ Spot spot_of(const TurnParams& p, const Place& x) {
  const PagedCache& c = p.c;
  if (x.t < 0) return Spot{-1, 0};
  const int page = p.table[static_cast<int64_t>(x.b) * p.max_pages + (x.t >> c.shift)];
  return Spot{static_cast<uint32_t>(page) < static_cast<uint32_t>(c.n_pages) ? page : -1, static_cast<int>(x.t & (c.page - 1))};
}

// Sum over the LPR lanes of a row, the same bits in all of them.
template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
  auto dpp = [](float y, auto ctrl) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(y), decltype(ctrl)::value, 0xF, 0xF, true));
  };
  x += dpp(x, std::integral_constant<int, 0xB1>{});                            // lanes 1 apart
  x += dpp(x, std::integral_constant<int, 0x4E>{});                            // 2 apart
  if constexpr (LPR >= 8) x += dpp(x, std::integral_constant<int, 0x141>{});   // the other half of 8
  if constexpr (LPR >= 16) x += dpp(x, std::integral_constant<int, 0x140>{});  // the other half of 16
  if constexpr (LPR >= 32) x = add_xor16(x);
  return x;
}

// Factors of a row: x becomes (x by) inv, with inv = 1 / sqrt(mean x^2 + eps). `by` is 1 but
// where inv is below the normal numbers.
struct Root {
  float by, inv;
};
// The factors from the row's sum of squares. Where that or eps leaves the range (or the sum
// is NaN), a lane's elements are squared again, scaled: by 2^-68, so that up to 128 squares of
// the largest number stay below 2^127, or by 2^64, where x below 2^-46 still has squares
// and the smallest eps is 2^-21.
template <int LPR, int N>
__device__ __forceinline__ Root inverse_root(float sq, const float (&x)[N], float per, float eps) {
  const float a = __builtin_fmaf(sq, per, eps);
  Root r = {1.f, __builtin_amdgcn_rsqf(a)};
  const bool high = !(a < __builtin_inff()), far = high || a < 0x1p-100f;
  if (__any(far)) {
    const float f = high ? 0x1p-68f : 0x1p64f;
    float again = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) again = __builtin_fmaf(x[i] * f, x[i] * f, again);
    const float root = __builtin_amdgcn_rsqf(__builtin_fmaf(row_sum<LPR>(again), per, eps * f * f));
    if (far) r = high ? Root{0x1p-32f, root * 0x1p-36f} : Root{1.f, root * 0x1p64f};
  }
  return r;
}

// Cosines and sines of one token's pairs, a pair a lane, for its wave through LDS.
__device__ __forceinline__ void put_angles(const TurnParams& p, int64_t tok, float (*cs)[kMaxPairs]) {
  const int lane = threadIdx.x & 63;
  if (lane < p.n_pairs) {
    const int ax = p.axis ? p.axis[lane] : 0;
    float cc = kStays, ss = 0.f;
    if (ax < p.n_axes) angle(p.positions[tok * p.n_axes + ax], p.inv_freq[lane], cc, ss);
    cs[0][lane] = cc;
    cs[1][lane] = ss;
  }
  wave_lds_order();
}

// Queries or keys of one token: where they lie, where they go.
template <class T>
struct Segment {
  const T *in, *weight;
  T* out;
  int64_t ld;
  int h0, h1;
};
template <class T, bool CACHE>
__device__ __forceinline__ Segment<T> segment(const TurnParams& p, int64_t tok, int seg, int h0, int h1, const Spot& spot) {
  Segment<T> g;
  g.h0 = seg ? max(h0, p.H) - p.H : h0;
  g.h1 = seg ? h1 - p.H : min(h1, p.H);
  g.in = static_cast<const T*>(seg ? p.k : p.q) + tok * (seg ? p.k_stride : p.q_stride);
  g.weight = static_cast<const T*>(seg ? p.wk : p.wq);
  g.ld = p.dh;
  if (CACHE && seg) {
    if (spot.page < 0) g.h1 = g.h0;  // nowhere
    g.out = static_cast<T*>(p.c.K) + (((static_cast<int64_t>(spot.page) * p.c.H) << p.c.shift) + spot.row) * p.dh;
    g.ld <<= p.c.shift;
  } else {
    g.out = static_cast<T*>(seg ? p.k_out : p.q_out) + tok * (seg ? p.ko_stride : p.qo_stride);
  }
  return g;
}

// Heads [h0, h1) of one token's rows (queries first, then keys), a wave's work, where
// 16-byte pieces lie in one half (or hold whole pairs, IL). A lane has two pieces of a
// row, in halves those whose elements are pairs, so that half as many lanes as pieces
// share a row and nothing passes between them but the sum of squares. The factors,
// cosines and sines times the weights, stay in registers for all heads. Without a norm the
// results are in every bit the rotation's own, whose order of the two products this
// keeps.
template <class T, int DH, bool IL, bool CACHE>
__device__ __forceinline__ void turn_whole(const TurnParams& p, int64_t tok, int h0, int h1, float (*cs)[kMaxPairs]) {
  constexpr int V = 16 / sizeof(T), LPR = DH / V / 2, HS = 64 / LPR;
  const int lane = threadIdx.x & 63, n = p.n_pairs, hl = lane / LPR, u = lane % LPR;
  // pieces A and B: a turned unit's, or two of those past the pairs
  const int np = IL ? 0 : n / V;
  const int oa = IL ? 2 * u * V : u < np ? u * V : 2 * n + (u - np) * 2 * V, ob = !IL && u < np ? oa + n : oa + V;
  const Segment<T> gq = segment<T, false>(p, tok, 0, h0, h1, Spot{-1, 0});
  Segment<T> gk = segment<T, false>(p, tok, 1, h0, h1, Spot{-1, 0});
  // steps of HS heads, those of the queries first; a step's rows are asked for two before
  const int nq = max(gq.h1 - gq.h0 + HS - 1, 0) / HS;
  int steps = nq;
  u32x4 a, b, a1, b1, a2, b2;
  auto request = [&](int st, u32x4& x, u32x4& y) {
    if (st >= steps) return;
    const T* in = st < nq ? gq.in : gk.in;
    const int h = st < nq ? min(gq.h0 + st * HS + hl, gq.h1 - 1) : min(gk.h0 + (st - nq) * HS + hl, gk.h1 - 1);
    x = *reinterpret_cast<const u32x4*>(in + static_cast<int64_t>(h) * DH + oa);
    y = *reinterpret_cast<const u32x4*>(in + static_cast<int64_t>(h) * DH + ob);
  };
  request(0, a, b);
  request(1, a1, b1);
  if constexpr (CACHE) {
    const Place at = place_of(p, tok);
    put_angles(p, tok, cs);
    gk = segment<T, true>(p, tok, 1, h0, h1, spot_of(p, at));
  } else {
    put_angles(p, tok, cs);
  }
  steps += max(gk.h1 - gk.h0 + HS - 1, 0) / HS;
  if (nq == 0) request(0, a, b);
  if (nq <= 1) request(1, a1, b1);
  bool some = false;
  uint32_t stay = 0;                   // pairs that are not turned
  float ca[V], sa[V], sb[V], cb[V];    // y0 = x0 ca - x1 sb, y1 = x0 sa + x1 cb
#pragma unroll 1
  for (int st = 0; st < steps; ++st) {
    const Segment<T>& g = st < nq ? gq : gk;
    request(st + 2, a2, b2);
    if (st == 0 || st == nq) {
      stay = 0;
#pragma unroll
      for (int x = 0; x < V; ++x) {
        const int j = u * V + x;  // the pair, in pairs those of piece A, then B
        const bool in = IL ? j < n : u < np, on = in && cs[0][in ? j : 0] != kStays;
        const float c = on ? cs[0][j] : 1.f, s = on ? cs[1][j] : 0.f;
        stay |= on ? 0u : 1u << x;
        float w0 = 1.f, w1 = 1.f;
        if (g.weight) {
          const int e = IL ? oa + 2 * x : oa + x;
          w0 = tof(g.weight[e]);
          w1 = tof(g.weight[IL ? e + 1 : ob + x]);
        }
        ca[x] = c * w0;
        sa[x] = s * w0;
        sb[x] = s * w1;
        cb[x] = c * w1;
      }
      some = __any(stay != 0u);
    }
    const int h = st < nq ? gq.h0 + st * HS + hl : gk.h0 + (st - nq) * HS + hl;
    float v[2 * V];  // x0, x1 of each pair
#pragma unroll
    for (int x = 0; x < V; ++x) {
      const T* pa = reinterpret_cast<const T*>(&a);
      const T* pb = reinterpret_cast<const T*>(&b);
      if constexpr (IL) {
        v[2 * x] = tof(x < V / 2 ? pa[2 * x] : pb[2 * x - V]);
        v[2 * x + 1] = tof(x < V / 2 ? pa[2 * x + 1] : pb[2 * x + 1 - V]);
      } else {
        v[2 * x] = tof(pa[x]);
        v[2 * x + 1] = tof(pb[x]);
      }
    }
    if (g.weight) {  // the root before the weights, whose products with x may leave the range
      float sq = 0.f;
#pragma unroll
      for (int x = 0; x < 2 * V; ++x) sq = __builtin_fmaf(v[x], v[x], sq);
      const Root root = inverse_root<LPR>(row_sum<LPR>(sq), v, 1.f / DH, p.eps);
      if (__any(root.by != 1.f))
#pragma unroll
        for (int x = 0; x < 2 * V; ++x) v[x] *= root.by;
#pragma unroll
      for (int x = 0; x < 2 * V; ++x) v[x] *= root.inv;
    }
    float y[2 * V];
#pragma unroll
    for (int x = 0; x < V; ++x) {
      y[2 * x] = __builtin_fmaf(v[2 * x], ca[x], -(v[2 * x + 1] * sb[x]));
      y[2 * x + 1] = __builtin_fmaf(v[2 * x], sa[x], v[2 * x + 1] * cb[x]);
    }
    if (some) {  // pairs that are not turned (a zero times what is not finite would reach the other)
#pragma unroll
      for (int x = 0; x < V; ++x) {
        const bool on = !((stay >> x) & 1u);
        y[2 * x] = on ? y[2 * x] : v[2 * x] * ca[x];
        y[2 * x + 1] = on ? y[2 * x + 1] : v[2 * x + 1] * cb[x];
      }
    }
    u32x4 ya, yb;
    T* ta = reinterpret_cast<T*>(&ya);
    T* tb = reinterpret_cast<T*>(&yb);
#pragma unroll
    for (int x = 0; x < V; ++x) {
      if constexpr (IL) {
        (x < V / 2 ? ta : tb)[2 * x % V] = fromf<T>(y[2 * x]);
        (x < V / 2 ? ta : tb)[2 * x % V + 1] = fromf<T>(y[2 * x + 1]);
      } else {
        ta[x] = fromf<T>(y[2 * x]);
        tb[x] = fromf<T>(y[2 * x + 1]);
      }
    }
    if (some && !g.weight) {  // neither normed nor turned: its bits, a NaN's too
      const T* pa = reinterpret_cast<const T*>(&a);
      const T* pb = reinterpret_cast<const T*>(&b);
#pragma unroll
      for (int x = 0; x < V; ++x) {
        const bool on = !((stay >> x) & 1u);
        if constexpr (IL) {
          T* to = (x < V / 2 ? ta : tb) + 2 * x % V;
          const T* from = (x < V / 2 ? pa : pb) + 2 * x % V;
          to[0] = on ? to[0] : from[0];
          to[1] = on ? to[1] : from[1];
        } else {
          ta[x] = on ? ta[x] : pa[x];
          tb[x] = on ? tb[x] : pb[x];
        }
      }
    }
    if (h < g.h1) {
      T* to = g.out + h * g.ld;
      *reinterpret_cast<u32x4*>(to + oa) = ya;
      *reinterpret_cast<u32x4*>(to + ob) = yb;
    }
    a = a1, b = b1;
    a1 = a2, b1 = b2;
  }
}

// The same for any number of pairs. A lane holds one 16-byte piece; in halves the other
// elements of its pairs lie n behind or before, so the rows of a step go through LDS (with
// room before and behind them), where a piece that element n cuts takes two reads.
// Other elements from other lanes need the LDS and a wait a step; the even ways above do not.
template <class T, int DH, bool IL, bool CACHE>
__device__ __forceinline__ void turn_any(const TurnParams& p, int64_t tok, int h0, int h1, char* stage, float (*cs)[kMaxPairs]) {
  constexpr int V = 16 / sizeof(T), U = 2, LPR = DH / V, HS = 64 / LPR;
  const int lane = threadIdx.x & 63, n = p.n_pairs, hl = lane / LPR, e0 = lane % LPR * V;
  Spot spot = {-1, 0};
  if constexpr (CACHE) spot = spot_of(p, place_of(p, tok));
  bool first = true;
  uint32_t turn = 0;  // elements that are turned
#pragma unroll 1
  for (int seg = 0; seg < 2; ++seg) {
    const Segment<T> g = segment<T, CACHE>(p, tok, seg, h0, h1, spot);
    if (g.h0 >= g.h1) continue;
    float f1[V], f2[V], wt[V];
    bool fresh = true;
    for (int hb = g.h0; hb < g.h1; hb += HS * U) {
      u32x4 a[U];
#pragma unroll
      for (int i = 0; i < U; ++i)
        a[i] = *reinterpret_cast<const u32x4*>(g.in + static_cast<int64_t>(min(hb + i * HS + hl, g.h1 - 1)) * DH + e0);
      if (first) {
        first = false;
        put_angles(p, tok, cs);
      }
      if (fresh) {
        fresh = false;
        turn = 0;
#pragma unroll
        for (int x = 0; x < V; ++x) {
          const int e = e0 + x, j = IL ? e / 2 : e < n ? e : e - n, o = IL ? e ^ 1 : e < n ? e + n : e < 2 * n ? e - n : e;
          const bool in = e < 2 * n, on = in && cs[0][in ? j : 0] != kStays, low = IL ? e % 2 == 0 : e < n;
          turn |= on ? 1u << x : 0u;
          wt[x] = g.weight ? tof(g.weight[e]) : 1.f;
          f1[x] = (on ? cs[0][j] : 1.f) * wt[x];
          f2[x] = (on ? (low ? -cs[1][j] : cs[1][j]) : 0.f) * (g.weight ? tof(g.weight[o]) : 1.f);
        }
      }
      if constexpr (!IL) {
#pragma unroll
        for (int i = 0; i < U; ++i) *reinterpret_cast<u32x4*>(stage + 16 + (i * 64 + lane) * 16) = a[i];
        wave_lds_order();
      }
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int h = hb + i * HS + hl;
        u32x4 b = a[i], d = a[i];
        if constexpr (!IL) {
          const char* me = stage + 16 + (i * 64 + lane) * 16;
          const int off = n * static_cast<int>(sizeof(T));
          if (e0 < n) __builtin_memcpy(&b, me + off, 16);
          if (e0 + V > n && e0 < 2 * n) __builtin_memcpy(&d, me - off, 16);
        }
        const T* xa = reinterpret_cast<const T*>(&a[i]);
        const T* xb = reinterpret_cast<const T*>(&b);
        const T* xd = reinterpret_cast<const T*>(&d);
        float v[V];
        Root root = {1.f, 1.f};
#pragma unroll
        for (int x = 0; x < V; ++x) v[x] = tof(xa[x]);
        if (g.weight) {
          float sq = 0.f;
#pragma unroll
          for (int x = 0; x < V; ++x) sq = __builtin_fmaf(v[x], v[x], sq);
          root = inverse_root<LPR>(row_sum<LPR>(sq), v, 1.f / DH, p.eps);
        }
        u32x4 y;
        T* vy = reinterpret_cast<T*>(&y);
#pragma unroll
        for (int x = 0; x < V; ++x) {
          const float mine = v[x] * root.by * root.inv;
          const float other = tof(IL ? xa[x ^ 1] : e0 + x < n ? xb[x] : xd[x]) * root.by * root.inv;
          const bool on = (turn >> x) & 1u;
          const float r = on ? __builtin_fmaf(mine, f1[x], other * f2[x]) : mine * wt[x];
          vy[x] = on || g.weight ? fromf<T>(r) : xa[x];
        }
        if (h < g.h1) *reinterpret_cast<u32x4*>(g.out + h * g.ld + e0) = y;
      }
      wave_lds_order();
    }
  }
}

constexpr int kStage = 2 * 64 * 16 + 32;  // bytes of a wave's rows in LDS
template <class T, int DH, bool IL, bool WHOLE, bool CACHE>
__device__ __forceinline__ void turn_rows(const TurnParams& p, int64_t tok, int h0, int h1, char* stage, float (*cs)[kMaxPairs]) {
  if constexpr (WHOLE)
    turn_whole<T, DH, IL, CACHE>(p, tok, h0, h1, cs);
  else
    turn_any<T, DH, IL, CACHE>(p, tok, h0, h1, stage, cs);
}

// A wave turns heads [hw * chunk, ...) of one token. Bound by memory: 16 times 2048 tokens
// of 32 + 8 heads of 128 dims from a fused projection (671 MB) 141 us, 4.8 TB/s, what a copy
// reaches (float32, 1.34 GB, 256 us). One token: 4.2 us, the launch and two loads behind each other.
template <class T, int DH, bool IL, bool WHOLE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(4))) void k_norm_rotary(TurnParams p, int chunks, int chunk) {
  __shared__ __attribute__((aligned(16))) char stage[4][WHOLE ? 16 : kStage];
  __shared__ float cs[4][2][kMaxPairs];
  const int w = threadIdx.x >> 6;
  const unsigned job = blockIdx.x * 4 + w, tok = job / static_cast<unsigned>(chunks);  // fewer than 2^26
  if (tok >= static_cast<unsigned>(p.B) * static_cast<unsigned>(p.T)) return;
  const int h0 = static_cast<int>(job - tok * static_cast<unsigned>(chunks)) * chunk;
  turn_rows<T, DH, IL, WHOLE, false>(p, tok, h0, min(h0 + chunk, p.H + p.Hkv), stage[w], cs[w]);
}

// Slots of the `run` tokens from n0 on (tokens of all sequences one after another): behind
// their page-mates, by an exclusive sum over the run and the 256 tokens before it. False
// if none of them goes anywhere.
constexpr int kRun = 128;
struct RunMeta {
  int page[kRun];  // -1: dropped
  uint32_t mask[kRun];
  int slot[kRun];
  int sum[256 + kRun], wsum[4], any;
};
template <class F>
__device__ __forceinline__ bool run_meta(const TurnParams& p, int64_t n0, int run, int h, RunMeta& m, F meanwhile) {
  const PagedCache& c = p.c;
  const int tid = threadIdx.x;
  const int64_t all = static_cast<int64_t>(p.B) * p.T, w0 = n0 - 256, tok = min(n0 + tid, all - 1);
  const uint32_t gm = group_bits(c.G);
  uint32_t mk[2];  // of the window, two tokens a thread
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int64_t t = w0 + 2 * tid + x;
    mk[x] = 2 * tid + x < 256 + run && t >= 0 && t < all ? p.mask[t] & gm : 0u;
  }
  const uint32_t whole = p.mask[tok];
  Spot s = spot_of(p, place_of(p, tok));
  if (tid >= run || n0 + tid >= all) s.page = -1;
  meanwhile();
  const int j = static_cast<int>(static_cast<unsigned>(tok) % static_cast<unsigned>(p.T));
  const int64_t meta = (static_cast<int64_t>(s.page) << c.shift) + s.row;
  int used = 0;
  if (s.page >= 0 && s.row > j) used = c.slot[meta - j - 1] + __popc(c.mask[meta - j - 1] & gm);
  if (tid == 0) m.any = 0;
  const int cnt = __popc(mk[0]), before = group_scan<256, false>(cnt + __popc(mk[1]), m.wsum);
  if (tid < (256 + run) / 2) {
    m.sum[2 * tid] = before;
    m.sum[2 * tid + 1] = before + cnt;
  }
  __syncthreads();
  if (tid < run) {
    m.page[tid] = s.page;
    if (s.page >= 0) {
      m.any = 1;
      const int mates = min(s.row, j);  // new ones before it in its page
      used += m.sum[256 + tid] - m.sum[256 + tid - mates];
      m.mask[tid] = whole & gm;
      m.slot[tid] = used;
      if (h == 0) {
        c.mask[meta] = whole;
        c.slot[meta] = used;
      }
    }
  }
  __syncthreads();
  return m.any != 0;
}

// Four dims of a rotated value from dim d on into the groups that keep them.
template <class T>
__device__ __forceinline__ void put_dims(const PagedCache& c, int page, int h, uint32_t mask, int slot, int d, f32x4 z) {
  T v[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) v[x] = fromf<T>(z[x]);
  T* base = static_cast<T*>(c.V) + (static_cast<int64_t>(page) * c.H + h) * c.vcap * c.ds;
  auto at = [&](int g) {  // of group g, or null
    const uint32_t sl = static_cast<uint32_t>(slot) + __popc(mask & ((1u << g) - 1u));
    return ((mask >> g) & 1u) && sl < static_cast<uint32_t>(c.vcap) ? base + static_cast<int64_t>(sl) * c.ds : nullptr;
  };
  if (c.ds >= 4) {
    T* to = at(d / c.ds);
    if (to) __builtin_memcpy(__builtin_assume_aligned(to + d % c.ds, 4 * sizeof(T)), v, 4 * sizeof(T));
  } else {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      T* to = at(d / 2 + u);
      if (to) __builtin_memcpy(__builtin_assume_aligned(to, 2 * sizeof(T)), v + 2 * u, 2 * sizeof(T));
    }
  }
}

// z = R_h^T v of a run's tokens for one head, on the matrix cores: dims of z are the
// product's rows, tokens its columns, 16 a wave. R_h lies in LDS.
template <class T, int DH>
struct Values {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int EP = 16 / sizeof(T), ROWB = DH * sizeof(T), KS = ROWB / 64, MB = DH / 16;
  static constexpr int LD = ROWB + (kBf16 ? 32 : 16), BYTES = DH * LD;
};
template <class T, int DH, class Load>
__device__ __forceinline__ void rotate_run(const TurnParams& p, int64_t n0, int run, int h, const RunMeta& m, const char* R,
                                           u32x4 (&vf)[Values<T, DH>::KS], Load load) {
  using L = Values<T, DH>;
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef s16x4 __attribute__((address_space(3))) * p3;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, l16 = lane & 15, g4 = lane >> 4;
#pragma unroll 1
  for (int t = 16 * w; t < run; t += 64) {
    f32x4 z[L::MB];
#pragma unroll
    for (int mb = 0; mb < L::MB; ++mb) z[mb] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < L::KS; ++j)
#pragma unroll
      for (int mb = 0; mb < L::MB; ++mb) {
        if constexpr (L::kBf16) {
          const char* r = R + (32 * j + 8 * g4 + l16 / 4) * L::LD + 8 * (l16 % 4) + 32 * mb;
          const bf16x4 a0 = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((p3)(r)));
          const bf16x4 a1 = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((p3)(r + 4 * L::LD)));
          z[mb] = mfma_16x16x32(__builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7), __builtin_bit_cast(bf16x8, vf[j]), z[mb]);
        } else {
          const f32x4 x = __builtin_bit_cast(f32x4, vf[j]);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float a = *reinterpret_cast<const float*>(R + (16 * j + 4 * g4 + k) * L::LD + 4 * (16 * mb + l16));
            z[mb] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, x[k], z[mb], 0, 0, 0);
          }
        }
      }
    settle(z);
    if (t + 64 < run) load(t + 64);
    const int i = t + l16, page = m.page[i];
    if (page < 0) continue;
#pragma unroll
    for (int mb = 0; mb < L::MB; ++mb) put_dims<T>(p.c, page, h, m.mask[i], m.slot[i], 16 * mb + 4 * g4, z[mb]);
  }
}

// An append. The first workgroups turn the rows of queries and keys, the last `vals` bring
// the values of one head and run of tokens. 16 times up to 305 tokens of 32 + 32 heads from
// a fused projection (157 MB) 46 us, 3.4 TB/s, of which the rows alone would take 30; with
// the values first 49, with both kinds spread evenly 51. Without the norm 39: the vector
// units are busy too. float32 (314 MB) 105, 3.0 TB/s: R_h fills 66 KB of LDS, so two
// workgroups share a CU.
template <class T, int DH, bool IL, bool WHOLE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 3 : 2))) void k_append_rotary(TurnParams p, unsigned vals, int run, int chunks, int chunk) {
  using L = Values<T, DH>;
  constexpr int ROWS = (WHOLE ? 0 : 4 * kStage) + 4 * 2 * kMaxPairs * 4, META = sizeof(RunMeta);
  __shared__ __attribute__((aligned(16))) char smem[ROWS > L::BYTES + META ? ROWS : L::BYTES + META];
  const int tid = threadIdx.x, w = tid >> 6;
  if (blockIdx.x >= gridDim.x - vals) {
    const unsigned vi = blockIdx.x - (gridDim.x - vals);
    const int h = static_cast<int>(vi % p.c.H);
    const int64_t n0 = static_cast<int64_t>(vi / p.c.H) * run;
    RunMeta& m = *reinterpret_cast<RunMeta*>(smem + L::BYTES);
    if (p.Rm) {
      constexpr int PP = L::ROWB / 16, N = DH * PP / 256;
      const char* R = static_cast<const char*>(p.Rm) + static_cast<int64_t>(h) * DH * L::ROWB;
      const int64_t last = static_cast<int64_t>(p.B) * p.T - 1;
      u32x4 vf[L::KS], rf[N];
      auto load = [&](int t) {  // this lane's part of its tile's values
        const T* v = static_cast<const T*>(p.v) + min(n0 + t + (tid & 15), last) * p.v_stride + static_cast<int64_t>(h) * DH +
                     (tid & 63) / 16 * L::EP;
#pragma unroll
        for (int j = 0; j < L::KS; ++j) vf[j] = *reinterpret_cast<const u32x4*>(v + 4 * j * L::EP);
      };
#pragma unroll
      for (int i = 0; i < N; ++i) rf[i] = *reinterpret_cast<const u32x4*>(R + (tid + 256 * i) * 16);
      load(16 * w);
      // R_h goes to LDS while the places are on their way
      const bool any = run_meta(p, n0, run, h, m, [&] {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int u = tid + 256 * i;
          *reinterpret_cast<u32x4*>(smem + u / PP * L::LD + u % PP * 16) = rf[i];
        }
      });
      if (!any) return;
      rotate_run<T, DH>(p, n0, run, h, m, smem, vf, load);
    } else {
      if (!run_meta(p, n0, run, h, m, [] {})) return;
      for (int u = tid; u < run * (DH / 4); u += 256) {
        const int i = u / (DH / 4), d = u % (DH / 4) * 4;
        if (m.page[i] < 0) continue;
        const T* v = static_cast<const T*>(p.v) + (n0 + i) * p.v_stride + static_cast<int64_t>(h) * DH + d;
        put_dims<T>(p.c, m.page[i], h, m.mask[i], m.slot[i], d, f32x4{tof(v[0]), tof(v[1]), tof(v[2]), tof(v[3])});
      }
    }
    return;
  }
  const unsigned job = blockIdx.x * 4 + w, tok = job / static_cast<unsigned>(chunks);
  if (tok >= static_cast<unsigned>(p.B) * static_cast<unsigned>(p.T)) return;
  const int h0 = static_cast<int>(job - tok * static_cast<unsigned>(chunks)) * chunk;
  turn_rows<T, DH, IL, WHOLE, true>(p, tok, h0, min(h0 + chunk, p.H + p.Hkv), smem + (WHOLE ? 0 : w * kStage),
                                    reinterpret_cast<float(*)[kMaxPairs]>(smem + (WHOLE ? 0 : 4 * kStage)) + 2 * w);
}

// Heads of a wave, as the rotation's kernels choose.
int heads_of(size_t tok, int heads) { return tok >= 4096 ? heads : tok >= 1024 ? (heads + 1) / 2 : 8; }

template <class T>
bool whole(const TurnParams& p) {
  return (p.interleaved ? 2 * p.n_pairs : p.n_pairs) % (16 / static_cast<int>(sizeof(T))) == 0;
}

template <class T, int DH>
void launch(const TurnParams& p, hipStream_t s) {
  const int heads = p.H + p.Hkv;
  const size_t tok = static_cast<size_t>(p.B) * p.T;
  const int chunk = heads_of(tok, heads), chunks = (heads + chunk - 1) / chunk;
  auto kern = p.interleaved ? (whole<T>(p) ? k_norm_rotary<T, DH, true, true> : k_norm_rotary<T, DH, true, false>)
                            : (whole<T>(p) ? k_norm_rotary<T, DH, false, true> : k_norm_rotary<T, DH, false, false>);
  hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>((tok * chunks + 3) / 4)), dim3(256), 0, s, p, chunks, chunk);
}

template <class T, int DH>
void launch_in(const TurnParams& p, hipStream_t s) {
  const int heads = p.H + p.Hkv;
  const size_t tok = static_cast<size_t>(p.B) * p.T;
  const int chunk = heads_of(tok, heads), chunks = (heads + chunk - 1) / chunk;
  // runs of 128 tokens, which read R_h half as often, where 64 would make four
  // workgroups a CU and more (the case above, before its other steps, 56 -> 51 us)
  const int run = (tok + 63) / 64 * p.c.H > 1024 ? kRun : 64;
  const size_t vals = (tok + run - 1) / run * p.c.H;
  auto kern = p.interleaved ? (whole<T>(p) ? k_append_rotary<T, DH, true, true> : k_append_rotary<T, DH, true, false>)
                            : (whole<T>(p) ? k_append_rotary<T, DH, false, true> : k_append_rotary<T, DH, false, false>);
  hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(vals + (tok * chunks + 3) / 4)), dim3(256), 0, s, p, static_cast<unsigned>(vals),
                     run, chunks, chunk);
}

}  // namespace

hipError_t launch_norm_rotary(const TurnParams& p, bool bf16, hipStream_t s) {
  if (bf16)
    p.dh == 128 ? launch<__bf16, 128>(p, s) : launch<__bf16, 64>(p, s);
  else
    p.dh == 128 ? launch<float, 128>(p, s) : launch<float, 64>(p, s);
  return hipGetLastError();
}

hipError_t launch_append_rotary(const TurnParams& p, bool bf16, hipStream_t s) {
  if (bf16)
    p.dh == 128 ? launch_in<__bf16, 128>(p, s) : launch_in<__bf16, 64>(p, s);
  else
    p.dh == 128 ? launch_in<float, 128>(p, s) : launch_in<float, 64>(p, s);
  return hipGetLastError();
}

}  // namespace rolesub
