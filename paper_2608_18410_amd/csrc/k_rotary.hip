// Queries and keys turned by their positions, with several position axes:
//   a_i = pos[axis(i)] * inv_freq[i],
//   y_i = x_i cos a_i - x_j sin a_i,  y_j = x_i sin a_i + x_j cos a_i.
#include "common.hpp"
#include "launch.hpp"

namespace rolesub {
namespace {

constexpr int kMaxPairs = 64;
constexpr float kStays = 2.f;  // in a cosine's place: no axis turns the pair

// cos and sin of pos * f. The product of a 31-bit integer and a 24-bit float and its
// share of a turn are held in two doubles each, and whole turns are taken off both before
// anything is rounded to 32 bits. Two doubles hold a turn to 2^-105 of it, so the angle
// is right to its 32-bit rounding while |pos * f| stays below 2^75. Nothing may be fused
// here but what says so: t - rint(t) from the unrounded product would count te twice.
__device__ __forceinline__ void angle(int32_t pos, float f, float& c, float& s) {
#pragma clang fp contract(off)
  constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnLo = -0x1.6b01ec5417056p-57;  // 1 / (2 pi)
  const double x = pos, y = f, p = x * y, pe = __builtin_fma(x, y, -p);
  const double t = p * kTurn, te = __builtin_fma(p, kTurn, -t) + __builtin_fma(p, kTurnLo, pe * kTurn);
  const double r = (t - __builtin_rint(t)) + (te - __builtin_rint(te));
  sincospif(static_cast<float>(r + r), &s, &c);  // half turns, in [-1, 1]
}

// Rows of whole 16-byte pieces: a wave turns heads [hw * chunk, ...) of one token.
// Lane u of a head's np units holds the unit's cosines and sines for all its heads:
// unit u is the pieces at u*V and n + u*V (halves), or the one piece of pairs at
// u*V (interleaved). Bound by memory: 32768 tokens of 32 + 8 heads of 128 (bf16, a
// view of a fused projection) move 671 MB in 124 us, 5.4 TB/s; one thread per pair
// and head took 289.
template <class T, bool IL>
__global__ __launch_bounds__(256) void k_rotary_rows(RotaryParams p, int chunks, int chunk) {
  constexpr int V = 16 / sizeof(T), NC = IL ? V / 2 : V, U = 4;
  __shared__ __attribute__((aligned(16))) float cs[4][2][kMaxPairs];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t job = static_cast<int64_t>(blockIdx.x) * 4 + w;
  const int64_t tok = job / chunks;
  if (tok >= static_cast<int64_t>(p.B) * p.T) return;
  const int n = p.n_pairs, np = n / NC, hs = 64 / np;  // units of a head, heads of a step
  const int hl = lane / np, u = lane - hl * np;
  const int h0 = static_cast<int>(job % chunks) * chunk, h1 = min(h0 + chunk, p.H + p.Hkv);
  const bool on = hl < hs;
  const int oa = u * V, ob = n + u * V;
  auto at = [&](int h, bool out) -> char* {
    const bool isq = h < p.H;
    const void* base = out ? (isq ? p.q_out : p.k_out) : (isq ? p.q : p.k);
    const int64_t st = out ? (isq ? p.qo_stride : p.ko_stride) : (isq ? p.q_stride : p.k_stride);
    return static_cast<char*>(const_cast<void*>(base)) + (tok * st + static_cast<int64_t>(isq ? h : h - p.H) * p.dh) * sizeof(T);
  };
  float c[NC] = {}, s[NC] = {};
  uint32_t stay = 0;  // pairs that no axis turns: copied (a zero times what is not finite would reach the other)
  bool first = true, some = false;
  for (int hb = h0; hb < h1; hb += hs * U) {
    u32x4 a[U], b[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int h = hb + i * hs + hl;
      if (on && h < h1) {
        const char* x = at(h, false);
        a[i] = *reinterpret_cast<const u32x4*>(x + oa * sizeof(T));
        if constexpr (!IL) b[i] = *reinterpret_cast<const u32x4*>(x + ob * sizeof(T));
      }
    }
    if (first) {  // while the first rows are on their way: a pair a lane, then through LDS
      first = false;
      if (lane < n) {
        const int ax = p.axis ? p.axis[lane] : 0;
        float cc = kStays, ss = 0.f;
        if (ax < p.n_axes) angle(p.positions[tok * p.n_axes + ax], p.inv_freq[lane], cc, ss);
        cs[w][0][lane] = cc;
        cs[w][1][lane] = p.inverse ? -ss : ss;
      }
      wave_lds_order();
      if (on)
#pragma unroll
        for (int x = 0; x < NC; x += 2) {  // NC is even, units start at even pairs
          const float2 cv = *reinterpret_cast<const float2*>(&cs[w][0][u * NC + x]);
          const float2 sv = *reinterpret_cast<const float2*>(&cs[w][1][u * NC + x]);
          c[x] = cv.x;
          c[x + 1] = cv.y;
          s[x] = sv.x;
          s[x + 1] = sv.y;
          stay |= (cv.x == kStays ? 1u << x : 0u) | (cv.y == kStays ? 2u << x : 0u);
        }
      some = __any(stay != 0u);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int h = hb + i * hs + hl;
      if (!on || h >= h1) continue;
      char* y = at(h, true);
      u32x4 ya, yb;
      const T* xa = reinterpret_cast<const T*>(&a[i]);
      const T* xb = reinterpret_cast<const T*>(&b[i]);
      T* va = reinterpret_cast<T*>(&ya);
      T* vb = reinterpret_cast<T*>(&yb);
#pragma unroll
      for (int x = 0; x < NC; ++x) {
        const float p0 = tof(IL ? xa[2 * x] : xa[x]), p1 = tof(IL ? xa[2 * x + 1] : xb[x]);
        const float r0 = p0 * c[x] - p1 * s[x], r1 = p0 * s[x] + p1 * c[x];
        if constexpr (IL) {
          va[2 * x] = fromf<T>(r0);
          va[2 * x + 1] = fromf<T>(r1);
        } else {
          va[x] = fromf<T>(r0);
          vb[x] = fromf<T>(r1);
        }
      }
      if (some) {
#pragma unroll
        for (int x = 0; x < NC; ++x) {
          if (!((stay >> x) & 1u)) continue;
          if constexpr (IL) {
            va[2 * x] = xa[2 * x];
            va[2 * x + 1] = xa[2 * x + 1];
          } else {
            va[x] = xa[x];
            vb[x] = xb[x];
          }
        }
      }
      *reinterpret_cast<u32x4*>(y + oa * sizeof(T)) = ya;
      if constexpr (!IL) *reinterpret_cast<u32x4*>(y + ob * sizeof(T)) = yb;
    }
  }
  // dims past the pairs
  const int rest = (p.dh - 2 * n) / V;
  for (int i = lane; i < (h1 - h0) * rest; i += 64) {
    const int h = h0 + i / rest, o = (2 * n + i % rest * V) * static_cast<int>(sizeof(T));
    *reinterpret_cast<u32x4*>(at(h, true) + o) = *reinterpret_cast<const u32x4*>(at(h, false) + o);
  }
}

// Any number of pairs: a wave turns heads [hw * chunk, ...) of one token, a lane one
// 16-byte piece of a row, with the cosines and sines of its elements in registers for
// all heads. In halves the other elements of its pairs lie n behind or before: one more
// load of the same row at whatever alignment, two in the piece that element n cuts. Such
// a load may begin before the row or end past it, but stays within the rows of the
// tensor; the first and the last token's come one by one. In pairs (IL) the piece holds
// them. A wave has loaded a row whole before it writes it, so rows may be turned in
// place. 32768 tokens of 32 + 8 heads of 128 (bf16) and 63 pairs in halves take 211 us, bound by
// the loads off their alignment (the cut piece's one by one: 232; a thread for each pair
// and head: 304); 33712 of 16 + 16 heads and 50 pairs in pairs (552 MB) 108, 5.1 TB/s.
template <class T, bool IL>
__global__ __launch_bounds__(256) void k_rotary_any(RotaryParams p, int chunks, int chunk) {
  constexpr int V = 16 / sizeof(T), U = 4;
  __shared__ float cs[4][2][kMaxPairs];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t job = static_cast<int64_t>(blockIdx.x) * 4 + w;
  const int64_t tok = job / chunks;
  if (tok >= static_cast<int64_t>(p.B) * p.T) return;
  const int n = p.n_pairs, lpr = p.dh / V, hs = 64 / lpr;  // lanes of a row, heads of a step
  const int hl = lane / lpr, e0 = lane % lpr * V;
  const int h0 = static_cast<int>(job % chunks) * chunk, h1 = min(h0 + chunk, p.H + p.Hkv);
  if (lane < n) {
    const int ax = p.axis ? p.axis[lane] : 0;
    float c = kStays, s = 0.f;
    if (ax < p.n_axes) angle(p.positions[tok * p.n_axes + ax], p.inv_freq[lane], c, s);
    cs[w][0][lane] = c;
    cs[w][1][lane] = p.inverse ? -s : s;
  }
  wave_lds_order();
  float c[V], s[V];
  uint32_t turn = 0;  // elements that are turned; the others are copied
#pragma unroll
  for (int x = 0; x < V; ++x) {
    const int e = e0 + x, i = IL ? e / 2 : e < n ? e : e - n;
    const bool on = e < 2 * n && cs[w][0][e < 2 * n ? i : 0] != kStays, low = IL ? e % 2 == 0 : e < n;
    c[x] = on ? cs[w][0][on ? i : 0] : 1.f;
    s[x] = on ? (low ? -cs[w][1][on ? i : 0] : cs[w][1][on ? i : 0]) : 0.f;
    turn |= on ? 1u << x : 0u;
  }
  const bool edge = tok == 0 || tok == static_cast<int64_t>(p.B) * p.T - 1;
  const bool low = !IL && e0 < n, high = !IL && e0 + V > n && e0 < 2 * n;  // pieces of either half
  for (int hb = h0; hb < h1; hb += hs * U) {
    u32x4 a[U], b[U], d[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int h = hb + i * hs + hl;
      if (h >= h1) continue;
      const bool isq = h < p.H;
      const T* row = static_cast<const T*>(isq ? p.q : p.k) + tok * (isq ? p.q_stride : p.k_stride) +
                     static_cast<int64_t>(isq ? h : h - p.H) * p.dh;
      a[i] = *reinterpret_cast<const u32x4*>(row + e0);
      if constexpr (!IL) {
        b[i] = d[i] = a[i];
        if (!edge) {
          if (low) __builtin_memcpy(&b[i], row + e0 + n, 16);
          if (high) __builtin_memcpy(&d[i], row + e0 - n, 16);
        } else {
          T* vb = reinterpret_cast<T*>(&b[i]);
#pragma unroll
          for (int x = 0; x < V; ++x) {
            const int e = e0 + x;
            vb[x] = row[e < n ? e + n : e < 2 * n ? e - n : e];
          }
          d[i] = b[i];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int h = hb + i * hs + hl;
      if (h >= h1) continue;
      const bool isq = h < p.H;
      T* row = static_cast<T*>(isq ? p.q_out : p.k_out) + tok * (isq ? p.qo_stride : p.ko_stride) +
               static_cast<int64_t>(isq ? h : h - p.H) * p.dh;
      const T* xa = reinterpret_cast<const T*>(&a[i]);
      const T* xb = reinterpret_cast<const T*>(&b[i]);
      const T* xd = reinterpret_cast<const T*>(&d[i]);
      u32x4 y;
      T* vy = reinterpret_cast<T*>(&y);
#pragma unroll
      for (int x = 0; x < V; ++x) {
        const float r = tof(xa[x]) * c[x] + tof(IL ? xa[x ^ 1] : e0 + x < n ? xb[x] : xd[x]) * s[x];
        vy[x] = (turn >> x) & 1u ? fromf<T>(r) : xa[x];
      }
      *reinterpret_cast<u32x4*>(row + e0) = y;
    }
  }
}

template <class T>
void launch(const RotaryParams& p, hipStream_t s) {
  constexpr int V = 16 / sizeof(T);
  const int heads = p.H + p.Hkv;
  const size_t tok = static_cast<size_t>(p.B) * p.T;
  // a wave per token where there are tokens enough for every wave slot (256 CUs of
  // 16 waves and more): its cosines serve all heads; with fewer the heads are split
  const int chunk = tok >= 4096 ? heads : tok >= 1024 ? (heads + 1) / 2 : 8;
  const int chunks = (heads + chunk - 1) / chunk;
  const dim3 grid(static_cast<unsigned>((tok * chunks + 3) / 4));
  const bool whole = (p.interleaved ? 2 * p.n_pairs : p.n_pairs) % V == 0;  // pieces lie in one half
  auto kern = p.interleaved ? (whole ? k_rotary_rows<T, true> : k_rotary_any<T, true>)
                            : (whole ? k_rotary_rows<T, false> : k_rotary_any<T, false>);
  hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, p, chunks, chunk);
}

}  // namespace

hipError_t launch_rotary(const RotaryParams& p, bool bf16, hipStream_t s) {
  if (bf16)
    launch<__bf16>(p, s);
  else
    launch<float>(p, s);
  return hipGetLastError();
}

}  // namespace rolesub
