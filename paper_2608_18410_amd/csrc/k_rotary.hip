// Queries and keys turned by their positions, with several position axes:
//   a_i = pos[axis(i)] * inv_freq[i],
//   y_i = x_i cos a_i - x_j sin a_i,  y_j = x_i sin a_i + x_j cos a_i.
#include "common.hpp"
#include "launch.hpp"

namespace rolesub {
namespace {

constexpr int kMaxPairs = 64;

// cos and sin of pos * f. The product of a 31-bit integer and a 24-bit float and its
// share of a turn are held in two doubles each, and whole turns are taken off before
// anything is rounded to 32 bits: exact for every position and frequency.
__device__ __forceinline__ void angle(int32_t pos, float f, float& c, float& s) {
  constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnLo = -0x1.6b01ec5417056p-57;  // 1 / (2 pi)
  const double x = pos, y = f, p = x * y, pe = __builtin_fma(x, y, -p);
  const double t = p * kTurn, te = __builtin_fma(p, kTurn, -t) + __builtin_fma(p, kTurnLo, pe * kTurn);
  const double r = (t - __builtin_rint(t)) + te;
  sincospif(static_cast<float>(r + r), &s, &c);  // half turns, in [-1, 1]
}

// Rows of whole 16-byte pieces: a wave turns heads [hw * chunk, ...) of one token.
// Lane u of a head's np units holds the unit's cosines and sines for all its heads:
// unit u is the pieces at u*V and n + u*V (halves), or the one piece of pairs at
// u*V (interleaved). Bound by memory: 32768 tokens of 32 + 8 heads of 128 (bf16, a
// view of a fused projection) move 671 MB in 124 us, 5.4 TB/s; one thread per pair
// and head (below) took 289.
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
  bool first = true;
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
        float cc = 1.f, ss = 0.f;
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
        }
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

// Any number of pairs. One workgroup turns the heads [blockIdx.y * hpb, ...) of one token: one thread
// per pair (and per dim past the pairs) and head.
template <class T>
__global__ __launch_bounds__(256) void k_rotary_any(RotaryParams p, int hpb) {
  __shared__ float cs[kMaxPairs], sn[kMaxPairs];
  const int64_t tok = blockIdx.x;
  const int tid = threadIdx.x, n = p.n_pairs;
  if (tid < n) {
    const int ax = p.axis ? p.axis[tid] : 0;
    float c = 1.f, s = 0.f;
    if (ax < p.n_axes) angle(p.positions[tok * p.n_axes + ax], p.inv_freq[tid], c, s);
    cs[tid] = c;
    sn[tid] = p.inverse ? -s : s;
  }
  __syncthreads();
  const int units = p.dh - n;  // pairs, then single dims
  const int h0 = blockIdx.y * hpb, h1 = min(h0 + hpb, p.H + p.Hkv);
  for (int i = tid; i < (h1 - h0) * units; i += 256) {
    const int h = h0 + i / units, u = i % units;
    const T* src;
    T* dst;
    if (h < p.H) {
      src = static_cast<const T*>(p.q) + tok * p.q_stride + static_cast<int64_t>(h) * p.dh;
      dst = static_cast<T*>(p.q_out) + tok * p.qo_stride + static_cast<int64_t>(h) * p.dh;
    } else {
      src = static_cast<const T*>(p.k) + tok * p.k_stride + static_cast<int64_t>(h - p.H) * p.dh;
      dst = static_cast<T*>(p.k_out) + tok * p.ko_stride + static_cast<int64_t>(h - p.H) * p.dh;
    }
    if (u >= n) {
      dst[n + u] = src[n + u];
      continue;
    }
    const int a = p.interleaved ? 2 * u : u, b = p.interleaved ? 2 * u + 1 : n + u;
    const float xa = tof(src[a]), xb = tof(src[b]), c = cs[u], s = sn[u];
    dst[a] = fromf<T>(xa * c - xb * s);
    dst[b] = fromf<T>(xa * s + xb * c);
  }
}

template <class T>
void launch(const RotaryParams& p, hipStream_t s) {
  constexpr int V = 16 / sizeof(T);
  const int heads = p.H + p.Hkv;
  const size_t tok = static_cast<size_t>(p.B) * p.T;
  if ((p.interleaved ? 2 * p.n_pairs : p.n_pairs) % V) {
    constexpr int hpb = 16;
    const dim3 grid(static_cast<unsigned>(tok), (heads + hpb - 1) / hpb);
    hipLaunchKernelGGL(k_rotary_any<T>, grid, dim3(256), 0, s, p, hpb);
    return;
  }
  // a wave per token where there are tokens enough for every wave slot (256 CUs of
  // 16 waves and more): its cosines serve all heads; with fewer the heads are split
  const int chunk = tok >= 4096 ? heads : tok >= 1024 ? (heads + 1) / 2 : 8;
  const int chunks = (heads + chunk - 1) / chunk;
  const dim3 grid(static_cast<unsigned>((tok * chunks + 3) / 4));
  auto kern = p.interleaved ? k_rotary_rows<T, true> : k_rotary_rows<T, false>;
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
