// Few pages of a long history: the bounds of each page's keys, and the scores that pages
// are chosen by for each query.
#include <algorithm>

#include "common.hpp"
#include "launch.hpp"

namespace rolesub {
namespace {

// Bounds of a page's keys in every dim, a wave for each page and head: 16-byte pieces of
// its rows, then the lanes of one piece. fminf and fmaxf pass over NaN. Whole pages are
// gone over again, as what a page holds may have moved.
template <class T, int DH>
__global__ __launch_bounds__(256) void k_page_bounds(BoundsParams p, int np) {
  constexpr int V = 16 / sizeof(T), LPR = DH / V, RPI = 64 / LPR, U = 4;
  const PagedCache& c = p.c;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t job = static_cast<int64_t>(blockIdx.x) * 4 + w, pages = static_cast<int64_t>(p.B) * np;
  if (job >= pages * c.H) return;
  const int h = static_cast<int>(job % c.H), i = static_cast<int>(job / c.H % np), b = static_cast<int>(job / c.H / np);
  const int64_t cap = static_cast<int64_t>(p.max_pages) << c.shift;
  const int64_t len = min(static_cast<int64_t>(max(p.lens[b], 0)), cap);
  const int64_t pi = (max(len - p.T, static_cast<int64_t>(0)) >> c.shift) + i, t0 = pi << c.shift;
  if (t0 >= len) return;
  const int page = p.table[static_cast<int64_t>(b) * p.max_pages + pi];
  if (static_cast<uint32_t>(page) >= static_cast<uint32_t>(c.n_pages)) return;
  const int n = static_cast<int>(min(len - t0, static_cast<int64_t>(c.page)));
  const int64_t head = static_cast<int64_t>(page) * c.H + h;
  const char* k = static_cast<const char*>(c.K) + (head << c.shift) * DH * static_cast<int64_t>(sizeof(T)) + lane % LPR * 16;
  float lo[V], hi[V];
#pragma unroll
  for (int x = 0; x < V; ++x) lo[x] = __builtin_inff(), hi[x] = -__builtin_inff();
  for (int r0 = lane / LPR; r0 < n; r0 += RPI * U) {
    u32x4 a[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {  // past the last row: it again
      const int r = min(r0 + u * RPI, n - 1);
      a[u] = *reinterpret_cast<const u32x4*>(k + r * DH * static_cast<int>(sizeof(T)));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const T* x = reinterpret_cast<const T*>(&a[u]);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        lo[i] = fminf(lo[i], tof(x[i]));
        hi[i] = fmaxf(hi[i], tof(x[i]));
      }
    }
  }
#pragma unroll
  for (int o = LPR; o < 64; o <<= 1)
#pragma unroll
    for (int x = 0; x < V; ++x) {
      lo[x] = fminf(lo[x], __shfl_xor(lo[x], o, kWave));
      hi[x] = fmaxf(hi[x], __shfl_xor(hi[x], o, kWave));
    }
  if (lane >= 2 * LPR) return;
  u32x4 out;
  T* o = reinterpret_cast<T*>(&out);
#pragma unroll
  for (int x = 0; x < V; ++x) o[x] = fromf<T>(lane < LPR ? lo[x] : hi[x]);
  *reinterpret_cast<u32x4*>(static_cast<char*>(p.bounds) + head * 2 * DH * sizeof(T) + lane * 16) = out;
}

// Scores of 64 pages of one key head for the rows of a sequence: the highest that a key
// within the bounds could have, sum_d (q < 0 ? q lo : q hi) = sum_d (q- lo + q+ hi), summed in
// 64 bits (the products are exact there) and rounded once, so that the choice does not
// hang on the order of the sum. A page a lane, a quarter of the dims a wave; the queries'
// parts come from LDS, the same for all lanes.
template <class T, int DH, int RC>
__global__ __launch_bounds__(256) void k_page_scores(SelectParams p, int np) {
  constexpr int V = 16 / sizeof(T), ROWB = 2 * DH * sizeof(T), LD = ROWB + 16, QD = DH / 4;
  __shared__ __attribute__((aligned(16))) char s_b[64 * LD];
  __shared__ __attribute__((aligned(16))) double s_q[RC][2][DH];
  __shared__ double s_sum[4][RC][64];
  const PagedCache& c = p.c;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  int lin = blockIdx.x;
  const int i0 = lin % np * 64;
  lin /= np;
  const int h = lin % c.H, b = lin / c.H;
  const int32_t* table = p.table + static_cast<int64_t>(b) * p.max_pages;
  const int64_t len = min(min(static_cast<int64_t>(max(p.lens[b], 0)), static_cast<int64_t>(p.max_len)),
                          static_cast<int64_t>(p.max_pages) << c.shift);
  auto pages_of = [&](int j) {
    const int64_t n = p.visible ? min(len, static_cast<int64_t>(max(p.visible[static_cast<int64_t>(b) * p.Tq + j], 0))) : len;
    return static_cast<int>((n + c.page - 1) >> c.shift);
  };
  if (i0 == 0)
    for (int j = tid; j < p.Tq; j += 256) p.counts[(static_cast<int64_t>(b) * p.Tq + j) * c.H + h] = pages_of(j);
  const int total = static_cast<int>((len + c.page - 1) >> c.shift);
  if (i0 >= total) return;
  // the bounds, rows of whole pieces
  constexpr int LPR = ROWB / 16;
  for (int u = tid; u < 64 * LPR; u += 256) {
    const int i = i0 + u / LPR;
    const int page = i < total ? table[i] : -1;
    u32x4 x = {0, 0, 0, 0};
    if (static_cast<uint32_t>(page) < static_cast<uint32_t>(c.n_pages))
      x = *reinterpret_cast<const u32x4*>(static_cast<const char*>(p.bounds) + (static_cast<int64_t>(page) * c.H + h) * ROWB + u % LPR * 16);
    *reinterpret_cast<u32x4*>(s_b + u / LPR * LD + u % LPR * 16) = x;
  }
  const int mine = i0 + lane < total ? table[i0 + lane] : -1;
  const bool there = static_cast<uint32_t>(mine) < static_cast<uint32_t>(c.n_pages);
  const int rows = p.Tq * p.rep;
  float best = -__builtin_inff();
  bool nan = false;
  for (int r0 = 0; r0 < rows; r0 += RC) {
    __syncthreads();
    for (int u = tid; u < RC * DH; u += 256) {
      const int r = r0 + u / DH, d = u % DH;
      float q = 0.f;
      if (r < rows)
        q = tof(static_cast<const T*>(p.q)[(static_cast<int64_t>(b) * p.Tq + r / p.rep) * p.q_stride + (h * p.rep + r % p.rep) * DH + d]);
      s_q[u / DH][0][d] = q < 0.f ? static_cast<double>(q) : 0.;
      s_q[u / DH][1][d] = q < 0.f ? 0. : static_cast<double>(q);  // NaN here
    }
    __syncthreads();
    double sum[RC];
#pragma unroll
    for (int r = 0; r < RC; ++r) sum[r] = 0.;
#pragma unroll 1
    for (int d = w * QD; d < (w + 1) * QD; d += V)
#pragma unroll
      for (int side = 0; side < 2; ++side) {
        const u32x4 a = *reinterpret_cast<const u32x4*>(s_b + lane * LD + (side * DH + d) * sizeof(T));
        const T* x = reinterpret_cast<const T*>(&a);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const double y = tof(x[i]);
#pragma unroll
          for (int r = 0; r < RC; ++r) sum[r] = __builtin_fma(s_q[r][side][d + i], y, sum[r]);
        }
      }
#pragma unroll
    for (int r = 0; r < RC; ++r) s_sum[w][r][lane] = sum[r];
    __syncthreads();
    // the first wave, row after row: of a query's heads the highest
    if (w == 0) {
      for (int r = 0; r < RC && r0 + r < rows; ++r) {
        float x = static_cast<float>((s_sum[0][r][lane] + s_sum[1][r][lane]) + (s_sum[2][r][lane] + s_sum[3][r][lane]));
        if (__any(x != x)) {  // an infinite bound times the zero of the other side's part
          double y = 0.;
#pragma unroll 1
          for (int d = 0; d < DH; ++d) {
            const bool low = s_q[r][0][d] != 0.;
            y += s_q[r][low ? 0 : 1][d] * tof(reinterpret_cast<const T*>(s_b + lane * LD)[low ? d : DH + d]);
          }
          x = x != x ? static_cast<float>(y) : x;
        }
        best = fmaxf(best, x);
        nan |= x != x;
        const int rr = r0 + r;
        if (rr % p.rep == p.rep - 1) {
          if (i0 + lane < total)
            p.scores[((static_cast<int64_t>(b) * p.Tq + rr / p.rep) * c.H + h) * p.ld + i0 + lane] =
                there && !nan ? best : __builtin_nanf("");
          best = -__builtin_inff();
          nan = false;
        }
      }
    }
  }
}

}  // namespace

hipError_t launch_page_bounds(const BoundsParams& p, bool bf16, hipStream_t s) {
  const int np = static_cast<int>(std::min<int64_t>(p.max_pages, ((p.c.page - 1 + static_cast<int64_t>(p.T) - 1) >> p.c.shift) + 1));
  const int64_t jobs = static_cast<int64_t>(p.B) * np * p.c.H;
  auto kern = bf16 ? (p.c.dh == 128 ? k_page_bounds<__bf16, 128> : k_page_bounds<__bf16, 64>)
                   : (p.c.dh == 128 ? k_page_bounds<float, 128> : k_page_bounds<float, 64>);
  hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>((jobs + 3) / 4)), dim3(256), 0, s, p, np);
  return hipGetLastError();
}

hipError_t launch_page_scores(const SelectParams& p, bool bf16, hipStream_t s) {
  const int np = std::max(1, (p.ld + 63) / 64);  // one at least: it writes the counts
  const int64_t wgs = static_cast<int64_t>(p.B) * p.c.H * np;
  constexpr int RC = 4;
  auto kern = bf16 ? (p.c.dh == 128 ? k_page_scores<__bf16, 128, RC> : k_page_scores<__bf16, 64, RC>)
                   : (p.c.dh == 128 ? k_page_scores<float, 128, RC> : k_page_scores<float, 64, RC>);
  hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(wgs)), dim3(256), 0, s, p, np);
  return hipGetLastError();
}

}  // namespace rolesub
