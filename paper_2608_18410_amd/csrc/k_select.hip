// Few pages of a long history: the bounds of each page's keys, and the scores that pages
// are chosen by for each query.
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "launch.hpp"

namespace rolesub {
namespace {

// Bounds of a page's keys in every dim, a wave for each page and hpw heads: 16-byte pieces of
// its rows, then the lanes of one piece. fminf and fmaxf pass over NaN. Whole pages are
// gone over again, as what a page holds may have moved. Where a sequence ends inside a page
// that others have in the same place, the longest of them counts: all that write its
// bounds then write the same. A chain of loads (length, page, rows): 3 to 4 us for one
// of 32 heads, 5.0 for 8 sequences with a page of 64 tokens each. 256 sequences and 32 heads on
// pages of 16 take 8.4, 1024 22.4: 1.4 of it to look at the others' lengths and pages, where a
// look for each head took 3 and 47.
template <class T, int DH, int U>
__global__ __launch_bounds__(256) void k_page_bounds(BoundsParams p, int np, int hpw) {
  constexpr int V = 16 / sizeof(T), LPR = DH / V, RPI = 64 / LPR;
  __shared__ int s_n[4];
  const PagedCache& c = p.c;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nt = static_cast<int>(blockDim.x), nw = nt / 64, wh = nw * hpw;
  const int hb = (c.H + wh - 1) / wh, h0 = static_cast<int>(blockIdx.x % hb) * wh;
  const int i = static_cast<int>(blockIdx.x / hb % np), b = static_cast<int>(blockIdx.x / hb / np);
  const int64_t cap = static_cast<int64_t>(p.max_pages) << c.shift;
  const bool alone = p.B <= 64;  // a wave looks at all sequences itself
  const int first = p.lens[min(alone ? lane : tid, p.B - 1)];  // of the sequences, one a lane
  const int64_t len = min(static_cast<int64_t>(max(p.lens[b], 0)), cap);
  const int64_t pi = (max(len - p.T, static_cast<int64_t>(0)) >> c.shift) + i, t0 = pi << c.shift;
  if (t0 >= len) return;
  int n = static_cast<int>(min(len - t0, static_cast<int64_t>(c.page)));
  const int page = p.table[static_cast<int64_t>(b) * p.max_pages + pi];
  if (n < c.page) {
    for (int x = alone ? lane : tid; x < p.B; x += nt) {
      const int64_t other = min(static_cast<int64_t>(max(x < nt ? first : p.lens[x], 0)), cap);
      if (other > t0 + n && p.table[static_cast<int64_t>(x) * p.max_pages + pi] == page)
        n = static_cast<int>(min(other - t0, static_cast<int64_t>(c.page)));
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) n = max(n, __shfl_xor(n, o, kWave));
    if (!alone) {
      if (lane == 0) s_n[w] = n;
      __syncthreads();
      for (int x = 0; x < nw; ++x) n = max(n, s_n[x]);
    }
  }
  if (static_cast<uint32_t>(page) >= static_cast<uint32_t>(c.n_pages)) return;
  for (int h = h0 + w; h < min(h0 + wh, c.H); h += nw) {
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
        for (int v = 0; v < V; ++v) {
          lo[v] = fminf(lo[v], tof(x[v]));
          hi[v] = fmaxf(hi[v], tof(x[v]));
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
    u32x4 out;
    T* o = reinterpret_cast<T*>(&out);
#pragma unroll
    for (int x = 0; x < V; ++x) o[x] = fromf<T>(lane < LPR ? lo[x] : hi[x]);
    if (lane < 2 * LPR) *reinterpret_cast<u32x4*>(static_cast<char*>(p.bounds) + head * 2 * DH * sizeof(T) + lane * 16) = out;
  }
}

// What the lane D away (D in 1, 2, 4, 8, 16; within rows of 2 D lanes) holds.
template <int D>
__device__ __forceinline__ uint32_t away(uint32_t x) {
  constexpr int quad1 = 0xB1, quad2 = 0x4E, mirror8 = 0x141, mirror16 = 0x140, quad_back = 0x1B;
  if constexpr (D == 1) return __builtin_amdgcn_update_dpp(0, x, quad1, 0xF, 0xF, true);
  if constexpr (D == 2) return __builtin_amdgcn_update_dpp(0, x, quad2, 0xF, 0xF, true);
  // lane i of 8 holds what lane 7 - i did, then quads are turned back
  if constexpr (D == 4)
    return __builtin_amdgcn_update_dpp(0, __builtin_amdgcn_update_dpp(0, x, mirror8, 0xF, 0xF, true), quad_back, 0xF, 0xF, true);
  // 15 - i, then 7 - i
  if constexpr (D == 8)
    return __builtin_amdgcn_update_dpp(0, __builtin_amdgcn_update_dpp(0, x, mirror16, 0xF, 0xF, true), mirror8, 0xF, 0xF, true);
  if constexpr (D == 16) return __shfl_xor(x, 16, kWave);
}
template <int D>
__device__ __forceinline__ double away(double x) {
  u32x2 v = __builtin_bit_cast(u32x2, x);
  v[0] = away<D>(v[0]);
  v[1] = away<D>(v[1]);
  return __builtin_bit_cast(double, v);
}

// N sums over the lanes of a row, N = 2^k: each step leaves a lane half of them, the lower
// one where its bit D is clear, so that at the end the lanes hold one each (N > lanes: a
// few; N < lanes: several lanes the same). x[0 ..] are the lane's.
template <int D, int N>
__device__ __forceinline__ void share_sums(double* x) {
  if constexpr (D > 0) {
    if constexpr (N > 1) {
      const bool up = threadIdx.x & D;
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const double keep = up ? x[i + N / 2] : x[i], give = up ? x[i] : x[i + N / 2];
        x[i] = keep + away<D>(give);
      }
    } else {
      x[0] += away<D>(x[0]);
    }
    share_sums<D / 2, (N > 1 ? N / 2 : 1)>(x);
  }
}

// Tokens of sequence b that any query sees, and pages of them that query j does.
__device__ __forceinline__ int64_t tokens_of(const SelectParams& p, int b) {
  return min(min(static_cast<int64_t>(max(p.lens[b], 0)), static_cast<int64_t>(p.max_len)),
             static_cast<int64_t>(p.max_pages) << p.c.shift);
}
__device__ __forceinline__ int pages_of(const SelectParams& p, int b, int j, int64_t len) {
  if (p.visible) len = min(len, static_cast<int64_t>(max(p.visible[static_cast<int64_t>(b) * p.Tq + j], 0)));
  return static_cast<int>((len + p.c.page - 1) >> p.c.shift);
}

// Scores of a few pages of one key head for a sequence's queries, a wave's work: the
// highest that a key within the bounds could have, sum_d (q < 0 ? q lo : q hi), summed in
// 64 bits and rounded once, so that the choice does not hang on the order of the sum. A
// lane has a 16-byte piece of both bounds of a page, and its part of RC queries in 64
// bits; the lanes of a page add up. All bounds of a wave are asked for at once.
template <class T, int DH, int RC>
struct PageScores {
  // pages of a step, steps; lanes of a page; sums of a lane at the end, lanes with the same one
  static constexpr int V = 16 / sizeof(T), LPR = DH / V, PS = 64 / LPR, U = 4, N = RC * U;
  static constexpr int LEFT = N > LPR ? N / LPR : 1, SHARED = LPR > N ? LPR / N : 1;
  u32x4 lo[U], hi[U];
  uint32_t there = 0;

  // pages i0 .. i0 + PS U - 1 of `total`
  __device__ __forceinline__ void load(const SelectParams& p, int b, int h, int i0, int total) {
    const PagedCache& c = p.c;
    const int lane = threadIdx.x & 63;
    const int32_t* table = p.table + static_cast<int64_t>(b) * p.max_pages;
    there = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * PS + lane / LPR, page = i < total ? table[i] : -1;
      const bool in = static_cast<uint32_t>(page) < static_cast<uint32_t>(c.n_pages);
      there |= in ? 1u << u : 0u;
      const T* at = static_cast<const T*>(p.bounds) + (static_cast<int64_t>(in ? page : 0) * c.H + h) * 2 * DH + lane % LPR * V;
      lo[u] = *reinterpret_cast<const u32x4*>(at);
      hi[u] = *reinterpret_cast<const u32x4*>(at + DH);
    }
  }

  // put(i, score) for each of them, for query j
  template <class Put>
  __device__ __forceinline__ void score(const SelectParams& p, int b, int j, int h, int i0, int total, Put put) const {
    const PagedCache& c = p.c;
    const int lane = threadIdx.x & 63, lr = lane % LPR, d0 = lr * V;
    // The sums' numbers are 4 r + u, their bits from the highest those of the lane from
    // LPR / 2 on: the lane's steps and rows, and which of its LEFT sums are which.
    const int mine = lr / SHARED * LEFT;
    float best[LEFT];  // of the query's heads, of the rows that the lane has sums of
    bool nan[LEFT];
#pragma unroll
    for (int x = 0; x < LEFT; ++x) best[x] = -__builtin_inff(), nan[x] = false;
#pragma unroll 1
    for (int r0 = 0; r0 < p.rep; r0 += RC) {
      double q[RC][V], sum[N];
#pragma unroll
      for (int r = 0; r < RC; ++r) {  // past the last head: it again
        const u32x4 x = *reinterpret_cast<const u32x4*>(static_cast<const T*>(p.q) + (static_cast<int64_t>(b) * p.Tq + j) * p.q_stride +
                                                        (h * p.rep + min(r0 + r, p.rep - 1)) * DH + d0);
#pragma unroll
        for (int i = 0; i < V; ++i) q[r][i] = tof(reinterpret_cast<const T*>(&x)[i]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int r = 0; r < RC; ++r) {
          const T* l = reinterpret_cast<const T*>(&lo[u]);
          const T* g = reinterpret_cast<const T*>(&hi[u]);
          double x = 0.;
#pragma unroll
          for (int i = 0; i < V; ++i) x = __builtin_fma(q[r][i], static_cast<double>(q[r][i] < 0. ? tof(l[i]) : tof(g[i])), x);
          sum[r * U + u] = x;
        }
      share_sums<LPR / 2, N>(sum);
#pragma unroll
      for (int x = 0; x < LEFT; ++x) {
        const float y = static_cast<float>(sum[x]);
        best[x] = fmaxf(best[x], y);
        nan[x] |= y != y;
      }
    }
    // the highest over the rows, which lie on lanes LPR / 2 and LPR / 4 apart, in an order
    // in which NaN is above all numbers
#pragma unroll
    for (int x = 0; x < LEFT; ++x) {
      uint32_t k = nan[x] ? 0xFFFFFFFFu : order_key(best[x]);
      if constexpr (RC == 4) {
        k = max(k, away<LPR / 2>(k));
        k = max(k, away<LPR / 4>(k));
      }
      // lanes whose rows' bits are clear have the steps mine ..
      const int u = mine + x, i = i0 + u * PS + lane / LPR;
      if (mine < U && lr % SHARED == 0 && i < total)
        put(i, ((there >> (u & 3)) & 1u) && k != 0xFFFFFFFFu ? __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k) : __builtin_nanf(""));
    }
  }
};

// Long histories: the scores to memory, for the selection that follows. Bound by memory and
// by the 64-bit products: 8 sequences of 110001 to 131071 tokens, pages of 64 and 8 key
// heads of 4 rows (62 MB) 22 us, 2.8 TB/s, with the vector units busy for 10.
template <class T, int DH, int RC>
__global__ __launch_bounds__(256) void k_page_scores(SelectParams p, int np) {
  typedef PageScores<T, DH, RC> S;
  const PagedCache& c = p.c;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int lin = blockIdx.x;  // heads fastest: their bounds lie behind each other
  const int h = lin % c.H;
  lin /= c.H;
  const int i0 = (lin % np * 4 + w) * S::PS * S::U, b = lin / np;
  const int64_t len = tokens_of(p, b);
  if (i0 == 0)
    for (int j = lane; j < p.Tq; j += 64) p.counts[(static_cast<int64_t>(b) * p.Tq + j) * c.H + h] = pages_of(p, b, j, len);
  const int total = static_cast<int>((len + c.page - 1) >> c.shift);
  if (i0 >= total) return;
  S s;
  s.load(p, b, h, i0, total);
  for (int j = 0; j < p.Tq; ++j)
    s.score(p, b, j, h, i0, total, [&](int i, float x) { p.scores[((static_cast<int64_t>(b) * p.Tq + j) * c.H + h) * p.ld + i] = x; });
}

// Up to kFewPages pages: scores and choice in one workgroup for each query and key head. A
// page's rank is the number of pages above it, counted by a thread each: no histogram
// and three barriers, where the selection's own kernel has ten and a launch before it. 176
// pages of 32 heads 8 us (16 with 512 threads that rank in a loop of 32-bit halves), 128 of
// 32 sequences and 8 heads of 4 rows 9.5.
constexpr int kFewWg = 1024;
template <class T, int DH, int RC>
__global__ __launch_bounds__(kFewWg) void k_select_few(SelectParams p) {
  typedef PageScores<T, DH, RC> S;
  __shared__ __attribute__((aligned(16))) uint64_t s_key[kFewPages + 8];  // the score, then the lower index first
  __shared__ int s_cnt[kFewWg / 64];
  const PagedCache& c = p.c;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = blockIdx.x % c.H, j = blockIdx.x / c.H % p.Tq, b = blockIdx.x / c.H / p.Tq;
  const int n = pages_of(p, b, j, tokens_of(p, b));
  int32_t* out = p.sel + static_cast<int64_t>(blockIdx.x) * p.n_sel;
  if (n <= p.n_sel) {
    for (int i = tid; i < p.n_sel; i += kFewWg) out[i] = i < n ? i : -1;
    return;
  }
  // of pages [lo, hi) the `need` highest, equal ones by lower index
  const int lo = p.first, hi = n - p.recent, need = p.n_sel - p.first - p.recent;
  S s;
  for (int i0 = w * S::PS * S::U; i0 < n; i0 += kFewWg / 64 * S::PS * S::U) {
    s.load(p, b, h, i0, n);
    s.score(p, b, j, h, i0, n, [&](int i, float x) {
      s_key[i] = i >= lo && i < hi ? static_cast<uint64_t>(order_key(x)) << 32 | static_cast<uint32_t>(~i) : 0u;
    });
  }
  if (tid < 8) s_key[n + tid] = 0;  // n is below kFewPages + 1
  __syncthreads();
  int rank = 0;
  if (64 * w < n) {
    const uint64_t key = s_key[min(tid, n)];
#pragma unroll 1
    for (int x = 0; x < n; x += 8) {
      uint64_t k[8];
#pragma unroll
      for (int y = 0; y < 8; ++y) k[y] = s_key[x + y];
#pragma unroll
      for (int y = 0; y < 8; ++y) rank += k[y] > key;
    }
  }
  const bool on = tid < n && (tid < lo || tid >= hi || rank < need);
  const uint64_t all = __ballot(on);
  if (lane == 0) s_cnt[w] = __popcll(all);
  __syncthreads();
  int at = __popcll(all & ((1ull << lane) - 1ull));
#pragma unroll
  for (int v = 0; v < kFewWg / 64; ++v) at += v < w ? s_cnt[v] : 0;
  if (on) out[at] = tid;
}

}  // namespace

hipError_t launch_page_bounds(const BoundsParams& p, bool bf16, hipStream_t s) {
  const int np = static_cast<int>(std::min<int64_t>(p.max_pages, ((p.c.page - 1 + static_cast<int64_t>(p.T) - 1) >> p.c.shift) + 1));
  // a wave takes one head, or a workgroup takes all where looking at the other sequences is
  // more than a load, or workgroups are many anyway
  const int64_t pages = static_cast<int64_t>(p.B) * np;
  const int nw = std::min(p.c.H, 4), most = (p.c.H + nw - 1) / nw, hpw = p.B > 256 || pages * p.c.H > (1 << 20) ? most : 1;
  const int64_t wgs = pages * ((most + hpw - 1) / hpw);
  // loads of a wave in flight: a page's of up to 16 KB
  auto some = bf16 ? (p.c.dh == 128 ? k_page_bounds<__bf16, 128, 4> : k_page_bounds<__bf16, 64, 4>)
                   : (p.c.dh == 128 ? k_page_bounds<float, 128, 4> : k_page_bounds<float, 64, 4>);
  auto many = bf16 ? (p.c.dh == 128 ? k_page_bounds<__bf16, 128, 16> : k_page_bounds<__bf16, 64, 16>)
                   : (p.c.dh == 128 ? k_page_bounds<float, 128, 16> : k_page_bounds<float, 64, 16>);
  auto kern = p.c.page * p.c.dh * (bf16 ? 2 : 4) <= 4096 ? some : many;
  hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(wgs)), dim3(64 * nw), 0, s, p, np, hpw);
  return hipGetLastError();
}

hipError_t launch_page_scores(const SelectParams& p, bool bf16, hipStream_t s) {
  // pages of a workgroup's four waves: 64 of 256 bytes a bound, 128 of 128, 32 of 512
  const int wide = p.c.dh * (bf16 ? 2 : 4), some = 4 * 4 * 1024 / wide;
  const int np = std::max(1, (p.ld + some - 1) / some);  // one at least: it writes the counts
  const int64_t wgs = static_cast<int64_t>(p.B) * p.c.H * np;
  auto many = bf16 ? (p.c.dh == 128 ? k_page_scores<__bf16, 128, 4> : k_page_scores<__bf16, 64, 4>)
                   : (p.c.dh == 128 ? k_page_scores<float, 128, 4> : k_page_scores<float, 64, 4>);
  auto one = bf16 ? (p.c.dh == 128 ? k_page_scores<__bf16, 128, 1> : k_page_scores<__bf16, 64, 1>)
                  : (p.c.dh == 128 ? k_page_scores<float, 128, 1> : k_page_scores<float, 64, 1>);
  hipLaunchKernelGGL(p.rep == 1 ? one : many, dim3(static_cast<unsigned>(wgs)), dim3(256), 0, s, p, np);
  return hipGetLastError();
}

hipError_t launch_select_few(const SelectParams& p, bool bf16, hipStream_t s) {
  auto many = bf16 ? (p.c.dh == 128 ? k_select_few<__bf16, 128, 4> : k_select_few<__bf16, 64, 4>)
                   : (p.c.dh == 128 ? k_select_few<float, 128, 4> : k_select_few<float, 64, 4>);
  auto one = bf16 ? (p.c.dh == 128 ? k_select_few<__bf16, 128, 1> : k_select_few<__bf16, 64, 1>)
                  : (p.c.dh == 128 ? k_select_few<float, 128, 1> : k_select_few<float, 64, 1>);
  hipLaunchKernelGGL(p.rep == 1 ? one : many, dim3(static_cast<unsigned>(p.B) * p.Tq * p.c.H), dim3(kFewWg), 0, s, p);
  return hipGetLastError();
}

}  // namespace rolesub
