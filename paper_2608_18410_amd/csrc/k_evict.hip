// Which tokens of a cache stay: the first, the latest, and of the others those
// with the most accumulated attention weight (equal ones by lower index).
//
// The weights become order-preserving 32-bit keys. The smallest key that stays is
// found digit by digit from the top (11, 11 and 10 bits): a histogram of the digit
// over the keys that share the digits found so far, and the digit at which the
// count from above reaches what is to be kept. A token then stays when its key is
// above that one, or equal to it with fewer equal ones before it than are left to
// keep; its place in the output is the count of such tokens before it.
// A call is a chain of short dependent steps; what it has to read (4 bytes a token)
// takes far less than the chain.
#include <algorithm>

#include "common.hpp"
#include "launch.hpp"

namespace rolesub {
namespace {

constexpr int kBins = 2048;
__device__ __forceinline__ constexpr int level_shift(int level) { return level == 0 ? 21 : level == 1 ? 10 : 0; }
__host__ __device__ __forceinline__ constexpr int level_bins(int level) { return level == 2 ? 1024 : 2048; }
// whether a key has the digits found before this level, and its digit there
__device__ __forceinline__ bool level_has(int level, uint32_t key, uint32_t found) {
  return level == 0 || (level == 1 ? key >> 21 : key >> 10) == found;
}
__device__ __forceinline__ int level_digit(int level, uint32_t key) {
  return (key >> level_shift(level)) & (level_bins(level) - 1);
}

// The largest digit that at least `need` (>= 1) keys reach, and how many are above
// it. Thread t holds the counts of bins top - j, top = NB - 1 - t * PER.
template <int NT, int PER>
__device__ __forceinline__ void find_digit(const int* cnt, int need, int* wsum, int* s_out, int& digit, int& above) {
  int mine = 0;
#pragma unroll
  for (int j = 0; j < PER; ++j) mine += cnt[j];
  int e = group_scan<NT, true>(mine, wsum);
  if (e < need && need <= e + mine) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      if (e < need && need <= e + cnt[j]) {
        s_out[0] = NT * PER - 1 - static_cast<int>(threadIdx.x) * PER - j;
        s_out[1] = e;
      }
      e += cnt[j];
    }
  }
  __syncthreads();
  digit = s_out[0];
  above = s_out[1];
}

struct Range {
  int len, n, lo, hi, need;  // tokens [lo, hi) compete for `need` places
};
__device__ __forceinline__ Range range_of(const EvictParams& p, int b) {
  Range r;
  r.len = min(max(p.lens[b], 0), p.max_len);
  r.n = min(r.len, p.keep);
  r.lo = p.first;
  r.hi = r.len - p.recent;
  r.need = p.keep - p.first - p.recent;
  return r;
}

// One workgroup per sequence of at most NT * ITS tokens, whose keys stay in registers.
// Bound by its barriers: 361 tokens 5.3 us, 2048 6.4.
template <int NT, int ITS>
__global__ __launch_bounds__(NT) void k_evict_one(EvictParams p) {
  constexpr int NW = NT / 64;
  __shared__ int hist[kBins];
  __shared__ int wsum[NW], s_out[2], cnt[ITS * NW];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const Range r = range_of(p, b);
  int32_t* out = p.keep_idx + static_cast<int64_t>(b) * p.keep;
  if (tid == 0) p.n_keep[b] = r.n;
  if (r.len <= p.keep) {
    for (int j = tid; j < p.keep; j += NT) out[j] = j < r.n ? j : -1;
    return;
  }
  const float* mass = p.mass + static_cast<int64_t>(b) * p.mass_ld;
  uint32_t key[ITS];
#pragma unroll
  for (int i = 0; i < ITS; ++i) {
    const int t = i * NT + tid;
    key[i] = t >= r.lo && t < r.hi ? order_key(mass[t]) : 0u;
  }
  uint32_t thr = 0xFFFFFFFFu;  // above every key
  int ties = 0;
  if (r.need > 0) {
    uint32_t found = 0;
    int need = r.need;
#pragma unroll
    for (int level = 0; level < 3; ++level) {
      constexpr int PER = kBins / NT;
      const int nb = level_bins(level);
      for (int i = tid; i < kBins; i += NT) hist[i] = 0;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < ITS; ++i) {
        const int t = i * NT + tid;
        if (t >= r.lo && t < r.hi && level_has(level, key[i], found)) atomicAdd(&hist[level_digit(level, key[i])], 1);
      }
      __syncthreads();
      int c[PER];
#pragma unroll
      for (int j = 0; j < PER; ++j) c[j] = hist[kBins - 1 - tid * PER - j];  // bins past nb hold zero
      int d, above;
      find_digit<NT, PER>(c, need, wsum, s_out, d, above);
      found = level == 0 ? d : found * nb + d;
      need -= above;
    }
    thr = found;
    ties = need;
  }
  uint64_t bg[ITS], be[ITS];
#pragma unroll
  for (int i = 0; i < ITS; ++i) {
    const int t = i * NT + tid;
    const bool mid = t >= r.lo && t < r.hi;
    bg[i] = __ballot(t < r.len && (!mid || key[i] > thr));
    be[i] = __ballot(mid && key[i] == thr);
    if (lane == 0) cnt[i * NW + w] = __popcll(bg[i]) | (__popcll(be[i]) << 16);
  }
  __syncthreads();
  const int mine = tid < ITS * NW ? cnt[tid] : 0;  // both counts stay below 2^15 in sum
  const int before = group_scan<NT, true>(mine, wsum);
  if (tid < ITS * NW) cnt[tid] = before;
  __syncthreads();
  const uint64_t below = (1ull << lane) - 1ull;
#pragma unroll
  for (int i = 0; i < ITS; ++i) {
    const int t = i * NT + tid, s = cnt[i * NW + w];
    const int pg = (s & 0xFFFF) + __popcll(bg[i] & below), pe = (s >> 16) + __popcll(be[i] & below);
    if (((bg[i] >> lane) & 1) || (((be[i] >> lane) & 1) && pe < ties)) out[pg + min(pe, ties)] = t;
  }
}

// Longer sequences: C chunks of each, a workgroup a chunk, a launch a level. Every
// workgroup leaves its histogram; those of the next launch add them up, each for
// itself, so that nothing is cleared and no count depends on an order. Bound by the four
// launches: 4 sequences of 131071 tokens 27 us, of which the 2.1 MB take 0.4.
struct EvictWs {
  uint16_t* hist[3];  // [B][C][bins], counts of at most kMaxChunk
  int* above[2];      // [B][C] keys above the digit found at levels 0, 1
  int* state[2];      // [B][2] digits found, keys left to keep, after levels 0, 1
};

constexpr int kPassWg = 512;
constexpr int kChunk = 4096;    // tokens of a workgroup's round: 8 a thread, all requested at once
constexpr int kMaxChunks = 64;  // histograms that each workgroup adds up
constexpr int kMaxWgs = 512;
constexpr int kMaxChunk = 61440;  // except where chunks would pass this (counts are kept in 16 bits)

template <int LEVEL>
__global__ __launch_bounds__(kPassWg) void k_evict_pass(EvictParams p, EvictWs ws, int C, int chunk) {
  constexpr int NT = kPassWg, ITS = kChunk / NT, NW = NT / 64;
  __shared__ int hist[LEVEL < 3 ? level_bins(LEVEL % 3) : 1];
  __shared__ int wsum[NT / 64], s_out[2], cnt[LEVEL == 3 ? 64 : 1];
  const int b = blockIdx.x / C, c = blockIdx.x % C, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  // the last level's histograms are asked for before anything else is known (rows past
  // the sequence's chunks are not counted)
  constexpr int L = LEVEL > 0 ? LEVEL - 1 : 0, PNB = level_bins(L), PER = PNB / NT, ROWS = LEVEL > 0 ? 32 : 1;
  typedef uint16_t vec __attribute__((ext_vector_type(PER)));
  const uint16_t* rows = ws.hist[L] + static_cast<int64_t>(b) * C * PNB + (PNB - (tid + 1) * PER);
  vec v[ROWS];
  if constexpr (LEVEL > 0)
#pragma unroll
    for (int x = 0; x < ROWS; ++x) v[x] = *reinterpret_cast<const vec*>(rows + static_cast<int64_t>(min(x, C - 1)) * PNB);
  const Range r = range_of(p, b);
  int32_t* out = p.keep_idx + static_cast<int64_t>(b) * p.keep;
  if (LEVEL == 3 && c == 0 && tid == 0) p.n_keep[b] = r.n;
  if (r.len <= p.keep) {
    if (LEVEL == 3)
      for (int64_t j = c * NT + tid; j < p.keep; j += static_cast<int64_t>(C) * NT) out[j] = j < r.n ? static_cast<int>(j) : -1;
    return;
  }
  const int t0 = c * chunk;  // chunk * C stays within 2^31
  if (t0 >= r.len) return;
  const int t1 = min(t0 + chunk, r.len), used = (r.len + chunk - 1) / chunk;
  const float* mass = p.mass + static_cast<int64_t>(b) * p.mass_ld;
  // the first round's weights (up to 64 chunks the only one) arrive meanwhile
  float first[ITS];
#pragma unroll
  for (int i = 0; i < ITS; ++i) {
    const int t = t0 + i * NT + tid;
    first[i] = t < t1 && t >= r.lo && t < r.hi ? mass[t] : 0.f;
  }
  uint32_t found = 0;
  int need = r.need, eq_before = 0, gt_before = 0;
  if (LEVEL > 0 && need > 0) {
    constexpr int NB = PNB;
    if (L > 0) {
      found = ws.state[L - 1][2 * b];
      need = ws.state[L - 1][2 * b + 1];
    }
    int sum[PER] = {}, own[PER] = {}, pre[PER] = {};
    for (int x0 = 0; x0 < used; x0 += ROWS) {
      if (x0 > 0)
#pragma unroll
        for (int x = 0; x < ROWS; ++x)
          v[x] = *reinterpret_cast<const vec*>(rows + static_cast<int64_t>(min(x0 + x, C - 1)) * PNB);
#pragma unroll
      for (int x = 0; x < ROWS; ++x)
#pragma unroll
        for (int j = 0; j < PER; ++j) {
          const int n = x0 + x < used ? v[x][PER - 1 - j] : 0;
          sum[j] += n;
          own[j] = x0 + x == c ? n : own[j];
          pre[j] += x0 + x < c ? n : 0;
        }
    }
    int d, above;
    find_digit<NT, PER>(sum, need, wsum, s_out, d, above);
    found = L == 0 ? d : found * NB + d;
    need -= above;
    int mine = 0, eq = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int bin = NB - 1 - tid * PER - j;
      mine += bin > d ? (LEVEL == 3 ? pre[j] : own[j]) : 0;
      eq += bin == d ? pre[j] : 0;
    }
    if (LEVEL < 3) {
      const int a = group_scan<NT, true>(mine, wsum) + mine;  // the last thread holds the sum
      if (tid == NT - 1) ws.above[L][static_cast<int64_t>(b) * C + c] = a;
      if (c == 0 && tid == 0) {
        ws.state[L][2 * b] = found;
        ws.state[L][2 * b + 1] = need;
      }
    } else {
      for (int x = tid; x < c; x += NT)
        mine += ws.above[0][static_cast<int64_t>(b) * C + x] + ws.above[1][static_cast<int64_t>(b) * C + x];
      const int g = group_scan<NT, true>(mine, wsum) + mine;
      if (tid == NT - 1) s_out[0] = g;  // s_out was read before the scan's barriers
      const int e = group_scan<NT, true>(eq, wsum) + eq;
      if (tid == NT - 1) s_out[1] = e;
      __syncthreads();
      gt_before = s_out[0];
      eq_before = s_out[1];
    }
  }
  if constexpr (LEVEL < 3) {
    constexpr int NB = level_bins(LEVEL % 3);
    if (need <= 0 && r.need <= 0) return;
    for (int i = tid; i < NB; i += NT) hist[i] = 0;
    __syncthreads();
    for (int s0 = t0; s0 < t1; s0 += kChunk)
#pragma unroll
      for (int i = 0; i < ITS; ++i) {
        const int t = s0 + i * NT + tid;
        if (t >= t1 || t < r.lo || t >= r.hi) continue;
        const uint32_t k = order_key(s0 == t0 ? first[i] : mass[t]);
        if (level_has(LEVEL, k, found)) atomicAdd(&hist[level_digit(LEVEL, k)], 1);
      }
    __syncthreads();
    uint16_t* h = ws.hist[LEVEL] + (static_cast<int64_t>(b) * C + c) * NB;
    for (int i = tid; i < NB; i += NT) h[i] = static_cast<uint16_t>(hist[i]);
  } else {
    const uint32_t thr = r.need > 0 ? found : 0xFFFFFFFFu;
    const int ties = r.need > 0 ? need : 0;
    // safe tokens before the chunk
    gt_before += min(t0, r.lo) + max(0, t0 - r.hi);
    for (int s0 = t0; s0 < t1; s0 += ITS * NT) {
      uint64_t bg[ITS], be[ITS];
#pragma unroll
      for (int i = 0; i < ITS; ++i) {
        const int t = s0 + i * NT + tid;
        const bool in = t < t1, mid = in && t >= r.lo && t < r.hi;
        const uint32_t k = mid ? order_key(s0 == t0 ? first[i] : mass[t]) : 0u;
        bg[i] = __ballot(in && (!mid || k > thr));
        be[i] = __ballot(mid && k == thr);
      }
      __syncthreads();  // the last round's counts were read
#pragma unroll
      for (int i = 0; i < ITS; ++i)
        if (lane == 0) cnt[i * NW + w] = __popcll(bg[i]) | (__popcll(be[i]) << 16);
      __syncthreads();
      // the 64 counts: every wave adds them up for itself
      const int mine = cnt[lane];
      int s = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(s, o, kWave);
        if (lane >= o) s += y;
      }
      const int all = __shfl(s, 63, kWave), before = s - mine;
      const uint64_t below = (1ull << lane) - 1ull;
#pragma unroll
      for (int i = 0; i < ITS; ++i) {
        const int q = __shfl(before, i * NW + w, kWave);
        const int pg = gt_before + (q & 0xFFFF) + __popcll(bg[i] & below);
        const int pe = eq_before + (q >> 16) + __popcll(be[i] & below);
        if (((bg[i] >> lane) & 1) || (((be[i] >> lane) & 1) && pe < ties)) out[pg + min(pe, ties)] = s0 + i * NT + tid;
      }
      gt_before += all & 0xFFFF;
      eq_before += all >> 16;
    }
  }
}

constexpr int kOneWg = 16384;   // tokens whose keys one workgroup holds in registers

// Tokens of a workgroup: a round, or more where a sequence or the batch has many (each
// workgroup adds up the histograms of all its sequence's: 66 sequences of 63549 tokens
// 128 -> 118 us with compaction, 20 of 131071 76 -> 72).
int chunk_of(int B, int max_len) {
  const int64_t c = std::max((static_cast<int64_t>(max_len) + kMaxChunks - 1) / kMaxChunks,
                             (static_cast<int64_t>(max_len) * B + kMaxWgs - 1) / kMaxWgs);
  return static_cast<int>(std::min<int64_t>(kMaxChunk, std::max<int64_t>(kChunk, (c + kChunk - 1) / kChunk * kChunk)));
}

size_t hist_bytes(size_t n) { return (n * (2048 + 2048 + 1024) * sizeof(uint16_t) + 15) & ~static_cast<size_t>(15); }

}  // namespace

size_t evict_ws_bytes(int B, int max_len) {
  if (max_len <= kOneWg) return 0;
  // at least the chunks of every shorter length
  const size_t C = std::max(std::min((max_len + kChunk - 1) / kChunk, kMaxChunks), (max_len + kMaxChunk - 1) / kMaxChunk);
  return hist_bytes(B * C) + (B * C * 2 + static_cast<size_t>(B) * 4) * sizeof(int);
}

hipError_t launch_evict(const EvictParams& p, hipStream_t s) {
  const dim3 one(static_cast<unsigned>(p.B));
  if (p.max_len <= 1024) {
    hipLaunchKernelGGL((k_evict_one<256, 4>), one, dim3(256), 0, s, p);
  } else if (p.max_len <= 2048) {
    hipLaunchKernelGGL((k_evict_one<512, 4>), one, dim3(512), 0, s, p);
  } else if (p.max_len <= 4096) {
    hipLaunchKernelGGL((k_evict_one<1024, 4>), one, dim3(1024), 0, s, p);
  } else if (p.max_len <= kOneWg) {
    hipLaunchKernelGGL((k_evict_one<1024, 16>), one, dim3(1024), 0, s, p);
  } else {
    const int chunk = chunk_of(p.B, p.max_len), C = (p.max_len + chunk - 1) / chunk;
    const size_t n = static_cast<size_t>(p.B) * C;
    EvictWs ws;
    uint16_t* bins = static_cast<uint16_t*>(p.ws);
    for (int l = 0; l < 3; ++l) {
      ws.hist[l] = bins;
      bins += n * level_bins(l);
    }
    int* at = reinterpret_cast<int*>(static_cast<char*>(p.ws) + hist_bytes(n));
    for (int l = 0; l < 2; ++l) {
      ws.above[l] = at;
      at += n;
    }
    for (int l = 0; l < 2; ++l) {
      ws.state[l] = at;
      at += 2 * static_cast<size_t>(p.B);
    }
    const dim3 grid(static_cast<unsigned>(n));
    hipLaunchKernelGGL(k_evict_pass<0>, grid, dim3(kPassWg), 0, s, p, ws, C, chunk);
    hipLaunchKernelGGL(k_evict_pass<1>, grid, dim3(kPassWg), 0, s, p, ws, C, chunk);
    hipLaunchKernelGGL(k_evict_pass<2>, grid, dim3(kPassWg), 0, s, p, ws, C, chunk);
    hipLaunchKernelGGL(k_evict_pass<3>, grid, dim3(kPassWg), 0, s, p, ws, C, chunk);
  }
  return hipGetLastError();
}

}  // namespace rolesub
