// Which tokens of a cache stay: the first, the latest, and of the others those
// with the most accumulated attention weight.
#include "common.hpp"
#include "launch.hpp"

namespace rolesub {
namespace {

// One workgroup of 1024 threads per sequence. The weights become order-preserving
// keys; the smallest key that stays is found bit by bit (32 counts), then the kept
// tokens are written in index order by a running sum over chunks of 1024.
__global__ __launch_bounds__(1024) void k_evict(EvictParams p) {
  __shared__ int cnt[2][16];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int len = min(max(p.lens[b], 0), p.max_len), n = min(len, p.keep);
  int32_t* out = p.keep_idx + static_cast<int64_t>(b) * p.keep;
  if (tid == 0) p.n_keep[b] = n;
  for (int j = n + tid; j < p.keep; j += 1024) out[j] = -1;
  if (len <= p.keep) {
    for (int j = tid; j < n; j += 1024) out[j] = j;
    return;
  }
  const float* mass = p.mass + static_cast<int64_t>(b) * p.mass_ld;
  const int lo = p.first, hi = len - p.recent, need = p.keep - p.first - p.recent;
  int turn = 0;
  auto total = [&](int c) {  // sum over the workgroup of a per-wave count
    if (lane == 0) cnt[turn][w] = c;
    __syncthreads();
    int s = 0;
    for (int v = 0; v < 16; ++v) s += cnt[turn][v];
    turn ^= 1;
    return s;
  };
  uint32_t thr = 0;  // largest key that at least `need` tokens reach
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t t = thr | (1u << bit);
    int c = 0;
    for (int i = lo + tid; i - tid < hi; i += 1024) c += __popcll(__ballot(i < hi && order_key(mass[i]) >= t));
    if (total(c) >= need) thr = t;
  }
  int c = 0;
  for (int i = lo + tid; i - tid < hi; i += 1024) c += __popcll(__ballot(i < hi && order_key(mass[i]) > thr));
  const int ties = need - total(c);  // equal keys to keep, the lowest indices first
  int at = 0, eq = 0;
  for (int i0 = 0; i0 < len; i0 += 1024) {
    const int i = i0 + tid;
    const bool safe = i < len && (i < lo || i >= hi), mid = i < len && !safe;
    const uint32_t k = mid ? order_key(mass[i]) : 0u;
    const uint64_t be = __ballot(mid && k == thr), below = (1ull << lane) - 1ull;
    if (lane == 0) cnt[turn][w] = __popcll(be);
    __syncthreads();
    int pe = eq + __popcll(be & below);
    for (int v = 0; v < 16; ++v) {
      pe += v < w ? cnt[turn][v] : 0;
      eq += cnt[turn][v];
    }
    turn ^= 1;
    const bool kept = safe || (mid && (k > thr || (k == thr && pe < ties)));
    const uint64_t bk = __ballot(kept);
    if (lane == 0) cnt[turn][w] = __popcll(bk);
    __syncthreads();
    int pk = at + __popcll(bk & below);
    for (int v = 0; v < 16; ++v) {
      pk += v < w ? cnt[turn][v] : 0;
      at += cnt[turn][v];
    }
    turn ^= 1;
    if (kept) out[pk] = i;
  }
}

}  // namespace

size_t evict_ws_bytes(int B, int max_len) {
  (void)B;
  (void)max_len;
  return 0;
}

hipError_t launch_evict(const EvictParams& p, hipStream_t s) {
  hipLaunchKernelGGL(k_evict, dim3(static_cast<unsigned>(p.B)), dim3(1024), 0, s, p);
  return hipGetLastError();
}

}  // namespace rolesub
