// Drafted tokens that form a tree: the bits of their ancestors, and the accepted path
// moved behind the cached tokens.
#include <algorithm>

#include "common.hpp"
#include "launch.hpp"

namespace rolesub {
namespace {

constexpr int kWords = kMaxTree / 32;

// One workgroup a tree, a thread a token. A token's bits cover its ancestors up to a
// distance that doubles each step, as it takes over those of the last ancestor it knows
// of and that one's last: T tokens need log2(T) steps however deep the tree. A load, the
// steps and a store behind each other: 1.8 us for one tree of 8, 4.9 for 32 of 24.
__global__ __launch_bounds__(kMaxTree) void k_tree_masks(TreeParams p) {
  __shared__ uint32_t s_bits[kMaxTree][kWords + 1];
  __shared__ int s_up[kMaxTree];
  const int j = threadIdx.x, words = (p.T + 31) / 32;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * p.T + j;
  const bool on = j < p.T;
  int up = -1;
  if (on) {
    up = p.parents[at];
    up = up >= 0 && up < j ? up : -1;
  }
  uint32_t bits[kWords];
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    bits[i] = j / 32 == i ? 1u << (j % 32) : 0u;
    s_bits[j][i] = bits[i];
  }
  s_up[j] = up;
  for (int d = 1; d < p.T; d *= 2) {
    __syncthreads();
    int next = -1;
    if (up >= 0) {
      next = s_up[up];
#pragma unroll
      for (int i = 0; i < kWords; ++i) bits[i] |= s_bits[up][i];
    }
    __syncthreads();
    up = next;
    s_up[j] = up;
#pragma unroll
    for (int i = 0; i < kWords; ++i) s_bits[j][i] = bits[i];
  }
  if (!on) return;
  int n = -1;
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    n += __popc(bits[i]);
    if (i < words) p.tree[at * words + i] = bits[i];
  }
  if (p.depth) p.depth[at] = n;
}

// The path of sequence b: the accepted token's bits in order.
struct Path {
  int n;        // tokens on it
  int64_t len;  // cached tokens before it
};
template <int NT>
__device__ __forceinline__ Path path_of(const AcceptParams& p, int b, int16_t* s_path, int* wsum, int* s_n) {
  const int tid = threadIdx.x, words = (p.T + 31) / 32, leaf = p.leaf[b];
  const int64_t cap = static_cast<int64_t>(p.max_pages) << p.c.shift;
  bool on = false;
  if (tid < p.T && leaf >= 0 && leaf < p.T)
    on = (p.tree[((p.trees > 1 ? static_cast<int64_t>(b) * p.T : 0) + leaf) * words + tid / 32] >> (tid % 32)) & 1u;
  const int before = group_scan<NT, false>(on, wsum);
  if (on) s_path[before] = static_cast<int16_t>(tid);
  if (tid == NT - 1) *s_n = before + on;
  __syncthreads();
  return Path{*s_n, min(static_cast<int64_t>(max(p.lens[b], 0)), cap)};
}

// Where tokens lie: the row of head 0 in K, and of their groups' first slot in V.
struct Place {
  int page, row;  // -1: none
};
__device__ __forceinline__ Place place_of(const AcceptParams& p, int b, int64_t t) {
  const PagedCache& c = p.c;
  if ((t >> c.shift) >= p.max_pages) return Place{-1, 0};
  const int page = p.table[static_cast<int64_t>(b) * p.max_pages + (t >> c.shift)];
  return Place{static_cast<uint32_t>(page) < static_cast<uint32_t>(c.n_pages) ? page : -1, static_cast<int>(t & (c.page - 1))};
}

// The i-th token of the path: where it comes from and goes, its mask and slots. The new
// slots start behind the last cached token's in the first page and at 0 in the others.
struct Move {
  Place from, to;
  uint32_t mask;
  int old_slot, slot;
};
template <int NT>
__device__ __forceinline__ Move move_of(const AcceptParams& p, int b, const Path& path, const int16_t* s_path, int* wsum, int* s_sum) {
  const PagedCache& c = p.c;
  const int tid = threadIdx.x, r0 = static_cast<int>(path.len & (c.page - 1));
  const uint32_t gm = group_bits(c.G);
  Move m = {{-1, 0}, {-1, 0}, 0u, 0, 0};
  int used = 0;
  if (tid < path.n) {
    m.from = place_of(p, b, path.len + s_path[tid]);
    m.to = place_of(p, b, path.len + tid);
    if (m.from.page >= 0) {
      const int64_t at = (static_cast<int64_t>(m.from.page) << c.shift) + m.from.row;
      m.mask = c.mask[at];
      m.old_slot = c.slot[at];
    }
    if (r0 + tid < c.page && r0 > 0 && m.to.page >= 0) {
      const int64_t at = (static_cast<int64_t>(m.to.page) << c.shift) + r0 - 1;
      used = c.slot[at] + __popc(c.mask[at] & gm);
    }
  }
  const int before = group_scan<NT, true>(__popc(m.mask & gm), wsum);
  if (tid < kMaxTree) s_sum[tid] = before;
  __syncthreads();
  const int first = max(((r0 + tid) & ~(c.page - 1)) - r0, 0);  // of the path's tokens in this page
  if (tid < path.n) m.slot = used + before - s_sum[first];
  return m;
}

// The keys and kept groups of hpb heads. Tokens move to lower places in ascending order,
// and so do their groups within a page, so what a step of the loop writes is read by no
// later one; within a step everything is read before anything is written. A page's other
// heads are other workgroups' and the masks and slots that all of them read are written
// by the next launch, unless a workgroup has all heads (WHOLE). VB: bytes of a value
// piece, the group's or 16. A chain of dependent loads (bits, length, pages, masks, rows): 5
// us for one of 8 drafted tokens and 32 heads; 32 sequences of 60 (15 MB each way) 9.5, and
// 3 for their masks and slots.
template <int VB> struct Bytes;
template <> struct Bytes<4> { typedef uint32_t t; };
template <> struct Bytes<8> { typedef u32x2 t; };
template <> struct Bytes<16> { typedef u32x4 t; };
template <int VB, int NT, bool WHOLE>
__global__ __launch_bounds__(NT) void k_accept(AcceptParams p, int hpb, int e) {
  typedef typename Bytes<VB>::t piece;
  __shared__ int16_t s_path[kMaxTree];
  __shared__ int wsum[NT / 64], s_n, s_sum[kMaxTree];
  __shared__ int64_t s_kfrom[kMaxTree], s_kto[kMaxTree], s_vfrom[kMaxTree], s_vto[kMaxTree];  // of head 0
  __shared__ int s_old[kMaxTree], s_new[kMaxTree], s_cnt[kMaxTree];
  const PagedCache& c = p.c;
  const int b = blockIdx.x, tid = threadIdx.x;
  const Path path = path_of<NT>(p, b, s_path, wsum, &s_n);
  if (WHOLE && tid == 0 && p.new_lens) p.new_lens[b] = static_cast<int32_t>(path.len + path.n);
  if (path.n == 0) return;
  const Move m = move_of<NT>(p, b, path, s_path, wsum, s_sum);
  const int row = c.dh * e, gb = c.ds * e;
  if (tid < path.n) {
    auto rows = [&](Place x) { return ((static_cast<int64_t>(x.page) * c.H) << c.shift) + x.row; };
    const bool same = m.from.page == m.to.page && m.from.row == m.to.row && m.old_slot == m.slot;
    s_kfrom[tid] = m.from.page < 0 ? -1 : rows(m.from);
    s_kto[tid] = m.to.page < 0 || same ? -1 : rows(m.to);
    s_vfrom[tid] = static_cast<int64_t>(m.from.page) * c.H * c.vcap;
    s_vto[tid] = static_cast<int64_t>(m.to.page) * c.H * c.vcap;
    s_old[tid] = m.old_slot;
    s_new[tid] = m.slot;
    s_cnt[tid] = __popc(m.mask & group_bits(c.G));
  }
  __syncthreads();
  const int h0 = blockIdx.y * hpb, nh = min(hpb, c.H - h0);
  const int kp = row / 16, vp = row / VB, gp = gb / VB, per = kp + vp, items = path.n * nh * per;
  for (int u0 = 0; u0 < items; u0 += NT * 4) {
    u32x4 xk[4];
    piece xv[4];
    char* to[4];
    bool key[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int u = u0 + NT * i + tid, q = u % per, h = h0 + u / per % nh, t = u / (per * nh);
      to[i] = nullptr;
      key[i] = q < kp;
      if (u >= items || s_kto[t] < 0) continue;
      if (key[i]) {
        xk[i] = u32x4{0, 0, 0, 0};
        const int64_t head = static_cast<int64_t>(h) << c.shift;
        if (s_kfrom[t] >= 0) xk[i] = *reinterpret_cast<const u32x4*>(static_cast<const char*>(c.K) + (s_kfrom[t] + head) * row + 16 * q);
        to[i] = static_cast<char*>(c.K) + (s_kto[t] + head) * row + 16 * q;
      } else {
        const int g = (q - kp) / gp;
        const uint32_t from = static_cast<uint32_t>(s_old[t]) + g, dst = static_cast<uint32_t>(s_new[t]) + g;
        if (g >= s_cnt[t] || dst >= static_cast<uint32_t>(c.vcap)) continue;
        const int64_t head = static_cast<int64_t>(h) * c.vcap;
        xv[i] = piece{};
        if (from < static_cast<uint32_t>(c.vcap))
          xv[i] = *reinterpret_cast<const piece*>(static_cast<const char*>(c.V) + (s_vfrom[t] + head + from) * gb + (q - kp) % gp * VB);
        to[i] = static_cast<char*>(c.V) + (s_vto[t] + head + dst) * gb + (q - kp) % gp * VB;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (!to[i]) continue;
      if (key[i])
        *reinterpret_cast<u32x4*>(to[i]) = xk[i];
      else
        *reinterpret_cast<piece*>(to[i]) = xv[i];
    }
  }
  if (WHOLE && tid < path.n && m.to.page >= 0) {
    const int64_t at = (static_cast<int64_t>(m.to.page) << c.shift) + m.to.row;
    c.mask[at] = m.mask;
    c.slot[at] = m.slot;
  }
}

// Their masks and slots, and the new lengths.
__global__ __launch_bounds__(256) void k_accept_meta(AcceptParams p) {
  __shared__ int16_t s_path[kMaxTree];
  __shared__ int wsum[4], s_n, s_sum[kMaxTree];
  const PagedCache& c = p.c;
  const int b = blockIdx.x, tid = threadIdx.x;
  const Path path = path_of<256>(p, b, s_path, wsum, &s_n);
  if (tid == 0 && p.new_lens) p.new_lens[b] = static_cast<int32_t>(path.len + path.n);
  if (path.n == 0) return;
  const Move m = move_of<256>(p, b, path, s_path, wsum, s_sum);
  __syncthreads();  // all is read
  if (tid < path.n && m.to.page >= 0) {
    const int64_t at = (static_cast<int64_t>(m.to.page) << c.shift) + m.to.row;
    c.mask[at] = m.mask;
    c.slot[at] = m.slot;
  }
}

}  // namespace

hipError_t launch_tree_masks(const TreeParams& p, hipStream_t s) {
  hipLaunchKernelGGL(k_tree_masks, dim3(static_cast<unsigned>(p.B)), dim3((p.T + 63) / 64 * 64), 0, s, p);
  return hipGetLastError();
}

// Pieces of a sequence up to which one workgroup moves them all. With the append before it:
// one sequence of 8 tokens and 32 heads (8 thousand) 24.2 -> 21.3 us against two launches, but
// 32 of 60 (61 thousand) 23.8 -> 29.3.
constexpr int64_t kWholePieces = 32768;
hipError_t launch_accept(const AcceptParams& p, bool bf16, hipStream_t s) {
  const int e = bf16 ? 2 : 4, gb = p.c.ds * e;
  // few pieces: one workgroup a sequence, without the second launch
  const int64_t pieces = static_cast<int64_t>(p.T) * p.c.H * (p.c.dh * e / 16 + p.c.dh * e / std::min(gb, 16));
  if (pieces <= kWholePieces) {
    auto kern = gb >= 16 ? k_accept<16, 1024, true> : gb == 8 ? k_accept<8, 1024, true> : k_accept<4, 1024, true>;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(p.B)), dim3(1024), 0, s, p, p.c.H, e);
    return hipGetLastError();
  }
  constexpr int hpb = 4;
  auto kern = gb >= 16 ? k_accept<16, 256, false> : gb == 8 ? k_accept<8, 256, false> : k_accept<4, 256, false>;
  hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(p.B), (p.c.H + hpb - 1) / hpb), dim3(256), 0, s, p, hpb, e);
  hipLaunchKernelGGL(k_accept_meta, dim3(static_cast<unsigned>(p.B)), dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace rolesub
