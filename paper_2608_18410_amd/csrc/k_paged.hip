// The paged routed cache's writers: new tokens appended (the pack of Sec. 3.2, a
// page at a time), and kept tokens moved to other pages.
#include "common.hpp"
#include "launch.hpp"

namespace rolesub {
namespace {

constexpr int kMaxPage = 256;

__device__ __forceinline__ uint32_t group_bits(int G) { return G >= 32 ? 0xFFFFFFFFu : (1u << G) - 1u; }

// Exclusive sum over the 256 threads of a workgroup.
__device__ __forceinline__ int scan256(int x, int* wsum) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int s = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(s, o, kWave);
    if (lane >= o) s += y;
  }
  if (lane == 63) wsum[w] = s;
  __syncthreads();
  int base = 0;
  for (int v = 0; v < w; ++v) base += wsum[v];
  return base + s - x;
}

template <int VB> struct Piece;
template <> struct Piece<4> { typedef uint32_t t; };
template <> struct Piece<8> { typedef u32x2 t; };
template <> struct Piece<16> { typedef u32x4 t; };

// New tokens of one page. One workgroup: sequence b, the i-th page its new tokens
// touch, heads [blockIdx.y * hpb, ...). The page's new tokens [t0, t1) take slots
// behind those its last cached token holds; an exclusive sum of their counts gives
// each its first. VB: bytes of a value piece, the group's or 16.
template <int VB>
__global__ __launch_bounds__(256) void k_append(AppendParams p, int np, int hpb, int e) {
  __shared__ uint32_t s_mask[kMaxPage];
  __shared__ int32_t s_slot[kMaxPage];
  __shared__ int wsum[4];
  typedef typename Piece<VB>::t piece;
  const PagedCache& c = p.c;
  const int b = blockIdx.x / np, i = blockIdx.x % np, tid = threadIdx.x;
  const int64_t cap = static_cast<int64_t>(p.max_pages) << c.shift;
  const int64_t len = min(static_cast<int64_t>(max(p.lens[b], 0)), cap);
  const int n = p.n_new ? min(max(p.n_new[b], 0), p.T) : p.T;
  const int64_t pg = (len >> c.shift) + i, t0 = max(pg << c.shift, len),
                t1 = min(min((pg + 1) << c.shift, len + n), cap);
  if (t0 >= t1) return;
  const int32_t page = p.table[static_cast<int64_t>(b) * p.max_pages + pg];
  if (static_cast<uint32_t>(page) >= static_cast<uint32_t>(c.n_pages)) return;
  const int m = static_cast<int>(t1 - t0), r0 = static_cast<int>(t0 & (c.page - 1));
  const int64_t j0 = static_cast<int64_t>(b) * p.T + (t0 - len);  // first new token's row of k, z and mask
  const int64_t meta = static_cast<int64_t>(page) << c.shift;
  const uint32_t gm = group_bits(c.G);
  const uint32_t mine = tid < m ? p.mask[j0 + tid] & gm : 0u;
  int base = 0;
  if (r0 > 0) base = c.slot[meta + r0 - 1] + __popc(c.mask[meta + r0 - 1] & gm);
  const int at = base + scan256(__popc(mine), wsum);
  if (tid < m) {
    s_mask[tid] = mine;
    s_slot[tid] = at;
    if (blockIdx.y == 0) {
      c.mask[meta + r0 + tid] = p.mask[j0 + tid];
      c.slot[meta + r0 + tid] = at;
    }
  }
  __syncthreads();
  const int h0 = blockIdx.y * hpb, nh = min(hpb, c.H - h0);
  const int row = c.dh * e, kp = row / 16, vp = row / VB, gb = c.ds * e;
  // keys: [head][token][piece] in the page's order
  for (int u = tid; u < nh * m * kp; u += 256) {
    const int q = u % kp, t = (u / kp) % m, h = h0 + u / (kp * m);
    const u32x4 x = *reinterpret_cast<const u32x4*>(static_cast<const char*>(p.k) + (j0 + t) * p.k_stride * e +
                                                    static_cast<int64_t>(h) * row + 16 * q);
    *reinterpret_cast<u32x4*>(static_cast<char*>(c.K) +
                              (((static_cast<int64_t>(page) * c.H + h) << c.shift) + r0 + t) * row + 16 * q) = x;
  }
  for (int u = tid; u < nh * m * vp; u += 256) {
    const int q = u % vp, t = (u / vp) % m, h = h0 + u / (vp * m);
    const int g = q * VB / gb;
    const uint32_t mk = s_mask[t];
    const int sl = s_slot[t] + __popc(mk & ((1u << g) - 1u));
    if (!((mk >> g) & 1u) || static_cast<uint32_t>(sl) >= static_cast<uint32_t>(c.vcap)) continue;
    const piece x = *reinterpret_cast<const piece*>(static_cast<const char*>(p.z) + (j0 + t) * p.z_stride * e +
                                                    static_cast<int64_t>(h) * row + VB * q);
    *reinterpret_cast<piece*>(static_cast<char*>(c.V) +
                              ((static_cast<int64_t>(page) * c.H + h) * c.vcap + sl) * gb + (q * VB) % gb) = x;
  }
}

// Kept tokens into one new page. One workgroup: sequence b, its i-th new page,
// heads [blockIdx.y * hpb, ...). Each new token's source page, row and slot come
// from its old index; its new slots from an exclusive sum over the page.
template <int VB>
__global__ __launch_bounds__(256) void k_compact(CompactParams p, int np, int hpb, int e) {
  __shared__ uint32_t s_mask[kMaxPage];
  __shared__ int32_t s_slot[kMaxPage], s_from[kMaxPage], s_page[kMaxPage], s_row[kMaxPage];
  __shared__ int wsum[4];
  typedef typename Piece<VB>::t piece;
  const PagedCache &c = p.src, &d = p.dst;
  const int b = blockIdx.x / np, i = blockIdx.x % np, tid = threadIdx.x;
  const int n = min(max(p.n_keep[b], 0), p.keep);
  const int j0 = i << c.shift, m = min(n - j0, c.page);
  if (m <= 0) return;
  const uint32_t gm = group_bits(c.G);
  uint32_t mine = 0, whole = 0;
  int from = 0, spage = -1, srow = 0;
  if (tid < m) {
    const int32_t t = p.keep_idx[static_cast<int64_t>(b) * p.keep + j0 + tid];
    const int pi = t >> c.shift;
    if (t >= 0 && pi < p.max_pages) spage = p.table[static_cast<int64_t>(b) * p.max_pages + pi];
    if (static_cast<uint32_t>(spage) >= static_cast<uint32_t>(c.n_pages)) spage = -1;
    srow = t & (c.page - 1);
    if (spage >= 0) {
      const int64_t meta = (static_cast<int64_t>(spage) << c.shift) + srow;
      whole = c.mask[meta];
      mine = whole & gm;
      from = c.slot[meta];
    }
    if (p.mass_out && blockIdx.y == 0) {
      const bool in = t >= 0 && t < p.mass_ld;
      p.mass_out[static_cast<int64_t>(b) * p.mass_out_ld + j0 + tid] =
          in ? p.mass_in[static_cast<int64_t>(b) * p.mass_ld + t] : 0.f;
    }
  }
  if (i >= p.dst_max_pages) return;
  const int32_t page = p.dst_table[static_cast<int64_t>(b) * p.dst_max_pages + i];
  if (static_cast<uint32_t>(page) >= static_cast<uint32_t>(d.n_pages)) return;
  const int at = scan256(__popc(mine), wsum);
  if (tid < m) {
    s_mask[tid] = mine;
    s_slot[tid] = at;
    s_from[tid] = from;
    s_page[tid] = spage;
    s_row[tid] = srow;
    if (blockIdx.y == 0) {
      const int64_t meta = (static_cast<int64_t>(page) << c.shift) + tid;
      d.mask[meta] = whole;
      d.slot[meta] = at;
    }
  }
  __syncthreads();
  const int h0 = blockIdx.y * hpb, nh = min(hpb, c.H - h0);
  const int row = c.dh * e, kp = row / 16, vp = row / VB, gb = c.ds * e;
  for (int u = tid; u < nh * m * kp; u += 256) {
    const int q = u % kp, t = (u / kp) % m, h = h0 + u / (kp * m);
    u32x4 x = {0, 0, 0, 0};
    if (s_page[t] >= 0)
      x = *reinterpret_cast<const u32x4*>(
          static_cast<const char*>(c.K) +
          (((static_cast<int64_t>(s_page[t]) * c.H + h) << c.shift) + s_row[t]) * row + 16 * q);
    *reinterpret_cast<u32x4*>(static_cast<char*>(d.K) +
                              (((static_cast<int64_t>(page) * c.H + h) << c.shift) + t) * row + 16 * q) = x;
  }
  for (int u = tid; u < nh * m * vp; u += 256) {
    const int q = u % vp, t = (u / vp) % m, h = h0 + u / (vp * m);
    const int g = q * VB / gb;
    const uint32_t mk = s_mask[t];
    const int r = __popc(mk & ((1u << g) - 1u)), sl = s_slot[t] + r, fr = s_from[t] + r;
    if (!((mk >> g) & 1u) || static_cast<uint32_t>(sl) >= static_cast<uint32_t>(d.vcap)) continue;
    piece x = {};
    if (static_cast<uint32_t>(fr) < static_cast<uint32_t>(c.vcap))
      x = *reinterpret_cast<const piece*>(static_cast<const char*>(c.V) +
                                          ((static_cast<int64_t>(s_page[t]) * c.H + h) * c.vcap + fr) * gb +
                                          (q * VB) % gb);
    *reinterpret_cast<piece*>(static_cast<char*>(d.V) +
                              ((static_cast<int64_t>(page) * c.H + h) * d.vcap + sl) * gb + (q * VB) % gb) = x;
  }
}

}  // namespace

hipError_t launch_append(const AppendParams& p, bool bf16, hipStream_t s) {
  const int e = bf16 ? 2 : 4, gb = p.c.ds * e, hpb = 4;
  const int np = ((p.c.page - 1 + p.T - 1) >> p.c.shift) + 1;
  const dim3 grid(static_cast<unsigned>(p.B) * np, (p.c.H + hpb - 1) / hpb);
  auto kern = gb >= 16 ? k_append<16> : gb == 8 ? k_append<8> : k_append<4>;
  hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, p, np, hpb, e);
  return hipGetLastError();
}

hipError_t launch_compact(const CompactParams& p, bool bf16, hipStream_t s) {
  const int e = bf16 ? 2 : 4, gb = p.src.ds * e, hpb = 4;
  const int np = ((p.keep - 1) >> p.src.shift) + 1;
  const dim3 grid(static_cast<unsigned>(p.B) * np, (p.src.H + hpb - 1) / hpb);
  auto kern = gb >= 16 ? k_compact<16> : gb == 8 ? k_compact<8> : k_compact<4>;
  hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, p, np, hpb, e);
  return hipGetLastError();
}

}  // namespace rolesub
