// The paged routed cache's writers: new tokens appended (the pack of Sec. 3.2, a
// page at a time), and kept tokens moved to other pages.
#include "common.hpp"
#include "launch.hpp"

namespace rolesub {
namespace {

constexpr int kMaxPage = 256;

template <int VB> struct Piece;
template <> struct Piece<4> { typedef uint32_t t; };
template <> struct Piece<8> { typedef u32x2 t; };
template <> struct Piece<16> { typedef u32x4 t; };

// A few new tokens of one page, every piece of its heads a thread's. One workgroup: sequence b, the i-th page its new tokens
// touch, heads [blockIdx.y * hpb, ...). The page's new tokens [t0, t1) take slots
// behind those its last cached token holds; an exclusive sum of their counts gives
// each its first. VB: bytes of a value piece, the group's or 16. Bound by the chain length,
// page, last token, copy: 64 new tokens of 32 heads (0.4 MB) 3.7 us.
template <int VB>
__global__ __launch_bounds__(256) void k_append_few(AppendParams p, int np, int hpb, int e) {
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
  const int at = base + group_scan<256, false>(__popc(mine), wsum);
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

// What a workgroup knows of its page's tokens while it copies them: the row each
// token's key comes from (of head 0; negative: zeros), how far its groups' slots move
// (of head 0), and whose group every slot holds (kNone: zeros).
constexpr uint16_t kNone = 0xFFFF;
struct PageMap {
  int64_t krow[kMaxPage], vmove[kMaxPage];
  uint16_t owner[kMaxPage * 32];
};

// Plain accesses, or ones that leave the caches to other data: a move reads and writes
// each byte once, and what it writes is not read soon (32 sequences of up to 2048
// tokens 49 -> 44 us with the selection, 16 of 32 heads 68 -> 60, 4 of 131071 80 -> 73).
// Appended tokens are read by the next attention call and stay.
template <bool NT, class P>
__device__ __forceinline__ P get(const P* p) {
  if constexpr (NT) return __builtin_nontemporal_load(p);
  return *p;
}
template <bool NT, class P>
__device__ __forceinline__ void put(P x, P* p) {
  if constexpr (NT)
    __builtin_nontemporal_store(x, p);
  else
    *p = x;
}

// Rows and slots of HB heads from h0, the same piece of every head by one thread, so
// that HB * U loads are on their way at once and each address is worked out once.
// Keys: rows of 2^lkp pieces; tokens [0, m) go to rows r0 + t of the page. Values:
// slots [0, slots), whole groups of gb bytes in pieces of VB.
template <int VB, int HB, bool NT>
__device__ __forceinline__ void copy_page(const PageMap& g, const char* ksrc, int64_t krowb, int64_t khead, const char* vsrc,
                                          int64_t vhead, const PagedCache& d, int64_t page, int r0, int m,
                                          int slots, int h0, int e) {
  constexpr int U = 8 / HB;
  typedef typename Piece<VB>::t piece;
  const int tid = threadIdx.x, row = d.dh * e, lkp = __builtin_ctz(row / 16), gb = d.ds * e;
  char* kd = static_cast<char*>(d.K) + (((page * d.H + h0) << d.shift) + r0) * row;
  const int64_t kdh = static_cast<int64_t>(row) << d.shift;
  for (int u0 = tid; u0 < m << lkp; u0 += 256 * U) {
    u32x4 x[U][HB];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = u0 + 256 * i, t = min(u >> lkp, m - 1), q = u & ((1 << lkp) - 1);
      const int64_t kr = g.krow[t];
#pragma unroll
      for (int h = 0; h < HB; ++h) {
        x[i][h] = u32x4{0, 0, 0, 0};
        if (kr >= 0 && h0 + h < d.H) x[i][h] = get<NT>(reinterpret_cast<const u32x4*>(ksrc + kr * krowb + (h0 + h) * khead + 16 * q));
      }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = u0 + 256 * i;
      if (u >= m << lkp) continue;
#pragma unroll
      for (int h = 0; h < HB; ++h)
        if (h0 + h < d.H) put<NT>(x[i][h], reinterpret_cast<u32x4*>(kd + h * kdh + 16 * static_cast<int64_t>(u)));
    }
  }
  const int lpg = __builtin_ctz(gb / VB);  // pieces of a group
  char* vd = static_cast<char*>(d.V) + (page * d.H + h0) * d.vcap * static_cast<int64_t>(gb);
  const int64_t vdh = static_cast<int64_t>(d.vcap) * gb;
  const int p1 = slots << lpg;
  for (int u0 = tid; u0 < p1; u0 += 256 * U) {
    piece x[U][HB];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = min(u0 + 256 * i, p1 - 1), sl = u >> lpg, t = g.owner[sl];
      const bool in = t != kNone;
      const char* v = vsrc + (in ? g.vmove[t] + sl : 0) * gb + (u & ((1 << lpg) - 1)) * VB;
#pragma unroll
      for (int h = 0; h < HB; ++h) {
        x[i][h] = piece{};
        if (in && h0 + h < d.H) x[i][h] = get<NT>(reinterpret_cast<const piece*>(v + (h0 + h) * vhead));
      }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = u0 + 256 * i;
      if (u >= p1) continue;
#pragma unroll
      for (int h = 0; h < HB; ++h)
        if (h0 + h < d.H) put<NT>(x[i][h], reinterpret_cast<piece*>(vd + h * vdh + VB * static_cast<int64_t>(u)));
    }
  }
}

// Many new tokens, a page of them a workgroup: sequence b, the i-th page its new
// tokens touch, HB heads. The groups of a new token lie apart in z (every G-th is
// there), so a slot's source is its token's row and the group it holds. 16 times up to 305
// tokens of 32 heads (67 MB) 17.5 us, 3.8 TB/s: a copy's rate, behind what comes before any
// copy: length, page and masks one after another, the exclusive sum, and each token's
// entries of owner and s_group, up to G in turn by its one thread.
template <int VB, int HB>
__global__ __launch_bounds__(256) void k_append(AppendParams p, int np, int e) {
  __shared__ PageMap g;
  __shared__ uint8_t s_group[kMaxPage * 32];
  __shared__ int wsum[4], s_total;
  typedef typename Piece<VB>::t piece;
  constexpr int U = 8 / HB;
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
  const uint32_t whole = tid < m ? p.mask[j0 + tid] : 0u, mine = whole & gm;
  int base = 0;
  if (r0 > 0) base = c.slot[meta + r0 - 1] + __popc(c.mask[meta + r0 - 1] & gm);
  const int cnt = __popc(mine), at = group_scan<256, false>(cnt, wsum);
  if (tid == 255) s_total = at + cnt;
  if (tid < m) {
    g.krow[tid] = j0 + tid;
    uint32_t left = mine;
    for (int x = 0; x < cnt; ++x, left &= left - 1) {
      g.owner[at + x] = static_cast<uint16_t>(tid);
      s_group[at + x] = static_cast<uint8_t>(__builtin_ctz(left));
    }
    if (blockIdx.y == 0) {
      c.mask[meta + r0 + tid] = whole;
      c.slot[meta + r0 + tid] = base + at;
    }
  }
  __syncthreads();
  const int row = c.dh * e, gb = c.ds * e, h0 = blockIdx.y * HB;
  copy_page<VB, HB, false>(g, static_cast<const char*>(p.k), p.k_stride * e, row, nullptr, 0, c, page, r0, m, 0, h0, e);
  const int lpg = __builtin_ctz(gb / VB);
  char* vd = static_cast<char*>(c.V) + (static_cast<int64_t>(page) * c.H + h0) * c.vcap * static_cast<int64_t>(gb);
  const int64_t vdh = static_cast<int64_t>(c.vcap) * gb;
  for (int u0 = tid; u0 < s_total << lpg; u0 += 256 * U) {
    piece x[U][HB];
#pragma unroll
    for (int y = 0; y < U; ++y) {
      const int u = min(u0 + 256 * y, (s_total << lpg) - 1), sl = u >> lpg;
      const char* z = static_cast<const char*>(p.z) + (j0 + g.owner[sl]) * p.z_stride * e + s_group[sl] * gb +
                      (u & ((1 << lpg) - 1)) * VB;
#pragma unroll
      for (int h = 0; h < HB; ++h)
        if (h0 + h < c.H) x[y][h] = *reinterpret_cast<const piece*>(z + (h0 + h) * row);
    }
#pragma unroll
    for (int y = 0; y < U; ++y) {
      const int u = u0 + 256 * y;
      const int64_t sl = static_cast<int64_t>(base) + (u >> lpg);
      if (u >= s_total << lpg || sl < 0 || sl >= c.vcap) continue;
#pragma unroll
      for (int h = 0; h < HB; ++h)
        if (h0 + h < c.H)
          *reinterpret_cast<piece*>(vd + h * vdh + sl * gb + (u & ((1 << lpg) - 1)) * VB) = x[y][h];
    }
  }
}

// Kept tokens into one new page. One workgroup: sequence b, its i-th new page, HB
// heads. Each new token's source page, row and slot come from its old index; its new
// slots from an exclusive sum over the page. Bound by memory: 32 sequences that keep up
// to 777 of 2048 tokens (8 heads; 146 MB) 36 us, 4.1 TB/s; 4 that keep 8192 of 131071 (210
// MB) 48 us, 4.4.
template <int VB, int HB>
__global__ __launch_bounds__(256) void k_compact(CompactParams p, int np, int e) {
  __shared__ PageMap g;
  __shared__ int wsum[4], s_total;
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
  const int cnt = __popc(mine), at = group_scan<256, false>(cnt, wsum);
  if (tid == 255) s_total = at + cnt;
  if (tid < m) {
    g.krow[tid] = spage < 0 ? -1 : ((static_cast<int64_t>(spage) * c.H) << c.shift) + srow;
    g.vmove[tid] = static_cast<int64_t>(spage) * c.H * c.vcap + from - at;
    for (int x = 0; x < cnt; ++x) {
      const uint32_t fr = static_cast<uint32_t>(from) + x;
      g.owner[at + x] = fr < static_cast<uint32_t>(c.vcap) ? static_cast<uint16_t>(tid) : kNone;
    }
    if (blockIdx.y == 0) {
      const int64_t meta = (static_cast<int64_t>(page) << c.shift) + tid;
      d.mask[meta] = whole;
      d.slot[meta] = at;
    }
  }
  __syncthreads();
  const int row = c.dh * e, gb = c.ds * e;
  copy_page<VB, HB, true>(g, static_cast<const char*>(c.K), row, static_cast<int64_t>(row) << c.shift,
                    static_cast<const char*>(c.V), static_cast<int64_t>(c.vcap) * gb, d, page, 0, m,
                    min(s_total, d.vcap), blockIdx.y * HB, e);
}

// Heads of a workgroup: four, whose loads then share their addresses' work, where
// that leaves two workgroups for each of the 256 CUs.
bool four_heads(size_t pages, int H) { return pages * ((H + 3) / 4) >= 512; }

}  // namespace

hipError_t launch_append(const AppendParams& p, bool bf16, hipStream_t s) {
  const int e = bf16 ? 2 : 4, gb = p.c.ds * e;
  const int np = ((p.c.page - 1 + p.T - 1) >> p.c.shift) + 1;
  const size_t pages = static_cast<size_t>(p.B) * np;
  if (p.T < 8) {
    constexpr int hpb = 8;
    auto kern = gb >= 16 ? k_append_few<16> : gb == 8 ? k_append_few<8> : k_append_few<4>;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(pages), (p.c.H + hpb - 1) / hpb), dim3(256), 0, s, p, np, hpb, e);
  } else if (four_heads(pages, p.c.H)) {
    auto kern = gb >= 16 ? k_append<16, 4> : gb == 8 ? k_append<8, 4> : k_append<4, 4>;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(pages), (p.c.H + 3) / 4), dim3(256), 0, s, p, np, e);
  } else {
    auto kern = gb >= 16 ? k_append<16, 1> : gb == 8 ? k_append<8, 1> : k_append<4, 1>;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(pages), p.c.H), dim3(256), 0, s, p, np, e);
  }
  return hipGetLastError();
}

hipError_t launch_compact(const CompactParams& p, bool bf16, hipStream_t s) {
  const int e = bf16 ? 2 : 4, gb = p.src.ds * e;
  const int np = ((p.keep - 1) >> p.src.shift) + 1;
  const size_t pages = static_cast<size_t>(p.B) * np;
  if (four_heads(pages, p.src.H)) {
    auto kern = gb >= 16 ? k_compact<16, 4> : gb == 8 ? k_compact<8, 4> : k_compact<4, 4>;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(pages), (p.src.H + 3) / 4), dim3(256), 0, s, p, np, e);
  } else {
    auto kern = gb >= 16 ? k_compact<16, 1> : gb == 8 ? k_compact<8, 1> : k_compact<4, 1>;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(pages), p.src.H), dim3(256), 0, s, p, np, e);
  }
  return hipGetLastError();
}

}  // namespace rolesub
