// Attention of drafted tokens that form a tree, over the paged cache: the kernels of
// decode.hpp, and one for more rows than a matrix product's 16.
#include "decode.hpp"

namespace rolesub {
namespace {

// The end of a split, as add_waves: RB blocks of rows of each wave at once.
template <class T, int DH, int RB>
__device__ __forceinline__ void add_blocks(const DecodeParams& p, int b, int h, int rtile, int sp, const float* m, float* l,
                                           const f32x4 (*acc)[Tile<T, DH>::MB], char* smem, float (*s_m)[16 * RB],
                                           float (*s_l)[16 * RB]) {
  using L = Tile<T, DH>;
  constexpr int MB = L::MB, RLD = L::RLD, ROWS = 16 * RB;
  const PagedCache& c = p.c;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g4 = lane >> 4;
  Rotation<T, DH> rot;
  if (p.n_split == 1) rot.load(p, h);
#pragma unroll
  for (int n = 0; n < RB; ++n) {
    l[n] = add_xor32(add_xor16(l[n]));
    if (g4 == 0) {
      s_m[w][16 * n + l16] = m[n];
      s_l[w][16 * n + l16] = l[n];
    }
  }
  __syncthreads();  // also: no wave reads its tile any more
  float* red = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int n = 0; n < RB; ++n) {
    float M = s_m[0][16 * n + l16];
#pragma unroll
    for (int v = 1; v < 4; ++v) M = fmaxf(M, s_m[v][16 * n + l16]);
    const float f = weight_of(m[n], M);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
      *reinterpret_cast<f32x4*>(red + (w * ROWS + 16 * n + l16) * RLD + 16 * mb + 4 * g4) = acc[n][mb] * f;
  }
  __syncthreads();
  const int64_t rows0 = (static_cast<int64_t>(b) * c.H + h) * p.R;
#pragma unroll 1
  for (int u = tid; u < ROWS * (DH / 4); u += 256) {
    const int row = u / (DH / 4), d = u % (DH / 4) * 4, rg = rtile * ROWS + row;
    float M = s_m[0][row];
#pragma unroll
    for (int v = 1; v < 4; ++v) M = fmaxf(M, s_m[v][row]);
    float sum = 0.f;
    f32x4 a = {0, 0, 0, 0};
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      sum += s_l[v][row] * weight_of(s_m[v][row], M);
      a += *reinterpret_cast<const f32x4*>(red + (v * ROWS + row) * RLD + d);
    }
    if (p.n_split == 1) {
      if (rg >= p.R || sum == 0.f) a = f32x4{0, 0, 0, 0};
      else a /= sum;
      *reinterpret_cast<f32x4*>(red + row * RLD + d) = a;  // read by this thread only
    }
    if (rg >= p.R) continue;
    const int64_t at = (rows0 + rg) * p.n_split + sp;
    if (p.n_split > 1) {
      *reinterpret_cast<f32x4*>(p.part + at * DH + d) = a;
      if (d == 0) *reinterpret_cast<float2*>(p.stat + 2 * at) = float2{M, sum};
    }
  }
  if (p.n_split == 1) {
    __syncthreads();
#pragma unroll 1
    for (int n = 0; n < RB; ++n) {
      const int r0 = (rtile * RB + n) * 16;
      if (r0 < p.R) finish_rows<T, DH>(p, b, h, r0, red + 16 * n * RLD, rot);
    }
  }
}

// One split of one key head and two blocks of 16 rows, both of them every wave's, which
// takes every fourth tile of tokens: keys come from memory straight into the products'
// operands, and a tile's expanded values are read from LDS once for both blocks. No wave
// waits for another before the end. (k_decode_rows, whose waves share tiles and have 16 rows
// each, reads every tile from LDS once a wave, which took as long there as the products did,
// and waits a barrier a tile: as it is, and with eight waves and 128 rows, it took 136 and
// 129 us for 32 sequences of 256 to 4096 tokens, 8 key heads of 96 rows, against 88 here; 64
// rows 92 against 73, 240 rows 207 against 176, all with two parts of a weight. Three, as it
// is, take 90, 76 and 181 with two input sets in turn, and 83 for the 96 rows where one
// set stays in the caches. Three blocks leave one wave a SIMD its
// registers: 184. Eight waves a workgroup, one workgroup a CU: 111, as the chain of loads
// before the first product and the one behind the last, some 12 us in all, then have
// nothing beside them.) The row tiles of one item read the same keys and values one after
// the other on one XCD: half of the reads find their lines in its cache.
// That chain and the longest sequence bound it: of the cycles in which a CU has waves the
// vector units issue in 47 % and the matrix units work in 24 %. Sequences of 64 tokens, which
// have the chain alone, take 31 us where k_decode_rows took 23.
template <class T, int DH, int SUB>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void k_tree_rows(DecodeParams p) {
  using L = Tile<T, DH>;
  constexpr int TK = L::TK, NB = L::NB, KS = L::KS, NVI = L::NVI, MB = L::MB;
  constexpr int STEP = 4 * TK, TPP = 64 / NB, ROWS = kTreeRows, RB = ROWS / 16;  // TPP: tiles whose pages one load brings
  constexpr int SMEM = RB * 4 * L::RB > 4 * L::ZB ? RB * 4 * L::RB : 4 * L::ZB;
  __shared__ __attribute__((aligned(16))) char smem[SMEM];
  __shared__ u32x2 s_rec[4][TK];
  __shared__ float s_m[4][ROWS], s_l[4][ROWS];
  __shared__ uint32_t s_bits[ROWS * kTreeRow];
  __shared__ int s_b;
  const PagedCache& c = p.c;
  // the row tiles of one split are eight workgroups apart, on one XCD at about one time
  const int nrt = (p.R + ROWS - 1) / ROWS, group = blockIdx.x / (8 * nrt), in = blockIdx.x % (8 * nrt), rtile = in / 8;
  int h, b, sp;
  if (group * 8 + in % 8 >= p.B * c.H * p.n_split) return;
  place_item(p, group * 8 + in % 8, nrt, reinterpret_cast<int*>(smem), s_b, h, b, sp);
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15,
            g4 = lane >> 4;
  const int c0 = sp * p.chunk, first = c0 + w * TK;
  const rsrc_t r_table = make_rsrc(p.table + static_cast<int64_t>(b) * p.max_pages,
                                   clamp_bytes(static_cast<size_t>(p.max_pages) * 4));
  const int shift = c.shift, pmask = c.page - 1;
  int pgs;  // lane j: the page of block j % NB of the (j / NB)-th of TPP tiles
  auto request_pages = [&](int i) {  // of tiles i .. i + TPP - 1
    const int t = first + i * STEP + lane / NB * STEP + lane % NB * 16;
    pgs = static_cast<int>(bload4(r_table, static_cast<uint32_t>(t >> shift) * 4u));  // past the row: 0
  };
  request_pages(0);
  const int len = tokens_of<kTree>(p, b);
  if (c0 >= len && p.n_split > 1) return;
  const uint32_t gm = group_bits(c.G);
  const int gb = c.ds * static_cast<int>(sizeof(T));

  TreeBits<ROWS> bits;
  bits.load(p, b, rtile * ROWS);
  u32x4 qf[RB][KS];
  View v[RB];
  int low = 0x7FFFFFFF, top = 0;
#pragma unroll
  for (int n = 0; n < RB; ++n) {
    const int r = (rtile * RB + n) * 16 + l16;
    int reach;
    load_query<T, DH>(p, b, h, r, g4, qf[n]);
    v[n] = look<kTree>(p, b, r, len, s_bits + (n * 16 + l16) * kTreeRow, reach);
    top = max(top, reach);
    low = min(low, r < p.R ? v[n].lim : 0x7FFFFFFF);
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) {
    top = max(top, __shfl_xor(top, o, kWave));
    low = min(low, __shfl_xor(low, o, kWave));
  }
  const int least = __builtin_amdgcn_readfirstlane(low);
  const int end = min(c0 + p.chunk, __builtin_amdgcn_readfirstlane(top));
  const uint32_t meta_bytes = static_cast<uint32_t>(c.n_pages) << (shift + 2);  // below 2 GiB
  const rsrc_t r_mask = make_rsrc(c.mask, meta_bytes), r_slot = make_rsrc(c.slot, meta_bytes);
  // bytes of a head's part of a page, and of a page (below 2 GiB)
  const uint32_t kstep = static_cast<uint32_t>(c.page) * L::ROWB, vstep = static_cast<uint32_t>(c.vcap) * gb;
  const uint32_t kpage = kstep * c.H, vpage = vstep * c.H;
  const char* khead = static_cast<const char*>(c.K) + static_cast<size_t>(h) * kstep;
  const char* vhead = static_cast<const char*>(c.V) + static_cast<size_t>(h) * vstep;

  // a lane's pieces of the values: always the same part of a row
  const int pc = lane % L::LPT, vt = lane / L::LPT;
  const int vg = SUB == 1 ? pc * 16 / gb : pc * SUB;
  const uint32_t vin = SUB == 1 ? static_cast<uint32_t>(pc * 16 % gb) : 0u;
  char* zt = smem + w * L::ZB;
  u32x2* rec = s_rec[w];

  float m[RB], l[RB];
  f32x4 acc[RB][MB];
#pragma unroll
  for (int n = 0; n < RB; ++n) {
    m[n] = -__builtin_inff();
    l[n] = 0.f;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) acc[n][mb] = f32x4{0, 0, 0, 0};
  }
  {
    int pg1[NB];   // pages of the next tile, whose masks and slots are on their way
    uint32_t mk1 = 0;
    int sl1 = 0;
    u32x4 kf[NB][KS], vf[NVI];
    bool there[NB], there1[NB];

    auto take_pages = [&](int i) {  // of tile i, pages that are none as -1
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int t = first + i * STEP + 16 * nb, pg = __builtin_amdgcn_readlane(pgs, i % TPP * NB + nb);
        pg1[nb] = t < end && static_cast<uint32_t>(pg) < static_cast<uint32_t>(c.n_pages) ? pg : -1;
      }
    };
    auto request_meta = [&](int i) {  // of the pages pg1
      const int t = first + i * STEP + lane, pg = NB == 2 && lane >= 16 ? pg1[NB - 1] : pg1[0];
      const uint32_t off = oob_unless(lane < TK && t < end && pg >= 0,
                                      (static_cast<uint32_t>(pg) << (shift + 2)) + static_cast<uint32_t>(t & pmask) * 4u);
      mk1 = bload4(r_mask, off);
      sl1 = static_cast<int>(bload4(r_slot, off));
    };
    auto request_keys = [&](int i) {
      const int t0 = first + i * STEP;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        there1[nb] = pg1[nb] >= 0;
        const rsrc_t rk = make_rsrc(khead + static_cast<uint64_t>(max(pg1[nb], 0)) * kpage, there1[nb] ? kstep : 0u);
        const uint32_t ko = static_cast<uint32_t>(((t0 + 16 * nb) & pmask) + l16) * L::ROWB + 16 * g4;
#pragma unroll
        for (int j = 0; j < KS; ++j) kf[nb][j] = bload16(rk, ko + 64 * j);
      }
    };
    auto request_values = [&]() {
      if (lane < TK) rec[lane] = u32x2{mk1 & gm, static_cast<uint32_t>(sl1)};
      wave_lds_order();
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        constexpr int N = NVI / NB;
        u32x2 tk[N];
#pragma unroll
        for (int x = 0; x < N; ++x) tk[x] = rec[(nb * N + x) * L::TPI + vt];
        const rsrc_t rv = make_rsrc(vhead + static_cast<uint64_t>(max(pg1[nb], 0)) * vpage, there1[nb] ? vstep : 0u);
#pragma unroll
        for (int x = 0; x < N; ++x)
          vf[nb * N + x] = request_piece<SUB>(rv, tk[x].x, tk[x].y, vg, vin, gb, static_cast<uint32_t>(c.vcap));
      }
    };
    auto next_pages = [&](int i) {
      if (i % TPP == 0) {
        request_pages(i);
        arrived(pgs);
      }
      take_pages(i);
    };

    take_pages(0);
    request_meta(0);
    request_keys(0);
    request_values();
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) there[nb] = there1[nb];
    next_pages(1);
    request_meta(1);
    bits.put(s_bits, len - v[0].base);
    __syncthreads();
#pragma unroll 1
    for (int i = 0, t0 = first; t0 < end; ++i, t0 += STEP) {
      // scores: tokens are the rows of the product, queries its columns
      f32x4 s[RB][NB];
#pragma unroll
      for (int n = 0; n < RB; ++n)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) s[n][nb] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)  // in the order the keys arrive
#pragma unroll
        for (int j = 0; j < KS; ++j)
#pragma unroll
          for (int n = 0; n < RB; ++n) s[n][nb] = score_step<T>(kf[nb][j], qf[n][j], s[n][nb]);
      // the tile's kept groups into their places, dropped ones as zeros
#pragma unroll
      for (int x = 0; x < NVI; ++x) *reinterpret_cast<u32x4*>(zt + (x * L::TPI + vt) * L::ZLD + 16 * pc) = vf[x];
      wave_lds_order();
      uint32_t ok = 0;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) ok |= there[nb] ? 1u << nb : 0u;
      request_keys(i + 1);
      request_values();
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) there[nb] = there1[nb];
      next_pages(i + 2);
      request_meta(i + 2);
#pragma unroll
      for (int n = 0; n < RB; ++n)
        soften<T, DH, true, kTree>(p, s[n], ok, t0, nullptr, v[n], least, end, 0, nullptr, nullptr, m[n], l[n], acc[n]);
      weigh_blocks<T, DH, RB>(zt, s, acc);
      wave_lds_order();
    }
  }
#pragma unroll
  for (int n = 0; n < RB; ++n) {
    bool bad = false;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int x = 0; x < 4; ++x) bad |= !__builtin_isfinite(acc[n][mb][x]);
    if (__any(bad)) one_by_one<T, DH, kTree>(p, b, h, (rtile * RB + n) * 16 + l16, first, STEP, end, v[n], zt, m[n], l[n], acc[n]);
  }
  add_blocks<T, DH, RB>(p, b, h, rtile, sp, m, l, acc, smem, s_m, s_l);
}

template <class T, int DH>
void go_rows(const DecodeParams& p, hipStream_t s) {
  const int sub = p.c.ds >= Tile<T, DH>::EP ? 1 : Tile<T, DH>::EP / p.c.ds;
  auto kern = sub == 1 ? k_tree_rows<T, DH, 1> : k_tree_rows<T, DH, 2>;
  if constexpr (sizeof(T) == 2) {
    if (sub == 4) kern = k_tree_rows<T, DH, 4>;
  }
  const unsigned items = static_cast<unsigned>(p.B) * p.c.H * p.n_split;
  hipLaunchKernelGGL(kern, dim3((items + 7) / 8 * 8 * ((p.R + kTreeRows - 1) / kTreeRows)), dim3(256), 0, s, p);
}

template <class T, int DH>
hipError_t launch_rows(DecodeParams p, hipStream_t s) {
  p.ordered = p.n_split == 1 && p.B > 1 && p.B <= kOrderMax && p.max_len >= 512;
  go_rows<T, DH>(p, s);
  launch_join<T, DH, kTree>(p, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_decode_tree(const DecodeParams& p, bool bf16, hipStream_t s) {
  if (p.R <= 16) return launch_any<kTree>(p, bf16, s);
  if (bf16) return p.c.dh == 128 ? launch_rows<__bf16, 128>(p, s) : launch_rows<__bf16, 64>(p, s);
  return p.c.dh == 128 ? launch_rows<float, 128>(p, s) : launch_rows<float, 64>(p, s);
}

}  // namespace rolesub
