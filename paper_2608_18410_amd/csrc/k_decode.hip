// Attention of new tokens over the paged routed cache, split over its length.
//
//   s[r,t] = scale <q_r, k_t>,  P = softmax over the tokens a row sees,
//   u_r    = sum_t P[r,t] (M_t z_t),  out_r = R_h u_r
//
// The rows of one key head are its rep = Hq / H query heads times Tq queries, in
// blocks of 16. Splits of `chunk` tokens are computed by separate workgroups into
// partial sums with their maximum and sum of exponentials, which k_join adds and
// rotates back; a single split is finished where it was computed.
#include <algorithm>

#include "common.hpp"
#include "launch.hpp"

namespace rolesub {
namespace {

// Four bf16 rows of 16 columns, transposed: 16 lanes give the addresses of the
// rows' 8-byte quarters, lane i gets column i of the four rows.
__device__ __forceinline__ bf16x4 lds_read_tr(const char* p) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef s16x4 __attribute__((address_space(3))) * p3;
  return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((p3)(p)));
}

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// Factor of sums taken against the maximum m once the maximum is M. Sums without a
// score above -inf are zeros, or NaN where a score was: they are added as they are.
__device__ __forceinline__ float weight_of(float m, float M) { return m == -__builtin_inff() ? 1.f : exp2_(m - M); }

template <class T, int DH>
struct Tile {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int TK = kBf16 ? 32 : 16, NB = TK / 16;  // tokens of a wave's tile, 16-token blocks
  static constexpr int EP = 16 / sizeof(T);                 // elements of a 16-byte piece
  static constexpr int KS = DH * sizeof(T) / 64;            // 64-byte steps of a row
  static constexpr int ROWB = DH * sizeof(T);
  static constexpr int LPT = ROWB / 16, TPI = 64 / LPT, NVI = TK / TPI;
  // LDS rows padded so that the transposed reads (bf16) or the four tokens of a
  // step (f32) fall on different banks
  static constexpr int ZLD = ROWB + (kBf16 ? 32 : 16);
  static constexpr int ZB = TK * ZLD;
  static constexpr int RLD = DH + 4;  // floats of a row while the waves' sums are added
  static constexpr int RB = 16 * RLD * 4;
  static constexpr int SMEM = 4 * ZB > 4 * RB ? 4 * ZB : 4 * RB;
  static constexpr int MB = DH / 16;
};

__device__ __forceinline__ int tokens_of(const DecodeParams& p, int b) {
  const int64_t cap = static_cast<int64_t>(p.max_pages) << p.c.shift;
  return static_cast<int>(min(static_cast<int64_t>(min(max(p.lens[b], 0), p.max_len)), cap));
}

template <bool ONCE>
__device__ __forceinline__ u32x4 bload16_hint(rsrc_t r, uint32_t off) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, static_cast<int>(off), 0, ONCE ? 2 : 0));
}

// Eight floats as the sum of three bf16 each: 8 of their 24 bits a part, and exact, as
// what a part leaves is a difference of near floats (down to 2^-110, where the last part
// leaves the range). Two parts, 17 bits, put float32 outputs off by up to 2^-16; the
// third costs 7 % where rows share tiles (16 sequences of up to 361 tokens and 56
// queries, 32 heads 29.2 -> 31.1 us, 8 of 305 and 305 52 -> 56.5) and nothing where
// calls are bound by memory. An infinity's other parts are NaN.
constexpr int kParts = 3;
__device__ __forceinline__ void split_bf16(f32x4 a, f32x4 b, bf16x8 (&part)[kParts]) {
  u32x4 v[kParts];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f32x2 x = i < 2 ? f32x2{a[2 * i], a[2 * i + 1]} : f32x2{b[2 * i - 4], b[2 * i - 3]};
#pragma unroll
    for (int n = 0; n < kParts; ++n) {
      v[n][i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
      x = f32x2{x[0] - __uint_as_float(v[n][i] << 16), x[1] - __uint_as_float(v[n][i] & 0xFFFF0000u)};
    }
  }
#pragma unroll
  for (int n = 0; n < kParts; ++n) part[n] = __builtin_bit_cast(bf16x8, v[n]);
}

// Order of N steps of R LDS reads that feed M matrix products each: the reads run A
// steps ahead (left to itself the compiler waits for each).
template <int N, int R, int M, int A>
__device__ __forceinline__ void reads_ahead() {
  constexpr int kDsRead = 0x100, kMfma = 0x008;
  __builtin_amdgcn_sched_group_barrier(kDsRead, A * R, 0);
#pragma unroll
  for (int i = 0; i + A < N; ++i) {
    __builtin_amdgcn_sched_group_barrier(kMfma, M, 0);
    __builtin_amdgcn_sched_group_barrier(kDsRead, R, 0);
  }
  __builtin_amdgcn_sched_group_barrier(kMfma, A * M, 0);
}

// Waits here for a load. In a branch, so that what follows it does not wait on every
// path: there the wait would be for whatever else is under way.
__device__ __forceinline__ void arrived(int& x) { asm volatile("" : "+v"(x)); }

// Waits until a matrix product's result may be read by other instructions. In straight
// code the compiler keeps the states between them (8 for the bf16 product, 10 for the
// float32 one). Without this, the assembly of k_join in bf16 has products into
// accumulation registers, a branch (around the way without a rotation), and on its taken
// side v_accvgpr_read of them three instructions later; the first elements came out
// stale. Placed after products that end a block; tests/test_mfma_waits.py looks at the
// assembly for any other.
template <int N>
__device__ __forceinline__ void settle(f32x4 (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));
  asm volatile("s_nop 15" : "+v"(x[0]));
#pragma unroll
  for (int i = 1; i < N; ++i) asm volatile("" : "+v"(x[i]));
}

// R_h's rows for the matrix cores: wave w's blocks of 16 output dims, w, w + 4, ...
template <class T, int DH>
struct Rotation {
  using L = Tile<T, DH>;
  static constexpr int N = L::MB / 4;
  u32x4 a[N][L::KS];
  __device__ __forceinline__ void load(const DecodeParams& p, int h) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, l16 = lane & 15, g4 = lane >> 4;
    if (!p.Rm) return;
    const T* R = static_cast<const T*>(p.Rm) + (static_cast<int64_t>(h) * DH + 16 * w + l16) * DH + g4 * L::EP;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < L::KS; ++j) a[i][j] = *reinterpret_cast<const u32x4*>(R + 64 * i * DH + 4 * j * L::EP);
  }
};

// Output rows [r0, r0 + 16) of key head h from their normalised sums u (LDS, rows of
// RLD floats; rows past R are zero): out = R_h u on the matrix cores, R's rows as
// the product's rows. The sums enter as bf16 parts, or in f32. All 256 threads.
template <class T, int DH>
__device__ __forceinline__ void finish_rows(const DecodeParams& p, int b, int h, int r0, const float* u,
                                            const Rotation<T, DH>& rot) {
  using L = Tile<T, DH>;
  constexpr int KS = L::KS, EP = L::EP, N = L::MB / 4;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, l16 = lane & 15, g4 = lane >> 4;
  const int r = r0 + l16;
  const float* ur = u + l16 * L::RLD;
  f32x4 o[N];
  if (p.Rm) {
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      const int d = (4 * j + g4) * EP;
      if constexpr (L::kBf16) {
        bf16x8 part[kParts];
        split_bf16(*reinterpret_cast<const f32x4*>(ur + d), *reinterpret_cast<const f32x4*>(ur + d + 4), part);
#pragma unroll
        for (int n = 0; n < kParts; ++n)
#pragma unroll
          for (int i = 0; i < N; ++i) o[i] = mfma_16x16x32(__builtin_bit_cast(bf16x8, rot.a[i][j]), part[n], o[i]);
      } else {
        const f32x4 uf = *reinterpret_cast<const f32x4*>(ur + d);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const f32x4 af = __builtin_bit_cast(f32x4, rot.a[i][j]);
#pragma unroll
          for (int x = 0; x < 4; ++x) o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(af[x], uf[x], o[i], 0, 0, 0);
        }
      }
    }
    settle(o);
    if constexpr (L::kBf16) {
      // infinite sums, whose other parts are NaN, once more from the float32 numbers (16
      // sequences and 56 queries, as above: 32.4 us; with a test of every part 34.8)
      bool bad = false;
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int x = 0; x < 4; ++x) bad |= !__builtin_isfinite(o[i][x]);
      if (__any(bad)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const T* R = static_cast<const T*>(p.Rm) + (static_cast<int64_t>(h) * DH + 16 * (w + 4 * i) + 4 * g4) * DH;
          o[i] = f32x4{0, 0, 0, 0};
#pragma unroll 1
          for (int d = 0; d < DH; ++d)
#pragma unroll
            for (int x = 0; x < 4; ++x) o[i][x] += tof(R[x * DH + d]) * ur[d];
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = *reinterpret_cast<const f32x4*>(ur + 16 * (w + 4 * i) + 4 * g4);
  }
  if (r >= p.R) return;
  const int64_t at = ((static_cast<int64_t>(b) * p.Tq + r / p.rep) * p.Hq + h * p.rep + r % p.rep) * DH + 16 * w + 4 * g4;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (p.out_f32 || !L::kBf16) {
      *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + at + 64 * i) = o[i];
    } else {
      const u32x2 v = {pack_bf16x2(o[i][0], o[i][1]), pack_bf16x2(o[i][2], o[i][3])};
      *reinterpret_cast<u32x2*>(static_cast<T*>(p.out) + at + 64 * i) = v;
    }
  }
}

// One 64-byte step of the scores of 16 tokens (rows) and 16 queries (columns).
template <class T>
__device__ __forceinline__ f32x4 score_step(u32x4 k, u32x4 q, f32x4 s) {
  if constexpr (sizeof(T) == 2) {
    return mfma_16x16x32(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q), s);
  } else {
    const f32x4 a = __builtin_bit_cast(f32x4, k), x = __builtin_bit_cast(f32x4, q);
#pragma unroll
    for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], x[i], s, 0, 0, 0);
    return s;
  }
}

// A 16-byte part of a token's expanded value row: the parts of its kept groups, zeros
// for dropped ones. vg: the part's first group; vin: its place in the group where
// that is wider (SUB == 1).
template <int SUB>
__device__ __forceinline__ u32x4 request_piece(rsrc_t rv, uint32_t mask, uint32_t slot, int vg, uint32_t vin, int gb,
                                               uint32_t vcap) {
  uint32_t sl = slot + __popc(mask & ((1u << vg) - 1u));
  if constexpr (SUB == 1) return bload16(rv, ((mask >> vg) & 1u) && sl < vcap ? sl * gb + vin : kOOB);
  u32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int u = 0; u < SUB; ++u) {
    const bool on = (mask >> (vg + u)) & 1u;
    const uint32_t off = on && sl < vcap ? sl * gb : kOOB;
    if constexpr (SUB == 2) {
      const u32x2 y = bload8(rv, off);
      v[2 * u] = y.x;
      v[2 * u + 1] = y.y;
    } else {
      v[u] = bload4(rv, off);
    }
    sl += on;
  }
  return v;
}

// A tile's scores s become weights: exponentials against the reference m, which the
// sums l and acc are kept against. It is raised, and they are scaled, only when some
// row's maximum passes it by more than 2^8: up to there nothing can overflow, and
// what the weights round to is relative to themselves. ok: blocks of 16 tokens that
// are there; lim: tokens the lane's row sees, least: those all rows see. SHORT: tiles
// that all rows see whole take a way without the comparisons (worth it where the
// kernel is bound by such instructions; the branch costs registers). Scores that are kept
// for the tokens' weights go to px, or to lx in LDS where there is one row.
template <class T, int DH, bool SHORT>
__device__ __forceinline__ void soften(const DecodeParams& p, f32x4* s, uint32_t ok, int t0, int lim, int least, int end,
                                       int r, float* px, float* lx, float& m, float& l, f32x4* acc) {
  using L = Tile<T, DH>;
  constexpr int NB = L::NB;
  constexpr float kSlack = 8.f;
  const int g4 = (threadIdx.x & 63) >> 4;
  if (SHORT && t0 + L::TK <= least && ok == (1u << NB) - 1u) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int x = 0; x < 4; ++x) s[nb][x] *= p.scale;
  } else {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const bool see = ((ok >> nb) & 1u) && t0 + 16 * nb + 4 * g4 + x < lim;
        s[nb][x] = see ? s[nb][x] * p.scale : -__builtin_inff();
      }
  }
  if (lx) {
    if ((threadIdx.x & 15) == 0)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) *reinterpret_cast<f32x4*>(lx + 16 * nb + 4 * g4) = s[nb];
  } else if (px) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int t = t0 + 16 * nb + 4 * g4;
      if (r < p.R && t < end) *reinterpret_cast<f32x4*>(px + t) = s[nb];
    }
  }
  float mx = s[0][0];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int x = 0; x < 4; ++x) mx = fmaxf(mx, s[nb][x]);
  mx = max_xor32(max_xor16(mx));
  if (__any(mx > m + kSlack)) {
    const float mn = fmaxf(m, mx), al = mn == -__builtin_inff() ? 0.f : exp2_(m - mn);
    m = mn;
    l *= al;
#pragma unroll
    for (int mb = 0; mb < L::MB; ++mb) acc[mb] *= al;
  }
  const float ms = m == -__builtin_inff() ? 0.f : m;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      s[nb][x] = exp2_(s[nb][x] - ms);
      l += s[nb][x];
    }
}

// The tile's values times its weights s, added to the sums (dims the rows of the
// product, queries its columns). A: steps by which LDS reads run ahead.
template <class T, int DH, int A>
__device__ __forceinline__ void weigh_tile(const char* zt, const f32x4* s, f32x4* acc) {
  using L = Tile<T, DH>;
  const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4;
  if constexpr (L::kBf16) {
    bf16x8 part[kParts];
    split_bf16(s[0], s[L::NB - 1], part);
    const char* zr = zt + (4 * g4 + l16 / 4) * L::ZLD + 8 * (l16 % 4);
#pragma unroll
    for (int mb = 0; mb < L::MB; ++mb) {
      const bf16x4 a0 = lds_read_tr(zr + 32 * mb), a1 = lds_read_tr(zr + 16 * L::ZLD + 32 * mb);
      const bf16x8 a = __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
      for (int n = 0; n < kParts; ++n) acc[mb] = mfma_16x16x32(a, part[n], acc[mb]);
    }
    if constexpr (A > 0) reads_ahead<L::MB, 2, kParts, A>();
  } else {
#pragma unroll
    for (int mb = 0; mb < L::MB; ++mb)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const float a = *reinterpret_cast<const float*>(zt + (4 * g4 + x) * L::ZLD + 4 * (16 * mb + l16));
        acc[mb] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, s[0][x], acc[mb], 0, 0, 0);
      }
  }
}

// A lane's part of row r's query: the dims that its part of a key is multiplied by.
template <class T, int DH>
__device__ __forceinline__ void load_query(const DecodeParams& p, int b, int h, int r, int g4, u32x4* qf) {
  using L = Tile<T, DH>;
#pragma unroll
  for (int j = 0; j < L::KS; ++j) qf[j] = u32x4{0, 0, 0, 0};
  if (r >= p.R) return;
  const T* q = static_cast<const T*>(p.q) + (static_cast<int64_t>(b) * p.Tq + r / p.rep) * p.q_stride +
               static_cast<int64_t>(h * p.rep + r % p.rep) * DH;
#pragma unroll
  for (int j = 0; j < L::KS; ++j) qf[j] = *reinterpret_cast<const u32x4*>(q + (4 * j + g4) * L::EP);
}

// A wave's sums again, token by token, where they were not finite: an infinity or
// NaN in a value then reaches the rows that see its token and no other (a matrix
// product multiplies it by their zeros). Scores and weights are the same; the sums
// stay in LDS, so that this takes no registers from the loop it follows.
template <class T, int DH>
__device__ __forceinline__ void one_by_one(const DecodeParams& p, int b, int h, int r, int first, int step, int end,
                                           int lim, char* zt, float& m, float& l, f32x4* acc) {
  using L = Tile<T, DH>;
  constexpr int KS = L::KS, MB = L::MB;
  static_assert(L::ZB >= 16 * DH * 4, "a wave's sums fit its tile");
  const PagedCache& c = p.c;
  const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4;
  const uint32_t gm = group_bits(c.G);
  float* sum = reinterpret_cast<float*>(zt) + l16 * DH + 4 * g4;  // this lane's: dims 16 mb + 4 g4 + 0..3
  m = -__builtin_inff();
  l = 0.f;
#pragma unroll 1
  for (int d = 0; d < DH; d += 16) *reinterpret_cast<f32x4*>(sum + d) = f32x4{0, 0, 0, 0};
#pragma unroll 1
  for (int tile = first; tile < end; tile += step)
#pragma unroll 1
    for (int t0 = tile; t0 < min(tile + L::TK, end); t0 += 16) {
      const int pg = p.table[static_cast<int64_t>(b) * p.max_pages + (t0 >> c.shift)];
      if (static_cast<uint32_t>(pg) >= static_cast<uint32_t>(c.n_pages)) continue;
      const int row = t0 & (c.page - 1);
      const int64_t head = static_cast<int64_t>(pg) * c.H + h;
      const char* kp = static_cast<const char*>(c.K) + ((head << c.shift) + row + l16) * L::ROWB + 16 * g4;
      u32x4 qf[KS];
      load_query<T, DH>(p, b, h, r, g4, qf);
      f32x4 s = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < KS; ++j) s = score_step<T>(*reinterpret_cast<const u32x4*>(kp + 64 * j), qf[j], s);
      float mx = -__builtin_inff();
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        s[x] = t0 + 4 * g4 + x < lim ? s[x] * p.scale : -__builtin_inff();
        mx = fmaxf(mx, s[x]);
      }
      mx = max_xor32(max_xor16(mx));
      const float mn = fmaxf(m, mx), ms = mn == -__builtin_inff() ? 0.f : mn, al = exp2_(m - ms);
      m = mn;
      l *= al;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        s[x] = exp2_(s[x] - ms);
        l += s[x];
      }
#pragma unroll 1
      for (int d = 0; d < DH; d += 16) *reinterpret_cast<f32x4*>(sum + d) *= al;
#pragma unroll 1
      for (int tk = 0; tk < min(16, end - t0); ++tk) {  // lane group tk / 4 holds its weights
        const float mine = tk % 4 == 0 ? s[0] : tk % 4 == 1 ? s[1] : tk % 4 == 2 ? s[2] : s[3];
        const float pv = __shfl(mine, 16 * (tk / 4) + l16, kWave);
        const int64_t meta = (static_cast<int64_t>(pg) << c.shift) + row + tk;
        const uint32_t mk = c.mask[meta] & gm, slot = static_cast<uint32_t>(c.slot[meta]);
        if (t0 + tk >= lim) continue;
#pragma unroll 1
        for (int x = 0; x < DH / 4; ++x) {
          const int d = x / 4 * 16 + x % 4, g = (d + 4 * g4) / c.ds;
          const uint32_t sl = slot + __popc(mk & ((1u << g) - 1u));
          if (((mk >> g) & 1u) && sl < static_cast<uint32_t>(c.vcap))
            sum[d] += pv * tof(static_cast<const T*>(c.V)[(head * c.vcap + sl) * c.ds + (d + 4 * g4) % c.ds]);
        }
      }
    }
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) acc[mb] = *reinterpret_cast<f32x4*>(sum + 16 * mb);
}

// The end of a split: the sums of the waves of each row block added in their order,
// and left for k_join or, where there is no other split, finished. All 256 threads.
template <class T, int DH, int WR>
__device__ __forceinline__ void add_waves(const DecodeParams& p, int b, int h, int rtile, int sp, float m, float l,
                                          const f32x4* acc, char* smem, float (*s_m)[16], float (*s_l)[16]) {
  using L = Tile<T, DH>;
  constexpr int MB = L::MB, RLD = L::RLD, WT = 4 / WR;
  const PagedCache& c = p.c;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g4 = lane >> 4;
  Rotation<T, DH> rot;
  if (p.n_split == 1) rot.load(p, h);
  // the sums of the waves of one row block, in their order
  l = add_xor32(add_xor16(l));
  if (g4 == 0) {
    s_m[w][l16] = m;
    s_l[w][l16] = l;
  }
  __syncthreads();  // also: no wave reads its tile any more
  float* red = reinterpret_cast<float*>(smem);
  {
    float M = s_m[w % WR][l16];
#pragma unroll
    for (int v = 1; v < WT; ++v) M = fmaxf(M, s_m[w % WR + v * WR][l16]);
    const float f = weight_of(m, M);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
      *reinterpret_cast<f32x4*>(red + (w * 16 + l16) * RLD + 16 * mb + 4 * g4) = acc[mb] * f;
  }
  __syncthreads();
  const int64_t rows0 = (static_cast<int64_t>(b) * c.H + h) * p.R;
#pragma unroll 1
  for (int u = tid; u < 16 * WR * (DH / 4); u += 256) {
    const int row = u / (DH / 4), d = u % (DH / 4) * 4, rb = row / 16, rr = row % 16, rg = rtile * 16 * WR + row;
    float M = s_m[rb][rr];
#pragma unroll
    for (int v = 1; v < WT; ++v) M = fmaxf(M, s_m[rb + v * WR][rr]);
    float sum = 0.f;
    f32x4 a = {0, 0, 0, 0};
#pragma unroll
    for (int v = 0; v < WT; ++v) {
      sum += s_l[rb + v * WR][rr] * weight_of(s_m[rb + v * WR][rr], M);
      a += *reinterpret_cast<const f32x4*>(red + ((rb + v * WR) * 16 + rr) * RLD + d);
    }
    if (p.n_split == 1) {
      if (rg >= p.R || sum == 0.f) a = f32x4{0, 0, 0, 0};
      else a /= sum;
      *reinterpret_cast<f32x4*>(red + (rb * 16 + rr) * RLD + d) = a;  // read by this thread only
    }
    if (rg >= p.R) continue;
    const int64_t at = (rows0 + rg) * p.n_split + sp;
    if (p.n_split > 1) *reinterpret_cast<f32x4*>(p.part + at * DH + d) = a;
    if (d == 0 && p.stat) {
      p.stat[2 * at] = M;
      p.stat[2 * at + 1] = sum;
    }
  }
  if (p.n_split == 1) {
    __syncthreads();
#pragma unroll 1
    for (int rb = 0; rb < WR; ++rb) {
      const int r0 = (rtile * WR + rb) * 16;
      if (r0 < p.R) finish_rows<T, DH>(p, b, h, r0, red + rb * 16 * RLD, rot);
    }
  }
}

// Sequence of the o-th group of workgroups where every workgroup takes a whole one:
// the longest first, and every other round of 256 workgroups (one for each CU) in the
// opposite order, so that a CU which starts with a long sequence goes on with a short
// one. The order is worked out from the lengths by each workgroup for itself, which
// pays where all workgroups are resident at once (up to three a CU: nothing else
// evens them out) and each has some tokens to read: 64 sequences of 256 to 2048
// tokens, 8 key heads, 58.5 -> 52.0 us, but 64 of 1152 48.1 -> 49.7, and 128 of 305, 32
// key heads, 100 -> 123.
constexpr int kOrderMax = 256;
constexpr int kOrderWgs = 768;
__device__ __forceinline__ int in_order(const DecodeParams& p, int o, int wgs, int* s_len, int& s_b) {
  const int q = max(1, 256 / wgs), j = o / q, n = min(q, p.B - j * q);
  const int want = j * q + (j & 1 ? n - 1 - o % q : o % q);
  const int t = threadIdx.x;
  s_len[t] = t < p.B ? p.lens[t] : -0x7FFFFFFF - 1;
  __syncthreads();
  const int mine = s_len[t];
  int rank = 0;
  for (int x = 0; x < p.B; x += 4) {
    const int4 v = *reinterpret_cast<const int4*>(s_len + x);
    rank += (v.x > mine || (v.x == mine && x < t)) + (v.y > mine || (v.y == mine && x + 1 < t)) +
            (v.z > mine || (v.z == mine && x + 2 < t)) + (v.w > mine || (v.w == mine && x + 3 < t));
  }
  if (t < p.B && rank == want) s_b = t;
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(s_b);
}

// A workgroup's rows, head, sequence and split. Workgroups start in the order of their
// numbers, their XCDs take turns, and only a sequence's last splits can be empty. So the
// splits' numbers change slowest, eight by eight (one by one where there are fewer):
// the full ones start first, the heads of a sequence read its masks and slots through
// one XCD's cache, and each sequence begins on another XCD. 34 sequences of 236 to 15420
// tokens, 8 key heads of 4 rows: 183 us; with the splits' numbers changing fastest,
// 256, as full and empty ones then meet on the same XCDs. Four of 30000 to 120000, 16
// heads: 340, and 410 with the eight apart.
__device__ __forceinline__ void place(const DecodeParams& p, int nrt, int* s_len, int& s_b, int& rtile, int& h, int& b, int& sp) {
  int lin = blockIdx.x;
  rtile = lin % nrt;
  lin /= nrt;
  if (p.n_split == 1) {
    h = lin % p.c.H;
    b = p.ordered ? in_order(p, lin / p.c.H, p.c.H * nrt, s_len, s_b) : lin / p.c.H;
    sp = 0;
    return;
  }
  const int most = p.n_split >= 8 ? 8 : 1, heads = p.B * p.c.H, s0 = lin / (heads * most) * most;
  const int n = min(most, p.n_split - s0);
  lin -= s0 * heads;
  sp = lin % n;
  lin /= n;
  h = lin % p.c.H;
  b = lin / p.c.H;
  sp = s0 + (sp + b) % n;
}

// One split of one key head and 16 * WR rows: wave w takes row block w % WR and every
// (4 / WR)-th tile of tokens. Nothing is shared between the waves until their sums
// are added, so no wave waits for another: each loads its next tile's keys and
// kept groups into registers while it works on the current one, and the masks and
// slots that address them a tile earlier still. A block of 16 tokens lies in one
// page, so its keys and its groups are each one buffer resource: a dropped group or
// a page that is none is an offset past it, which reads zeros and moves nothing.
// SUB: value groups in a 16-byte piece of a row (1: a piece lies in one group).
// ONCE: keys are loaded so that they leave the caches to other data (kOnceTokens).
// Bound by memory from a few thousand tokens on: 64 sequences of 256 to 2048 tokens, 8
// key heads of 4 rows (219 MB) 46 us, 4.7 TB/s; two of 131071 tokens and 32 heads (3.36
// GB) 547 us, 6.1 TB/s, and 608 where the scores are stored for the weights, more
// than their 33 MB explain. Below that by a chain of dependent loads (length, page, mask, key and value): one
// of 305 tokens 8 us.
template <class T, int DH, int WR, int SUB, bool ONCE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(DH == 128 ? (sizeof(T) == 2 ? 3 : 2) : 4))) void k_decode(DecodeParams p) {
  using L = Tile<T, DH>;
  constexpr int TK = L::TK, NB = L::NB, EP = L::EP, KS = L::KS, NVI = L::NVI, MB = L::MB, RLD = L::RLD;
  constexpr int WT = 4 / WR, STEP = WT * TK, TPP = 64 / NB;  // tiles whose pages one load brings
  __shared__ __attribute__((aligned(16))) char smem[L::SMEM];
  __shared__ u32x2 s_rec[4][TK];
  __shared__ float s_m[4][16], s_l[4][16];
  const PagedCache& c = p.c;
  const int nrt = (p.R + 16 * WR - 1) / (16 * WR);
  __shared__ int s_b;
  int rtile, h, b, sp;
  place(p, nrt, reinterpret_cast<int*>(smem), s_b, rtile, h, b, sp);
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15,
            g4 = lane >> 4;
  const int len = tokens_of(p, b), c0 = sp * p.chunk;
  if (c0 >= len && (p.n_split > 1 || sp > 0)) return;
  const uint32_t gm = group_bits(c.G);
  const int shift = c.shift, pmask = c.page - 1, gb = c.ds * static_cast<int>(sizeof(T));

  // this lane's row, its query and the tokens it sees
  const int r = (rtile * WR + w % WR) * 16 + l16;
  int lim = 0;
  u32x4 qf[KS];
  load_query<T, DH>(p, b, h, r, g4, qf);
  if (r < p.R) lim = p.visible ? min(len, max(p.visible[static_cast<int64_t>(b) * p.Tq + r / p.rep], 0)) : len;
  int top = lim, low = r < p.R ? lim : 0x7FFFFFFF;
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) {
    top = max(top, __shfl_xor(top, o, kWave));
    low = min(low, __shfl_xor(low, o, kWave));
  }
  const int least = __builtin_amdgcn_readfirstlane(low);
  const int end = min(c0 + p.chunk, __builtin_amdgcn_readfirstlane(top));
  const int first = c0 + (w / WR) * TK;

  const rsrc_t r_table = make_rsrc(p.table + static_cast<int64_t>(b) * p.max_pages,
                                   clamp_bytes(static_cast<size_t>(p.max_pages) * 4));
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
  constexpr int XW = WR == 1 ? 4 : 1;
  __shared__ __attribute__((aligned(16))) float s_x[XW][256];
  float* px = p.x ? p.x + ((static_cast<int64_t>(b) * c.H + h) * p.R + (p.R == 1 ? 0 : r)) * p.x_ld : nullptr;

  float m = -__builtin_inff(), l = 0.f;
  f32x4 acc[MB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) acc[mb] = f32x4{0, 0, 0, 0};
  {
    int pgs = -1;     // lane j: the page of block j % NB of the (j / NB)-th of TPP tiles
    int pg1[NB];      // pages of the next tile, whose masks and slots are on their way
    uint32_t mk1 = 0;
    int sl1 = 0;
    u32x4 kf[NB][KS], vf[NVI];
    bool there[NB], there1[NB];

    // pages of tiles i .. i + TPP - 1
    auto request_pages = [&](int i) {
      const int t = first + i * STEP + lane / NB * STEP + lane % NB * 16;
      pgs = static_cast<int>(bload4(r_table, static_cast<uint32_t>(t >> shift) * 4u));  // past the row: 0
    };
    auto take_pages = [&](int i) {  // of tile i, pages that are none as -1
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int t = first + i * STEP + 16 * nb, v = __builtin_amdgcn_readlane(pgs, i % TPP * NB + nb);
        pg1[nb] = t < end && static_cast<uint32_t>(v) < static_cast<uint32_t>(c.n_pages) ? v : -1;
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
        for (int j = 0; j < KS; ++j) kf[nb][j] = bload16_hint<ONCE>(rk, ko + 64 * j);
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
        for (int x = 0; x < N; ++x) {
          vf[nb * N + x] = request_piece<SUB>(rv, tk[x].x, tk[x].y, vg, vin, gb, static_cast<uint32_t>(c.vcap));
        }
      }
    };
    auto next_pages = [&](int i) {
      if (i % TPP == 0) {
        request_pages(i);
        arrived(pgs);
      }
      take_pages(i);
    };

    request_pages(0);  // before the lengths are looked at
    take_pages(0);
    request_meta(0);
    request_keys(0);
    request_values();
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) there[nb] = there1[nb];
    next_pages(1);
    request_meta(1);
#pragma unroll 1
    for (int i = 0, t0 = first; t0 < end; ++i, t0 += STEP) {
      // scores: tokens are the rows of the product, queries its columns
      f32x4 s[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {  // in the order the keys arrive
        s[nb] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < KS; ++j) s[nb] = score_step<T>(kf[nb][j], qf[j], s[nb]);
      }
      // the tile's kept groups into their places, dropped ones as zeros
#pragma unroll
      for (int x = 0; x < NVI; ++x) *reinterpret_cast<u32x4*>(zt + (x * L::TPI + vt) * L::ZLD + 16 * pc) = vf[x];
      wave_lds_order();
      bool now[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) now[nb] = there[nb];
      request_keys(i + 1);
      request_values();
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) there[nb] = there1[nb];
      next_pages(i + 2);
      request_meta(i + 2);
      uint32_t ok = 0;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) ok |= now[nb] ? 1u << nb : 0u;
      // one row's scores are kept in pieces of 1 KB where there are that many: two of
      // 131071 tokens and 32 heads 645 -> 632 us, 8 of 8192 and 8 heads 50.5 -> 49, but one
      // of 305 8.1 -> 8.6
      constexpr int XL = TK / 4, XT = 64 / XL;  // lanes of a tile's scores, tiles of a store
      const bool alone = WR == 1 && p.x && p.R == 1 && p.chunk >= XT * STEP;
      soften<T, DH, false>(p, s, ok, t0, lim, least, end, r, px, alone ? s_x[w % XW] + i % XT * TK : nullptr, m, l, acc);
      if (alone && (i % XT == XT - 1 || t0 + STEP >= end)) {
        wave_lds_order();
        const int k = lane / XL, t = t0 + (k - i % XT) * STEP + lane % XL * 4;
        if (k <= i % XT && t < end) *reinterpret_cast<f32x4*>(px + t) = *reinterpret_cast<const f32x4*>(s_x[w % XW] + 4 * lane);
      }
      weigh_tile<T, DH, 0>(zt, s, acc);
      wave_lds_order();
    }
  }
  bool bad = false;
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
#pragma unroll
    for (int x = 0; x < 4; ++x) bad |= !__builtin_isfinite(acc[mb][x]);
  if (__any(bad)) one_by_one<T, DH>(p, b, h, r, first, STEP, end, lim, zt, m, l, acc);

  add_waves<T, DH, WR>(p, b, h, rtile, sp, m, l, acc, smem, s_m, s_l);
}

// One split of one key head and 64 rows, 16 a wave: the four waves share each tile of
// tokens. Its keys and kept groups come into registers a tile ahead, a quarter a
// wave, and go from there to one of two LDS tiles, so that one barrier a tile is
// enough: between two barriers the waves write the next tile and compute on this one.
// (With a tile to each wave, as above, every wave fetches and expands all of it:
// 16 sequences of up to 361 tokens and 56 queries took 42 us.) Those 16, 32 heads, take 32
// us; 64 of 361 108. No one unit bounds it: of the waves' time there a third is spent
// waiting for data or a barrier and a third for a turn to issue, among 267 vector
// instructions a tile and wave, 32 of them products; 12 instructions fewer changed nothing.
// A quarter of the LDS cycles are bank conflicts.
template <class T, int DH, int SUB>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(DH == 128 ? 3 : 4))) void k_decode_rows(DecodeParams p) {
  using L = Tile<T, DH>;
  constexpr int TK = L::TK, NB = L::NB, EP = L::EP, KS = L::KS, MB = L::MB;
  constexpr int KLD = L::ROWB + 16, KB = TK * KLD, BUF = KB + L::ZB;
  constexpr int TPP = 256 / L::LPT, NP = TK / TPP;  // tokens of a pass of the workgroup, passes
  static_assert(NP >= 1 && (16 % TPP == 0 || TPP % 16 == 0), "a wave's pass lies in one block of 16 tokens");
  constexpr int SMEM = 2 * BUF > 4 * L::RB ? 2 * BUF : 4 * L::RB;
  constexpr int TPG = 64 / NB;  // tiles whose pages one load brings
  __shared__ __attribute__((aligned(16))) char smem[SMEM];
  __shared__ float s_m[4][16], s_l[4][16];
  static_assert(SMEM / 4 >= 16 * DH * 4, "a wave's sums fit its quarter");
  const PagedCache& c = p.c;
  const int nrt = (p.R + 63) / 64;
  __shared__ int s_b;
  int rtile, h, b, sp;
  place(p, nrt, reinterpret_cast<int*>(smem), s_b, rtile, h, b, sp);
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15,
            g4 = lane >> 4;
  const int len = tokens_of(p, b), c0 = sp * p.chunk;
  if (c0 >= len && p.n_split > 1) return;
  const uint32_t gm = group_bits(c.G);
  const int shift = c.shift, pmask = c.page - 1, gb = c.ds * static_cast<int>(sizeof(T));
  const int r = (rtile * 4 + w) * 16 + l16;
  u32x4 qf[KS];
  load_query<T, DH>(p, b, h, r, g4, qf);
  int lim = 0;
  if (r < p.R) lim = p.visible ? min(len, max(p.visible[static_cast<int64_t>(b) * p.Tq + r / p.rep], 0)) : len;
  int top = lim, low = r < p.R ? lim : 0x7FFFFFFF;
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) {
    top = max(top, __shfl_xor(top, o, kWave));
    low = min(low, __shfl_xor(low, o, kWave));
  }
  const int least = __builtin_amdgcn_readfirstlane(low);
  if (lane == 0) s_m[w][0] = __int_as_float(top);
  __syncthreads();
  int all = max(max(__float_as_int(s_m[0][0]), __float_as_int(s_m[1][0])),
                max(__float_as_int(s_m[2][0]), __float_as_int(s_m[3][0])));
  const int end = min(c0 + p.chunk, __builtin_amdgcn_readfirstlane(all));

  const rsrc_t r_table = make_rsrc(p.table + static_cast<int64_t>(b) * p.max_pages,
                                   clamp_bytes(static_cast<size_t>(p.max_pages) * 4));
  const uint32_t meta_bytes = static_cast<uint32_t>(c.n_pages) << (shift + 2);  // below 2 GiB
  const rsrc_t r_mask = make_rsrc(c.mask, meta_bytes), r_slot = make_rsrc(c.slot, meta_bytes);
  // bytes of a head's part of a page, and of a page (below 2 GiB)
  const uint32_t kstep = static_cast<uint32_t>(c.page) * L::ROWB, vstep = static_cast<uint32_t>(c.vcap) * gb;
  const uint32_t kpage = kstep * c.H, vpage = vstep * c.H;
  const char* khead = static_cast<const char*>(c.K) + static_cast<size_t>(h) * kstep;
  const char* vhead = static_cast<const char*>(c.V) + static_cast<size_t>(h) * vstep;

  // this thread's pieces: part pc of tokens vt + TPP x of every tile
  const int pc = tid % L::LPT, vt = tid / L::LPT;
  const int vg = SUB == 1 ? pc * 16 / gb : pc * SUB;
  const uint32_t vin = SUB == 1 ? static_cast<uint32_t>(pc * 16 % gb) : 0u;
  float* px = p.x ? p.x + ((static_cast<int64_t>(b) * c.H + h) * p.R + r) * p.x_ld : nullptr;

  int pgs = 0;                    // lane j: the page of block j % NB of the (j / NB)-th of TPG tiles
  uint32_t there = 0, now = 0;    // bit nb: that block's page is one (of the tile in registers, in hand)
  int pg1[NP], pgm[NP];           // pages of this wave's passes: of the tile whose masks are asked for next
  uint32_t mk[NP];
  int sl0[NP];
  u32x4 kf[NP], vf[NP];
  auto block_of = [&](int x) { return (x * TPP + w * (64 / L::LPT)) / 16; };  // of this wave's pass x
  auto take_pages = [&](int i) {
    if (i % TPG == 0) {
      const int t = c0 + i * TK + lane / NB * TK + lane % NB * 16;
      pgs = static_cast<int>(bload4(r_table, static_cast<uint32_t>(t >> shift) * 4u));  // past the row: 0
      arrived(pgs);
    }
    there = 0;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int v = __builtin_amdgcn_readlane(pgs, i % TPG * NB + nb);
      const bool in = c0 + i * TK + 16 * nb < end && static_cast<uint32_t>(v) < static_cast<uint32_t>(c.n_pages);
      there |= in ? 1u << nb : 0u;
#pragma unroll
      for (int x = 0; x < NP; ++x)
        if (block_of(x) == nb) pg1[x] = in ? v : -1;
    }
  };
  auto request_meta = [&](int i) {
#pragma unroll
    for (int x = 0; x < NP; ++x) {
      const int t = c0 + i * TK + x * TPP + vt;
      const uint32_t off = oob_unless(t < end && pg1[x] >= 0,
                                      (static_cast<uint32_t>(pg1[x]) << (shift + 2)) + static_cast<uint32_t>(t & pmask) * 4u);
      mk[x] = bload4(r_mask, off);
      sl0[x] = static_cast<int>(bload4(r_slot, off));
      pgm[x] = pg1[x];
    }
  };
  auto request_tile = [&](int i) {  // whose masks have been asked for
#pragma unroll
    for (int x = 0; x < NP; ++x) {
      const rsrc_t rk = make_rsrc(khead + static_cast<uint64_t>(max(pgm[x], 0)) * kpage, pgm[x] >= 0 ? kstep : 0u);
      const int t = c0 + i * TK + x * TPP + vt;
      kf[x] = bload16(rk, static_cast<uint32_t>(t & pmask) * L::ROWB + 16 * pc);
    }
#pragma unroll
    for (int x = 0; x < NP; ++x) {
      const rsrc_t rv = make_rsrc(vhead + static_cast<uint64_t>(max(pgm[x], 0)) * vpage, pgm[x] >= 0 ? vstep : 0u);
      vf[x] = request_piece<SUB>(rv, mk[x] & gm, static_cast<uint32_t>(sl0[x]), vg, vin, gb, static_cast<uint32_t>(c.vcap));
    }
  };
  auto put_tile = [&](char* buf) {
#pragma unroll
    for (int x = 0; x < NP; ++x) {
      *reinterpret_cast<u32x4*>(buf + (x * TPP + vt) * KLD + 16 * pc) = kf[x];
      *reinterpret_cast<u32x4*>(buf + KB + (x * TPP + vt) * L::ZLD + 16 * pc) = vf[x];
    }
  };

  float m = -__builtin_inff(), l = 0.f;
  f32x4 acc[MB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) acc[mb] = f32x4{0, 0, 0, 0};
  uint32_t there0, there1;
  take_pages(0);
  there0 = there;
  request_meta(0);
  request_tile(0);
  take_pages(1);
  there1 = there;
  request_meta(1);
  put_tile(smem);
  request_tile(1);
  take_pages(2);
  request_meta(2);
#pragma unroll 1
  for (int i = 0, t0 = c0; t0 < end; ++i, t0 += TK) {
    __syncthreads();
    const char* buf = smem + (i & 1) * BUF;
    now = there0;
    put_tile(smem + ((i + 1) & 1) * BUF);
    there0 = there1;
    there1 = there;
    request_tile(i + 2);
    take_pages(i + 3);
    request_meta(i + 3);
    f32x4 s[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) s[nb] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < KS; ++j)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
        s[nb] = score_step<T>(*reinterpret_cast<const u32x4*>(buf + (16 * nb + l16) * KLD + 64 * j + 16 * g4), qf[j], s[nb]);
    soften<T, DH, true>(p, s, now, t0, lim, least, end, r, px, nullptr, m, l, acc);
    weigh_tile<T, DH, 2>(buf + KB, s, acc);
  }
  __syncthreads();
  bool bad = false;
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
#pragma unroll
    for (int x = 0; x < 4; ++x) bad |= !__builtin_isfinite(acc[mb][x]);
  if (__any(bad)) one_by_one<T, DH>(p, b, h, r, c0, TK, end, lim, smem + w * (SMEM / 4), m, l, acc);
  add_waves<T, DH, 4>(p, b, h, rtile, sp, m, l, acc, smem, s_m, s_l);
}

// The maxima and sums of exponentials of J rows from their splits' statistics; `step`
// lanes share a row's splits. The rows' loads are in flight together, and a lane's first
// split is read once.
template <int J>
__device__ __forceinline__ void join_stat(const float* const (&st)[J], int ns, int from, int step, float (&M)[J], float (&sum)[J]) {
  float2 v[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    v[j] = float2{-__builtin_inff(), 0.f};
    if (from < ns) v[j] = *reinterpret_cast<const float2*>(st[j] + 2 * from);
  }
#pragma unroll
  for (int j = 0; j < J; ++j) M[j] = v[j].x;
  for (int i = from + step; i < ns; i += step)
#pragma unroll
    for (int j = 0; j < J; ++j) M[j] = fmaxf(M[j], st[j][2 * i]);
  for (int o = 1; o < step; o <<= 1)
#pragma unroll
    for (int j = 0; j < J; ++j) M[j] = fmaxf(M[j], __shfl_xor(M[j], o, kWave));
#pragma unroll
  for (int j = 0; j < J; ++j) sum[j] = v[j].y * weight_of(v[j].x, M[j]);
  for (int i = from + step; i < ns; i += step)
#pragma unroll
    for (int j = 0; j < J; ++j) sum[j] += st[j][2 * i + 1] * weight_of(st[j][2 * i], M[j]);
  for (int o = 1; o < step; o <<= 1)
#pragma unroll
    for (int j = 0; j < J; ++j) sum[j] += __shfl_xor(sum[j], o, kWave);
}

// The splits of 16 rows of one key head added, normalised and rotated back.
template <class T, int DH>
__device__ __forceinline__ void join_rows(const DecodeParams& p, int64_t blk, char* smem) {
  using L = Tile<T, DH>;
  constexpr int Q = DH / 4;  // 16-byte pieces of a row
  float* u = reinterpret_cast<float*>(smem);                      // [16][RLD]
  f32x4* red = reinterpret_cast<f32x4*>(smem + L::RB);            // [256]
  float* s_M = reinterpret_cast<float*>(smem + L::RB + 4096);     // [16] maxima, [16] sums
  const PagedCache& c = p.c;
  const int nrb = (p.R + 15) / 16, tid = threadIdx.x;
  const int r0 = static_cast<int>(blk % nrb) * 16, h = static_cast<int>(blk / nrb % c.H), b = static_cast<int>(blk / nrb / c.H);
  Rotation<T, DH> rot;
  rot.load(p, h);
  const int ns = (tokens_of(p, b) + p.chunk - 1) / p.chunk, nr = min(16, p.R - r0);
  const int64_t cell0 = ((static_cast<int64_t>(b) * c.H + h) * p.R + r0) * p.n_split;
  {
    const int row = tid / 16;
    const float* const st[1] = {p.stat + 2 * (cell0 + static_cast<int64_t>(min(row, nr - 1)) * p.n_split)};
    float M[1], sum[1];
    join_stat(st, ns, tid % 16, 16, M, sum);
    if (tid % 16 == 0) {
      s_M[row] = M[0];
      s_M[16 + row] = row >= nr ? 0.f : sum[0];
    }
  }
  __syncthreads();
  // few rows: their splits are shared out among groups of threads
  const int items = nr * Q, groups = max(1, 256 / items);
  for (int it0 = 0; it0 < 16 * Q; it0 += 256) {
    const int it = it0 + tid % (groups > 1 ? items : 256), g = groups > 1 ? tid / items : 0;
    f32x4 a = {0, 0, 0, 0};
    const int row = it / Q, d = it % Q;
    if (row < nr && g < groups) {
      const int64_t cell = cell0 + static_cast<int64_t>(row) * p.n_split;
      const float M = s_M[row];
#pragma unroll 4
      for (int i = g; i < ns; i += groups)
        a += *reinterpret_cast<const f32x4*>(p.part + (cell + i) * DH + 4 * d) * weight_of(p.stat[2 * (cell + i)], M);
    }
    if (groups > 1) {
      red[tid] = a;
      __syncthreads();
      if (tid < items)
        for (int v = 1; v < groups; ++v) a += red[tid + v * items];
      if (tid < items) *reinterpret_cast<f32x4*>(u + row * L::RLD + 4 * d) = s_M[16 + row] == 0.f ? f32x4{0, 0, 0, 0} : a / s_M[16 + row];
      for (int z = tid; z < (16 - nr) * Q; z += 256)
        *reinterpret_cast<f32x4*>(u + (nr + z / Q) * L::RLD + z % Q * 4) = f32x4{0, 0, 0, 0};
      break;
    }
    *reinterpret_cast<f32x4*>(u + row * L::RLD + 4 * d) = s_M[16 + row] == 0.f ? f32x4{0, 0, 0, 0} : a / s_M[16 + row];
  }
  __syncthreads();
  finish_rows<T, DH>(p, b, h, r0, u, rot);
}

// mass_out[b,t] = decay mass_in[b,t] + the token's weight in every row. A workgroup
// takes `per` blocks of TB tokens, and the lanes of one every (256 / TB)-th row each: the rows' sums of
// exponentials first, J rows of each 8 lanes at a time, while the first scores are on
// their way.
constexpr int kMassRows = 512;
template <int J>
__device__ __forceinline__ void row_sums(const DecodeParams& p, int b, int q1, int64_t row0, int n, int ns, int len, float* s_lse, int* s_lim) {
  const int tid = threadIdx.x;
  for (int q0 = 0; q0 < n; q0 += 32 * J) {
    const float* st[J];
    float M[J], l[J];
    int lim[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int q = min(q0 + 32 * j + tid / 8, n - 1);
      st[j] = p.stat + 2 * (row0 + q) * p.n_split;
      lim[j] = p.visible ? p.visible[static_cast<int64_t>(b) * p.Tq + (q1 + q) % p.R / p.rep] : len;
    }
    join_stat<J>(st, ns, tid % 8, 8, M, l);
    if (tid % 8 == 0)
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int q = q0 + 32 * j + tid / 8;
        s_lse[q] = M[j] + __log2f(l[j]);  // -inf where nothing was seen
        s_lim[q] = l[j] == 0.f || q >= n ? 0 : lim[j];
      }
  }
}
// U: scores of a lane in flight, and as many that it works on; PH lanes share a token.
template <int J, int U, int PH>
__device__ __forceinline__ float add_rows(const DecodeParams& p, int b, int q1, int64_t row0, int n, int ns, int len, int t, int ph,
                                          bool fresh, float sum, float* s_lse, int* s_lim) {
  const float* px = p.x + row0 * p.x_ld + min(t, p.x_ld - 1);
  float x[U], y[U] = {};
#pragma unroll
  for (int i = 0; i < U; ++i) x[i] = px[static_cast<int64_t>(min(PH * i + ph, n - 1)) * p.x_ld];
  if (fresh) {
    row_sums<J>(p, b, q1, row0, n, ns, len, s_lse, s_lim);
    __syncthreads();
  }
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += PH * U) {
    if (i0 + PH * U < n)
#pragma unroll
      for (int i = 0; i < U; ++i) y[i] = px[static_cast<int64_t>(min(i0 + PH * (U + i) + ph, n - 1)) * p.x_ld];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int q = i0 + PH * i + ph;
      sum += t < s_lim[q] ? exp2_(x[i] - s_lse[q]) : 0.f;
      x[i] = y[i];
    }
  }
  return sum;
}
template <int TB>
__device__ __forceinline__ void add_mass(const DecodeParams& p, int64_t blk, int nblk, int per, char* smem) {
  constexpr int PH = 256 / TB;
  float* s_lse = reinterpret_cast<float*>(smem);
  int* s_lim = reinterpret_cast<int*>(smem + kMassRows * 4);
  float* s_sum = reinterpret_cast<float*>(smem + kMassRows * 8);
  const int b = static_cast<int>(blk / nblk), tid = threadIdx.x, ph = tid / TB, len = tokens_of(p, b);
  const int first = static_cast<int>(blk % nblk) * TB * per, end = min(len, first + TB * per);
  const int ns = (len + p.chunk - 1) / p.chunk;
  const int rows = p.c.H * p.R;  // at most 2^28: a launch has 16 threads a row and less than 2^32
  const int64_t row0 = static_cast<int64_t>(b) * rows;
#pragma unroll 1
  for (int t0 = first; t0 < end; t0 += TB) {
    const int t = t0 + tid % TB;
    float sum = 0.f;
    for (int q0 = 0; q0 < rows; q0 += kMassRows) {
      const int n = min(rows - q0, kMassRows);
      const bool fresh = t0 == first || rows > kMassRows;
      if (q0 || t0 > first) __syncthreads();
      sum = n <= 32 ? add_rows<1, 32 / PH, PH>(p, b, q0, row0 + q0, n, ns, len, t, ph, fresh, sum, s_lse, s_lim)
                    : add_rows<4, TB == 64 ? 16 : 8, PH>(p, b, q0, row0 + q0, n, ns, len, t, ph, fresh, sum, s_lse, s_lim);
    }
    s_sum[tid] = sum;
    __syncthreads();
    if (ph == 0 && t < len) {
      sum = 0.f;
#pragma unroll
      for (int i = 0; i < PH; i += 4)
        sum += (s_sum[TB * i + tid] + s_sum[TB * (i + 1) + tid]) + (s_sum[TB * (i + 2) + tid] + s_sum[TB * (i + 3) + tid]);
      const int64_t at = static_cast<int64_t>(b) * p.mass_ld + t;
      p.mass_out[at] = p.mass_in ? p.decay * p.mass_in[at] + sum : sum;
    }
  }
}

// What follows the splits: the first `joins` workgroups finish the outputs, the
// others add the weights. A chain of dependent loads, 5 us for one of 305 tokens and 32
// heads; two of 131071 read 34 MB of scores and 32 splits' sums in 21 us.
template <class T, int DH>
__global__ __launch_bounds__(256) void k_join(DecodeParams p, int joins, int nblk, int tb, int per) {
  using L = Tile<T, DH>;
  __shared__ __attribute__((aligned(16))) char smem[L::RB + 4096 + 128];
  static_assert(sizeof(smem) >= kMassRows * 8 + 1024, "both halves fit");
  if (static_cast<int>(blockIdx.x) < joins)
    join_rows<T, DH>(p, blockIdx.x, smem);
  else if (tb == 64)
    add_mass<64>(p, static_cast<int64_t>(blockIdx.x) - joins, nblk, per, smem);
  else
    add_mass<16>(p, static_cast<int64_t>(blockIdx.x) - joins, nblk, 1, smem);
}

// Blocks of 16 rows of a workgroup. From 17 rows on a tile of bfloat16 tokens is worth
// sharing among all four waves where its keys and values are 32 KB and more (4: dims
// of 128): 8 sequences of 8192 tokens, 8 key heads of 32 rows 75 -> 69 us, 42 of 4748 to
// 12482 of 20 rows 391 -> 281, but 64 of 361 of 24 rows 26.9 -> 28.3; dims of 64, 8 of 8192
// of 20 rows 37.9 -> 40.7; float32, 8 of 8192 of 20 rows 143 -> 180.
constexpr bool share_from_17(bool bf16, int dh) { return bf16 && dh == 128; }
int row_blocks(int R, bool bf16, int dh) { return R <= 16 ? 1 : R <= 32 && !share_from_17(bf16, dh) ? 2 : 4; }

// Sequences from which on keys pass the caches by: 64 of up to 2048 tokens and 8 key
// heads 51.5 -> 47, 64 of 1152 49.5 -> 45.5, two of 131071 and 32 heads 560 -> 550 us, but
// 128 of 305 and 32 heads 100 -> 107. Not where scores are kept for the tokens' weights,
// whose stores go through the same caches: two of 131071 and 32 heads 631 -> 676, and 8
// heads of 4 rows 182 -> 195, four of 32768 and 32 heads 319 -> 335, though shorter
// batches would gain (64 of up to 2048, 8 heads of 4 rows 64.6 -> 59.2).
constexpr int kOnceTokens = 1024;

template <class T, int DH, int WR, int SUB>
auto kernel_of(const DecodeParams& p) {
  if constexpr (WR == 4)
    return k_decode_rows<T, DH, SUB>;
  else
    return p.max_len >= kOnceTokens && !p.x ? k_decode<T, DH, WR, SUB, true> : k_decode<T, DH, WR, SUB, false>;
}

template <class T, int DH, int WR>
void go(const DecodeParams& p, hipStream_t s) {
  const int sub = p.c.ds >= Tile<T, DH>::EP ? 1 : Tile<T, DH>::EP / p.c.ds;
  auto kern = sub == 1 ? kernel_of<T, DH, WR, 1>(p) : kernel_of<T, DH, WR, 2>(p);
  if constexpr (sizeof(T) == 2) {
    if (sub == 4) kern = kernel_of<T, DH, WR, 4>(p);
  }
  const int nrt = (p.R + 16 * WR - 1) / (16 * WR);
  hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(nrt) * p.n_split * p.c.H * p.B), dim3(256), 0, s, p);
}

template <class T, int DH>
hipError_t launch(DecodeParams p, hipStream_t s) {
  const int WR = row_blocks(p.R, sizeof(T) == 2, DH);
  const int64_t wgs = static_cast<int64_t>(p.B) * p.c.H * ((p.R + 63) / 64);
  p.ordered = p.n_split == 1 && p.B > 1 && p.B <= kOrderMax && wgs > 256 && wgs <= kOrderWgs && p.max_len >= 512;
  if (WR == 1)
    go<T, DH, 1>(p, s);
  else if (WR == 4)
    go<T, DH, 4>(p, s);
  else if constexpr (!share_from_17(sizeof(T) == 2, DH))
    go<T, DH, 2>(p, s);
  const int joins = p.n_split > 1 ? (p.R + 15) / 16 * p.c.H * p.B : 0;
  const int64_t blocks = static_cast<int64_t>(p.B) * ((p.max_len + 63) / 64), rows = static_cast<int64_t>(p.c.H) * p.R;
  // many rows and blocks of 64 tokens on half the CUs or fewer: of 16 (305 tokens and 1280
  // rows 55 -> 35 us, two of 3447 and 528 rows 73 -> 55)
  const int tb = blocks <= 128 && rows > 128 ? 16 : 64;
  // many blocks: up to eight a workgroup, for which it takes the rows' sums once (64
  // sequences of 16384 tokens, 8 key heads of 4 rows 719 -> 705 us; 8 of 20000, 4 of 64 139 -> 141)
  const int per = rows > kMassRows ? 1 : static_cast<int>(std::min<int64_t>(8, std::max<int64_t>(1, blocks / 1024)));
  const int nblk = p.mass_out ? (p.max_len + tb * per - 1) / (tb * per) : 0;
  if (joins + nblk > 0)
    hipLaunchKernelGGL((k_join<T, DH>), dim3(static_cast<unsigned>(joins) + static_cast<unsigned>(nblk) * p.B), dim3(256),
                       0, s, p, joins, nblk, tb, per);
  return hipGetLastError();
}

// Workgroups that the splits are made for: two for each of the 256 CUs. More splits
// cost more to add up than they even out: 64 sequences of 256 to 2048 tokens and 8
// key heads take 60 us in one split each, 73 in two, 66 in four; 16 of 361 tokens
// and 56 queries 40 against 64. Short sequences in one split without the weights, whose
// adding takes the second launch anyway, would save that launch (one of 305 tokens, 32
// heads: 12.2 against 14.4 us), but a call's outputs would then depend on whether it
// adds up weights.
constexpr int64_t kSplitWgs = 512;
// Splits of more than 2048 tokens cost next to nothing to add up, and up to 2048
// workgroups of them even out a ragged batch: 34 sequences of 236 to 15420 tokens, 8 key
// heads of 4 rows 259 -> 183 us, 23 of 7727 to 22794 290 -> 215, 34 of 8192 192 -> 170. Not
// where one split each is had in order of length: 64 of 256 to 16384 302 -> 347.
constexpr int64_t kLongUnits = 16, kLongWgs = 2048;
constexpr int64_t kMaxSplits = 256;  // that k_join adds up

size_t up256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

}  // namespace

DecodePlan decode_plan(int B, int H, int R, int dh, int max_len, bool mass) {
  DecodePlan d;
  const int nrt = (R + 63) / 64;  // whatever row_blocks says
  const int64_t units = (static_cast<int64_t>(max_len) + 127) / 128;  // of 128 tokens, a tile for each of four waves
  const int64_t wgs = static_cast<int64_t>(B) * H * nrt;
  const int64_t least = (units + kMaxSplits - 1) / kMaxSplits;
  int64_t per = std::max((units * wgs + kSplitWgs - 1) / kSplitWgs, least);
  if (per > kLongUnits && (per < units || wgs > kOrderWgs))
    per = std::max({kLongUnits, (units * wgs + kLongWgs - 1) / kLongWgs, least});
  d.chunk = static_cast<int>(128 * std::max<int64_t>(1, std::min(per, units)));
  d.n_split = std::max(1, static_cast<int>((static_cast<int64_t>(max_len) + d.chunk - 1) / d.chunk));
  d.x_ld = (max_len + 3) / 4 * 4;
  const size_t rows = static_cast<size_t>(B) * H * R, cells = rows * d.n_split;
  d.off_stat = d.n_split > 1 ? up256(cells * dh * 4) : 0;
  d.off_x = d.off_stat + (d.n_split > 1 || (mass && max_len > 0) ? up256(cells * 8) : 0);
  d.bytes = d.off_x + (mass ? up256(rows * d.x_ld * 4) : 0);
  // what to ask a caller for: a bound on the above that does not fall as B, Tq or
  // max_len grows (n_split <= kSplitWgs / wgs + 1, or for splits of kLongUnits and more
  // kLongWgs / wgs + 1 and units / kLongUnits + 1; R <= 64 nrt)
  const size_t r64 = std::min<size_t>(R, 64);
  const size_t longs = std::min(r64 * kLongWgs, rows * static_cast<size_t>(units / kLongUnits)) + rows;
  const size_t most = std::min(rows * static_cast<size_t>(std::min(units, kMaxSplits)), std::max(r64 * kSplitWgs + rows, longs));
  d.ask = up256(most * dh * 4) + up256(most * 8) + (mass ? up256(rows * d.x_ld * 4) : 0);
  return d;
}

hipError_t launch_decode(const DecodeParams& p, bool bf16, hipStream_t s) {
  if (bf16) return p.c.dh == 128 ? launch<__bf16, 128>(p, s) : launch<__bf16, 64>(p, s);
  return p.c.dh == 128 ? launch<float, 128>(p, s) : launch<float, 64>(p, s);
}

}  // namespace rolesub
