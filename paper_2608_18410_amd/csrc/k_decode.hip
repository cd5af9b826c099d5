// Attention of new tokens over the paged routed cache, split over its length.
//
//   s[r,t] = scale <q_r, k_t>,  P = softmax over the tokens a row sees,
//   u_r    = sum_t P[r,t] (M_t z_t),  out_r = R_h u_r
//
// The rows of one key head are its rep = Hq / H query heads times Tq queries.
// Splits of `chunk` tokens are computed by separate workgroups into partial sums
// with their maximum and sum of exponentials; k_join adds them and rotates back.
#include <algorithm>

#include "common.hpp"
#include "launch.hpp"

namespace rolesub {
namespace {

__device__ __forceinline__ uint32_t group_bits(int G) { return G >= 32 ? 0xFFFFFFFFu : (1u << G) - 1u; }

// Four bf16 rows of 16 columns, transposed: 16 lanes give the addresses of the
// rows' 8-byte quarters, lane i gets column i of the four rows.
__device__ __forceinline__ bf16x4 lds_read_tr(const char* p) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef s16x4 __attribute__((address_space(3))) * p3;
  return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((p3)(p)));
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// Factor of sums taken against the maximum m once the maximum is M. Sums without a
// score above -inf are zeros, or NaN where a score was: they are added as they are.
__device__ __forceinline__ float weight_of(float m, float M) { return m == -__builtin_inff() ? 1.f : exp2_(m - M); }

struct alignas(16) TokenRec {
  uint32_t mask;
  int32_t slot, page, pad;
};

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
  static constexpr int SMEM = 4 * ZB > 4 * 16 * RLD * 4 ? 4 * ZB : 4 * 16 * RLD * 4;
  static constexpr int MB = DH / 16;
};

// SUB: value groups in a 16-byte piece of a row (1: a piece lies in one group).
template <class T, int DH, int RT, int SUB>
__global__ __launch_bounds__(256) void k_decode(DecodeParams p) {
  using L = Tile<T, DH>;
  constexpr int TK = L::TK, NB = L::NB, EP = L::EP, KS = L::KS, NVI = L::NVI, MB = L::MB, RLD = L::RLD;
  __shared__ __attribute__((aligned(16))) char smem[L::SMEM];
  __shared__ TokenRec s_rec[4][TK];
  __shared__ float s_m[4][16 * RT], s_l[4][16 * RT];
  const PagedCache& c = p.c;
  const int nrt = (p.R + 16 * RT - 1) / (16 * RT);
  int lin = blockIdx.x;
  const int rtile = lin % nrt;
  lin /= nrt;
  const int sp = lin % p.n_split;
  lin /= p.n_split;
  const int h = lin % c.H, b = lin / c.H;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15,
            g4 = lane >> 4;
  const int64_t cap = static_cast<int64_t>(p.max_pages) << c.shift;
  const int len = static_cast<int>(min(static_cast<int64_t>(min(max(p.lens[b], 0), p.max_len)), cap));
  const int c0 = sp * p.chunk;
  if (c0 >= len) return;
  const uint32_t gm = group_bits(c.G);

  int lim[RT];  // tokens this lane's rows see
  int top = 0;
  uint4 qf[RT][KS];
#pragma unroll
  for (int k = 0; k < RT; ++k) {
    const int r = (rtile * RT + k) * 16 + l16;
    lim[k] = 0;
#pragma unroll
    for (int j = 0; j < KS; ++j) qf[k][j] = uint4{0, 0, 0, 0};
    if (r < p.R) {
      const int jq = r / p.rep, hq = h * p.rep + r % p.rep;
      lim[k] = p.visible ? min(len, max(p.visible[static_cast<int64_t>(b) * p.Tq + jq], 0)) : len;
      const T* q = static_cast<const T*>(p.q) + (static_cast<int64_t>(b) * p.Tq + jq) * p.q_stride +
                   static_cast<int64_t>(hq) * DH;
#pragma unroll
      for (int j = 0; j < KS; ++j) qf[k][j] = *reinterpret_cast<const uint4*>(q + (4 * j + g4) * EP);
    }
    top = max(top, lim[k]);
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) top = max(top, __shfl_xor(top, o, kWave));
  const int end = min(c0 + p.chunk, __builtin_amdgcn_readfirstlane(top));

  float m[RT], l[RT];
  f32x4 acc[RT][MB];
  char* zt = smem + w * L::ZB;
  TokenRec* rec = s_rec[w];
  // The second round runs only where the first one's sums are not finite: it adds
  // token by token, so that an infinity or NaN in a value reaches the rows that
  // see its token and no other (a matrix product multiplies it by their zeros).
#pragma unroll 1
  for (int round = 0; round < 2; ++round) {
#pragma unroll
    for (int k = 0; k < RT; ++k) {
      m[k] = -__builtin_inff();
      l[k] = 0.f;
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) acc[k][mb] = f32x4{0, 0, 0, 0};
    }
#pragma unroll 1
    for (int t0 = c0 + w * TK; t0 < end; t0 += 4 * TK) {
      TokenRec mine = {0, 0, -1, 0};
      if (lane < TK && t0 + lane < end) {
        const int t = t0 + lane;
        const int32_t pg = p.table[static_cast<int64_t>(b) * p.max_pages + (t >> c.shift)];
        if (static_cast<uint32_t>(pg) < static_cast<uint32_t>(c.n_pages)) {
          const int64_t meta = (static_cast<int64_t>(pg) << c.shift) + (t & (c.page - 1));
          mine = TokenRec{c.mask[meta] & gm, c.slot[meta], pg, 0};
        }
      }
      if (lane < TK) rec[lane] = mine;
      wave_lds_order();
      // scores: tokens are the rows of the product, queries its columns
      bool there[NB];
      f32x4 s[RT][NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int pg = __builtin_amdgcn_readlane(mine.page, 16 * nb);  // a page holds whole blocks of 16 tokens
        there[nb] = pg >= 0;
#pragma unroll
        for (int k = 0; k < RT; ++k) s[k][nb] = f32x4{0, 0, 0, 0};
        if (!there[nb]) continue;
        const int row = (t0 + 16 * nb) & (c.page - 1);
        const char* kp = static_cast<const char*>(c.K) +
                         (((static_cast<int64_t>(pg) * c.H + h) << c.shift) + row + l16) * L::ROWB + 16 * g4;
        uint4 kf[KS];
#pragma unroll
        for (int j = 0; j < KS; ++j) kf[j] = *reinterpret_cast<const uint4*>(kp + 64 * j);
#pragma unroll
        for (int j = 0; j < KS; ++j)
#pragma unroll
          for (int k = 0; k < RT; ++k) {
            if constexpr (L::kBf16) {
              s[k][nb] = mfma_16x16x32(__builtin_bit_cast(bf16x8, kf[j]), __builtin_bit_cast(bf16x8, qf[k][j]), s[k][nb]);
            } else {
              const f32x4 a = __builtin_bit_cast(f32x4, kf[j]), q = __builtin_bit_cast(f32x4, qf[k][j]);
#pragma unroll
              for (int i = 0; i < 4; ++i) s[k][nb] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], q[i], s[k][nb], 0, 0, 0);
            }
          }
      }
      // the tile's kept groups into their places, dropped ones as zeros
#pragma unroll
      for (int i = 0; i < NVI; ++i) {
        const int tk = i * L::TPI + lane / L::LPT, pc = lane % L::LPT;
        const TokenRec r = rec[tk];
        const int64_t base = (static_cast<int64_t>(r.page) * c.H + h) * c.vcap;
        uint4 v = {0, 0, 0, 0};
        if constexpr (SUB == 1) {
          const int g = pc * EP / c.ds, sl = r.slot + __popc(r.mask & ((1u << g) - 1u));
          if (((r.mask >> g) & 1u) && static_cast<uint32_t>(sl) < static_cast<uint32_t>(c.vcap))
            v = *reinterpret_cast<const uint4*>(static_cast<const T*>(c.V) + (base + sl) * c.ds + pc * EP % c.ds);
        } else {
          constexpr int W = 4 / SUB;  // 32-bit words of a group
          uint32_t* vv = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
          for (int u = 0; u < SUB; ++u) {
            const int g = pc * SUB + u, sl = r.slot + __popc(r.mask & ((1u << g) - 1u));
            if (((r.mask >> g) & 1u) && static_cast<uint32_t>(sl) < static_cast<uint32_t>(c.vcap)) {
              const uint32_t* src = reinterpret_cast<const uint32_t*>(static_cast<const T*>(c.V) + (base + sl) * c.ds);
#pragma unroll
              for (int x = 0; x < W; ++x) vv[u * W + x] = src[x];
            }
          }
        }
        *reinterpret_cast<uint4*>(zt + tk * L::ZLD + 16 * pc) = v;
      }
      wave_lds_order();
      // softmax against the running maximum
#pragma unroll
      for (int k = 0; k < RT; ++k) {
        float mx = -__builtin_inff();
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool see = there[nb] && t0 + 16 * nb + 4 * g4 + i < lim[k];
            s[k][nb][i] = see ? s[k][nb][i] * p.scale : -__builtin_inff();
            mx = fmaxf(mx, s[k][nb][i]);
          }
          const int r = (rtile * RT + k) * 16 + l16, t = t0 + 16 * nb + 4 * g4;
          if (p.x && r < p.R && t < end)
            *reinterpret_cast<f32x4*>(p.x + ((static_cast<int64_t>(b) * c.H + h) * p.R + r) * p.x_ld + t) = s[k][nb];
        }
        mx = max_xor32(max_xor16(mx));
        const float mn = fmaxf(m[k], mx), ms = mn == -__builtin_inff() ? 0.f : mn;
        const float al = exp2_(m[k] - ms);
        m[k] = mn;
        float sum = 0.f;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            s[k][nb][i] = exp2_(s[k][nb][i] - ms);
            sum += s[k][nb][i];
          }
        l[k] = l[k] * al + sum;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) acc[k][mb] *= al;
      }
      if (round == 0) {
        if constexpr (L::kBf16) {
          // weights as two bf16 each, so that their rounding stays below the output's
          bf16x8 hi[RT], lo[RT];
#pragma unroll
          for (int k = 0; k < RT; ++k)
#pragma unroll
            for (int x = 0; x < 8; ++x) {
              const float pv = s[k][x / 4][x % 4];
              hi[k][x] = fromf<bf16>(pv);
              lo[k][x] = fromf<bf16>(pv - tof(hi[k][x]));
            }
          const char* zr = zt + (4 * g4 + l16 / 4) * L::ZLD + 8 * (l16 % 4);
#pragma unroll
          for (int mb = 0; mb < MB; ++mb) {
            const bf16x4 a0 = lds_read_tr(zr + 32 * mb), a1 = lds_read_tr(zr + 16 * L::ZLD + 32 * mb);
            const bf16x8 a = __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int k = 0; k < RT; ++k) {
              acc[k][mb] = mfma_16x16x32(a, hi[k], acc[k][mb]);
              acc[k][mb] = mfma_16x16x32(a, lo[k], acc[k][mb]);
            }
          }
        } else {
#pragma unroll
          for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float a = *reinterpret_cast<const float*>(zt + (4 * g4 + i) * L::ZLD + 4 * (16 * mb + l16));
#pragma unroll
              for (int k = 0; k < RT; ++k)
                acc[k][mb] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, s[k][0][i], acc[k][mb], 0, 0, 0);
            }
        }
      } else {
#pragma unroll 1
        for (int q = 0; q < 4; ++q)  // tokens 4q + i of each block: lane group q holds their weights
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int tk = 16 * nb + 4 * q + i;
              const T* z = reinterpret_cast<const T*>(zt + tk * L::ZLD);
#pragma unroll
              for (int k = 0; k < RT; ++k) {
                const float pv = __shfl(s[k][nb][i], 16 * q + l16, kWave);
                if (t0 + tk < lim[k])
#pragma unroll
                  for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int x = 0; x < 4; ++x) acc[k][mb][x] += pv * tof(z[16 * mb + 4 * g4 + x]);
              }
            }
      }
      wave_lds_order();
    }
    bool bad = false;
#pragma unroll
    for (int k = 0; k < RT; ++k)
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int x = 0; x < 4; ++x) bad |= !__builtin_isfinite(acc[k][mb][x]);
    if (!__any(bad)) break;
  }

  // the four waves' sums, in the order of the waves
#pragma unroll
  for (int k = 0; k < RT; ++k) {
    l[k] = add_xor32(add_xor16(l[k]));
    if (g4 == 0) {
      s_m[w][16 * k + l16] = m[k];
      s_l[w][16 * k + l16] = l[k];
    }
  }
  float* red = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int k = 0; k < RT; ++k) {
    __syncthreads();
    const int rr = 16 * k + l16;
    const float M = fmaxf(fmaxf(s_m[0][rr], s_m[1][rr]), fmaxf(s_m[2][rr], s_m[3][rr]));
    const float f = weight_of(m[k], M);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
      *reinterpret_cast<f32x4*>(red + (w * 16 + l16) * RLD + 16 * mb + 4 * g4) = acc[k][mb] * f;
    __syncthreads();
    for (int u = tid; u < 16 * DH / 4; u += 256) {
      const int row = u / (DH / 4), d = u % (DH / 4) * 4, r = (rtile * RT + k) * 16 + row;
      if (r >= p.R) continue;
      f32x4 a = *reinterpret_cast<const f32x4*>(red + row * RLD + d);
#pragma unroll
      for (int v = 1; v < 4; ++v) a += *reinterpret_cast<const f32x4*>(red + (v * 16 + row) * RLD + d);
      const int64_t at = ((static_cast<int64_t>(b) * c.H + h) * p.R + r) * p.n_split + sp;
      *reinterpret_cast<f32x4*>(p.part + at * DH + d) = a;
      if (d == 0) {
        const int rw = 16 * k + row;
        const float M2 = fmaxf(fmaxf(s_m[0][rw], s_m[1][rw]), fmaxf(s_m[2][rw], s_m[3][rw]));
        float sum = 0.f;
        for (int v = 0; v < 4; ++v) sum += s_l[v][rw] * weight_of(s_m[v][rw], M2);
        p.stat[2 * at] = M2;
        p.stat[2 * at + 1] = sum;
      }
    }
  }
}

// The splits of one query head's row added, normalised and rotated back.
template <class T, int DH>
__global__ __launch_bounds__(DH) void k_join(DecodeParams p) {
  __shared__ float u[DH];
  const PagedCache& c = p.c;
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;  // [b][h][r]
  const int r = static_cast<int>(row % p.R), h = static_cast<int>(row / p.R % c.H);
  const int b = static_cast<int>(row / p.R / c.H);
  const int64_t cap = static_cast<int64_t>(p.max_pages) << c.shift;
  const int len = static_cast<int>(min(static_cast<int64_t>(min(max(p.lens[b], 0), p.max_len)), cap));
  const int ns = (len + p.chunk - 1) / p.chunk;
  const float* st = p.stat + 2 * row * p.n_split;
  float M = -__builtin_inff(), sum = 0.f, x = 0.f;
  for (int i = 0; i < ns; ++i) M = fmaxf(M, st[2 * i]);
  for (int i = 0; i < ns; ++i) {
    const float f = weight_of(st[2 * i], M);
    sum += f * st[2 * i + 1];
    x += f * p.part[(row * p.n_split + i) * DH + tid];
  }
  x = sum == 0.f ? 0.f : x / sum;
  if (p.lse && tid == 0) p.lse[row] = sum == 0.f ? -__builtin_inff() : M + __log2f(sum);
  if (p.Rm) {
    u[tid] = x;
    __syncthreads();
    const T* R = static_cast<const T*>(p.Rm) + (static_cast<int64_t>(h) * DH + tid) * DH;
    x = 0.f;
    for (int j = 0; j < DH; ++j) x += tof(R[j]) * u[j];
  }
  const int64_t o = ((static_cast<int64_t>(b) * p.Tq + r / p.rep) * p.Hq + h * p.rep + r % p.rep) * DH + tid;
  if (p.out_f32)
    static_cast<float*>(p.out)[o] = x;
  else
    static_cast<T*>(p.out)[o] = fromf<T>(x);
}

// mass_out[b,t] = decay mass_in[b,t] + the token's weight in every row.
__global__ __launch_bounds__(256) void k_mass(DecodeParams p, int nblk) {
  const PagedCache& c = p.c;
  const int b = blockIdx.x / nblk, t = blockIdx.x % nblk * 256 + threadIdx.x;
  const int64_t cap = static_cast<int64_t>(p.max_pages) << c.shift;
  const int len = static_cast<int>(min(static_cast<int64_t>(min(max(p.lens[b], 0), p.max_len)), cap));
  if (t >= len) return;
  float sum = 0.f;
  for (int64_t hr = 0; hr < static_cast<int64_t>(c.H) * p.R; ++hr) {
    const int64_t row = static_cast<int64_t>(b) * c.H * p.R + hr;
    const int lim = p.visible ? p.visible[static_cast<int64_t>(b) * p.Tq + hr % p.R / p.rep] : len;
    const float lse = p.lse[row];
    if (t < lim && lse != -__builtin_inff()) sum += exp2_(p.x[row * p.x_ld + t] - lse);
  }
  const int64_t at = static_cast<int64_t>(b) * p.mass_ld + t;
  p.mass_out[at] = p.mass_in ? p.decay * p.mass_in[at] + sum : sum;
}

template <class T, int DH, int RT>
void go(const DecodeParams& p, dim3 grid, hipStream_t s) {
  const int sub = p.c.ds >= Tile<T, DH>::EP ? 1 : Tile<T, DH>::EP / p.c.ds;
  auto kern = sub == 1 ? k_decode<T, DH, RT, 1> : k_decode<T, DH, RT, 2>;
  if constexpr (sizeof(T) == 2) {
    if (sub == 4) kern = k_decode<T, DH, RT, 4>;
  }
  hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, p);
}

int row_blocks(int R) { return R <= 16 ? 1 : R <= 32 ? 2 : 4; }  // blocks of 16 rows a workgroup takes

template <class T, int DH>
hipError_t launch(const DecodeParams& p, hipStream_t s) {
  const int RT = row_blocks(p.R), nrt = (p.R + 16 * RT - 1) / (16 * RT);
  const dim3 grid(static_cast<unsigned>(nrt) * p.n_split * p.c.H * p.B);
  if (p.n_split > 0) {
    if (RT == 1)
      go<T, DH, 1>(p, grid, s);
    else if (RT == 2)
      go<T, DH, 2>(p, grid, s);
    else
      go<T, DH, 4>(p, grid, s);
  }
  hipLaunchKernelGGL((k_join<T, DH>), dim3(static_cast<unsigned>(p.B) * p.c.H * p.R), dim3(DH), 0, s, p);
  if (p.mass_out && p.max_len > 0) {
    const int nblk = (p.max_len + 255) / 256;
    hipLaunchKernelGGL(k_mass, dim3(static_cast<unsigned>(p.B) * nblk), dim3(256), 0, s, p, nblk);
  }
  return hipGetLastError();
}

constexpr int64_t kSplitWgs = 2048;  // workgroups that the splits are made for

size_t up256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

}  // namespace

DecodePlan decode_plan(int B, int H, int R, int dh, int max_len, bool mass) {
  DecodePlan d;
  const int RT = row_blocks(R), nrt = (R + 16 * RT - 1) / (16 * RT);
  const int64_t units = (static_cast<int64_t>(max_len) + 127) / 128;  // of 128 tokens, a tile for each of four waves
  const int64_t wgs = static_cast<int64_t>(B) * H * nrt;
  const int64_t per = std::max<int64_t>(1, (units * wgs + kSplitWgs - 1) / kSplitWgs);
  d.chunk = static_cast<int>(128 * std::max<int64_t>(1, std::min(per, units)));
  d.n_split = static_cast<int>((static_cast<int64_t>(max_len) + d.chunk - 1) / d.chunk);
  d.x_ld = (max_len + 3) / 4 * 4;
  const size_t rows = static_cast<size_t>(B) * H * R, cells = rows * d.n_split;
  d.off_stat = up256(cells * dh * 4);
  d.off_x = d.off_stat + up256(cells * 8);
  d.off_lse = d.off_x + (mass ? up256(rows * d.x_ld * 4) : 0);
  d.bytes = d.off_lse + (mass ? up256(rows * 4) : 0);
  // what to ask a caller for: a bound on the above that does not fall as B, Tq or
  // max_len grows (n_split <= kSplitWgs / wgs + 1 and R <= 64 nrt)
  const size_t most = std::min(rows * static_cast<size_t>(units),
                               std::min<size_t>(R, 64) * static_cast<size_t>(kSplitWgs) + rows);
  d.ask = up256(most * dh * 4) + up256(most * 8) + (mass ? up256(rows * d.x_ld * 4) + up256(rows * 4) : 0);
  return d;
}

hipError_t launch_decode(const DecodeParams& p, bool bf16, hipStream_t s) {
  if (bf16) return p.c.dh == 128 ? launch<__bf16, 128>(p, s) : launch<__bf16, 64>(p, s);
  return p.c.dh == 128 ? launch<float, 128>(p, s) : launch<float, 64>(p, s);
}

}  // namespace rolesub
