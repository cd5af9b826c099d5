// Queries and keys turned by their positions, with several position axes:
//   a_i = pos[axis(i)] * inv_freq[i],
//   y_i = x_i cos a_i - x_j sin a_i,  y_j = x_i sin a_i + x_j cos a_i.
#include "common.hpp"
#include "launch.hpp"

namespace rolesub {
namespace {

constexpr int kMaxPairs = 64;

// cos and sin of 2 pi times the product pos * f / (2 pi), reduced in 64 bits: the
// product of a 31-bit integer and a 24-bit float is exact to 2 ulp of a double,
// and the turns it makes are removed before anything is rounded to 32 bits.
__device__ __forceinline__ void angle(int32_t pos, float f, float& c, float& s) {
  double t = static_cast<double>(pos) * static_cast<double>(f) * 0.15915494309189533577;
  t -= __builtin_rint(t);
  const float x = static_cast<float>(t + t);  // half turns, in [-1, 1]
  sincospif(x, &s, &c);
}

// One workgroup turns the heads [blockIdx.y * hpb, ...) of one token: one thread
// per pair (and per dim past the pairs) and head.
template <class T>
__global__ __launch_bounds__(256) void k_rotary(RotaryParams p, int hpb) {
  __shared__ float cs[kMaxPairs], sn[kMaxPairs];
  const int64_t tok = blockIdx.x;
  const int tid = threadIdx.x, n = p.n_pairs;
  if (tid < n) {
    const int ax = p.axis ? p.axis[tid] : 0;
    float c = 1.f, s = 0.f;
    if (ax < p.n_axes) angle(p.positions[tok * p.n_axes + ax], p.inv_freq[tid], c, s);
    cs[tid] = c;
    sn[tid] = p.inverse ? -s : s;
  }
  __syncthreads();
  const int units = p.dh - n;  // pairs, then single dims
  const int h0 = blockIdx.y * hpb, h1 = min(h0 + hpb, p.H + p.Hkv);
  for (int i = tid; i < (h1 - h0) * units; i += 256) {
    const int h = h0 + i / units, u = i % units;
    const T* src;
    T* dst;
    if (h < p.H) {
      src = static_cast<const T*>(p.q) + tok * p.q_stride + static_cast<int64_t>(h) * p.dh;
      dst = static_cast<T*>(p.q_out) + tok * p.qo_stride + static_cast<int64_t>(h) * p.dh;
    } else {
      src = static_cast<const T*>(p.k) + tok * p.k_stride + static_cast<int64_t>(h - p.H) * p.dh;
      dst = static_cast<T*>(p.k_out) + tok * p.ko_stride + static_cast<int64_t>(h - p.H) * p.dh;
    }
    if (u >= n) {
      dst[n + u] = src[n + u];
      continue;
    }
    const int a = p.interleaved ? 2 * u : u, b = p.interleaved ? 2 * u + 1 : n + u;
    const float xa = tof(src[a]), xb = tof(src[b]), c = cs[u], s = sn[u];
    dst[a] = fromf<T>(xa * c - xb * s);
    dst[b] = fromf<T>(xa * s + xb * c);
  }
}

}  // namespace

hipError_t launch_rotary(const RotaryParams& p, bool bf16, hipStream_t s) {
  const int heads = p.H + p.Hkv, hpb = 16;
  const dim3 grid(static_cast<unsigned>(p.B) * p.T, (heads + hpb - 1) / hpb);
  if (bf16)
    hipLaunchKernelGGL(k_rotary<__bf16>, grid, dim3(256), 0, s, p, hpb);
  else
    hipLaunchKernelGGL(k_rotary<float>, grid, dim3(256), 0, s, p, hpb);
  return hipGetLastError();
}

}  // namespace rolesub
