// Angles of pairs of dims turned by positions, for the kernels that turn them.
#pragma once
#include "common.hpp"

namespace rolesub {
namespace {

constexpr int kMaxPairs = 64;
constexpr float kStays = 2.f;  // in a cosine's place: no axis turns the pair

// cos and sin of pos * f. The product of a 31-bit integer and a 24-bit float and its
// share of a turn are held in two doubles each, and whole turns are taken off both before
// anything is rounded to 32 bits. Two doubles hold a turn to 2^-105 of it, so the angle
// is right to its 32-bit rounding while |pos * f| stays below 2^75. Nothing may be fused
// here but what says so: t - rint(t) from the unrounded product would count te twice.
__device__ __forceinline__ void angle(int32_t pos, float f, float& c, float& s) {
#pragma clang fp contract(off)
  constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnLo = -0x1.6b01ec5417056p-57;  // 1 / (2 pi)
  const double x = pos, y = f, p = x * y, pe = __builtin_fma(x, y, -p);
  const double t = p * kTurn, te = __builtin_fma(p, kTurn, -t) + __builtin_fma(p, kTurnLo, pe * kTurn);
  const double r = (t - __builtin_rint(t)) + (te - __builtin_rint(te));
  sincospif(static_cast<float>(r + r), &s, &c);  // half turns, in [-1, 1]
}

}  // namespace
}  // namespace rolesub
