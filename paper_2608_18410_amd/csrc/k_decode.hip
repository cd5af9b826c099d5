// Attention over the tokens that rows see of the paged cache from its start: the kernels
// of decode.hpp, and how calls are split.
#include "decode.hpp"

namespace rolesub {
namespace {

// Workgroups that the splits are made for: two for each of the 256 CUs. More splits
// cost more to add up than they even out: 64 sequences of 256 to 2048 tokens and 8
// key heads take 60 us in one split each, 73 in two, 66 in four; 16 of 361 tokens
// and 56 queries 40 against 64. Short sequences in one split without the weights, whose
// adding takes the second launch anyway, would save that launch (one of 305 tokens, 32
// heads: 12.2 against 14.4 us), but a call's outputs would then depend on whether it
// adds up weights.
constexpr int64_t kSplitWgs = 512;
// The same for drafted tokens of up to 16 rows, whose tiles take longer (32 sequences of 256
// to 4096 tokens, 8 key heads of 16 rows: 107 us with 512, 101 with 1024, 113 with 1536), and
// of more, in blocks of kTreeRows: 8 of those sequences, of 96 rows, 60 us with 256, 53 with
// 512, 46 with 768 and 50 with 1024. Where the blocks fill the card without splits, two to a
// CU, splits only add: 32 of those sequences of 64 rows 73 us in one, 98 in two, of 96 rows
// 88 and 113, of 64 rows and up to 16384 tokens 217 and 258; nothing longer was measured, and
// all of this with two parts of a weight, where three take 3 % more.
constexpr int64_t kTreeWgs = 1024, kTreeRowsWgs = 768, kTreeFull = 512, kTreeWhole = 128;
// Up to 512 tokens these and listed pages, whose calls add up no weights, have one split
// where 16 rows or fewer share it: 8 drafted tokens over 305 and 32 heads 24.9 -> 22.2 us
// with the masks, 24 pages of 16 chosen of 176 35.7 -> 31.9 with the choice. From 60 rows on
// they are slower (25.2 -> 27.4), and so are 1024 listed tokens (35.6 -> 37.7).
constexpr int64_t kShortUnits = 4;
// Splits of more than 2048 tokens cost next to nothing to add up, and up to 2048
// workgroups of them even out a ragged batch: 34 sequences of 236 to 15420 tokens, 8 key
// heads of 4 rows 259 -> 183 us, 23 of 7727 to 22794 290 -> 215, 34 of 8192 192 -> 170. Not
// where one split each is had in order of length: 64 of 256 to 16384 302 -> 347.
constexpr int64_t kLongUnits = 16, kLongWgs = 2048;
constexpr int64_t kMaxSplits = 256;  // that k_join adds up

size_t up256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

}  // namespace

DecodePlan decode_plan(int B, int H, int R, int dh, int max_len, bool mass, DecodeKind kind) {
  DecodePlan d;
  const int64_t want = kind != DecodeKind::tree ? kSplitWgs : R > 16 ? kTreeRowsWgs : kTreeWgs;
  const int tile = kind == DecodeKind::tree ? kTreeRows : 64;  // rows of a workgroup, whatever row_blocks says
  const int nrt = (R + tile - 1) / tile;
  const int64_t units = (static_cast<int64_t>(max_len) + 127) / 128;  // of 128 tokens, a tile for each of four waves
  const int64_t wgs = static_cast<int64_t>(B) * H * nrt;
  const int64_t least = (units + kMaxSplits - 1) / kMaxSplits;
  int64_t per = std::max((units * wgs + want - 1) / want, least);
  if (per > kLongUnits && (per < units || wgs > kOrderWgs))
    per = std::max({kLongUnits, (units * wgs + kLongWgs - 1) / kLongWgs, least});
  if (kind == DecodeKind::tree && R > 16 && wgs >= kTreeFull && units <= kTreeWhole) per = units;
  if (kind != DecodeKind::paged && units <= kShortUnits && R <= 16) per = units;
  d.chunk = static_cast<int>(128 * std::max<int64_t>(1, std::min(per, units)));
  d.n_split = std::max(1, static_cast<int>((static_cast<int64_t>(max_len) + d.chunk - 1) / d.chunk));
  d.x_ld = (max_len + 3) / 4 * 4;
  const size_t rows = static_cast<size_t>(B) * H * R, cells = rows * d.n_split;
  d.off_stat = d.n_split > 1 ? up256(cells * dh * 4) : 0;
  d.off_x = d.off_stat + (d.n_split > 1 || (mass && max_len > 0) ? up256(cells * 8) : 0);
  d.bytes = d.off_x + (mass ? up256(rows * d.x_ld * 4) : 0);
  // what to ask a caller for: a bound on the above that does not fall as B, Tq or
  // max_len grows (n_split <= want / wgs + 1, or for splits of kLongUnits and more
  // kLongWgs / wgs + 1 and units / kLongUnits + 1; R <= tile * nrt)
  const size_t most_r = std::min(R, tile);
  size_t short_rows = most_r * want;  // n_split times rows, but for one a row
  if (kind == DecodeKind::tree && R > 16) short_rows = std::max(short_rows, static_cast<size_t>(16 * kTreeWgs));
  const size_t longs = std::min(most_r * kLongWgs, rows * static_cast<size_t>(units / kLongUnits)) + rows;
  const size_t most = std::min(rows * static_cast<size_t>(std::min(units, kMaxSplits)), std::max(short_rows + rows, longs));
  d.ask = up256(most * dh * 4) + up256(most * 8) + (mass ? up256(rows * d.x_ld * 4) : 0);
  return d;
}

hipError_t launch_decode(const DecodeParams& p, bool bf16, hipStream_t s) { return launch_any<kPrefix>(p, bf16, s); }

}  // namespace rolesub
