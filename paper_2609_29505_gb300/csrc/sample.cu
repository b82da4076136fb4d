// A token drawn from each row of logits: temperature, top-k, min-p and top-p, from two given random numbers.
//
// With x = scale z, w_i = e^(x_i - max x), and the tokens in the order (z descending, index ascending):
//   K1 = the first top_k of the order that have w_i >= min_p;  K = the shortest prefix of K1 with a mass (sum of w)
//   of at least top_p times K1's.
// The vocabulary is cut into blocks of 512 tokens.  The first block whose cumulative mass (of K alone) is above
// u0 mass(K) is drawn, then the first token in it whose cumulative mass is above u1 mass(block).
//
// Why two steps: one fp32 number has 24 bits, too few for a tail of 126464 tokens.  And why blocks: a border between tokens
// moves with every rounding of the sum before it, so that a draw among 1e5 tokens by fp32 sums is another token than by exact
// ones once in a hundred rows.  A block's border is met with 500 times less often, so that fp32 sums do unless the number
// falls within their error of a border, which is seen, and the masses are taken anew; inside a block, and where a cut is
// looked for, masses are whole numbers (weight() below): their sums have no error and no order.
//
// A row is read once from HBM, by tiles of 16 KB that bulk copies bring into a ring of three: warps take blocks and leave their maxima
// and, where masses are needed, their sums of exponentials against the maximum (kError below).  What comes after looks, from L2, only
// at blocks whose maximum reaches a bound zl that the cut is not below:
//   top-k: the k-th largest of the blocks' maxima, for large k a quantile of a sample of the row;  min-p: max + ln(min_p) / scale;
//   top-p alone: the 64th largest of the maxima where the maxima above it already have the mass; else from the sample (one token of 8
//   in a histogram of its weights), which also gives a bound zh that the cut is not above.
// What lies between the bounds is listed.  For top-p alone the tail below zl is summed in fp32 as well: what is not kept has the share
// 1 - top_p at most, so that the cut depends on the tail's error and, by 1 - top_p, on the row's; where it does (one row in twenty of a
// broad distribution) both masses are taken anew.  The blocks' masses lose the tail and what of the list is not kept.  If the cut
// is not between the bounds after all, which counts and sums tell, the whole row is searched.
// The cut is found in the list, or the row, by histograms of counts and masses over the order's integers, 1024 bins at a time,
// down to 256 tokens, which are ranked by comparing all with all.
//
// Many rows: a CTA of 256 threads each (64 or 128 for short rows), three or four per SM, so that one's search hides
// behind the others' reading.  Few: a cluster reads a row, and takes the bracket between the bounds together.
//
// Measured (GB300, replayed from a graph; a copy moves 6.7 TB/s): every token of 2048 of 4096 x 126464 fp16 93 us = 5.6 TB/s (over other
// buffers of the same size up to 156, where a copy and the scoring kernel take as long as everywhere: not known why), of 1024 x
// 126464 fp32 81 us = 6.4: HBM, and for 16-bit logits the issue slots (60% busy) and exponentials (73% of their rate).  A persistent
// form with 16 streaming warps per SM and finishing warps was slower everywhere (96 and 83 us; 1500 x 126464 147 against 135).
// 1003 x 32003 fp32 with every filter 46 us: a row is 18 thousand clocks of reading and 15 of steps one after another.
// 1024 x 126464 bf16, top-p 0.9 of a broad distribution (2900 tokens): 336 us: 200 thousand clocks a row, half of them the
// bracket (300 instructions a block), in 2.25 rounds of 456 rows; two or four CTAs per SM instead of three: 347 and 336 us.
// One row of 126464: 5.8 us, with top-p 17 to 30, latency; 634 where tens of thousands of tokens are kept, which the row is searched for.
#include <math.h>

#include "sample.cuh"

namespace sgd {
namespace {

using namespace rows;

template <typename T>
cudaError_t rows_of_type(const SampleArgs& a, cudaStream_t s) {
  const SampleParams& p = a.p;
  const bool filter = (p.top_k > 0 && p.top_k < p.vocab) || p.min_p > 0.0 || p.top_p < 1.0;
  return filter ? sample_rows<T, true>(a, s) : sample_rows<T, false>(a, s);
}

}  // namespace

cudaError_t sample_launch(const SampleParams& p, cudaStream_t s) {
  const float f = p.scale < 0x1p-64f ? 0x1p-64f : 1.f, scale = p.scale / f;
  const double c = static_cast<double>(scale) * 1.4426950408889634073599;
  SampleArgs a{p, f, static_cast<float>(c), 0.f, scale, p.min_p > 0.0 ? log(p.min_p) / static_cast<double>(p.scale) : -HUGE_VAL,
               (p.vocab + SGD_SAMPLE_BLOCK - 1) / SGD_SAMPLE_BLOCK, device_status_ptr()};
  a.c_lo = static_cast<float>(c - static_cast<double>(a.c));
  if (p.dtype == SGD_F16) return rows_of_type<f16>(a, s);
  if (p.dtype == SGD_BF16) return rows_of_type<bf16>(a, s);
  return rows_of_type<float>(a, s);
}

}  // namespace sgd
