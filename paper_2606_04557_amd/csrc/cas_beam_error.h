// How exact the sums of beam search's selection are.
#pragma once

namespace cas {

// Up to here the scan's terms are one multiply-add and an exponential, beyond they have another form (cas_beam_step.hip).
constexpr float kFarLogit = 64.0f;

// How far ln sum exp(x - most) may be off by what the scan rounds; most is the
// largest logit, lowest the lowest ref that terms which count were made with.
// With d = x - ref, relative to itself and in units of 2^-24 a term is off
//   near (|ref| <= kFarLogit):  by its argument's rounding, |d|, and by that of log2 e, 0.23 |x|;
//   far:                        by two roundings of the argument, 2 |d|, and by that of log2 e, 0.23 |d|;
// and by the exponential's unit (2) and eleven additions at most. |d| is most - x at most, and above 0 most - lowest and
// 16 at most. |x| is |most| more than most - x at most, and 64 more than |d| where a near form was taken. Weighted by the terms' share of the
// sum, most - x is ln V - ln sum at most (the entropy of V tokens is at most ln V). All refs lie between lowest and most:
// where these are on both sides of a border, either form may have been taken. For V up to 2^30 all in all under 6e-6.
constexpr double sum_error(double ln_vocab, double ln_sum, double lowest, double most) {
  const double above = most - lowest > 16.0 ? 16.0 : most > lowest ? most - lowest : 0.0;
  const double d = ln_vocab - ln_sum + above, size = most < 0.0 ? -most : most;
  const double near = 1.25 * d + 0.25 * (size < 80.0 ? size : 80.0), far = 2.25 * d;
  const bool only_near = lowest >= -kFarLogit && most <= kFarLogit;
  return ((only_near || near > far ? near : far) + 13.0) * 0x1p-24;
}

}  // namespace cas
