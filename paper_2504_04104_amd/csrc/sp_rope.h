// Rotary positions: the frequencies of the pairs, and what a rotation is to the kernels.  Host part in plain C++.
//
//   pair t of a head's first `dims` columns, (t, t + dims / 2) in halves or (2t, 2t + 1) interleaved, at position p:
//   (a, b) -> gain * (a cos - b sin, b cos + a sin) at the angle p * freq[t]; the other columns pass.
#pragma once
#include <cmath>
#include <stdint.h>

#define SP_ROPE_PAIRS 64          // of a stage's heads (d_head up to 128, latent part up to 128)

// A stage's rotation, by value.  on 0: the config's, theta^(-2t / d) over whole heads in halves.
struct StageRope {
  double freq[SP_ROPE_PAIRS];
  float gain;
  int on;
  int dims;
  int layout;                      // 0 halves, 1 interleaved
};

// freq[t], t < dims / 2, of theta^(-2t / dims) scaled for contexts `factor` times as long as the `original` ones:
//   1 linear: all of them divided by factor
//   2 bands:  by the turns that a pair makes within the original context: as they are from `second` turns on, divided by factor up
//             to `first` turns, blended linearly in the turns in between
//   3 ramp:   by the pair's number: as they are up to the one that makes `first` turns, divided by factor from the one that makes
//             `second` turns on (first > second), blended linearly in the number in between
inline void rope_frequencies(int dims, double theta, int scaling, double factor, double original, double first, double second, double* freq) {
  const double two_pi = 6.283185307179586476925286766559;
  double lo = 0., hi = 1.;
  if (scaling == 3) {
    auto pair_of = [&](double turns) { return dims * std::log(original / (turns * two_pi)) / (2. * std::log(theta)); };
    lo = std::floor(pair_of(first));
    hi = std::ceil(pair_of(second));
    if (lo < 0.) lo = 0.;
    if (hi > dims - 1.) hi = dims - 1.;
    if (hi - lo < 0.001) hi = lo + 0.001;
  }
  for (int t = 0; t < dims / 2; ++t) {
    const double f = std::pow(theta, -2. * t / dims);
    double keep = 1.;               // share of the frequency as it is
    if (scaling == 1) keep = 0.;
    if (scaling == 2) keep = (original * f / two_pi - first) / (second - first);
    if (scaling == 3) keep = 1. - (t - lo) / (hi - lo);
    keep = keep < 0. ? 0. : keep > 1. ? 1. : keep;
    freq[t] = scaling == 0 ? f : keep * f + (1. - keep) * f / factor;
  }
}
