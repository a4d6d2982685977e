// Host side of the rotary positions: argument checks and the frequency table.
#include "rope.h"

#include <algorithm>
#include <cmath>

namespace ppas {

namespace {

bool positive(double v) { return std::isfinite(v) && v > 0; }

}  // namespace

// The fields that do not depend on the head.
static ppas_status check_rope(const ppas_rope& r) {
  if (r.layout != PPAS_ROPE_HALF && r.layout != PPAS_ROPE_INTERLEAVED) return PPAS_EINVAL;
  if (r.rotary_dim < 2 || r.rotary_dim % 2 != 0 || r.rotary_dim > 2 * kRopeMaxPairs) return PPAS_EINVAL;
  if (!positive(r.theta)) return PPAS_EINVAL;
  if (!(r.magnitude == 0 || positive(r.magnitude)) || !std::isfinite(float(r.magnitude))) return PPAS_EINVAL;
  if (r.scaling < PPAS_ROPE_PLAIN || r.scaling > PPAS_ROPE_RAMP) return PPAS_EINVAL;
  if (r.scaling == PPAS_ROPE_PLAIN) return PPAS_OK;
  if (!positive(r.factor)) return PPAS_EINVAL;
  if (r.scaling == PPAS_ROPE_BANDS || r.scaling == PPAS_ROPE_RAMP) {
    if (r.original_len < 1 || !positive(r.low) || !positive(r.high) || !(r.low < r.high)) return PPAS_EINVAL;
    if (r.scaling == PPAS_ROPE_RAMP && !(r.theta > 1)) return PPAS_EINVAL;
  }
  return PPAS_OK;
}

// Radians per position of every pair, in 64 bits. Every call makes the table, so that its
// time counts: u_j = u_8k u_(j - 8k) takes 24 exponentials for 128 pairs (a power each took
// 3 us for 64). Their arguments, a few tens at most, are within 2^-52 of themselves, and
// the frequencies so within 1e-14.
static void frequencies(const ppas_rope& r, double* w) {
  const double R = r.rotary_dim;
  double base = r.theta;
  if (r.scaling == PPAS_ROPE_BASE && r.rotary_dim > 2) base *= std::pow(r.factor, R / (R - 2));
  const double ln = std::log(base);
  const int32_t pairs = r.rotary_dim / 2;
  double fine[8];
  for (int32_t j = 0; j < 8; ++j) fine[j] = std::exp(-2.0 * j / R * ln);
  for (int32_t j = 0; j < pairs; j += 8) {
    const double coarse = std::exp(-2.0 * j / R * ln);
    for (int32_t i = 0; i < std::min(8, pairs - j); ++i) w[j + i] = coarse * fine[i];
  }
  switch (r.scaling) {
    case PPAS_ROPE_LINEAR:
      for (int32_t j = 0; j < pairs; ++j) w[j] /= r.factor;
      break;
    case PPAS_ROPE_BANDS:
      for (int32_t j = 0; j < pairs; ++j) {
        const double turns = r.original_len * w[j] / (2.0 * M_PI);   // over the original length
        const double keep = std::min(1.0, std::max(0.0, (turns - r.low) / (r.high - r.low)));
        w[j] *= keep + (1.0 - keep) / r.factor;
      }
      break;
    case PPAS_ROPE_RAMP: {
      // the pair that makes b turns over the original length
      auto pair_of = [&](double b) { return R * std::log(r.original_len / (2.0 * M_PI * b)) / (2.0 * ln); };
      const double first = std::max(std::floor(pair_of(r.high)), 0.0), last = std::min(std::ceil(pair_of(r.low)), R - 1);
      for (int32_t j = 0; j < pairs; ++j) {
        const double t = j <= first ? 0.0 : j >= last ? 1.0 : (j - first) / (last - first);
        w[j] *= 1.0 - t + t / r.factor;
      }
      break;
    }
    default: break;
  }
}

ppas_status rope_frequencies(const ppas_rope* rope, int32_t head_dim, double* w) {
  if (!rope || rope->rotary_dim > head_dim) return PPAS_EINVAL;
  const ppas_status st = check_rope(*rope);
  if (st != PPAS_OK) return st;
  frequencies(*rope, w);
  // Every pair has to turn (a base or factor at the ends of fp64's range can leave it), and at most
  // 2^12 times per position: an angle at position 2^31 is then known to 2^-10 of a turn. Far beyond
  // it would be a whole number of turns, whatever the position, and then infinite.
  for (int32_t j = 0; j < rope->rotary_dim / 2; ++j)
    if (!positive(w[j]) || w[j] > 4096 * 2.0 * M_PI) return PPAS_EINVAL;
  return PPAS_OK;
}

ppas_status rope_table(const ppas_rope* rope, int32_t head_dim, RopeTable& t) {
  const ppas_status st = rope_frequencies(rope, head_dim, t.turns);
  if (st != PPAS_OK) return st;
  t.layout = rope->layout;
  t.pairs = rope->rotary_dim / 2;
  t.magnitude = rope->magnitude == 0 ? 1.f : float(rope->magnitude);
  for (int32_t j = 0; j < t.pairs; ++j) t.turns[j] *= 1 / (2.0 * M_PI);
  return PPAS_OK;
}

}  // namespace ppas
