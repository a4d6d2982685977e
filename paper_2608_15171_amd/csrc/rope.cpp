// Host side of the rotary positions: argument checks and the frequency table.
#include "rope.h"

#include <algorithm>
#include <cmath>
#include <cstring>

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

double rope_frequency(const ppas_rope& r, int32_t j) {
  const double R = r.rotary_dim;
  double base = r.theta;
  if (r.scaling == PPAS_ROPE_BASE && r.rotary_dim > 2) base *= std::pow(r.factor, R / (R - 2));
  const double w = std::pow(base, -2.0 * j / R);
  switch (r.scaling) {
    case PPAS_ROPE_LINEAR: return w / r.factor;
    case PPAS_ROPE_BANDS: {
      const double turns = r.original_len * w / (2.0 * M_PI);   // over the original length
      const double keep = std::min(1.0, std::max(0.0, (turns - r.low) / (r.high - r.low)));
      return w * (keep + (1.0 - keep) / r.factor);
    }
    case PPAS_ROPE_RAMP: {
      // the pair that makes b turns over the original length
      auto pair_of = [&](double b) { return R * std::log(r.original_len / (2.0 * M_PI * b)) / (2.0 * std::log(r.theta)); };
      const double first = std::max(std::floor(pair_of(r.high)), 0.0), last = std::min(std::ceil(pair_of(r.low)), R - 1);
      const double t = j <= first ? 0.0 : j >= last ? 1.0 : (j - first) / (last - first);
      return w * (1.0 - t + t / r.factor);
    }
    default: return w;
  }
}

ppas_status rope_table(const ppas_rope* rope, int32_t head_dim, const RopeTable** table) {
  static_assert(sizeof(ppas_rope) == 4 * sizeof(int32_t) + 5 * sizeof(double), "compared byte by byte: no padding");
  thread_local ppas_rope last{};   // rotary_dim 0: none
  thread_local RopeTable kept;
  if (!rope || rope->rotary_dim > head_dim) return PPAS_EINVAL;
  if (std::memcmp(&last, rope, sizeof(last)) != 0 || last.rotary_dim == 0) {
    const ppas_rope r = *rope;
    const ppas_status st = check_rope(r);
    if (st != PPAS_OK) return st;
    last = ppas_rope{};
    kept.layout = r.layout;
    kept.pairs = r.rotary_dim / 2;
    kept.magnitude = r.magnitude == 0 ? 1.f : float(r.magnitude);
    for (int32_t j = 0; j < kept.pairs; ++j) {
      const double w = rope_frequency(r, j);
      // every pair has to turn (a base or factor at the ends of fp64's range can leave it)
      if (!positive(w)) return PPAS_EINVAL;
      kept.turns[j] = w / (2.0 * M_PI);
    }
    last = r;
  }
  if (table) *table = &kept;
  return PPAS_OK;
}

}  // namespace ppas
