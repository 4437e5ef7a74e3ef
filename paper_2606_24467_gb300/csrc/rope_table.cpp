// Rotary frequencies and the table that the kernels rotate by (host only).
//
// A frequency f (radians a position) is held as f / 2 pi turns modulo one, in
// units of 2^-64: the product with a 32-bit position, modulo 2^64, is then the
// angle with no rounding but that of the table, 2^-64 of a turn and |f| 2^-55 (the
// quotient is a double) a position.
#include <cmath>
#include <cstdint>
#include <cstring>

#include "compresskv.h"

namespace {

constexpr double kTwoPi = 6.283185307179586476925286766559;
constexpr int kMaxPairs = 64;

bool rot_dim_ok(int32_t d) { return d >= 2 && d <= 2 * kMaxPairs && d % 2 == 0; }

double clip01(double x) { return x < 0.0 ? 0.0 : x > 1.0 ? 1.0 : x; }

}  // namespace

extern "C" {

int compresskv_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor,
                                double original_length, double low, double high, double* frequencies) {
  if (!frequencies || !rot_dim_ok(rot_dim)) return CKV_ERR_INVALID_ARG;
  if (scaling < CKV_ROPE_PLAIN || scaling > CKV_ROPE_RAMP) return CKV_ERR_INVALID_ARG;
  if (!(base > 0.0) || std::isinf(base)) return CKV_ERR_INVALID_ARG;
  const int pairs = rot_dim / 2;
  if (scaling != CKV_ROPE_PLAIN && (!(factor >= 1.0) || std::isinf(factor))) return CKV_ERR_INVALID_ARG;
  if (scaling == CKV_ROPE_BASE) {
    if (rot_dim == 2) return CKV_ERR_INVALID_ARG;
    base *= std::pow(factor, static_cast<double>(rot_dim) / (rot_dim - 2));
    if (std::isinf(base)) return CKV_ERR_INVALID_ARG;
  }
  const bool by_turns = scaling == CKV_ROPE_WAVES || scaling == CKV_ROPE_RAMP;
  if (by_turns && (!(original_length > 0.0) || std::isinf(original_length) || !(low > 0.0) ||
                   !(high > low) || std::isinf(high)))
    return CKV_ERR_INVALID_ARG;
  // RAMP: the pair whose wave makes t turns over the original length, i with
  // original_length base^(-2i / rot_dim) = 2 pi t
  double first = 0.0, last = 0.0;
  if (scaling == CKV_ROPE_RAMP) {
    if (!(base > 1.0)) return CKV_ERR_INVALID_ARG;
    const double per = rot_dim / (2.0 * std::log(base));
    first = std::fmax(std::floor(per * std::log(original_length / (kTwoPi * high))), 0.0);
    // (at most the last channel's number, not the last pair's: a pair of fewer turns
    // than `low` need not exist)
    last = std::fmin(std::ceil(per * std::log(original_length / (kTwoPi * low))), rot_dim - 1.0);
    if (!(last > first)) last = first + 1e-3;  // one step
  }
  for (int i = 0; i < pairs; ++i) {
    const double f = std::pow(base, -2.0 * i / rot_dim);
    double keep = 1.0;
    if (scaling == CKV_ROPE_LINEAR) keep = 0.0;
    if (scaling == CKV_ROPE_WAVES) keep = clip01((original_length * f / kTwoPi - low) / (high - low));
    if (scaling == CKV_ROPE_RAMP) keep = 1.0 - clip01((i - first) / (last - first));
    if (scaling == CKV_ROPE_PLAIN || scaling == CKV_ROPE_BASE)
      frequencies[i] = f;
    else
      frequencies[i] = f * keep + f / factor * (1.0 - keep);
  }
  return CKV_OK;
}

int compresskv_rope_init(ckv_rope* r, int32_t rot_dim, int32_t interleaved, const double* frequencies,
                         double scale) {
  if (!r || !frequencies || !rot_dim_ok(rot_dim)) return CKV_ERR_INVALID_ARG;
  const float s = static_cast<float>(scale);
  if (!std::isfinite(s)) return CKV_ERR_INVALID_ARG;
  for (int i = 0; i < rot_dim / 2; ++i)
    if (!(std::fabs(frequencies[i]) <= 1048576.0)) return CKV_ERR_INVALID_ARG;
  std::memset(r, 0, sizeof(*r));
  r->rot_dim = rot_dim;
  r->interleaved = interleaved != 0;
  r->scale = s;
  for (int i = 0; i < rot_dim / 2; ++i) {
    // (negated as an integer: one minus a small part keeps fewer of its bits)
    const double t = std::fabs(frequencies[i]) / kTwoPi;
    const uint64_t part = static_cast<uint64_t>(std::ldexp(t - std::floor(t), 64));
    r->turns[i] = frequencies[i] < 0.0 ? 0 - part : part;
  }
  return CKV_OK;
}

}  // extern "C"
