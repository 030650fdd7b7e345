// rotary_host.cpp -- the rotation's angles.  Host C++ only; no HIP calls.
#include "rotary_host.hpp"

#include <cmath>

namespace splat {

splat_status rotary_build(const splat_rotary_desc& d, const splat_rotary_axes* axes,
                          HostRotary& out, std::string& err) {
  auto bad = [&](const char* what) {
    err = what;
    return SPLAT_ERR_INVALID_ARG;
  };
  if (d.max_len < 1 || d.max_len > SPLAT_ROTARY_MAX_LEN)
    return bad("max_len must be in [1, SPLAT_ROTARY_MAX_LEN]");
  if (d.rot_dim < 16 || d.rot_dim > 128 || d.rot_dim % 16 != 0)
    return bad("rot_dim must be a multiple of 16 in [16, 128]");
  if (d.interleaved != 0 && d.interleaved != 1) return bad("interleaved must be 0 or 1");
  if (!(d.base > 1.0) || !std::isfinite(d.base)) return bad("base must be a finite number above 1");
  if (!(d.factor >= 1.0) || !std::isfinite(d.factor))
    return bad("factor must be a finite number of at least 1");
  if (!(d.magnitude > 0.0) || !std::isfinite(d.magnitude))
    return bad("magnitude must be a finite number above 0");
  const bool ramp = d.ramp_lo != 0.0 || d.ramp_hi != 0.0;
  if (ramp && !(d.ramp_lo >= 0.0 && d.ramp_hi > d.ramp_lo && std::isfinite(d.ramp_hi)))
    return bad("a ramp needs 0 <= ramp_lo < ramp_hi");
  if (ramp && d.original_len < 1) return bad("a ramp needs original_len >= 1");
  const int32_t n = d.rot_dim / 2;
  const splat_rotary_axes one{1, {n}, 0, 0};
  const splat_rotary_axes& x = axes ? *axes : one;
  if (x.n < 1 || x.n > SPLAT_ROTARY_MAX_AXES)
    return bad("axes must be in [1, SPLAT_ROTARY_MAX_AXES]");
  int64_t pairs = 0;
  for (int32_t a = 0; a < SPLAT_ROTARY_MAX_AXES; ++a) {
    if (a < x.n ? x.pairs[a] < 1 : x.pairs[a] != 0)
      return bad("each axis must have at least one pair, and no pairs stand past the last axis");
    pairs += x.pairs[a];
  }
  if (pairs != n) return bad("the axes' pairs must be rot_dim / 2 in all");
  if ((x.cyclic != 0 && x.cyclic != 1) || (x.restart != 0 && x.restart != 1))
    return bad("cyclic and restart must be 0 or 1");
  out.desc = d;
  out.axes = x.n;
  out.axis.clear();
  // whole axes in turn, or a pair of each
  int32_t used[SPLAT_ROTARY_MAX_AXES] = {0};
  std::vector<int32_t> number;     // of each pair among its axis's
  for (int32_t a = 0; (int32_t)out.axis.size() < n; a = (a + 1) % x.n)
    for (int32_t k = x.cyclic ? 1 : x.pairs[a]; k > 0 && used[a] < x.pairs[a]; --k) {
      out.axis.push_back((uint8_t)a);
      number.push_back(used[a]++);
    }
  out.frequency.resize(n);
  for (int32_t t = 0; t < n; ++t) {
    const double f = x.restart ? std::pow(d.base, -(double)number[t] / x.pairs[out.axis[t]])
                               : std::pow(d.base, -2.0 * t / d.rot_dim);
    double keep = 0.0;
    if (ramp) {
      const double turns = d.original_len * f / (2.0 * 3.14159265358979323846);
      keep = (turns - d.ramp_lo) / (d.ramp_hi - d.ramp_lo);
      keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
    }
    out.frequency[t] = f * keep + f / d.factor * (1.0 - keep);
  }
  return SPLAT_OK;
}

// Rounded once, from angles in 64 bits: in fp32 position 65536's angle would be
// off by 2^-9.
std::vector<float> rotary_table(const HostRotary& r) {
  std::vector<float> out(2 * (size_t)r.desc.max_len * r.frequency.size());
  float* p = out.data();
  for (int32_t i = 0; i < r.desc.max_len; ++i)
    for (double f : r.frequency) {
      *p++ = (float)(std::cos(i * f) * r.desc.magnitude);
      *p++ = (float)(std::sin(i * f) * r.desc.magnitude);
    }
  return out;
}

}  // namespace splat
