// rotary_host.hpp -- the position rotation's angles (no HIP).
#pragma once

#include <string>
#include <vector>

#include "../../include/splat.h"

namespace splat {

struct HostRotary {
  splat_rotary_desc desc;
  int32_t axes;                    // 1: every pair turns by the one position
  std::vector<uint8_t> axis;       // rot_dim / 2: each pair's
  std::vector<double> frequency;   // rot_dim / 2: angle per position of each pair
};

// axes: may be null
splat_status rotary_build(const splat_rotary_desc& desc, const splat_rotary_axes* axes,
                          HostRotary& out, std::string& err);

// max_len x rot_dim / 2 x (cosine, sine), times magnitude
std::vector<float> rotary_table(const HostRotary& r);

}  // namespace splat
