// rotary_host.hpp -- the position rotation's angles (no HIP).
#pragma once

#include <string>
#include <vector>

#include "../../include/splat.h"

namespace splat {

struct HostRotary {
  splat_rotary_desc desc;
  std::vector<double> frequency;   // rot_dim / 2: angle per position of each pair
};

splat_status rotary_build(const splat_rotary_desc& desc, HostRotary& out, std::string& err);

// max_len x rot_dim / 2 x (cosine, sine), times magnitude
std::vector<float> rotary_table(const HostRotary& r);

}  // namespace splat
