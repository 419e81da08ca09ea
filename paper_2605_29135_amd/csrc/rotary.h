// rotary.h -- the rotation of heads by their position, shared by the attention blocks.
#pragma once

#include <hip/hip_runtime.h>

namespace moe {
namespace dev {

// Rotation of dimension pair (i, i + d/2) at position p: angle p * theta^(-2i/d).  The angle is formed and
// reduced to [-pi, pi] in double, so thousands of positions keep full single precision in cos and sin.
__device__ __forceinline__ void rope_cs(int p, int i, int d, float theta, float &c, float &s) {
    const double inv_freq = exp2(-2.0 * double(i) / double(d) * log2(double(theta)));
    const double ang = double(p) * inv_freq;
    constexpr double kTwoPi = 6.283185307179586;
    const double r = fma(-rint(ang * (1.0 / kTwoPi)), kTwoPi, ang);
    double sd, cd;
    sincos(r, &sd, &cd);
    c = float(cd);
    s = float(sd);
}

}  // namespace dev
}  // namespace moe
