// Angles of the rotary embedding, shared by the kernels that rotate.
#pragma once

#include <cuda_runtime.h>
#include <math.h>

#include "../../include/hpd.h"

namespace hpd {

struct InvFreq { double f[64]; };                    // theta^(-2i/D), i < D/2 <= 64

// Angles reach thousands of radians, where an fp32 product pos * inv_freq already loses ~1e-4 rad: the product and its
// reduction to [-pi, pi] are taken in fp64 (2*pi split in two doubles), and only the reduced angle goes through the fp32 sine and cosine.
__device__ __forceinline__ void rotary_angle(int pos, double inv_freq, float& cosine, float& sine)
{
    const double ang = static_cast<double>(pos) * inv_freq;
    const double k = rint(ang * 0.15915494309189535);                       // turns
    double r = fma(-k, 6.283185307179586, ang);                             // minus k * 2*pi (high part, then the rest)
    r = fma(-k, 2.4492935982947064e-16, r);
    sincosf(static_cast<float>(r), &sine, &cosine);
}

// Each thread keeps the table of its last (theta, D): a model asks for the same one layer after layer, and 64 powers take 3 us.
inline const InvFreq& inv_freq_table(const hpd_geom& g)
{
    static thread_local InvFreq t;
    static thread_local float theta = -1.f;
    static thread_local int dim = 0;
    if (g.rope_theta != theta || g.D != dim) {
        for (int i = 0; i < g.D / 2; ++i) t.f[i] = pow(static_cast<double>(g.rope_theta), -2.0 * i / static_cast<double>(g.D));
        theta = g.rope_theta; dim = g.D;
    }
    return t;
}

}  // namespace hpd
