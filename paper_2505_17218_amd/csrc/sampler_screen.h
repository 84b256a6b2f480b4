// Screening of the Gumbel-max samplers (gfx950): bounds on an entry's exact score that need no
// exact noise.  Shared by the full-vocabulary sampler and the truncated one, which draw with the
// same noise.  Built with -ffp-contract=off, as sampler_math.h.
#pragma once

#include "common.h"
#include "sampler_math.h"

namespace dash {

// bound on |cheap noise - exact noise|: 8x the exhaustive maximum (1.9e-6) on gfx950
constexpr float kScreenTol = 1.6e-5f;

DASH_DEV bool better(float s, int i, float bs, int bi) { return s > bs || (s == bs && i < bi); }

// -ln(-ln u) with the hardware logarithm; u = ((x >> 8) | 1) 2^-24 as in gumbel_from_bits
DASH_DEV float cheap_gumbel(uint32_t x) {
    const float u = (float)((x >> 8) | 1u) * (1.0f / 16777216.0f);
    return -__logf(-__logf(u));
}

// Interval half-width around a cheap score sa that contains the exact score.
DASH_DEV float screen_margin(float sa) { return kScreenTol + fabsf(sa) * (1.0f / 1048576.0f); }

// Upper bound on the exact noise of the random word x, from its leading ones alone:
// k leading ones leave u < 1 - 2^-(k+1), and -ln(1 - e) >= e gives
// g = -ln(-ln u) < -ln(2^-(k+1)) = (k+1) ln 2 (0.6931472f is above ln 2; at most 25
// terms, so the product's rounding stays far inside the margin added by the caller).
DASH_DEV float noise_bound(uint32_t x) { return (float)(min(__clz(~x), 24) + 1) * 0.6931472f; }

// Maximum over the wave's 64 lanes, returned wave-uniform: data-parallel-primitive moves
// within each row of 16 lanes (quad swaps, then the half-row and row mirrors), row
// broadcasts up to lane 63, then that lane read into a scalar register.  Every step is a
// register move inside the vector unit; exchanges through LDS (one per xor distance)
// each waited for the LDS round trip.
DASH_DEV float wave_max_f(float v) {
    int x = __float_as_int(v);
    x = __float_as_int(fmaxf(__int_as_float(x), __int_as_float(__builtin_amdgcn_update_dpp(x, x, 0xB1, 0xF, 0xF, false))));
    x = __float_as_int(fmaxf(__int_as_float(x), __int_as_float(__builtin_amdgcn_update_dpp(x, x, 0x4E, 0xF, 0xF, false))));
    x = __float_as_int(fmaxf(__int_as_float(x), __int_as_float(__builtin_amdgcn_update_dpp(x, x, 0x141, 0xF, 0xF, false))));
    x = __float_as_int(fmaxf(__int_as_float(x), __int_as_float(__builtin_amdgcn_update_dpp(x, x, 0x140, 0xF, 0xF, false))));
    // row_bcast15 into rows 1 and 3, row_bcast31 into rows 2 and 3 (rows not in the mask keep x)
    x = __float_as_int(fmaxf(__int_as_float(x), __int_as_float(__builtin_amdgcn_update_dpp(x, x, 0x142, 0xA, 0xF, false))));
    x = __float_as_int(fmaxf(__int_as_float(x), __int_as_float(__builtin_amdgcn_update_dpp(x, x, 0x143, 0xC, 0xF, false))));
    return __int_as_float(__builtin_amdgcn_readlane(x, 63));
}

}  // namespace dash
