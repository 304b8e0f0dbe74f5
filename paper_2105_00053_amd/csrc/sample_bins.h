// The draw's first bins of floats: what is counted and what is looked for later are the same logits, as both ask here.
#pragma once

#include "posit_core.h"

namespace pnn {

constexpr int SAMPLE_BITS = 11, SAMPLE_BINS = 1 << SAMPLE_BITS;

// Bins to one of a logit's unit: the range whose weights are not nothing, s + 3 powers of two, over all bins but the last, which holds what lies below it; 0, and all in
// one bin, where the largest alone is asked for
PNN_HD float sample_bin_scale(int shift, double inverse, bool greedy) {
    return greedy ? 0.f : fminf((float)((SAMPLE_BINS - 1) * inverse / ((shift + 3) * 0.6931471805599453)), 1e38f);
}
// The bin of a logit that is not above `top`, by its difference to that; -1, none, of -inf.  (A difference that is infinite falls into the last bin, times a scale of 0 too.)
PNN_HD int sample_float_bin(float v, float top, float scale) {
    return v > -__builtin_huge_valf() ? (int)fminf((top - v) * scale, (float)(SAMPLE_BINS - 1)) : -1;
}

}  // namespace pnn
