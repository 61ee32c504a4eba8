// The join of attention's parts, where a long range of states is split over workgroups: one kernel for all that do so.
#pragma once

#include "hp_device.hpp"
#include "hp_operators.h"

namespace hp {

constexpr int kMostParts = kWave;                  // a lane for each

// Each part's softmax over what it saw: products [splits][rows * heads_q][dim], divided by the part's sum of exponentials,
// and lse2 [splits][rows * heads_q], its logarithm to base two, -inf where the part saw nothing.
struct Parts {
    float *products, *lse2;
    int32_t splits;
};

// out, and lse (natural; may be NULL), of all parts together.  HP_OK or HP_EHIP.
int join_parts(const Parts &n, int dtype, int64_t rows, int heads_q, int dim, const hp_heads_t &out, float *lse, hipStream_t s);

}  // namespace hp
