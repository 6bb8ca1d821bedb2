// A rotary table on one device, made by psattn_rope.hip, read by its kernels and by psattn_rope_apply.hip.
#pragma once
#include <cstdint>

#include "psattn.h"

struct psattn_rope {
    int32_t head_dim = 0;
    int32_t rotary_dim = 0;    // the first dimensions of a head, that are turned
    int32_t layout = PSATTN_ROPE_HALF;
    int32_t max_positions = 0;
    int device = -1;
    float* d_table = nullptr;  // [max_positions][rotary_dim]: cosines of the pairs' angles | sines
};

namespace psattn {

constexpr int32_t kRopeMostDims = 512;  // of a head

}  // namespace psattn
