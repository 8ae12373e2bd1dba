// What a call of surel_sample_classes is given.
#pragma once

#include <stdint.h>

namespace surel {

struct SampleArgs {
    const char* logits = nullptr;
    int64_t row = 0;    // bytes
    int32_t n_rows = 0, n_classes = 0;
    const float *u = nullptr, *temperature = nullptr;
    const int32_t* top_k = nullptr;
    const float *top_p = nullptr, *min_p = nullptr;
    int32_t* chosen = nullptr;
    float* logp = nullptr;
    uint32_t* err = nullptr;
};

}  // namespace surel
