// What the kernels of the softmax loss share.
#pragma once

#include "matrix_tile.h"

namespace surel {

struct LossArgs {
    const char *h = nullptr, *w = nullptr;  // [n_rows][dim], [n_classes][dim]
    const int32_t* labels = nullptr;        // < 0: the row does not count
    int32_t n_rows = 0, n_classes = 0, dim = 0;
    uint32_t* err = nullptr;
};

// A row's label, -1 where it does not count.
__device__ __forceinline__ int label_of(const LossArgs& a, int row) {
    const int label = a.labels[row];
    if (label < a.n_classes) return label < 0 ? -1 : label;
    atomicOr(a.err, kDevBadLabel);
    return -1;
}

// How work on `tiles` tiles of the stationary side and `steps` steps along the streamed one is cut: into
// parts of the streamed side, so that workgroups (tiles * parts of them) fill the device evenly.  Parts are
// numbered fastest and a multiple of 8 of them stays on one XCD each, whose L2 then holds what they stream.
// part_cost: what a part of all tiles costs beside its work, in steps of a workgroup.
inline int parts_for(int64_t tiles, int64_t steps, int slots, int most, double part_cost) {
    int best = 1;
    double least = 1e300;
    for (int parts = 1; parts <= most && parts <= steps; parts = parts < 8 ? 2 * parts : parts + 8) {
        const double rounds = ceil((double)(tiles * parts) / slots);
        // (2: what a workgroup costs beside its steps)
        const double time = rounds * (ceil((double)steps / parts) + 2) + (parts > 1 ? parts * part_cost : 0.0);
        if (time < 0.97 * least) least = time, best = parts;
    }
    return best;
}

}  // namespace surel
