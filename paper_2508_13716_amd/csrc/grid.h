// Sizes of launches whose workgroups stride over their jobs.
#pragma once

#include <cstdint>

namespace capgnn {

// A launch holds fewer than 2^32 threads in a dimension: up to 2^30 of them, and the workgroups take further jobs in turn.
constexpr unsigned stride_grid(int64_t jobs, int threads) {
    const int64_t most = (int64_t(1) << 30) / threads;
    return static_cast<unsigned>(jobs < most ? jobs : most);
}

}  // namespace capgnn
