// How the gradient of layer norm is cut into runs of rows: by the number and width of the rows alone, since the order of the sums
// over rows goes by it.
#pragma once
#include <cstdint>

namespace ivk {
namespace {

constexpr uint32_t kThreads = 512;
constexpr uint32_t kWideWarps = 8;
constexpr uint64_t kWidest = 8u * kThreads * 2u;      // columns of the kernel that reads its rows once
constexpr uint64_t kMostParts = 148;      // runs of rows: one for each of a B200's SMs, whatever GPU it is
constexpr uint32_t kPartRows = 2;         // and no fewer rows than this per group of threads, if there are that many

// Threads of a row's group.
inline uint32_t threads_for(uint64_t dim) {
    uint32_t t = 8;
    while (t < kThreads && 8u * (uint64_t)t < dim) t *= 2u;
    return t;
}
inline uint64_t part_count(uint64_t n, uint32_t groups) {
    const uint64_t parts = (n + (uint64_t)groups * kPartRows - 1) / ((uint64_t)groups * kPartRows);
    return parts < kMostParts ? (parts ? parts : 1u) : kMostParts;
}
inline uint64_t parts_for(uint64_t n, uint64_t dim) {
    if (dim <= kWidest) return part_count(n, kThreads / threads_for(dim));
    const uint64_t tiles = (dim + 255u) / 256u, most = 2368u / tiles ? 2368u / tiles : 1u, parts = part_count(n, kWideWarps);
    return parts < most ? parts : most;                  // 16 CTAs for each of a B200's SMs, all tiles together
}

}  // namespace
}  // namespace ivk
