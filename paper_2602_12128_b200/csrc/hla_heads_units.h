// Which rows the groups of lanes of the head preparation's forward go through.  Plain C++, for the kernel, its launch and tests on the CPU.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define HLA_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define HLA_HOST_DEVICE inline
#endif

namespace hla {
namespace heads {

// A group's unit is one token of one run of heads (of one tensor).  The units of a run are filled up to whole warps: a warp's groups then have one
// run, so they take the branches that depend on the tensor together, as the shuffles within them need.
struct Units {
    uint32_t tokens, per_run, all;
};
HLA_HOST_DEVICE Units units_of(uint32_t tokens, uint32_t runs, int log_lanes) {
    const uint32_t groups = 32u >> log_lanes, per_run = (tokens + groups - 1) / groups * groups;
    return {tokens, per_run, per_run * runs};
}

struct Unit {
    uint32_t run, token;
    bool live;      // else run and token are those of another unit, and nothing is read or written
};
HLA_HOST_DEVICE Unit unit_of(const Units& u, uint32_t unit) {
    if (unit >= u.all) return {0, 0, false};      // (whole warps)
    const uint32_t run = unit / u.per_run, token = unit - run * u.per_run;
    return {run, token < u.tokens ? token : 0, token < u.tokens};
}

}  // namespace heads
}  // namespace hla
