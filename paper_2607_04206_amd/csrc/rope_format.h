// Plan blob of rotary positions (rope_plan.cpp writes it, rope.hip reads it):
// a header and the turns per position of every pair, position independent like
// the other plans.
#pragma once

#include <stdint.h>

namespace sangam {

constexpr uint32_t kRopePlanMagic = 0x50525347u;  // "GSRP"
constexpr uint32_t kRopePlanVersion = 1;
constexpr int kRopeMaxDim = 512;

struct RopePlanHeader {
    uint32_t magic;
    uint32_t version;
    uint64_t total_bytes;
    int32_t rot_dim;
    int32_t interleaved;
    float magnitude;
    int32_t reserved;
    uint64_t off_turns;  // double[rot_dim / 2]
};

static_assert(sizeof(RopePlanHeader) == 40, "RopePlanHeader layout is part of the blob format");

}  // namespace sangam
