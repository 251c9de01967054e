// The attention kernels' launchers (fq_attn.hip chooses between them).
#pragma once

#include <atomic>

#include "fq_attn_device.hpp"
#include "fq_launch.hpp"

namespace fq {

// rows: of a workgroup, 128 or (head sizes up to 128) 256
hipError_t launch_attention_tile(bool cached, const AttnArgs &a, const Split &sp, int rows, hipStream_t s);
hipError_t launch_attention_stream(bool cached, const AttnArgs &a, const Split &sp, hipStream_t s);

}  // namespace fq
