// The persistent kernel of the INT8 gated block (gated_stream.hip): does it serve these operands, and its launch (validated arguments, M and F >= 1;
// tile: one of GATED_*).
#pragma once
#include "common.h"

namespace ibert {

// Tiles: 128 tokens by 128 channels, 256 by 128, 128 by 64 (two workgroups to a compute unit).
enum { GATED_LOW = 1, GATED_TALL = 2, GATED_NARROW = 3 };

bool gated_stream_ok(const ibert_gated_desc& d, const int8_t* A, const int8_t* W);
int launch_gated_stream(const ibert_gated_desc& d, const int8_t* A, const int8_t* W, const int32_t* bias, const int32_t* mult, const int32_t* shift, int8_t* C, int tile,
                        hipStream_t stream);

}  // namespace ibert
