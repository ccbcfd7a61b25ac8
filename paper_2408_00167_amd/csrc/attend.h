// Launchers of the kernels behind finch_rotate, finch_quantize and finch_attend; each returns
// hipGetLastError() after the launch.
#pragma once

#include "attend_common.h"

namespace finch {

hipError_t launch_attend_rows(int head_dim, bool eight, const AttendParams& p, hipStream_t s);
hipError_t launch_attend_rows16(int head_dim, bool eight, const AttendParams& p, hipStream_t s);
hipError_t launch_attend_tiles(int head_dim, bool eight, const AttendParams& p, hipStream_t s);
hipError_t launch_attend_rows_f32(int head_dim, const AttendParams& p, hipStream_t s);
// joins the splits of tiles of `tile_rows` rows and `tile_keys` keys; rows_max: of a problem
hipError_t launch_attend_join(int head_dim, bool bf16, int tile_rows, int tile_keys, int rows_max, const AttendParams& p, hipStream_t s);
hipError_t launch_rotate(int head_dim, bool bf16, const finch_rotary& how, const finch_rows* descs, int n, int group, int n_max,
                         hipStream_t s);
hipError_t launch_quantize(int head_dim, bool bf16, const finch_quantization* descs, int n, int n_max, int block, hipStream_t s);

}  // namespace finch
