// Launchers of the kernels behind finch_rotate, finch_quantize and finch_attend; each returns
// hipGetLastError() after the launch.
#pragma once

#include "attend_common.h"

namespace finch {

hipError_t launch_attend_rows(int head_dim, bool eight, const AttendParams& p, int workgroups, hipStream_t s);
hipError_t launch_attend_rows16(int head_dim, bool eight, const AttendParams& p, int workgroups, hipStream_t s);
hipError_t launch_attend_tiles(int head_dim, bool eight, const AttendParams& p, int workgroups, hipStream_t s);
hipError_t launch_attend_rows_f32(int head_dim, const AttendParams& p, int workgroups, hipStream_t s);
// joins the splits of `tiles` tiles of `tile_rows` rows and `tile_keys` keys, of `problems` problems of at most rows_max rows each; p's
// runs are those with splits and start at their first tile of rows
hipError_t launch_attend_join(int head_dim, bool bf16, int tile_rows, int tile_keys, int rows_max, int problems, int tiles, AttendParams& p, hipStream_t s);
hipError_t launch_rotate(int head_dim, bool bf16, const finch_rotary& how, const finch_rows* descs, int n, int group, int n_max,
                         hipStream_t s);
hipError_t launch_quantize(int head_dim, bool bf16, const finch_quantization* descs, int n, int n_max, int block, hipStream_t s);

}  // namespace finch
