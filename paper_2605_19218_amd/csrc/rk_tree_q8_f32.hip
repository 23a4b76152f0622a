// Attention of several query rows a KV head (rk_attn_rows.hpp), 8-bit cache, fp32 rows.
#include <type_traits>
#include "rk_attn_rows.hpp"

namespace rk {
hipError_t launch_rows_q8_f32(const RowsArgs& a, int, hipStream_t st) { return launch_rows_fmt<ROWS_Q8_F32>(a, st); }
hipError_t launch_window_rows_q8_f32(const WindowRowsArgs& a, hipStream_t st) { return launch_window_fmt<ROWS_Q8_F32>(a, st); }
}  // namespace rk
