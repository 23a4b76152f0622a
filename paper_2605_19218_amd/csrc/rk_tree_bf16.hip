// Attention of several query rows a KV head (rk_attn_rows.hpp, rk_attn_block.hpp), packed bf16 cache, bf16 rows.
#include <type_traits>
#include "rk_attn_block.hpp"

namespace rk {
hipError_t launch_rows_bf16(const RowsArgs& a, int rows, hipStream_t st)
{
    return rows == 16 ? launch_rows_fmt<ROWS_BF16>(a, st) : launch_block_fmt<ROWS_BF16>(a, rows, st);
}
hipError_t launch_window_rows_bf16(const WindowRowsArgs& a, hipStream_t st) { return launch_window_fmt<ROWS_BF16>(a, st); }
}  // namespace rk
