// Attention of several query rows a KV head (rk_attn_rows.hpp, rk_attn_block.hpp), 8-bit cache, bf16 rows.
#include <type_traits>
#include "rk_attn_block.hpp"

namespace rk {
hipError_t launch_rows_q8_bf16(const RowsArgs& a, int rows, hipStream_t st)
{
    return rows == 16 ? launch_rows_fmt<ROWS_Q8_BF16>(a, st) : launch_block_fmt<ROWS_Q8_BF16>(a, rows, st);
}
}  // namespace rk
