// Attention of several query rows a KV head (rk_attn_rows.hpp, rk_attn_block.hpp), 8-bit cache, bf16 rows.
#include <type_traits>
#include "rk_attn_block.hpp"

namespace rk {
hipError_t launch_rows_q8_bf16(const RowsArgs& a, int nrb16, hipStream_t st) 
{
    return nrb16 <= 2 ? launch_rows_fmt<ROWS_Q8_BF16>(a, nrb16, st) : launch_block_fmt<ROWS_Q8_BF16>(a, nrb16, st);
}
}  // namespace rk
