// What follows the attention of several query rows a KV head (rk_attn_rows.hpp): the fold of its partials, and the way of the accepted drafts
// into the text segment.
#include <type_traits>
#include "rk_attn_rows.hpp"

namespace rk {

// out = sum_i acc_i w_i / sum_i l_i w_i, w_i = 2^(m_i - M).  32 lanes take a row, 4 channels each.  WIDE: the eight groups of 32 lanes of a
// work-group share the partials of one row, for few rows with many partials; else a group has a row of its own.  Bound by two round trips, and by
// memory from some thousand rows on: 2 us for 32 rows x 8 partials, 8 for 3584 x 16 (31 MB, which the L2 holds in part), 9.4 for 14336 x 7.  WIDE against not, us
// of the whole call: 512 rows x 16 17.5 / 20.4, 896 x 16 23.0 / 25.8, 1792 x 16 65.6 / 67.5, 3584 x 16 80.1 / 77.4, 7168 x 8 81.2 / 75.1.
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void rows_merge(const float* __restrict__ ws_m, const float* __restrict__ ws_l, const float* __restrict__ ws_acc,
                                                  T* __restrict__ out, int rows, int S, int Hq, int n_tok, const int32_t* __restrict__ n_drafts)
{
    __shared__ f32x4 part[WIDE ? 8 : 1][32];
    __shared__ float den[WIDE ? 8 : 1];
    const int tid = threadIdx.x, p = tid & 31, grp = tid >> 5;
    const int row = WIDE ? blockIdx.x : blockIdx.x * 8 + grp;
    if (row >= rows) return;
    const int bt = row / Hq, b = bt / n_tok;
    if (n_drafts && bt - b * n_tok >= n_drafts[b]) return;       // (rows behind the last draft stay as they were)
    f32x4 num;
    float sum;
    merge_row<WIDE ? 2 : 4>(ws_m + (size_t)row * S, ws_l + (size_t)row * S, ws_acc + (size_t)row * S * D, S, WIDE ? grp : 0, WIDE ? 8 : 1, p, num, sum);
    if constexpr (WIDE) {
        part[grp][p] = num;
        if (p == 0) den[grp] = sum;
        __syncthreads();
        if (grp) return;
#pragma unroll
        for (int k = 1; k < 8; ++k) {
            num += part[k][p];
            sum += den[k];
        }
    }
    const float inv = 1.f / sum;
    T* o = out + (size_t)row * D + 4 * p;
#pragma unroll
    for (int e = 0; e < 4; ++e) st_elem(o + e, sum == 0.f ? 0.f : num[e] * inv);
}

hipError_t launch_rows_merge(int dtype, const RowsArgs& a, hipStream_t st)
{
    const int rows = a.B * a.T * a.Hq, S = a.Sv + a.Sr;
    auto go = [&](auto t) {
        typedef decltype(t) E;
        if (S > 4 && rows <= 2048)
            rows_merge<E, true><<<rows, 256, 0, st>>>(a.ws_m, a.ws_l, a.ws_acc, (E*)a.out, rows, S, a.Hq, a.T, a.draft_k ? a.n_drafts : nullptr);
        else
            rows_merge<E, false><<<(rows + 7) / 8, 256, 0, st>>>(a.ws_m, a.ws_l, a.ws_acc, (E*)a.out, rows, S, a.Hq, a.T,
                                                                 a.draft_k ? a.n_drafts : nullptr);
        return hipGetLastError();
    };
    return dtype == 0 ? go(0.f) : go(bf16_t{});
}

// ---------------------------------------------------------------------------
// The accepted path of a tree: rows of the drafts, in the path's order, behind the text segment.  A work-group copies eight rows of a head, 16
// bytes a lane.  Bound by its round trips (length and path, then a row): 2.5 us for 4 rows of 8 heads, 6.9 for 64 sequences x 32 heads.  The path ends at its first entry that is no draft, and where the segment is full.  The last work-group of a sequence writes the
// length: len_out may be the length that all of them read.
template <typename T>
__global__ __launch_bounds__(256) void append_path(PathArgs A, int32_t* __restrict__ tickets, int apart)
{
    constexpr int PR = D * (int)sizeof(T) / 16;          // 16-byte pieces of a row
    const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 63;
    const int len = A.text_len[b];
    const int drafts = min(max(A.n_drafts ? A.n_drafts[b] : A.T, 0), A.T);
    const int mine = A.path[(size_t)b * A.P + min(lane, A.P - 1)];
    const uint64_t bad = __ballot(!(lane < A.P && mine >= 0 && mine < drafts));
    int n = bad ? __builtin_ctzll(bad) : 64;
    n = min(n, max(A.n_path[b], 0));
    n = len < 0 ? 0 : min(n, max(A.text_cap - len, 0));
    const int first = blockIdx.x * 8;
    for (int i = tid; i < 8 * 2 * PR; i += 256) {
        const int row = i / (2 * PR), rest = i - row * 2 * PR, piece = rest & (PR - 1), j = first + row;
        const int from = __shfl(mine, j & 63);           // (all lanes take part: no lane leaves the loop before the others)
        if (j >= n) continue;
        const int64_t src = (int64_t)b * A.draft_sb + (int64_t)h * A.draft_sh + (int64_t)from * A.draft_st;
        const int64_t dst = (int64_t)b * A.text_sb + (int64_t)h * A.text_sh + (int64_t)(len + j) * A.text_st;
        if (rest < PR) ((uint4*)((T*)A.text_k + dst))[piece] = ((const uint4*)((const T*)A.draft_k + src))[piece];
        else ((uint4*)((T*)A.text_v + dst))[piece] = ((const uint4*)((const T*)A.draft_v + src))[piece];
    }
    __syncthreads();
    if (tid == 0 && atomicAdd(tickets + (size_t)b * apart, 1) == (int)(gridDim.x * gridDim.y) - 1) {
        tickets[(size_t)b * apart] = 0;
        A.len_out[b] = len + n;
    }
}

hipError_t launch_append_path(int dtype, const PathArgs& a, int32_t* tickets, hipStream_t st)
{
    const dim3 grid((a.P + 7) / 8, a.Hkv, a.B);
    if (dtype == 0) append_path<float><<<grid, 256, 0, st>>>(a, tickets, tickets_apart(a.B));
    else append_path<bf16_t><<<grid, 256, 0, st>>>(a, tickets, tickets_apart(a.B));
    return hipGetLastError();
}

}  // namespace rk
