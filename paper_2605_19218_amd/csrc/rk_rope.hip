// Positions of several axes on the rows of queries and Keys, and new tokens into the text segment with their positions on.
//
//   angle(t, i) = pos[axis(i)][t] inv_freq[i],  (x, y) of pair i -> (x cos - y sin, x sin + y cos)
//
// The angle is needed modulo a turn, and a far position times a frequency in fp32 has lost those bits (a position of 10^6 would be off by up to 0.03 radians): the
// product and its division by 2 pi are fp64, and what is left of a turn, within half of one, is fp32 again, where sincospi takes it.  Pairs, products and
// sums are fp32, rounded once.
// Pairs of halves: eight lanes take a row, eight pairs each, in pieces of eight channels, 8 o ..+7 and n_pairs + 8 o ..+7, so that a pair's two channels are in one lane; neighbours, and halves
// that are no multiple of eight, sixteen lanes.  Sines and cosines are the same in all heads of a token: a work-group makes those of its tokens once, in LDS, and takes the tokens' heads in the
// order in which they lie in memory.  (Made by each lane for its own pairs, a wave taking eight tokens through head after head: 50 us in place of 43 below.)
// Bound by memory: 28 + 4 heads x 71000 tokens of bf16 270 us, 1.44 GB, 5.3 TB/s; fp32, 32 + 32 heads x 2944 tokens from memory 43 us, 193 MB, 4.5 TB/s (a copy of as many bytes 37); 28 +
// 4 + 4 heads x 4400 tokens into segments 23.5 us, 116 MB, 4.9 TB/s; one token of 64 sequences x 96 heads 3.5 us. 328 MB, 40 heads: bf16 x 16000 tokens 64 pairs 67 us, neighbours 71, 13 pairs 75 (117 with
// the pairs' other channels read one by one, 89 with each of a lane's pieces waited for before the next was asked for), 63 87 (99); fp32 x 8000 65, 68, 70, 74.
#include <type_traits>
#include "rk_kernels.hpp"

namespace rk {

namespace {

// Eight channels of a row, in memory and as fp32.
template <typename T> struct Piece;
template <> struct Piece<bf16_t> {
    uint4 d;
    __device__ __forceinline__ void load(const bf16_t* p) { d = *(const uint4*)p; }
    __device__ __forceinline__ void load_anywhere(const bf16_t* p) { __builtin_memcpy(&d, p, 16); }
    __device__ __forceinline__ void store(bf16_t* p) const { *(uint4*)p = d; }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
        const uint32_t w[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, (bf16x2){(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
        d = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <> struct Piece<float> {
    f32x4 a, b;
    __device__ __forceinline__ void load(const float* p) { a = *(const f32x4*)p; b = *(const f32x4*)(p + 4); }
    __device__ __forceinline__ void load_anywhere(const float* p)
    {
        __builtin_memcpy(&a, p, 16);
        __builtin_memcpy(&b, p + 4, 16);
    }
    __device__ __forceinline__ void store(float* p) const { *(f32x4*)p = a; *(f32x4*)(p + 4) = b; }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
    }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) { a[i] = x[i]; b[i] = x[4 + i]; }
    }
};

// VEC: pairs of halves, a multiple of 8, so that a lane's are all there or none, in two aligned pieces; else a lane has one piece (sixteen lanes a row): neighbours are all in it (fp32, 64 pairs,
// 40 heads x 8000 tokens 68 us, in two pieces of sixteen channels a lane 83), the other channels of pairs of halves it reads from where they are, at any alignment.
// A work-group takes TOKENS tokens (one, where there are fewer) through 1 << log_heads heads, a token's heads one after another, which is how a projection leaves them.
template <typename T, bool VEC, int TOKENS>
__global__ __launch_bounds__(TOKENS == 1 ? 1024 : 256) void rope_rows(RopeArgs A, int log_heads, int32_t* __restrict__ tickets, int apart)
{
    constexpr int LANES = VEC ? 8 : 16, ANGLES = VEC ? 64 : 128;
    // by pairs; else by channels, what its own number and the pair's other one are taken times
    __shared__ __attribute__((aligned(16))) float cosines[TOKENS][ANGLES], sines[TOKENS][ANGLES];
    const int tid = threadIdx.x, o = tid % LANES, b = blockIdx.z, t0 = blockIdx.x * TOKENS, h0 = blockIdx.y << log_heads;
    const int nq = A.q ? A.Hq : 0, nk = A.k ? A.Hkv : 0, heads = nq + nk + (A.v ? A.Hkv : 0);
    const bool adj = A.pairing != 0;
    const int np = A.n_pairs;

    const int n = min(max(A.n_dev ? A.n_dev[b] : A.n, 0), A.n);
    const int len = A.len ? A.len[b] : 0;
    const int fit = A.len ? (len < 0 ? 0 : min(n, max(A.cap - len, 0))) : n;      // rows of Keys and Values that are written

    if (t0 < n) {
        for (int x = tid; x < TOKENS * 64; x += blockDim.x) {
            const int t = t0 + (x >> 6), i = x & 63;
            if (t >= n || i >= np) continue;
            const int a = (int)((i < 32 ? A.axes[0] : A.axes[1]) >> (2 * (i & 31))) & 3;
            const double turns = (double)A.pos[a * A.pos_sa + (int64_t)b * A.pos_sb + t] * (double)A.inv_freq[i] * 0.15915494309189533577;
            float s, c;
            sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
            if (A.inverse) s = -s;
            const int one = VEC ? i : adj ? 2 * i : i, two = adj ? 2 * i + 1 : np + i;
            cosines[x >> 6][one] = c;
            sines[x >> 6][one] = VEC ? s : -s;
            if (!VEC) {
                cosines[x >> 6][two] = c;
                sines[x >> 6][two] = s;
            }
        }
        __syncthreads();
        for (int r = tid / LANES; r < TOKENS << log_heads; r += blockDim.x / LANES) {
            const int tl = r >> log_heads, t = t0 + tl, h = h0 + (r & ((1 << log_heads) - 1));
            if (t >= n || h >= heads) continue;
            const bool turned = h < nq + nk;
            const T* from;
            T* to;
            if (h < nq) {
                from = (const T*)A.q + (int64_t)b * A.q_sb + (int64_t)h * A.q_sh + (int64_t)t * A.q_st;
                to = (T*)A.qo + (int64_t)b * A.qo_sb + (int64_t)h * A.qo_sh + (int64_t)t * A.qo_st;
            } else {
                if (t >= fit) continue;
                const int hk = turned ? h - nq : h - nq - nk;
                from = turned ? (const T*)A.k + (int64_t)b * A.k_sb + (int64_t)hk * A.k_sh + (int64_t)t * A.k_st
                              : (const T*)A.v + (int64_t)b * A.v_sb + (int64_t)hk * A.v_sh + (int64_t)t * A.v_st;
                to = (turned ? (T*)A.ko : (T*)A.vo) + (int64_t)b * A.ko_sb + (int64_t)hk * A.ko_sh + (int64_t)(len + t) * A.ko_st;
            }
            Piece<T> u, v;
            float x[8], y[8], c[8], s[8];
            if constexpr (VEC) {
                const bool mine = turned && 8 * o < np;
                u.load(from + (mine ? 8 * o : 16 * o));
                v.load(from + (mine ? np + 8 * o : 16 * o + 8));
                if (mine) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) { c[e] = cosines[tl][8 * o + e]; s[e] = sines[tl][8 * o + e]; }
                    u.get(x);
                    v.get(y);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float a0 = x[e], a1 = y[e];
                        x[e] = fmaf(a0, c[e], -a1 * s[e]);
                        y[e] = fmaf(a0, s[e], a1 * c[e]);
                    }
                    u.set(x);
                    v.set(y);
                }
                u.store(to + (mine ? 8 * o : 16 * o));
                v.store(to + (mine ? np + 8 * o : 16 * o + 8));
            } else {
                u.load(from + 8 * o);
                const bool mine = turned && 8 * o < 2 * np, first_half = 8 * o < np, ends = first_half && 8 * o + 8 > np;
                Piece<T> w;
                if (!adj && mine) {
                    // (np is 63 at most here, so that eight from 8 o + np on end inside the row; where a half ends inside a piece, the others' are the row's first)
                    v.load_anywhere(from + (first_half ? 8 * o + np : 8 * o - np));
                    if (ends) w.load(from);
                }
                // A result may lie over its source, and the row's lanes read each other's channels: all of them are one wave's, and none of it stores before all have read.
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
                if (mine) {
                    u.get(x);
                    if (adj) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] = x[e ^ 1];
                    } else {
                        v.get(y);
                        if (ends) {
                            float z[8];
                            w.get(z);
#pragma unroll
                            for (int k = 1; k < 8; ++k)
                                if ((np & 7) == k)
#pragma unroll
                                    for (int e = k; e < 8; ++e) y[e] = z[e - k];
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) { c[e] = cosines[tl][8 * o + e]; s[e] = sines[tl][8 * o + e]; }
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (8 * o + e < 2 * np) x[e] = fmaf(x[e], c[e], y[e] * s[e]);
                    u.set(x);
                }
                u.store(to + 8 * o);
            }
        }
    }

    if (!A.len_out) return;
    if (A.len_out != A.len || gridDim.x * gridDim.y == 1) {
        __syncthreads();
        if (tid == 0 && blockIdx.x == 0 && blockIdx.y == 0) A.len_out[b] = len + fit;
        return;
    }
    // len_out is the length that all work-groups of the sequence read: the last of them writes it
    __syncthreads();
    if (tid == 0 && atomicAdd(tickets + (size_t)b * apart, 1) == (int)(gridDim.x * gridDim.y) - 1) {
        tickets[(size_t)b * apart] = 0;
        A.len_out[b] = len + fit;
    }
}

}  // namespace

hipError_t launch_rope(int dtype, const RopeArgs& a, int32_t* tickets, int n_cu, hipStream_t st)
{
    const int heads = (a.q ? a.Hq : 0) + (a.k ? a.Hkv : 0) + (a.v ? a.Hkv : 0);
    auto go = [&](auto e, auto vec) {
        typedef decltype(e) T;
        constexpr bool VEC = decltype(vec)::value;
        constexpr int lanes = VEC ? 8 : 16, rows = 256 / lanes;       // of a row; of a work-group's step
        int log_heads = 0;
        if (a.n < ROPE_TOKENS) {
            // a token's heads in one work-group, up to 1024 lanes
            while ((1 << log_heads) < heads && (lanes << log_heads) < 1024) ++log_heads;
            const int threads = lanes << log_heads < 64 ? 64 : lanes << log_heads;
            rope_rows<T, VEC, 1><<<dim3(a.n, (heads + (1 << log_heads) - 1) >> log_heads, a.B), threads, 0, st>>>(a, log_heads, tickets, tickets_apart(a.B));
        } else {
            const int blocks = (a.n + ROPE_TOKENS - 1) / ROPE_TOKENS;
            // eight heads, or fewer that leave four work-groups a compute unit, but a step of a work-group at least (fp32, 32 + 32 heads x 2944 tokens with 8, 16, 32 heads
            // 43.4, 46.1, 46.2 us; 28 + 4 heads x 71000 tokens 270, 272, 277; 28 + 4 + 4 x 4400 tokens, appended 26.2, 28.8, 33.8)
            while ((1 << log_heads) < heads && log_heads < 3) ++log_heads;
            while (ROPE_TOKENS << log_heads > rows && (int64_t)a.B * blocks * ((heads + (1 << log_heads) - 1) >> log_heads) < 4 * n_cu) --log_heads;
            rope_rows<T, VEC, ROPE_TOKENS><<<dim3(blocks, (heads + (1 << log_heads) - 1) >> log_heads, a.B), 256, 0, st>>>(a, log_heads, tickets, tickets_apart(a.B));
        }
        return hipGetLastError();
    };
    auto by_type = [&](auto vec) { return dtype == 0 ? go(0.f, vec) : go(bf16_t{}, vec); };
    return a.pairing == 0 && a.n_pairs % 8 == 0 ? by_type(std::true_type{}) : by_type(std::false_type{});
}

}  // namespace rk
