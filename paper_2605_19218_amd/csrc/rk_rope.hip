// Positions of several axes on the rows of queries and Keys, and new tokens into the text segment with their positions on.
//
//   angle(t, i) = pos[axis(i)][t] inv_freq[i],  (x, y) of pair i -> (x cos - y sin, x sin + y cos)
//
// The angle is needed modulo a turn, and a far position times a frequency in fp32 has lost those bits (a position of 10^6 would be off by 0.06 radians): the
// product and its division by 2 pi are fp64, and what is left of a turn, within half of one, is fp32 again, where sincospi takes it.  Pairs, products and
// sums are fp32, rounded once.
// Eight lanes take a row, eight pairs each, in 16-byte pieces: channels 8 o ..+7 and n_pairs + 8 o ..+7 (or 16 o ..+15 for neighbours), so that a pair's two channels
// are in one lane.  Its sines and cosines are the same in all heads of a token, so a wave takes eight tokens through several heads with them in registers; with fewer than eight
// tokens it takes one through eight heads.
#include <type_traits>
#include "rk_kernels.hpp"

namespace rk {

namespace {

// Eight channels of a row, in memory and as fp32.
template <typename T> struct Piece;
template <> struct Piece<bf16_t> {
    uint4 d;
    __device__ __forceinline__ void load(const bf16_t* p) { d = *(const uint4*)p; }
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

// VEC: n_pairs is a multiple of 8, so that pieces are aligned and a lane's pairs are all there or none; else element by element.
// ONE: a wave's eight rows are heads of one token, else eight tokens of a head, and `heads_per` heads follow each other.
template <typename T, bool VEC, bool ONE>
__global__ __launch_bounds__(ONE ? 1024 : 256) void rope_rows(RopeArgs A, int heads_per, int32_t* __restrict__ tickets, int apart)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, o = lane & 7, slot = lane >> 3, b = blockIdx.z;
    const int nq = A.q ? A.Hq : 0, nk = A.k ? A.Hkv : 0, heads = nq + nk + (A.v ? A.Hkv : 0);
    const int t = ONE ? blockIdx.x : (blockIdx.x * 4 + wave) * 8 + slot;
    const int h0 = ONE ? (blockIdx.y * (blockDim.x >> 6) + wave) * 8 + slot : blockIdx.y * heads_per;
    const int h1 = min(heads, ONE ? h0 + 1 : h0 + heads_per);
    const bool adj = A.pairing != 0;
    const int np = A.n_pairs;

    const int n = min(max(A.n_dev ? A.n_dev[b] : A.n, 0), A.n);
    const int len = A.len ? A.len[b] : 0;
    const int fit = A.len ? (len < 0 ? 0 : min(n, max(A.cap - len, 0))) : n;      // rows of Keys and Values that are written

    if (t < n && h0 < h1) {
        float c[8], s[8];
        int p[RK_AXES];
#pragma unroll
        for (int a = 0; a < RK_AXES; ++a) p[a] = a < A.n_axes ? A.pos[a * A.pos_sa + (int64_t)b * A.pos_sb + t] : 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = 8 * o + e;
            const uint64_t word = o < 4 ? A.axes[0] : A.axes[1];
            const int a = (int)(word >> (2 * (i & 31))) & 3;
            const int at = a < 2 ? (a == 0 ? p[0] : p[1]) : (a == 2 ? p[2] : p[3]);
            const double turns = (double)at * (double)(i < np ? A.inv_freq[i] : 0.f) * 0.15915494309189533577;
            sincospif(2.f * (float)(turns - rint(turns)), &s[e], &c[e]);
            s[e] = A.inverse ? -s[e] : s[e];
        }
        // where row t of head h is read and written; false: it is not written
        auto place = [&](int h, const T*& from, T*& to, bool& turned) {
            turned = h < nq + nk;
            if (h < nq) {
                from = (const T*)A.q + (int64_t)b * A.q_sb + (int64_t)h * A.q_sh + (int64_t)t * A.q_st;
                to = (T*)A.qo + (int64_t)b * A.qo_sb + (int64_t)h * A.qo_sh + (int64_t)t * A.qo_st;
                return true;
            }
            const int hk = turned ? h - nq : h - nq - nk;
            from = turned ? (const T*)A.k + (int64_t)b * A.k_sb + (int64_t)hk * A.k_sh + (int64_t)t * A.k_st
                          : (const T*)A.v + (int64_t)b * A.v_sb + (int64_t)hk * A.v_sh + (int64_t)t * A.v_st;
            to = (turned ? (T*)A.ko : (T*)A.vo) + (int64_t)b * A.ko_sb + (int64_t)hk * A.ko_sh + (int64_t)(len + t) * A.ko_st;
            return t < fit;
        };
        for (int h = h0; h < h1; ++h) {
            const T* from;
            T* to;
            bool turned;
            if (!place(h, from, to, turned)) continue;
            if constexpr (VEC) {
                const bool mine = turned && 8 * o < np;
                const int c0 = mine && !adj ? 8 * o : 16 * o, c1 = mine && !adj ? np + 8 * o : 16 * o + 8;
                Piece<T> u, v;
                u.load(from + c0);
                v.load(from + c1);
                if (mine) {
                    float x[8], y[8];
                    u.get(x);
                    v.get(y);
                    if (adj) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float a0 = x[2 * e], a1 = x[2 * e + 1], b0 = y[2 * e], b1 = y[2 * e + 1];
                            x[2 * e] = fmaf(a0, c[e], -a1 * s[e]);
                            x[2 * e + 1] = fmaf(a0, s[e], a1 * c[e]);
                            y[2 * e] = fmaf(b0, c[4 + e], -b1 * s[4 + e]);
                            y[2 * e + 1] = fmaf(b0, s[4 + e], b1 * c[4 + e]);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float a0 = x[e], a1 = y[e];
                            x[e] = fmaf(a0, c[e], -a1 * s[e]);
                            y[e] = fmaf(a0, s[e], a1 * c[e]);
                        }
                    }
                    u.set(x);
                    v.set(y);
                }
                u.store(to + c0);
                v.store(to + c1);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int i = 8 * o + e;
                    const bool mine = i < np;
                    const int c0 = mine && !adj ? i : 2 * i, c1 = mine && !adj ? np + i : 2 * i + 1;
                    if (turned && mine) {
                        const float a0 = ld_elem(from + c0), a1 = ld_elem(from + c1);
                        st_elem(to + c0, fmaf(a0, c[e], -a1 * s[e]));
                        st_elem(to + c1, fmaf(a0, s[e], a1 * c[e]));
                    } else {
                        const T a0 = from[c0], a1 = from[c1];
                        to[c0] = a0;
                        to[c1] = a1;
                    }
                }
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
        if (a.n < 8) {
            const int waves = (heads + 7) / 8, each = waves < 16 ? waves : 16;
            rope_rows<T, VEC, true><<<dim3(a.n, (waves + each - 1) / each, a.B), 64 * each, 0, st>>>(a, 1, tickets, tickets_apart(a.B));
        } else {
            const int64_t groups = (int64_t)a.B * ((a.n + 31) / 32);
            int per = 8;
            while (per > 1 && groups * ((heads + per - 1) / per) < 2 * n_cu) per /= 2;
            rope_rows<T, VEC, false><<<dim3((a.n + 31) / 32, (heads + per - 1) / per, a.B), 256, 0, st>>>(a, per, tickets, tickets_apart(a.B));
        }
        return hipGetLastError();
    };
    auto by_type = [&](auto vec) { return dtype == 0 ? go(0.f, vec) : go(bf16_t{}, vec); };
    return a.n_pairs % 8 == 0 ? by_type(std::true_type{}) : by_type(std::false_type{});
}

}  // namespace rk
