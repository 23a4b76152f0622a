// Attention of several query rows a KV head over one rotated cache: drafted tokens (a tree of them, with the text segment and the drafts'
// own full-width rows) over the packed or the 8-bit cache, and the single token over the 8-bit cache.
//
//   row (t, h) of KV head hk: x_c = q R_r . k~_c + q . delta_mu, x_m = q . k_m (text rows, and drafts that mask[t] names),
//   out = softmax(scale x) . (V_c, V_m)       one softmax; a row that sees nothing: zeros.
//
// A KV head's T G rows share its Keys and Values, so a work-group takes 16 rows (a matrix-core column each) over one stretch of
// tokens, a wave 32 tokens at a time: every Key and Value is requested once for all the rows, straight into the registers that feed the matrix
// cores, and nothing passes through LDS in the loop.  Both products are turned so that a lane keeps one row: S^T = K q^T leaves lane (g, n)
// with row n's scores of tokens 4 g ..+3, which is how O^T = V^T P^T wants them as its B operand, and every accumulator of the lane belongs to row
// n as well.  So the running maximum and sum are per lane, and a new maximum rescales without any exchange.
// The running maximum follows a row's true one only when it falls behind by 2^8: weights stay below 256, and the accumulators are
// rescaled a few times instead of at every new maximum.  Maxima, sums and accumulators are fp32.  Over 16-bit products the weights go as two
// bf16 parts (17 bits), as q R_r does; with fp32 rows three (all 24); a code is exact in one.
// Stretches: the cache's 32-token tiles are shared by the first Sv splits, the text's and the drafts' by the others, by the sequence's own lengths;
// rows_merge folds the partials (inside the launch, by the work-group that ends last, it took up to 3 us more: one work-group reads all of a unit).  More than 16
// rows are blocks of 16 that read the same tokens, on one XCD, out of its L2, up to where attn_block is faster.  (Two blocks of 16 in one wave
// shared each read, but their accumulators wandered between the two halves of the register file at every tile: 32 rows, 32 units x 16000 tokens 45.8 us, as
// two work-groups 44.1; 8 x 16000 20.2 and 16.4.)
// What bounds it: memory and its latency.  One token over 8 bits, 28 rows of 4 KV heads x 8 x 16384 tokens, r = 64: 20.2 us for 103 MB, 5.1 TB/s; 32 heads x 2880
// tokens with fp32 rows 10.3 us; 8 heads x 1024 tokens 6.1 us, of which launch, length, rotation and the first tiles' round trips are all but 1.
#pragma once
#include "rk_kernels.hpp"

namespace rk {

enum { ROWS_BF16 = 0, ROWS_F32 = 1, ROWS_Q8_BF16 = 2, ROWS_Q8_F32 = 3 };

constexpr float ROWS_NEG_INF = -__builtin_huge_valf();
constexpr int PARK = 17;         // 16 rows' pieces, and one: lanes that read pieces side by side meet other banks

__device__ __forceinline__ float rows_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// one bf16 part of a weight or a query after another
template <int NP>
__device__ __forceinline__ void parts_of(const float (&x)[8], bf16x8 (&p)[NP])
{
    if constexpr (NP == 2) {
        split_bf16x8(x, p[0], p[1]);
    } else {
        float rest[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
        for (int k = 0; k < NP; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[k][i] = (__bf16)rest[i];
                rest[i] -= (float)p[k][i];
            }
    }
}

// eight codes (two words) as bf16: exact, so the high halves of the floats are all there is
__device__ __forceinline__ bf16x8 codes_bf16(uint32_t lo, uint32_t hi)
{
    uint32_t d[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = i < 2 ? lo : hi;
        const int s = 16 * (i & 1);
        const float a = (float)((int32_t)(w << (24 - s)) >> 24), b = (float)((int32_t)(w << (16 - s)) >> 24);
        d[i] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    }
    return __builtin_bit_cast(bf16x8, make_uint4(d[0], d[1], d[2], d[3]));
}

// The softmax state of a wave: row n in the lanes (., n).
struct RowState {
    float m, l;                  // log2 domain; l: this lane's tokens only, until the end
    f32x4 O[8];
    __device__ __forceinline__ void clear()
    {
        m = ROWS_NEG_INF;
        l = 0.f;
#pragma unroll
        for (int cb = 0; cb < 8; ++cb) O[cb] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    // scores of 32 tokens -> weights
    __device__ __forceinline__ void weigh(f32x4 (&s)[2])
    {
        const float mt = groups_max(fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                                          fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3]))));
        if (__any(mt > m + 8.f)) {
            const float m_new = fmaxf(m, mt);
            const float alpha = m > ROWS_NEG_INF ? rows_exp2(m - m_new) : 0.f;      // (0 . 0 before the first score)
            l *= alpha;
#pragma unroll
            for (int cb = 0; cb < 8; ++cb) O[cb] *= alpha;
            m = m_new;
        }
        const float ref = m > ROWS_NEG_INF ? m : 0.f;         // every score so far may be minus infinity: no weight, not NaN
        float sum = 0.f;
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int ii = 0; ii < 4; ++ii) {
                s[tb][ii] = rows_exp2(s[tb][ii] - ref);
                sum += s[tb][ii];
            }
        l += sum;
    }
};

// ---- tiles of the caches: 32 tokens, R channels (rp of them stored) ------------
// bf16: K [tb][i] octet 4 i + g of token 16 tb + n; V [cb] the eight tokens of group g, channel 16 cb + n
template <int R>
struct TileBf16 {
    uint4 k[2][R / 32], v[8];
    __device__ __forceinline__ void load(const char* Ku, const char* Vu, int tok0, int rp, int lane)
    {
        const int g = lane >> 4;
        const char* kb = Ku + (size_t)(tok0 >> 4) * (32 * rp);
        const char* vb = Vu + (size_t)(tok0 >> 5) * 8192;
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int i = 0; i < R / 32; ++i) {
                const bool in = i < R / 32 - 1 || 32 * i + 8 * g < rp;
                k[tb][i] = *(const uint4*)(kb + tb * 32 * rp + (in ? 1024 * i + 16 * lane : 16 * (lane & 15)));
            }
#pragma unroll
        for (int cb = 0; cb < 8; ++cb) v[cb] = *(const uint4*)(vb + 1024 * cb + 16 * lane);
    }
};
// 8 bits: K [i] octet 4 i + g of tokens n and 16 + n; V [cp] channel blocks 2 cp and 2 cp + 1; steps of tokens 4 g ..+3 of both halves
template <int R>
struct TileQ8 {
    uint4 k[R / 32], v[4], st[2];
    __device__ __forceinline__ void load(const char* Ku, const char* Vu, int tok0, int rp, int lane)
    {
        const int g = lane >> 4;
        const char* kb = Ku + (size_t)(tok0 >> 5) * q8_kblock(rp);
        const char* vb = Vu + (size_t)(tok0 >> 5) * 4096;
#pragma unroll
        for (int i = 0; i < R / 32; ++i) {
            const bool in = i < R / 32 - 1 || 32 * i + 8 * g < rp;      // (what stands there instead meets zeros of q R_r; a code is finite)
            k[i] = *(const uint4*)(kb + (in ? 1024 * i + 16 * lane : 16 * (lane & 15)));
        }
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) st[tb] = *(const uint4*)(kb + 32 * rp + 64 * tb + 16 * g);
#pragma unroll
        for (int cp = 0; cp < 4; ++cp) v[cp] = *(const uint4*)(vb + 1024 * cp + 16 * lane);
    }
};
// fp32: K [tb][i] channels 16 i + 4 g ..+3 of token 16 tb + n; V [cb] as bf16
template <int R>
struct TileF32 {
    f32x4 k[2][R / 16], v[8][2];
    __device__ __forceinline__ void load(const char* Ku, const char* Vu, int tok0, int rp, int lane)
    {
        const int g = lane >> 4, n = lane & 15;
        const char* kb = Ku + (size_t)(tok0 >> 4) * (64 * rp);
        const char* vb = Vu + (size_t)(tok0 >> 5) * 16384;
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int i = 0; i < R / 16; ++i) {
                const bool in = i < R / 16 - 1 || 16 * i < rp;          // (the last sixteen: all stored, or none)
                k[tb][i] = *(const f32x4*)(kb + tb * 64 * rp + (in ? 1024 * i : 0) + 512 * (g >> 1) + 32 * n + 16 * (g & 1));
            }
#pragma unroll
        for (int cb = 0; cb < 8; ++cb) {
            v[cb][0] = *(const f32x4*)(vb + 2048 * cb + 32 * lane);
            v[cb][1] = *(const f32x4*)(vb + 2048 * cb + 32 * lane + 16);
        }
    }
};

// The rotated queries as B operands, and what a tile does with them.
template <int FMT, int R>
struct CacheRows {
    static constexpr bool Q8 = FMT >= ROWS_Q8_BF16, F32 = FMT == ROWS_F32;
    static constexpr int NP = FMT == ROWS_Q8_F32 ? 3 : 2, KS = R / 32;
    bf16x8 qf[F32 ? 1 : KS][NP];
    f32x4 q4[F32 ? R / 16 : 1];

    // qt: [16][R + 4] of LDS
    __device__ __forceinline__ void take(const float* qt, float scale_log2, int g, int n)
    {
        const float* row = qt + n * (R + 4);
        if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < R / 16; ++i) q4[i] = *(const f32x4*)(row + 16 * i + 4 * g) * scale_log2;
        } else {
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const f32x4 a = *(const f32x4*)(row + 32 * i + 8 * g) * scale_log2, b = *(const f32x4*)(row + 32 * i + 8 * g + 4) * scale_log2;
                const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
                parts_of<NP>(x, qf[i]);
            }
        }
    }

    // `left`: tokens of the tile that exist
    __device__ __forceinline__ void step(TileF32<R>& T, RowState& st, int left, int rp, int g)
    {
        f32x4 s[2];
        if (rp < R) {
#pragma unroll
            for (int tb = 0; tb < 2; ++tb) T.k[tb][R / 16 - 1] = (f32x4){0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            s[tb] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < R / 16; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    s[tb] = __builtin_amdgcn_mfma_f32_16x16x4f32(T.k[tb][i][e], q4[i][e], s[tb], 0, 0, 0);
        }
        if (left < 32) {
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                for (int ii = 0; ii < 4; ++ii) {
                    const bool in = 16 * tb + 4 * g + ii < left;
                    s[tb][ii] = in ? s[tb][ii] : ROWS_NEG_INF;
#pragma unroll
                    for (int cb = 0; cb < 8; ++cb) T.v[cb][tb][ii] = in ? T.v[cb][tb][ii] : 0.f;
                }
        }
        st.weigh(s);
#pragma unroll
        for (int cb = 0; cb < 8; ++cb)
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                for (int ii = 0; ii < 4; ++ii)
                    st.O[cb] = __builtin_amdgcn_mfma_f32_16x16x4f32(T.v[cb][tb][ii], s[tb][ii], st.O[cb], 0, 0, 0);
    }

    __device__ __forceinline__ void step(TileBf16<R>& T, RowState& st, int left, int rp, int g)
    {
        f32x4 s[2];
        if (rp < R && g >= 2) {
#pragma unroll
            for (int tb = 0; tb < 2; ++tb) T.k[tb][KS - 1] = make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            s[tb] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KS; ++i)
#pragma unroll
                for (int p = NP - 1; p >= 0; --p)
                    s[tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, T.k[tb][i]), qf[i][p], s[tb], 0, 0, 0);
        }
        if (left < 32) {
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                for (int ii = 0; ii < 4; ++ii) {
                    const bool in = 16 * tb + 4 * g + ii < left;
                    s[tb][ii] = in ? s[tb][ii] : ROWS_NEG_INF;
                    const uint32_t keep = in ? ~0u : (ii & 1 ? 0x0000ffffu : 0xffff0000u);
#pragma unroll
                    for (int cb = 0; cb < 8; ++cb) {
                        uint32_t& w = tb ? (ii < 2 ? T.v[cb].z : T.v[cb].w) : (ii < 2 ? T.v[cb].x : T.v[cb].y);
                        w &= keep;
                    }
                }
        }
        st.weigh(s);
        bf16x8 p[2];
        const float x[8] = {s[0][0], s[0][1], s[0][2], s[0][3], s[1][0], s[1][1], s[1][2], s[1][3]};
        parts_of<2>(x, p);
#pragma unroll
        for (int cb = 0; cb < 8; ++cb)
#pragma unroll
            for (int k = 1; k >= 0; --k)
                st.O[cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, T.v[cb]), p[k], st.O[cb], 0, 0, 0);
    }

    __device__ __forceinline__ void step(TileQ8<R>& T, RowState& st, int left, int rp, int g)
    {
        f32x4 s[2];
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            s[tb] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const bf16x8 kf = tb ? codes_bf16(T.k[i].z, T.k[i].w) : codes_bf16(T.k[i].x, T.k[i].y);
#pragma unroll
                for (int p = NP - 1; p >= 0; --p)
                    s[tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[i][p], s[tb], 0, 0, 0);
            }
        }
        // a token's step is a factor of its score, the Value's one of its weight
        float vs[2][4];
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int ii = 0; ii < 4; ++ii) {
                const uint32_t w = ii == 0 ? T.st[tb].x : ii == 1 ? T.st[tb].y : ii == 2 ? T.st[tb].z : T.st[tb].w;
                const float ks = __uint_as_float(w << 16);
                vs[tb][ii] = __uint_as_float(w & 0xffff0000u);
                s[tb][ii] *= ks;
            }
        if (left < 32) {
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                for (int ii = 0; ii < 4; ++ii) {
                    const bool in = 16 * tb + 4 * g + ii < left;
                    vs[tb][ii] = in ? vs[tb][ii] : 0.f;
                    s[tb][ii] = in ? s[tb][ii] : ROWS_NEG_INF;
                }
        }
        st.weigh(s);
        bf16x8 p[NP];
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s[e >> 2][e & 3] * vs[e >> 2][e & 3];
        parts_of<NP>(x, p);
#pragma unroll
        for (int cb = 0; cb < 8; ++cb) {
            const uint4 w = T.v[cb >> 1];
            const bf16x8 vf = cb & 1 ? codes_bf16(w.z, w.w) : codes_bf16(w.x, w.y);
#pragma unroll
            for (int k = NP - 1; k >= 0; --k)
                st.O[cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[k], st.O[cb], 0, 0, 0);
        }
    }
};

template <int FMT, int R> struct TileOf;
template <int R> struct TileOf<ROWS_BF16, R> { typedef TileBf16<R> type; };
template <int R> struct TileOf<ROWS_F32, R> { typedef TileF32<R> type; };
template <int R> struct TileOf<ROWS_Q8_BF16, R> { typedef TileQ8<R> type; };
template <int R> struct TileOf<ROWS_Q8_F32, R> { typedef TileQ8<R> type; };

// ---- full-width rows: the text segment and the drafts ---------------------------
// Row-major, so the Value operand holds channel 8 m + cb where the cache's holds 16 cb + m: lane (g, m) loads channels 8 m ..+7 of the eight
// tokens of its group (bf16: the 8 x 8 transpose of a lane's own registers, at use).
__device__ __forceinline__ uint32_t dword_of(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// What a weight of 0 does not erase: a Value that is no number.  Where a draft holds one it is left out of the product (clean()), and behind the loop the
// rows that see the draft get it added: a sum of it is it (or NaN, of both infinities).
__device__ __forceinline__ bool no_number(uint32_t fp32_bits) { return (fp32_bits & 0x7f800000u) == 0x7f800000u; }
// a bit a token of the tile, the same in all lanes, from a bit a token slot of this lane's group
__device__ __forceinline__ uint32_t tokens_of(uint32_t slots, int g)
{
    uint32_t t = (slots & 15) << (4 * g) | (slots >> 4) << (16 + 4 * g);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) t |= (uint32_t)__shfl_xor((int)t, o);
    return __builtin_amdgcn_readfirstlane(t);
}

struct PlainRowsBf16 {
    bf16x8 qf[4];
    uint4 k[2][4], v[8];
    __device__ __forceinline__ void take(const bf16_t* qrow, int g)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) qf[i] = *(const bf16x8*)(qrow + 32 * i + 8 * g);
    }
    // rows r0 ..+31 of kp, vp; those from `rows` on repeat the last
    __device__ __forceinline__ void load(const bf16_t* kp, const bf16_t* vp, int64_t stride, int r0, int rows, int g, int n)
    {
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            const bf16_t* row = kp + (int64_t)min(r0 + 16 * tb + n, rows - 1) * stride + 8 * g;
#pragma unroll
            for (int i = 0; i < 4; ++i) k[tb][i] = *(const uint4*)(row + 32 * i);
        }
#pragma unroll
        for (int jj = 0; jj < 8; ++jj) v[jj] = *(const uint4*)(vp + (int64_t)min(r0 + (jj < 4 ? 4 * g + jj : 12 + 4 * g + jj), rows - 1) * stride + 8 * n);
    }
    __device__ __forceinline__ void scores(f32x4 (&s)[2], float scale_log2)
    {
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            s[tb] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                s[tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[tb][i]), qf[i], s[tb], 0, 0, 0);
            s[tb] *= scale_log2;
        }
    }
    __device__ __forceinline__ void drop(int jj)
    {
        v[jj] = make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ bool odd() const
    {
        bool any = false;
#pragma unroll
        for (int jj = 0; jj < 8; ++jj)
#pragma unroll
            for (int w = 0; w < 4; ++w) any |= no_number(dword_of(v[jj], w)) || no_number(dword_of(v[jj], w) << 16);
        return any;
    }
    __device__ __forceinline__ uint32_t clean(int g)
    {
        uint32_t slots = 0;
#pragma unroll
        for (int jj = 0; jj < 8; ++jj) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = dword_of(v[jj], i);
                const uint32_t keep = (no_number(w[i]) ? 0u : 0xffff0000u) | (no_number(w[i] << 16) ? 0u : 0xffffu);
                slots |= keep == ~0u ? 0u : 1u << jj;
                w[i] &= keep;
            }
            v[jj] = make_uint4(w[0], w[1], w[2], w[3]);
        }
        return tokens_of(slots, g);
    }
    // channel e of eight of a draft, where it is no number
    struct Eight {
        uint4 d;
        __device__ __forceinline__ explicit Eight(const bf16_t* p) : d(*(const uint4*)p) {}
        __device__ __forceinline__ float odd(int e) const
        {
            const uint32_t w = e & 1 ? dword_of(d, e >> 1) & 0xffff0000u : dword_of(d, e >> 1) << 16;
            return no_number(w) ? __uint_as_float(w) : 0.f;
        }
    };
    __device__ __forceinline__ uint4 column(int cb) const
    {
        const uint32_t sel = (cb & 1) ? 0x07060302u : 0x05040100u;
        uint4 d;
        d.x = __builtin_amdgcn_perm(dword_of(v[1], cb >> 1), dword_of(v[0], cb >> 1), sel);
        d.y = __builtin_amdgcn_perm(dword_of(v[3], cb >> 1), dword_of(v[2], cb >> 1), sel);
        d.z = __builtin_amdgcn_perm(dword_of(v[5], cb >> 1), dword_of(v[4], cb >> 1), sel);
        d.w = __builtin_amdgcn_perm(dword_of(v[7], cb >> 1), dword_of(v[6], cb >> 1), sel);
        return d;
    }
    __device__ __forceinline__ void accumulate(const f32x4 (&s)[2], f32x4 (&O)[8]) const
    {
        bf16x8 p[2];
        const float x[8] = {s[0][0], s[0][1], s[0][2], s[0][3], s[1][0], s[1][1], s[1][2], s[1][3]};
        parts_of<2>(x, p);
#pragma unroll
        for (int cb = 0; cb < 8; ++cb) {
            const bf16x8 vf = __builtin_bit_cast(bf16x8, column(cb));
#pragma unroll
            for (int k2 = 1; k2 >= 0; --k2)
                O[cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[k2], O[cb], 0, 0, 0);
        }
    }
};

struct PlainRowsF32 {
    f32x4 qf[8], k[2][8], v[8][2];
    __device__ __forceinline__ void take(const float* qrow, int g)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) qf[i] = *(const f32x4*)(qrow + 16 * i + 4 * g);
    }
    __device__ __forceinline__ void load(const float* kp, const float* vp, int64_t stride, int r0, int rows, int g, int n)
    {
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            const float* row = kp + (int64_t)min(r0 + 16 * tb + n, rows - 1) * stride + 4 * g;
#pragma unroll
            for (int i = 0; i < 8; ++i) k[tb][i] = *(const f32x4*)(row + 16 * i);
        }
#pragma unroll
        for (int jj = 0; jj < 8; ++jj) {
            const float* row = vp + (int64_t)min(r0 + (jj < 4 ? 4 * g + jj : 12 + 4 * g + jj), rows - 1) * stride + 8 * n;
            v[jj][0] = *(const f32x4*)row;
            v[jj][1] = *(const f32x4*)(row + 4);
        }
    }
    __device__ __forceinline__ void scores(f32x4 (&s)[2], float scale_log2)
    {
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            s[tb] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    s[tb] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[tb][i][e], qf[i][e], s[tb], 0, 0, 0);
            s[tb] *= scale_log2;
        }
    }
    __device__ __forceinline__ void drop(int jj)
    {
        v[jj][0] = v[jj][1] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ bool odd() const
    {
        bool any = false;
#pragma unroll
        for (int jj = 0; jj < 8; ++jj)
#pragma unroll
            for (int c = 0; c < 8; ++c) any |= no_number(__float_as_uint(v[jj][c >> 2][c & 3]));
        return any;
    }
    __device__ __forceinline__ uint32_t clean(int g)
    {
        uint32_t slots = 0;
#pragma unroll
        for (int jj = 0; jj < 8; ++jj)
#pragma unroll
            for (int c = 0; c < 8; ++c)
                if (no_number(__float_as_uint(v[jj][c >> 2][c & 3]))) {
                    slots |= 1u << jj;
                    v[jj][c >> 2][c & 3] = 0.f;
                }
        return tokens_of(slots, g);
    }
    struct Eight {
        f32x4 a, b;
        __device__ __forceinline__ explicit Eight(const float* p) : a(*(const f32x4*)p), b(*(const f32x4*)(p + 4)) {}
        __device__ __forceinline__ float odd(int e) const
        {
            const float x = e < 4 ? a[e & 3] : b[e & 3];
            return no_number(__float_as_uint(x)) ? x : 0.f;
        }
    };
    __device__ __forceinline__ void accumulate(const f32x4 (&s)[2], f32x4 (&O)[8]) const
    {
#pragma unroll
        for (int cb = 0; cb < 8; ++cb)
#pragma unroll
            for (int jj = 0; jj < 8; ++jj)
                O[cb] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[jj][cb >> 2][cb & 3], s[jj >> 2][jj & 3], O[cb], 0, 0, 0);
    }
};

// q R_r of this work-group's rows into qt [16][R + 4], and q . delta_mu of row n: D^T[j][row] = R_r^T . q^T, column blocks
// of R_r shared by the waves.  q in bf16 is exact and R_r goes as head and remainder; in fp32 all of it is fp32.  load() asks for
// everything, make() waits for it.
template <typename T, int R> struct Rotation;
template <int R>
struct Rotation<bf16_t, R> {
    static constexpr int NW = (R + 63) / 64;
    bf16x8 qf[4];
    float x[NW][4][8];
    f32x4 dm[8];
    __device__ __forceinline__ void load(const bf16_t* qrow, const float* Ru, const float* dp, int r, int wave, int g, int n)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) qf[i] = *(const bf16x8*)(qrow + 32 * i + 8 * g);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const int j = min(16 * (wave + 4 * w) + n, r - 1);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[w][i][e] = Ru[(32 * i + 8 * g + e) * r + j];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) dm[i] = *(const f32x4_any*)(dp + 32 * (i >> 1) + 8 * g + 4 * (i & 1));
    }
    __device__ __forceinline__ void make(float* qt, float& bias, bool biased, int r, int wave, int g, int n)
    {
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const int jb = wave + 4 * w;
            if (16 * jb >= R) break;
            f32x4 acc = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[w][i][e] = 16 * jb + n < r ? x[w][i][e] : 0.f;
                bf16x8 hi, lo;
                split_bf16x8(x[w][i], hi, lo);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, qf[i], acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, qf[i], acc, 0, 0, 0);
            }
            *(f32x4*)(qt + n * (R + 4) + 16 * jb + 4 * g) = acc;
        }
        bias = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) bias = fmaf((float)qf[i][e], dm[2 * i + (e >> 2)][e & 3], bias);
        bias = biased ? groups_sum(bias) : 0.f;
    }
};
template <int R>
struct Rotation<float, R> {
    static constexpr int NW = (R + 63) / 64;
    f32x4 qf[8];
    float x[NW][8][4];
    f32x4 dm[8];
    __device__ __forceinline__ void load(const float* qrow, const float* Ru, const float* dp, int r, int wave, int g, int n)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) qf[i] = *(const f32x4*)(qrow + 16 * i + 4 * g);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const int j = min(16 * (wave + 4 * w) + n, r - 1);
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[w][i][e] = Ru[(16 * i + 4 * g + e) * r + j];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) dm[i] = *(const f32x4_any*)(dp + 16 * i + 4 * g);
    }
    __device__ __forceinline__ void make(float* qt, float& bias, bool biased, int r, int wave, int g, int n)
    {
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const int jb = wave + 4 * w;
            if (16 * jb >= R) break;
            f32x4 acc = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(16 * jb + n < r ? x[w][i][e] : 0.f, qf[i][e], acc, 0, 0, 0);
            *(f32x4*)(qt + n * (R + 4) + 16 * jb + 4 * g) = acc;
        }
        bias = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) bias = fmaf(qf[i][e], dm[i][e], bias);
        bias = biased ? groups_sum(bias) : 0.f;
    }
};

// The weight of a partial (m, l) under the maximum M of all: one that nothing weighs in has none, and a NaN stays one.
__device__ __forceinline__ float partial_weight(float m, float l, float M)
{
    return l == 0.f ? 0.f : rows_exp2(m - (M > ROWS_NEG_INF ? M : 0.f));
}

// Partials first, first + step, ... of the S of a row, by 32 lanes with four channels each: sum l_i w_i and sum acc_i w_i, w_i = 2^(m_i - M), M the maximum
// of all S.  MC (up to eight) partials' loads at once.
template <int MC>
__device__ __forceinline__ void merge_row(const float* m, const float* l, const float* acc, int S, int first, int step, int p, f32x4& num, float& sum)
{
    float M = ROWS_NEG_INF;
    for (int i = p; i < S; i += 32) M = fmaxf(M, m[i]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
    num = (f32x4){0.f, 0.f, 0.f, 0.f};
    sum = 0.f;
    for (int i0 = first; i0 < S; i0 += MC * step) {
        f32x4 av[MC];
#pragma unroll
        for (int k = 0; k < MC; ++k) av[k] = *(const f32x4*)(acc + (size_t)min(i0 + k * step, S - 1) * D + 4 * p);
        const int mine = i0 + (p & 7) * step, at = min(mine, S - 1);       // lane k of each eight: partial k's weight
        const float mv = m[at], lv = (p & 7) < MC && mine < S ? l[at] : 0.f;
        const float w = partial_weight(mv, lv, M), lw = lv * w;
#pragma unroll
        for (int k = 0; k < MC; ++k) {
            sum += __shfl(lw, k, 8);
            const float wk = __shfl(w, k, 8);
            if (i0 + k * step < S) num += av[k] * wk;
        }
    }
}

// Which stretch and rows a work-group takes.  Work-groups go to the XCDs in turn by their index: the row blocks of a stretch follow each other on one
// XCD, and read it from its L2; the stretches are dealt over all of them.
__device__ __forceinline__ bool rows_place(const RowsArgs& A, int& split, int& u, int& block)
{
    const uint32_t units = A.B * A.Hkv, xcd = blockIdx.x & 7, turn = blockIdx.x >> 3, pair = turn / A.nrb * 8 + xcd;
    block = turn % A.nrb;
    split = pair / units;
    u = pair - split * units;
    return pair < units * (A.Sv + A.Sr);
}
inline dim3 rows_grid(const RowsArgs& a)
{
    const int64_t units = (int64_t)a.B * a.Hkv, x = (units * (a.Sv + a.Sr) + 7) / 8 * 8 * a.nrb;
    return dim3(x > 0x7fffffff ? 0 : (uint32_t)x);
}

template <int FMT, int R>
__global__ __launch_bounds__(256, FMT == ROWS_F32 ? 1 : 2) void attn_rows(RowsArgs A)
{
    constexpr bool F32IO = FMT == ROWS_F32 || FMT == ROWS_Q8_F32;
    typedef typename std::conditional<F32IO, float, bf16_t>::type T;
    typedef typename std::conditional<F32IO, PlainRowsF32, PlainRowsBf16>::type Plain;
    constexpr int POOL = 16 * (R + 4) > 4 * 32 * PARK * 4 ? 16 * (R + 4) : 4 * 32 * PARK * 4;
    __shared__ __attribute__((aligned(16))) float pool[POOL];           // q R_r, and at the end the four waves' accumulators of 16 rows
    __shared__ float sm_m[4][16], sm_l[4][16];

    int split, u, block;
    if (!rows_place(A, split, u, block)) return;
    const int b = u / A.Hkv, hk = u - b * A.Hkv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, n = lane & 15;
    const int S = A.Sv + A.Sr;
    const int row0 = block * 16;                           // rows of the KV head: token by token, its G heads
    if (row0 >= A.T * A.G) return;
    const int row = min(row0 + n, A.T * A.G - 1), tok = row / A.G;      // lane (., n): its row and the row's token
    const T* qrow = (const T*)A.q + ((size_t)(b * A.T + tok) * A.Hq + hk * A.G + (row - tok * A.G)) * D;
    auto drafts_of = [&]() { return A.draft_k ? min(max(A.n_drafts ? A.n_drafts[b] : A.T, 0), A.T) : 0; };
    int live = A.T;                                        // tokens whose rows are asked for

    RowState st;                                      // (cleared only in front of the loops: its registers are the prologue's until then)
    const bool cache = split < A.Sv;
    if (cache) {
        typedef typename TileOf<FMT, R>::type Tile;
        constexpr int ES = FMT == ROWS_F32 ? 4 : 2;
        const size_t slab = slab_tokens(A.cap);
        const bool q8 = FMT >= ROWS_Q8_BF16;
        const char* Ku = (const char*)A.Kc + (q8 ? (size_t)u * (slab / 32) * q8_kblock(A.rp) : (size_t)u * slab * A.rp * ES);
        const char* Vu = (const char*)A.Vc + (size_t)u * slab * D * (q8 ? 1 : ES);
        auto share = [&](int len, int& t0, int& t1) {      // the split's tiles
            const int tiles = (len + 31) / 32;
            t0 = (int)((int64_t)tiles * split / A.Sv);
            t1 = (int)((int64_t)tiles * (split + 1) / A.Sv);
        };
        // Everything is asked for before the length is known, which is a round trip of its own: the first tile where it lies if the
        // sequence is as long as the host's bound (else it is asked for again).
        int e0, e1, t0, t1;
        share(min(A.max_len, A.cap), e0, e1);
        Rotation<T, R> rot;
        const float* Ru = A.Rr + (size_t)u * D * A.r;
        rot.load(qrow, Ru, A.dmu ? A.dmu + (size_t)u * D : Ru, A.r, wave, g, n);      // (any address that can be read, without a bias)
        Tile X, Y;
        X.load(Ku, Vu, 32 * max(min(e0 + wave, e1 - 1), 0), A.rp, lane);
        __builtin_amdgcn_sched_barrier(0);
        const int len = min(max(A.seq_len[b], 0), A.cap);
        if (A.draft_k) live = drafts_of();
        if (row0 >= live * A.G) return;
        share(len, t0, t1);
        if (t0 < t1) {
            int t = t0 + wave;                             // (a wave without a tile reads the last one, and leaves it)
            if (t0 != e0 || t1 != e1) X.load(Ku, Vu, 32 * min(t, t1 - 1), A.rp, lane);
            float bias;
            rot.make(pool, bias, A.dmu != nullptr, A.r, wave, g, n);
            lds_barrier();
            CacheRows<FMT, R> rows;
            rows.take(pool, A.scale_log2, g, n);
            st.clear();
#pragma unroll 1
            for (; t < t1; t += 8) {
                Y.load(Ku, Vu, 32 * min(t + 4, t1 - 1), A.rp, lane);
                __builtin_amdgcn_sched_barrier(0);
                rows.step(X, st, len - 32 * t, A.rp, g);
                if (t + 4 >= t1) break;
                X.load(Ku, Vu, 32 * min(t + 8, t1 - 1), A.rp, lane);
                __builtin_amdgcn_sched_barrier(0);
                rows.step(Y, st, len - 32 * (t + 4), A.rp, g);
            }
            // the bias joins only now: it is the same for all of the cache, and would cost the scores bits
            st.m += bias * A.scale_log2;
        } else {
            st.clear();
        }
    } else {
        // tiles of 32 rows: first the text's, then the drafts'
        const int drafts = drafts_of();
        if (A.draft_k) live = drafts;
        if (row0 >= live * A.G) return;
        st.clear();
        const int text = A.text_k ? min(max(A.text_len ? A.text_len[b] : A.text_max, 0), A.text_max) : 0;
        const int tt = (text + 31) / 32, tiles = tt + (drafts + 31) / 32, k = split - A.Sv;
        const int t0 = (int)((int64_t)tiles * k / A.Sr), t1 = (int)((int64_t)tiles * (k + 1) / A.Sr);
        if (t0 < t1) {
            const T* tk = (const T*)A.text_k + (int64_t)b * A.text_sb + (int64_t)hk * A.text_sh;
            const T* tv = (const T*)A.text_v + (int64_t)b * A.text_sb + (int64_t)hk * A.text_sh;
            const T* dk = (const T*)A.draft_k + (int64_t)b * A.draft_sb + (int64_t)hk * A.draft_sh;
            const T* dv = (const T*)A.draft_v + (int64_t)b * A.draft_sb + (int64_t)hk * A.draft_sh;
            Plain X;
            X.take(qrow, g);
            uint64_t odd = 0;                              // drafts whose Values hold one that is no number
#pragma unroll 1
            for (int t = t0 + wave; t < t1; t += 4) {
                const bool own = t >= tt;                  // drafts
                const int r0 = 32 * (own ? t - tt : t), rows = own ? drafts : text;
                X.load(own ? dk : tk, own ? dv : tv, own ? A.draft_st : A.text_st, r0, rows, g, n);
                f32x4 s[2];
                X.scores(s, A.scale_log2);
                uint64_t mask = ~0ull;
                if (own) {
                    mask = A.mask ? A.mask[(size_t)b * A.T + tok] : (2ull << tok) - 1;
                    mask >>= r0;
                }
                const int left = rows - r0;
                mask &= left >= 32 ? 0xffffffffull : (1ull << left) - 1;
                const uint32_t lo = (uint32_t)mask >> (4 * g);
                const uint32_t see = (lo & 15) | ((lo >> 12) & 0xf0);      // bit e: row n sees token slot e of this lane's group
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    s[e >> 2][e & 3] = (see >> e) & 1 ? s[e >> 2][e & 3] : ROWS_NEG_INF;
                    if (r0 + (e < 4 ? 4 * g + e : 12 + 4 * g + e) >= rows) X.drop(e);
                }
                st.weigh(s);
                if (own && __any(X.odd())) odd |= (uint64_t)X.clean(g) << r0;
                X.accumulate(s, st.O);
            }
#pragma unroll 1
            for (; odd; odd &= odd - 1) {                  // (accumulator (cb, ii) is channel 32 g + 8 ii + cb)
                const int j = __builtin_ctzll(odd);
#pragma unroll
                for (int ii = 0; ii < 4; ++ii) {
                    const typename Plain::Eight x(dv + (int64_t)j * A.draft_st + 32 * g + 8 * ii);
                    const uint64_t mask = A.mask ? A.mask[(size_t)b * A.T + tok] : (2ull << tok) - 1;
#pragma unroll
                    for (int cb = 0; cb < 8; ++cb) st.O[cb][ii] += (mask >> j) & 1 ? x.odd(cb) : 0.f;
                }
            }
        }
    }

    // The four waves' states become one partial (or, of a single split, the result).  Parked as quads of channels:
    // [wave][channels 4 p ..+3][row].
    f32x4* park = (f32x4*)pool + wave * 32 * PARK;
    __syncthreads();
#pragma unroll
    for (int cb = 0; cb < 8; ++cb) {
        if (cache) park[(4 * cb + g) * PARK + n] = st.O[cb];
        else {                                         // accumulator (cb, ii) is channel 32 g + 8 ii + cb there
            const int ii = cb >> 1, h = cb & 1;
            park[(8 * g + cb) * PARK + n] = (f32x4){st.O[4 * h][ii], st.O[4 * h + 1][ii], st.O[4 * h + 2][ii], st.O[4 * h + 3][ii]};
        }
    }
    const float l = groups_sum(st.l);
    if (g == 0) { sm_m[wave][n] = st.m; sm_l[wave][n] = l; }
    __syncthreads();
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int i = tid + 256 * half, row = i >> 5, p = i & 31, mine = row0 + row;
        if (mine >= live * A.G) continue;
        const float M = fmaxf(fmaxf(sm_m[0][row], sm_m[1][row]), fmaxf(sm_m[2][row], sm_m[3][row]));
        f32x4 acc = (f32x4){0.f, 0.f, 0.f, 0.f};
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float x = partial_weight(sm_m[w][row], sm_l[w][row], M);
            acc += ((const f32x4*)pool)[(w * 32 + p) * PARK + row] * x;
            sum = fmaf(sm_l[w][row], x, sum);
        }
        const int tm = mine / A.G;
        const size_t to = (size_t)(b * A.T + tm) * A.Hq + hk * A.G + (mine - tm * A.G);
        if (S == 1) {
            const float inv = 1.f / sum;
            T* o = (T*)A.out + to * D + 4 * p;
#pragma unroll
            for (int e = 0; e < 4; ++e) st_elem(o + e, sum == 0.f ? 0.f : acc[e] * inv);
        } else {
            const size_t slot = to * S + split;
            *(f32x4*)(A.ws_acc + slot * D + 4 * p) = acc;
            if (p == 0) { A.ws_m[slot] = M; A.ws_l[slot] = sum; }
        }
    }
}

template <int FMT>
static hipError_t launch_rows_fmt(const RowsArgs& a, hipStream_t st)
{
    const dim3 grid = rows_grid(a);
    if (!grid.x) return hipErrorInvalidValue;
    switch ((a.r + 31) / 32) {
        case 1: attn_rows<FMT, 32><<<grid, 256, 0, st>>>(a); break;
        case 2: attn_rows<FMT, 64><<<grid, 256, 0, st>>>(a); break;
        case 3: attn_rows<FMT, 96><<<grid, 256, 0, st>>>(a); break;
        default: attn_rows<FMT, 128><<<grid, 256, 0, st>>>(a); break;
    }
    return hipGetLastError();
}

}  // namespace rk
