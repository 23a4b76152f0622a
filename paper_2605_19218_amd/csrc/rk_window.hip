// Attention of new tokens (a prompt, or a part of one) over the text segment that holds them, with a sliding window and sinks.
//
//   token t of sequence b stands at p = len - n + t and sees row j <= p with j < sinks or p - j < window (window 0: every j <= p);
//   out = softmax(scale q . k) v over what it sees, zeros if that is nothing.
//
// The rows of a KV head are its n tokens with the G query heads of each, token by token, so that a work-group's rows share Keys, Values and nearly
// all of what they see. A wave owns 32 rows; a stage of 32 tokens goes through LDS once for the four of them. Products are turned as in attn_rows: S^T = K q^T
// leaves lane (h, n) = (lane / 32, lane % 32) with row n's scores of tokens 8 j + 4 h ..+3, which is how O^T = V^T P^T takes the weights, and all
// of a lane's accumulators are row n's: the running maximum and sum cost one exchange between the two halves of a wave.
// The tiles that a row block sees are the sinks' and those from the window's edge of its first token to its last token; only tiles on an edge are masked.
// What a masked Value holds must not reach a sum, and a weight of 0 does not erase an infinity: in masked tiles Values that are no
// numbers are left out of the product and added behind it, for the rows that see them.
#include <type_traits>
#include "rk_attn_block.hpp"

namespace rk {

namespace {

constexpr int PROMPT_ROWS = 128, PROMPT_TOKENS = 32;

// Slots of 16 bytes of a token's row in LDS lie permuted by the token, so that eight tokens' same slot, and four tokens' same pair of slots, are in other banks.
__device__ __forceinline__ int slot_of(int token, int slot) { return slot ^ (2 * (token & 3) | ((token >> 2) & 1)); }

__device__ __forceinline__ bool odd_value(uint32_t bits) { return (bits & 0x7f800000u) == 0x7f800000u; }

// What a row sees.
struct Sight {
    int p, window, sinks;        // window: 2^30 or more when there is none
    __device__ __forceinline__ bool of(int j) const { return j <= p && (j < sinks || p - j < window); }
};

struct PromptBf16 {
    typedef bf16_t T;
    static constexpr int ROW = 256, TILE = PROMPT_TOKENS * ROW;       // bytes of a token's Key (or Value) and of a stage's
    bf16x8 q[8];
    uint4 k[2], v[2];
    __device__ __forceinline__ void take(const T* row, int h)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = *(const bf16x8*)(row + 16 * i + 8 * h);
    }
    __device__ __forceinline__ void load(const T* kp, const T* vp, int64_t st, int j0, int last, int tid)
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t at = (int64_t)min(j0 + 16 * i + (tid >> 4), last) * st + 8 * (tid & 15);
            k[i] = *(const uint4*)(kp + at);
            v[i] = *(const uint4*)(vp + at);
        }
    }
    __device__ __forceinline__ void store(char* kb, char* vb, int tid) const
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int m = 16 * i + (tid >> 4), at = m * ROW + 16 * slot_of(m, tid & 15);
            *(uint4*)(kb + at) = k[i];
            *(uint4*)(vb + at) = v[i];
        }
    }
    __device__ __forceinline__ void scores(const char* kb, f32x16& s, int h, int n) const
    {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bf16x8 a = *(const bf16x8*)(kb + n * ROW + 16 * slot_of(n, 2 * i + h));
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[i], s, 0, 0, 0);
        }
    }
    // CLEAN: Values that are no numbers count as 0; the answer: whether there are any
    template <bool CLEAN>
    __device__ __forceinline__ bool product(const char* vb, const f32x16& w, f32x16 (&O)[4], int lane) const
    {
        const int h = lane >> 5, nh = (lane >> 4) & 1, i = lane & 15;
        bool odd = false;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            uint32_t p[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = __builtin_bit_cast(uint32_t, (bf16x2){(__bf16)w[8 * t + 2 * e], (__bf16)w[8 * t + 2 * e + 1]});
            const bf16x8 b = __builtin_bit_cast(bf16x8, make_uint4(p[0], p[1], p[2], p[3]));
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t a[4];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int m = 16 * t + 8 * x + 4 * h + (i >> 2);
                    typedef __attribute__((address_space(3))) s16x4* Lds;
                    const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(vb + m * ROW + 16 * slot_of(m, 4 * c + 2 * nh + ((i & 3) >> 1)) + 8 * (i & 1)));
                    const uint2 z = __builtin_bit_cast(uint2, y);
                    a[2 * x] = z.x;
                    a[2 * x + 1] = z.y;
                }
                if constexpr (CLEAN) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t keep = (odd_value(a[e]) ? 0u : 0xffff0000u) | (odd_value(a[e] << 16) ? 0u : 0xffffu);
                        odd |= keep != ~0u;
                        a[e] &= keep;
                    }
                }
                O[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, make_uint4(a[0], a[1], a[2], a[3])), b, O[c], 0, 0, 0);
            }
        }
        return odd;
    }
    // channel of accumulator i of block c
    static __device__ __forceinline__ int channel(int c, int i, int h) { return 32 * c + 8 * (i >> 2) + 4 * h + (i & 3); }
    static __device__ __forceinline__ float value(const char* vb, int m, int ch)
    {
        return bf16_to_f32(*(const bf16_t*)(vb + m * ROW + 16 * slot_of(m, ch >> 3) + 2 * (ch & 7)));
    }
};

struct PromptF32 {
    typedef float T;
    static constexpr int ROW = 512, TILE = PROMPT_TOKENS * ROW;
    f32x4 q[16];
    uint4 k[4], v[4];
    __device__ __forceinline__ void take(const T* row, int h)
    {
#pragma unroll
        for (int i = 0; i < 16; ++i) q[i] = *(const f32x4*)(row + 8 * i + 4 * h);
    }
    __device__ __forceinline__ void load(const T* kp, const T* vp, int64_t st, int j0, int last, int tid)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t at = (int64_t)min(j0 + 8 * i + (tid >> 5), last) * st + 4 * (tid & 31);
            k[i] = *(const uint4*)(kp + at);
            v[i] = *(const uint4*)(vp + at);
        }
    }
    __device__ __forceinline__ void store(char* kb, char* vb, int tid) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int m = 8 * i + (tid >> 5), at = m * ROW + 16 * slot_of(m, tid & 31);
            *(uint4*)(kb + at) = k[i];
            *(uint4*)(vb + at) = v[i];
        }
    }
    __device__ __forceinline__ void scores(const char* kb, f32x16& s, int h, int n) const
    {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const f32x4 a = *(const f32x4*)(kb + n * ROW + 16 * slot_of(n, 2 * i + h));
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], q[i][e], s, 0, 0, 0);
        }
    }
    template <bool CLEAN>
    __device__ __forceinline__ bool product(const char* vb, const f32x16& w, f32x16 (&O)[4], int lane) const
    {
        const int h = lane >> 5, n = lane & 31;
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int m = 8 * (i >> 2) + 4 * h + (i & 3);
            f32x4 a = *(const f32x4*)(vb + m * ROW + 16 * slot_of(m, n));
            if constexpr (CLEAN) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (odd_value(__float_as_uint(a[c]))) {
                        odd = true;
                        a[c] = 0.f;
                    }
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) O[c] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[c], w[i], O[c], 0, 0, 0);
        }
        return odd;
    }
    static __device__ __forceinline__ int channel(int c, int i, int h) { return 4 * (8 * (i >> 2) + 4 * h + (i & 3)) + c; }
    static __device__ __forceinline__ float value(const char* vb, int m, int ch)
    {
        return *(const float*)(vb + m * ROW + 16 * slot_of(m, ch >> 2) + 4 * (ch & 3));
    }
};

template <typename P>
__global__ __launch_bounds__(256, 2) void attn_prompt(PrefillArgs A)
{
    typedef typename P::T T;
    __shared__ __attribute__((aligned(16))) char lds[4 * P::TILE];    // two stages of Keys and Values

    // blocks with more to see first
    const uint32_t u = blockIdx.x / (uint32_t)(A.blocks * A.S), rest = blockIdx.x - u * (uint32_t)(A.blocks * A.S);
    const int block = A.blocks - 1 - (int)(rest / A.S), split = rest % A.S;
    const int b = u / A.Hkv, hk = u - b * A.Hkv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, n = lane & 31;

    const int len = min(max(A.len ? A.len[b] : A.max_len, 0), A.max_len), fresh = min(max(A.n_dev ? A.n_dev[b] : A.n, 0), A.n);
    const int first = len - fresh;                         // the first new token's position
    const int64_t rows = (int64_t)fresh * A.G, row0 = (int64_t)block * PROMPT_ROWS;
    if (row0 >= rows) return;
    auto token = [&](int64_t r) { return (int)((r < rows ? r : rows - 1) / A.G); };
    const int64_t row = row0 + 32 * wave + n, mine = row < rows ? row : rows - 1;
    const int tok = token(row), head = hk * A.G + (int)(mine - (int64_t)tok * A.G);
    const int window = A.window > 0 ? A.window : 0x7fffffff;
    const Sight sight{first + tok, window, A.sinks};

    P tile;
    tile.take((const T*)A.q + (int64_t)b * A.q_sb + (int64_t)head * A.q_sh + (int64_t)tok * A.q_st, h);

    // tiles that any row of the block sees: `few` of the sinks, and from `from` on
    const int p_hi = first + token(row0 + PROMPT_ROWS - 1), p_lo = max(first + token(row0), 0);
    int few = 0, from = 0, tiles = 0;
    if (p_hi >= 0) {
        const int lo = A.window > 0 ? max(p_lo - A.window + 1, 0) : 0;
        from = lo / PROMPT_TOKENS;
        few = min((min(A.sinks, lo) + PROMPT_TOKENS - 1) / PROMPT_TOKENS, from);
        tiles = few + p_hi / PROMPT_TOKENS - from + 1;
    }
    const int i0 = (int)((int64_t)tiles * split / A.S), i1 = (int)((int64_t)tiles * (split + 1) / A.S);
    auto start = [&](int i) { return PROMPT_TOKENS * (i < few ? i : i - few + from); };
    const int w_lo = first + token(row0 + 32 * wave), w_hi = first + token(row0 + 32 * wave + 31);     // positions of the wave's rows

    const T* kp = (const T*)A.k + (int64_t)b * A.sb + (int64_t)hk * A.sh;
    const T* vp = (const T*)A.v + (int64_t)b * A.sb + (int64_t)hk * A.sh;
    float m = ROWS_NEG_INF, l = 0.f;                       // log2 domain; l: this lane's tokens only, until the end
    f32x16 O[4];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[c][i] = 0.f;

    if (i0 < i1) {
        tile.load(kp, vp, A.st, start(i0), len - 1, tid);
        tile.store(lds, lds + P::TILE, tid);
    }
    __syncthreads();
    for (int i = i0; i < i1; ++i) {
        const char* kb = lds + ((i - i0) & 1) * 2 * P::TILE;
        char* next = lds + ((i - i0 + 1) & 1) * 2 * P::TILE;
        if (i + 1 < i1) tile.load(kp, vp, A.st, start(i + 1), len - 1, tid);
        const int j0 = start(i), j1 = j0 + PROMPT_TOKENS - 1;
        const bool none = j0 > w_hi || (j0 >= A.sinks && w_lo - j1 >= window);
        if (!none) {
            const bool all = j1 <= w_lo && (j1 < A.sinks || w_hi - j0 < window);
            f32x16 s;
            tile.scores(kb, s, h, n);
            float mt = ROWS_NEG_INF;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[e] *= A.scale_log2;
                if (!all) s[e] = sight.of(j0 + 8 * (e >> 2) + 4 * h + (e & 3)) ? s[e] : ROWS_NEG_INF;
                mt = fmaxf(mt, s[e]);
            }
            mt = halves_max(mt);
            // (the maximum moves when it is behind by 2^8, as in attn_rows; a sum that holds an infinity may not meet a factor of 0)
            if (__any(mt > m + 8.f)) {
                const float m_new = fmaxf(m, mt), alpha = m > ROWS_NEG_INF ? fmaxf(rows_exp2(m - m_new), 0x1p-126f) : 0.f;
                l *= alpha;
                if (m > ROWS_NEG_INF) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) O[c] *= alpha;
                }
                m = m_new;
            }
            const float ref = m > ROWS_NEG_INF ? m : 0.f;
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[e] = rows_exp2(s[e] - ref);
                sum += s[e];
            }
            l += sum;
            if (all) {
                tile.template product<false>(kb + P::TILE, s, O, lane);
            } else if (__any(tile.template product<true>(kb + P::TILE, s, O, lane))) {
#pragma unroll 1
                for (int j = 0; j < PROMPT_TOKENS; ++j) {
                    const bool seen = sight.of(j0 + j);
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const float x = P::value(kb + P::TILE, j, P::channel(c, e, h));
                            O[c][e] += seen && odd_value(__float_as_uint(x)) ? x : 0.f;
                        }
                }
            }
        }
        if (i + 1 < i1) tile.store(next, next + P::TILE, tid);
        __syncthreads();
    }

    l = halves_sum(l);
    if (row >= rows) return;
    if (A.S == 1) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        T* o = (T*)A.out + (int64_t)b * A.o_sb + (int64_t)head * A.o_sh + (int64_t)tok * A.o_st;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int e = 0; e < 16; ++e) st_elem(o + P::channel(c, e, h), l == 0.f ? 0.f : O[c][e] * inv);
    } else {
        const size_t slot = ((size_t)u * A.n * A.G + row) * A.S + split;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int e = 0; e < 16; ++e) A.ws_acc[slot * D + P::channel(c, e, h)] = O[c][e];
        if (h == 0) { A.ws_m[slot] = m; A.ws_l[slot] = l; }
    }
}


// ---- bf16, many rows: 64 rows a wave ------------------------------------------------
// A stage of 64 tokens, three of them in LDS: loads go there without passing through registers, two stages ahead. Rows in two groups of 32, so that a Key or Value
// read from LDS feeds two products.
// In LDS a token's row is its 256 bytes, slots permuted as slot_of() says: what a load leaves is lane by lane, so it is the lanes' addresses that are permuted.
constexpr int WIDE_ROWS = 256, WIDE_TOKENS = 64, WIDE_ROW = 256, WIDE_VALUES = WIDE_TOKENS * WIDE_ROW, WIDE_STAGE = 2 * WIDE_VALUES;
constexpr int WIDE_LDS = 3 * WIDE_STAGE;      // and a flag

__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p; }
// 16 bytes a lane from `from` to LDS at `to` (of the wave) + 16 lane. (Not the builtin: behind it every read of LDS waits for all loads.) What is asked for
// is there after stage_wait().
__device__ __forceinline__ void load_to_lds(const void* from, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(to), "v"(from) : "m0", "memory");
}
// this wave's loads but the last N are there
template <int N>
__device__ __forceinline__ void stage_wait() { asm volatile("s_waitcnt vmcnt(%0)" : : "i"(N) : "memory"); }

struct WideRows {
    bf16x8 q[2][8];
    f32x16 O[2][4];
    float m[2], l[2];
    Sight sight[2];
    float c;                     // scale, log2 domain

    // Accumulators and queries stay in the half of the register file that only matrix instructions read and write.
    __device__ __forceinline__ void hold()
    {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
#pragma unroll
            for (int b = 0; b < 4; ++b) asm volatile("" : "+a"(O[g][b]));
#pragma unroll
            for (int i = 0; i < 8; ++i) asm volatile("" : "+a"(q[g][i]));
        }
    }
    // S^T of a tile's 32 tokens; ka: this lane's places of pieces 0..3 of the tile's first token
    __device__ __forceinline__ void scores(const char* lds, const int (&ka)[4], int at, f32x16 (&s)[2]) const
    {
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[g][i] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bf16x8 a = *(const bf16x8*)(lds + ka[i & 3] + at + 128 * (i >> 2));
#pragma unroll
            for (int g = 0; g < 2; ++g) s[g] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[g][i], s[g], 0, 0, 0);
        }
    }
    // the running maxima, after the tile's own
    __device__ __forceinline__ void follow(const f32x16 (&s)[2])
    {
        float mt[2];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            mt[g] = s[g][0];
#pragma unroll
            for (int i = 1; i < 16; ++i) mt[g] = fmaxf(mt[g], s[g][i]);
            mt[g] = halves_max(mt[g]) * c;
        }
        if (__any(mt[0] > m[0] + 8.f || mt[1] > m[1] + 8.f)) {
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const float m_new = fmaxf(m[g], mt[g]), alpha = m[g] > ROWS_NEG_INF ? rows_exp2(m[g] - m_new) : 1.f;
                l[g] *= alpha;
#pragma unroll
                for (int b = 0; b < 4; ++b) O[g][b] *= alpha;
                m[g] = m_new;
            }
        }
    }
    __device__ __forceinline__ void weigh(f32x16& s, int g, bf16x8 (&p)[2])
    {
        const float ref = m[g] > ROWS_NEG_INF ? m[g] : 0.f;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[i] = rows_exp2(fmaf(s[i], c, -ref));
            sum += s[i];
        }
        l[g] += sum;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = __builtin_bit_cast(uint32_t, (bf16x2){(__bf16)s[8 * t + 2 * e], (__bf16)s[8 * t + 2 * e + 1]});
            p[t] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
        }
    }
    // channels 32 b + lane % 32 of the tile's tokens 16 t + (4 h ..+3, 8 + 4 h ..+3); va: this lane's places of blocks 0 and 1
    static __device__ __forceinline__ bf16x8 values(const char* lds, const int (&va)[2], int at, int t, int b)
    {
        uint2 a[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            typedef __attribute__((address_space(3))) s16x4* Lds;
            a[x] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(lds + va[b & 1] + at + (16 * t + 8 * x) * WIDE_ROW + 128 * (b >> 1))));
        }
        return __builtin_bit_cast(bf16x8, make_uint4(a[0].x, a[0].y, a[1].x, a[1].y));
    }
    // a tile on an edge: what a row does not see has no score
    __device__ __forceinline__ void hide(f32x16 (&s)[2], int j0, int h) const
    {
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[g][i] = sight[g].of(j0 + 8 * (i >> 2) + 4 * h + (i & 3)) ? s[g][i] : ROWS_NEG_INF;
    }
    // One tile (Values at vt): scores s of it into O; the scores of the next tile (Keys at kt) into `next`.
    __device__ __forceinline__ void tile(f32x16 (&s)[2], f32x16 (&next)[2], const char* lds, const int (&ka)[4], int kt, const int (&va)[2], int vt)
    {
        bf16x8 p[2][2];
        follow(s);
        hold();
        scores(lds, ka, kt, next);
        weigh(s[0], 0, p[0]);
        weigh(s[1], 1, p[1]);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const bf16x8 a = values(lds, va, vt, t, b);
#pragma unroll
                for (int g = 0; g < 2; ++g) O[g][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, p[g][t], O[g][b], 0, 0, 0);
            }
    }
};

__global__ __launch_bounds__(256, 1) void attn_prompt_wide(PrefillArgs A)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t u = blockIdx.x / (uint32_t)(A.blocks * A.S), rest = blockIdx.x - u * (uint32_t)(A.blocks * A.S);
    const int block = A.blocks - 1 - (int)(rest / A.S), split = rest % A.S;
    const int b = u / A.Hkv, hk = u - b * A.Hkv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, n = lane & 31;

    const int len = min(max(A.len ? A.len[b] : A.max_len, 0), A.max_len), fresh = min(max(A.n_dev ? A.n_dev[b] : A.n, 0), A.n);
    const int first = len - fresh;
    const int rows = fresh * A.G, row0 = block * WIDE_ROWS;
    if (row0 >= rows) return;
    auto token = [&](int r) { return (int)((uint32_t)min(r, rows - 1) / (uint32_t)A.G); };
    const int window = A.window > 0 ? A.window : 0x7fffffff;

    WideRows W;
    W.c = A.scale_log2;
    int tok[2], head[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        const int mine = min(row0 + 64 * wave + 32 * g + n, rows - 1);
        tok[g] = token(mine);
        head[g] = hk * A.G + mine - tok[g] * A.G;
        W.sight[g] = Sight{first + tok[g], window, A.sinks};
        W.m[g] = ROWS_NEG_INF;
        W.l[g] = 0.f;
        const bf16_t* q = (const bf16_t*)A.q + (int64_t)b * A.q_sb + (int64_t)head[g] * A.q_sh + (int64_t)tok[g] * A.q_st;
#pragma unroll
        for (int i = 0; i < 8; ++i) W.q[g][i] = *(const bf16x8*)(q + 16 * i + 8 * h);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) W.O[g][c][i] = 0.f;
    }

    // stages that any row of the block sees: `few` of the sinks, and from `from` on
    const int p_hi = first + token(row0 + WIDE_ROWS - 1), p_lo = max(first + token(row0), 0);
    int few = 0, from = 0, stages = 0;
    if (p_hi >= 0) {
        const int lo = A.window > 0 ? max(p_lo - A.window + 1, 0) : 0;
        from = lo / WIDE_TOKENS;
        few = min((min(A.sinks, lo) + WIDE_TOKENS - 1) / WIDE_TOKENS, from);
        stages = few + p_hi / WIDE_TOKENS - from + 1;
    }
    const int i0 = (int)((int64_t)stages * split / A.S), i1 = (int)((int64_t)stages * (split + 1) / A.S);
    auto start = [&](int i) { return WIDE_TOKENS * (i < few ? i : i - few + from); };
    const int w_lo = first + token(row0 + 64 * wave), w_hi = first + token(row0 + 64 * wave + 63);      // positions of the wave's rows

    const bf16_t* kp = (const bf16_t*)A.k + (int64_t)b * A.sb + (int64_t)hk * A.sh;
    const bf16_t* vp = (const bf16_t*)A.v + (int64_t)b * A.sb + (int64_t)hk * A.sh;
    int* odd = (int*)(lds + WIDE_LDS);
    if (i0 < i1) {
        // rows 16 wave + 4 i + lane / 16 of a stage, i < 4: their 16-byte pieces, in the order that slot_of() undoes
        const uint32_t base = __builtin_amdgcn_readfirstlane(lds_address(lds)) + 16 * WIDE_ROW * wave;
        auto fetch = [&](int i, int buf) {
            const int j = start(i) + 16 * wave + (lane >> 4);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int64_t at = (int64_t)min(j + 4 * x, len - 1) * A.st + 8 * slot_of(4 * x + (lane >> 4), lane & 15);
                load_to_lds(kp + at, base + buf + 4 * WIDE_ROW * x);
                load_to_lds(vp + at, base + buf + WIDE_VALUES + 4 * WIDE_ROW * x);
            }
        };
        // Stages that not all of the block's rows see whole: what a masked Value holds may not meet a weight of 0, so what is no number becomes 0 there.
        auto edge = [&](int j) { return !(j + WIDE_TOKENS - 1 <= p_lo && (j + WIDE_TOKENS - 1 < A.sinks || p_hi - j < window)) || first + token(row0) < 0; };
        auto clean = [&](char* buf) {
#pragma unroll 1
            for (int x = 0; x < 4; ++x) {
                uint4* at = (uint4*)(buf + WIDE_VALUES + 4096 * x + 16 * tid);
                const uint4 d = *at;
                uint32_t w[4] = {d.x, d.y, d.z, d.w};
                bool any = false;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t keep = (odd_value(w[e]) ? 0u : 0xffff0000u) | (odd_value(w[e] << 16) ? 0u : 0xffffu);
                    any |= keep != ~0u;
                    w[e] &= keep;
                }
                if (any) {
                    *at = make_uint4(w[0], w[1], w[2], w[3]);
                    *odd = 1;
                }
            }
        };
        fetch(i0, 0);
        fetch(min(i0 + 1, i1 - 1), WIDE_STAGE);
        if (tid == 0) *odd = 0;
        stage_wait<8>();
        lds_barrier();
        if (edge(start(i0))) {
            clean(lds);
            lds_barrier();
        }
        int ka[4], va[2];
#pragma unroll
        for (int i = 0; i < 4; ++i) ka[i] = n * WIDE_ROW + 16 * slot_of(n, 2 * i + h);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = 4 * h + ((lane & 15) >> 2);
            va[i] = r * WIDE_ROW + 16 * slot_of(r, 4 * i + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + 8 * (lane & 1);
        }
        f32x16 s0[2], s1[2];
        W.scores(lds, ka, 0, s0);
        int now = 0, next = WIDE_STAGE, behind = 2 * WIDE_STAGE;
#pragma unroll 1
        for (int i = i0; i < i1; ++i) {
            W.hold();
            const int j0 = start(i);
            fetch(min(i + 2, i1 - 1), behind);
            auto inside = [&](int j) { return j + 31 <= w_lo && (j + 31 < A.sinks || w_hi - j < window); };
            if (!inside(j0)) W.hide(s0, j0, h);
            W.tile(s0, s1, lds, ka, now + 32 * WIDE_ROW, va, now + WIDE_VALUES);
            // the next stage's loads are all but the last eight, which are the ones behind it
            stage_wait<8>();
            lds_barrier();
            if (i + 1 < i1 && edge(start(i + 1))) {
                clean(lds + next);
                lds_barrier();
            }
            if (!inside(j0 + 32)) W.hide(s1, j0 + 32, h);
            W.tile(s1, s0, lds, ka, next, va, now + WIDE_VALUES + 32 * WIDE_ROW);
            lds_barrier();
            const int t = now;
            now = next;
            next = behind;
            behind = t;
        }
        stage_wait<0>();             // (what was asked for twice, at the end)
        // The Values that were left out join the rows that see them: a sum of one is it, or NaN.
        if (*odd) {
#pragma unroll 1
            for (int i = i0; i < i1; ++i) {
                const int j0 = start(i);
                if (!edge(j0)) continue;
#pragma unroll 1
                for (int j = j0; j < min(j0 + WIDE_TOKENS, len); ++j)
#pragma unroll
                    for (int b = 0; b < 4; ++b)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const uint2 d = *(const uint2*)(vp + (int64_t)j * A.st + 32 * b + 8 * q + 4 * h);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const uint32_t w = e < 2 ? d.x : d.y, v = e & 1 ? w & 0xffff0000u : w << 16;
#pragma unroll
                                for (int g = 0; g < 2; ++g) W.O[g][b][4 * q + e] += odd_value(v) && W.sight[g].of(j) ? __uint_as_float(v) : 0.f;
                            }
                        }
            }
        }
    }

#pragma unroll
    for (int g = 0; g < 2; ++g) {
        const float l = halves_sum(W.l[g]);
        const int row = row0 + 64 * wave + 32 * g + n;
        if (row >= rows) continue;
        if (A.S == 1) {
            const float inv = l == 0.f ? 0.f : 1.f / l;
            bf16_t* o = (bf16_t*)A.out + (int64_t)b * A.o_sb + (int64_t)head[g] * A.o_sh + (int64_t)tok[g] * A.o_st;
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = l == 0.f ? 0.f : W.O[g][c][4 * q + e] * inv;
                    *(uint2*)(o + 32 * c + 8 * q + 4 * h) =
                        make_uint2(__builtin_bit_cast(uint32_t, (bf16x2){(__bf16)x[0], (__bf16)x[1]}), __builtin_bit_cast(uint32_t, (bf16x2){(__bf16)x[2], (__bf16)x[3]}));
                }
        } else {
            const size_t slot = ((size_t)u * A.n * A.G + row) * A.S + split;
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *(f32x4*)(A.ws_acc + slot * D + 32 * c + 8 * q + 4 * h) = (f32x4){W.O[g][c][4 * q], W.O[g][c][4 * q + 1], W.O[g][c][4 * q + 2], W.O[g][c][4 * q + 3]};
            if (h == 0) { A.ws_m[slot] = W.m[g]; A.ws_l[slot] = l; }
        }
    }
}

// The fold of the splits' partials: 32 lanes a row, four channels each (see rows_merge).
template <typename T>
__global__ __launch_bounds__(256) void prompt_merge(PrefillArgs A)
{
    const int p = threadIdx.x & 31;
    const int64_t per = (int64_t)A.n * A.G, at = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), u = at / per, row = at - u * per;
    const int b = (int)(u / A.Hkv), hk = (int)(u - (int64_t)b * A.Hkv);
    if (b >= A.B) return;
    const int fresh = min(max(A.n_dev ? A.n_dev[b] : A.n, 0), A.n);
    if (row >= (int64_t)fresh * A.G) return;
    f32x4 num;
    float sum;
    merge_row<4>(A.ws_m + at * A.S, A.ws_l + at * A.S, A.ws_acc + at * A.S * D, A.S, 0, 1, p, num, sum);
    const int tok = (int)(row / A.G), head = hk * A.G + (int)(row - (int64_t)tok * A.G);
    const float inv = 1.f / sum;
    T* o = (T*)A.out + (int64_t)b * A.o_sb + (int64_t)head * A.o_sh + (int64_t)tok * A.o_st + 4 * p;
#pragma unroll
    for (int e = 0; e < 4; ++e) st_elem(o + e, sum == 0.f ? 0.f : num[e] * inv);
}

}  // namespace

int prefill_block_rows(int dtype) { return dtype == 0 ? PROMPT_ROWS : WIDE_ROWS; }

hipError_t launch_prefill(int dtype, const PrefillArgs& a, hipStream_t st)
{
    const int64_t units = (int64_t)a.B * a.Hkv, groups = units * a.blocks * a.S;
    if (groups > 0x7fffffff || (units * a.n * a.G + 7) / 8 > 0x7fffffff) return hipErrorInvalidValue;
    if (dtype == 0) attn_prompt<PromptF32><<<(uint32_t)groups, 256, 0, st>>>(a);
    else {
        const hipError_t e = allow_dynamic_lds((const void*)attn_prompt_wide, WIDE_LDS + 16);
        if (e != hipSuccess) return e;
        attn_prompt_wide<<<(uint32_t)groups, 256, WIDE_LDS + 16, st>>>(a);
    }
    if (a.S > 1) {
        const uint32_t g = (uint32_t)((units * a.n * a.G + 7) / 8);
        if (dtype == 0) prompt_merge<float><<<g, 256, 0, st>>>(a);
        else prompt_merge<bf16_t><<<g, 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

}  // namespace rk
