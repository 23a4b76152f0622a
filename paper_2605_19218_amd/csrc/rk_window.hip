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

// Which rows and splits a work-group takes: the last blocks of all KV heads first, which see most, so that the short ones fill the gaps at the end; a head's
// work-groups go to the same XCDs, which read its Keys and Values from their L2.
__device__ __forceinline__ void prompt_place(const PrefillArgs& A, int& block, int& split, int& u)
{
    const uint32_t units = A.B * A.Hkv, rank = blockIdx.x / units;
    u = blockIdx.x - rank * units;
    block = A.blocks - 1 - (int)(rank / A.S);
    split = rank % A.S;
}

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

    int block, split, u;
    prompt_place(A, block, split, u);
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
// A stage of 64 tokens, four of them in LDS: loads go there without passing through registers, two stages ahead, one barrier a stage. Rows in two groups of 32, so that a Key or Value
// read from LDS feeds two products.
// In LDS a token's row is its 256 bytes, slots permuted as slot_of() says: what a load leaves is lane by lane, so it is the lanes' addresses that are permuted.
constexpr int WIDE_ROWS = 256, WIDE_TOKENS = 64, WIDE_ROW = 256, WIDE_VALUES = WIDE_TOKENS * WIDE_ROW, WIDE_STAGE = 2 * WIDE_VALUES;
constexpr int WIDE_LDS = 4 * WIDE_STAGE;      // and a flag

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
    // a tile's 32 Keys; ka: this lane's places of pieces 0..3 of the tile's first token
    static __device__ __forceinline__ void keys(const char* lds, const int (&ka)[4], int at, bf16x8 (&k)[8])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) k[i] = *(const bf16x8*)(lds + ka[i & 3] + at + 128 * (i >> 2));
    }
    // S^T of them
    __device__ __forceinline__ void scores(const bf16x8 (&k)[8], f32x16 (&s)[2]) const
    {
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[g][i] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int g = 0; g < 2; ++g) s[g] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[i], q[g][i], s[g], 0, 0, 0);
    }
    // the largest score of each group's row among this lane's tokens
    static __device__ __forceinline__ float most(const f32x16& s)
    {
        float a = fmaxf(s[0], s[1]), b = fmaxf(s[2], s[3]);
#pragma unroll
        for (int i = 4; i < 16; i += 4) {
            a = fmaxf(fmaxf(a, s[i]), s[i + 1]);
            b = fmaxf(fmaxf(b, s[i + 2]), s[i + 3]);
        }
        return fmaxf(a, b);
    }
    // the running maxima, after a tile's
    __device__ __forceinline__ void follow(const float (&top)[2])
    {
        float mt[2];
#pragma unroll
        for (int g = 0; g < 2; ++g) mt[g] = halves_max(top[g]) * c;
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
    // half x of channels 32 b + lane % 32 of the tile's tokens 16 t + (4 h ..+3, 8 + 4 h ..+3); va: this lane's places of blocks 0 and 1
    static __device__ __forceinline__ s16x4 values(const char* lds, const int (&va)[2], int at, int t, int b, int x)
    {
        typedef __attribute__((address_space(3))) s16x4* Lds;
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(lds + va[b & 1] + at + (16 * t + 8 * x) * WIDE_ROW + 128 * (b >> 1)));
    }
    // a tile on an edge: what a row does not see has no score
    __device__ __forceinline__ void hide(f32x16 (&s)[2], float (&top)[2], int j0, int h) const
    {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[g][i] = sight[g].of(j0 + 8 * (i >> 2) + 4 * h + (i & 3)) ? s[g][i] : ROWS_NEG_INF;
            top[g] = most(s[g]);
        }
    }
    // Scores belong into the other half of the register file, where the vector instructions are that they are for; the compiler would have them beside the accumulators and
    // copy them (64 instructions a tile). The vector instructions that read them come 300 cycles behind, matrix instructions of the same group two behind.
    static __device__ __forceinline__ void score(f32x16& s, const bf16x8& k, const bf16x8& q, bool begin)
    {
        if (begin) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(k), "a"(q));
        else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(k), "a"(q));
    }
    // One tile (Values at vt): scores s of it, whose largest are `top`, into O; the scores of the next tile (Keys k) into `next`, its largest into `top`; the Keys of
    // the one behind it (at kt) into k.
    // A wave has its SIMD for itself, so what runs beside the matrix instructions is what stands between them: 32 of 32 cycles, of which the first 24 have beside them
    // the weights, 16 pairs of 52 cycles (the exponentials 16 each), two in three instructions' time, and the last eight the maxima; LDS is read one piece a step.
    __device__ __forceinline__ void tile(f32x16 (&s)[2], f32x16 (&next)[2], float (&top)[2], bf16x8 (&k)[8], const char* lds, const int (&ka)[4], int kt,
                                         const int (&va)[2], int vt)
    {
        follow(top);
        hold();
        const float ref[2] = {m[0] > ROWS_NEG_INF ? m[0] : 0.f, m[1] > ROWS_NEG_INF ? m[1] : 0.f};
        float sum[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
        uint32_t p[2][8];
        s16x4 v[2][4][2];
        __builtin_amdgcn_sched_barrier(0);
        auto weigh = [&](int pair) {             // of rows' group pair / 8, tokens 2 (pair % 8) and the next
            const int g = pair >> 3, e = 2 * (pair & 7);
            s[g][e] = rows_exp2(fmaf(s[g][e], c, -ref[g]));
            s[g][e + 1] = rows_exp2(fmaf(s[g][e + 1], c, -ref[g]));
        };
        auto pack = [&](int pair) {
            const int g = pair >> 3, e = 2 * (pair & 7);
            sum[g][0] += s[g][e];
            sum[g][1] += s[g][e + 1];
            p[g][pair & 7] = __builtin_bit_cast(uint32_t, (bf16x2){(__bf16)s[g][e], (__bf16)s[g][e + 1]});
        };
#pragma unroll
        for (int x = 0; x < 32; ++x) {
            if (x < 16) {
                const int g = x & 1, i = x >> 1;
                score(next[g], k[i], q[g][i], i == 0);
                v[x >> 3][(x >> 1) & 3][x & 1] = values(lds, va, vt, x >> 3, (x >> 1) & 3, x & 1);
            } else {
                const int g = (x >> 3) & 1, t = (x >> 2) & 1, b = x & 3;
                const uint2 v0 = __builtin_bit_cast(uint2, v[t][b][0]), v1 = __builtin_bit_cast(uint2, v[t][b][1]);
                O[g][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, make_uint4(v0.x, v0.y, v1.x, v1.y)),
                                                                  __builtin_bit_cast(bf16x8, make_uint4(p[g][4 * t], p[g][4 * t + 1], p[g][4 * t + 2], p[g][4 * t + 3])),
                                                                  O[g][b], 0, 0, 0);
                if (x >= 24) k[x - 24] = *(const bf16x8*)(lds + ka[x & 3] + kt + 128 * ((x - 24) >> 2));
            }
            // pairs 2 y and 2 y + 1 in steps 3 y ..+2, each one's sums and rounding a step behind
            if (x < 24 && x % 3 < 2) weigh(2 * (x / 3) + x % 3);
            if (x < 25 && x % 3 == 1) pack(2 * (x / 3));
            if (x < 25 && x % 3 == 2) pack(2 * (x / 3) + 1);
            if (x == 26) top[0] = most(next[0]);
            if (x == 28) top[1] = most(next[1]);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int g = 0; g < 2; ++g) l[g] += sum[g][0] + sum[g][1];
    }
};

__global__ __launch_bounds__(256, 1) void attn_prompt_wide(PrefillArgs A)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int block, split, u;
    prompt_place(A, block, split, u);
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
#pragma unroll
        for (int i = 0; i < 3; ++i) fetch(min(i0 + i, i1 - 1), i * WIDE_STAGE);
        if (tid == 0) *odd = 0;
        stage_wait<16>();
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
        bf16x8 k[8];
        float top[2];
        WideRows::keys(lds, ka, 0, k);
        W.scores(k, s0);
        WideRows::keys(lds, ka, 32 * WIDE_ROW, k);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            asm volatile("" : "+v"(s0[g]));
            top[g] = WideRows::most(s0[g]);
        }
        int now = 0;
#pragma unroll 1
        for (int i = i0; i < i1; ++i) {
            W.hold();
            const int j0 = start(i), next = (now + WIDE_STAGE) & (4 * WIDE_STAGE - 1);
            // The next stage's loads are all but the last eight.  Behind the barrier it is there for all waves, and nobody reads the one before this any more.
            stage_wait<8>();
            lds_barrier();
            fetch(min(i + 3, i1 - 1), (now + 3 * WIDE_STAGE) & (4 * WIDE_STAGE - 1));
            if (i + 1 < i1 && edge(start(i + 1))) {
                clean(lds + next);
                lds_barrier();
            }
            auto inside = [&](int j) { return j + 31 <= w_lo && (j + 31 < A.sinks || w_hi - j < window); };
            if (!inside(j0)) W.hide(s0, top, j0, h);
            W.tile(s0, s1, top, k, lds, ka, next, va, now + WIDE_VALUES);
            if (!inside(j0 + 32)) W.hide(s1, top, j0 + 32, h);
            W.tile(s1, s0, top, k, lds, ka, next + 32 * WIDE_ROW, va, now + WIDE_VALUES + 32 * WIDE_ROW);
            now = next;
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
