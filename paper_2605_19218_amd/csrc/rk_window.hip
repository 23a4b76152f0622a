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

int prefill_block_rows(int) { return PROMPT_ROWS; }

hipError_t launch_prefill(int dtype, const PrefillArgs& a, hipStream_t st)
{
    const int64_t units = (int64_t)a.B * a.Hkv, groups = units * a.blocks * a.S;
    if (groups > 0x7fffffff || (units * a.n * a.G + 7) / 8 > 0x7fffffff) return hipErrorInvalidValue;
    if (dtype == 0) attn_prompt<PromptF32><<<(uint32_t)groups, 256, 0, st>>>(a);
    else attn_prompt<PromptBf16><<<(uint32_t)groups, 256, 0, st>>>(a);
    if (a.S > 1) {
        const uint32_t g = (uint32_t)((units * a.n * a.G + 7) / 8);
        if (dtype == 0) prompt_merge<float><<<g, 256, 0, st>>>(a);
        else prompt_merge<bf16_t><<<g, 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

}  // namespace rk
