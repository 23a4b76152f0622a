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
// With 16-bit rows a weight is rounded to one bf16 part for its product with the Values, off by 2^-8 of itself at most: a mean's error of a step of its own rounding, 0.0020 of the largest output where
// that rounding alone makes 0.0015 to 0.0017.  Two parts, as attn_rows and attn_block have them, are half as many products again where prompts are bound by products.
#include <type_traits>
#include "rk_attn_block.hpp"

namespace rk {

namespace {

// LDS serves 256 bytes at a time, and a row of 16-bit numbers in it is 256 bytes: slots of 16 bytes lie permuted by the token, so that sixteen Keys' same slot are sixteen slots, and
// the two pairs of slots that 32 lanes read of four Values' rows are eight pairs. (fp32 rows are twice as long: eight Keys' same slot.)
__device__ __forceinline__ int key_slot(int token, int slot) { return slot ^ (4 * (token & 3) | ((token >> 2) & 3)); }
__device__ __forceinline__ int value_slot(int token, int slot) { return slot ^ 4 * (token & 3); }
__device__ __forceinline__ int slot_of(int token, int slot) { return slot ^ (2 * (token & 3) | ((token >> 2) & 1)); }

__device__ __forceinline__ bool odd_value(uint32_t bits) { return (bits & 0x7f800000u) == 0x7f800000u; }

// What a row sees.
struct Sight {
    int p, window, sinks;        // window: 2^30 when there is none
    __device__ __forceinline__ bool of(int j) const { return j <= p && (j < sinks || p - j < window); }
    static __device__ __forceinline__ uint32_t below(int x) { return x >= 32 ? ~0u : (1u << max(x, 0)) - 1; }
    // a bit for each of rows j ..+31 (a p in front of row 0 sees none, whatever the second difference wraps to)
    __device__ __forceinline__ uint32_t bits(int j) const { return below(p - j + 1) & (~below((int)((uint32_t)p - (uint32_t)window - (uint32_t)j + 1u)) | below(sinks - j)); }
    // scores of a lane's tokens j + 8 (i / 4) + i % 4: minus infinity where they are not seen
    __device__ __forceinline__ void hide(f32x16& s, int j) const
    {
        const uint32_t seen = bits(j);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t all = (uint32_t)((int32_t)(seen << (31 - 8 * (i >> 2) - (i & 3))) >> 31);
            s[i] = __uint_as_float((__float_as_uint(s[i]) & all) | (0xff800000u & ~all));
        }
    }
};

__device__ __forceinline__ uint32_t over(uint32_t x, const Divisor& d) { return (uint32_t)((uint64_t)x * d.m >> (31 + d.s)); }

// The splits of a block.
__device__ __forceinline__ int prompt_splits(const PrefillArgs& A, int block)
{
    int splits = 1;
#pragma unroll
    for (int i = 0; i < PREFILL_CUTS; ++i) splits += block >= A.cut[i] ? 1 : 0;
    return A.S > PREFILL_CUTS + 1 ? A.S : splits;
}

// Which rows and splits a work-group takes: the last blocks of all KV heads first, which see most, so that the short ones fill the gaps at the end; a head's
// work-groups go to the same XCDs, which read its Keys and Values from their L2.  (No branches: with one the wide kernel spills.)
__device__ __forceinline__ void prompt_place(const PrefillArgs& A, int& block, int& split, int& splits, int& u)
{
    const uint32_t units = A.B * A.Hkv, rank = over(blockIdx.x, A.by_units);
    u = blockIdx.x - rank * units;
    int at = (int)rank, end = A.blocks;          // rank among the blocks in front of `end`
    bool found = A.S > PREFILL_CUTS + 1;
    splits = found ? A.S : 1;
#pragma unroll
    for (int i = PREFILL_CUTS; i > 0; --i) {
        const int cut = A.cut[i - 1], count = (end - cut) * (i + 1);
        const bool here = !found && at < count;
        splits = here ? i + 1 : splits;
        found = found || here;
        at -= found ? 0 : count;
        end = found ? end : cut;
    }
    const int each = (int)((uint32_t)at / (uint32_t)splits);
    block = end - 1 - each;
    split = at - each * splits;
}

__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p; }
// 16 bytes a lane from `from` to LDS at `to` (of the wave) + 16 lane. (Not the builtin: behind it every read of LDS waits for all loads.) What is asked for
// is there after stage_wait(). (What is the wave's has to be said where code is not optimised.)
__device__ __forceinline__ void load_to_lds(const void* from, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(from) : "m0", "memory");
}
// The same with the address as a sum: of the wave (from, to + step) and of the lane, 32 bits.
template <int STEP>
__device__ __forceinline__ void load_to_lds(const char* from, uint32_t lane_bytes, uint32_t to)
{
#ifdef __OPTIMIZE__
    asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3" : : "s"(to), "i"(STEP), "v"(lane_bytes), "s"(from) : "m0", "scc", "memory");
#else                            // (a wave's address is in no scalar register then)
    load_to_lds(from + lane_bytes, to + STEP);
#endif
}
// this wave's loads but the last N are there
template <int N>
__device__ __forceinline__ void stage_wait() { asm volatile("s_waitcnt vmcnt(%0)" : : "i"(N) : "memory"); }


// What a block of `size` rows sees, in stages of TOKENS rows of the segment: `few` of the sinks, and from `from` on.
template <int TOKENS>
struct Prompt {
    int b, hk, len, first, rows, row0, window, sinks, p_lo, p_hi, few, from, i0, i1;
    bool before;                 // some of the rows stand in front of row 0
    __device__ __forceinline__ Prompt(const PrefillArgs& A, int u, int block, int split, int splits, int size)
    {
        b = over(u, A.by_hkv);
        hk = u - b * A.Hkv;
        len = min(max(A.len ? A.len[b] : A.max_len, 0), A.max_len);
        const int fresh = min(max(A.n_dev ? A.n_dev[b] : A.n, 0), A.n);
        first = len - fresh;
        rows = fresh * A.G;
        row0 = block * size;
        window = A.window > 0 ? min(A.window, 1 << 30) : 1 << 30;
        sinks = A.sinks;
        if (row0 >= rows) return;
        p_lo = first + token(A, row0);
        p_hi = first + token(A, row0 + size - 1);
        before = p_lo < 0;
        p_lo = max(p_lo, 0);
        int stages = 0;
        few = from = 0;
        if (p_hi >= 0) {
            const int lo = A.window > 0 ? max(p_lo - A.window + 1, 0) : 0;
            from = lo / TOKENS;
            few = min((min(sinks, lo) + TOKENS - 1) / TOKENS, from);
            stages = few + p_hi / TOKENS - from + 1;
        }
        // (stages and splits stay below 2^25 and 2^6)
        i0 = (int)((uint32_t)stages * (uint32_t)split / (uint32_t)splits);
        i1 = (int)((uint32_t)stages * (uint32_t)(split + 1) / (uint32_t)splits);
    }
    __device__ __forceinline__ int token(const PrefillArgs& A, int r) const { return (int)over(min(r, rows - 1), A.by_g); }
    __device__ __forceinline__ int start(int i) const { return TOKENS * (i < few ? i : i - few + from); }
    // whether all rows from position lo to hi see rows j ..+n-1
    __device__ __forceinline__ bool inside(int j, int n, int lo, int hi) const { return j + n - 1 <= lo && (j + n - 1 < sinks || hi - j < window); }
    // Which of the block's tiles of SIZE rows, counted through its stages, inside() says yes for, for positions lo to hi: those in front of `a`, and `n` from `b` on.
    struct Inside {
        int a, b, n;
        __device__ __forceinline__ bool of(int tile) const { return tile < a || (uint32_t)(tile - b) < (uint32_t)n; }
    };
    template <int SIZE>
    __device__ __forceinline__ Inside tiles_inside(int lo, int hi) const
    {
        constexpr int PER = TOKENS / SIZE;
        const int whole = (lo + 1) / SIZE;       // tiles that end in front of lo's next row (none for a lo in front of row 0)
        const int moved = PER * (from - few), first = max(hi - window + SIZE, 0) / SIZE;
        Inside t;
        t.a = max(min(sinks / SIZE, whole), 0);
        if (few < from) t.a = min(t.a, PER * few);
        t.b = max(first - moved, few < from ? PER * few : 0);
        t.n = max(whole - moved - t.b, 0);
        return t;
    }
    // whether a stage is masked for some row of the block
    __device__ __forceinline__ bool edge(int j) const { return before || !inside(j, TOKENS, p_lo, p_hi); }
};

// Values of a stage in LDS that are no numbers become 0 (what a masked one holds may not meet a weight of 0), and the flag says that there were any
template <typename T>
__device__ __forceinline__ void clean_values(char* values, int bytes, int* odd, int tid)
{
#pragma unroll 1
    for (int x = 16 * tid; x < bytes; x += 4096) {
        const uint4 d = *(const uint4*)(values + x);
        uint32_t w[4] = {d.x, d.y, d.z, d.w};
        bool any = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t keep = sizeof(T) == 4 ? (odd_value(w[e]) ? 0u : ~0u) : (odd_value(w[e]) ? 0u : 0xffff0000u) | (odd_value(w[e] << 16) ? 0u : 0xffffu);
            any |= keep != ~0u;
            w[e] &= keep;
        }
        if (any) {
            *(uint4*)(values + x) = make_uint4(w[0], w[1], w[2], w[3]);
            *odd = 1;
        }
    }
}

// ---- fp32, 128 rows ----------------------------------------------------------------
// 32 rows a wave, 128 a work-group, two work-groups a compute unit; stages of 32 tokens in LDS, two of them. Bound by the fp32 matrix instructions: 128 of 64 cycles
// for a tile, to some 500 cycles of vector instructions (8 x 28 heads, 500 tokens on 8000 3945 us, 120 TFLOP/s; the matrix cores are busy for 78 % of the cycles).
constexpr int F32_ROWS = 128, F32_TOKENS = 32, F32_ROW = 512, F32_VALUES = F32_TOKENS * F32_ROW, F32_STAGE = 2 * F32_VALUES;

__global__ __launch_bounds__(256, 2) void attn_prompt_f32(PrefillArgs A)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int block, split, splits, u;
    prompt_place(A, block, split, splits, u);
    const Prompt<F32_TOKENS> P(A, u, block, split, splits, F32_ROWS);
    if (P.row0 >= P.rows) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, n = lane & 31;
    const int row = P.row0 + 32 * wave + n, mine = min(row, P.rows - 1), tok = P.token(A, mine), head = P.hk * A.G + mine - tok * A.G;
    const Sight sight{P.first + tok, P.window, P.sinks};
    const int w_lo = P.first + P.token(A, P.row0 + 32 * wave), w_hi = P.first + P.token(A, P.row0 + 32 * wave + 31);

    f32x4 q[16];
    const float* qp = (const float*)A.q + (int64_t)P.b * A.q_sb + (int64_t)head * A.q_sh + (int64_t)tok * A.q_st;
#pragma unroll
    for (int i = 0; i < 16; ++i) q[i] = *(const f32x4*)(qp + 8 * i + 4 * h);
    const float* kp = (const float*)A.k + (int64_t)P.b * A.sb + (int64_t)P.hk * A.sh;
    const float* vp = (const float*)A.v + (int64_t)P.b * A.sb + (int64_t)P.hk * A.sh;
    float m = ROWS_NEG_INF, l = 0.f;
    f32x16 O[4];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[c][i] = 0.f;

    int* odd = (int*)(lds + 2 * F32_STAGE);
    if (P.i0 < P.i1) {
        // rows 8 wave + 2 x + lane / 32 of a stage, x < 4
        const uint32_t base = __builtin_amdgcn_readfirstlane(lds_address(lds)) + 8 * F32_ROW * wave;
        auto fetch = [&](int i, int buf) {
            const int j = P.start(i) + 8 * wave + h;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int64_t at = (int64_t)min(j + 2 * x, P.len - 1) * A.st + 4 * slot_of(2 * x + h, n);
                load_to_lds(kp + at, base + buf + 2 * F32_ROW * x);
                load_to_lds(vp + at, base + buf + F32_VALUES + 2 * F32_ROW * x);
            }
        };
        fetch(P.i0, 0);
        if (tid == 0) *odd = 0;
        int ka[4], va[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            ka[i] = n * F32_ROW + 16 * slot_of(n, 2 * i + h);
            va[i] = F32_VALUES + (4 * h + i) * F32_ROW + 16 * slot_of(4 * h + i, n);
        }
        int now = 0;
#pragma unroll 1
        for (int i = P.i0; i < P.i1; ++i) {
            const int j0 = P.start(i);
            stage_wait<0>();
            lds_barrier();               // (this stage is there for all waves, and nobody reads the one before it any more)
            fetch(min(i + 1, P.i1 - 1), now ^ F32_STAGE);
            if (P.edge(j0)) {
                clean_values<float>(lds + now + F32_VALUES, F32_VALUES, odd, tid);
                lds_barrier();
            }
            now ^= F32_STAGE;
            if (j0 > w_hi) continue;     // (behind all of this wave's rows)
            const char* at = lds + (now ^ F32_STAGE);
            f32x16 s;
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                const f32x4 a = *(const f32x4*)(at + ka[x & 3] + 128 * (x >> 2));
#pragma unroll
                for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], q[x][e], s, 0, 0, 0);
            }
            if (!P.inside(j0, F32_TOKENS, w_lo, w_hi)) sight.hide(s, j0 + 4 * h);
            __builtin_amdgcn_s_setprio(1);       // (the other wave of the SIMD has its products; 32 heads x 2944 tokens 601 us without, 593 with)
            float mt = s[0];
#pragma unroll
            for (int e = 1; e < 16; ++e) mt = fmaxf(mt, s[e]);
            mt = halves_max(mt) * A.scale_log2;
            if (__any(mt > m + 8.f)) {
                const float m_new = fmaxf(m, mt), alpha = m > ROWS_NEG_INF ? rows_exp2(m - m_new) : 1.f;
                l *= alpha;
#pragma unroll
                for (int c = 0; c < 4; ++c) O[c] *= alpha;
                m = m_new;
            }
            const float ref = m > ROWS_NEG_INF ? m : 0.f;
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[e] = rows_exp2(fmaf(s[e], A.scale_log2, -ref));
                sum += s[e];
            }
            l += sum;
            __builtin_amdgcn_s_setprio(0);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const f32x4 a = *(const f32x4*)(at + va[e & 3] + 8 * F32_ROW * (e >> 2));
#pragma unroll
                for (int c = 0; c < 4; ++c) O[c] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[c], s[e], O[c], 0, 0, 0);
            }
        }
        stage_wait<0>();
        // The Values that were left out join the rows that see them: a sum of one is it, or NaN.  (O[c][i] is channel 4 (8 (i / 4) + 4 h + i % 4) + c)
        if (*odd) {
#pragma unroll 1
            for (int i = P.i0; i < P.i1; ++i) {
                const int j0 = P.start(i);
                if (!P.edge(j0)) continue;
#pragma unroll 1
                for (int j = j0; j < min(j0 + F32_TOKENS, P.len); ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const f32x4 v = *(const f32x4*)(vp + (int64_t)j * A.st + 4 * (8 * (e >> 2) + 4 * h + (e & 3)));
#pragma unroll
                        for (int c = 0; c < 4; ++c) O[c][e] += odd_value(__float_as_uint(v[c])) && sight.of(j) ? v[c] : 0.f;
                    }
            }
        }
    }

    l = halves_sum(l);
    if (row >= P.rows) return;
    const float inv = splits > 1 ? 1.f : l == 0.f ? 0.f : 1.f / l;
    const size_t slot = ((size_t)u * A.n * A.G + row) * A.S + split;
    float* o = splits > 1 ? A.ws_acc + slot * D : (float*)A.out + (int64_t)P.b * A.o_sb + (int64_t)head * A.o_sh + (int64_t)tok * A.o_st;
    const bool none = splits == 1 && l == 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e)
        *(f32x4*)(o + 4 * (8 * (e >> 2) + 4 * h + (e & 3))) = none ? (f32x4){0.f, 0.f, 0.f, 0.f} : (f32x4){O[0][e], O[1][e], O[2][e], O[3][e]} * inv;
    if (splits > 1 && h == 0) { A.ws_m[slot] = m; A.ws_l[slot] = l; }
}

// ---- fp32, many rows: products of bf16 parts ---------------------------------------
// The bf16 matrix instructions are 16 times as fast as the fp32 ones. A number is exactly the sum of three bf16 parts, and of the nine products of two numbers' parts the six
// large ones leave out less than 2^-24 of the product: 96 instructions of 32 cycles for a tile in place of 128 of 64. Queries are in parts once, weights in registers, Keys and
// Values on their way into LDS, once for the 256 rows of the eight waves: each thread asks for eight channels of a Key and of a Value a stage ahead (into a place of its own in LDS), and
// writes their parts for all. Of the two waves of a SIMD one does that in front of its products, the other behind them.
// 8 x 28 heads, 500 tokens on 8000 2325 us, 204 TFLOP/s, 1220 of issued products: what a large bf16 matrix product reaches here. 32 heads x 2944 tokens 417 to 424 us, 169 TFLOP/s, where
// the work-groups, one a compute unit and some three times as long as others, leave a fifth of the compute units' time unused.
// What that holds for: numbers from 2^-100 on (of smaller ones, parts below the smallest normal number may count as 0, less than 2^-125 of the number in all). Above the largest bf16
// number the first part is rounded towards zero (2^-23 of a product left out there), and an infinity has no other parts, so that finite numbers have finite parts. An infinity times a part of 0 is NaN:
// Values that are no numbers are left out in every stage and join the rows that see them behind the loop, as on edges in the other kernels; for Keys and queries the header says it.
// (Looking for such numbers costs 1.5 %: 32 heads x 2944 tokens 410 -> 417 us, 8 x 28 heads, 500 tokens on 8000 2290 -> 2325.)
constexpr int PARTS_ROWS = 256, PARTS_TOKENS = 32, PARTS_PLANE = PARTS_TOKENS * 256, PARTS_STAGE = 6 * PARTS_PLANE, PARTS_RAW = 2 * PARTS_STAGE,
              PARTS_LDS = PARTS_RAW + 8 * 4096;        // planes [stage][Keys 3, Values 3]; eight waves' own places; and a flag

// The bits of the largest of eight numbers' sizes (more than an infinity's where one is no number).
__device__ __forceinline__ uint32_t largest(const float (&x)[8])
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    return top;
}
// eight numbers in parts; top: largest() of them, or less where it is known to be no more than the largest bf16 number
__device__ __forceinline__ void parts3(const float (&x)[8], bf16x8 (&p)[3], uint32_t top = 0)
{
    constexpr uint32_t MOST = 0x7f7f0000u;       // the largest bf16 number
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = x[i];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = __builtin_bit_cast(uint32_t, (bf16x2){(__bf16)r[2 * i], (__bf16)r[2 * i + 1]});
            if (k < 2) {
                r[2 * i] -= __uint_as_float(w[i] << 16);
                r[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
            }
        }
        if (k == 0 && top > MOST) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t bits = __float_as_uint(x[i]), size = bits & 0x7fffffffu, first = bits & 0xffff0000u;
                if (size > MOST && size <= 0x7f800000u) {
                    w[i >> 1] = i & 1 ? (w[i >> 1] & 0xffffu) | first : (w[i >> 1] & 0xffff0000u) | first >> 16;
                    r[i] = size == 0x7f800000u ? 0.f : x[i] - __uint_as_float(first);
                }
            }
        }
        p[k] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
    }
}
// the six products, small ones first
__device__ __forceinline__ void product3(const bf16x8 (&a)[3], const bf16x8 (&b)[3], f32x16& s)
{
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[2], b[0], s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0], b[2], s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[1], b[1], s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[1], b[0], s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0], b[1], s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0], b[0], s, 0, 0, 0);
}

__global__ __launch_bounds__(512, 2) void attn_prompt_parts(PrefillArgs A)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int block, split, splits, u;
    prompt_place(A, block, split, splits, u);
    const Prompt<PARTS_TOKENS> P(A, u, block, split, splits, PARTS_ROWS);
    if (P.row0 >= P.rows) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, n = lane & 31;
    const int row = P.row0 + 32 * wave + n, mine = min(row, P.rows - 1), tok = P.token(A, mine), head = P.hk * A.G + mine - tok * A.G;
    const Sight sight{P.first + tok, P.window, P.sinks};
    const int w_lo = P.first + P.token(A, P.row0 + 32 * wave), w_hi = P.first + P.token(A, P.row0 + 32 * wave + 31);

    bf16x8 q[8][3];
    const float* qp = (const float*)A.q + (int64_t)P.b * A.q_sb + (int64_t)head * A.q_sh + (int64_t)tok * A.q_st;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const f32x4 a = *(const f32x4*)(qp + 16 * i + 8 * h), b = *(const f32x4*)(qp + 16 * i + 8 * h + 4);
        const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        parts3(x, q[i], largest(x));
    }
    const float* kp = (const float*)A.k + (int64_t)P.b * A.sb + (int64_t)P.hk * A.sh;
    const float* vp = (const float*)A.v + (int64_t)P.b * A.sb + (int64_t)P.hk * A.sh;
    float m = ROWS_NEG_INF, l = 0.f;
    f32x16 O[4];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[c][i] = 0.f;

    int* odd = (int*)(lds + PARTS_LDS);
    if (tid == 0) *odd = 0;
    __syncthreads();
    if (P.i0 < P.i1) {
        // this thread's token of a stage, and its eight channels
        const int token = tid >> 4, eight = tid & 15;
        char* own = lds + PARTS_RAW + 4096 * wave + 16 * lane;
        const uint32_t base = __builtin_amdgcn_readfirstlane(lds_address(lds)) + PARTS_RAW + 4096 * wave;
        auto fetch = [&](int i) {
            const int64_t at = (int64_t)min(P.start(i) + token, P.len - 1) * A.st + 8 * eight;
            load_to_lds(kp + at, base);
            load_to_lds(kp + at + 4, base + 1024);
            load_to_lds(vp + at, base + 2 * 1024);
            load_to_lds(vp + at + 4, base + 3 * 1024);
        };
        // the parts of what was asked for as stage i; then stage `next` is asked for
        auto ready = [&](int i, int next, char* to) {
            stage_wait<0>();
            f32x4 raw[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) raw[x] = *(const f32x4*)(own + 1024 * x);
            asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
            __builtin_amdgcn_sched_barrier(0);
            fetch(next);
            const int kat = token * 256 + 16 * key_slot(token, eight), vat = token * 256 + 16 * value_slot(token, eight);
            bf16x8 p[3];
            const float a[8] = {raw[0][0], raw[0][1], raw[0][2], raw[0][3], raw[1][0], raw[1][1], raw[1][2], raw[1][3]};
            parts3(a, p, largest(a));
#pragma unroll
            for (int k = 0; k < 3; ++k) *(bf16x8*)(to + k * PARTS_PLANE + kat) = p[k];
            float b[8] = {raw[2][0], raw[2][1], raw[2][2], raw[2][3], raw[3][0], raw[3][1], raw[3][2], raw[3][3]};
            const uint32_t top = largest(b);
            if (top >= 0x7f800000u) {            // Values that are no numbers count as 0
#pragma unroll
                for (int e = 0; e < 8; ++e) b[e] = odd_value(__float_as_uint(b[e])) ? 0.f : b[e];
                atomicOr(odd, P.edge(P.start(i)) ? 1 : 2);
            }
            parts3(b, p, top);
#pragma unroll
            for (int k = 0; k < 3; ++k) *(bf16x8*)(to + (3 + k) * PARTS_PLANE + vat) = p[k];
        };
        int ka[8], va[4];
#pragma unroll
        for (int i = 0; i < 8; ++i) ka[i] = n * 256 + 16 * key_slot(n, 2 * i + h);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 4 * h + ((lane & 15) >> 2);
            va[i] = 3 * PARTS_PLANE + r * 256 + 16 * value_slot(r, 4 * i + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + 8 * (lane & 1);
        }
        fetch(P.i0);
        ready(P.i0, min(P.i0 + 1, P.i1 - 1), lds);
        lds_barrier();
        int now = 0;
#pragma unroll 1
        for (int i = P.i0; i < P.i1; ++i) {
            const int j0 = P.start(i);
            const char* at = lds + now;
            char* other = lds + (now ^ PARTS_STAGE);
            now ^= PARTS_STAGE;
            const bool more = i + 1 < P.i1;
            if (more && wave < 4) ready(i + 1, min(i + 2, P.i1 - 1), other);
            if (j0 <= w_hi) {                    // (else behind all of this wave's rows)
                f32x16 s;
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    bf16x8 a[3];
#pragma unroll
                    for (int k = 0; k < 3; ++k) a[k] = *(const bf16x8*)(at + k * PARTS_PLANE + ka[x]);
                    product3(a, q[x], s);
                }
                if (!P.inside(j0, PARTS_TOKENS, w_lo, w_hi)) sight.hide(s, j0 + 4 * h);
                float mt = s[0];
#pragma unroll
                for (int e = 1; e < 16; ++e) mt = fmaxf(mt, s[e]);
                mt = halves_max(mt) * A.scale_log2;
                if (__any(mt > m + 8.f)) {
                    const float m_new = fmaxf(m, mt), alpha = m > ROWS_NEG_INF ? rows_exp2(m - m_new) : 1.f;
                    l *= alpha;
#pragma unroll
                    for (int c = 0; c < 4; ++c) O[c] *= alpha;
                    m = m_new;
                }
                const float ref = m > ROWS_NEG_INF ? m : 0.f;
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    s[e] = rows_exp2(fmaf(s[e], A.scale_log2, -ref));
                    sum += s[e];
                }
                l += sum;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    bf16x8 w[3];
                    const float x[8] = {s[8 * t], s[8 * t + 1], s[8 * t + 2], s[8 * t + 3], s[8 * t + 4], s[8 * t + 5], s[8 * t + 6], s[8 * t + 7]};
                    parts3(x, w);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        bf16x8 a[3];
#pragma unroll
                        for (int k = 0; k < 3; ++k) {
                            typedef __attribute__((address_space(3))) s16x4* Lds;
                            uint2 d[2];
#pragma unroll
                            for (int y = 0; y < 2; ++y)
                                d[y] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                                     (Lds)(at + k * PARTS_PLANE + va[c] + (16 * t + 8 * y) * 256)));
                            a[k] = __builtin_bit_cast(bf16x8, make_uint4(d[0].x, d[0].y, d[1].x, d[1].y));
                        }
                        product3(a, w, O[c]);
                    }
                }
            }
            if (more && wave >= 4) ready(i + 1, min(i + 2, P.i1 - 1), other);
            lds_barrier();
        }
        stage_wait<0>();
        // The Values that were left out join the rows that see them: a sum of one is it, or NaN.
        if (const int found = *odd) {            // 1: in stages on an edge, 2: in others
#pragma unroll 1
            for (int i = P.i0; i < P.i1; ++i) {
                const int j0 = P.start(i);
                if (!(found & (P.edge(j0) ? 1 : 2))) continue;
#pragma unroll 1
                for (int j = j0; j < min(j0 + PARTS_TOKENS, P.len); ++j)
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const f32x4 v = *(const f32x4*)(vp + (int64_t)j * A.st + 32 * c + 8 * e + 4 * h);
#pragma unroll
                            for (int x = 0; x < 4; ++x) O[c][4 * e + x] += odd_value(__float_as_uint(v[x])) && sight.of(j) ? v[x] : 0.f;
                        }
            }
        }
    }

    l = halves_sum(l);
    if (row >= P.rows) return;
    const float inv = splits > 1 ? 1.f : l == 0.f ? 0.f : 1.f / l;
    const size_t slot = ((size_t)u * A.n * A.G + row) * A.S + split;
    float* o = splits > 1 ? A.ws_acc + slot * D : (float*)A.out + (int64_t)P.b * A.o_sb + (int64_t)head * A.o_sh + (int64_t)tok * A.o_st;
    const bool none = splits == 1 && l == 0.f;
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            *(f32x4*)(o + 32 * c + 8 * e + 4 * h) =
                none ? (f32x4){0.f, 0.f, 0.f, 0.f} : (f32x4){O[c][4 * e], O[c][4 * e + 1], O[c][4 * e + 2], O[c][4 * e + 3]} * inv;
    if (splits > 1 && h == 0) { A.ws_m[slot] = m; A.ws_l[slot] = l; }
}

// ---- bf16, many rows: 64 rows a wave ------------------------------------------------
// A stage of 64 tokens, four of them in LDS: loads go there without passing through registers, two stages ahead, one barrier a stage. Rows in two groups of 32, so that a Key or Value
// read from LDS feeds two products. (With 32 rows a wave and two waves a SIMD LDS would have to deliver 128 bytes a cycle, all it has.)
// 28 heads x 16384 tokens, all visible 1613 us, 1193 TFLOP/s; with a window of 4096 771 to 780, 1080 to 1090; 32 x 2944 85, 835 (a large library product reaches 1161 here). A wave has its
// SIMD for itself and issues an instruction in 4 to 5 cycles, so their number bounds it: of some 210 a tile 32 are products of 32 cycles, 32 exponentials of 16. What took instructions away took time
// away: loads' addresses as a wave's and a lane's part 814 -> 800, one exclusive or for each LDS address 800 -> 787, sums by pairs of rounded weights (they divide what those weights made), kept
// over tiles like the maxima's limits, 787 -> 780; and branches beside products in place of between them 837 -> 826.
// A work-group's beginning and end take 12 us, a stage 1.55.
// In LDS a token's row is its 256 bytes, slots permuted as key_slot() and value_slot() say: what a load leaves is lane by lane, so it is the lanes' addresses that are permuted.
constexpr int WIDE_ROWS = 256, WIDE_TOKENS = 64, WIDE_ROW = 256, WIDE_VALUES = WIDE_TOKENS * WIDE_ROW, WIDE_STAGE = 2 * WIDE_VALUES;
constexpr int WIDE_LDS = 4 * WIDE_STAGE;      // and a flag

struct WideRows {
    bf16x8 q[2][8];
    f32x16 O[2][4];
    float m[2], l[2][2];         // running maximum, and sum in two halves
    float ref[2], limit[2];      // by m: what weights are taken relative to, and the score (not scaled) that the maximum moves for
    Sight sight[2];
    float c, inv_c;              // scale, log2 domain

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
    // Piece i of a tile's 32 Keys (slots 2 i + h, permuted: key_slot); ka: where this lane's piece 0 of the stage is in LDS, `more`: the tile in it.
    static __device__ __forceinline__ bf16x8 key(uint32_t ka, int more, int i)
    {
        typedef const __attribute__((address_space(3))) char* Lds;
        return *(const __attribute__((address_space(3))) bf16x8*)((Lds)(uintptr_t)(ka ^ 32 * i) + more);
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
    // The same, for scores that came out of assembly: of those the compiler makes each maximum's operands canonical first, 12 instructions more a tile. (What it reads is long done, and so is
    // what it writes when row_most() takes it.)
    static __device__ __forceinline__ float most3(const f32x16& s)
    {
        float a, b;
        asm("v_max3_f32 %0, %2, %3, %4\n\tv_max3_f32 %1, %5, %6, %7\n\tv_max3_f32 %0, %0, %8, %9\n\tv_max3_f32 %1, %1, %10, %11\n\t"
            "v_max3_f32 %0, %0, %12, %13\n\tv_max3_f32 %1, %1, %14, %15\n\tv_max3_f32 %0, %0, %16, %17\n\tv_max_f32 %0, %0, %1"
            : "=&v"(a), "=&v"(b)
            : "v"(s[0]), "v"(s[1]), "v"(s[2]), "v"(s[3]), "v"(s[4]), "v"(s[5]), "v"(s[6]), "v"(s[7]), "v"(s[8]), "v"(s[9]), "v"(s[10]), "v"(s[11]), "v"(s[12]), "v"(s[13]),
              "v"(s[14]), "v"(s[15]));
        return a;
    }
    // (of the whole row)
    static __device__ __forceinline__ float row_most(float mine)
    {
        const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(mine), __float_as_uint(mine), false, false);
        float d;
        asm("v_max_f32 %0, %1, %2" : "=v"(d) : "v"(b[0]), "v"(b[1]));      // (as halves_max(), no canonical operands)
        return d;
    }
    __device__ __forceinline__ void settle(int g)
    {
        ref[g] = m[g] > ROWS_NEG_INF ? m[g] : 0.f;
        limit[g] = (m[g] + 8.f) * inv_c;
    }
    __device__ __forceinline__ bool behind(const float (&top)[2]) const { return __any(top[0] > limit[0] || top[1] > limit[1]); }
    // the running maxima move to a tile's
    __device__ __forceinline__ void follow(const float (&top)[2])
    {
        hold();                  // (or they would be copied in front of the branch, for every tile)
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const float m_new = fmaxf(m[g], top[g] * c), alpha = m[g] > ROWS_NEG_INF ? rows_exp2(m[g] - m_new) : 1.f;
            l[g][0] *= alpha;
            l[g][1] *= alpha;
#pragma unroll
            for (int b = 0; b < 4; ++b) O[g][b] *= alpha;
            m[g] = m_new;
            settle(g);
        }
    }
    // half x of channels 32 b + lane % 32 of the tile's tokens 16 t + (4 h ..+3, 8 + 4 h ..+3); va: where this lane's place of block 0 of the stage is in LDS (see value_slot), `more`: the tile in it
    static __device__ __forceinline__ s16x4 values(uint32_t va, int more, int t, int b, int x)
    {
        typedef __attribute__((address_space(3))) char* Lds;
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)((Lds)(uintptr_t)(va ^ 64 * b) + more + (16 * t + 8 * x) * WIDE_ROW));
    }
    // a tile on an edge: what a row does not see has no score
    __device__ __forceinline__ void hide(f32x16 (&s)[2], float (&top)[2], int j0, int h) const
    {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            sight[g].hide(s[g], j0 + 4 * h);
            top[g] = row_most(most(s[g]));
        }
    }
    // Scores belong into the other half of the register file, where the vector instructions are that they are for; the compiler would have them beside the accumulators and
    // copy them (64 instructions a tile). The vector instructions that read them come 300 cycles behind, matrix instructions of the same group two behind.
    static __device__ __forceinline__ void score(f32x16& s, const bf16x8& k, const bf16x8& q, bool begin)
    {
        if (begin) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(k), "a"(q));
        else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(k), "a"(q));
    }
    // One tile (vt of a stage's Values at va): scores s of it, whose largest are `top`, into O; the scores of the next tile (Keys k) into `next`, its largest into `top`; the Keys of
    // the one behind it (kt of a stage's at ka) into k.
    // A wave has its SIMD for itself, so what runs beside the matrix instructions is what stands between them: 32 of 32 cycles. Behind the first stand the branches (what is to be hidden,
    // maxima that move): in front of them the matrix cores would wait. 24 have beside them the weights, 16 pairs of 52 cycles (the exponentials 16 each), two in three instructions'
    // time, and the last eight the maxima and beside(0..7), a load of a later stage each; LDS is read one piece a step.
    template <typename E, typename F>
    __device__ __forceinline__ void tile(f32x16 (&s)[2], f32x16 (&next)[2], float (&top)[2], bf16x8 (&k)[8], uint32_t ka, int kt, uint32_t va, int vt,
                                         E edge, F beside)
    {
        uint32_t p[2][8];
        s16x4 v[2][4][2];
        auto weigh = [&](int pair) {             // of rows' group pair / 8, tokens 2 (pair % 8) and the next
            const int g = pair >> 3, e = 2 * (pair & 7);
            s[g][e] = rows_exp2(fmaf(s[g][e], c, -ref[g]));
            s[g][e + 1] = rows_exp2(fmaf(s[g][e + 1], c, -ref[g]));
        };
        auto pack = [&](int pair) {
            const int g = pair >> 3, e = 2 * (pair & 7);
            const bf16x2 w = {(__bf16)s[g][e], (__bf16)s[g][e + 1]};
            p[g][pair & 7] = __builtin_bit_cast(uint32_t, w);
            l[g][pair & 1] = __builtin_amdgcn_fdot2_f32_bf16(w, (bf16x2){(__bf16)1.f, (__bf16)1.f}, l[g][pair & 1], false);
        };
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int x = 0; x < 32; ++x) {
            if (x < 16) {
                const int g = x & 1, i = x >> 1;
                score(next[g], k[i], q[g][i], i == 0);
                v[x >> 3][(x >> 1) & 3][x & 1] = values(va, vt, x >> 3, (x >> 1) & 3, x & 1);
            } else {
                const int g = (x >> 3) & 1, t = (x >> 2) & 1, b = x & 3;
                const uint2 v0 = __builtin_bit_cast(uint2, v[t][b][0]), v1 = __builtin_bit_cast(uint2, v[t][b][1]);
                O[g][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, make_uint4(v0.x, v0.y, v1.x, v1.y)),
                                                                  __builtin_bit_cast(bf16x8, make_uint4(p[g][4 * t], p[g][4 * t + 1], p[g][4 * t + 2], p[g][4 * t + 3])),
                                                                  O[g][b], 0, 0, 0);
                if (x >= 24) k[x - 24] = key(ka, kt, x - 24);
            }
            if (x == 0) {
                edge();
                if (behind(top)) follow(top);
                hold();
            }
            // pairs 2 y and 2 y + 1 in steps 1 + 3 y ..+2, each one's sums and rounding a step behind
            const int y = x - 1;
            if (y >= 0 && y < 24 && y % 3 < 2) weigh(2 * (y / 3) + y % 3);
            if (y >= 0 && y < 25 && y % 3 == 1) pack(2 * (y / 3));
            if (y >= 0 && y < 25 && y % 3 == 2) pack(2 * (y / 3) + 1);
            if (x == 26 || x == 28) top[x / 2 - 13] = most3(next[x / 2 - 13]);
            if (x == 29 || x == 30) top[x - 29] = row_most(top[x - 29]);
            if (x == 24) beside(std::integral_constant<int, 0>{});
            if (x == 25) beside(std::integral_constant<int, 1>{});
            if (x == 26) beside(std::integral_constant<int, 2>{});
            if (x == 27) beside(std::integral_constant<int, 3>{});
            if (x == 28) beside(std::integral_constant<int, 4>{});
            if (x == 29) beside(std::integral_constant<int, 5>{});
            if (x == 30) beside(std::integral_constant<int, 6>{});
            if (x == 31) beside(std::integral_constant<int, 7>{});
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

__global__ __launch_bounds__(256, 1) void attn_prompt_wide(PrefillArgs A)
{
    extern __shared__ __attribute__((aligned(256))) char lds[];
    int block, split, splits, u;
    prompt_place(A, block, split, splits, u);
    const Prompt<WIDE_TOKENS> P(A, u, block, split, splits, WIDE_ROWS);
    if (P.row0 >= P.rows) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, n = lane & 31;

    WideRows W;
    W.c = A.scale_log2;
    W.inv_c = 1.f / W.c;
    int tok[2], head[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        const int mine = min(P.row0 + 64 * wave + 32 * g + n, P.rows - 1);
        tok[g] = P.token(A, mine);
        head[g] = P.hk * A.G + mine - tok[g] * A.G;
        W.sight[g] = Sight{P.first + tok[g], P.window, P.sinks};
        W.m[g] = ROWS_NEG_INF;
        W.l[g][0] = W.l[g][1] = 0.f;
        const bf16_t* q = (const bf16_t*)A.q + (int64_t)P.b * A.q_sb + (int64_t)head[g] * A.q_sh + (int64_t)tok[g] * A.q_st;
#pragma unroll
        for (int i = 0; i < 8; ++i) W.q[g][i] = *(const bf16x8*)(q + 16 * i + 8 * h);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) W.O[g][c][i] = 0.f;
    }

    const int w_lo = P.first + P.token(A, P.row0 + 64 * wave), w_hi = P.first + P.token(A, P.row0 + 64 * wave + 63);      // positions of the wave's rows
    const bf16_t* kp = (const bf16_t*)A.k + (int64_t)P.b * A.sb + (int64_t)P.hk * A.sh;
    const bf16_t* vp = (const bf16_t*)A.v + (int64_t)P.b * A.sb + (int64_t)P.hk * A.sh;
    int* odd = (int*)(lds + WIDE_LDS);
    if (P.i0 < P.i1) {
        // Rows 16 wave + 4 x + lane / 16 of a stage, x < 4: their 16-byte pieces, in the order that reading them undoes.  A lane's places in a stage are the same in all of
        // them; in one that reaches behind the last row they repeat it.  (Bytes in 32 bits: rows are less than 2^24 elements apart.)
        const uint32_t base = __builtin_amdgcn_readfirstlane(lds_address(lds)) + 16 * WIDE_ROW * wave;
        const int64_t step = 2 * WIDE_TOKENS * A.st, apart = (const char*)vp - (const char*)kp;
        uint32_t place[2][4];            // of Keys, of Values
        auto places = [&](int last) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int token = 4 * x + (lane >> 4);
                const uint32_t row = 2 * (uint32_t)min(16 * wave + token, last) * (uint32_t)A.st;
                place[0][x] = row + 16 * key_slot(token, lane & 15);
                place[1][x] = row + 16 * value_slot(token, lane & 15);
            }
        };
        places(WIDE_TOKENS);
        const int tail = P.len % WIDE_TOKENS ? P.few + P.len / WIDE_TOKENS - P.from : -1;        // the stage that reaches behind the last row
        const char* from = (const char*)kp + P.start(P.i0) * (step / WIDE_TOKENS);               // the stage that is asked for: i
        if (P.i0 == tail) places((P.len - 1) % WIDE_TOKENS);
        auto aim = [&](int i) {          // from the one in front of it (there is none behind the last: that is asked for again)
            if (i < P.i1) {
                from += i == P.few ? step * (P.from - P.few + 1) : step;
                if (i == tail) places((P.len - 1) % WIDE_TOKENS);
            }
        };
        auto load = [&](auto piece, int buf) {
            constexpr int x = decltype(piece)::value >> 1, v = decltype(piece)::value & 1;
            load_to_lds<v * WIDE_VALUES + 4 * WIDE_ROW * x>(v ? from + apart : from, place[v][x], base + buf);
        };
        auto fetch = [&](int buf) {
            load(std::integral_constant<int, 0>{}, buf); load(std::integral_constant<int, 1>{}, buf);
            load(std::integral_constant<int, 2>{}, buf); load(std::integral_constant<int, 3>{}, buf);
            load(std::integral_constant<int, 4>{}, buf); load(std::integral_constant<int, 5>{}, buf);
            load(std::integral_constant<int, 6>{}, buf); load(std::integral_constant<int, 7>{}, buf);
        };
        fetch(0);
        aim(P.i0 + 1);
        fetch(WIDE_STAGE);
        aim(P.i0 + 2);
        fetch(2 * WIDE_STAGE);
        const auto whole = P.before ? typename Prompt<WIDE_TOKENS>::Inside{0, 0, 0} : P.template tiles_inside<WIDE_TOKENS>(P.p_lo, P.p_hi);      // stages that no row's edge is in
        const auto inside = P.template tiles_inside<32>(w_lo, w_hi);
        if (tid == 0) *odd = 0;
        stage_wait<16>();
        lds_barrier();
        if (!whole.of(P.i0)) {
            clean_values<bf16_t>(lds + WIDE_VALUES, WIDE_VALUES, odd, tid);
            lds_barrier();
        }
        const uint32_t at = lds_address(lds), vr = 4 * h + ((lane & 15) >> 2), ka = at + n * WIDE_ROW + 16 * key_slot(n, h);
        const uint32_t va = at + WIDE_VALUES + vr * WIDE_ROW + 16 * value_slot(vr, 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + 8 * (lane & 1);
        f32x16 s0[2], s1[2];
        bf16x8 k[8];
        float top[2];
#pragma unroll
        for (int x = 0; x < 8; ++x) k[x] = WideRows::key(ka, 0, x);
        W.scores(k, s0);
#pragma unroll
        for (int x = 0; x < 8; ++x) k[x] = WideRows::key(ka, 32 * WIDE_ROW, x);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            asm volatile("" : "+v"(s0[g]));
            top[g] = W.row_most(WideRows::most(s0[g]));
        }
        // the first tile's maxima are the running ones, with nothing to scale
        if (!inside.of(2 * P.i0)) W.hide(s0, top, P.start(P.i0), h);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            W.m[g] = top[g] * W.c;
            W.settle(g);
        }
        int now = 0;
#pragma unroll 1
        for (int i = P.i0; i < P.i1; ++i) {
            W.hold();
            const int next = (now + WIDE_STAGE) & (4 * WIDE_STAGE - 1);
            // The next stage's loads are all but the last eight.  Behind the barrier it is there for all waves, and nobody reads the one before this any more.
            stage_wait<8>();
            lds_barrier();
            aim(i + 3);
            const int later = (now + 3 * WIDE_STAGE) & (4 * WIDE_STAGE - 1);
            if (i + 1 < P.i1 && !whole.of(i + 1)) {
                clean_values<bf16_t>(lds + next + WIDE_VALUES, WIDE_VALUES, odd, tid);
                lds_barrier();
            }
            W.tile(
                s0, s1, top, k, ka + next, 0, va + now, 0, [&]() { if (!inside.of(2 * i)) W.hide(s0, top, P.start(i), h); }, [&](auto x) { load(x, later); });
            W.tile(
                s1, s0, top, k, ka + next, 32 * WIDE_ROW, va + now, 32 * WIDE_ROW, [&]() { if (!inside.of(2 * i + 1)) W.hide(s1, top, P.start(i) + 32, h); },
                [](auto) {});
            now = next;
        }
        stage_wait<0>();             // (what was asked for twice, at the end)
        // The Values that were left out join the rows that see them: a sum of one is it, or NaN.
        if (*odd) {
#pragma unroll 1
            for (int i = P.i0; i < P.i1; ++i) {
                const int j0 = P.start(i);
                if (!P.edge(j0)) continue;
#pragma unroll 1
                for (int j = j0; j < min(j0 + WIDE_TOKENS, P.len); ++j)
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

    // Rows go out through LDS, sixteen lanes a row: as they lie in the accumulators each store would be 16 bytes of 32 rows.
    if (splits == 1) {
        lds_barrier();               // (nobody reads a stage any more)
        char* own = lds + wave * WIDE_STAGE;
        int64_t* places = (int64_t*)(own + 64 * WIDE_ROW);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const float l = halves_sum(W.l[g][0] + W.l[g][1]), inv = l == 0.f ? 0.f : 1.f / l;
            if (h == 0)
                places[32 * g + n] = P.row0 + 64 * wave + 32 * g + n < P.rows ? (int64_t)P.b * A.o_sb + (int64_t)head[g] * A.o_sh + (int64_t)tok[g] * A.o_st : -1;
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = l == 0.f ? 0.f : W.O[g][c][4 * q + e] * inv;
                    *(uint2*)(own + (32 * g + n) * WIDE_ROW + 16 * ((4 * c + q) ^ (n & 15)) + 8 * h) =
                        make_uint2(__builtin_bit_cast(uint32_t, (bf16x2){(__bf16)x[0], (__bf16)x[1]}), __builtin_bit_cast(uint32_t, (bf16x2){(__bf16)x[2], (__bf16)x[3]}));
                }
        }
#pragma unroll 4
        for (int x = 0; x < 16; ++x) {
            const int r = 4 * x + (lane >> 4);
            const int64_t place = places[r];
            const uint4 d = *(const uint4*)(own + r * WIDE_ROW + 16 * ((lane & 15) ^ (r & 15)));
            if (place >= 0) *(uint4*)((bf16_t*)A.out + place + 8 * (lane & 15)) = d;
        }
        return;
    }
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        const float l = halves_sum(W.l[g][0] + W.l[g][1]);
        const int row = P.row0 + 64 * wave + 32 * g + n;
        if (row >= P.rows) continue;
        const size_t slot = ((size_t)u * A.n * A.G + row) * A.S + split;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(f32x4*)(A.ws_acc + slot * D + 32 * c + 8 * q + 4 * h) = (f32x4){W.O[g][c][4 * q], W.O[g][c][4 * q + 1], W.O[g][c][4 * q + 2], W.O[g][c][4 * q + 3]};
        if (h == 0) { A.ws_m[slot] = W.m[g]; A.ws_l[slot] = l; }
    }
}

// ---- bf16, few rows ------------------------------------------------------------------
// 32 rows a work-group, whose four waves take a tile of 32 tokens each in turn: what a short prompt waits for is its chain of round trips, so nothing in it is
// waited for by four waves, every wave has its next tile on the way into its own part of LDS, and the waves meet once, to join their sums. 40 tokens of 8 units of 4 heads behind 1000, a window
// of 512: 7.6 us and 3.6 for the fold (256 rows a work-group: 18.8 and 3.9); a work-group takes 9 us, and 1.35 for each four tiles.
constexpr int FEW_ROWS = 32, FEW_TOKENS = 32, FEW_TILE = 2 * FEW_TOKENS * 256, FEW_WAVE = 2 * FEW_TILE, FEW_LDS = 4 * FEW_WAVE;
constexpr int FEW_PARK = 33;     // 32 rows' quads, and one: lanes that write quads side by side meet other banks

// The fold of the four waves' sums of 32 rows, parked: 32 lanes a row, four channels each.
template <typename T>
__device__ __forceinline__ void few_fold(const PrefillArgs& A, const Prompt<FEW_TOKENS>& P, int u, int split, int splits, const f32x4* park, float (&sm_m)[4][32], float (&sm_l)[4][32],
                                         float m, float l, int tid)
{
    if ((tid & 32) == 0) {
        sm_m[tid >> 6][tid & 31] = m;
        sm_l[tid >> 6][tid & 31] = l;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int r = 8 * k + (tid >> 5), p = tid & 31, row = P.row0 + r;
        if (row >= P.rows) continue;
        const float M = fmaxf(fmaxf(sm_m[0][r], sm_m[1][r]), fmaxf(sm_m[2][r], sm_m[3][r]));
        f32x4 acc = (f32x4){0.f, 0.f, 0.f, 0.f};
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float x = partial_weight(sm_m[w][r], sm_l[w][r], M);
            acc += park[(w * 32 + p) * FEW_PARK + r] * x;
            sum = fmaf(sm_l[w][r], x, sum);
        }
        if (splits == 1) {
            const int t = P.token(A, row), hd = P.hk * A.G + row - t * A.G;
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = sum == 0.f ? 0.f : acc[e] * inv;
            T* o = (T*)A.out + (int64_t)P.b * A.o_sb + (int64_t)hd * A.o_sh + (int64_t)t * A.o_st + 4 * p;
            if constexpr (sizeof(T) == 4) *(f32x4*)o = (f32x4){x[0], x[1], x[2], x[3]};
            else *(uint2*)o = make_uint2(__builtin_bit_cast(uint32_t, (bf16x2){(__bf16)x[0], (__bf16)x[1]}), __builtin_bit_cast(uint32_t, (bf16x2){(__bf16)x[2], (__bf16)x[3]}));
        } else {
            const size_t slot = ((size_t)u * A.n * A.G + row) * A.S + split;
            *(f32x4*)(A.ws_acc + slot * D + 4 * p) = acc;
            if (p == 0) { A.ws_m[slot] = M; A.ws_l[slot] = sum; }
        }
    }
}

__global__ __launch_bounds__(256, 1) void attn_prompt_few(PrefillArgs A)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ float sm_m[4][32], sm_l[4][32];
    int block, split, splits, u;
    prompt_place(A, block, split, splits, u);
    const Prompt<FEW_TOKENS> P(A, u, block, split, splits, FEW_ROWS);
    if (P.row0 >= P.rows) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, n = lane & 31;
    const int mine = min(P.row0 + n, P.rows - 1), tok = P.token(A, mine), head = P.hk * A.G + mine - tok * A.G;
    const Sight sight{P.first + tok, P.window, P.sinks};
    const bf16_t* kp = (const bf16_t*)A.k + (int64_t)P.b * A.sb + (int64_t)P.hk * A.sh;
    const bf16_t* vp = (const bf16_t*)A.v + (int64_t)P.b * A.sb + (int64_t)P.hk * A.sh;

    bf16x8 q[8];
    const bf16_t* qp = (const bf16_t*)A.q + (int64_t)P.b * A.q_sb + (int64_t)head * A.q_sh + (int64_t)tok * A.q_st;
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = *(const bf16x8*)(qp + 16 * i + 8 * h);

    char* own = lds + wave * FEW_WAVE;
    const uint32_t base = __builtin_amdgcn_readfirstlane(lds_address(own));
    // rows 4 x + lane / 16 of a tile, x < 8
    auto fetch = [&](int i, int buf) {
        const int j = P.start(i);
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const int token = 4 * x + (lane >> 4);
            const int64_t at = (int64_t)min(j + token, P.len - 1) * A.st;
            load_to_lds(kp + at + 8 * key_slot(token, lane & 15), base + buf + 1024 * x);
            load_to_lds(vp + at + 8 * value_slot(token, lane & 15), base + buf + FEW_TILE / 2 + 1024 * x);
        }
    };
    int ka[8], va[4];
#pragma unroll
    for (int i = 0; i < 8; ++i) ka[i] = n * 256 + 16 * key_slot(n, 2 * i + h);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 4 * h + ((lane & 15) >> 2);
        va[i] = FEW_TILE / 2 + r * 256 + 16 * value_slot(r, 4 * i + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + 8 * (lane & 1);
    }
    float m = ROWS_NEG_INF, l = 0.f;
    f32x16 O[4];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[c][i] = 0.f;
    bool odd = false;
    int now = 0;
    if (P.i0 + wave < P.i1) fetch(P.i0 + wave, 0);
#pragma unroll 1
    for (int i = P.i0 + wave; i < P.i1; i += 4) {
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");     // (nothing reads the other tile's place any more)
        if (i + 4 < P.i1) {
            fetch(i + 4, now ^ FEW_TILE);
            stage_wait<16>();
        } else {
            stage_wait<0>();
        }
        const int j0 = P.start(i);
        const char* at = own + now;
        f32x16 s;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
        for (int x = 0; x < 8; ++x) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8*)(at + ka[x]), q[x], s, 0, 0, 0);
        const bool edge = P.edge(j0);
        if (edge) sight.hide(s, j0 + 4 * h);
        float mt = s[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mt = fmaxf(mt, s[e]);
        mt = halves_max(mt) * A.scale_log2;
        if (__any(mt > m + 8.f)) {
            const float m_new = fmaxf(m, mt), alpha = m > ROWS_NEG_INF ? rows_exp2(m - m_new) : 1.f;
            l *= alpha;
#pragma unroll
            for (int c = 0; c < 4; ++c) O[c] *= alpha;
            m = m_new;
        }
        const float ref = m > ROWS_NEG_INF ? m : 0.f;
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s[e] = rows_exp2(fmaf(s[e], A.scale_log2, -ref));
            sum += s[e];
        }
        l += sum;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = __builtin_bit_cast(uint32_t, (bf16x2){(__bf16)s[8 * t + 2 * e], (__bf16)s[8 * t + 2 * e + 1]});
            const bf16x8 p = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t a[4];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    typedef __attribute__((address_space(3))) s16x4* Lds;
                    const uint2 d = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + va[c] + (16 * t + 8 * x) * 256)));
                    a[2 * x] = d.x;
                    a[2 * x + 1] = d.y;
                }
                if (edge) {                  // Values that are no numbers count as 0 where they may be masked
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t keep = (odd_value(a[e]) ? 0u : 0xffff0000u) | (odd_value(a[e] << 16) ? 0u : 0xffffu);
                        odd |= keep != ~0u;
                        a[e] &= keep;
                    }
                }
                O[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, make_uint4(a[0], a[1], a[2], a[3])), p, O[c], 0, 0, 0);
            }
        }
        now ^= FEW_TILE;
    }
    // ... and join the rows that see them behind the loop: a sum of one is it, or NaN.
    if (__any(odd)) {
#pragma unroll 1
        for (int i = P.i0 + wave; i < P.i1; i += 4) {
            const int j0 = P.start(i);
            if (!P.edge(j0)) continue;
#pragma unroll 1
            for (int j = j0; j < min(j0 + FEW_TOKENS, P.len); ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint2 d = *(const uint2*)(vp + (int64_t)j * A.st + 32 * c + 8 * e + 4 * h);
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const uint32_t w = x < 2 ? d.x : d.y, v = x & 1 ? w & 0xffff0000u : w << 16;
                            O[c][4 * e + x] += odd_value(v) && sight.of(j) ? __uint_as_float(v) : 0.f;
                        }
                    }
        }
    }

    // the four waves' sums: quads of channels, [wave][channels 4 p ..+3][row]
    l = halves_sum(l);
    __syncthreads();
    f32x4* park = (f32x4*)lds;
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            park[(wave * 32 + 8 * c + 2 * e + h) * FEW_PARK + n] = (f32x4){O[c][4 * e], O[c][4 * e + 1], O[c][4 * e + 2], O[c][4 * e + 3]};
    few_fold<bf16_t>(A, P, u, split, splits, park, sm_m, sm_l, m, l, tid);
}

// ---- fp32, few rows ------------------------------------------------------------------
// The same with fp32 products: a wave's tile is 32 KB of LDS, so it has one, whose Keys' half is asked for again as soon as the scores are there, and whose Values' half behind the products.
// 40 tokens of 8 units of 4 heads behind 1000, a window of 512: 16.6 us with the fold (128 rows a work-group: 21.9), 100 tokens 11.2 (15.0), 512 units of 4 heads, 4 tokens on 500 62 (131).
// Bound by round trips, and by the fp32 products, 8200 cycles a tile.
constexpr int FEW32_VALUES = FEW_TOKENS * F32_ROW, FEW32_WAVE = 2 * FEW32_VALUES, FEW32_LDS = 4 * FEW32_WAVE;

__global__ __launch_bounds__(256, 1) void attn_prompt_few_f32(PrefillArgs A)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ float sm_m[4][32], sm_l[4][32];
    int block, split, splits, u;
    prompt_place(A, block, split, splits, u);
    const Prompt<FEW_TOKENS> P(A, u, block, split, splits, FEW_ROWS);
    if (P.row0 >= P.rows) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, n = lane & 31;
    const int mine = min(P.row0 + n, P.rows - 1), tok = P.token(A, mine), head = P.hk * A.G + mine - tok * A.G;
    const Sight sight{P.first + tok, P.window, P.sinks};
    const float* kp = (const float*)A.k + (int64_t)P.b * A.sb + (int64_t)P.hk * A.sh;
    const float* vp = (const float*)A.v + (int64_t)P.b * A.sb + (int64_t)P.hk * A.sh;

    f32x4 q[16];
    const float* qp = (const float*)A.q + (int64_t)P.b * A.q_sb + (int64_t)head * A.q_sh + (int64_t)tok * A.q_st;
#pragma unroll
    for (int i = 0; i < 16; ++i) q[i] = *(const f32x4*)(qp + 8 * i + 4 * h);

    char* own = lds + wave * FEW32_WAVE;
    const uint32_t base = __builtin_amdgcn_readfirstlane(lds_address(own));
    // rows 2 x + lane / 32 of a tile, x < 16
    auto fetch = [&](const float* from, int i, int half) {
        const int j = P.start(i);
#pragma unroll
        for (int x = 0; x < 16; ++x) load_to_lds(from + (int64_t)min(j + 2 * x + h, P.len - 1) * A.st + 4 * slot_of(2 * x + h, n), base + half + 2 * F32_ROW * x);
    };
    int ka[4], va[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        ka[i] = n * F32_ROW + 16 * slot_of(n, 2 * i + h);
        va[i] = FEW32_VALUES + (4 * h + i) * F32_ROW + 16 * slot_of(4 * h + i, n);
    }
    float m = ROWS_NEG_INF, l = 0.f;
    f32x16 O[4];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[c][i] = 0.f;
    bool odd = false;
    if (P.i0 + wave < P.i1) {
        fetch(kp, P.i0 + wave, 0);
        fetch(vp, P.i0 + wave, FEW32_VALUES);
    }
#pragma unroll 1
    for (int i = P.i0 + wave; i < P.i1; i += 4) {
        const int j0 = P.start(i);
        const bool edge = P.edge(j0), more = i + 4 < P.i1;
        stage_wait<16>();                // (all but the Values)
        f32x16 s;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            const f32x4 a = *(const f32x4*)(own + ka[x & 3] + 128 * (x >> 2));
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], q[x][e], s, 0, 0, 0);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");     // (nothing reads the Keys any more)
        if (more) fetch(kp, i + 4, 0);
        if (edge) sight.hide(s, j0 + 4 * h);
        float mt = s[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mt = fmaxf(mt, s[e]);
        mt = halves_max(mt) * A.scale_log2;
        if (__any(mt > m + 8.f)) {
            const float m_new = fmaxf(m, mt), alpha = m > ROWS_NEG_INF ? rows_exp2(m - m_new) : 1.f;
            l *= alpha;
#pragma unroll
            for (int c = 0; c < 4; ++c) O[c] *= alpha;
            m = m_new;
        }
        const float ref = m > ROWS_NEG_INF ? m : 0.f;
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s[e] = rows_exp2(fmaf(s[e], A.scale_log2, -ref));
            sum += s[e];
        }
        l += sum;
        if (more) stage_wait<16>();      // (all but the next Keys)
        else stage_wait<0>();
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            f32x4 a = *(const f32x4*)(own + va[e & 3] + 8 * F32_ROW * (e >> 2));
            if (edge) {                  // Values that are no numbers count as 0 where they may be masked
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const bool no = odd_value(__float_as_uint(a[c]));
                    odd |= no;
                    a[c] = no ? 0.f : a[c];
                }
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) O[c] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[c], s[e], O[c], 0, 0, 0);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");     // (nor the Values)
        if (more) fetch(vp, i + 4, FEW32_VALUES);
    }
    // ... and join the rows that see them behind the loop: a sum of one is it, or NaN.  (O[c][e] is channel 4 (8 (e / 4) + 4 h + e % 4) + c)
    if (__any(odd)) {
#pragma unroll 1
        for (int i = P.i0 + wave; i < P.i1; i += 4) {
            const int j0 = P.start(i);
            if (!P.edge(j0)) continue;
#pragma unroll 1
            for (int j = j0; j < min(j0 + FEW_TOKENS, P.len); ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const f32x4 v = *(const f32x4*)(vp + (int64_t)j * A.st + 4 * (8 * (e >> 2) + 4 * h + (e & 3)));
#pragma unroll
                    for (int c = 0; c < 4; ++c) O[c][e] += odd_value(__float_as_uint(v[c])) && sight.of(j) ? v[c] : 0.f;
                }
        }
    }

    // the four waves' sums: quads of channels, [wave][channels 4 p ..+3][row]
    l = halves_sum(l);
    __syncthreads();
    f32x4* park = (f32x4*)lds;
#pragma unroll
    for (int e = 0; e < 16; ++e) park[(wave * 32 + 8 * (e >> 2) + 4 * h + (e & 3)) * FEW_PARK + n] = (f32x4){O[0][e], O[1][e], O[2][e], O[3][e]};
    few_fold<float>(A, P, u, split, splits, park, sm_m, sm_l, m, l, tid);
}

// The fold of the splits' partials, of the blocks that are in splits: 32 lanes a row, four channels each (see rows_merge).
template <typename T>
__global__ __launch_bounds__(256) void prompt_merge(PrefillArgs A)
{
    const int p = threadIdx.x & 31;
    // (all of these are below 2^31)
    const uint32_t first = (A.S > PREFILL_CUTS + 1 ? 0 : A.cut[0]) * A.rows, all = (uint32_t)A.n * A.G, x = blockIdx.x * 8 + (threadIdx.x >> 5), u = over(x, A.by_merged),
                   row = x - u * (all - first) + first;
    const int b = (int)over(u, A.by_hkv), hk = (int)u - b * A.Hkv;
    if (b >= A.B) return;
    const int fresh = min(max(A.n_dev ? A.n_dev[b] : A.n, 0), A.n);
    if (row >= (uint32_t)fresh * A.G) return;
    f32x4 num;
    float sum;
    const int64_t at = ((int64_t)u * all + row) * A.S;
    merge_row<4>(A.ws_m + at, A.ws_l + at, A.ws_acc + at * D, prompt_splits(A, (int)(row >> __builtin_ctz(A.rows))), 0, 1, p, num, sum);
    const int tok = (int)over(row, A.by_g), head = hk * A.G + (int)row - tok * A.G;
    const float inv = 1.f / sum;
    T* o = (T*)A.out + (int64_t)b * A.o_sb + (int64_t)head * A.o_sh + (int64_t)tok * A.o_st + 4 * p;
#pragma unroll
    for (int e = 0; e < 4; ++e) st_elem(o + e, sum == 0.f ? 0.f : num[e] * inv);
}

}  // namespace

hipError_t launch_prefill(int dtype, const PrefillArgs& args, hipStream_t st)
{
    PrefillArgs a = args;
    const int64_t units = (int64_t)a.B * a.Hkv;
    int64_t groups = units * a.blocks * a.S, merged = units * a.n * a.G;
    if (a.S <= PREFILL_CUTS + 1) {
        groups = units * a.blocks;
        for (int i = 0; i < PREFILL_CUTS; ++i) groups += units * (a.blocks - a.cut[i]);
        merged -= units * a.cut[0] * a.rows;
    }
    a.by_units = divisor((uint32_t)units);
    a.by_hkv = divisor((uint32_t)a.Hkv);
    a.by_g = divisor((uint32_t)a.G);
    a.by_merged = divisor(a.S > 1 ? (uint32_t)(merged / units) : 1);
    if (groups > 0x7fffffff || (merged + 7) / 8 > 0x7fffffff) return hipErrorInvalidValue;
    auto go = [&](void (*kernel)(PrefillArgs), int lds, int threads = 256) {
        const hipError_t e = allow_dynamic_lds((const void*)kernel, lds);
        if (e != hipSuccess) return e;
        kernel<<<(uint32_t)groups, threads, lds, st>>>(a);
        return hipGetLastError();
    };
    hipError_t e;
    if (dtype == 0 && a.rows == PARTS_ROWS) e = go(attn_prompt_parts, PARTS_LDS + 16, 512);
    else if (dtype == 0 && a.rows == FEW_ROWS) e = go(attn_prompt_few_f32, FEW32_LDS);
    else if (dtype == 0) e = go(attn_prompt_f32, 2 * F32_STAGE + 16);
    else if (a.rows == FEW_ROWS) e = go(attn_prompt_few, FEW_LDS);
    else e = go(attn_prompt_wide, WIDE_LDS + 16);
    if (e != hipSuccess || a.S == 1) return e;
    const uint32_t g = (uint32_t)((merged + 7) / 8);
    if (dtype == 0) prompt_merge<float><<<g, 256, 0, st>>>(a);
    else prompt_merge<bf16_t><<<g, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace rk
