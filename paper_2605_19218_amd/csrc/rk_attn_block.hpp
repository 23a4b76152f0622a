// Attention of many query rows a KV head (more than 32: trees of drafts on grouped-query layers), bf16 rows, over the packed bf16 or the 8-bit
// cache.  The mathematics, the splits and the partials are those of attn_rows (rk_attn_rows.hpp); what differs is who holds what:
//
// attn_rows gives every wave other tokens and the same rows, which is right while memory is the bound.  With many rows the matrix cores are, and a
// wave that keeps 64 rows' accumulators beside its tiles needs more registers than there are.  Here a work-group stages the tokens in LDS, once for
// all its rows, as operands of v_mfma_f32_32x32x16_bf16, and a wave owns 32 rows: 64 registers of accumulators, so that two waves
// share a SIMD and one's softmax runs under the other's products.  A tile of 32 tokens read from LDS (12 KB at r = 64) feeds 24 instructions of 32
// cycles.  8-bit codes become bf16 on their way into LDS, once for the work-group.  What is requested of memory is DEPTH stages ahead, in registers: a
// round trip to HBM takes as long as two or three stages' arithmetic (three stages do not fit beside 128 channels).
// What bounds it: no one thing.  Of a SIMD's cycles the products take 34 %, the vector instructions between them (weights, their two parts, codes) 28 % over the packed and
// 38 over the 8-bit cache, and 38 and 28 % neither: waits at a stage's barrier, and for LDS in front of it.  112 rows x 32 units x 16384 tokens, r = 64, 1024 text rows: 65 us, 57
// GFLOP issued, 870 TFLOP/s; 448 rows over 8 bits: 214 to 219 us, 187 GFLOP, 860.  (Eight waves behind one barrier took 221 us for what two work-groups of four took 209; one bf16 part of the weights would save a third of the
// products, and the error would be that of the result's own rounding.)
//   S^T[token][row] = K . q~^T, O^T[channel][row] = V^T . P^T: lane (h, n) = (lane / 32, lane % 32) holds row n's scores of tokens 8 j + 4 h ..+3,
//   j < 4.  Step s of the second product takes j = s and j = s + 2 of them as they are: tokens 4 g ..+3 and 16 + 4 g ..+3, g = 2 s + h, which is a
//   16-byte piece of the Value cache; a Key operand is one of the Key cache.  So the stages are copied piece by piece.
// RW: row groups of a work-group, 32 rows each; the 4 / RW waves of a group take a tile of a stage each.  128 rows; over 8 bits also 64, whose codes take
// as long to convert for fewer rows but leave no wave idle.
#pragma once
#include "rk_attn_rows.hpp"

namespace rk {

constexpr int BLOCK_NT = 256;                            // four waves, a SIMD each; two work-groups a compute unit
constexpr int BLOCK_V = 16384, BLOCK_BUF = 32768;       // in a buffer: Keys of up to 64 tokens and 128 channels, their Values behind them
constexpr int BLOCK_LDS = 2 * BLOCK_BUF + 2 * 512 + 64; // two buffers; steps of Keys and Values; flags

__device__ __forceinline__ float halves_sum(float v)
{
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float halves_max(float v)
{
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// places in a tile: octet o of token m; channel 16 cb + n, tokens 4 g ..+3 and 16 + 4 g ..+3
__device__ __forceinline__ int key_place(int o, int m) { return o * 512 + m * 16; }
__device__ __forceinline__ int value_place(int cb, int g, int n) { return (cb >> 1) * 2048 + g * 512 + ((cb & 1) * 16 + n) * 16; }

// two weights as bf16 head and remainder: heads cut off, not rounded, which the remainder (8 bits of what is left) makes up for
__device__ __forceinline__ void cut_bf16x2(float a, float b, uint32_t& hi, uint32_t& lo)
{
    const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
    hi = __builtin_amdgcn_perm(y, x, 0x07060302u);
    const float ra = a - __uint_as_float(x & 0xffff0000u), rb = b - __uint_as_float(y & 0xffff0000u);
    lo = __builtin_bit_cast(uint32_t, (bf16x2){(__bf16)ra, (__bf16)rb});
}

struct BlockState {
    float m, l;
    float limit;                 // what a score may exceed `m` by before it moves: 2^8, or nothing before the first score
    f32x16 below;                // - m in every place (0 before the first score): what the first product starts from
    f32x16 O[4];
    __device__ __forceinline__ void clear()
    {
        m = limit = ROWS_NEG_INF;
        l = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) below[i] = 0.f;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) O[c][i] = 0.f;
    }
    // s: scores of a tile, with `below` added
    __device__ __forceinline__ void weigh(f32x16& s)
    {
        float mt = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mt = fmaxf(mt, s[i]);
        if (__any(mt > limit)) {
            const float m_new = fmaxf(m, halves_max(mt) - below[0]);
            const float alpha = m > ROWS_NEG_INF ? rows_exp2(m - m_new) : 0.f, ref = m_new > ROWS_NEG_INF ? m_new : 0.f;
            const float down = ref + below[0];
            l *= alpha;
#pragma unroll
            for (int c = 0; c < 4; ++c) O[c] *= alpha;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[i] -= down;
                below[i] = -ref;
            }
            m = m_new;
            limit = m_new > ROWS_NEG_INF ? 8.f : ROWS_NEG_INF;
        }
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[i] = rows_exp2(s[i]);
            sum += s[i];
        }
        l += sum;
    }
    // P . V of a tile: vt [channel block][step][lane]
    __device__ __forceinline__ void accumulate(const f32x16& p, const char* vt, int lane)
    {
        bf16x8 w[2][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) cut_bf16x2(p[4 * t + 8 * (i >> 1) + 2 * (i & 1)], p[4 * t + 8 * (i >> 1) + 2 * (i & 1) + 1], hi[i], lo[i]);
            w[t][0] = __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
            w[t][1] = __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const bf16x8 v = *(const bf16x8*)(vt + c * 2048 + t * 1024 + lane * 16);
                O[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w[t][1], O[c], 0, 0, 0);
                O[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w[t][0], O[c], 0, 0, 0);
            }
    }
    // A draft's Value v (this lane's four channels of each eight) where it is no number, for a row that sees it (see attn_rows).
    __device__ __forceinline__ void add_odd(const bf16_t* v, bool seen)
    {
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint2 d = *(const uint2*)(v + 32 * c + 8 * q);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t x = e & 1 ? (e < 2 ? d.x : d.y) & 0xffff0000u : (e < 2 ? d.x : d.y) << 16;
                    O[c][4 * q + e] += seen && (x & 0x7f800000u) == 0x7f800000u ? __uint_as_float(x) : 0.f;
                }
            }
    }
};

// TG tiles of the cache on their way into LDS: [tile][octet][token] and, BLOCK_V behind, [tile][channel block][step][lane].  A wave's pieces lie in
// one tile each, so that an address is a uniform base and an offset that never changes.  (`last`: the sequence's last tile, taken instead of one
// behind it.)
template <int TG>
__device__ __forceinline__ int tile_of(int s, int t, int last) { return TG == 1 ? s : min(TG * s + t, last); }
template <int FMT, int R, int TG> struct CacheStage;
template <int R>
struct CacheStage<ROWS_BF16, R, 1> {
    static constexpr int KP = 4 * R, NK = (KP + BLOCK_NT - 1) / BLOCK_NT, DEPTH = R > 96 ? 2 : 3;
    uint4 k[NK], v[2];
    // tile s of the sequence
    __device__ __forceinline__ void load(const char* Ku, const char* Vu, int s, int, int rp, int tid, int)
    {
#pragma unroll
        for (int j = 0; j < NK; ++j) {           // piece: [octet][token]
            const int p = (BLOCK_NT * j + tid) % KP, m = p & 31, o = p >> 5;
            k[j] = *(const uint4*)(Ku + (size_t)s * (64 * rp) + (uint32_t)((m >> 4) * (32 * rp) + (8 * o < rp ? o : 0) * 256 + (m & 15) * 16));
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) v[j] = *(const uint4*)(Vu + (size_t)s * 8192 + (uint32_t)(j * 4096 + tid * 16));
    }
    // `left`: tokens of the tile that exist; Values behind them may be anything
    __device__ __forceinline__ void store(char* buf, float*, int left, int tid)
    {
#pragma unroll
        for (int j = 0; j < NK; ++j)
            if (BLOCK_NT * (j + 1) <= KP || BLOCK_NT * j + tid < KP) *(uint4*)(buf + (BLOCK_NT * j + tid) * 16) = k[j];
        const int n = tid & 15, g = (tid >> 4) & 3;
        if (left < 32) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                uint32_t x[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = 16 * (i >> 1) + 4 * g + 2 * (i & 1);
                    x[i] &= t + 1 < left ? ~0u : t < left ? 0xffffu : 0u;
                }
                v[j] = make_uint4(x[0], x[1], x[2], x[3]);
            }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) *(uint4*)(buf + BLOCK_V + value_place(4 * j + (tid >> 6), g, n)) = v[j];
    }
};
template <int R, int TG>
struct CacheStage<ROWS_Q8_BF16, R, TG> {
    static constexpr int KP = TG * 2 * R, NK = (KP + BLOCK_NT - 1) / BLOCK_NT, DEPTH = 3;
    uint4 k[NK], v[TG];
    uint32_t step;
    __device__ __forceinline__ void load(const char* Ku, const char* Vu, int s, int last, int rp, int tid, int wave)
    {
        const size_t kblk = q8_kblock(rp);
#pragma unroll
        for (int j = 0; j < NK; ++j) {           // piece: [tile][octet][token n, and 16 + n]
            const int tile = min((BLOCK_NT * j + 64 * wave) / (2 * R), TG - 1), p = (BLOCK_NT * j + tid) % (2 * R), n = p & 15, o = p >> 4;
            k[j] = *(const uint4*)(Ku + (size_t)tile_of<TG>(s, tile, last) * kblk + (uint32_t)((8 * o < rp ? o : 0) * 256 + n * 16));
        }
#pragma unroll
        for (int j = 0; j < TG; ++j) v[j] = *(const uint4*)(Vu + (size_t)tile_of<TG>(s, j, last) * 4096 + (uint32_t)(tid * 16));
        const int a = TG * s, b = tile_of<TG>(s, TG - 1, last);
        step = *(const uint32_t*)(Ku + (size_t)a * kblk + (uint32_t)(32 * rp + (tid & 32 ? (b - a) * (int)kblk : 0) + (tid & 31) * 4));
    }
    // `left`: tokens of the stage that exist
    __device__ __forceinline__ void store(char* buf, float* steps, int left, int tid)
    {
#pragma unroll
        for (int j = 0; j < NK; ++j) {
            const int p = BLOCK_NT * j + tid, n = p & 15, o = p >> 4;       // (octets of the tiles one after another)
            if (BLOCK_NT * (j + 1) <= KP || p < KP) {
                *(uint4*)(buf + key_place(o, n)) = __builtin_bit_cast(uint4, codes_bf16(k[j].x, k[j].y));
                *(uint4*)(buf + key_place(o, 16 + n)) = __builtin_bit_cast(uint4, codes_bf16(k[j].z, k[j].w));
            }
        }
        const int n = tid & 15, g = (tid >> 4) & 3, cp = tid >> 6;
#pragma unroll
        for (int j = 0; j < TG; ++j) {
            char* to = buf + BLOCK_V + j * 8192;
            *(uint4*)(to + value_place(2 * cp, g, n)) = __builtin_bit_cast(uint4, codes_bf16(v[j].x, v[j].y));
            *(uint4*)(to + value_place(2 * cp + 1, g, n)) = __builtin_bit_cast(uint4, codes_bf16(v[j].z, v[j].w));
        }
        asm volatile("" : "+v"(step));             // (waited for by all: a load that only some wait for is waited for with all others, later)
        if (tid < 32 * TG) {
            steps[tid] = __uint_as_float(step << 16);
            steps[64 + tid] = tid < left ? __uint_as_float(step & 0xffff0000u) : 0.f;
        }
    }
};

// 64 full-width rows: threads 0..127 take the Keys, the others the Values, eight tokens by eight channels each, transposed in registers.
struct PlainStage {
    uint4 x[8];
    // token (of 64) of Value x[j]: the eight slots of (tile, g)
    static __device__ __forceinline__ int token(int tid, int j) { return 32 * ((tid >> 6) & 1) + 4 * ((tid >> 4) & 3) + (j < 4 ? j : 12 + j); }
    __device__ __forceinline__ void load(const bf16_t* kp, const bf16_t* vp, int64_t stride, int r0, int rows, int tid)
    {
        if (tid < 128) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                x[j] = *(const uint4*)(kp + (int64_t)min(r0 + (tid >> 2) + 32 * (j >> 2), rows - 1) * stride + 8 * ((tid & 3) + 4 * (j & 3)));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = *(const uint4*)(vp + (int64_t)min(r0 + token(tid, j), rows - 1) * stride + 8 * (tid & 15));
        }
    }
    // `odd` (drafts): a bit for each whose Value holds one that is no number; nothing of that goes into the product
    __device__ __forceinline__ void store(char* buf, uint32_t* odd, int r0, int rows, int tid)
    {
        if (tid < 128) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int t = (tid >> 2) + 32 * (j >> 2);
                *(uint4*)(buf + (t >> 5) * 8192 + key_place((tid & 3) + 4 * (j & 3), t & 31)) = x[j];
            }
        } else {
            const int co = tid & 15;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (r0 + token(tid, j) >= rows) x[j] = make_uint4(0, 0, 0, 0);
            if (odd) {
                bool any = false;
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) any |= (dword_of(x[j], i) & 0x7f800000u) == 0x7f800000u || (dword_of(x[j], i) & 0x7f80u) == 0x7f80u;
                if (any) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        uint32_t w[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            w[i] = dword_of(x[j], i);
                            w[i] &= ((w[i] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u) | ((w[i] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu);
                        }
                        if (w[0] != x[j].x || w[1] != x[j].y || w[2] != x[j].z || w[3] != x[j].w) atomicOr(odd + (token(tid, j) >> 5), 1u << (token(tid, j) & 31));
                        x[j] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
            }
            char* to = buf + BLOCK_V + ((tid >> 6) & 1) * 8192 + value_place(co >> 1, (tid >> 4) & 3, 8 * (co & 1));
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t sel = (k & 1) ? 0x07060302u : 0x05040100u;
                uint4 d;
                d.x = __builtin_amdgcn_perm(dword_of(x[1], k >> 1), dword_of(x[0], k >> 1), sel);
                d.y = __builtin_amdgcn_perm(dword_of(x[3], k >> 1), dword_of(x[2], k >> 1), sel);
                d.z = __builtin_amdgcn_perm(dword_of(x[5], k >> 1), dword_of(x[4], k >> 1), sel);
                d.w = __builtin_amdgcn_perm(dword_of(x[7], k >> 1), dword_of(x[6], k >> 1), sel);
                *(uint4*)(to + 16 * k) = d;
            }
        }
    }
};

template <int FMT, int R, int RW>
__global__ __launch_bounds__(BLOCK_NT, 2) void attn_block(RowsArgs A)
{
    constexpr bool Q8 = FMT == ROWS_Q8_BF16;
    constexpr int TG = 4 / RW;           // waves of a row group: each takes a tile of a stage
    extern __shared__ __attribute__((aligned(16))) char lds[];
    float* steps = (float*)(lds + 2 * BLOCK_BUF);                  // [buffer][Keys 64, Values 64]
    uint32_t* odd = (uint32_t*)(steps + 256);                      // a bit a draft

    int split, u, block;
    if (!rows_place(A, split, u, block)) return;
    const int b = u / A.Hkv, hk = u - b * A.Hkv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, n = lane & 31;
    const int S = A.Sv + A.Sr;
    if (block * 32 * RW >= A.T * A.G) return;
    const int row0 = (block * RW + wave % RW) * 32, row = row0 + n;
    const int rc = min(row, A.T * A.G - 1), tok = rc / A.G;
    const size_t at = (size_t)(b * A.T + tok) * A.Hq + hk * A.G + (rc - tok * A.G);

    // What needs no length is asked for first: a length is a round trip of its own.
    bf16x8 qf[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) qf[i] = *(const bf16x8*)((const bf16_t*)A.q + at * D + 16 * i + 8 * h);
    int live = A.T;                      // tokens whose rows are asked for
    auto drafts_of = [&]() { return A.draft_k ? min(max(A.n_drafts ? A.n_drafts[b] : A.T, 0), A.T) : 0; };
    BlockState st;                       // (cleared only in front of the loops: its registers are the prologue's until then)
    if (split < A.Sv) {
        const float* Ru = A.Rr + (size_t)u * D * A.r;
        constexpr int NF = R / 16;               // fragments of R_r^T a wave makes ready: 32 columns, 16 channels each
        float x[NF][8];
#pragma unroll
        for (int w = 0; w < NF; ++w) {
            const int f = 4 * w + wave, j = 32 * (f >> 3) + n;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[w][e] = Ru[(16 * (f & 7) + 8 * h + e) * A.r + min(j, A.r - 1)];
        }
        f32x4 dm[16];
        const float* dp = A.dmu ? A.dmu + (size_t)u * D : Ru;      // (any address that can be read, without a bias)
#pragma unroll
        for (int i = 0; i < 16; ++i) dm[i] = *(const f32x4_any*)(dp + 16 * (i >> 1) + 8 * h + 4 * (i & 1));
        __builtin_amdgcn_sched_barrier(0);
        if (A.draft_k) live = drafts_of();
        if (block * 32 * RW >= live * A.G) return;
        const bool active = row0 < live * A.G;                     // (a wave without rows helps with the staging)
        constexpr int DEPTH = CacheStage<FMT, R, TG>::DEPTH;
        const int len = __builtin_amdgcn_readfirstlane(min(max(A.seq_len[b], 0), A.cap)), stages = (len + 32 * TG - 1) / (32 * TG), last = (len + 31) / 32 - 1;
        const int s0 = (int)((int64_t)stages * split / A.Sv), s1 = (int)((int64_t)stages * (split + 1) / A.Sv);
        const size_t slab = slab_tokens(A.cap);
        const char* Ku = (const char*)A.Kc + (Q8 ? (size_t)u * (slab / 32) * q8_kblock(A.rp) : (size_t)u * slab * A.rp * 2);
        const char* Vu = (const char*)A.Vc + (size_t)u * slab * D * (Q8 ? 1 : 2);
        if (s0 < s1) {
            CacheStage<FMT, R, TG> X[DEPTH];
#pragma unroll
            for (int k = 0; k < DEPTH; ++k) {
                X[k].load(Ku, Vu, min(s0 + k, s1 - 1), last, A.rp, tid, wave);
                __builtin_amdgcn_sched_barrier(0);                 // (in this order, as the loop's waits count them)
            }
            // R_r^T as A operands, head and remainder, in LDS; then this wave's rows of q R_r
#pragma unroll
            for (int w = 0; w < NF; ++w) {
                const int f = 4 * w + wave, j = 32 * (f >> 3) + n;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[w][e] = j < A.r ? x[w][e] : 0.f;
                bf16x8 hi, lo;
                split_bf16x8(x[w], hi, lo);
                *(bf16x8*)(lds + (2 * f) * 1024 + lane * 16) = hi;
                *(bf16x8*)(lds + (2 * f + 1) * 1024 + lane * 16) = lo;
            }
            float bias = 0.f;
            if (A.dmu) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) bias = fmaf((float)qf[i][e], dm[2 * i + (e >> 2)][e & 3], bias);
                bias = halves_sum(bias) * A.scale_log2;
            }
            lds_barrier();
            bf16x8 qr[R / 16][2];
#pragma unroll
            for (int jb = 0; jb < R / 32; ++jb) {
                f32x16 acc;
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[i] = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bf16x8 hi = *(const bf16x8*)(lds + (2 * (8 * jb + i)) * 1024 + lane * 16);
                    const bf16x8 lo = *(const bf16x8*)(lds + (2 * (8 * jb + i) + 1) * 1024 + lane * 16);
                    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lo, qf[i], acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(hi, qf[i], acc, 0, 0, 0);
                }
                // row n's channels 8 j + 4 h ..+3 of the block -> 16 t + 8 h ..+7: the lanes' halves change places
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    float y[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[8 * t + e]), __float_as_uint(acc[8 * t + 4 + e]), false, false);
                        y[e] = __uint_as_float(w[0]) * A.scale_log2;
                        y[4 + e] = __uint_as_float(w[1]) * A.scale_log2;
                    }
                    split_bf16x8(y, qr[2 * jb + t][0], qr[2 * jb + t][1]);
                }
            }
            lds_barrier();
            X[0].store(lds, steps, len - 32 * TG * s0, tid);
            lds_barrier();

            st.clear();
            int buf = 0;
            // one stage from LDS; the next out of X, and the one DEPTH behind that asked for.  (Past the end the last is asked for again.)
            auto pass = [&](CacheStage<FMT, R, TG>& next, CacheStage<FMT, R, TG>& mine, int s) {
                mine.load(Ku, Vu, min(s + DEPTH, s1 - 1), last, A.rp, tid, wave);
                const int tile = wave / RW, left = len - 32 * (TG * s + tile);
                if (active && left > 0) {
                    const char* kt = lds + buf * BLOCK_BUF + tile * (64 * R);
                    const char* vt = lds + buf * BLOCK_BUF + BLOCK_V + tile * 8192;
                    f32x16 p;
                    if constexpr (Q8) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) p[i] = 0.f;
                    } else {
                        p = st.below;
                    }
#pragma unroll
                    for (int i = 0; i < R / 16; ++i) {
                        if (i == R / 16 - 1 && A.rp < R) break;        // (no such channels)
                        const bf16x8 k = *(const bf16x8*)(kt + i * 1024 + lane * 16);
                        p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qr[i][1], p, 0, 0, 0);
                        p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qr[i][0], p, 0, 0, 0);
                    }
                    const float* ks = steps + buf * 128 + 32 * tile + 4 * h;
                    if constexpr (Q8) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const f32x4 w = *(const f32x4*)(ks + 8 * q);
#pragma unroll
                            for (int i = 0; i < 4; ++i) p[4 * q + i] = fmaf(p[4 * q + i], w[i], st.below[0]);
                        }
                    }
                    if (left < 32) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) p[i] = 8 * (i >> 2) + 4 * h + (i & 3) < left ? p[i] : ROWS_NEG_INF;
                    }
                    st.weigh(p);
                    if constexpr (Q8) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const f32x4 w = *(const f32x4*)(ks + 64 + 8 * q);
#pragma unroll
                            for (int i = 0; i < 4; ++i) p[4 * q + i] *= w[i];
                        }
                    }
                    st.accumulate(p, vt, lane);
                }
                buf ^= 1;
                next.store(lds + buf * BLOCK_BUF, steps + buf * 128, len - 32 * TG * (s + 1), tid);
                lds_barrier();
            };
#pragma unroll 1
            for (int s = s0; s < s1; s += DEPTH) {
#pragma unroll
                for (int k = 0; k < DEPTH; ++k) {
                    if (s + k >= s1) break;
                    pass(X[(k + 1) % DEPTH], X[k], s + k);
                }
            }
            // the bias joins only now, see attn_rows
            st.m += bias;
        } else {
            st.clear();
        }
    } else {
        const int drafts = drafts_of();
        if (A.draft_k) live = drafts;
        if (block * 32 * RW >= live * A.G) return;
        const bool active = row0 < live * A.G;
        st.clear();
        const int text = A.text_k ? min(max(A.text_len ? A.text_len[b] : A.text_max, 0), A.text_max) : 0;
        const int tt = (text + 63) / 64, stages = tt + (drafts > 0), k = split - A.Sv;
        const int s0 = (int)((int64_t)stages * k / A.Sr), s1 = (int)((int64_t)stages * (k + 1) / A.Sr);
        if (s0 < s1) {
            const bf16_t* tk = (const bf16_t*)A.text_k + (int64_t)b * A.text_sb + (int64_t)hk * A.text_sh;
            const bf16_t* tv = (const bf16_t*)A.text_v + (int64_t)b * A.text_sb + (int64_t)hk * A.text_sh;
            const bf16_t* dk = (const bf16_t*)A.draft_k + (int64_t)b * A.draft_sb + (int64_t)hk * A.draft_sh;
            const bf16_t* dv = (const bf16_t*)A.draft_v + (int64_t)b * A.draft_sb + (int64_t)hk * A.draft_sh;
            PlainStage X[2];
            auto load = [&](PlainStage& x, int s) {
                const bool own = s >= tt;
                x.load(own ? dk : tk, own ? dv : tv, own ? A.draft_st : A.text_st, own ? 0 : 64 * s, own ? drafts : text, tid);
            };
            auto store = [&](PlainStage& x, int s, int buf) {
                x.store(lds + buf * BLOCK_BUF, s >= tt && s < s1 ? odd : nullptr, s >= tt ? 0 : 64 * s, s >= tt ? drafts : text, tid);
            };
            load(X[0], s0);
            load(X[1], min(s0 + 1, s1 - 1));
            uint64_t mask = ~0ull;
            if (A.draft_k) mask = A.mask ? A.mask[(size_t)b * A.T + tok] : (2ull << tok) - 1;
            if (tid < 2) odd[tid] = 0;
            lds_barrier();
            store(X[0], s0, 0);
            lds_barrier();
            int buf = 0;
            auto pass = [&](PlainStage& next, PlainStage& mine, int s) {
                const bool own = s >= tt;
                load(mine, min(s + 2, s1 - 1));
                if (active) {
#pragma unroll 1
                    for (int tile = wave / RW; tile < 2; tile += TG) {
                        const char* kt = lds + buf * BLOCK_BUF + tile * 8192;
                        const char* vt = lds + buf * BLOCK_BUF + BLOCK_V + tile * 8192;
                        const int left = (own ? drafts : text - 64 * s) - 32 * tile;
                        if (left <= 0) break;
                        f32x16 p;
#pragma unroll
                        for (int i = 0; i < 16; ++i) p[i] = 0.f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8*)(kt + i * 1024 + lane * 16), qf[i], p, 0, 0, 0);
                        uint32_t word = own ? (uint32_t)(mask >> (32 * tile)) : ~0u;                // (drafts: two tiles at most)
                        if (left < 32) word &= (1u << left) - 1;
                        word >>= 4 * h;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const bool in = (word >> (8 * (i >> 2) + (i & 3))) & 1;
                            p[i] = in ? fmaf(p[i], A.scale_log2, st.below[0]) : ROWS_NEG_INF;
                        }
                        st.weigh(p);
                        st.accumulate(p, vt, lane);
                    }
                }
                buf ^= 1;
                store(next, s + 1, buf);
                lds_barrier();
            };
#pragma unroll 1
            for (int s = s0; s < s1; s += 2) {
                pass(X[1], X[0], s);
                if (s + 1 >= s1) break;
                pass(X[0], X[1], s + 1);
            }
            if (s1 > tt && active) {
                // (a tile's are added by the wave that took it)
#pragma unroll 1
                for (uint64_t left = ((uint64_t)odd[1] << 32) | odd[0]; left; left &= left - 1) {
                    const int j = __builtin_ctzll(left);
                    if ((j >> 5) % TG == wave / RW) st.add_odd(dv + (int64_t)j * A.draft_st + 4 * h, (mask >> j) & 1);
                }
            }
        }
    }

    // the waves of a row group: pairs of states, one of them parked in LDS
    st.l = halves_sum(st.l);
#pragma unroll
    for (int half = TG / 2; half > 0; half >>= 1) {
        const int part = wave / RW;
        float* park = (float*)lds + ((part % half) * RW + wave % RW) * (64 * 66) + lane;
        __syncthreads();
        if (part >= half && part < 2 * half) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int i = 0; i < 16; ++i) park[64 * (16 * c + i)] = st.O[c][i];
            park[64 * 64] = st.m;
            park[64 * 65] = st.l;
        }
        __syncthreads();
        if (part < half) {
            const float m2 = park[64 * 64], l2 = park[64 * 65], M = fmaxf(st.m, m2);
            const float w1 = partial_weight(st.m, st.l, M), w2 = partial_weight(m2, l2, M);
            st.m = M;
            st.l = st.l * w1 + l2 * w2;
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int i = 0; i < 16; ++i) st.O[c][i] = st.O[c][i] * w1 + park[64 * (16 * c + i)] * w2;
        }
    }
    if (wave >= RW || row >= live * A.G) return;
    if (S == 1) {
        const float inv = 1.f / st.l;
        bf16_t* o = (bf16_t*)A.out + at * D + 4 * h;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int e = 0; e < 4; ++e) st_elem(o + 32 * c + 8 * q + e, st.l == 0.f ? 0.f : st.O[c][4 * q + e] * inv);
    } else {
        const size_t slot = at * S + split;
        float* o = A.ws_acc + slot * D + 4 * h;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(f32x4*)(o + 32 * c + 8 * q) = (f32x4){st.O[c][4 * q], st.O[c][4 * q + 1], st.O[c][4 * q + 2], st.O[c][4 * q + 3]};
        if (h == 0) { A.ws_m[slot] = st.m; A.ws_l[slot] = st.l; }
    }
}

template <int FMT, int R, int RW>
static hipError_t launch_block_rw(dim3 grid, const RowsArgs& a, hipStream_t st)
{
    const hipError_t e = allow_dynamic_lds((const void*)attn_block<FMT, R, RW>, BLOCK_LDS);
    if (e != hipSuccess) return e;
    attn_block<FMT, R, RW><<<grid, BLOCK_NT, BLOCK_LDS, st>>>(a);
    return hipGetLastError();
}
// rows: of a work-group, 128, or over the 8-bit cache 64
template <int FMT, int R>
static hipError_t launch_block_r(int rows, dim3 grid, const RowsArgs& a, hipStream_t st)
{
    if constexpr (FMT == ROWS_Q8_BF16)
        if (rows == 64) return launch_block_rw<FMT, R, 2>(grid, a, st);
    return launch_block_rw<FMT, R, 4>(grid, a, st);
}
template <int FMT>
static hipError_t launch_block_fmt(const RowsArgs& a, int rows, hipStream_t st)
{
    const dim3 grid = rows_grid(a);
    if (!grid.x) return hipErrorInvalidValue;
    switch ((a.r + 31) / 32) {
        case 1: return launch_block_r<FMT, 32>(rows, grid, a, st);
        case 2: return launch_block_r<FMT, 64>(rows, grid, a, st);
        case 3: return launch_block_r<FMT, 96>(rows, grid, a, st);
        default: return launch_block_r<FMT, 128>(rows, grid, a, st);
    }
}

}  // namespace rk
