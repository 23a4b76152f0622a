// Attention of many query rows a KV head (more than 32: trees of drafts on grouped-query layers), bf16 rows, over the packed bf16 or the 8-bit
// cache.  The mathematics, the splits and the partials are those of attn_rows (rk_attn_rows.hpp); what differs is who holds what:
//
// attn_rows gives every wave other tokens and the same rows, which is right while memory is the bound.  From 64 rows on the matrix cores are, and a
// wave that keeps 64 rows' accumulators beside its tiles needs more registers than there are.  Here a work-group stages 64 tokens at a time in
// LDS, once for all its rows, as operands of v_mfma_f32_32x32x16_bf16, and a wave owns 32 rows: 64 registers of accumulators, so that two waves
// share a SIMD and one's softmax runs under the other's products.  A tile read from LDS (12 KB at r = 64) feeds 24 instructions of 32 cycles.
// 8-bit codes become bf16 on their way into LDS, once for the work-group.
//   S^T[token][row] = K . q~^T, O^T[channel][row] = V^T . P^T: lane (h, n) = (lane / 32, lane % 32) holds row n's scores of tokens 8 j + 4 h ..+3,
//   j < 4, and feeds them to the second product as they are: slot (h, e) of a 16-deep step is token (channel) 8 (e / 4) + 4 h + e % 4 in both
//   products, for both operands.  So the queries go from their rotation into the first product, and the weights into the second, without an
//   exchange between lanes; the staging puts halves of its 16-byte pieces where that order wants them.
// RW: row groups of a work-group (4: 128 rows; 2: 64 rows, and the waves of a row group take one of the two tiles each).
#pragma once
#include "rk_attn_rows.hpp"

namespace rk {

constexpr int BLOCK_BUF = 32768;                        // a stage: 64 tokens' Keys (up to 128 channels), then their Values
constexpr int BLOCK_LDS = 2 * BLOCK_BUF + 2 * 512 + 64; // two of them; steps of Keys and Values; flags

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

// where the Keys of octet o, token m of a 32-token tile go: its two halves, 512 bytes apart
__device__ __forceinline__ void put_key(char* kt, int o, int m, uint4 v)
{
    char* to = kt + (o >> 1) * 1024 + m * 16 + (o & 1) * 8;
    *(uint2*)to = make_uint2(v.x, v.y);
    *(uint2*)(to + 512) = make_uint2(v.z, v.w);
}
// the Values of channel 16 cb + n, tokens 4 g ..+3 and 16 + 4 g ..+3 of a tile
__device__ __forceinline__ void put_value(char* vt, int cb, int g, int n, uint4 v)
{
    char* to = vt + (cb >> 1) * 2048 + (g & 1) * 512 + ((cb & 1) * 16 + n) * 16 + (g >> 1) * 8;
    *(uint2*)to = make_uint2(v.x, v.y);
    *(uint2*)(to + 1024) = make_uint2(v.z, v.w);
}

struct BlockState {
    float m, l;
    f32x16 O[4];
    __device__ __forceinline__ void clear()
    {
        m = ROWS_NEG_INF;
        l = 0.f;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) O[c][i] = 0.f;
    }
    __device__ __forceinline__ void weigh(f32x16& s)
    {
        float mt = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mt = fmaxf(mt, s[i]);
        mt = halves_max(mt);
        if (__any(mt > m + 8.f)) {
            const float m_new = fmaxf(m, mt), alpha = m > ROWS_NEG_INF ? rows_exp2(m - m_new) : 0.f;
            l *= alpha;
#pragma unroll
            for (int c = 0; c < 4; ++c) O[c] *= alpha;
            m = m_new;
        }
        const float ref = m > ROWS_NEG_INF ? m : 0.f;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[i] = rows_exp2(s[i] - ref);
            sum += s[i];
        }
        l += sum;
    }
    // P . V of a tile: vt [channel block][step][lane]
    template <bool ODD>
    __device__ __forceinline__ void accumulate(const f32x16& p, const char* vt, int lane)
    {
        bf16x8 w[2][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float x[8] = {p[8 * t], p[8 * t + 1], p[8 * t + 2], p[8 * t + 3], p[8 * t + 4], p[8 * t + 5], p[8 * t + 6], p[8 * t + 7]};
            split_bf16x8(x, w[t][0], w[t][1]);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint4 d = *(const uint4*)(vt + c * 2048 + t * 1024 + lane * 16);
                if constexpr (ODD) {
                    uint32_t* x = (uint32_t*)&d;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        x[i] &= ((x[i] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u) | ((x[i] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu);
                }
                const bf16x8 v = __builtin_bit_cast(bf16x8, d);
                O[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w[t][1], O[c], 0, 0, 0);
                O[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w[t][0], O[c], 0, 0, 0);
            }
    }
    // Values that are no numbers, for the rows that see them (see attn_rows): bit i of `see` is score i
    __device__ __forceinline__ void add_odd(uint32_t see, const char* vt, int lane)
    {
#pragma unroll 1
        for (int kind = 0; kind < 3; ++kind)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                f32x16 cnt;
#pragma unroll
                for (int i = 0; i < 16; ++i) cnt[i] = 0.f;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const uint4 d = *(const uint4*)(vt + c * 2048 + t * 1024 + lane * 16);
                    uint32_t x[4], a[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t w = dword_of(d, i);
                        x[i] = (pick_odd(w << 16, kind) ? 0x3f80u : 0u) | (pick_odd(w & 0xffff0000u, kind) ? 0x3f800000u : 0u);
                        a[i] = ((see >> (8 * t + 2 * i)) & 1 ? 0x3f80u : 0u) | ((see >> (8 * t + 2 * i + 1)) & 1 ? 0x3f800000u : 0u);
                    }
                    cnt = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, make_uint4(x[0], x[1], x[2], x[3])),
                                                                  __builtin_bit_cast(bf16x8, make_uint4(a[0], a[1], a[2], a[3])), cnt, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) O[c][i] += cnt[i] > 0.f ? odd_value(kind) : 0.f;
            }
    }
};

// A stage of 64 tokens of the cache on its way into LDS.
template <int FMT, int R> struct CacheStage;
template <int R>
struct CacheStage<ROWS_BF16, R> {
    uint4 k[R / 32], v[4];
    // tiles 2 s and 2 s + 1 of the sequence (`last`: its last tile, taken instead of one behind it)
    __device__ __forceinline__ void load(const char* Ku, const char* Vu, int s, int last, int rp, int tid)
    {
        const int n = tid & 15, tb = (tid >> 4) & 3, o0 = tid >> 6;
        const char* kb = Ku + (size_t)(2 * min(2 * s + (tb >> 1), last) + (tb & 1)) * (32 * rp) + n * 16;
#pragma unroll
        for (int j = 0; j < R / 32; ++j) {
            const int o = 4 * j + o0;
            const uint4 x = *(const uint4*)(kb + (8 * o < rp ? o : 0) * 256);
            k[j] = 8 * o < rp ? x : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = *(const uint4*)(Vu + (size_t)min(2 * s + (j >> 1), last) * 8192 + (j & 1) * 4096 + tid * 16);
    }
    // `left`: tokens of the stage that exist
    __device__ __forceinline__ void store(char* kt, char* vt, float*, int left, int tid)
    {
        const int n = tid & 15, tb = (tid >> 4) & 3, o0 = tid >> 6;
#pragma unroll
        for (int j = 0; j < R / 32; ++j) put_key(kt + (tb >> 1) * (64 * R), 4 * j + o0, (tb & 1) * 16 + n, k[j]);
        const int g = (tid >> 4) & 3;
        if (left < 64) {             // Values behind the end may be anything
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t x[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (32 * (j >> 1) + (i < 4 ? 4 * g + i : 12 + 4 * g + i) >= left) x[i >> 1] &= i & 1 ? 0x0000ffffu : 0xffff0000u;
                v[j] = make_uint4(x[0], x[1], x[2], x[3]);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) put_value(vt + (j >> 1) * 8192, 4 * (j & 1) + (tid >> 6), g, n, v[j]);
    }
};
template <int R>
struct CacheStage<ROWS_Q8_BF16, R> {
    static constexpr int NK = (R + 63) / 64;
    uint4 k[NK], v[2];
    uint32_t step;
    __device__ __forceinline__ void load(const char* Ku, const char* Vu, int s, int last, int rp, int tid)
    {
        const size_t kblk = q8_kblock(rp);
#pragma unroll
        for (int j = 0; j < NK; ++j) {
            const int p = 256 * j + tid, n = p & 15, o = (p >> 4) % (R / 8), tile = min((p >> 4) / (R / 8), 1);
            k[j] = *(const uint4*)(Ku + (size_t)min(2 * s + tile, last) * kblk + (8 * o < rp ? o : 0) * 256 + n * 16);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) v[j] = *(const uint4*)(Vu + (size_t)min(2 * s + j, last) * 4096 + tid * 16);
        step = *(const uint32_t*)(Ku + (size_t)min(2 * s + ((tid >> 5) & 1), last) * kblk + 32 * rp + (tid & 31) * 4);
    }
    __device__ __forceinline__ void store(char* kt, char* vt, float* steps, int left, int tid)
    {
#pragma unroll
        for (int j = 0; j < NK; ++j) {
            const int p = 256 * j + tid, n = p & 15, o = (p >> 4) % (R / 8), tile = (p >> 4) / (R / 8);
            if (tile < 2) {              // (codes are finite, and meet zeros of q R_r behind the last octet)
                put_key(kt + tile * (64 * R), o, n, __builtin_bit_cast(uint4, codes_bf16(k[j].x, k[j].y)));
                put_key(kt + tile * (64 * R), o, 16 + n, __builtin_bit_cast(uint4, codes_bf16(k[j].z, k[j].w)));
            }
        }
        const int n = tid & 15, g = (tid >> 4) & 3, cp = tid >> 6;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            put_value(vt + j * 8192, 2 * cp, g, n, __builtin_bit_cast(uint4, codes_bf16(v[j].x, v[j].y)));
            put_value(vt + j * 8192, 2 * cp + 1, g, n, __builtin_bit_cast(uint4, codes_bf16(v[j].z, v[j].w)));
        }
        if (tid < 64) {
            steps[tid] = __uint_as_float(step << 16);
            steps[64 + tid] = tid < left ? __uint_as_float(step & 0xffff0000u) : 0.f;
        }
    }
};

// 64 full-width rows: threads 0..127 take the Keys, the others the Values, eight tokens by eight channels each, transposed in registers.
struct PlainStage {
    uint4 x[8];
    __device__ __forceinline__ void load(const bf16_t* kp, const bf16_t* vp, int64_t stride, int r0, int rows, int tid)
    {
        if (tid < 128) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                x[j] = *(const uint4*)(kp + (int64_t)min(r0 + (tid >> 2) + 32 * (j >> 2), rows - 1) * stride + 8 * ((tid & 3) + 4 * (j & 3)));
        } else {
            const int sg = (tid >> 4) & 7, t0 = 16 * (sg >> 1) + 4 * (sg & 1);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = *(const uint4*)(vp + (int64_t)min(r0 + t0 + (j < 4 ? j : 4 + j), rows - 1) * stride + 8 * (tid & 15));
        }
    }
    // whether the Values hold one that is no number, by wave
    __device__ __forceinline__ void store(char* kt, char* vt, int* odd, int r0, int rows, int tid)
    {
        bool any = false;
        if (tid < 128) {
#pragma unroll
            for (int j = 0; j < 8; ++j) put_key(kt + (j >> 2) * 8192, (tid & 3) + 4 * (j & 3), tid >> 2, x[j]);
        } else {
            const int sg = (tid >> 4) & 7, t0 = 16 * (sg >> 1) + 4 * (sg & 1), co = tid & 15;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (r0 + t0 + (j < 4 ? j : 4 + j) >= rows) x[j] = make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t w = dword_of(x[j], i);
                    any |= (w & 0x7f800000u) == 0x7f800000u || (w & 0x7f80u) == 0x7f80u;
                }
            }
            char* to = vt + (sg >> 2) * 8192 + (co >> 2) * 2048 + ((sg >> 1) & 1) * 1024 + (sg & 1) * 512 + 8 * (co & 3) * 16;
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
        any = __any(any);
        if ((tid & 63) == 0) odd[tid >> 6] = any;
    }
};

template <int FMT, int R, int RW>
__global__ __launch_bounds__(256, 2) void attn_block(RowsArgs A)
{
    constexpr bool Q8 = FMT == ROWS_Q8_BF16;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    float* steps = (float*)(lds + 2 * BLOCK_BUF);                  // [buffer][Keys 64, Values 64]
    int* odd = (int*)(steps + 256);                                // [buffer][wave]

    const uint32_t turn = blockIdx.x >> 3;                         // (the row blocks of a stretch follow each other on one XCD)
    const uint32_t pair = turn / A.nrb * 8 + (blockIdx.x & 7), block = turn % A.nrb;
    const uint32_t units = A.B * A.Hkv;
    if (pair >= units * (A.Sv + A.Sr)) return;
    const int split = pair / units, u = pair - split * units, b = u / A.Hkv, hk = u - b * A.Hkv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, n = lane & 31;
    const int S = A.Sv + A.Sr;
    const int drafts = A.draft_k ? min(max(A.n_drafts ? A.n_drafts[b] : A.T, 0), A.T) : 0;
    const int live = A.draft_k ? drafts : A.T;
    if ((int)block * 32 * RW >= live * A.G) return;
    const int row0 = (block * RW + wave % RW) * 32, row = row0 + n;
    const bool active = row0 < live * A.G;                         // (a wave without rows helps with the staging)
    const int rc = min(row, A.T * A.G - 1), tok = rc / A.G;
    const size_t at = (size_t)(b * A.T + tok) * A.Hq + hk * A.G + (rc - tok * A.G);

    // q: slot (h, e) of step i is channel 16 i + 8 (e / 4) + 4 h + e % 4
    bf16x8 qf[8];
    {
        const bf16_t* q = (const bf16_t*)A.q + at * D + 4 * h;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint2 a = *(const uint2*)(q + 16 * i), c = *(const uint2*)(q + 16 * i + 8);
            qf[i] = __builtin_bit_cast(bf16x8, make_uint4(a.x, a.y, c.x, c.y));
        }
    }
    BlockState st;
    st.clear();
    const int tile0 = RW == 4 ? 0 : wave >> 1, tile1 = RW == 4 ? 2 : tile0 + 1;

    if (split < A.Sv) {
        const int len = min(max(A.seq_len[b], 0), A.cap), stages = (len + 63) / 64, last = (len + 31) / 32 - 1;
        const int s0 = (int)((int64_t)stages * split / A.Sv), s1 = (int)((int64_t)stages * (split + 1) / A.Sv);
        const size_t slab = slab_tokens(A.cap);
        const char* Ku = (const char*)A.Kc + (Q8 ? (size_t)u * (slab / 32) * q8_kblock(A.rp) : (size_t)u * slab * A.rp * 2);
        const char* Vu = (const char*)A.Vc + (size_t)u * slab * D * (Q8 ? 1 : 2);
        if (s0 < s1) {
            CacheStage<FMT, R> X;
            X.load(Ku, Vu, s0, last, A.rp, tid);
            // R_r^T as A operands, head and remainder, in LDS; then this wave's rows of q R_r
            const float* Ru = A.Rr + (size_t)u * D * A.r;
            for (int f = wave; f < R / 4; f += 4) {
                const int j = 32 * (f >> 3) + n;
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = Ru[(16 * (f & 7) + 8 * (e >> 2) + 4 * h + (e & 3)) * A.r + min(j, A.r - 1)];
                    x[e] = j < A.r ? v : 0.f;
                }
                bf16x8 hi, lo;
                split_bf16x8(x, hi, lo);
                *(bf16x8*)(lds + (2 * f) * 1024 + lane * 16) = hi;
                *(bf16x8*)(lds + (2 * f + 1) * 1024 + lane * 16) = lo;
            }
            float bias = 0.f;
            if (A.dmu) {
                const float* dm = A.dmu + (size_t)u * D + 4 * h;
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) bias = fmaf((float)qf[i][e], dm[16 * i + 8 * (e >> 2) + (e & 3)], bias);
                bias = halves_sum(bias) * A.scale_log2;
            }
            __syncthreads();
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
                acc *= A.scale_log2;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const float x[8] = {acc[8 * t], acc[8 * t + 1], acc[8 * t + 2], acc[8 * t + 3], acc[8 * t + 4], acc[8 * t + 5], acc[8 * t + 6], acc[8 * t + 7]};
                    split_bf16x8(x, qr[2 * jb + t][0], qr[2 * jb + t][1]);
                }
            }
            __syncthreads();
            X.store(lds, lds + BLOCK_BUF / 2, steps, len - 64 * s0, tid);
            __syncthreads();
            int buf = 0;
#pragma unroll 1
            for (int s = s0; s < s1; ++s) {
                if (s + 1 < s1) X.load(Ku, Vu, s + 1, last, A.rp, tid);
                if (active) {
#pragma unroll 1
                    for (int tile = tile0; tile < tile1; ++tile) {
                        const char* kt = lds + buf * BLOCK_BUF + tile * (64 * R);
                        const char* vt = lds + buf * BLOCK_BUF + BLOCK_BUF / 2 + tile * 8192;
                        const int left = len - 64 * s - 32 * tile;
                        if (left <= 0) break;
                        f32x16 x;
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
                        for (int i = 0; i < R / 16; ++i) {
                            const bf16x8 k = *(const bf16x8*)(kt + i * 1024 + lane * 16);
                            x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qr[i][1], x, 0, 0, 0);
                            x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qr[i][0], x, 0, 0, 0);
                        }
                        const float* ks = steps + buf * 128 + 32 * tile + 4 * h;
                        if constexpr (Q8) {
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                const f32x4 w = *(const f32x4*)(ks + 8 * q);
#pragma unroll
                                for (int i = 0; i < 4; ++i) x[4 * q + i] *= w[i];
                            }
                        }
                        if (left < 32) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) x[i] = 8 * (i >> 2) + 4 * h + (i & 3) < left ? x[i] : ROWS_NEG_INF;
                        }
                        st.weigh(x);
                        if constexpr (Q8) {
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                const f32x4 w = *(const f32x4*)(ks + 64 + 8 * q);
#pragma unroll
                                for (int i = 0; i < 4; ++i) x[4 * q + i] *= w[i];
                            }
                        }
                        st.accumulate<false>(x, vt, lane);
                    }
                }
                if (s + 1 < s1) {
                    buf ^= 1;
                    X.store(lds + buf * BLOCK_BUF, lds + buf * BLOCK_BUF + BLOCK_BUF / 2, steps + buf * 128, len - 64 * (s + 1), tid);
                    __syncthreads();
                }
            }
            st.m += bias;                // (see attn_rows)
        }
    } else {
        const int text = A.text_k ? min(max(A.text_len ? A.text_len[b] : A.text_max, 0), A.text_max) : 0;
        const int tt = (text + 63) / 64, stages = tt + (drafts > 0), k = split - A.Sv;
        const int s0 = (int)((int64_t)stages * k / A.Sr), s1 = (int)((int64_t)stages * (k + 1) / A.Sr);
        if (s0 < s1) {
            const bf16_t* tk = (const bf16_t*)A.text_k + (int64_t)b * A.text_sb + (int64_t)hk * A.text_sh;
            const bf16_t* tv = (const bf16_t*)A.text_v + (int64_t)b * A.text_sb + (int64_t)hk * A.text_sh;
            const bf16_t* dk = (const bf16_t*)A.draft_k + (int64_t)b * A.draft_sb + (int64_t)hk * A.draft_sh;
            const bf16_t* dv = (const bf16_t*)A.draft_v + (int64_t)b * A.draft_sb + (int64_t)hk * A.draft_sh;
            uint64_t mask = ~0ull;
            if (A.draft_k) mask = A.mask ? A.mask[(size_t)b * A.T + tok] : (2ull << tok) - 1;
            PlainStage X;
            auto load = [&](int s) {
                const bool own = s >= tt;
                X.load(own ? dk : tk, own ? dv : tv, own ? A.draft_st : A.text_st, own ? 0 : 64 * s, own ? drafts : text, tid);
            };
            auto store = [&](int s, int buf) {
                X.store(lds + buf * BLOCK_BUF, lds + buf * BLOCK_BUF + BLOCK_BUF / 2, odd + 4 * buf, s >= tt ? 0 : 64 * s, s >= tt ? drafts : text, tid);
            };
            load(s0);
            store(s0, 0);
            __syncthreads();
            int buf = 0;
#pragma unroll 1
            for (int s = s0; s < s1; ++s) {
                const bool own = s >= tt;
                if (s + 1 < s1) load(s + 1);
                if (active) {
                    const bool strange = own && (odd[4 * buf + 2] | odd[4 * buf + 3]);
#pragma unroll 1
                    for (int tile = tile0; tile < tile1; ++tile) {
                        const char* kt = lds + buf * BLOCK_BUF + tile * 8192;
                        const char* vt = lds + buf * BLOCK_BUF + BLOCK_BUF / 2 + tile * 8192;
                        const int left = (own ? drafts : text - 64 * s) - 32 * tile;
                        if (left <= 0) break;
                        f32x16 x;
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8*)(kt + i * 1024 + lane * 16), qf[i], x, 0, 0, 0);
                        uint32_t word = own ? (uint32_t)(mask >> (32 * tile)) : ~0u, see = 0;
                        if (left < 32) word &= (1u << left) - 1;
                        word >>= 4 * h;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const bool in = (word >> (8 * (i >> 2) + (i & 3))) & 1;
                            x[i] = in ? x[i] * A.scale_log2 : ROWS_NEG_INF;
                            see |= (uint32_t)in << i;
                        }
                        st.weigh(x);
                        if (strange) {
                            st.add_odd(see, vt, lane);
                            st.accumulate<true>(x, vt, lane);
                        } else {
                            st.accumulate<false>(x, vt, lane);
                        }
                    }
                }
                if (s + 1 < s1) {
                    buf ^= 1;
                    store(s + 1, buf);
                    __syncthreads();
                }
            }
        }
    }

    st.l = halves_sum(st.l);
    if constexpr (RW == 2) {             // the two tiles' states of a row group
        float* park = (float*)lds + (wave & 1) * 64 * 66 + lane;
        __syncthreads();
        if (wave >= 2) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int i = 0; i < 16; ++i) park[64 * (16 * c + i)] = st.O[c][i];
            park[64 * 64] = st.m;
            park[64 * 65] = st.l;
        }
        __syncthreads();
        if (wave >= 2) return;
        const float m2 = park[64 * 64], l2 = park[64 * 65], M = fmaxf(st.m, m2);
        const float w1 = partial_weight(st.m, st.l, M), w2 = partial_weight(m2, l2, M);
        st.m = M;
        st.l = st.l * w1 + l2 * w2;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) st.O[c][i] = st.O[c][i] * w1 + park[64 * (16 * c + i)] * w2;
    }
    if (row >= live * A.G) return;
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
    attn_block<FMT, R, RW><<<grid, 256, BLOCK_LDS, st>>>(a);
    return hipGetLastError();
}
template <int FMT, int R>
static hipError_t launch_block_r(int nrb16, dim3 grid, const RowsArgs& a, hipStream_t st)
{
    return nrb16 == 4 ? launch_block_rw<FMT, R, 2>(grid, a, st) : launch_block_rw<FMT, R, 4>(grid, a, st);
}
template <int FMT>
static hipError_t launch_block_fmt(const RowsArgs& a, int nrb16, hipStream_t st)
{
    const int64_t pairs = (int64_t)a.B * a.Hkv * (a.Sv + a.Sr), blocks = (pairs + 7) / 8 * 8 * a.nrb;
    if (blocks > 0x7fffffff) return hipErrorInvalidValue;
    const dim3 grid((uint32_t)blocks);
    switch ((a.r + 31) / 32) {
        case 1: return launch_block_r<FMT, 32>(nrb16, grid, a, st);
        case 2: return launch_block_r<FMT, 64>(nrb16, grid, a, st);
        case 3: return launch_block_r<FMT, 96>(nrb16, grid, a, st);
        default: return launch_block_r<FMT, 128>(nrb16, grid, a, st);
    }
}

}  // namespace rk
