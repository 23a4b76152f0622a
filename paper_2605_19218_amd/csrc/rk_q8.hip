// The 8-bit caches: written for a prompt (compress_q8), for one token (append_q8), and read back (unpack_q8).
//
// A row x of a head, the rotated Key k R_r (in fp32) or a Value, is held as whole numbers c = round(x / s), |c| <= 127, and ONE step s for
// the row, the bfloat16 next above or at max |x| / 127.  Upwards, so that no element passes 127; sixteen bits are enough for a step, since
// the codes are made with the rounded one (it costs at most 2^-7 of the step itself, and halves what the steps take).  A row with an infinity or
// a NaN has s = NaN: all of it reads back as NaN.  A row whose largest element is below 2^-100 has s = 0 (1 / s stays finite).
// What bounds these kernels is memory; the layout (rk_device.hpp) is made for the attention that reads it.  Measured at r = 64 in bf16: 32 heads x 16384 prompt
// tokens written in 90 us (380 MB, 4.2 TB/s; of its cycles the vector instructions take 36 %, the products 11), read back in 43.5 (304 MB, 7.0 TB/s); a token of 64 x 32 heads
// appended in 13.6 us (67 MB of R_r, 4.9 TB/s), of 8 heads, r = 32, in 4.  In fp32: 158 us (640 MB, 4.1 TB/s), 173 (505 MB, 2.9: two 16-byte stores a lane, each of half a
// line's pieces), 12.4.
#include "rk_kernels.hpp"

namespace rk {

// The step of a row from the bits of its largest magnitude, and 1 / s to 1 ulp (0 where every code is 0).  The product with 1 / 127 falls short of the quotient by
// 4e-9 of itself, so that a quotient that is a bfloat16 comes out as that; one that lies a rounding above it comes down to it (two of 2^23 magnitudes a binade), which
// the remainder shows: 127 s has 15 bits.  Every magnitude of a binade was compared with the quotient in 64 bits.  (The two divisions, ten rows a lane
// and block, were a third of the kernel's instructions.)
__device__ __forceinline__ float row_step(uint32_t top, float& inv)
{
    uint32_t up = (__float_as_uint(__uint_as_float(top) * (1.f / 127.f)) + 0xffffu) & 0xffff0000u;
    up += fmaf(-127.f, __uint_as_float(up), __uint_as_float(top)) > 0.f ? 0x10000u : 0u;
    const bool finite = top < 0x7f800000u, tiny = top < 0x0d800000u;        // 2^-100
    inv = finite && !tiny ? __builtin_amdgcn_rcpf(__uint_as_float(up)) : 0.f;
    return __uint_as_float(!finite ? 0x7fc00000u : tiny ? 0u : up);
}
// The code, in the low byte: 1.5 2^23 + c is c's two's complement there, and the sum is rounded once, to the nearest even.  x / s as a division rounds it: x times the
// reciprocal, and the remainder, which is exact since s has 8 bits, once more by it.  A quotient half way between two codes then comes out as that, and no other one
// does: the next lie more than half a unit of fp32's last place away.  (x / s of every step's and every fp32 x's mantissa was compared in 64 bits, with reciprocals off by a unit
// each way.  x times the reciprocal alone takes the other code for some of the ties, which a twentieth of normal bfloat16 rows have.)  A row that is no
// number gets any code: its step is NaN.
__device__ __forceinline__ uint32_t code_of(float x, float s, float inv)
{
    const float q = x * inv;
    return __float_as_uint(fmaf(fmaf(-q, s, x), inv, q) + 12582912.f);
}
// Of a bfloat16 x: what is no tie lies 2^-9 and more from one, so that the quotient rounded to 2^-11 (the last place at 1.5 2^12) tells them apart, and two
// operations do (every x and step, as above; with four, 32 heads x 16384 tokens written and read back took 133.5 us for 132.7).
__device__ __forceinline__ uint32_t code_of_bf16(float x, float inv) { return __float_as_uint(fmaf(x, inv, 6144.f) + (12582912.f - 6144.f)); }
template <typename T>
__device__ __forceinline__ uint32_t code_of_stored(float x, float s, float inv)
{
    return sizeof(T) == 2 ? code_of_bf16(x, inv) : code_of(x, s, inv);
}
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// maximum over the lanes l % 16 + 16 g, and over an aligned group of 16 lanes (as whole numbers: a NaN is the largest)
__device__ __forceinline__ uint32_t groups_umax(uint32_t v)
{
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max((uint32_t)a[0], (uint32_t)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max((uint32_t)b[0], (uint32_t)b[1]);
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true);
}
__device__ __forceinline__ uint32_t row16_umax(uint32_t v)
{
    v = max(v, dpp_u32<0xB1>(v));
    v = max(v, dpp_u32<0x4E>(v));
    v = max(v, dpp_u32<0x141>(v));
    return max(v, dpp_u32<0x140>(v));
}

// eight channels of a row
__device__ __forceinline__ void load8(const bf16_t* p, float (&x)[8])
{
    const uint4 v = *(const uint4*)p;
    const uint32_t d[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(d[i] << 16);
        x[2 * i + 1] = __uint_as_float(d[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8])
{
    const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = a[i];
        x[4 + i] = b[i];
    }
}

// ---------------------------------------------------------------------------
// Prompt rows.  A wave takes blocks of 32 tokens.  Keys: D^T[channel j][token] = R_r^T . K^T on v_mfma_f32_16x16x32_bf16, R_r as three bf16 parts in LDS (made
// once a work-group), which hold all of its 24 bits, an fp32 Key likewise, without the three smallest of the nine products (2^-24 of |k| |R_r|): k R_r is what
// fp32 products and sums make of it, so that a token gets the same codes by a prompt and by itself but for the order of the sums (with two parts, 2^-17 of |R_r| off, one code
// in some ten thousand was another one).  Lane (g, n) then holds channels 16 jb + 4 g ..+3 of tokens n and 16 + n: the row's maximum is two lane swaps, and
// a swap of halves between two jb makes the 16 bytes of the layout (one octet of both tokens).
// Values: lane (g, n) takes channels 8 n ..+7 of the eight tokens whose codes the layout puts side by side, the bytes are transposed in
// the lane, and go through LDS into the layout.  What a unit reads is asked for before the block's arithmetic, a block a wave; three work-groups a
// compute unit hide the rest (registers spent on fewer bank conflicts in the Values' transposition cost more than it gave).
// Grid: (blocks of `each` tokens, h_kv, b).
constexpr int write_waves(int R) { return R > 96 ? 8 : 4; }              // (one work-group fits into a compute unit's LDS at R = 128)
constexpr int WRITE_V = 1024;                                            // LDS of a wave for its Value codes
constexpr int write_lds(int R) { return R * D * 6 + write_waves(R) * WRITE_V; }
// an fp32 Key's eight channels as three parts of 8 bits: the first cut off, so that the largest numbers have one
__device__ __forceinline__ void key_parts(const float (&x)[8], bf16x8 (&p)[3])
{
    uint32_t h[4], m[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = x[2 * i], b = x[2 * i + 1];
        h[i] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
        const float ra = a - __uint_as_float(__float_as_uint(a) & 0xffff0000u), rb = b - __uint_as_float(__float_as_uint(b) & 0xffff0000u);
        m[i] = __builtin_bit_cast(uint32_t, (bf16x2){(__bf16)ra, (__bf16)rb});
        const float sa = ra - __uint_as_float(m[i] << 16), sb = rb - __uint_as_float(m[i] & 0xffff0000u);
        l[i] = __builtin_bit_cast(uint32_t, (bf16x2){(__bf16)sa, (__bf16)sb});
    }
    p[0] = __builtin_bit_cast(bf16x8, make_uint4(h[0], h[1], h[2], h[3]));
    p[1] = __builtin_bit_cast(bf16x8, make_uint4(m[0], m[1], m[2], m[3]));
    p[2] = __builtin_bit_cast(bf16x8, make_uint4(l[0], l[1], l[2], l[3]));
}

template <typename T, int R>
__global__ __launch_bounds__(64 * write_waves(R)) void compress_q8(RowsDev keys, RowsDev vals, int Hkv, int cap, int r, int each,
                                                                   const float* __restrict__ Rr, uint8_t* __restrict__ Kq, uint8_t* __restrict__ Vq,
                                                                   int32_t* __restrict__ seq_len_out)
{
    constexpr int JB = R / 16, NW = write_waves(R);
    constexpr bool F32 = sizeof(T) == 4;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    bf16x8* frag = (bf16x8*)smem;               // [i][jb][part][lane]
    unsigned char* vcodes = smem + R * D * 6 + (threadIdx.x >> 6) * WRITE_V;
    const int h = blockIdx.y, b = blockIdx.z, u = b * Hkv + h;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, n = lane & 15;
    const int n_b = min(rows_count(keys, b), cap);
    if (blockIdx.x == 0 && h == 0 && tid == 0 && seq_len_out) seq_len_out[b] = n_b;
    const int64_t first = (int64_t)blockIdx.x * each;
    if (first >= n_b) return;
    const int blk0 = (int)first, blk1 = (int)min(first + each, (int64_t)n_b);

    const float* Ru = Rr + (size_t)u * D * r;
    for (int f = wave; f < JB * 4; f += NW) {
        const int i = f / JB, j = 16 * (f - i * JB) + n, c0 = 32 * i + 8 * g;
        bf16x8 part[3];
#pragma unroll
        for (int jj = 0; jj < 8; ++jj) {
            const float v = Ru[(c0 + jj) * r + min(j, r - 1)];
            __bf16 hi, mid, lo;
            split3_bf16(j < r ? v : 0.f, hi, mid, lo);
            part[0][jj] = hi;
            part[1][jj] = mid;
            part[2][jj] = lo;
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) frag[(3 * f + p) * 64 + lane] = part[p];
    }
    __syncthreads();

    const int rp = keep_padded(r);
    const size_t blocks = slab_tokens(cap) / 32, kblk = q8_kblock(rp);
    uint8_t* Ku = Kq + (size_t)u * blocks * kblk;
    uint8_t* Vu = Vq + (size_t)u * blocks * (32 * D);
    const T* kdata = (const T*)keys.data + (int64_t)b * keys.sb + (int64_t)h * keys.sh;
    const T* vdata = (const T*)vals.data + (int64_t)b * vals.sb + (int64_t)h * vals.sh;
    const int32_t* list = keys.tok_idx ? keys.tok_idx + keys.tok_off[b] : nullptr;
    auto row_of = [&](int t) {                  // rows behind the last are clamped to it and not stored
        t = min(t, n_b - 1);
        return list ? (int64_t)list[t] : (int64_t)t;
    };

#pragma unroll 1
    for (int t0 = blk0 + 32 * wave; t0 < blk1; t0 += 32 * NW) {
        const bool full = t0 + 32 <= n_b;
        uint8_t* kb = Ku + (size_t)(t0 >> 5) * kblk;
        uint8_t* vb = Vu + (size_t)(t0 >> 5) * (32 * D);
        uint16_t* steps = (uint16_t*)(kb + 32 * rp);         // (Key, Value) of a token side by side

        // ---- Values: requested first, they are used last
        float xv[8][8];
#pragma unroll
        for (int jj = 0; jj < 8; ++jj) {
            const int tl = jj < 4 ? 4 * g + jj : 12 + 4 * g + jj;
            load8(vdata + row_of(t0 + tl) * vals.st + 8 * n, xv[jj]);
        }
        // ---- Keys
        f32x4 acc[2][JB];
#pragma unroll
        for (int jb = 0; jb < JB; ++jb) acc[0][jb] = acc[1][jb] = (f32x4){0.f, 0.f, 0.f, 0.f};
        {
            float x[F32 ? 2 : 1][4][8];
            bf16x8 kf[2][4];
#pragma unroll
            for (int tb = 0; tb < 2; ++tb) {
                const T* kr = kdata + row_of(t0 + 16 * tb + n) * keys.st + 8 * g;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (F32) load8(kr + 32 * i, x[tb][i]);
                    else kf[tb][i] = *(const bf16x8*)(kr + 32 * i);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                constexpr int NP = F32 ? 3 : 1;
                bf16x8 k[2][NP];
#pragma unroll
                for (int tb = 0; tb < 2; ++tb) {
                    if constexpr (F32) key_parts(x[tb][i], k[tb]);
                    else k[tb][0] = kf[tb][i];
                }
#pragma unroll
                for (int jb = 0; jb < JB; ++jb) {
                    bf16x8 a[3];
#pragma unroll
                    for (int p = 0; p < 3; ++p) a[p] = frag[((i * JB + jb) * 3 + p) * 64 + lane];
#pragma unroll
                    for (int sum = 2; sum >= 0; --sum)              // (the smallest products first)
#pragma unroll
                        for (int p = sum; p >= 0; --p)
                            if (sum - p < NP)
#pragma unroll
                                for (int tb = 0; tb < 2; ++tb)
                                    acc[tb][jb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[p], k[tb][sum - p], acc[tb][jb], 0, 0, 0);
                }
            }
        }
        float inv[2], ks[2];
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            uint32_t top = 0;
#pragma unroll
            for (int jb = 0; jb < JB; ++jb)
#pragma unroll
                for (int ii = 0; ii < 4; ++ii) top = max(top, mag(acc[tb][jb][ii]));
            ks[tb] = row_step(groups_umax(top), inv[tb]);
        }
#pragma unroll
        for (int jb = 0; jb < JB; jb += 2) {
            uint32_t piece[4];
#pragma unroll
            for (int tb = 0; tb < 2; ++tb) {
                uint32_t w[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const f32x4 a = acc[tb][jb + e];
                    w[e] = low_bytes(code_of(a[0], ks[tb], inv[tb]), code_of(a[1], ks[tb], inv[tb]), code_of(a[2], ks[tb], inv[tb]), code_of(a[3], ks[tb], inv[tb]));
                }
                // odd lane groups give their half of jb and get the even ones' half of jb + 1
                const auto x = __builtin_amdgcn_permlane16_swap(w[0], w[1], false, false);
                piece[2 * tb] = x[0];
                piece[2 * tb + 1] = x[1];
            }
            const int oct = 2 * (jb + (g & 1)) + (g >> 1);
            if (8 * oct < rp) {
                uint8_t* to = kb + oct * 256 + n * 16;
                if (full || t0 + 16 + n < n_b) *(uint4*)to = make_uint4(piece[0], piece[1], piece[2], piece[3]);
                else if (t0 + n < n_b) *(uint2*)to = make_uint2(piece[0], piece[1]);
            }
        }
        {
            const int tl = 16 * (g & 1) + n;
            if (g < 2 && t0 + tl < n_b) steps[2 * tl] = (uint16_t)(__float_as_uint(g ? ks[1] : ks[0]) >> 16);
        }

        // ---- Values
        uint32_t lo4[8], hi4[8];
        float vs[8], vinv[8];
#pragma unroll
        for (int jj = 0; jj < 8; ++jj) {
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) top = max(top, mag(xv[jj][k]));
            vs[jj] = row_step(row16_umax(top), vinv[jj]);
        }
        auto code = [&](float x, int jj) { return code_of_stored<T>(x, vs[jj], vinv[jj]); };
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            lo4[k] = low_bytes(code(xv[0][k], 0), code(xv[1][k], 1), code(xv[2][k], 2), code(xv[3][k], 3));
            hi4[k] = low_bytes(code(xv[4][k], 4), code(xv[5][k], 5), code(xv[6][k], 6), code(xv[7][k], 7));
        }
        uint32_t mine = 0;
#pragma unroll
        for (int jj = 0; jj < 8; ++jj) mine = n == jj ? __float_as_uint(vs[jj]) >> 16 : mine;
        {
            const int tl = (n & 7) < 4 ? 4 * g + (n & 7) : 12 + 4 * g + (n & 7);
            if (n < 8 && t0 + tl < n_b) steps[2 * tl + 1] = (uint16_t)mine;
        }
        // channel 8 n + k is place 8 (n % 2) + k of channel block n / 2; blocks lie in pairs
        uint8_t* to = vb + (n >> 2) * 1024 + g * 256 + (n & 1) * 128;
        if (full) {
            // through LDS, so that a store is a kilobyte on end (from the lanes as they are, 64 bytes a lane in four stores, the
            // stores of a block touched every line of it four times), a kilobyte at a time: what LDS is left makes a third work-group on a compute unit
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (n >> 2 == j) {
                    unsigned char* at = vcodes + g * 256 + (n & 1) * 128 + (n & 2) * 4;
#pragma unroll
                    for (int k = 0; k < 8; ++k) *(uint2*)(at + 16 * k) = make_uint2(lo4[k], hi4[k]);
                }
                wave_lds_fence();
                *(uint4*)(vb + 1024 * j + 16 * lane) = *(const uint4*)(vcodes + 16 * lane);
                wave_lds_fence();
            }
        } else {
            to += (n & 2) * 4;
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int jj = 0; jj < 8; ++jj) {
                    const int tl = jj < 4 ? 4 * g + jj : 12 + 4 * g + jj;
                    if (t0 + tl < n_b) to[16 * k + jj] = (uint8_t)((jj < 4 ? lo4[k] : hi4[k]) >> (8 * (jj & 3)));
                }
        }
    }
}

// ---------------------------------------------------------------------------
// One token a sequence: k~ = k R_r in fp32, thread (half, j) of 2 x 128 sums 64 channels of column j.  Bound by round trips: half of R_r's column is asked for
// beside the length and the inputs, the other half in flight behind it (64 x 32 heads, r = 64, appended and read back: 47.7 us with none ahead, 45.7 with 16, 45.6
// with 32, 46.1 with all 64).  The last work-group of a sequence writes the new length: seq_len_out may be seq_len itself, which all of them read.
template <typename T>
__global__ __launch_bounds__(256) void append_q8(int Hkv, int cap, int r, const T* __restrict__ k_new, const T* __restrict__ v_new,
                                                 const float* __restrict__ Rr, uint8_t* __restrict__ Kq, uint8_t* __restrict__ Vq,
                                                 const int32_t* seq_len, int32_t* seq_len_out, int32_t* __restrict__ tickets, int apart)
{
    constexpr int AHEAD = 32;            // channels
    __shared__ float ks[D], part[D];
    __shared__ uint32_t tops[4];
    const int h = blockIdx.x, b = blockIdx.y, u = b * Hkv + h;
    const int tid = threadIdx.x, wave = tid >> 6, j = tid & 127, half = tid >> 7;
    const int len = seq_len[b];
    const bool room = len >= 0 && len < cap;
    float x = 0.f;
    const float* Rc = Rr + (size_t)u * D * r + (size_t)(64 * half) * r + min(j, r - 1);
    float w[AHEAD];
#pragma unroll
    for (int c = 0; c < AHEAD; ++c) w[c] = Rc[c * r];
    if (half) x = ld_elem(v_new + (size_t)u * D + j);
    else ks[j] = ld_elem(k_new + (size_t)u * D + j);
    __syncthreads();
    float a = 0.f;
#pragma unroll
    for (int c = 0; c < AHEAD; ++c) a = fmaf(ks[64 * half + c], w[c], a);
#pragma unroll 16
    for (int c = AHEAD; c < 64; ++c) a = fmaf(ks[64 * half + c], Rc[c * r], a);
    if (half) part[j] = a;
    __syncthreads();
    if (!half) x = j < r ? a + part[j] : 0.f;       // waves 0 and 1: the rotated Key; 2 and 3: the Value
    uint32_t top = mag(x);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    if ((tid & 63) == 0) tops[wave] = top;
    __syncthreads();
    float inv;
    const float step = row_step(max(tops[2 * half], tops[2 * half + 1]), inv);
    if (room) {
        const int rp = keep_padded(r);
        const size_t blocks = slab_tokens(cap) / 32;
        uint8_t* kb = Kq + ((size_t)u * blocks + (len >> 5)) * q8_kblock(rp);
        const uint8_t code = (uint8_t)code_of(x, step, inv);
        if (half) Vq[(size_t)u * blocks * (32 * D) + q8_vidx(len, j)] = code;
        else if (j < rp) kb[q8_kplace(len, j)] = code;
        if (j == 0) ((uint16_t*)(kb + 32 * rp))[2 * (len & 31) + half] = (uint16_t)(__float_as_uint(step) >> 16);
    }
    if (tid == 0 && atomicAdd(tickets + (size_t)b * apart, 1) == Hkv - 1) {
        tickets[(size_t)b * apart] = 0;
        seq_len_out[b] = room ? len + 1 : len;
    }
}

// ---------------------------------------------------------------------------
// Both caches back to rows, a wave a block of 32 tokens: what was read 16 bytes a lane is written as whole rows, the Values by the same
// transpose of bytes as above.  Bound by memory (two of three bytes are written at r = 64 in bf16), for short heads by the round trips to the length and
// to the codes: PIECES, of a lane's Keys (R / 32), are counted at compile time so that all loads of a block are in flight at once (64 x 32 heads of up to 150
// tokens, appended to and read back: 45.7 us with three round trips a block, 44.6).
__device__ __forceinline__ float code_at(uint32_t w, int i) { return (float)((int32_t)(w << (24 - 8 * i)) >> 24); }
__device__ __forceinline__ void store8(bf16_t* p, const float (&x)[8])
{
    uint32_t d[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] = __builtin_bit_cast(uint32_t, (bf16x2){(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
    nt_store16(p, make_uint4(d[0], d[1], d[2], d[3]));
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8])
{
    nt_store16(p, make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])));
    nt_store16(p + 4, make_uint4(__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7])));
}

template <typename T, int PIECES>
__global__ __launch_bounds__(256) void unpack_q8(int Hkv, int cap, int r, const uint8_t* __restrict__ Kq, const uint8_t* __restrict__ Vq,
                                                 const int32_t* __restrict__ seq_len, T* __restrict__ k_rows, T* __restrict__ v_rows)
{
    const int h = blockIdx.y, b = blockIdx.z;
    const size_t u = (size_t)b * Hkv + h;
    const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
    const int t0 = (blockIdx.x * 4 + (threadIdx.x >> 6)) * 32;
    const int len = seq_len ? min(max(seq_len[b], 0), cap) : cap;
    if (t0 >= len) return;
    const int rp = keep_padded(r), octs = (r + 7) / 8;
    const size_t blocks = slab_tokens(cap) / 32;
    const uint8_t* kb = Kq + (u * blocks + (t0 >> 5)) * q8_kblock(rp);
    const uint32_t* steps = (const uint32_t*)(kb + 32 * rp);       // (Key, Value) of a token
    // everything is asked for first: the Values' codes and steps, the Keys' pieces (consecutive lanes take consecutive octets of a token: whole rows are
    // written; the last pieces may be read twice)
    uint2 raw[8];
    uint4 vst[2];
    if (v_rows) {
        const uint8_t* from = Vq + (u * blocks + (t0 >> 5)) * (size_t)(32 * D) + (n >> 2) * 1024 + g * 256 + (n & 1) * 128 + (n & 2) * 4;
#pragma unroll
        for (int k = 0; k < 8; ++k) raw[k] = *(const uint2*)(from + 16 * k);
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) vst[tb] = *(const uint4*)(steps + 16 * tb + 4 * g);
    }
    if (k_rows) {
        uint4 piece[PIECES];
        uint32_t kst[PIECES][2];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int p = min(lane + 64 * i, 16 * octs - 1), tn = p / octs, oct = p - tn * octs;
            piece[i] = *(const uint4*)(kb + oct * 256 + tn * 16);
            kst[i][0] = steps[tn];
            kst[i][1] = steps[16 + tn];
        }
        const bool wide = r % 8 == 0 && ((uintptr_t)k_rows & 15) == 0;
        T* to = k_rows + (u * cap + t0) * (size_t)r;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int p = lane + 64 * i, tn = p / octs, oct = p - tn * octs;
            if (p >= 16 * octs) break;
#pragma unroll
            for (int tb = 0; tb < 2; ++tb) {
                const int tl = 16 * tb + tn;
                if (t0 + tl >= len) continue;
                const float s = __uint_as_float(kst[i][tb] << 16);
                float x[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const uint32_t w = tb ? (c < 4 ? piece[i].z : piece[i].w) : (c < 4 ? piece[i].x : piece[i].y);
                    x[c] = code_at(w, c & 3) * s;
                }
                T* at = to + (size_t)tl * r + 8 * oct;
                if (wide) store8(at, x);
                else
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        if (8 * oct + c < r) st_elem(at + c, x[c]);
            }
        }
    }
    if (v_rows) {
        const bool wide = ((uintptr_t)v_rows & 15) == 0;
        T* to = v_rows + (u * cap + t0) * (size_t)D;
#pragma unroll
        for (int jj = 0; jj < 8; ++jj) {
            const int tl = jj < 4 ? 4 * g + jj : 12 + 4 * g + jj;
            if (t0 + tl >= len) continue;
            const uint4 w = vst[jj >> 2];
            const float s = __uint_as_float(((jj & 3) == 0 ? w.x : (jj & 3) == 1 ? w.y : (jj & 3) == 2 ? w.z : w.w) & 0xffff0000u);
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = code_at(jj < 4 ? raw[k].x : raw[k].y, jj & 3) * s;
            T* at = to + (size_t)tl * D + 8 * n;
            if (wide) store8(at, x);
            else
#pragma unroll
                for (int k = 0; k < 8; ++k) st_elem(at + k, x[k]);
        }
    }
}

// ---------------------------------------------------------------------------
template <typename T, int R>
static hipError_t compress_q8_r(const RowsDev& keys, const RowsDev& vals, int B, int Hkv, int cap, int r, int each, const float* Rr, uint8_t* Kq,
                                uint8_t* Vq, int32_t* seq_len_out, hipStream_t st)
{
    constexpr int lds = write_lds(R);
    const hipError_t e = allow_dynamic_lds((const void*)compress_q8<T, R>, lds);
    if (e != hipSuccess) return e;
    const int nb = keys.n_tokens > 0 ? (int)(((int64_t)keys.n_tokens + each - 1) / each) : 1;
    compress_q8<T, R><<<dim3(nb, Hkv, B), 64 * write_waves(R), lds, st>>>(keys, vals, Hkv, cap, r, each, Rr, Kq, Vq, seq_len_out);
    return hipGetLastError();
}

hipError_t launch_compress_q8(int dtype, const RowsDev& keys, const RowsDev& vals, int B, int Hkv, int cap, int r, const float* Rr, void* Kq,
                              void* Vq, int32_t* seq_len_out, int n_cu, hipStream_t st)
{
    // Tokens of a work-group: the count whose rounds of work-groups (as many of them on a compute unit as their LDS lets) come out shortest, each counted with
    // 96 tokens more for making R_r ready.  With 128 / 256 / 512 (us): r = 64, bf16, 32768 tokens x heads 10.0 / 18.7 / 30.8, 65536 15.9 / 20.4 / 32.4, 131072 27.2 / 25.4
    // / 34.0, 256000 48.9 / 46.6 / 45.1, 524288 109 / 98 / 110, 1280000 238 / 218 / 222; fp32 131072 40.2 / 37.8 / 43.8, 524288 174 / 165 / 159; r = 128, bf16
    // 65536 28.7 / 19.7 / 27.3, 131072 53.8 / 37.0 / 33.9, 524288 242 / 161 / 149.
    const int64_t R = (r + 31) / 32 * 32, side = (int64_t)n_cu * (163840 / write_lds((int)R));
    int each = 128;
    int64_t best = INT64_MAX;
    for (int e = 32 * write_waves((int)R); e <= 512; e *= 2) {
        const int64_t groups = ((int64_t)keys.n_tokens + e - 1) / e * B * Hkv, cost = (groups + side - 1) / side * (e + 96);
        if (cost < best) { best = cost; each = e; }
    }
    auto go = [&](auto t) {
        typedef decltype(t) T;
        uint8_t *kq = (uint8_t*)Kq, *vq = (uint8_t*)Vq;
        const int w = (r + 31) / 32;
        if (w == 1) return compress_q8_r<T, 32>(keys, vals, B, Hkv, cap, r, each, Rr, kq, vq, seq_len_out, st);
        if (w == 2) return compress_q8_r<T, 64>(keys, vals, B, Hkv, cap, r, each, Rr, kq, vq, seq_len_out, st);
        if (w == 3) return compress_q8_r<T, 96>(keys, vals, B, Hkv, cap, r, each, Rr, kq, vq, seq_len_out, st);
        return compress_q8_r<T, 128>(keys, vals, B, Hkv, cap, r, each, Rr, kq, vq, seq_len_out, st);
    };
    return dtype == 0 ? go(0.f) : go(bf16_t{});
}

hipError_t launch_append_q8(int dtype, int B, int Hkv, int cap, int r, const void* k_new, const void* v_new, const float* Rr, void* Kq, void* Vq,
                            const int32_t* seq_len, int32_t* seq_len_out, int32_t* tickets, hipStream_t st)
{
    const dim3 grid(Hkv, B);
    if (dtype == 0)
        append_q8<float><<<grid, 256, 0, st>>>(Hkv, cap, r, (const float*)k_new, (const float*)v_new, Rr, (uint8_t*)Kq, (uint8_t*)Vq, seq_len,
                                               seq_len_out, tickets, tickets_apart(B));
    else
        append_q8<bf16_t><<<grid, 256, 0, st>>>(Hkv, cap, r, (const bf16_t*)k_new, (const bf16_t*)v_new, Rr, (uint8_t*)Kq, (uint8_t*)Vq, seq_len,
                                                seq_len_out, tickets, tickets_apart(B));
    return hipGetLastError();
}

hipError_t launch_unpack_q8(int dtype, int B, int Hkv, int cap, int r, const void* Kq, const void* Vq, const int32_t* seq_len, void* k_rows,
                            void* v_rows, hipStream_t st)
{
    const dim3 grid((cap + 127) / 128, Hkv, B);
    auto go = [&](auto t) {
        typedef decltype(t) T;
        const uint8_t *kq = (const uint8_t*)Kq, *vq = (const uint8_t*)Vq;
        T *k = (T*)k_rows, *v = (T*)v_rows;
        switch ((r + 31) / 32) {
            case 1: unpack_q8<T, 1><<<grid, 256, 0, st>>>(Hkv, cap, r, kq, vq, seq_len, k, v); break;
            case 2: unpack_q8<T, 2><<<grid, 256, 0, st>>>(Hkv, cap, r, kq, vq, seq_len, k, v); break;
            case 3: unpack_q8<T, 3><<<grid, 256, 0, st>>>(Hkv, cap, r, kq, vq, seq_len, k, v); break;
            default: unpack_q8<T, 4><<<grid, 256, 0, st>>>(Hkv, cap, r, kq, vq, seq_len, k, v); break;
        }
        return hipGetLastError();
    };
    return dtype == 0 ? go(0.f) : go(bf16_t{});
}

}  // namespace rk
