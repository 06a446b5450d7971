// coded_common.h -- reading the 8-bit paged KV cache: the codes' decoding, the
// tile loads and their MFMA operands.  Internal to the library.
//
// A cached value is code * scale, the code an e4m3 (OCP) number or an int8, the
// scale one fp32 per block of tokens and KV head.  Both kinds of code are bf16
// and fp16 numbers exactly (4 and 7 significant bits), so products run on the
// MFMA over decoded codes and the scales are applied in fp32: K's to the logits,
// V's to the probabilities before they are rounded.
#pragma once

#include "device_common.h"
#include "launch.h"
#include "verify_common.h"

namespace ssl {
namespace cc {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kRowBytes = kHeadDim;   // a cached row

// A logit's factor, sm_scale log2(e) times K's scale: above 0, whatever the two, so
// that a masked logit times it stays -inf (0 times it would be NaN).
__device__ __forceinline__ float logit_scale(float scale_log2, float ks) {
    constexpr float kLeast = 0x1p-126f;
    return fmaxf(scale_log2 * ks, kLeast);
}

// Four codes of a dword as two packed bf16 pairs.
template <bool kInt8>
__device__ __forceinline__ void decode4(uint32_t w, uint32_t& lo, uint32_t& hi) {
    if constexpr (kInt8) {
        // (a whole number up to 127 ends above bit 16 of its fp32 form)
        const float f0 = (float)(int8_t)w, f1 = (float)(int8_t)(w >> 8);
        const float f2 = (float)(int8_t)(w >> 16), f3 = (float)(int8_t)(w >> 24);
        lo = __builtin_amdgcn_perm(__float_as_uint(f1), __float_as_uint(f0), 0x07060302u);
        hi = __builtin_amdgcn_perm(__float_as_uint(f3), __float_as_uint(f2), 0x07060302u);
    } else {
        lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
        hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
    }
}

// The same as fp16 pairs.
__device__ __forceinline__ void decode4_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ f32x4 mfma_f16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Two rows' dwords x, y of the same four head-dim elements as four packed
// pairs (x's, y's), one per element.
template <bool kInt8>
__device__ __forceinline__ void decode_pairs(uint32_t x, uint32_t y, uint32_t (&p)[4]) {
    if constexpr (kInt8) {
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const float fx = (float)(int8_t)(x >> (8 * d)), fy = (float)(int8_t)(y >> (8 * d));
            p[d] = __builtin_amdgcn_perm(__float_as_uint(fy), __float_as_uint(fx), 0x07060302u);
        }
    } else {
        decode4<false>(__builtin_amdgcn_perm(y, x, 0x05010400u), p[0], p[1]);   // x0 y0 x1 y1
        decode4<false>(__builtin_amdgcn_perm(y, x, 0x07030602u), p[2], p[3]);   // x2 y2 x3 y3
    }
}

// The same as fp16 pairs.  int8: a biased byte below 0x64 in the high byte is
// 1024 + 128 + x, from which 1152 is taken (exact).
template <bool kInt8>
__device__ __forceinline__ void decode_pairs_f16(uint32_t x, uint32_t y, uint32_t (&p)[4]) {
    if constexpr (kInt8) {
        typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
        x ^= 0x80808080u;
        y ^= 0x80808080u;
        const uint32_t t[2] = {__builtin_amdgcn_perm(y, x, 0x05010400u), __builtin_amdgcn_perm(y, x, 0x07030602u)};
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const uint32_t u = __builtin_amdgcn_perm(0x64646464u, t[d >> 1], d & 1 ? 0x04030402u : 0x04010400u);
            p[d] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, u) - f16x2{(_Float16)1152.f, (_Float16)1152.f});
        }
    } else {
        decode4_f16(__builtin_amdgcn_perm(y, x, 0x05010400u), p[0], p[1]);   // x0 y0 x1 y1
        decode4_f16(__builtin_amdgcn_perm(y, x, 0x07030602u), p[2], p[3]);   // x2 y2 x3 y3
    }
}

// A row's probabilities and the weights of its value product.  A key's probability
// is held as p = 2^(y - M), M near the row's maximum of y: its sum and the scores
// come from it and do not depend on V.  Its weight, 2^y times its V scale s = 2^e r,
// is rounded to fp16, which gives it 11 bits, where bf16 would give 8 (a single bf16
// rounding of the weights is as large as the output's own).  So that weights keep
// within fp16's range whatever the scales, they are relative to a reference of
// their own, N, which follows the row's maximum of y + e: w = 2^(y + e - N) r.  (One
// reference for both would put p out of fp32's range where scales are far apart.)
// A reference is set kBelow under its maximum and moves when a key passes it by
// kAbove.  Weights then span 2^-24 (2^-31 of the largest) to 2^15.  References are
// whole numbers, so that moving them is exact.
constexpr float kBelow = 7.f, kAbove = 14.f;
constexpr float kNoRef = -3.402823466e38f;   // reference of a row without keys so far
// A partial output is relative to M, as its sum is, and held 2^-kPartialExp times:
// so a row's whole sum passes fp32's range only where its output is about to, and
// values down to 2^-90 keep their bits.
constexpr int kPartialExp = 36;
constexpr float kWhole = 0x1p36f;

// x >= 0 as 2^exponent(x) rest(x), rest(x) below 2
__device__ __forceinline__ float exponent(float x) { return (float)((int)(__float_as_uint(x) >> 23) - 127); }
__device__ __forceinline__ float rest(float x) { return __builtin_ldexpf(x, 127 - (int)(__float_as_uint(x) >> 23)); }

// The exponent that takes a wave's sum of w code (relative to M + D) to its share of
// the partial output relative to Mx.  Not a factor: D may lie past fp32's range.
__device__ __forceinline__ int partial_shift(float M, float D, float Mx) {
    return (int)fmaxf(M - Mx + D, -300.f) - kPartialExp;
}
__device__ __forceinline__ f32x4 times_2(f32x4 o, int shift) {
    return f32x4{__builtin_ldexpf(o[0], shift), __builtin_ldexpf(o[1], shift), __builtin_ldexpf(o[2], shift),
                 __builtin_ldexpf(o[3], shift)};
}

// p and w of the lane's eight keys of a tile for one row (y not yet scaled, masked
// keys -inf); D = N - M; more_p and more_o rescale what the row has summed.
template <typename MoreP, typename MoreO>
__device__ __forceinline__ void key_weights(const f32x4 (&y)[2], float scale, float ve, float vr, float& M, float& D, float& L,
                                            f32x4 (&p)[2], f32x4 (&w)[2], MoreP&& more_p, MoreO&& more_o) {
    constexpr float kFar = 100.f;   // 2^shift that a probability and its factor still hold together
    float mx = y[0][0];
#pragma unroll
    for (int e = 1; e < 8; ++e) mx = fmaxf(mx, y[e >> 2][e & 3]);
    const float over = __builtin_fmaf(mx, scale, -M);
    float shift = ve - D;   // w = p 2^shift vr
    bool far = false;
    if (__any(fmaxf(fmaxf(over, over + shift), shift - (kFar - kAbove)) > kAbove)) {
        // the wave's first tile, a key far above a reference, or scales far apart
        mx = fmaxf(mx, shfl_xor_f(mx, 16));
        mx = fmaxf(mx, shfl_xor_f(mx, 32)) * scale;
        const float N = M + D;
        const bool grow = mx > M + kAbove, grow_o = mx + ve > N + kAbove;
        const float Mn = grow ? ceilf(mx) - kBelow : M, Nn = grow_o ? ceilf(mx + ve) - kBelow : N;
        if (__any(grow && M != kNoRef)) {
            const float alpha = fast_exp2(M - Mn);   // (1 where it stays)
            L *= alpha;
            more_p(alpha, grow && M != kNoRef);
        }
        if (__any(grow_o && M != kNoRef)) more_o(fast_exp2(N - Nn));
        M = Mn;
        D = Nn - Mn;
        shift = ve - D;
        far = __any(shift > kFar);
    }
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        p[e >> 2][e & 3] = fast_exp2(__builtin_fmaf(y[e >> 2][e & 3], scale, -M));
        sum += p[e >> 2][e & 3];
    }
    L += sum;
    const float c = __builtin_ldexpf(vr, (int)shift);
    w[0] = p[0] * c;
    w[1] = p[1] * c;
    if (far) {   // (wave-uniform) a probability that fp32 does not hold may still count
        const float at = shift - M;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e >> 2][e & 3] = fast_exp2(__builtin_fmaf(y[e >> 2][e & 3], scale, at)) * vr;
    }
}

// A 32-key tile of codes in registers.
// K: lane (m16, G) holds one key of the half tile (+16 for t = 1; a_row_key(m16)
// where V's rows have to match), bytes 64 j + 16 G .. +16, so that a row is read
// in pieces of 16 bytes: MFMA k-block kb takes the eight of them from 8 (kb & 1)
// on, j = kb / 2, and q_dim() gives the head-dim elements that the Q operand
// matches them with.
// V: slot e = 4t + i is key 16t + G + 4i, and lane (m16, G) holds its head-dim
// elements 8 m16 .. +8.
struct KCodes {
    u32x4 k[2][2];
};
struct KVCodes {
    u32x4 k[2][2];
    u32x2 v[8];
};
__device__ __forceinline__ int q_dim(int kb, int G) { return 64 * (kb >> 1) + 16 * G + 8 * (kb & 1); }

template <bool kInt8>
__device__ __forceinline__ void decode_k(const u32x4 (&k)[2], u32x4 (&a)[4]) {
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
        uint32_t w0, w1, w2, w3;
        decode4<kInt8>(k[kb >> 1][2 * (kb & 1)], w0, w1);
        decode4<kInt8>(k[kb >> 1][2 * (kb & 1) + 1], w2, w3);
        a[kb] = u32x4{w0, w1, w2, w3};
    }
}

// O^T += V^T P^T for one head-dim dword h (elements 4h .. 4h + 3 of the lane's eight).
template <bool kInt8, bool kF16 = false>
__device__ __forceinline__ void decode_v(const u32x2 (&v)[8], int h, u32x4 (&a)[4]) {
#pragma unroll
    for (int s2 = 0; s2 < 4; ++s2) {
        uint32_t p[4];
        if constexpr (kF16) decode_pairs_f16<kInt8>(v[2 * s2][h], v[2 * s2 + 1][h], p);
        else decode_pairs<kInt8>(v[2 * s2][h], v[2 * s2 + 1][h], p);
#pragma unroll
        for (int d = 0; d < 4; ++d) a[d][s2] = p[d];
    }
}

// Where a wave's tiles of one run are: lane l has tile first + kWaves * l (a
// run has at most vc::kPageRunTiles tiles of the workgroup), found once with
// all its table and scale loads in flight together, and a tile reads its lane
// back with readlane.  backwards: tile t is the (ntile - 1 - t)-th in key order.
// Page ids outside the pool are clamped into it.
struct TileRun {
    uint32_t off_lo, off_hi;   // byte offset of the tile in the pool of codes
    float ks, ve, vr;          // its scales, V's as 2^ve vr (a scale block holds whole tiles)
    int first;
};

__device__ __forceinline__ TileRun tile_run(const CodedKV& c, const int32_t* table, int n_kv, int head, int page_size,
                                            int key_begin, int ntile, int first, int lane, bool backwards = false) {
    TileRun r;
    r.first = first;
    const int t = min(first + vc::kWaves * lane, ntile - 1);
    const int key = key_begin + (backwards ? ntile - 1 - t : t) * vc::kTile;
    const int blk = key / page_size, o = key - blk * page_size;
    const int page = min(max(table[blk], 0), c.n_pages - 1);
    const size_t unit = (size_t)page * n_kv + head;
    const size_t off = (unit * page_size + o) * kRowBytes;
    const size_t at = unit * c.page_scales + (o >> c.scale_shift);
    r.off_lo = (uint32_t)off;
    r.off_hi = (uint32_t)(off >> 32);
    r.ks = c.k_scale[at];
    const float vs = c.v_scale[at];
    r.ve = exponent(vs);
    r.vr = rest(vs);
    return r;
}

__device__ __forceinline__ float lane_f(float x, int l) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), l));
}

__device__ __forceinline__ size_t tile_off(const TileRun& r, int t) {
    const int l = (t - r.first) / vc::kWaves;
    return (size_t)(uint32_t)__builtin_amdgcn_readlane((int)r.off_hi, l) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((int)r.off_lo, l);
}

// The tile as a buffer of its valid rows: rows past the sequence read as code
// 0, so that what stands behind it is never used.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t code_rsrc(const uint8_t* base, int rows) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, min(rows, vc::kTile) * kRowBytes, 0x00027000);
}

constexpr int kNonTemporal = 2;   // the buffer instructions' nt bit

template <bool kNt>
__device__ __forceinline__ void load_k_codes(const uint8_t* base, int rows, int G, int key, u32x4 (&k)[2][2]) {
    const __amdgpu_buffer_rsrc_t r = code_rsrc(base, rows);
    const int off = key * kRowBytes + 16 * G;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < 2; ++j)
            k[t][j] = __builtin_bit_cast(
                u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off + 16 * t * kRowBytes + 64 * j, 0, kNt ? kNonTemporal : 0));
}

template <bool kNt>
__device__ __forceinline__ void load_v_codes(const uint8_t* base, int rows, int m16, int G, u32x2 (&v)[8]) {
    const __amdgpu_buffer_rsrc_t r = code_rsrc(base, rows);
    const int off = G * kRowBytes + 8 * m16;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(
                                             r, off + (16 * (e >> 2) + 4 * (e & 3)) * kRowBytes, 0, kNt ? kNonTemporal : 0));
}

// The verify rows of an item in LDS, kQStride bytes each (no bank conflicts: a
// lane group's sixteen rows fall on different banks), zero past the last:
// q_load() requests them, q_store() puts them there, q_operand() reads a row's
// MFMA k-block in the order of the K codes.
constexpr int kQStride = kHeadDim * 2 + 16;

template <int NRT>
__device__ __forceinline__ void q_load(const VerifyArgs& a, int b, int c, int nq, int qoff, u32x4 (&q)[NRT]) {
    const int g = a.group;
#pragma unroll
    for (int rt = 0; rt < NRT; ++rt) {
        const int row = rt * 16 + ((int)threadIdx.x >> 4), jl = row / g;
        q[rt] = u32x4{0u, 0u, 0u, 0u};
        if (row < nq * g)
            q[rt] = ld_u32x4(a.q + (((size_t)b * a.max_q + qoff + jl) * a.n_q_heads + c * g + (row - jl * g)) * kHeadDim +
                             8 * (threadIdx.x & 15));
    }
}
template <int NRT>
__device__ __forceinline__ void q_store(const u32x4 (&q)[NRT], char* lds) {
#pragma unroll
    for (int rt = 0; rt < NRT; ++rt)
        *reinterpret_cast<u32x4*>(lds + (rt * 16 + ((int)threadIdx.x >> 4)) * kQStride + 16 * (threadIdx.x & 15)) = q[rt];
}
// A lane's place in the rows, taken anew for each tile: the rows are read from
// LDS there (kept in registers over the loop, 16 of them per row tile would
// halve the waves that a SIMD holds).
__device__ __forceinline__ int q_place(int m16, int G) {
    int at = m16 * kQStride + 32 * G;
    asm volatile("" : "+v"(at));
    return at;
}
__device__ __forceinline__ u32x4 q_operand(const char* lds, int place, int rt, int kb) {
    return *reinterpret_cast<const u32x4*>(lds + place + rt * 16 * kQStride + 2 * q_dim(kb, 0));
}

}  // namespace cc
}  // namespace ssl
