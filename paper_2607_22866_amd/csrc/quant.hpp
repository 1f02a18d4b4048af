// Values in 8 bits with a scale: E4M3 in blocks of 128, and integers by rows.
#pragma once

#include "dense.hpp"

namespace gm {

constexpr int SB = GMAGNUS_SCALE_BLOCK;
constexpr float FP8_MAX = 448.f;
constexpr float SCALE_MIN = 0x1p-126f;
constexpr float INT8_MAX_F = 127.f;

// Magnitudes compare as their bits, NaN above infinity above the rest.
GM_DEV uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

GM_DEV float block_scale(uint32_t most) {
    const float s = __uint_as_float(most) / FP8_MAX;
    return s < SCALE_MIN ? SCALE_MIN : s;  // (a NaN stays)
}

GM_DEV float to_range(float x, float scale) {
    const float v = x / scale;
    return v > FP8_MAX ? FP8_MAX : v < -FP8_MAX ? -FP8_MAX : v;
}

GM_DEV uint32_t pack_fp8(float a, float b, float c, float d) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}

// Eight bytes, of which `valid` are there, at any alignment.
GM_DEV void store_bytes8(uint8_t *p, int valid, const uint32_t (&w)[2]) {
    if (valid >= 8) {
        struct Bytes8 {
            uint32_t v[2] __attribute__((packed, aligned(1)));
        };
        *reinterpret_cast<Bytes8 *>(p) = Bytes8{{w[0], w[1]}};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) p[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
    }
}

GM_DEV void store_fp8x8(uint8_t *p, int valid, const float (&v)[8], float scale) {
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = to_range(v[i], scale);
    const uint32_t w[2] = {pack_fp8(r[0], r[1], r[2], r[3]), pack_fp8(r[4], r[5], r[6], r[7])};
    store_bytes8(p, valid, w);
}

// 16 bytes, those from `valid` on zero and not read.
GM_DEV u32x4 load16(const uint8_t *p, int64_t valid) {
    u32x4 r = {0, 0, 0, 0};
    if (valid >= 16) {
        const Bytes16<1> b = *reinterpret_cast<const Bytes16<1> *>(p);
        r = u32x4{b.v[0], b.v[1], b.v[2], b.v[3]};
    } else if (valid > 0) {
        uint32_t e[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] = p[i < valid ? i : 0];
#pragma unroll
        for (int i = 0; i < 16; ++i) r[i >> 2] |= (i < valid ? e[i] : 0u) << (8 * (i & 3));
    }
    return r;
}

// The 16 bytes at `at` of a row of n bytes, zeros past its end, where nothing is read: the row's last 16 bytes where
// these would pass it, moved down. (Element by element they would take more registers than all else in the kernels
// that use this; a branch on what is there would wait for each load.)
GM_DEV u32x4 cut_piece(const uint8_t *row, int64_t at, int64_t n) {
    if (n >= 16) {
        const int64_t from = at < n - 16 ? at : n - 16, past = at - from;
        const int move = past < 16 ? (int)past : 16;
        const Bytes16<1> b = *reinterpret_cast<const Bytes16<1> *>(row + from);
        const bool all = move & 16, two = move & 8, one = move & 4;
        const uint32_t c[4] = {two ? b.v[2] : b.v[0], two ? b.v[3] : b.v[1], two ? 0 : b.v[2], two ? 0 : b.v[3]};
        const uint32_t d[5] = {one ? c[1] : c[0], one ? c[2] : c[1], one ? c[3] : c[2], one ? 0 : c[3], 0};
        u32x4 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = all ? 0u : __builtin_amdgcn_alignbyte(d[i + 1], d[i], move & 3);
        return r;
    }
    uint64_t v[2] = {0, 0};  // (a row of less than a piece)
#pragma unroll 1
    for (int i = 0; i < (int)(n - at); ++i) {
        const uint64_t x = (uint64_t)row[at + i] << (8 * (i & 7));
        v[0] |= i < 8 ? x : 0;
        v[1] |= i < 8 ? 0 : x;
    }
    return u32x4{(uint32_t)v[0], (uint32_t)(v[0] >> 32), (uint32_t)v[1], (uint32_t)(v[1] >> 32)};
}

// The scale of a row of 8-bit integers.
GM_DEV float row_scale(uint32_t most) {
    const float s = __uint_as_float(most) / INT8_MAX_F;
    return s < SCALE_MIN ? SCALE_MIN : s;  // (a NaN stays)
}

// v / scale as the division rounds it, by 1 / scale, which costs a division for eight values rather than for each: the
// quotient is corrected by what it leaves of v. (That makes it the division's at all quotients near an odd multiple of
// 2^-7 times a power of two, where 8-bit roundings have their borders: computed for every scale's mantissa and the
// seven values around each. Uncorrected it lies on the other side of the border at one in twelve of these. What is
// left of v may pass the end of fp32 where the scale is below 2^-90: both are taken 2^60 times there. An infinite scale,
// whose inverse is 0, corrects nothing: 0 and NaN, as the division gives. Zeros keep their sign, of v and q s
// subtracted in this order.)
GM_DEV void quotients(const float (&v)[8], float scale, float inverse, float (&r)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = v[i];
    const bool small = scale < 0x1p-90f;
    if (__builtin_expect(ballot(small) != 0, 0)) {  // (of any lane)
        const float up = small ? 0x1p60f : 1.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] *= up;
        scale *= up;
        inverse *= small ? 0x1p-60f : 1.f;
    }
    if (inverse == 0.f) scale = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = r[i] * inverse;
        r[i] = __builtin_fmaf(-__builtin_fmaf(q, scale, -r[i]), inverse, q);
    }
}

// The bytes of store_fp8x8 by 1 / scale. (No clamp: 448 and a unit at most, which is 448 in E4M3.)
GM_DEV void store_fp8x8_by(uint8_t *p, int valid, const float (&v)[8], float scale, float inverse) {
    float r[8];
    quotients(v, scale, inverse, r);
    const uint32_t w[2] = {pack_fp8(r[0], r[1], r[2], r[3]), pack_fp8(r[4], r[5], r[6], r[7])};
    store_bytes8(p, valid, w);
}

// To the nearest integers, ties to even; a NaN as 0. (127 in magnitude and a unit at most before that.)
GM_DEV void store_int8x8_by(uint8_t *p, int valid, const float (&v)[8], float scale, float inverse) {
    float r[8];
    quotients(v, scale, inverse, r);
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = __builtin_rintf(r[i]);
        b[i] = (uint32_t)(int)(x == x ? x : 0.f);
    }
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)  // (the low bytes of four)
        w[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[4 * i + 3], b[4 * i + 2], 0x0c0c0400u),
                                     __builtin_amdgcn_perm(b[4 * i + 1], b[4 * i], 0x0c0c0400u), 0x05040100u);
    store_bytes8(p, valid, w);
}

}  // namespace gm
