// Shared pieces of the dense-operand kernels (routed expert products): 16-bit
// element types, eight elements at a time at any alignment, and the row tiles
// of ragged groups.
#pragma once

#include "common.hpp"
#include "host.hpp"

namespace gm {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// 16 bytes at the alignment of an element (the hardware takes any address).
template <int ALIGN>
struct Bytes16 {
    uint32_t v[4] __attribute__((packed, aligned(ALIGN)));
};

GM_DEV float to_f32(float x) { return x; }
GM_DEV float to_f32(__bf16 x) { return (float)x; }
GM_DEV float to_f32(_Float16 x) { return (float)x; }

// Two values rounded to nearest even, as 32 bits.
template <typename T>
GM_DEV uint32_t pack2(float a, float b);
template <>
GM_DEV uint32_t pack2<__bf16>(float a, float b) {
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}
template <>
GM_DEV uint32_t pack2<_Float16>(float a, float b) {
    const f16x2 v = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, v);
}

// 16 bytes of 16-bit elements, those from `valid` on as zeros; not read either.
template <typename T>
GM_DEV u32x4 load8(const T *p, int valid) {
    u32x4 r = {0, 0, 0, 0};
    if (valid >= 8) {
        const Bytes16<sizeof(T)> b = *reinterpret_cast<const Bytes16<sizeof(T)> *>(p);
        r = u32x4{b.v[0], b.v[1], b.v[2], b.v[3]};
    } else if (valid > 0) {
        const uint16_t *s = reinterpret_cast<const uint16_t *>(p);
        uint32_t e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = s[i < valid ? i : 0];
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i >> 1] |= (i < valid ? e[i] : 0u) << (16 * (i & 1));
    }
    return r;
}

// Eight elements as fp32, those from `valid` on zero.
template <typename T>
GM_DEV void load_f32x8(const T *p, int valid, float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
        if (valid >= 8) {
            const Bytes16<4> b0 = reinterpret_cast<const Bytes16<4> *>(p)[0], b1 = reinterpret_cast<const Bytes16<4> *>(p)[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = __uint_as_float(b0.v[i]);
                v[4 + i] = __uint_as_float(b1.v[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < valid ? p[i] : 0.f;
        }
    } else {
        typedef T vec __attribute__((ext_vector_type(8)));
        const vec x = __builtin_bit_cast(vec, load8(p, valid));
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)x[i];
    }
}

// Eight values rounded to T, of which `valid` are there, at any alignment.
template <typename T>
GM_DEV void store_f32(T *p, int valid, const float (&v)[8]) {
    if (valid >= 8) {
        if constexpr (sizeof(T) == 4) {
            Bytes16<4> b0, b1;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                b0.v[i] = __float_as_uint(v[i]);
                b1.v[i] = __float_as_uint(v[4 + i]);
            }
            reinterpret_cast<Bytes16<4> *>(p)[0] = b0;
            reinterpret_cast<Bytes16<4> *>(p)[1] = b1;
        } else {
            Bytes16<2> b;
#pragma unroll
            for (int i = 0; i < 4; ++i) b.v[i] = pack2<T>(v[2 * i], v[2 * i + 1]);
            *reinterpret_cast<Bytes16<2> *>(p) = b;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) p[i] = (T)v[i];
    }
}

// e^x for x up to MOST, by the hardware's power of two: what x log2(e) loses when it is
// rounded (|x| units of 2^-24 of the result) is multiplied in afterwards, so that a few
// units are off at any x. (From -200 on down the result is zero, for NaN too: an
// infinite logit, whose difference to itself that is, has a sum of zero and NaN weights.)
template <int MOST>
GM_DEV float exp_upto(float x) {
    constexpr float L = 0x1.715476p+0f, L_REST = 0x1.4ae0cp-26f, LN2 = 0x1.62e43p-1f;
    const float y = __builtin_amdgcn_fmed3f(x, -200.f, (float)MOST), t = y * L;
    const float rest = __builtin_fmaf(y, L_REST, __builtin_fmaf(y, L, -t));
    const float r = __builtin_amdgcn_exp2f(t);
    return __builtin_fmaf(r * LN2, rest, r);
}
GM_DEV float exp_neg(float x) { return exp_upto<0>(x); }

// sigma(g) and 1 - sigma(g) for g from -FAR on up, each to a few units (the latter zero soon after FAR). (The
// hardware's reciprocal is off by one.)
constexpr float FAR = 86.f;
GM_DEV void sigmoid(float g, float &s, float &rest) {
    const float z = exp_upto<(int)FAR + 1>(-g);
    s = __builtin_amdgcn_rcpf(1.f + z);
    rest = z * s;
}

// From -FAR on down sigma(g) is e^g to fp32's last place and may be below fp32's normal numbers where its product with g and
// u is not, so it is taken apart: e^g = m 2^k. (Below -300 m is zero: 2^-432 times g, u and a gradient is.)
GM_DEV float exp_apart(float g, int &k) {
    constexpr float L = 0x1.715476p+0f, L_REST = 0x1.4ae0cp-26f;
    const float y = __builtin_amdgcn_fmed3f(g, -300.f, 0.f), whole = __builtin_rintf(y * L);
    k = (int)whole;
    const float m = __builtin_amdgcn_exp2f(__builtin_fmaf(y, L_REST, __builtin_fmaf(y, L, -whole)));
    return g > -300.f ? m : 0.f;
}
// a b c m 2^k, rounded to fp32's range once, at the end.
GM_DEV float product_apart(float a, float b, float c, float m, int k) {
    const float p = __builtin_amdgcn_frexp_mantf(a) * __builtin_amdgcn_frexp_mantf(b) * __builtin_amdgcn_frexp_mantf(c) * m;
    return __builtin_amdgcn_ldexpf(p, __builtin_amdgcn_frexp_expf(a) + __builtin_amdgcn_frexp_expf(b) + __builtin_amdgcn_frexp_expf(c) + k);
}

// g sigma(g) u
GM_DEV float gated_near(float g, float u) {
    float s, rest;
    sigmoid(g, s, rest);
    return g * s * u;
}
GM_DEV float gated(float g, float u) {
    if (g >= -FAR) return gated_near(g, u);
    int k;
    const float m = exp_apart(g, k);
    return product_apart(g, u, 1.f, m, k);  // (of a NaN too)
}
// Whether any of a wave's lanes has one of eight below -FAR. (Negative numbers' bits are ordered as their magnitudes,
// above all others'.)
GM_DEV bool any_far(const float (&g)[8]) {
    uint32_t most = __float_as_uint(g[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) most = max(most, __float_as_uint(g[i]));
    return __builtin_expect(ballot(most > __float_as_uint(-FAR)) != 0, 0);
}
GM_DEV void gated8(const float (&g)[8], const float (&u)[8], float (&a)[8]) {
    if (any_far(g)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            a[i] = gated(g[i], u[i]);
            __builtin_amdgcn_sched_barrier(0);  // (one by one: what is common shall hold no registers for all of them)
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = gated_near(g[i], u[i]);
    }
}

GM_DEV uint32_t wave_max(uint32_t x) {
#define GM_STEP(ctrl, rows) \
    { const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xf, false); x = x > y ? x : y; }
    GM_STEP(0x111, 0xf) GM_STEP(0x112, 0xf) GM_STEP(0x114, 0xf) GM_STEP(0x118, 0xf) GM_STEP(0x142, 0xa) GM_STEP(0x143, 0xc)
#undef GM_STEP
    return (uint32_t)__builtin_amdgcn_readlane((int)x, GM_WAVE - 1);
}
GM_DEV float wave_sum(float x) {
#define GM_STEP(ctrl, rows) x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), ctrl, rows, 0xf, false));
    GM_STEP(0x111, 0xf) GM_STEP(0x112, 0xf) GM_STEP(0x114, 0xf) GM_STEP(0x118, 0xf) GM_STEP(0x142, 0xa) GM_STEP(0x143, 0xc)
#undef GM_STEP
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), GM_WAVE - 1));
}

GM_DEV f32x4 mfma_16x16x32(u32x4 a, u32x4 b, f32x4 c, __bf16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
GM_DEV f32x4 mfma_16x16x32(u32x4 a, u32x4 b, f32x4 c, _Float16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Rows [begin, end) of ragged group e, clamped to the rows there are; group
// n_groups is what lies past the last one, n_groups + 1 what lies before the first.
GM_DEV void group_rows(const int64_t *gp, int64_t n_groups, int64_t n_rows, int64_t e, int64_t &begin, int64_t &end) {
    int64_t b = gp[e <= n_groups ? e : 0], f = gp[e < n_groups ? e + 1 : 0];
    b = e <= n_groups ? b : 0;
    f = e == n_groups ? n_rows : f;
    begin = b < 0 ? 0 : b > n_rows ? n_rows : b;
    end = f < begin ? begin : f > n_rows ? n_rows : f;
}

// Row tiles of at most BM rows, group after group, the rows past the last group
// and those before the first as two more. With HALF a group's last tile of at most BM / 2 rows is a tile of
// that height, and those come after all others: less padding is computed, and
// the work groups that start last have little to do. A wave counts 64 groups at
// a time; all lanes get the same answer.
struct RowTiles {
    uint32_t full, half;
};

template <int BM, bool HALF>
GM_DEV void tiles_of(const int64_t *gp, int64_t n_groups, int64_t n_rows, int64_t e, int64_t &b, int64_t &f, int &full, int &half) {
    b = f = 0;
    if (e <= n_groups + 1) group_rows(gp, n_groups, n_rows, e, b, f);
    const int rows = (int)(f - b), rem = rows % BM;
    half = HALF && e < n_groups && rem > 0 && rem <= BM / 2;
    full = (rows + BM - 1) / BM - half;
}

template <int BM, bool HALF = false>
GM_DEV RowTiles count_row_tiles(const int64_t *gp, int64_t n_groups, int64_t n_rows, int64_t most) {
    const int lane = threadIdx.x & (GM_WAVE - 1);
    int n = 0, h = 0;
    for (int64_t e = lane; e <= n_groups + 1; e += GM_WAVE) {
        int64_t b, f;
        int full, half;
        tiles_of<BM, HALF>(gp, n_groups, n_rows, e, b, f, full, half);
        n += full;
        h += half;
    }
    const uint32_t full = wave_reduce_sum<int32_t>(n), half = HALF ? wave_reduce_sum<int32_t>(h) : 0, m = (uint32_t)most;
    // (`most`: what the rows allow, whatever group_ptr holds)
    const uint32_t f = full < m ? full : m;
    return RowTiles{f, half < m - f ? half : m - f};
}

struct RowTile {
    int64_t group;  // n_groups or above: rows of no group
    int64_t begin;  // first row
    int rows;       // at most BM, a half tile's at most BM / 2
};

// Tile t of the full (`half`: of the half) ones in the order above, t below their count.
template <int BM, bool HALF = false>
GM_DEV RowTile find_row_tile(const int64_t *gp, int64_t n_groups, int64_t n_rows, uint32_t t, bool half = false) {
    const int lane = threadIdx.x & (GM_WAVE - 1);
    int left = (int)t;
    for (int64_t e0 = 0; e0 <= n_groups + 1; e0 += GM_WAVE) {
        int64_t b, f;
        int n, h;
        tiles_of<BM, HALF>(gp, n_groups, n_rows, e0 + lane, b, f, n, h);
        if (HALF && half) n = h;
        const int upto = wave_incl_scan<int32_t>(n);
        const uint64_t hit = ballot(upto > left);
        if (hit) {
            const int src = __ffsll((unsigned long long)hit) - 1;
            const int in = left - (__builtin_amdgcn_readlane(upto, src) - __builtin_amdgcn_readlane(n, src));
            const int64_t gb = __builtin_amdgcn_readlane((int)b, src), gf = __builtin_amdgcn_readlane((int)f, src);
            const int64_t begin = HALF && half ? gf - (gf - gb) % BM : gb + (int64_t)in * BM;
            return RowTile{e0 + src, begin, (int)(gf - begin < BM ? gf - begin : BM)};
        }
        left -= __builtin_amdgcn_readlane(upto, GM_WAVE - 1);
    }
    return RowTile{n_groups, n_rows, 0};
}

// Upper bound of count_row_tiles on the host, which does not know the groups.
inline int64_t row_tiles_bound(int64_t n_groups, int64_t n_rows, int bm) {
    return n_rows / bm + (n_groups + 2 < n_rows ? n_groups + 2 : n_rows);
}

// Place of tile number b of n when each XCD gets a run of neighbours (the
// hardware deals consecutive work groups round-robin to the 8 XCDs). 32 bits: a
// tile's fixed work is worth counting when it has a step or two.
GM_DEV uint32_t xcd_place(uint32_t b, uint32_t n) {
    const uint32_t per = n / 8, rem = n % 8, x = b % 8;
    return x * per + (x < rem ? x : rem) + b / 8;
}

// Tile (row tile, column tile) number t: bands of 8 column tiles, row tiles
// within a band, so that the tiles in flight on one XCD share rows and columns.
GM_DEV void band_tile(uint32_t t, uint32_t n_row, uint32_t n_col, uint32_t &row, uint32_t &col) {
    constexpr uint32_t BAND = 8;
    if (n_col <= BAND) {
        row = t / n_col;
        col = t - row * n_col;
        return;
    }
    const uint32_t band = t / (n_row * BAND), r = t - band * n_row * BAND;
    const uint32_t w = n_col - band * BAND < BAND ? n_col - band * BAND : BAND;
    row = r / w;
    col = band * BAND + (r - row * w);
}

// f(T{}) for a type of fp32, bf16 or fp16.
template <class F>
inline void with_float(int32_t type, F &&f) {
    if (type == GMAGNUS_DATA_BF16)
        f(__bf16{});
    else if (type == GMAGNUS_DATA_FP16)
        f(_Float16{});
    else
        f(float{});
}

inline int data_size(int32_t type) {
    return type == GMAGNUS_DATA_FP32 ? 4 : type == GMAGNUS_DATA_FP8_E4M3 || type == GMAGNUS_DATA_INT8 ? 1 : 2;
}

inline bool is_float(int32_t type) { return type == GMAGNUS_DATA_FP32 || type == GMAGNUS_DATA_BF16 || type == GMAGNUS_DATA_FP16; }

// Common checks of a dense operand of an entry point (`last`: the last of the types it may have).
inline void check_dense(const gmagnus_dense_t *m, const char *name, int64_t n_rows, int64_t n_cols, int64_t n_stack = 1,
                        int32_t last = GMAGNUS_DATA_FP8_E4M3) {
    const std::string s(name);
    GM_REQUIRE(m != nullptr, GMAGNUS_ERROR_INVALID_VALUE, "NULL " + s);
    GM_REQUIRE(m->data_type >= GMAGNUS_DATA_FP32 && m->data_type <= last, GMAGNUS_ERROR_INVALID_VALUE,
               "unknown data type of " + s);
    GM_REQUIRE(m->n_rows == n_rows && m->n_cols == n_cols, GMAGNUS_ERROR_INVALID_VALUE,
               s + " is " + std::to_string(m->n_rows) + " x " + std::to_string(m->n_cols) + ", expected " +
                   std::to_string(n_rows) + " x " + std::to_string(n_cols));
    GM_REQUIRE(n_rows == 0 || m->row_stride >= n_cols, GMAGNUS_ERROR_INVALID_VALUE, "row stride of " + s + " below its columns");
    GM_REQUIRE(n_stack <= 1 || n_rows == 0 || m->stack_stride >= 0, GMAGNUS_ERROR_INVALID_VALUE, "negative stack stride of " + s);
    GM_REQUIRE(m->data != nullptr || n_rows == 0 || n_cols == 0 || n_stack == 0, GMAGNUS_ERROR_INVALID_VALUE,
               "NULL data of " + s);
    GM_REQUIRE(m->data == nullptr || (uintptr_t)m->data % data_size(m->data_type) == 0, GMAGNUS_ERROR_INVALID_VALUE,
               "data of " + s + " is not aligned to its type");
}

// One operand of a tile.
struct Side {
    const void *base;      // of the tile's first element (K_ROWS: of its first column)
    int64_t stride;        // elements between rows in memory
    const int32_t *index;  // row numbers in memory of the rows below, or null
    int64_t n_mem;         // rows in memory that an index may name
    int valid;             // elements of the tile's own axis
};

// Row `r`'s address, null where its index names none.
template <typename T>
GM_DEV const T *row_at(const Side &s, int64_t r) {
    if (s.index) {
        const int64_t i = s.index[r];
        return i < 0 || i >= s.n_mem ? nullptr : static_cast<const T *>(s.base) + i * s.stride;
    }
    return static_cast<const T *>(s.base) + r * s.stride;
}

// Four neighbours of an output row, from `first` on as many as there are, at any alignment.
template <typename OUT>
GM_DEV void store4(OUT *p, f32x4 v, int64_t left, int first = 0) {
    if (left >= 4 && first <= 0) {
        if constexpr (sizeof(OUT) == 4) {
            *reinterpret_cast<Bytes16<4> *>(p) = Bytes16<4>{{__float_as_uint(v[0]), __float_as_uint(v[1]),
                                                             __float_as_uint(v[2]), __float_as_uint(v[3])}};
        } else {
            struct Bytes8 {
                uint32_t v[2] __attribute__((packed, aligned(2)));
            };
            *reinterpret_cast<Bytes8 *>(p) = Bytes8{{pack2<OUT>(v[0], v[1]), pack2<OUT>(v[2], v[3])}};
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i >= first && i < left) p[i] = (OUT)v[i];
    }
}

// Rows of zeros.
template <typename OUT>
GM_DEV void zero_tile(OUT *out, int64_t stride, int rows, int cols) {
    for (int r = threadIdx.x / 64; r < rows; r += blockDim.x / 64)
        for (int c = threadIdx.x % 64; c < cols; c += 64) out[r * stride + c] = (OUT)0.f;
}

// Work groups of a launch: the kernels' loops take what exceeds this.
constexpr int64_t MAX_GRID = 1 << 22;
// (A launch has less than 2^32 threads: of work groups of 1024 fewer fit.)
constexpr int64_t max_grid(int threads) { return threads < 1024 ? MAX_GRID : ((int64_t(1) << 32) - 1) / threads; }

// Grouped rows and sides of matrices. The kernels count rows of a group, and
// elements of the reduction, in 32 bits, and go past their end by a few steps
// (384 elements) and round up to tiles (256 rows) before they compare.
constexpr int64_t MAX_SIDE = (int64_t(1) << 31) - 1025;

inline void check_groups(const gmagnus_groups_t *g) {
    GM_REQUIRE(g != nullptr, GMAGNUS_ERROR_INVALID_VALUE, "NULL groups");
    GM_REQUIRE(g->n_groups >= 1 && g->n_rows >= 0, GMAGNUS_ERROR_INVALID_VALUE, "groups: n_groups must be positive, n_rows not negative");
    GM_REQUIRE(g->group_ptr != nullptr, GMAGNUS_ERROR_INVALID_VALUE, "groups: NULL group_ptr");
    GM_REQUIRE(g->n_rows <= MAX_SIDE && g->n_groups < INT32_MAX, GMAGNUS_ERROR_UNSUPPORTED,
               "groups: more than 2^31 - 1025 rows or 2^31 - 2 groups");
}

// Rows that X has to have: its own with an index (and without grouped rows, where
// an empty index may be NULL), one for each grouped row otherwise.
inline int64_t x_rows(const gmagnus_groups_t &g, const gmagnus_dense_t &X) { return g.index || g.n_rows == 0 ? X.n_rows : g.n_rows; }

inline void check_side(int64_t n, const char *what) {
    GM_REQUIRE(n >= 1, GMAGNUS_ERROR_INVALID_VALUE, std::string(what) + " must be positive");
    GM_REQUIRE(n <= MAX_SIDE, GMAGNUS_ERROR_UNSUPPORTED, std::string(what) + " beyond 2^31 - 1025");
}

// 16-byte aligned rows (and matrices of a stack).
inline bool aligned16(const void *p, int64_t stride, int64_t stack, int size) {
    return (uintptr_t)p % 16 == 0 && stride * size % 16 == 0 && stack * size % 16 == 0;
}

}  // namespace gm
