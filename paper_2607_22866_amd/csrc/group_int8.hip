// Matrix products grouped by ragged runs of rows on 8-bit integers with a scale for
// each row of either operand:
//   Y[r,n] = sx[r] * sw[n] * (sum over k of x[r,k] * w[n,k])
// The sums are integers of 32 bits, exact in any order, and leave the matrix units
// once, when they are scaled: nothing is done between two steps of the reduction, as
// blocks of E4M3 with scales of their own need it.
#include "quant.hpp"
#include "tile.hpp"

namespace gm {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// 16x16x64; both operands' 16 bytes of a lane hold the same places of the reduction.
struct MulInt8 {
    typedef i32x4 sums;
    GM_DEV static i32x4 mul(u32x4 a, u32x4 b, i32x4 c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
    }
};

// 128 * 128 times as many products stay within 32 bits.
constexpr int64_t MAX_K = 131071;

struct Int8Args {
    const int64_t *gp;
    const int32_t *index;
    int64_t n_groups, n_rows, n_x, n, k;
    const uint8_t *x, *w;
    const float *sx, *sw;
    void *y;
    int64_t xs, ws, wg, swg, ys;  // strides: rows of X, rows of W, matrices of W, their scales, rows of Y
    int64_t max_row_tiles;
};

// Row of X that the tile's row r stands for, -1 if there is none.
GM_DEV int64_t x_row(const Int8Args &a, const RowTile &t, int r) {
    if (r >= t.rows) return -1;
    const int64_t i = a.index ? a.index[t.begin + r] : t.begin + r;
    return i >= a.n_x ? -1 : i;
}

// The scales of four neighbouring columns, zero past the last.
GM_DEV f32x4 four_scales(const float *s, int left) {
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = e < left ? s[e] : 0.f;
    return v;
}

GM_DEV f32x4 scaled(i32x4 v, float sx, f32x4 sw) {
    return f32x4{(float)v[0] * sx * sw[0], (float)v[1] * sx * sw[1], (float)v[2] * sx * sw[2], (float)v[3] * sx * sw[3]};
}

// What a wave scales its results with: its NP rows' and NQ times four columns' scales,
// fetched when the sums are whole.
template <int NP, int NQ>
struct Scales {
    float x[NP];
    f32x4 w[NQ];
    GM_DEV Scales(const Int8Args &a, const RowTile &t, int64_t n0, int cols, int p0, int q0) {
        const int lane = threadIdx.x & 63;
        const float *sw = a.sw + t.group * a.swg + n0;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int64_t r = x_row(a, t, p0 + 16 * i + lane % 16);
            x[i] = r < 0 ? 0.f : a.sx[r];
        }
#pragma unroll
        for (int j = 0; j < NQ; ++j) {
            const int c = q0 + 16 * j + lane / 16 * 4;
            w[j] = four_scales(sw + c, cols - c);
        }
    }
    GM_DEV f32x4 operator()(int i, int j, i32x4 v) const { return scaled(v, x[i], w[j]); }
};

// Any alignment: tiles of 128 x 128 staged through registers, four waves of 64 x 64,
// LDS rows of 128 bytes as the E4M3 tiles have them. One step's loads are in flight while
// the step before it is multiplied from one of two buffers; bound by loads at odd
// addresses: 4001 x 4001 x 4001 138-146 us, 0.9 POP/s, with rows of 4004 117 (with two steps'
// loads in flight, whose registers spill, 157); 20 groups of 35 rows, 1000 x 3000, 29 us.
constexpr int GEN_B = 128, GEN_T = 256;

template <typename OUT>
__global__ __launch_bounds__(GEN_T, 2) void k_group_product_int8_any(Int8Args a) {
    __shared__ u32x4 lds[4 * GEN_B * 8];
    const int n_k = (int)a.k;
    const int lane = threadIdx.x & 63, i16 = lane % 16, g = lane / 16, wv = threadIdx.x / 64;
    const int p0 = wv / 2 * 64, q0 = wv % 2 * 64;
    const uint32_t n_row = count_row_tiles<GEN_B>(a.gp, a.n_groups, a.n_rows, a.max_row_tiles).full;
    const uint32_t n_col = (uint32_t)((a.n + GEN_B - 1) / GEN_B), total = n_row * n_col;
    for (uint32_t blk = blockIdx.x; blk < total; blk += gridDim.x) {
        uint32_t tr, tc;
        band_tile(xcd_place(blk, total), n_row, n_col, tr, tc);
        const RowTile t = find_row_tile<GEN_B>(a.gp, a.n_groups, a.n_rows, tr);
        const int64_t n0 = (int64_t)tc * GEN_B;
        const int cols = (int)(a.n - n0 < GEN_B ? a.n - n0 : GEN_B);
        OUT *out = static_cast<OUT *>(a.y) + t.begin * a.ys + n0;
        if (t.group >= a.n_groups) {
            zero_tile(out, a.ys, t.rows, cols);
            continue;
        }
        const uint8_t *pr[4], *qr[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (threadIdx.x + i * GEN_T) / 8;
            // (columns that are not there read the last one, rows a row of W: the former's results are not stored, the
            // latter's are not or have the scale 0. Whole steps then have no branch, which would wait for each load)
            qr[i] = a.w + t.group * a.wg + (n0 + (r < cols ? r : cols - 1)) * a.ws;
            const int64_t xr = x_row(a, t, r);
            pr[i] = xr < 0 ? qr[i] : a.x + xr * a.xs;
        }
        i32x4 acc[4][4] = {};
        u32x4 vp[4], vq[4];
        auto load = [&](int k0) {
            if (k0 >= n_k) return;
            const int k = k0 + threadIdx.x % 8 * 16;
            if (n_k - k0 >= SB) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    vp[i] = load16(pr[i] + k, 16);
                    vq[i] = load16(qr[i] + k, 16);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    vp[i] = cut_piece(pr[i], k, n_k);
                    vq[i] = cut_piece(qr[i], k, n_k);
                }
            }
        };
        auto step = [&](int k0, int buffer) {
            u32x4 *lp = lds + buffer * 2 * GEN_B * 8, *lq = lp + GEN_B * 8;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = (threadIdx.x + i * GEN_T) / 8, at = r * 8 + ((threadIdx.x % 8) ^ (r / 2 % 8));
                lp[at] = vp[i];
                lq[at] = vq[i];
            }
            __syncthreads();
            load(k0 + SB);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 fp[4], fq[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int rp = p0 + 16 * i + i16, rq = q0 + 16 * i + i16;
                    fp[i] = lp[rp * 8 + ((h * 4 + g) ^ (rp / 2 % 8))];
                    fq[i] = lq[rq * 8 + ((h * 4 + g) ^ (rq / 2 % 8))];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j] = MulInt8::mul(fq[j], fp[i], acc[i][j]);
            }
        };
        load(0);
        __syncthreads();  // (the last tile's reads of LDS)
        for (int k0 = 0; k0 < n_k; k0 += 2 * SB) {
            step(k0, 0);
            if (k0 + SB < n_k) step(k0 + SB, 1);
        }
        const Scales<4, 4> s(a, t, n0, cols, p0, q0);
        __syncthreads();
        store_tile<OUT, GEN_B, GEN_B, 4, 4, GEN_T>(out, a.ys, t.rows, cols, p0, q0, reinterpret_cast<char *>(lds),
                                                   [&](int i, int j) { return s(i, j, acc[i][j]); });
    }
}

// Tiles brought straight from memory into LDS, as the 16-bit products have them (tile.hpp). One group of 8192 x 8192 x
// 8192 480 us, 2290 TOP/s (of zeros 3120); 16 groups of 1024 rows, 4096 x 4096, 258-269 us, 2040-2130,
// cut by chance 297-312: the matrix units are busy 53 % of the cycles in which a CU has work, and CUs have none in 15 %
// of the time.
template <typename OUT, int BP, int BQ, int WP, int WQ>
GM_DEV void tile_int8_fast(const Int8Args &a, const RowTile &t, int64_t n0, int cols, char *lds) {
    const int w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64));
    Dma p{reinterpret_cast<const char *>(a.x), span(a.n_x, a.xs, a.k), a.xs, nullptr, a.n_x, t.rows};
    if (a.index) {
        p.index = a.index + t.begin;
    } else {
        p.base += t.begin * a.xs;
        p.records = span(t.rows, a.xs, a.k);
    }
    const Dma q{reinterpret_cast<const char *>(a.w) + t.group * a.wg + n0 * a.ws, span(cols, a.ws, a.k), a.ws, nullptr, 0, cols};
    constexpr int MP = BP / WP, MQ = BQ / WQ;
    tile_fast<MulInt8, OUT, false, false, true, false, BP, BQ, WP, WQ>(
        p, q, (int)(a.k / 2), static_cast<OUT *>(a.y) + t.begin * a.ys + n0, a.ys, lds,
        [&] { return Scales<MP / 16, MQ / 16>(a, t, n0, cols, w / WQ * MP, w % WQ * MQ); });
}

template <typename OUT, int BP, int BQ, int WP, int WQ>
__global__ __launch_bounds__(64 * WP * WQ, 2) void k_group_product_int8_fast(Int8Args a) {
    extern __shared__ char lds_fast[];
    constexpr bool HALF = BP >= 128;
    const RowTiles n_row = count_row_tiles<BP, HALF>(a.gp, a.n_groups, a.n_rows, a.max_row_tiles);
    const uint32_t n_col = (uint32_t)((a.n + BQ - 1) / BQ), n_full = n_row.full * n_col, total = n_full + n_row.half * n_col;
    for (uint32_t b = blockIdx.x; b < total; b += gridDim.x) {
        const bool half = HALF && b >= n_full;
        uint32_t tr, tc;
        if (half)
            band_tile(xcd_place(b - n_full, total - n_full), n_row.half, n_col, tr, tc);
        else
            band_tile(xcd_place(b, n_full), n_row.full, n_col, tr, tc);
        const RowTile t = find_row_tile<BP, HALF>(a.gp, a.n_groups, a.n_rows, tr, half);
        const int64_t n0 = (int64_t)tc * BQ;
        const int cols = (int)(a.n - n0 < BQ ? a.n - n0 : BQ);
        if (t.group >= a.n_groups) {
            zero_tile(static_cast<OUT *>(a.y) + t.begin * a.ys + n0, a.ys, t.rows, cols);
            continue;
        }
        if constexpr (HALF)
            if (half) {
                tile_int8_fast<OUT, BP / 2, BQ, WP, WQ>(a, t, n0, cols, lds_fast);
                continue;
            }
        tile_int8_fast<OUT, BP, BQ, WP, WQ>(a, t, n0, cols, lds_fast);
    }
}

// Groups of a few rows: the weights' bytes are the bound, and go straight into the
// matrix unit's registers, any alignment. A work group takes 16 rows of a group and 16
// NT columns, its waves take turns at blocks of 128, FEW_U blocks' loads in flight
// each, and their sums are joined in LDS. 64 groups of 1 row, 2048 x 4096, 113 us (4.7 TB/s
// of weights), of 8 rows 116; one row, 4096 x 4096, 11.7 us with the call.
constexpr int FEW_U = 4;

template <typename OUT, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_group_product_int8_few(Int8Args a) {
    constexpr int BP = 16, BQ = 16 * NT, THREADS = 64 * WAVES;
    __shared__ int part[WAVES][BP][BQ + 4];
    const int lane = threadIdx.x & 63, i16 = lane % 16, g = lane / 16;
    const int w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64));
    const uint32_t n_row = count_row_tiles<BP>(a.gp, a.n_groups, a.n_rows, a.max_row_tiles).full;
    const uint32_t n_col = (uint32_t)((a.n + BQ - 1) / BQ), total = n_row * n_col;
    const int n_k = (int)a.k, full = n_k / SB;
    for (uint32_t b = blockIdx.x; b < total; b += gridDim.x) {
        const uint32_t tc = b / n_row, tr = b - tc * n_row;
        const int64_t q0 = (int64_t)tc * BQ;
        const RowTile t = find_row_tile<BP>(a.gp, a.n_groups, a.n_rows, tr);
        const int cols = (int)(a.n - q0 < BQ ? a.n - q0 : BQ);
        OUT *out = static_cast<OUT *>(a.y) + t.begin * a.ys + q0;
        if (t.group >= a.n_groups) {
            zero_tile(out, a.ys, t.rows, cols);
            continue;
        }
        const uint8_t *wr[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int c = 16 * j + i16;
            wr[j] = a.w + t.group * a.wg + (q0 + (c < cols ? c : cols - 1)) * a.ws;
        }
        // (a row that is not there reads another: its results are not stored, or are zeros)
        const int64_t xi = x_row(a, t, i16);
        const uint8_t *xr = xi < 0 ? wr[0] : a.x + xi * a.xs;
        i32x4 acc[NT] = {};
        auto block = [&](const u32x4(&fx)[2], const u32x4(&fw)[NT][2]) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[j] = MulInt8::mul(fw[j][h], fx[h], acc[j]);
        };
        for (int k0 = w; k0 < full; k0 += WAVES * FEW_U) {
            u32x4 fx[FEW_U][2], fw[FEW_U][NT][2];
#pragma unroll
            for (int u = 0; u < FEW_U; ++u) {
                const int kb = min(k0 + u * WAVES, full - 1);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int j = 0; j < NT; ++j) fw[u][j][h] = load16(wr[j] + kb * SB + h * 64 + g * 16, 16);
                    fx[u][h] = load16(xr + kb * SB + h * 64 + g * 16, 16);
                }
            }
#pragma unroll
            for (int u = 0; u < FEW_U; ++u)
                if (k0 + u * WAVES < full) block(fx[u], fw[u]);
        }
        if (full * SB < n_k && w == full % WAVES) {  // what is left of the last block
            u32x4 fx[2], fw[NT][2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = full * SB + h * 64 + g * 16;
#pragma unroll
                for (int j = 0; j < NT; ++j) fw[j][h] = load16(wr[j] + k, n_k - k);
                fx[h] = load16(xr + k, n_k - k);
            }
            block(fx, fw);
        }
        __syncthreads();  // (the last tile's sums)
#pragma unroll
        for (int j = 0; j < NT; ++j) *reinterpret_cast<i32x4 *>(&part[w][i16][16 * j + 4 * g]) = acc[j];
        __syncthreads();
        for (int i = threadIdx.x; i < t.rows * (BQ / 4); i += THREADS) {
            const int r = i / (BQ / 4), c = i % (BQ / 4) * 4;
            const int64_t x = x_row(a, t, r);
            const f32x4 sw = four_scales(a.sw + t.group * a.swg + q0 + c, cols - c);
            const float sx = x < 0 ? 0.f : a.sx[x];
            i32x4 s = *reinterpret_cast<const i32x4 *>(&part[0][r][c]);
#pragma unroll
            for (int v = 1; v < WAVES; ++v) s += *reinterpret_cast<const i32x4 *>(&part[v][r][c]);
            if (x < 0) s = i32x4{0, 0, 0, 0};
            store4(out + r * a.ys + c, scaled(s, sx, sw), cols - c);
        }
    }
}

// The kernel of a product, as for 16 bits (group.hip).
enum class Shape { FEW16, FEW64, ANY, T32, T64, T256 };

Shape int8_shape(const Int8Args &a) {
    const int64_t mean = (a.n_rows + a.n_groups - 1) / a.n_groups, groups = a.n_groups < a.n_rows ? a.n_groups : a.n_rows;
    const bool fast = fast_side(a.x, a.xs, 0, a.k, a.index ? a.n_x : 256, 1) &&
                      fast_side(a.w, a.ws, a.n_groups > 1 ? a.wg : 0, a.k, 256, 1);
    // 64 groups, 2048 x 4096, sizes as chance deals them: of 1, 4, 8, 12, 16 and 24 rows 64
    // columns a work group 78, 111, 117, 124, 144 and 178 us, tiles of 32 x 128 79, 157,
    // 161, 160, 159 and 173 (all rows in one of the groups, mean 8: 44 / 23, 16: 80 / 25);
    // one row, 4096 x 4096: 11.7 with 16 columns, 13.6 with 64, 4 groups 19.6 / 18.5; not
    // aligned, 2047 x 2047, 4 groups of 1 row 19.4 with 16 columns, staged tiles 25.5, 16
    // groups 73 / 27
    if (mean <= 16) {
        if (groups * ((a.n + 63) / 64) < 256) return Shape::FEW16;
        if (fast) return Shape::FEW64;
    }
    if (!fast) return Shape::ANY;
    // 256 x 256 tiles where they do not leave CUs without one and the columns' padding does not
    // grow by more than a third: of 32, 48, 64, 96, 128, 192 and 512 rows 137, 139, 139, 144, 157,
    // 163 and 356 us, tiles of 32 rows 152, 148, 146, 175, 202, 264 and 606, of 64 177, 172, 150,
    // 155, 180, 209 and 437 (of 40 rows 139, 133, 178; mean 128, all rows in one of the groups, 60
    // against 88); 8 groups of 512 rows, 1024 x 1024 (64 tiles) 19.1 against 12.2 with 64 rows, of
    // 1024 (128 tiles) 21.8 / 19.3
    const int64_t cols = (a.n + 255) / 256;
    if (mean >= 48 && (mean + 255) / 256 * cols * groups >= 128 && 3 * 2 * cols <= 4 * ((a.n + 127) / 128)) return Shape::T256;
    return mean <= 64 ? Shape::T32 : Shape::T64;
}

}  // namespace
}  // namespace gm

using namespace gm;

extern "C" gmagnus_status_t gmagnus_group_product_int8(const gmagnus_groups_t *groups, const gmagnus_dense_t *X,
                                                       const gmagnus_dense_t *X_scale, const gmagnus_dense_t *W,
                                                       const gmagnus_dense_t *W_scale, const gmagnus_dense_t *Y,
                                                       void *hip_stream) {
    return guarded([&] {
        check_groups(groups);
        GM_REQUIRE(X && W && Y && X_scale && W_scale, GMAGNUS_ERROR_INVALID_VALUE, "NULL X, W, Y or scale");
        const int64_t k = X->n_cols, n = Y->n_cols;
        check_side(k, "columns of X");
        check_side(n, "columns of Y");
        const int64_t n_x = x_rows(*groups, *X);
        check_dense(X, "X", n_x, k, 1, GMAGNUS_DATA_INT8);
        check_dense(X_scale, "X_scale", 1, n_x);
        check_dense(Y, "Y", groups->n_rows, n);
        check_dense(W, "W", n, k, groups->n_groups, GMAGNUS_DATA_INT8);
        check_dense(W_scale, "W_scale", groups->n_groups, n);
        GM_REQUIRE(n_x >= 0 && n_x < INT32_MAX, GMAGNUS_ERROR_UNSUPPORTED, "rows of X beyond 2^31 - 2");
        GM_REQUIRE(X->data_type == GMAGNUS_DATA_INT8 && W->data_type == GMAGNUS_DATA_INT8 &&
                       X_scale->data_type == GMAGNUS_DATA_FP32 && W_scale->data_type == GMAGNUS_DATA_FP32 &&
                       is_float(Y->data_type),
                   GMAGNUS_ERROR_INVALID_VALUE, "X and W must be int8, their scales fp32, Y fp32, bf16 or fp16");
        GM_REQUIRE(k <= MAX_K, GMAGNUS_ERROR_UNSUPPORTED, "columns of X beyond 131071: their sums leave 32 bits");
        if (groups->n_rows == 0) return;
        const Int8Args a{groups->group_ptr, groups->index, groups->n_groups, groups->n_rows, n_x, n, k,
                         (const uint8_t *)X->data, (const uint8_t *)W->data, (const float *)X_scale->data,
                         (const float *)W_scale->data, Y->data, X->row_stride, W->row_stride, W->stack_stride,
                         W_scale->row_stride, Y->row_stride, 0};
        hipStream_t s = (hipStream_t)hip_stream;
        with_float(Y->data_type, [&](auto o) {
            using O = decltype(o);
            auto go = [&](auto kernel, int bp, int bq, int threads, int lds) {
                Int8Args f = a;
                f.max_row_tiles = row_tiles_bound(a.n_groups, a.n_rows, bp);
                launch_fast(kernel, f.max_row_tiles * ((n + bq - 1) / bq), threads, lds, f, s);
            };
            switch (int8_shape(a)) {
            case Shape::FEW16: return go(k_group_product_int8_few<O, 1, 4>, 16, 16, 256, 0);
            case Shape::FEW64: return go(k_group_product_int8_few<O, 4, 4>, 16, 64, 256, 0);
            case Shape::ANY: return go(k_group_product_int8_any<O>, GEN_B, GEN_B, GEN_T, 0);
            case Shape::T32: return go(k_group_product_int8_fast<O, 32, 128, 1, 4>, 32, 128, 256, fast_bytes(32, 128));
            case Shape::T64: return go(k_group_product_int8_fast<O, 64, 128, 2, 2>, 64, 128, 256, fast_bytes(64, 128));
            case Shape::T256: return go(k_group_product_int8_fast<O, 256, 256, 2, 4>, 256, 256, 512, fast_bytes(256, 256));
            }
        });
        GM_CHECK_LAUNCH();
    });
}
