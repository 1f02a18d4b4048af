// Matrix products grouped by ragged runs of rows, 16-bit operands, fp32 sums:
//   Y[r,:]  = X[index[r],:] * W_e^T   (or * W_e) for the rows r of group e
//   D_e     = sum over group e's rows r of DY[r,:]^T * X[index[r],:]
//
// One kernel computes one BP x BQ tile of an output whose contiguous axis is
// q: out[p][q] = sum over k of P[p][k] * Q[q][k]. Each operand lies in memory
// with either k contiguous (rows of X, of W) or its own axis contiguous and k
// as the row number (W in the transposed product, both operands of the
// gradient). The matrix units take Q as their row operand and P as their column
// operand, so that a lane's four results are neighbours on the q axis.
#include "dense.hpp"

namespace gm {
namespace {

constexpr int BK = 64;  // reduction elements a step

// LDS layout of an operand tile, in 16-byte chunks (8 elements).
// k contiguous: 128-byte rows; chunk c of row r sits at c ^ swz(r).
// k as rows: rows of B elements; 32-byte unit u of row k sits at u ^ swz(k).
// Either swizzle spreads the chunks that a wave reads at once over the banks.
template <bool KROWS>
GM_DEV int swz(int r) {
    return KROWS ? (r & 3) | ((r >> 3) & 1) << 2 : (r >> 1) & 7;
}

// ---------------------------------------------------------------- any layout
// Tiles staged through registers: any alignment and stride. 128 x 128 tiles, four waves
// of 64 x 64.
constexpr int GEN_B = 128, GEN_T = 256;

template <typename T, bool KROWS>
struct Staged {
    static constexpr int N = GEN_B * BK / 8 / GEN_T;  // chunks a thread moves
    const T *row[N];
    u32x4 v[N];

    GM_DEV void init(const Side &s) {
        if constexpr (!KROWS) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int r = (threadIdx.x + i * GEN_T) / 8;
                row[i] = r < s.valid ? row_at<T>(s, r) : nullptr;
            }
        }
    }
    // chunk i of this thread, reduction elements k0 .. k0 + BK of n_k
    GM_DEV void load(const Side &s, int64_t k0, int64_t n_k) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = threadIdx.x + i * GEN_T;
            if constexpr (KROWS) {
                const int64_t k = k0 + c / (GEN_B / 8);
                const int col = c % (GEN_B / 8) * 8;
                const T *p = k < n_k && col < s.valid ? row_at<T>(s, k) : nullptr;
                v[i] = p ? load8(p + col, s.valid - col) : u32x4{0, 0, 0, 0};
            } else {
                const int64_t k = k0 + c % 8 * 8;
                const int64_t left = n_k - k;
                v[i] = row[i] ? load8(row[i] + k, left > 8 ? 8 : (int)left) : u32x4{0, 0, 0, 0};
            }
        }
    }
    GM_DEV void store(u32x4 *lds) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = threadIdx.x + i * GEN_T;
            if constexpr (KROWS) {
                const int k = c / (GEN_B / 8), s = c % (GEN_B / 8);
                lds[k * (GEN_B / 8) + (((s >> 1) ^ swz<true>(k)) << 1 | (s & 1))] = v[i];
            } else {
                const int r = c / 8;
                lds[r * 8 + ((c % 8) ^ swz<false>(r))] = v[i];
            }
        }
    }
};

// A wave's fragment of 16 rows from x0 and 32 reduction elements from 32 * kk:
// lane l holds row l % 16, elements 8 * (l / 16) .. + 8.
template <bool KROWS, int B>
GM_DEV u32x4 fragment(const u32x4 *lds, int x0, int kk) {
    const int lane = threadIdx.x & 63, i = lane % 16, g = lane / 16;
    if constexpr (KROWS) {
        // the transposing read: of 16 lanes, lane 4j + p brings four elements from
        // column 4p of row j; lane i gets column i of the four rows
        u32x2 h[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int k = kk * 32 + g * 8 + j * 4 + i / 4;
            const int u = (x0 / 16) ^ swz<true>(k);
            const char *p = reinterpret_cast<const char *>(lds) + k * (B * 2) + u * 32 + (i % 4) * 8;
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            h[j] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p));
        }
        return u32x4{h[0][0], h[0][1], h[1][0], h[1][1]};
    } else {
        const int r = x0 + i;
        return lds[r * 8 + ((kk * 4 + g) ^ swz<false>(r))];
    }
}

template <typename T, typename OUT, bool PK, bool QK>
GM_DEV void tile_any(const Side &p, const Side &q, int64_t n_k, OUT *out, int64_t out_stride, bool wide, u32x4 *lds) {
    u32x4 *lp = lds, *lq = lds + GEN_B * BK / 8;
    Staged<T, PK> sp;
    Staged<T, QK> sq;
    sp.init(p);
    sq.init(q);
    const int lane = threadIdx.x & 63, w = threadIdx.x / 64;
    const int p0 = w / 2 * 64, q0 = w % 2 * 64;
    f32x4 acc[4][4] = {};
    sp.load(p, 0, n_k);
    sq.load(q, 0, n_k);
    for (int64_t k0 = 0; k0 < n_k; k0 += BK) {
        __syncthreads();
        sp.store(lp);
        sq.store(lq);
        __syncthreads();
        if (k0 + BK < n_k) {
            sp.load(p, k0 + BK, n_k);
            sq.load(q, k0 + BK, n_k);
        }
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            u32x4 fp[4], fq[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                fp[i] = fragment<PK, GEN_B>(lp, p0 + 16 * i, kk);
                fq[i] = fragment<QK, GEN_B>(lq, q0 + 16 * i, kk);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = mfma_16x16x32(fq[j], fp[i], acc[i][j], T{});
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = p0 + 16 * i + lane % 16;
        if (r < p.valid) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int c = q0 + 16 * j + lane / 16 * 4;
                store4(out + r * out_stride + c, acc[i][j], q.valid - c, wide);
            }
        }
    }
}

struct ProductArgs {
    const int64_t *gp;
    const int32_t *index;
    int64_t n_groups, n_rows, n_x, n, k;
    const void *x, *w;
    void *y;
    int64_t xs, ws, wg, ys;  // strides: rows of X, rows of W, matrices of W, rows of Y
    bool wide;               // 16-byte aligned rows of Y
    int64_t max_row_tiles;   // what the rows allow, whatever group_ptr holds
};

template <typename T, typename OUT, bool TRANS>
__global__ __launch_bounds__(GEN_T) void k_group_product_any(ProductArgs a) {
    __shared__ u32x4 lds[2 * GEN_B * BK / 8];
    const int64_t n_row = min(count_row_tiles<GEN_B>(a.gp, a.n_groups, a.n_rows), a.max_row_tiles);
    const int64_t n_col = (a.n + GEN_B - 1) / GEN_B, total = n_row * n_col;
    for (int64_t b = blockIdx.x; b < total; b += gridDim.x) {
        int64_t tr, tc;
        band_tile(xcd_tile(b, total), n_row, n_col, tr, tc);
        const RowTile t = find_row_tile<GEN_B>(a.gp, a.n_groups, a.n_rows, tr);
        const int64_t q0 = tc * GEN_B;
        const int cols = (int)(a.n - q0 < GEN_B ? a.n - q0 : GEN_B);
        OUT *out = static_cast<OUT *>(a.y) + t.begin * a.ys + q0;
        if (t.group >= a.n_groups) {
            zero_tile(out, a.ys, t.rows, cols);
            continue;
        }
        Side p{a.x, a.xs, nullptr, a.n_x, t.rows};
        if (a.index)
            p.index = a.index + t.begin;
        else
            p.base = static_cast<const T *>(a.x) + t.begin * a.xs;
        const T *w = static_cast<const T *>(a.w) + t.group * a.wg + (TRANS ? q0 : q0 * a.ws);
        const Side q{w, a.ws, nullptr, 0, cols};
        tile_any<T, OUT, false, TRANS>(p, q, a.k, out, a.ys, a.wide, lds);
    }
}

struct OuterArgs {
    const int64_t *gp;
    const int32_t *index;
    int64_t n_groups, n_rows, n_x, n, k;
    const void *dy, *x;
    void *d;
    int64_t dys, xs, ds, dg;
    bool wide;
};

template <typename T, typename OUT>
__global__ __launch_bounds__(GEN_T) void k_group_outer_any(OuterArgs a) {
    __shared__ u32x4 lds[2 * GEN_B * BK / 8];
    const int64_t n_row = (a.n + GEN_B - 1) / GEN_B, n_col = (a.k + GEN_B - 1) / GEN_B;
    const int64_t per = n_row * n_col, total = per * a.n_groups;
    for (int64_t b = blockIdx.x; b < total; b += gridDim.x) {
        const int64_t t = xcd_tile(b, total), e = t / per;
        int64_t tr, tc, begin, end;
        band_tile(t - e * per, n_row, n_col, tr, tc);
        group_rows(a.gp, a.n_groups, a.n_rows, e, begin, end);
        const int64_t p0 = tr * GEN_B, q0 = tc * GEN_B;
        const Side p{static_cast<const T *>(a.dy) + begin * a.dys + p0, a.dys, nullptr, 0,
                     (int)(a.n - p0 < GEN_B ? a.n - p0 : GEN_B)};
        Side q{static_cast<const T *>(a.x) + q0, a.xs, nullptr, a.n_x, (int)(a.k - q0 < GEN_B ? a.k - q0 : GEN_B)};
        if (a.index)
            q.index = a.index + begin;
        else
            q.base = static_cast<const T *>(a.x) + begin * a.xs + q0;
        OUT *out = static_cast<OUT *>(a.d) + e * a.dg + p0 * a.ds + q0;
        tile_any<T, OUT, true, true>(p, q, end - begin, out, a.ds, a.wide, lds);
    }
}

bool is_16bit(int32_t t) { return t == GMAGNUS_DATA_BF16 || t == GMAGNUS_DATA_FP16; }

// f(T{}, OUT{}) for the operands' and the output's type
template <class F>
void with_elem(int32_t type, int32_t out, F &&f) {
    if (type == GMAGNUS_DATA_BF16) {
        if (out == GMAGNUS_DATA_FP32) f(__bf16{}, float{}); else f(__bf16{}, __bf16{});
    } else {
        if (out == GMAGNUS_DATA_FP32) f(_Float16{}, float{}); else f(_Float16{}, _Float16{});
    }
}

}  // namespace
}  // namespace gm

using namespace gm;

extern "C" gmagnus_status_t gmagnus_group_product(const gmagnus_groups_t *groups, const gmagnus_dense_t *X,
                                                  const gmagnus_dense_t *W, int32_t transposed,
                                                  const gmagnus_dense_t *Y, void *hip_stream) {
    return guarded([&] {
        check_groups(groups);
        GM_REQUIRE(X && W && Y, GMAGNUS_ERROR_INVALID_VALUE, "NULL X, W or Y");
        GM_REQUIRE(transposed == 0 || transposed == 1, GMAGNUS_ERROR_INVALID_VALUE, "transposed must be 0 or 1");
        const int64_t k = X->n_cols, n = Y->n_cols;
        check_side(k, "columns of X");
        check_side(n, "columns of Y");
        check_dense(X, "X", groups->index ? X->n_rows : groups->n_rows, k);
        check_dense(Y, "Y", groups->n_rows, n);
        check_dense(W, "W", transposed ? k : n, transposed ? n : k, groups->n_groups);
        GM_REQUIRE(X->n_rows >= 0 && X->n_rows < INT32_MAX, GMAGNUS_ERROR_UNSUPPORTED, "rows of X beyond 2^31 - 2");
        GM_REQUIRE(is_16bit(X->data_type) && W->data_type == X->data_type, GMAGNUS_ERROR_INVALID_VALUE,
                   "X and W must both be bf16 or both fp16");
        GM_REQUIRE(Y->data_type == X->data_type || Y->data_type == GMAGNUS_DATA_FP32, GMAGNUS_ERROR_INVALID_VALUE,
                   "Y must have the type of X, or fp32");
        if (groups->n_rows == 0) return;
        const int64_t row_tiles = row_tiles_bound(groups->n_groups, groups->n_rows, GEN_B);
        const ProductArgs a{groups->group_ptr, groups->index, groups->n_groups, groups->n_rows, X->n_rows, n, k,
                            X->data, W->data, Y->data, X->row_stride, W->row_stride, W->stack_stride, Y->row_stride,
                            aligned16(Y->data, Y->row_stride, 0, data_size(Y->data_type)), row_tiles};
        hipStream_t s = (hipStream_t)hip_stream;
        const int64_t tiles = row_tiles * ((n + GEN_B - 1) / GEN_B);
        const dim3 grid((unsigned)(tiles < MAX_GRID ? tiles : MAX_GRID));
        with_elem(X->data_type, Y->data_type, [&](auto t, auto o) {
            using T = decltype(t);
            using O = decltype(o);
            if (transposed)
                hipLaunchKernelGGL((k_group_product_any<T, O, true>), grid, dim3(GEN_T), 0, s, a);
            else
                hipLaunchKernelGGL((k_group_product_any<T, O, false>), grid, dim3(GEN_T), 0, s, a);
        });
        GM_CHECK_LAUNCH();
    });
}

extern "C" gmagnus_status_t gmagnus_group_outer(const gmagnus_groups_t *groups, const gmagnus_dense_t *DY,
                                                const gmagnus_dense_t *X, const gmagnus_dense_t *D, void *hip_stream) {
    return guarded([&] {
        check_groups(groups);
        GM_REQUIRE(DY && X && D, GMAGNUS_ERROR_INVALID_VALUE, "NULL DY, X or D");
        const int64_t n = DY->n_cols, k = X->n_cols;
        check_side(n, "columns of DY");
        check_side(k, "columns of X");
        check_dense(DY, "DY", groups->n_rows, n);
        check_dense(X, "X", groups->index ? X->n_rows : groups->n_rows, k);
        check_dense(D, "D", n, k, groups->n_groups);
        GM_REQUIRE(X->n_rows >= 0 && X->n_rows < INT32_MAX, GMAGNUS_ERROR_UNSUPPORTED, "rows of X beyond 2^31 - 2");
        GM_REQUIRE(is_16bit(X->data_type) && DY->data_type == X->data_type, GMAGNUS_ERROR_INVALID_VALUE,
                   "DY and X must both be bf16 or both fp16");
        GM_REQUIRE(D->data_type == X->data_type || D->data_type == GMAGNUS_DATA_FP32, GMAGNUS_ERROR_INVALID_VALUE,
                   "D must have the type of X, or fp32");
        GM_REQUIRE(groups->n_groups <= 1 || D->stack_stride >= (n - 1) * D->row_stride + k, GMAGNUS_ERROR_INVALID_VALUE,
                   "matrices of D overlap");
        const OuterArgs a{groups->group_ptr, groups->index, groups->n_groups, groups->n_rows, X->n_rows, n, k,
                          DY->data, X->data, D->data, DY->row_stride, X->row_stride, D->row_stride, D->stack_stride,
                          aligned16(D->data, D->row_stride, D->stack_stride, data_size(D->data_type))};
        hipStream_t s = (hipStream_t)hip_stream;
        const int64_t tiles = ((n + GEN_B - 1) / GEN_B) * ((k + GEN_B - 1) / GEN_B);
        const int64_t total = tiles > MAX_GRID / a.n_groups ? MAX_GRID : tiles * a.n_groups;
        with_elem(X->data_type, D->data_type, [&](auto t, auto o) {
            hipLaunchKernelGGL((k_group_outer_any<decltype(t), decltype(o)>), dim3((unsigned)total), dim3(GEN_T), 0, s, a);
        });
        GM_CHECK_LAUNCH();
    });
}
