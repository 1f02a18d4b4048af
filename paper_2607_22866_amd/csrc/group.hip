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
#include <type_traits>

#include "tile.hpp"

namespace gm {
namespace {

// ---------------------------------------------------------------- any layout
// Tiles staged through registers, for operands at any alignment: 128 x 128, four
// waves of 64 x 64. Two steps' loads are in flight in registers while a third
// step's tile is multiplied from one of two LDS buffers; bound by that staging
// (loads that cross lines, LDS writes). One group of 4001 x 4001 x 4001, fp16: 700
// TFLOP/s, transposed 730, gradient 690.
constexpr int GEN_B = 128, GEN_T = 256;

// IDX: k as rows, their numbers by an index.
template <typename T, bool KROWS, bool IDX>
struct Staged {
    static constexpr int N = GEN_B * BK / 8 / GEN_T;  // chunks a thread moves
    const T *at[N];   // chunk i: its row, null if it is not there; k as rows: its place in the next step
    uint32_t to[N];   // its place in the tile, in chunks
    int32_t ids[KROWS && IDX ? N : 1];

    GM_DEV static int row_of(int i) { return (threadIdx.x + i * GEN_T) / (KROWS ? GEN_B / 8 : 8); }
    GM_DEV static int elem_of() { return threadIdx.x % (KROWS ? GEN_B / 8 : 8) * 8; }

    GM_DEV void init(const Side &s) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = row_of(i), x = elem_of() / 8;
            if constexpr (KROWS) {
                to[i] = r * (GEN_B / 8) + (((x >> 1) ^ swz<true>(r)) << 1 | (x & 1));
                // (columns that are not there read the first ones: their results are not stored)
                at[i] = static_cast<const T *>(s.base) + (elem_of() < s.valid ? elem_of() : 0) + (IDX ? 0 : r * s.stride);
            } else {
                to[i] = r * 8 + (x ^ swz<false>(r));
                at[i] = r < s.valid ? row_at<T>(s, r) : nullptr;
            }
        }
    }
    // the rows' numbers of step k0, -1 where there is none
    GM_DEV void fetch_ids(const Side &s, int k0, int n_k) {
        if constexpr (KROWS && IDX) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int k = k0 + row_of(i);
                ids[i] = k < n_k ? s.index[k] : -1;
            }
        }
    }
    // the chunks of reduction elements k0 .. k0 + BK of n_k, step after step (by index: of the numbers fetched
    // last; the next step's are on their way before the chunks are, so that waiting for them does not wait
    // for these)
    GM_DEV void load(const Side &s, int k0, int n_k, u32x4(&v)[N]) {
        if constexpr (KROWS) {
            const int left = s.valid - (elem_of() < s.valid ? elem_of() : 0);
            const bool whole = (s.valid & 7) == 0;
            if constexpr (IDX) {
                int32_t now[N];
#pragma unroll
                for (int i = 0; i < N; ++i) now[i] = ids[i] >= (int)s.n_mem ? -1 : ids[i];
                fetch_ids(s, k0 + BK, n_k);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const T *p = at[i] + (int64_t)(now[i] < 0 ? 0 : now[i]) * s.stride;
                    v[i] = whole ? load8(p, 8) : load8(p, left);
                    if (now[i] < 0) v[i] = u32x4{0, 0, 0, 0};
                }
            } else if (whole && n_k - k0 >= BK) {
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] = load8(at[i], 8);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] = load8(at[i], k0 + row_of(i) < n_k ? left : 0);
            }
            if constexpr (!IDX)
#pragma unroll
                for (int i = 0; i < N; ++i) at[i] += BK * s.stride;
        } else {
            const int x = k0 + elem_of();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[i] = u32x4{0, 0, 0, 0};
                if (at[i]) v[i] = n_k - k0 >= BK ? load8(at[i] + x, 8) : load8(at[i] + x, n_k - x);
            }
        }
    }
    GM_DEV void store(u32x4 *lds, const u32x4(&v)[N]) const {
#pragma unroll
        for (int i = 0; i < N; ++i) lds[to[i]] = v[i];
    }
};

// First element of tile `t` of B on an axis of n elements that is contiguous in
// memory: the last tile is moved back to end with the axis, so that no piece of
// 8 elements is cut (16384 rows, 2047 x 2047, transposed product and gradient:
// 364 -> 239 us, 472 -> 323). What an earlier tile stores as well is skipped.
GM_DEV int64_t tile_start(int64_t t, int64_t n, int b) { return t * b + b > n && n > b ? n - b : t * b; }

template <typename T, typename OUT, bool PK, bool QK, bool QI>
GM_DEV void tile_any(const Side &p, const Side &q, int n_k, OUT *out, int64_t out_stride, int skip_p, int skip_q, u32x4 *lds) {
    constexpr int BUF = GEN_B * BK / 8;  // chunks of a tile
    Staged<T, PK, false> sp;
    Staged<T, QK, QI> sq;
    sp.init(p);
    sq.init(q);
    const int w = threadIdx.x / 64;
    const int p0 = w / 2 * 64, q0 = w % 2 * 64;
    const Reader<PK, GEN_B> rp(p0);
    const Reader<QK, GEN_B> rq(q0);
    f32x4 acc[4][4] = {};
    u32x4 vp[2][decltype(sp)::N], vq[2][decltype(sq)::N];
    auto load = [&](int k0, int set) {
        if (k0 < n_k) {
            sp.load(p, k0, n_k, vp[set]);
            sq.load(q, k0, n_k, vq[set]);
        }
    };
    auto step = [&](int k0, int set) {
        u32x4 *lp = lds + set * 2 * BUF, *lq = lp + BUF;
        sp.store(lp, vp[set]);
        sq.store(lq, vq[set]);
        __syncthreads();
        load(k0 + 2 * BK, set);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            u32x4 fp[4], fq[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                fp[i] = rp.get(reinterpret_cast<const char *>(lp), kk, i);
                fq[i] = rq.get(reinterpret_cast<const char *>(lq), kk, i);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = mfma_16x16x32(fq[j], fp[i], acc[i][j], T{});
        }
    };
    sq.fetch_ids(q, 0, n_k);
    load(0, 0);
    load(BK, 1);
    __syncthreads();  // (the last tile's reads of LDS)
    for (int k0 = 0; k0 < n_k; k0 += 2 * BK) {
        step(k0, 0);
        if (k0 + BK < n_k) step(k0 + BK, 1);
    }
    __syncthreads();
    store_tile<OUT, GEN_B, GEN_B, 4, 4, GEN_T>(out, out_stride, p.valid, q.valid, p0, q0, reinterpret_cast<char *>(lds),
                                               [&](int i, int j) { return acc[i][j]; }, skip_p, skip_q);
}

struct ProductArgs {
    const int64_t *gp;
    const int32_t *index;
    int64_t n_groups, n_rows, n_x, n, k;
    const void *x, *w;
    void *y;
    int64_t xs, ws, wg, ys;  // strides: rows of X, rows of W, matrices of W, rows of Y
    int64_t max_row_tiles;   // what the rows allow, whatever group_ptr holds
};

template <typename T, typename OUT, bool TRANS>
__global__ __launch_bounds__(GEN_T, 2) void k_group_product_any(ProductArgs a) {
    __shared__ u32x4 lds[4 * GEN_B * BK / 8];
    const uint32_t n_row = count_row_tiles<GEN_B>(a.gp, a.n_groups, a.n_rows, a.max_row_tiles).full;
    const uint32_t n_col = (uint32_t)((a.n + GEN_B - 1) / GEN_B), total = n_row * n_col;
    for (uint32_t b = blockIdx.x; b < total; b += gridDim.x) {
        uint32_t tr, tc;
        band_tile(xcd_place(b, total), n_row, n_col, tr, tc);
        const RowTile t = find_row_tile<GEN_B>(a.gp, a.n_groups, a.n_rows, tr);
        const int64_t q0 = TRANS ? tile_start(tc, a.n, GEN_B) : (int64_t)tc * GEN_B;
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
        tile_any<T, OUT, false, TRANS, false>(p, q, (int)a.k, out, a.ys, 0, (int)((int64_t)tc * GEN_B - q0), lds);
    }
}

template <typename T, typename OUT, bool TRANS, int BP, int BQ, int WP, int WQ>
__global__ __launch_bounds__(64 * WP * WQ, 2) void k_group_product_fast(ProductArgs a) {
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
        const int64_t q0 = (int64_t)tc * BQ;
        const int cols = (int)(a.n - q0 < BQ ? a.n - q0 : BQ);
        OUT *out = static_cast<OUT *>(a.y) + t.begin * a.ys + q0;
        if (t.group >= a.n_groups) {
            zero_tile(out, a.ys, t.rows, cols);
            continue;
        }
        Dma p{static_cast<const char *>(a.x), span(a.n_x, a.xs * 2, a.k * 2), a.xs * 2, nullptr, a.n_x, t.rows};
        if (a.index) {
            p.index = a.index + t.begin;
        } else {
            p.base += t.begin * p.stride;
            p.records = span(t.rows, p.stride, a.k * 2);
        }
        const char *w = static_cast<const char *>(a.w) + (t.group * a.wg + (TRANS ? q0 : q0 * a.ws)) * 2;
        const uint32_t wb = TRANS ? (uint32_t)cols * 2 : span(cols, a.ws * 2, a.k * 2);
        const Dma q{w, wb, a.ws * 2, nullptr, 0, cols};
        if constexpr (HALF)
            if (half) {
                tile_fast<Mul16<T>, OUT, false, TRANS, true, false, BP / 2, BQ, WP, WQ>(p, q, (int)a.k, out, a.ys, lds_fast, AsTheyAre{});
                continue;
            }
        tile_fast<Mul16<T>, OUT, false, TRANS, true, false, BP, BQ, WP, WQ>(p, q, (int)a.k, out, a.ys, lds_fast, AsTheyAre{});
    }
}

// ------------------------------------------------------------------ few rows
// Groups of a few rows each: the weights are read once and bound the time, so they
// go straight from memory into the matrix unit's registers, any alignment. A
// work group takes 16 rows of a group and 16 NT columns; its waves take turns at blocks
// of 64 reduction elements, FEW_U blocks' loads in flight each, and their sums
// are joined in LDS in the waves' order. A lane's 16 bytes of a row (chunks g
// and g + 4 of the block, the same for both operands) lie next to its
// neighbours'. 64 groups of 1 row, 2048 x 2048, bf16: 112 us (4.8 TB/s of weights);
// one row, 4096 x 4096: 11 us with the call.
constexpr int FEW_U = 4;

// Row of X that the tile's row r stands for, -1 if there is none.
GM_DEV int64_t x_row(const ProductArgs &a, const RowTile &t, int r) {
    if (r >= t.rows) return -1;
    const int64_t i = a.index ? a.index[t.begin + r] : t.begin + r;
    return i >= a.n_x ? -1 : i;
}

template <typename T, typename OUT, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_group_product_few(ProductArgs a) {
    constexpr int BP = 16, BQ = 16 * NT, THREADS = 64 * WAVES;
    __shared__ float part[WAVES][BP][BQ + 4];
    const int lane = threadIdx.x & 63, i16 = lane % 16, g = lane / 16;
    const int w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64));
    const uint32_t n_row = count_row_tiles<BP>(a.gp, a.n_groups, a.n_rows, a.max_row_tiles).full;
    const uint32_t n_col = (uint32_t)((a.n + BQ - 1) / BQ), total = n_row * n_col;
    const int n_k = (int)a.k, full = n_k / 64;
    for (uint32_t b = blockIdx.x; b < total; b += gridDim.x) {
        // the row tiles of a group meet its weights one after the other
        const uint32_t tc = b / n_row, tr = b - tc * n_row;
        const int64_t q0 = (int64_t)tc * BQ;
        const RowTile t = find_row_tile<BP>(a.gp, a.n_groups, a.n_rows, tr);
        const int cols = (int)(a.n - q0 < BQ ? a.n - q0 : BQ);
        OUT *out = static_cast<OUT *>(a.y) + t.begin * a.ys + q0;
        if (t.group >= a.n_groups) {
            zero_tile(out, a.ys, t.rows, cols);
            continue;
        }
        const T *xr, *wr[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int c = 16 * j + i16;
            wr[j] = static_cast<const T *>(a.w) + t.group * a.wg + (q0 + (c < cols ? c : cols - 1)) * a.ws;
        }
        // (a row that is not there reads another: its results are not stored)
        const int64_t xi = x_row(a, t, i16);
        xr = xi < 0 ? wr[0] : static_cast<const T *>(a.x) + xi * a.xs;
        f32x4 acc[NT] = {};
        for (int k0 = w; k0 < full; k0 += WAVES * FEW_U) {
            u32x4 fx[FEW_U][2], fw[FEW_U][NT][2];
#pragma unroll
            for (int u = 0; u < FEW_U; ++u) {
                const int at = min(k0 + u * WAVES, full - 1) * 64 + g * 8;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int j = 0; j < NT; ++j) fw[u][j][h] = load8(wr[j] + at + h * 32, 8);
                    fx[u][h] = load8(xr + at + h * 32, 8);
                }
            }
#pragma unroll
            for (int u = 0; u < FEW_U; ++u)
                if (k0 + u * WAVES < full)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int j = 0; j < NT; ++j) acc[j] = mfma_16x16x32(fw[u][j][h], fx[u][h], acc[j], T{});
        }
        if (full * 64 < n_k && w == full % WAVES) {  // what is left of the last block
            for (int h = 0; h < 2; ++h) {
                const int k = full * 64 + h * 32 + g * 8;
                u32x4 fw[NT];
#pragma unroll
                for (int j = 0; j < NT; ++j) fw[j] = load8(wr[j] + k, n_k - k);
                const u32x4 fx = load8(xr + k, n_k - k);
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[j] = mfma_16x16x32(fw[j], fx, acc[j], T{});
            }
        }
        __syncthreads();  // (the last tile's sums)
#pragma unroll
        for (int j = 0; j < NT; ++j) *reinterpret_cast<f32x4 *>(&part[w][i16][16 * j + 4 * g]) = acc[j];
        __syncthreads();
        for (int i = threadIdx.x; i < t.rows * (BQ / 4); i += THREADS) {
            const int r = i / (BQ / 4), c = i % (BQ / 4) * 4;
            f32x4 s = *reinterpret_cast<const f32x4 *>(&part[0][r][c]);
#pragma unroll
            for (int v = 1; v < WAVES; ++v) s += *reinterpret_cast<const f32x4 *>(&part[v][r][c]);
            if (x_row(a, t, r) < 0) s = f32x4{0, 0, 0, 0};
            store4(out + r * a.ys + c, s, cols - c);
        }
    }
}

struct OuterArgs {
    const int64_t *gp;
    const int32_t *index;
    int64_t n_groups, n_rows, n_x, n, k;
    const void *dy, *x;
    void *d;
    int64_t dys, xs, ds, dg;
    bool by_size;  // see outer_tile
};

// Tile t of the stack of gradients: its group, tile row and tile column. A tile
// costs as much as its group has rows, so where the groups are long (by_size) of
// each 64 the longest come first, and the last work groups to start have little
// to do; a group's tiles are spread over the XCDs, neighbours together. In order
// against by size, 16 groups of 1024 rows on the average, 2048 x 2048, bf16: equal
// groups 129 / 135 us, half of the rows in the last group 213 / 169, sizes that fall
// off exponentially 156 / 134; of 256 rows 62 / 70, 81 / 69, 64 / 63; 64 groups of 256
// rows 248 / 272, 378 / 303, 258 / 282. Ordering costs a tile one to two microseconds,
// so shorter groups are taken as they come (64 groups of 128 equal ones 192 / 219).
GM_DEV void outer_tile(const OuterArgs &a, uint32_t t, uint32_t n_row, uint32_t n_col, uint32_t &e, uint32_t &tr, uint32_t &tc) {
    const uint32_t per = n_row * n_col, place = t / per;
    e = place;
    if (a.by_size) {
        const uint32_t e0 = place / GM_WAVE * GM_WAVE;
        const int lane = threadIdx.x & 63, want = (int)(place - e0);
        int64_t b = 0, f = -1;
        if (e0 + lane < a.n_groups) group_rows(a.gp, a.n_groups, a.n_rows, e0 + lane, b, f);
        const int size = (int)(f - b);  // (lanes past the last group: -1, after all others)
        int rank = 0;
        for (int o = 0; o < GM_WAVE; ++o) {
            const int other = __builtin_amdgcn_readlane(size, o);
            rank += other > size || (other == size && o < lane);
        }
        e = e0 + __ffsll((unsigned long long)ballot(rank == want)) - 1;
    }
    band_tile(xcd_place(t - place * per, per), n_row, n_col, tr, tc);
}

template <typename T, typename OUT, bool IDX>
__global__ __launch_bounds__(GEN_T, 2) void k_group_outer_any(OuterArgs a) {
    __shared__ u32x4 lds[4 * GEN_B * BK / 8];
    const uint32_t n_row = (uint32_t)((a.n + GEN_B - 1) / GEN_B), n_col = (uint32_t)((a.k + GEN_B - 1) / GEN_B);
    const uint32_t total = n_row * n_col * (uint32_t)a.n_groups;
    for (uint32_t b = blockIdx.x; b < total; b += gridDim.x) {
        uint32_t e, tr, tc;
        int64_t begin, end;
        outer_tile(a, b, n_row, n_col, e, tr, tc);
        group_rows(a.gp, a.n_groups, a.n_rows, e, begin, end);
        const int64_t p0 = tile_start(tr, a.n, GEN_B), q0 = tile_start(tc, a.k, GEN_B);
        const Side p{static_cast<const T *>(a.dy) + begin * a.dys + p0, a.dys, nullptr, 0,
                     (int)(a.n - p0 < GEN_B ? a.n - p0 : GEN_B)};
        Side q{static_cast<const T *>(a.x) + q0, a.xs, nullptr, a.n_x, (int)(a.k - q0 < GEN_B ? a.k - q0 : GEN_B)};
        if constexpr (IDX) {
            q.index = a.index + begin;
            if (a.n_x == 0) end = begin;  // (no row to read: all zeros)
        } else {
            q.base = static_cast<const T *>(a.x) + begin * a.xs + q0;
        }
        OUT *out = static_cast<OUT *>(a.d) + e * a.dg + p0 * a.ds + q0;
        tile_any<T, OUT, true, true, IDX>(p, q, (int)(end - begin), out, a.ds, (int)((int64_t)tr * GEN_B - p0), (int)((int64_t)tc * GEN_B - q0), lds);
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

template <typename T, typename OUT, bool IDX, int BP, int BQ, int WP, int WQ>
__global__ __launch_bounds__(64 * WP * WQ, 2) void k_group_outer_fast(OuterArgs a) {
    extern __shared__ char lds_fast[];
    const uint32_t n_row = (uint32_t)((a.n + BP - 1) / BP), n_col = (uint32_t)((a.k + BQ - 1) / BQ);
    const uint32_t total = n_row * n_col * (uint32_t)a.n_groups;
    for (uint32_t b = blockIdx.x; b < total; b += gridDim.x) {
        uint32_t e, tr, tc;
        int64_t begin, end;
        outer_tile(a, b, n_row, n_col, e, tr, tc);
        group_rows(a.gp, a.n_groups, a.n_rows, e, begin, end);
        const int64_t p0 = (int64_t)tr * BP, q0 = (int64_t)tc * BQ;
        const int pv = (int)(a.n - p0 < BP ? a.n - p0 : BP), qv = (int)(a.k - q0 < BQ ? a.k - q0 : BQ);
        const Dma p{static_cast<const char *>(a.dy) + (begin * a.dys + p0) * 2, (uint32_t)(pv * 2), a.dys * 2, nullptr, 0, pv};
        Dma q{static_cast<const char *>(a.x) + q0 * 2, (uint32_t)(qv * 2), a.xs * 2, nullptr, a.n_x, qv};
        if constexpr (IDX) {
            q.index = a.index + begin;
            q.records = span(a.n_x, q.stride, qv * 2);
        } else {
            q.base += begin * q.stride;
        }
        OUT *out = static_cast<OUT *>(a.d) + e * a.dg + p0 * a.ds + q0;
        tile_fast<Mul16<T>, OUT, true, true, false, IDX, BP, BQ, WP, WQ>(p, q, (int)(end - begin), out, a.ds, lds_fast, AsTheyAre{});
    }
}

// The kernel of a product. The host knows the groups' mean size only; every
// kernel is right for any sizes.
enum class Shape { FEW16, FEW64, ANY, T32, T64, T256 };

Shape product_shape(const ProductArgs &a, bool transposed) {
    const int64_t mean = (a.n_rows + a.n_groups - 1) / a.n_groups, groups = a.n_groups < a.n_rows ? a.n_groups : a.n_rows;
    const bool fast = fast_side(a.x, a.xs, 0, a.k, a.index ? a.n_x : 256) &&
                      fast_side(a.w, a.ws, a.n_groups > 1 ? a.wg : 0, transposed ? a.n : a.k, 256);
    // Up to 16 rows a group the weights' bytes are all there is. 64 columns a work
    // group (64 groups, 2048 x 2048, sizes as chance deals them, of 1, 4 and 16 rows on
    // the average: 80, 111 and 142 us; tiles of 32 x 128 84, 149 and 156; of 24 rows 180
    // against 172) unless that leaves CUs without one, then 16 (4 groups of 1 row: 10.9
    // against 12.9). Rows that are not aligned are slower with 64 (64 groups of 1 row,
    // 2047 x 2047: 194 us, staged tiles 101), not with 16 (4 groups: 29 / 37). Where one
    // group has all the rows its weights are read for every 16 of them, from the
    // caches: mean 16, 77 against 24 us with tiles of 32 x 128.
    if (!transposed && mean <= 16) {
        if (groups * ((a.n + 63) / 64) < 256) return Shape::FEW16;
        if (fast) return Shape::FEW64;
    }
    if (!fast) return Shape::ANY;
    // Tiles of 32 rows or of 64 by the groups' height: of 48 rows 130 against 177 us, of
    // 64 rows 143 / 151, of 96 rows 169 / 152 (all rows in one of the groups, mean 64: 58 /
    // 50); transposed 24 rows 122 / 125, 32 rows 116 / 127, and of 48 rows still 128 / 133.
    if (mean <= (transposed ? 32 : 64)) return Shape::T32;
    return big_product_tiles(mean, a.n, groups) ? Shape::T256 : Shape::T64;
}

// Whether a gradient's tiles are 256 x 256 rather than 128 x 128. A tile takes as
// long as its group has rows, so there have to be several a CU to even that out,
// unless there is one group. Equal groups, then rows cut at random: 64 groups of 256
// rows on the average, 2048 x 2048 (4096 tiles), 289 against 407 us and 281 / 373, 768 x
// 1024 (768 tiles) 57 / 76 and 52 / 73; 16 groups of 1024 rows, 1024 x 1024 (256 tiles),
// 40 / 56 and 74 / 58; one group of 1024 rows, 4096 x 4096 (256 tiles), 35 / 41, 2048 x
// 2048 (64 tiles) 27 / 16. And not where padding grows by more than a third.
bool big_outer_tiles(int64_t n, int64_t k, int64_t n_groups) {
    const int64_t tiles = (n + 255) / 256 * ((k + 255) / 256), small = (n + 127) / 128 * ((k + 127) / 128);
    return tiles * n_groups >= (n_groups == 1 ? 192 : 512) && 3 * 4 * tiles <= 4 * small;
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
        check_dense(X, "X", x_rows(*groups, *X), k);
        check_dense(Y, "Y", groups->n_rows, n);
        check_dense(W, "W", transposed ? k : n, transposed ? n : k, groups->n_groups);
        GM_REQUIRE(X->n_rows >= 0 && X->n_rows < INT32_MAX, GMAGNUS_ERROR_UNSUPPORTED, "rows of X beyond 2^31 - 2");
        GM_REQUIRE(is_16bit(X->data_type) && W->data_type == X->data_type, GMAGNUS_ERROR_INVALID_VALUE,
                   "X and W must both be bf16 or both fp16");
        GM_REQUIRE(Y->data_type == X->data_type || Y->data_type == GMAGNUS_DATA_FP32, GMAGNUS_ERROR_INVALID_VALUE,
                   "Y must have the type of X, or fp32");
        if (groups->n_rows == 0) return;
        const ProductArgs a{groups->group_ptr, groups->index, groups->n_groups, groups->n_rows, X->n_rows, n, k,
                            X->data, W->data, Y->data, X->row_stride, W->row_stride, W->stack_stride, Y->row_stride, 0};
        hipStream_t s = (hipStream_t)hip_stream;
        const Shape shape = product_shape(a, transposed);
        with_elem(X->data_type, Y->data_type, [&](auto t, auto o) {
            using T = decltype(t);
            using O = decltype(o);
            auto launch = [&](auto kernel, int bp, int bq, int threads, int lds) {
                ProductArgs f = a;
                f.max_row_tiles = row_tiles_bound(a.n_groups, a.n_rows, bp);
                launch_fast(kernel, f.max_row_tiles * ((n + bq - 1) / bq), threads, lds, f, s);
            };
            auto fast = [&](auto trans) {
                constexpr bool TR = decltype(trans)::value;
                if (shape == Shape::T32)
                    launch(k_group_product_fast<T, O, TR, 32, 128, 1, 4>, 32, 128, 256, fast_bytes(32, 128));
                else if (shape == Shape::T64)
                    launch(k_group_product_fast<T, O, TR, 64, 128, 2, 2>, 64, 128, 256, fast_bytes(64, 128));
                else
                    launch(k_group_product_fast<T, O, TR, 256, 256, 2, 4>, 256, 256, 512, fast_bytes(256, 256));
            };
            if (shape == Shape::FEW16)
                launch(k_group_product_few<T, O, 1, 4>, 16, 16, 256, 0);
            else if (shape == Shape::FEW64)
                launch(k_group_product_few<T, O, 4, 4>, 16, 64, 256, 0);
            else if (shape == Shape::ANY && transposed)
                launch(k_group_product_any<T, O, true>, GEN_B, GEN_B, GEN_T, 0);
            else if (shape == Shape::ANY)
                launch(k_group_product_any<T, O, false>, GEN_B, GEN_B, GEN_T, 0);
            else if (transposed)
                fast(std::true_type{});
            else
                fast(std::false_type{});
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
        check_dense(X, "X", x_rows(*groups, *X), k);
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
                          groups->n_rows / groups->n_groups >= 256};
        hipStream_t s = (hipStream_t)hip_stream;
        const bool fast = fast_side(a.dy, a.dys, 0, n, BK) && fast_side(a.x, a.xs, 0, k, a.index ? a.n_x : BK);
        const bool big = big_outer_tiles(n, k, a.n_groups);
        with_elem(X->data_type, D->data_type, [&](auto t, auto o) {
            using T = decltype(t);
            using O = decltype(o);
            auto launch = [&](auto kernel, int b, int threads, int lds) {
                const int64_t tiles = (n + b - 1) / b * ((k + b - 1) / b);
                GM_REQUIRE(tiles < INT32_MAX / a.n_groups, GMAGNUS_ERROR_UNSUPPORTED, "2^31 tiles or more");
                launch_fast(kernel, tiles * a.n_groups, threads, lds, a, s);
            };
            auto go = [&](auto idx) {
                constexpr bool IX = decltype(idx)::value;
                if (!fast)
                    launch(k_group_outer_any<T, O, IX>, GEN_B, GEN_T, 0);
                else if (big)
                    launch(k_group_outer_fast<T, O, IX, 256, 256, 2, 4>, 256, 512, fast_bytes(256, 256));
                else
                    launch(k_group_outer_fast<T, O, IX, 128, 128, 2, 2>, 128, 256, fast_bytes(128, 128));
            };
            if (a.index)
                go(std::true_type{});
            else
                go(std::false_type{});
        });
        GM_CHECK_LAUNCH();
    });
}
