// What a layer of experts does to whole rows around its products: the root-mean-
// square norm with the residual's addition, the gate of a pair of columns, and
// the rounding of rows to 8-bit integers; each result in the rows' type, in 8 bits with
// scales, or both; and the gradients of the first two.
//   h = x + residual (rounded to its type),  y = h w / sqrt(mean(h^2) + eps)
//   a = silu(g) u for rows [g | u],          silu(g) = g / (1 + e^-g)
// All of it is bound by its bytes, so a row is read once and held in registers until
// what is needed of the whole row is known: eight columns of a piece to a lane, CH
// pieces, by one wave or by the W waves of a work group. Rows longer than that are
// read again for each thing to be known.
#include "quant.hpp"

namespace gm {
namespace {

enum class Op { NORM, GATE, COPY };
enum { IN_TYPE = 0, E4M3 = 1, INTEGER = 2 };  // the 8-bit result

struct RowArgs {
    const void *x, *r, *w;  // rows (of the gate: pairs), residual, weight; the latter two may be null
    void *total, *y;        // may be null
    uint8_t *q;
    float *scale;
    int64_t n_rows, n, xs, rs, ts, ys, qs, ss;
    int64_t stack_rows, xg, qg, sg;  // rows of each matrix of a stack, strides between those
    float eps;
    int format;
    bool w32;
    bool in_place;  // total is x or the residual
};

template <int ROR>
GM_DEV uint32_t max_with_ror(uint32_t x) {
    const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + ROR, 0xf, 0xf, false);
    return x > y ? x : y;
}
// The largest of 16 neighbouring lanes', in all of them.
GM_DEV uint32_t max16(uint32_t x) { return max_with_ror<1>(max_with_ror<2>(max_with_ror<4>(max_with_ror<8>(x)))); }

// Sums and maxima over the W waves of a row. Two sets of places (for pairs of sums two
// each): a set is written again behind the barrier of the next one, when all have read it.
template <int W>
struct Join {
    float (*part)[W];
    int turn = 0;
    GM_DEV float sum(float x) {
        x = wave_sum(x);
        if constexpr (W > 1) {
            float *p = part[turn];
            turn ^= 1;
            if ((threadIdx.x & 63) == 0) p[threadIdx.x / 64] = x;
            __syncthreads();
            x = p[0];
#pragma unroll
            for (int i = 1; i < W; ++i) x += p[i];
        }
        return x;
    }
    GM_DEV void sums(float &x, float &y) {
        x = wave_sum(x);
        y = wave_sum(y);
        if constexpr (W > 1) {
            float *p = part[turn], *q = part[turn + 2];
            turn ^= 1;
            if ((threadIdx.x & 63) == 0) {
                p[threadIdx.x / 64] = x;
                q[threadIdx.x / 64] = y;
            }
            __syncthreads();
            x = p[0];
            y = q[0];
#pragma unroll
            for (int i = 1; i < W; ++i) {
                x += p[i];
                y += q[i];
            }
        }
    }
    GM_DEV uint32_t most(uint32_t x) {
        x = wave_max(x);
        if constexpr (W > 1) {
            float *p = part[turn];
            turn ^= 1;
            if ((threadIdx.x & 63) == 0) p[threadIdx.x / 64] = __uint_as_float(x);
            __syncthreads();
            x = 0;
#pragma unroll
            for (int i = 0; i < W; ++i) x = max(x, __float_as_uint(p[i]));
        }
        return x;
    }
};

GM_DEV int columns_left(int64_t n, int64_t c) { return n - c >= 8 ? 8 : n > c ? (int)(n - c) : 0; }

// Eight columns, of which `valid` are there. WHOLE: all or none are, which leaves out what
// cut pieces take (the norm of 4096 bf16 columns 102 -> 84 registers).
template <bool WHOLE, typename T>
GM_DEV void load(const T *p, int valid, float (&v)[8]) {
    if constexpr (WHOLE) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
        if (valid > 0) load_f32x8(p, 8, v);
    } else {
        load_f32x8(p, valid, v);
    }
}
template <bool WHOLE, typename T>
GM_DEV void store(T *p, int valid, const float (&v)[8]) {
    if constexpr (WHOLE) {
        if (valid > 0) store_f32(p, 8, v);
    } else {
        store_f32(p, valid, v);
    }
}

// Eight columns as they lie in memory, for what is on its way while another row is worked on.
template <bool WHOLE, typename T>
struct Piece {
    u32x4 v[sizeof(T) / 2];
    GM_DEV void fetch(const T *p, int valid) {
        if constexpr (sizeof(T) == 2) {
            v[0] = load8(p, WHOLE ? (valid > 0 ? 8 : 0) : valid);
        } else {
            float x[8];
            load<WHOLE>(p, valid, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i / 4][i % 4] = __float_as_uint(x[i]);
        }
    }
    GM_DEV void get(float (&x)[8]) const {
        if constexpr (sizeof(T) == 2) {
            typedef T vec __attribute__((ext_vector_type(8)));
            const vec t = __builtin_bit_cast(vec, v[0]);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (float)t[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(v[i / 4][i % 4]);
        }
    }
};

// Of a weight of type T, or float32 (w32); null: ones.
template <bool WHOLE, typename T>
GM_DEV void load_weight(const void *w, bool w32, int64_t c, int valid, float (&v)[8]) {
    if (!w) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 1.f;
    } else if (w32) {
        load<WHOLE>(static_cast<const float *>(w) + c, valid, v);
    } else {
        load<WHOLE>(static_cast<const T *>(w) + c, valid, v);
    }
}

// Where row number `row` of a stack lies.
struct Place {
    int64_t g, r;
    GM_DEV Place(const RowArgs &a, int64_t row) {
        g = a.stack_rows == a.n_rows ? 0 : row / a.stack_rows;
        r = row - g * a.stack_rows;
    }
};

// Eight columns of what comes before anything is known of the row: the gate's and
// a copy's results, the norm's h (which goes to `total`, and is read there when `again`
// if x or the residual is that memory; reading those two again is quicker: 3277 x 20480 bf16 132 us for 138).
template <Op OP, bool WHOLE, typename T>
GM_DEV void load_piece(const RowArgs &a, const T *x, int64_t row, int64_t c, int valid, bool again, float (&v)[8]) {
    if (OP == Op::NORM && again && a.in_place) {
        load<WHOLE>(static_cast<const T *>(a.total) + row * a.ts + c, valid, v);
        return;
    }
    if constexpr (OP == Op::GATE) {
        float u[8];
        if (WHOLE && valid <= 0) {  // (both loads behind one branch, or the second waits for the first)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.f;
            return;
        }
        load_f32x8(x + c, WHOLE ? 8 : valid, v);
        load_f32x8(x + a.n + c, WHOLE ? 8 : valid, u);
        gated8(v, u, v);
        return;
    }
    load<WHOLE>(x + c, valid, v);
    if constexpr (OP == Op::NORM) {
        if (a.r) {
            float u[8];
            load<WHOLE>(static_cast<const T *>(a.r) + row * a.rs + c, valid, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = to_f32((T)(v[i] + u[i]));
            if (!again) store<WHOLE>(static_cast<T *>(a.total) + row * a.ts + c, valid, v);
        }
    }
}

// Eight columns of the results; E4M3: 16 lanes hold a block of 128.
template <bool WHOLE, typename T>
GM_DEV void store_piece(const RowArgs &a, const Place &at, int64_t row, int64_t c, int valid, const float (&v)[8], float scale, float inverse) {
    if (a.y) store<WHOLE>(static_cast<T *>(a.y) + row * a.ys + c, valid, v);
    uint8_t *q = a.q + at.g * a.qg + at.r * a.qs + c;
    if (a.format == E4M3) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, magnitude(v[i]));
        const float s = block_scale(max16(m));
        if (valid > 0) {
            store_fp8x8_by(q, WHOLE ? 8 : valid, v, s, 1.f / s);
            if (threadIdx.x % 16 == 0) a.scale[row * a.ss + c / SB] = s;
        }
    } else if (a.format == INTEGER) {
        if (valid > 0) store_int8x8_by(q, WHOLE ? 8 : valid, v, scale, inverse);
    }
}

// Bound by its bytes. Norm of 16384 x 4096 bf16 with residual, its sum and its results in bf16 and E4M3 114-118 us
// (5.1-5.3 TB/s; without the next row on its way 120), without residual to bf16 44 us (6.1), to E4M3 alone 50
// (4.0), to integers 52; gate of 32768 x 2048 to E4M3 64 us (5.2), to integers 70, 9001 x 1365 fp16 21-22 us (3.4);
// integers of 8192 x 4096 22 us (4.6), of 65536 x 777 50 (3.0). One row of 4096 with all results 3.5 us.
// Rows that end inside a piece have 16 to 96 bytes of scratch a lane, through which the next row passes in the norm of
// 2049 to 4096 columns: 16384 x 4095 with residual 156 us, 4096 columns 101.
template <Op OP, typename T, int W, int CH, bool WHOLE>
__global__ __launch_bounds__(W > 4 ? 64 * W : 256) void k_rows(RowArgs a) {
    constexpr int PER = W == 1 ? 4 : 1;  // rows of a work group
    __shared__ float part[2][W];
    Join<W> join{part};
    const int t = W == 1 ? threadIdx.x % 64 : threadIdx.x;
    int valid[CH];
    float w[OP == Op::NORM ? CH : 1][8];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int64_t c = (j * W * 64 + t) * 8;
        valid[j] = columns_left(a.n, c);
        if constexpr (OP == Op::NORM) load_weight<WHOLE, T>(a.w, a.w32, c, valid[j], w[j]);
    }
    const int64_t step = (int64_t)gridDim.x * PER;
    Piece<WHOLE, T> nx[CH], nr[CH];  // the next row (the gate's are long enough, and rows enough)
    auto fetch = [&](int64_t row) {
        const Place at(a, row);
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int64_t c = (j * W * 64 + t) * 8;
            nx[j].fetch(static_cast<const T *>(a.x) + at.g * a.xg + at.r * a.xs + c, valid[j]);
            if (OP == Op::NORM && a.r) nr[j].fetch(static_cast<const T *>(a.r) + row * a.rs + c, valid[j]);
        }
    };
    int64_t row = (int64_t)blockIdx.x * PER + (W == 1 ? threadIdx.x / 64 : 0);
    if constexpr (OP != Op::GATE)
        if (row < a.n_rows) fetch(row);
    for (; row < a.n_rows; row += step) {
        const Place at(a, row);
        float v[CH][8];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int64_t c = (j * W * 64 + t) * 8;
            if constexpr (OP != Op::GATE) {
                nx[j].get(v[j]);
                if (OP == Op::NORM && a.r) {
                    float u[8];
                    nr[j].get(u);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[j][i] = to_f32((T)(v[j][i] + u[i]));
                    store<WHOLE>(static_cast<T *>(a.total) + row * a.ts + c, valid[j], v[j]);
                }
            } else {
                load_piece<OP, WHOLE>(a, static_cast<const T *>(a.x) + row * a.xs, row, c, valid[j], false, v[j]);
            }
        }
        if constexpr (OP != Op::GATE)
            if (row + step < a.n_rows) fetch(row + step);
        if constexpr (OP == Op::NORM) {
            float s = 0.f;
#pragma unroll
            for (int j = 0; j < CH; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) s += v[j][i] * v[j][i];
            const float r = 1.f / sqrtf(join.sum(s) / (float)a.n + a.eps);
#pragma unroll
            for (int j = 0; j < CH; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[j][i] = i < valid[j] ? v[j][i] * r * w[j][i] : 0.f;
        }
        float scale = 0.f, inverse = 0.f;
        if (a.format == INTEGER) {
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < CH; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) m = max(m, magnitude(v[j][i]));
            scale = row_scale(join.most(m));
            inverse = 1.f / scale;
            if (t == 0) a.scale[at.g * a.sg + at.r] = scale;
        }
#pragma unroll
        for (int j = 0; j < CH; ++j) store_piece<WHOLE, T>(a, at, row, (j * W * 64 + t) * 8, valid[j], v[j], scale, inverse);
    }
}

// Rows of any length: what is to be known of a row is found in passes of their own.
constexpr int LONG_W = 16;

template <Op OP, typename T, bool WHOLE>
__global__ __launch_bounds__(64 * LONG_W) void k_rows_long(RowArgs a) {
    __shared__ float part[2][LONG_W];
    Join<LONG_W> join{part};
    constexpr int64_t STEP = 64 * LONG_W * 8;
    for (int64_t row = blockIdx.x; row < a.n_rows; row += gridDim.x) {
        const Place at(a, row);
        const T *x = static_cast<const T *>(a.x) + at.g * a.xg + at.r * a.xs;
        float v[8], w[8], r = 0.f, scale = 0.f, inverse = 0.f;
        if constexpr (OP == Op::NORM) {
            float s = 0.f;
            for (int64_t c0 = 0; c0 < a.n; c0 += STEP) {
                const int64_t c = c0 + threadIdx.x * 8;
                load_piece<OP, WHOLE>(a, x, row, c, columns_left(a.n, c), false, v);
                float p = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) p += v[i] * v[i];
                s += p;
            }
            r = 1.f / sqrtf(join.sum(s) / (float)a.n + a.eps);
        }
        auto piece = [&](int64_t c, int valid) {
            load_piece<OP, WHOLE>(a, x, row, c, valid, true, v);
            if constexpr (OP == Op::NORM) {
                load_weight<WHOLE, T>(a.w, a.w32, c, valid, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = i < valid ? v[i] * r * w[i] : 0.f;
            }
        };
        if (a.format == INTEGER) {
            uint32_t m = 0;
            for (int64_t c0 = 0; c0 < a.n; c0 += STEP) {
                const int64_t c = c0 + threadIdx.x * 8;
                piece(c, columns_left(a.n, c));
#pragma unroll
                for (int i = 0; i < 8; ++i) m = max(m, magnitude(v[i]));
            }
            scale = row_scale(join.most(m));
            inverse = 1.f / scale;
            if (threadIdx.x == 0) a.scale[at.g * a.sg + at.r] = scale;
        }
        for (int64_t c0 = 0; c0 < a.n; c0 += STEP) {
            const int64_t c = c0 + threadIdx.x * 8;
            const int valid = columns_left(a.n, c);
            piece(c, valid);
            store_piece<WHOLE, T>(a, at, row, c, valid, v, scale, inverse);
        }
    }
}

// ------------------------------------------------------------ norm's gradients
// With r = 1 / sqrt(mean(h^2) + eps), g = d_y w and c = mean(g h) r^2:
//   d_h = r (g - h c) + d_total,   d_w = sum over rows of d_y h r
// A work group takes rows in turns and holds its share of d_w in registers; the
// shares are added in their order by a second kernel, so results do not change from
// run to run. While a row's sums are joined the next row is on its way: 8192 x 4096 bf16
// with three operands 43-45 us, 6.0-6.2 TB/s (without 83); 1024 work groups 49, and the
// shares' sum 6 instead of 5. 4095 columns, which end inside a piece (176 to 213 registers
// and scratch), take 115 us with that sum, 4096 48.
struct NormBackArgs {
    const void *h, *w, *d_y, *d_total;
    void *d_h;
    float *share;    // [units][n], null: d_w is not wanted
    float *of_row;   // long rows: r and c
    int64_t n_rows, n, hs, ds, ts, os;
    float eps;
    bool w32;
};

template <typename T, int W, int CH, bool WHOLE>
__global__ __launch_bounds__(W > 4 ? 64 * W : 256) void k_norm_backward(NormBackArgs a) {
    constexpr int PER = W == 1 ? 4 : 1;
    __shared__ float part[4][W];
    __shared__ float whole[W == 1 ? CH * 512 : 1];
    Join<W> join{part};
    const int t = W == 1 ? threadIdx.x % 64 : threadIdx.x;
    const int64_t step = (int64_t)gridDim.x * PER;
    int valid[CH];
    float w[CH][8], share[CH][8] = {};
    Piece<WHOLE, T> nh[CH], nd[CH], nt[CH];  // of the next row
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int64_t c = (j * W * 64 + t) * 8;
            nh[j].fetch(static_cast<const T *>(a.h) + row * a.hs + c, valid[j]);
            nd[j].fetch(static_cast<const T *>(a.d_y) + row * a.ds + c, valid[j]);
            if (a.d_total) nt[j].fetch(static_cast<const T *>(a.d_total) + row * a.ts + c, valid[j]);
        }
    };
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int64_t c = (j * W * 64 + t) * 8;
        valid[j] = columns_left(a.n, c);
        load_weight<WHOLE, T>(a.w, a.w32, c, valid[j], w[j]);
    }
    int64_t row = (int64_t)blockIdx.x * PER + (W == 1 ? threadIdx.x / 64 : 0);
    if (row < a.n_rows) fetch(row);
    for (; row < a.n_rows; row += step) {
        float h[CH][8], d[CH][8], o[CH][8], square = 0.f, dot = 0.f;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            nh[j].get(h[j]);
            nd[j].get(d[j]);
            nt[j].get(o[j]);
        }
        if (row + step < a.n_rows) fetch(row + step);
#pragma unroll
        for (int j = 0; j < CH; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                square += h[j][i] * h[j][i];
                dot += d[j][i] * w[j][i] * h[j][i];
            }
        join.sums(square, dot);
        const float r = 1.f / sqrtf(square / (float)a.n + a.eps), c = r * (dot / (float)a.n) * r;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                share[j][i] += d[j][i] * (h[j][i] * r);
                const float x = r * (d[j][i] * w[j][i] - h[j][i] * c);
                o[j][i] = a.d_total ? x + o[j][i] : x;
            }
            store<WHOLE>(static_cast<T *>(a.d_h) + row * a.os + (j * W * 64 + t) * 8, valid[j], o[j]);
        }
    }
    if (!a.share) return;
    if constexpr (W == 1) {  // the four waves' shares
        for (int v = 0; v < 4; ++v) {
            if ((int)threadIdx.x / 64 == v)
#pragma unroll
                for (int j = 0; j < CH; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float *p = &whole[i * (CH * 64) + j * 64 + t];
                        *p = v ? *p + share[j][i] : share[j][i];
                    }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < CH * 512; c += 256)
            if (c < a.n) a.share[blockIdx.x * a.n + c] = whole[c % 8 * (CH * 64) + c / 8];
    } else {
#pragma unroll
        for (int j = 0; j < CH; ++j) store<WHOLE>(a.share + blockIdx.x * a.n + (j * W * 64 + t) * 8, valid[j], share[j]);
    }
}

// d_w from the units' shares: 64 columns a work group, a wave every 16th unit.
__global__ __launch_bounds__(1024) void k_add_shares(const float *share, int64_t n, int units, float *out) {
    __shared__ float part[16][64];
    const int x = threadIdx.x % 64, w = threadIdx.x / 64;
    for (int64_t c0 = (int64_t)blockIdx.x * 64; c0 < n; c0 += (int64_t)gridDim.x * 64) {
        const int64_t c = c0 + x;
        float s = 0.f;
        if (c < n)
#pragma unroll 8
            for (int u = w; u < units; u += 16) s += share[u * n + c];
        part[w][x] = s;
        __syncthreads();
        if (w == 0 && c < n) {
#pragma unroll
            for (int i = 1; i < 16; ++i) s += part[i][x];
            out[c] = s;
        }
        __syncthreads();
    }
}

// Rows of any length: r and c of each row, then the columns 512 at a time. 4096 rows of 12288
// columns 118 us, of 16384 163 (all is read twice).
template <typename T, bool WHOLE>
__global__ __launch_bounds__(64 * LONG_W) void k_norm_backward_rows(NormBackArgs a) {
    __shared__ float part[4][LONG_W];
    Join<LONG_W> join{part};
    for (int64_t row = blockIdx.x; row < a.n_rows; row += gridDim.x) {
        float square = 0.f, dot = 0.f;
        for (int64_t c0 = 0; c0 < a.n; c0 += 64 * LONG_W * 8) {
            const int64_t c = c0 + threadIdx.x * 8;
            const int valid = columns_left(a.n, c);
            float h[8], d[8], w[8], p = 0.f, q = 0.f;
            load<WHOLE>(static_cast<const T *>(a.h) + row * a.hs + c, valid, h);
            load<WHOLE>(static_cast<const T *>(a.d_y) + row * a.ds + c, valid, d);
            load_weight<WHOLE, T>(a.w, a.w32, c, valid, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p += h[i] * h[i];
                q += d[i] * w[i] * h[i];
            }
            square += p;
            dot += q;
        }
        join.sums(square, dot);
        if (threadIdx.x == 0) {
            const float r = 1.f / sqrtf(square / (float)a.n + a.eps);
            a.of_row[2 * row] = r;
            a.of_row[2 * row + 1] = r * (dot / (float)a.n) * r;
        }
    }
}

template <typename T, bool WHOLE>
__global__ __launch_bounds__(64) void k_norm_backward_columns(NormBackArgs a, int units) {
    const int64_t pieces = (a.n + 511) / 512;
    for (int64_t b = blockIdx.x; b < pieces * units; b += gridDim.x) {
        const int64_t u = b / pieces, c = (b - u * pieces) * 512 + threadIdx.x * 8;
        const int valid = columns_left(a.n, c);
        float w[8], share[8] = {};
        load_weight<WHOLE, T>(a.w, a.w32, c, valid, w);
        for (int64_t row = u; row < a.n_rows; row += units) {
            const float r = a.of_row[2 * row], cr = a.of_row[2 * row + 1];
            float h[8], d[8], o[8] = {};
            load<WHOLE>(static_cast<const T *>(a.h) + row * a.hs + c, valid, h);
            load<WHOLE>(static_cast<const T *>(a.d_y) + row * a.ds + c, valid, d);
            if (a.d_total) load<WHOLE>(static_cast<const T *>(a.d_total) + row * a.ts + c, valid, o);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                share[i] += d[i] * (h[i] * r);
                o[i] += r * (d[i] * w[i] - h[i] * cr);
            }
            store<WHOLE>(static_cast<T *>(a.d_h) + row * a.os + c, valid, o);
        }
        if (a.share) store<WHOLE>(a.share + u * a.n + c, valid, share);
    }
}

// ------------------------------------------------------------- gate's gradient
// With s = sigma(g): d_g = d_a u s (1 + g (1 - s)), d_u = d_a g s. Eight columns a
// lane, no row is needed as a whole. Where s is below fp32's normal numbers, or d_a u
// above its largest, the products are made of fractions and exponents. 16384 x 2048
// bf16 60 us, 9001 x 1365 fp16 23 us, 5.4 TB/s.
GM_DEV void gate_slopes(float g, float u, float d, float &d_g, float &d_u) {
    float s, rest;
    sigmoid(g, s, rest);
    d_g = d * u * (s * (1.f + g * rest));
    d_u = d * (g * s);
}
// (Values that are neither far nor too large: as above, whatever lies beside them.)
GM_DEV void gate_slopes_apart(float g, float u, float d, float &d_g, float &d_u) {
    if (g < -FAR) {
        int k;
        const float m = exp_apart(g, k);
        d_g = product_apart(d, u, 1.f + g, m, k);
        d_u = product_apart(d, g, 1.f, m, k);
    } else if (fabsf(d * u) == INFINITY) {
        float s, rest;
        sigmoid(g, s, rest);
        d_g = product_apart(d, u, s * (1.f + g * rest), 1.f, 0);
        d_u = d * (g * s);
    } else {
        gate_slopes(g, u, d, d_g, d_u);
    }
}

struct GateBackArgs {
    const void *h, *d_a;
    void *d_h;
    int64_t n_rows, n, hs, ds, os;
};

template <typename T, bool WHOLE>
__global__ __launch_bounds__(256) void k_gate_backward(GateBackArgs a) {
    const uint32_t pieces = (uint32_t)((a.n + 7) / 8);
    const int64_t total = a.n_rows * pieces;
    for (int64_t b = blockIdx.x * 256ll + threadIdx.x; b < total; b += gridDim.x * 256ll) {
        const int64_t row = total < INT32_MAX ? (uint32_t)b / pieces : b / pieces, c = (b - row * pieces) * 8;
        // (no lane is without columns: said outright, or each load has a branch and a wait of its own)
        const int valid = WHOLE ? 8 : columns_left(a.n, c);
        const T *h = static_cast<const T *>(a.h) + row * a.hs + c;
        T *o = static_cast<T *>(a.d_h) + row * a.os + c;
        float g[8], u[8], d[8];
        load<WHOLE>(h, valid, g);
        load<WHOLE>(h + a.n, valid, u);
        load<WHOLE>(static_cast<const T *>(a.d_a) + row * a.ds + c, valid, d);
        float most = 0.f;  // (a NaN leaves it as it is, and is one below)
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(d[i] * u[i]));
        if (any_far(g) || __builtin_expect(most == INFINITY, 0)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                gate_slopes_apart(g[i], u[i], d[i], u[i], d[i]);
                __builtin_amdgcn_sched_barrier(0);  // (as in gated8)
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) gate_slopes(g[i], u[i], d[i], u[i], d[i]);
        }
        store<WHOLE>(o, valid, u);
        store<WHOLE>(o + a.n, valid, d);
    }
}

// ------------------------------------------------------------------- host side
// Work groups, each of which takes rows in turns with the next one's loads on its way (and the norm's weight in
// registers). Norm of 16384 x 4096: 512 work groups 51 us, 1024 44, 2048 44, with residual and E4M3 result 88, 92, 90, of
// 8192 x 4096 30, 25, 25 and 45, 42, 42; with residual, 131072 x 256: 512 93, 2048 70. Integers, 8192 x 4096: 512 34,
// 1024 28, 2048 23, one for each row 23, 8192 x 8192 46, 42, 41, 48.
int64_t rows_grid(int64_t n, bool norm) { return norm && n > 512 ? 1024 : 2048; }
constexpr int64_t BACK_UNITS = 512;   // shares of d_w

int64_t back_units(int64_t t, int64_t n) {
    const int64_t per = n <= 1024 ? 4 : 1, units = (t + per - 1) / per;
    return units < BACK_UNITS ? units : BACK_UNITS;
}
// The longest rows that registers hold; the gradients hold four things of a row for the norm's two, which 16
// waves have no room for.
constexpr int64_t HELD = 64 * LONG_W * 2 * 8, HELD_BACK = HELD / 2;

struct BackLayout {
    int64_t share, of_row, bytes;
    BackLayout(int64_t t, int64_t n) {
        share = 0;
        of_row = (back_units(t, n) * n * 4 + 255) / 256 * 256;
        bytes = of_row + (n > HELD_BACK ? t * 8 : 0);
    }
};

bool back_sizes_ok(int64_t t, int64_t n) { return t >= 0 && t < INT32_MAX && n >= 1 && n <= MAX_SIDE; }

// f(W{}, CH{}, WHOLE{}): waves of a row of n columns and its pieces a lane (W 0: any length), and whether its
// pieces are whole.
template <class F>
void with_row(int64_t n, F &&f) {
    auto whole = [&](auto w, auto ch) {
        if (n % 8 == 0)
            f(w, ch, std::true_type{});
        else
            f(w, ch, std::false_type{});
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    using I2 = std::integral_constant<int, 2>;
    using I4 = std::integral_constant<int, 4>;
    using I8 = std::integral_constant<int, 8>;
    using I16 = std::integral_constant<int, 16>;
    if (n <= 512)
        whole(I1{}, I1{});
    else if (n <= 1024)
        whole(I1{}, I2{});
    else if (n <= 2048)
        whole(I4{}, I1{});
    else if (n <= 4096)
        whole(I4{}, I2{});
    else if (n <= 8192)
        whole(I8{}, I2{});
    else if (n <= HELD)
        whole(I16{}, I2{});
    else
        whole(I0{}, I0{});
}

template <Op OP>
void launch_rows(const RowArgs &a, int32_t type, hipStream_t s) {
    with_float(type, [&](auto v) {
        using T = decltype(v);
        with_row(a.n, [&](auto waves, auto pieces, auto whole) {
            constexpr int W = decltype(waves)::value, CH = decltype(pieces)::value;
            constexpr bool WHOLE = decltype(whole)::value;
            if constexpr (W == 0) {
                hipLaunchKernelGGL((k_rows_long<OP, T, WHOLE>), dim3(grid_for(a.n_rows, 1, 1 << 16)), dim3(64 * LONG_W), 0, s, a);
            } else {
                const int64_t most = OP == Op::GATE ? max_grid(W > 4 ? 64 * W : 256) : rows_grid(a.n, OP == Op::NORM);
                hipLaunchKernelGGL((k_rows<OP, T, W, CH, WHOLE>), dim3(grid_for(a.n_rows, W == 1 ? 4 : 1, most)),
                                   dim3(W > 4 ? 64 * W : 256), 0, s, a);
            }
        });
    });
    GM_CHECK_LAUNCH();
}

void check_rows_n(int64_t t, int64_t n, const char *name) {
    GM_REQUIRE(t >= 0, GMAGNUS_ERROR_INVALID_VALUE, std::string("negative rows of ") + name);
    GM_REQUIRE(t < INT32_MAX, GMAGNUS_ERROR_UNSUPPORTED, std::string("rows of ") + name + " beyond 2^31 - 2");
    check_side(n, "columns");
}

// A result or operand of the shape and type of the rows.
void check_like(const gmagnus_dense_t *m, const char *name, int64_t t, int64_t n, int32_t type) {
    check_dense(m, name, t, n);
    GM_REQUIRE(m->data_type == type, GMAGNUS_ERROR_INVALID_VALUE, std::string(name) + " has another type than the rows");
}

void check_weight(const gmagnus_dense_t *w, int64_t n, int32_t type) {
    if (!w) return;
    check_dense(w, "weight", 1, n);
    GM_REQUIRE(w->data_type == type || w->data_type == GMAGNUS_DATA_FP32, GMAGNUS_ERROR_INVALID_VALUE,
               "weight must have the type of the rows, or fp32");
}

// Whether rows of two matrices share memory (rows may lie between one another's).
bool overlap(const gmagnus_dense_t &a, const gmagnus_dense_t &b) {
    struct Place {
        int64_t at, rows, stride, width;  // in bytes
        explicit Place(const gmagnus_dense_t &m) {
            const int64_t size = data_size(m.data_type);
            at = (int64_t)(uintptr_t)m.data, rows = m.n_rows, width = m.n_cols * size, stride = m.row_stride * size;
            if (rows <= 1 || stride == width) width *= rows, stride = width, rows = rows > 0;
        }
        int64_t end() const { return at + (rows - 1) * stride + width; }
    };
    const Place p(a), q(b), &few = p.rows <= q.rows ? p : q, &many = p.rows <= q.rows ? q : p;
    if (p.rows == 0 || q.rows == 0 || p.end() <= q.at || q.end() <= p.at) return false;
    if (p.stride == q.stride) {  // row i can meet rows i + k and i + k - 1
        const int64_t w = p.stride, d = few.at - many.at, past = d + few.width - 1;
        const int64_t k = past >= 0 ? past / w : -((w - 1 - past) / w);
        for (int64_t j = k - 1; j <= k; ++j)
            if (j * w + many.width > d && (j < 0 ? -j : 0) < (few.rows < many.rows - j ? few.rows : many.rows - j)) return true;
        return false;
    }
    // (of the rows of `many` that begin before a row's end, the last one reaches furthest)
    for (int64_t i = 0; i < few.rows; ++i) {
        const int64_t from = few.at + i * few.stride, before = from + few.width - 1 - many.at;
        if (before < 0) continue;
        const int64_t j = before / many.stride < many.rows ? before / many.stride : many.rows - 1;
        if (many.at + j * many.stride + many.width > from) return true;
    }
    return false;
}

// An output may be an input itself; otherwise they have no memory in common.
void check_apart(const gmagnus_dense_t *out, const char *name, const gmagnus_dense_t *in, const char *other, bool may_be = true) {
    if (!out || !in || !out->data || !in->data) return;
    if (may_be && out->data == in->data && out->data_type == in->data_type && out->n_rows == in->n_rows && out->n_cols == in->n_cols &&
        (out->row_stride == in->row_stride || out->n_rows <= 1))
        return;
    GM_REQUIRE(!overlap(*out, *in), GMAGNUS_ERROR_INVALID_VALUE, std::string(name) + " overlaps " + other);
}

void check_eps(double eps) {
    GM_REQUIRE(eps >= 0 && eps <= 1e30, GMAGNUS_ERROR_INVALID_VALUE, "eps must be a number from 0 to 1e30");
}

// The results of n_stack matrices of t rows of n columns; fills their part of the kernel's arguments.
void check_results(RowArgs &a, const gmagnus_dense_t *Y, const gmagnus_dense_t *Q, const gmagnus_dense_t *scale, int64_t t,
                   int64_t n, int64_t n_stack, int32_t type) {
    GM_REQUIRE(Y || Q, GMAGNUS_ERROR_INVALID_VALUE, "neither a result in the rows' type nor one in 8 bits is wanted");
    GM_REQUIRE(!Q == !scale, GMAGNUS_ERROR_INVALID_VALUE, "an 8-bit result has its scale, and none has none");
    a.n_rows = n_stack * t;
    a.stack_rows = t;
    a.n = n;
    a.format = IN_TYPE;
    if (Y) {
        check_like(Y, "Y", t, n, type);
        a.y = Y->data;
        a.ys = Y->row_stride;
    }
    if (!Q) return;
    check_dense(Q, "Q", t, n, n_stack, GMAGNUS_DATA_INT8);
    GM_REQUIRE(Q->data_type == GMAGNUS_DATA_FP8_E4M3 || Q->data_type == GMAGNUS_DATA_INT8, GMAGNUS_ERROR_INVALID_VALUE,
               "Q must be E4M3 or int8");
    a.format = Q->data_type == GMAGNUS_DATA_INT8 ? INTEGER : E4M3;
    if (a.format == INTEGER) {
        check_dense(scale, "scale", n_stack, t);
        a.sg = scale->row_stride;
    } else {
        check_dense(scale, "scale", t, (n + SB - 1) / SB);
        a.ss = scale->row_stride;
    }
    GM_REQUIRE(scale->data_type == GMAGNUS_DATA_FP32, GMAGNUS_ERROR_INVALID_VALUE, "scale must be fp32");
    GM_REQUIRE(n_stack <= 1 || t == 0 || Q->stack_stride >= (t - 1) * Q->row_stride + n, GMAGNUS_ERROR_INVALID_VALUE,
               "matrices of Q overlap");
    a.q = (uint8_t *)Q->data;
    a.qs = Q->row_stride;
    a.qg = n_stack > 1 ? Q->stack_stride : 0;
    a.scale = (float *)scale->data;
}

}  // namespace
}  // namespace gm

using namespace gm;

extern "C" gmagnus_status_t gmagnus_rms_norm(const gmagnus_dense_t *X, const gmagnus_dense_t *residual,
                                             const gmagnus_dense_t *weight, double eps, const gmagnus_dense_t *total,
                                             const gmagnus_dense_t *Y, const gmagnus_dense_t *Q,
                                             const gmagnus_dense_t *scale, void *hip_stream) {
    return guarded([&] {
        GM_REQUIRE(X != nullptr, GMAGNUS_ERROR_INVALID_VALUE, "NULL X");
        const int64_t t = X->n_rows, n = X->n_cols;
        check_rows_n(t, n, "X");
        check_dense(X, "X", t, n);
        GM_REQUIRE(is_float(X->data_type), GMAGNUS_ERROR_INVALID_VALUE, "X must be fp32, bf16 or fp16");
        GM_REQUIRE(!residual == !total, GMAGNUS_ERROR_INVALID_VALUE, "a residual has its total, and none has none");
        if (residual) {
            check_like(residual, "residual", t, n, X->data_type);
            check_like(total, "total", t, n, X->data_type);
        }
        check_weight(weight, n, X->data_type);
        check_eps(eps);
        RowArgs a{};
        check_results(a, Y, Q, scale, t, n, 1, X->data_type);
        const gmagnus_dense_t *out[] = {total, Y, Q, scale};
        const char *names[] = {"total", "Y", "Q", "scale"};
        for (int i = 0; i < 4; ++i) {
            check_apart(out[i], names[i], X, "X");
            check_apart(out[i], names[i], residual, "residual");
            check_apart(out[i], names[i], weight, "weight", false);
            for (int j = 0; j < i; ++j) check_apart(out[i], names[i], out[j], names[j], false);
        }
        if (t == 0) return;
        a.x = X->data;
        a.xs = X->row_stride;
        if (residual) {
            a.r = residual->data;
            a.rs = residual->row_stride;
            a.total = total->data;
            a.in_place = total->data == X->data || total->data == residual->data;
            a.ts = total->row_stride;
        }
        a.w = weight ? weight->data : nullptr;
        a.w32 = weight && weight->data_type == GMAGNUS_DATA_FP32;
        a.eps = (float)eps;
        launch_rows<Op::NORM>(a, X->data_type, (hipStream_t)hip_stream);
    });
}

extern "C" gmagnus_status_t gmagnus_gate(const gmagnus_dense_t *H, const gmagnus_dense_t *Y, const gmagnus_dense_t *Q,
                                         const gmagnus_dense_t *scale, void *hip_stream) {
    return guarded([&] {
        GM_REQUIRE(H != nullptr, GMAGNUS_ERROR_INVALID_VALUE, "NULL H");
        const int64_t t = H->n_rows;
        check_rows_n(t, H->n_cols, "H");
        GM_REQUIRE(H->n_cols % 2 == 0, GMAGNUS_ERROR_INVALID_VALUE, "H must have an even number of columns");
        check_dense(H, "H", t, H->n_cols);
        GM_REQUIRE(is_float(H->data_type), GMAGNUS_ERROR_INVALID_VALUE, "H must be fp32, bf16 or fp16");
        RowArgs a{};
        check_results(a, Y, Q, scale, t, H->n_cols / 2, 1, H->data_type);
        if (t == 0) return;
        a.x = H->data;
        a.xs = H->row_stride;
        launch_rows<Op::GATE>(a, H->data_type, (hipStream_t)hip_stream);
    });
}

extern "C" gmagnus_status_t gmagnus_quantise_rows(const gmagnus_dense_t *X, int64_t n_stack, const gmagnus_dense_t *Q,
                                                  const gmagnus_dense_t *scale, void *hip_stream) {
    return guarded([&] {
        GM_REQUIRE(X && Q && scale, GMAGNUS_ERROR_INVALID_VALUE, "NULL X, Q or scale");
        const int64_t t = X->n_rows, n = X->n_cols;
        check_rows_n(t, n, "X");
        GM_REQUIRE(n_stack >= 0, GMAGNUS_ERROR_INVALID_VALUE, "negative stack");
        GM_REQUIRE(n_stack < INT32_MAX, GMAGNUS_ERROR_UNSUPPORTED, "stack beyond 2^31 - 2");
        check_dense(X, "X", t, n, n_stack);
        GM_REQUIRE(is_float(X->data_type), GMAGNUS_ERROR_INVALID_VALUE, "X must be fp32, bf16 or fp16");
        GM_REQUIRE(Q->data_type == GMAGNUS_DATA_INT8, GMAGNUS_ERROR_INVALID_VALUE, "Q must be int8");
        RowArgs a{};
        check_results(a, nullptr, Q, scale, t, n, n_stack, X->data_type);
        if (t == 0 || n_stack == 0) return;
        a.x = X->data;
        a.xs = X->row_stride;
        a.xg = n_stack > 1 ? X->stack_stride : 0;
        launch_rows<Op::COPY>(a, X->data_type, (hipStream_t)hip_stream);
    });
}

extern "C" int64_t gmagnus_rms_norm_backward_workspace_bytes(int64_t n_rows, int64_t n_cols) {
    return back_sizes_ok(n_rows, n_cols) ? BackLayout(n_rows, n_cols).bytes : 0;
}

extern "C" gmagnus_status_t gmagnus_rms_norm_backward(const gmagnus_dense_t *TOTAL, const gmagnus_dense_t *weight,
                                                      double eps, const gmagnus_dense_t *D_Y,
                                                      const gmagnus_dense_t *D_TOTAL, const gmagnus_dense_t *D_X,
                                                      float *d_weight, void *workspace, int64_t workspace_bytes,
                                                      void *hip_stream) {
    return guarded([&] {
        GM_REQUIRE(TOTAL != nullptr, GMAGNUS_ERROR_INVALID_VALUE, "NULL TOTAL");
        const int64_t t = TOTAL->n_rows, n = TOTAL->n_cols;
        check_rows_n(t, n, "TOTAL");
        check_dense(TOTAL, "TOTAL", t, n);
        GM_REQUIRE(is_float(TOTAL->data_type), GMAGNUS_ERROR_INVALID_VALUE, "TOTAL must be fp32, bf16 or fp16");
        check_like(D_Y, "D_Y", t, n, TOTAL->data_type);
        check_like(D_X, "D_X", t, n, TOTAL->data_type);
        if (D_TOTAL) check_like(D_TOTAL, "D_TOTAL", t, n, TOTAL->data_type);
        check_weight(weight, n, TOTAL->data_type);
        check_apart(D_X, "D_X", TOTAL, "TOTAL");
        check_apart(D_X, "D_X", D_Y, "D_Y");
        check_apart(D_X, "D_X", D_TOTAL, "D_TOTAL");
        check_eps(eps);
        GM_REQUIRE((uintptr_t)d_weight % 4 == 0, GMAGNUS_ERROR_INVALID_VALUE, "d_weight is not aligned to its type");
        hipStream_t s = (hipStream_t)hip_stream;
        if (t == 0) {
            if (d_weight) fill<float>(d_weight, 0.f, n, s);
            return;
        }
        const BackLayout l(t, n);
        GM_REQUIRE(workspace && workspace_bytes >= l.bytes, GMAGNUS_ERROR_INVALID_VALUE,
                   "workspace below gmagnus_rms_norm_backward_workspace_bytes");
        GM_REQUIRE((uintptr_t)workspace % 16 == 0, GMAGNUS_ERROR_INVALID_VALUE, "workspace is not 16-byte aligned");
        char *ws = static_cast<char *>(workspace);
        const int units = (int)back_units(t, n);
        const NormBackArgs a{TOTAL->data, weight ? weight->data : nullptr, D_Y->data, D_TOTAL ? D_TOTAL->data : nullptr,
                             D_X->data, d_weight ? (float *)(ws + l.share) : nullptr, (float *)(ws + l.of_row), t, n,
                             TOTAL->row_stride, D_Y->row_stride, D_TOTAL ? D_TOTAL->row_stride : 0, D_X->row_stride,
                             (float)eps, weight && weight->data_type == GMAGNUS_DATA_FP32};
        with_float(TOTAL->data_type, [&](auto v) {
            using T = decltype(v);
            with_row(n, [&](auto waves, auto pieces, auto whole) {
                constexpr int W = decltype(waves)::value, CH = decltype(pieces)::value;
            constexpr bool WHOLE = decltype(whole)::value;
                if constexpr (W == 0 || W == 16) {
                    hipLaunchKernelGGL((k_norm_backward_rows<T, WHOLE>), dim3(grid_for(t, 1, 1 << 16)), dim3(64 * LONG_W), 0, s, a);
                    hipLaunchKernelGGL((k_norm_backward_columns<T, WHOLE>), dim3(grid_for((n + 511) / 512 * units, 1, MAX_GRID)),
                                       dim3(64), 0, s, a, units);
                } else {
                    hipLaunchKernelGGL((k_norm_backward<T, W, CH, WHOLE>), dim3(units), dim3(W > 4 ? 64 * W : 256), 0, s, a);
                }
            });
        });
        if (d_weight)
            hipLaunchKernelGGL(k_add_shares, dim3(grid_for(n, 64, max_grid(1024))), dim3(1024), 0, s, a.share, n, units, d_weight);
        GM_CHECK_LAUNCH();
    });
}

extern "C" gmagnus_status_t gmagnus_gate_backward(const gmagnus_dense_t *H, const gmagnus_dense_t *D_A,
                                                  const gmagnus_dense_t *D_H, void *hip_stream) {
    return guarded([&] {
        GM_REQUIRE(H != nullptr, GMAGNUS_ERROR_INVALID_VALUE, "NULL H");
        const int64_t t = H->n_rows, n = H->n_cols / 2;
        check_rows_n(t, H->n_cols, "H");
        GM_REQUIRE(H->n_cols % 2 == 0, GMAGNUS_ERROR_INVALID_VALUE, "H must have an even number of columns");
        check_dense(H, "H", t, 2 * n);
        GM_REQUIRE(is_float(H->data_type), GMAGNUS_ERROR_INVALID_VALUE, "H must be fp32, bf16 or fp16");
        check_like(D_A, "D_A", t, n, H->data_type);
        check_like(D_H, "D_H", t, 2 * n, H->data_type);
        check_apart(D_H, "D_H", H, "H");
        check_apart(D_H, "D_H", D_A, "D_A");
        if (t == 0) return;
        const GateBackArgs a{H->data, D_A->data, D_H->data, t, n, H->row_stride, D_A->row_stride, D_H->row_stride};
        with_float(H->data_type, [&](auto v) {
            const dim3 grid(grid_for(t * ((n + 7) / 8), 256, MAX_GRID));
            if (n % 8 == 0)
                hipLaunchKernelGGL((k_gate_backward<decltype(v), true>), grid, dim3(256), 0, (hipStream_t)hip_stream, a);
            else
                hipLaunchKernelGGL((k_gate_backward<decltype(v), false>), grid, dim3(256), 0, (hipStream_t)hip_stream, a);
        });
        GM_CHECK_LAUNCH();
    });
}
