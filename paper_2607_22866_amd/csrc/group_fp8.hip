// Matrix products grouped by ragged runs of rows on 8-bit operands (E4M3) with
// a scale for each block of 128, and the rounding of matrices to that form.
//   Y[r,n] = sum over blocks b of sx[r,b] * sw[n/128,b] * (sum over k in b of x[r,k] * w[n,k])
// A step of the reduction is one block, so its sum leaves the matrix unit
// unscaled and is scaled as it joins the fp32 result. Within a block the unit
// adds 16 E4M3 products at a time, aligned to the largest and cut 13 bits below
// its leading one, and such groups in fp32 (measured; all of its 8-bit
// instructions do). Operands widened to 16 bits would not lose that, at half the
// rate; the operands' own rounding, 2^-4 each, is far above it.
#include "tile.hpp"

namespace gm {
namespace {

constexpr int SB = GMAGNUS_SCALE_BLOCK;
constexpr float FP8_MAX = 448.f;
constexpr float SCALE_MIN = 0x1p-126f;

// ----------------------------------------------------------------- quantise
struct QuantArgs {
    const void *x;
    uint8_t *q;
    float *scale;
    int64_t n_rows, n_cols, xs, xg, qs, qg, ss, sg, n_stack;
};

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

GM_DEV void store_fp8x8(uint8_t *p, int valid, const float (&v)[8], float scale) {
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = to_range(v[i], scale);
    const uint32_t w[2] = {pack_fp8(r[0], r[1], r[2], r[3]), pack_fp8(r[4], r[5], r[6], r[7])};
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

// One scale a row and 128 columns: 16 lanes a block, eight values a lane, a work
// group 16 blocks of one row or, of rows shorter than that, several rows. Bound by
// its bytes: 8192 x 8192 bf16 42-48 us, 4.2-4.8 TB/s; 16384 x 4096 45-47 us.
template <typename T>
__global__ __launch_bounds__(256) void k_quantise_rows(QuantArgs a) {
    const int blocks = (int)((a.n_cols + SB - 1) / SB), wide = blocks < 16 ? blocks : 16, per = 16 / wide;
    const int unit = threadIdx.x / 16, ur = unit / wide, ub = unit - ur * wide;
    const int64_t rows = a.n_stack * a.n_rows;
    for (int64_t row0 = (int64_t)blockIdx.x * per; row0 < rows; row0 += (int64_t)gridDim.x * per) {
        const int64_t row = row0 + ur;
        const bool mine = ur < per && row < rows;
        const int64_t g = a.n_stack == 1 || !mine ? 0 : row / a.n_rows, r = mine ? row - g * a.n_rows : 0;
        const T *x = static_cast<const T *>(a.x) + g * a.xg + r * a.xs;
        for (int b0 = 0; b0 < blocks; b0 += 2 * wide) {
            float v[2][8];
            int valid[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t c0 = (int64_t)(b0 + h * wide + ub) * SB + threadIdx.x % 16 * 8;
                valid[h] = !mine || c0 >= a.n_cols ? 0 : a.n_cols - c0 >= 8 ? 8 : (int)(a.n_cols - c0);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[h][i] = 0.f;
                if (valid[h] > 0) load_f32x8(x + c0, valid[h], v[h]);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int b = b0 + h * wide + ub;
                uint32_t m = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) m = max(m, magnitude(v[h][i]));
#pragma unroll
                for (int d = 1; d < 16; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d, 64));
                const float s = block_scale(m);
                if (valid[h] > 0) store_fp8x8(a.q + g * a.qg + r * a.qs + (int64_t)b * SB + threadIdx.x % 16 * 8, valid[h], v[h], s);
                if (mine && b < blocks && threadIdx.x % 16 == 0) a.scale[g * a.sg + r * a.ss + b] = s;
            }
        }
    }
}

// One scale for 128 x 128 values: a work group a block, kept in registers. Bound by
// its bytes in bf16 (8192 x 8192 42 us, 4.7 TB/s; 16 x 4096 x 4096 160 us, 5.0); in
// fp32, where a lane's 32 bytes are two loads, at half that (145 us, 2.3 TB/s; 523 us,
// 2.6).
template <typename T>
__global__ __launch_bounds__(256) void k_quantise_tiles(QuantArgs a) {
    __shared__ uint32_t part[4];
    const int64_t bc = (a.n_cols + SB - 1) / SB, br = (a.n_rows + SB - 1) / SB, total = a.n_stack * br * bc;
    for (int64_t u = blockIdx.x; u < total; u += gridDim.x) {
        const int64_t g = u / (br * bc), t = u - g * br * bc, tr = t / bc, tc = t - tr * bc;
        const int64_t c0 = tc * SB + threadIdx.x % 16 * 8;
        const int cols = c0 >= a.n_cols ? 0 : a.n_cols - c0 >= 8 ? 8 : (int)(a.n_cols - c0);
        float v[8][8];
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t r = tr * SB + i * 16 + threadIdx.x / 16;
            load_f32x8(static_cast<const T *>(a.x) + g * a.xg + (r < a.n_rows ? r : 0) * a.xs + (cols ? c0 : 0),
                       r < a.n_rows ? cols : 0, v[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) m = max(m, magnitude(v[i][j]));
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d, 64));
        if ((threadIdx.x & 63) == 0) part[threadIdx.x / 64] = m;
        __syncthreads();
        m = max(max(part[0], part[1]), max(part[2], part[3]));
        const float s = block_scale(m);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t r = tr * SB + i * 16 + threadIdx.x / 16;
            if (r < a.n_rows && cols > 0) store_fp8x8(a.q + g * a.qg + r * a.qs + c0, cols, v[i], s);
        }
        if (threadIdx.x == 0) a.scale[g * a.sg + tr * a.ss + tc] = s;
        __syncthreads();
    }
}

// ------------------------------------------------------------------ product
typedef int i32x8 __attribute__((ext_vector_type(8)));

// 16x16x128 on E4M3 operands (without the unit's own scales).
GM_DEV f32x4 mfma_fp8(u32x4 a0, u32x4 a1, u32x4 b0, u32x4 b1, f32x4 c) {
    const i32x8 a = {(int)a0[0], (int)a0[1], (int)a0[2], (int)a0[3], (int)a1[0], (int)a1[1], (int)a1[2], (int)a1[3]};
    const i32x8 b = {(int)b0[0], (int)b0[1], (int)b0[2], (int)b0[3], (int)b1[0], (int)b1[1], (int)b1[2], (int)b1[3]};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
}

struct Fp8Args {
    const int64_t *gp;
    const int32_t *index;
    int64_t n_groups, n_rows, n_x, n, k;
    const uint8_t *x, *w;
    const float *sx, *sw;
    void *y;
    int64_t xs, sxs, ws, wg, sws, swg, ys;
    int64_t max_row_tiles;
};

// Row of X that the tile's row r stands for, -1 if there is none.
GM_DEV int64_t x_row(const Fp8Args &a, const RowTile &t, int r) {
    if (r >= t.rows) return -1;
    const int64_t i = a.index ? a.index[t.begin + r] : t.begin + r;
    return i >= a.n_x ? -1 : i;
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

// Any alignment: tiles of 128 x 128 staged through registers, four waves of
// 64 x 64. LDS rows are one block of 128 bytes; chunk c of row r sits at
// c ^ (r / 2 % 8). A lane's 32 reduction bytes are chunks g and g + 4 of its row,
// the same for both operands (the order within a block does not matter). One
// buffer, one step's loads in flight: one group of 4001 x 4001 x 4001 177 us, 720
// TFLOP/s; 16 groups of 1024 rows, 2047 x 2047, 197 us, 700.
constexpr int GEN_B = 128, GEN_T = 256;

template <typename OUT>
__global__ __launch_bounds__(GEN_T, 2) void k_group_product_fp8_any(Fp8Args a) {
    __shared__ u32x4 lds[2 * GEN_B * 8];
    u32x4 *lp = lds, *lq = lds + GEN_B * 8;
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
        const float *sp[4];
        const float *sq = a.sw + t.group * a.swg + n0 / SB * a.sws;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (threadIdx.x + i * GEN_T) / 8;
            const int64_t xr = x_row(a, t, r), sr = x_row(a, t, p0 + 16 * i + i16);
            pr[i] = xr < 0 ? nullptr : a.x + xr * a.xs;
            qr[i] = r < cols ? a.w + t.group * a.wg + (n0 + r) * a.ws : nullptr;
            sp[i] = sr < 0 ? nullptr : a.sx + sr * a.sxs;
        }
        f32x4 acc[4][4] = {};
        u32x4 vp[4], vq[4];
        auto load = [&](int64_t k0) {
            const int64_t k = k0 + threadIdx.x % 8 * 16;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                vp[i] = pr[i] ? load16(pr[i] + k, a.k - k) : u32x4{0, 0, 0, 0};
                vq[i] = qr[i] ? load16(qr[i] + k, a.k - k) : u32x4{0, 0, 0, 0};
            }
        };
        load(0);
        for (int64_t k0 = 0; k0 < a.k; k0 += SB) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = (threadIdx.x + i * GEN_T) / 8, at = r * 8 + ((threadIdx.x % 8) ^ (r / 2 % 8));
                lp[at] = vp[i];
                lq[at] = vq[i];
            }
            __syncthreads();
            if (k0 + SB < a.k) load(k0 + SB);
            float s[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] = (sp[i] ? sp[i][k0 / SB] : 0.f) * sq[k0 / SB];
            u32x4 fp[4][2], fq[4][2];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int rp = p0 + 16 * i + i16, rq = q0 + 16 * i + i16;
                    fp[i][h] = lp[rp * 8 + ((h * 4 + g) ^ (rp / 2 % 8))];
                    fq[i][h] = lq[rq * 8 + ((h * 4 + g) ^ (rq / 2 % 8))];
                }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const f32x4 d = mfma_fp8(fq[j][0], fq[j][1], fp[i][0], fp[i][1], f32x4{0, 0, 0, 0});
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] += s[i] * d[e];
                }
        }
        __syncthreads();
        store_tile<OUT, GEN_B, GEN_B, 4, 4, GEN_T>(out, a.ys, t.rows, cols, p0, q0, reinterpret_cast<char *>(lds),
                                                   [&](int i, int j) { return acc[i][j]; });
    }
}

// Tiles brought straight from memory into LDS, as the 16-bit products have
// them (tile.hpp): a step is one block of 128 bytes a row. A wave takes its p
// rows 16 at a time against its 64 q columns. What the matrix units return for
// a block goes into the fp32 sums with the row's scale times the column
// block's, on the vector units while the other wave of the SIMD multiplies; the
// matrix units are busy half of the cycles (4096 x 4096 x 4096). One group of 8192 x
// 8192 x 8192: 2000-2300 TFLOP/s from card to card (of zeros, which draw less power,
// 2700); 16 groups of 1024 rows, 4096 x 4096, 1720-1920. The scales of X's rows come with their tile, 64 rows by each of the first waves.
template <int BP, int BQ>
constexpr int fast_lds() { return 2 * ((BP + BQ) * SB + ((BP + 63) / 64 * 64 + 64) * 4); }

template <typename OUT, int BP, int BQ, int WP, int WQ>
GM_DEV void tile_fp8_fast(const Fp8Args &a, const RowTile &t, int64_t n0, int cols, char *lds) {
    constexpr int THREADS = 64 * WP * WQ, MP = BP / WP, MQ = BQ / WQ, NP = MP / 16, NQ = MQ / 16;
    static_assert(NP % 2 == 0, "units alternate between two sets of fragments");
    constexpr int PB = BP * SB, QB = BQ * SB;
    char *lp = lds, *lq = lds + 2 * PB;
    float *ls = reinterpret_cast<float *>(lds + 2 * PB + 2 * QB);
    const int lane = threadIdx.x & 63, i16 = lane % 16, w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64));
    const int p0 = w / WQ * MP, q0 = w % WQ * MQ;
    Dma p{reinterpret_cast<const char *>(a.x), span(a.n_x, a.xs, a.k), a.xs, nullptr, a.n_x, t.rows};
    if (a.index) {
        p.index = a.index + t.begin;
    } else {
        p.base += t.begin * a.xs;
        p.records = span(t.rows, a.xs, a.k);
    }
    const Dma q{reinterpret_cast<const char *>(a.w) + t.group * a.wg + n0 * a.ws, span(cols, a.ws, a.k), a.ws,
                nullptr, 0, cols};
    // The step's scales come as single values: a row's to each thread of the first
    // RW waves, the column blocks' to the next waves (which repeat each other:
    // a branch around them would split the loop's body, and the compiler would move
    // the sums past it, out of the units).
    constexpr int RW = (BP + 63) / 64, SR = RW * 64 + 64;  // the rows' scales, then the column blocks'
    const int kb = (int)((a.k + SB - 1) / SB);
    const bool row_wave = w < RW;
    const float *s_base = row_wave ? a.sx : a.sw + t.group * a.swg + n0 / SB * a.sws;
    const int s_blocks = (cols + SB - 1) / SB;
    const uint32_t s_records = row_wave ? span(a.n_x, a.sxs * 4, kb * 4) : span(s_blocks, a.sws * 4, kb * 4);
    uint32_t sat = NOWHERE;
    if (row_wave && (int)threadIdx.x < t.rows) {
        const int64_t r = a.index ? a.index[t.begin + threadIdx.x] : t.begin + threadIdx.x;
        if (r >= 0 && r < a.n_x) sat = (uint32_t)(r * a.sxs * 4);
    } else if (!row_wave && lane < s_blocks) {
        sat = (uint32_t)(lane * a.sws * 4);
    }
    const int n_k = (int)(a.k / 2), steps = (n_k + BK - 1) / BK;  // (in pairs of bytes, as Feed counts)
    Feed<false, true, BP, THREADS> fp;
    Feed<false, false, BQ, THREADS> fq;
    fp.init(p);
    fq.init(q);
    const Reader<false, BP> rp(p0);
    const Reader<false, BQ> rq(q0);
    constexpr int LP = decltype(fp)::L, LQ = decltype(fq)::L;
    f32x4 acc[NP][NQ] = {};
    u32x4 a0[2], a1[2], b[NQ][2];
    float c0, c1;
    auto feed_p = [&](int s, int i) { fp.issue(p, lp + (s & 1) * PB, s * BK, n_k, i); };
    auto feed_q = [&](int s, int i) { fq.issue(q, lq + (s & 1) * QB, s * BK, n_k, i); };
    auto read_p = [&](int s, int u, u32x4(&f)[2], float &c) {
#pragma unroll
        for (int h = 0; h < 2; ++h) f[h] = rp.get(lp + (s & 1) * PB, h, u);
        c = ls[(s & 1) * SR + p0 + 16 * u + i16];
    };
    auto read_q = [&](int s, int j) {
#pragma unroll
        for (int h = 0; h < 2; ++h) b[j][h] = rq.get(lq + (s & 1) * QB, h, j);
    };
    auto feed_scales = [&](int s) {  // (past the last block: zeros, nothing is read)
        load_to_lds<4>(s_base, s_records, s < kb ? sat + (uint32_t)s * 4 : NOWHERE,
                       ls + (s & 1) * SR + (row_wave ? w : RW) * 64);
    };
    auto read_sq = [&](int s) { return ls[(s & 1) * SR + RW * 64 + q0 / SB]; };
    // a unit's products column by column, with a part of what else has to be issued after each
    auto unit = [&](int u, const u32x4(&f)[2], float sc, auto &&after) {
#pragma unroll
        for (int j = 0; j < NQ; ++j) {
            const f32x4 d = mfma_fp8(b[j][0], b[j][1], f[0], f[1], f32x4{0, 0, 0, 0});
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[u][j][e] += sc * d[e];
            after(j);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    wait_and_barrier();  // (the last tile's reads of LDS)
#pragma unroll
    for (int x = 0; x < LP; ++x) feed_p(0, x);
#pragma unroll
    for (int x = 0; x < LQ; ++x) feed_q(0, x);
    feed_scales(0);
    wait_and_barrier();
#pragma unroll
    for (int x = 0; x < LP; ++x) feed_p(1, x);
    feed_scales(1);
    read_p(0, 0, a0, c0);
#pragma unroll
    for (int j = 0; j < NQ; ++j) read_q(0, j);
    float sq = read_sq(0);
    // Steps past the last are fed as zeros and their fragments never used: one body for all steps.
    for (int s = 0; s < steps; ++s) {
        auto feed_at = [&](int u, int j) {  // the next tile's second operand, in the first unit
#pragma unroll
            for (int x = 0; x < LQ; ++x)
                if (u == 0 && x * NQ / LQ == j) feed_q(s + 1, x);
        };
#pragma unroll
        for (int u = 0; u + 2 < NP; u += 2) {
            read_p(s, u + 1, a1, c1);
            unit(u, a0, c0 * sq, [&](int j) { feed_at(u, j); });
            read_p(s, u + 2, a0, c0);
            unit(u + 1, a1, c1 * sq, [](int) {});
        }
        read_p(s, NP - 1, a1, c1);
        unit(NP - 2, a0, c0 * sq, [&](int j) { feed_at(NP - 2, j); });
        wait_and_barrier();
        feed_scales(s + 2);
        read_p(s + 1, 0, a0, c0);
        const float sn = read_sq(s + 1);
        unit(NP - 1, a1, c1 * sq, [&](int j) {
            read_q(s + 1, j);
#pragma unroll
            for (int x = 0; x < LP; ++x)
                if (x * NQ / LP == j) feed_p(s + 2, x);
        });
        sq = sn;
    }
    wait_and_barrier();  // (no load may be on its way to LDS when the work group ends)
    OUT *out = static_cast<OUT *>(a.y) + t.begin * a.ys + n0;
    store_tile<OUT, BP, BQ, NP, NQ, THREADS>(out, a.ys, t.rows, cols, p0, q0, lds, [&](int i, int j) { return acc[i][j]; });
}

template <typename OUT, int BP, int BQ, int WP, int WQ>
__global__ __launch_bounds__(64 * WP * WQ, 2) void k_group_product_fp8_fast(Fp8Args a) {
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
                tile_fp8_fast<OUT, BP / 2, BQ, WP, WQ>(a, t, n0, cols, lds_fast);
                continue;
            }
        tile_fp8_fast<OUT, BP, BQ, WP, WQ>(a, t, n0, cols, lds_fast);
    }
}

// Groups of a few rows: the weights' bytes are the bound, and go straight into the
// matrix unit's registers, any alignment (64 groups of 1 row, 2048 x 4096: 144 us,
// 4 rows 146; 3.7 TB/s of weights). A work group takes 16 rows of a group and 16 NT
// columns, its waves take turns at blocks of 128, FEW_U blocks' loads in flight
// each, and their sums are joined in LDS in the waves' order.
constexpr int FEW_U = 4;

template <typename OUT, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_group_product_fp8_few(Fp8Args a) {
    constexpr int BP = 16, BQ = 16 * NT, THREADS = 64 * WAVES;
    __shared__ float part[WAVES][BP][BQ + 4];
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
        // (a row that is not there reads another: its results are not stored)
        const int64_t xi = x_row(a, t, i16);
        const uint8_t *xr = xi < 0 ? wr[0] : a.x + xi * a.xs;
        const float *sq = a.sw + t.group * a.swg + q0 / SB * a.sws, *sp = xi < 0 ? sq : a.sx + xi * a.sxs;
        f32x4 acc[NT] = {};
        auto block = [&](const u32x4(&fx)[2], const u32x4(&fw)[NT][2], float s) {
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const f32x4 d = mfma_fp8(fw[j][0], fw[j][1], fx[0], fx[1], f32x4{0, 0, 0, 0});
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[j][e] += s * d[e];
            }
        };
        for (int k0 = w; k0 < full; k0 += WAVES * FEW_U) {
            u32x4 fx[FEW_U][2], fw[FEW_U][NT][2];
            float s[FEW_U];
#pragma unroll
            for (int u = 0; u < FEW_U; ++u) {
                const int kb = min(k0 + u * WAVES, full - 1);
                s[u] = sp[kb] * sq[kb];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int j = 0; j < NT; ++j) fw[u][j][h] = load16(wr[j] + kb * SB + h * 64 + g * 16, 16);
                    fx[u][h] = load16(xr + kb * SB + h * 64 + g * 16, 16);
                }
            }
#pragma unroll
            for (int u = 0; u < FEW_U; ++u)
                if (k0 + u * WAVES < full) block(fx[u], fw[u], s[u]);
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
            block(fx, fw, sp[full] * sq[full]);
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

// The kernel of a product, as for 16 bits (group.hip).
enum class Shape { FEW16, FEW64, ANY, T32, T64, T256 };

Shape fp8_shape(const Fp8Args &a) {
    const int64_t mean = (a.n_rows + a.n_groups - 1) / a.n_groups, groups = a.n_groups < a.n_rows ? a.n_groups : a.n_rows;
    const int64_t kb = (a.k + SB - 1) / SB;
    const bool fast = fast_side(a.x, a.xs, 0, a.k, a.index ? a.n_x : 256, 1) &&
                      fast_side(a.w, a.ws, a.n_groups > 1 ? a.wg : 0, a.k, 256, 1) &&
                      (a.n_x * a.sxs + kb) * 4 < (int64_t)NOWHERE && (2 * a.sws + kb) * 4 < (int64_t)NOWHERE;
    // 64 groups, 2048 x 4096, sizes as chance deals them: of 1, 4, 8 and 16 rows 64
    // columns a work group 103, 141, 156 and 181 us, tiles of 32 x 128 88, 173, 176 and
    // 177 (all rows in one of the groups, mean 8: 60 / 26); one row, 4096 x 4096: 11.7
    // with 16 columns, 13.8 with 64; 4 groups of 1 row, 2047 x 2047 (not aligned): 19.4,
    // staged tiles 27.4
    if (mean <= 8) {
        if (groups * ((a.n + 63) / 64) < 256) return Shape::FEW16;
        if (fast) return Shape::FEW64;
    }
    if (!fast) return Shape::ANY;
    // of 24 rows tiles of 32 rows 172, of 64 178; of 32 rows 137 / 176, of 96 206 / 162 (and of 48 still 148 / 173)
    if (mean <= 32) return Shape::T32;
    // of 96 rows 256 x 256 tiles 142 against 162, of 128 151 / 200, of 512 370 / 510
    return big_product_tiles(mean, a.n, groups) ? Shape::T256 : Shape::T64;
}

}  // namespace
}  // namespace gm

using namespace gm;

extern "C" gmagnus_status_t gmagnus_quantise_blocks(const gmagnus_dense_t *X, int64_t n_stack, int64_t block_rows,
                                                    const gmagnus_dense_t *Q, const gmagnus_dense_t *scale,
                                                    void *hip_stream) {
    return guarded([&] {
        GM_REQUIRE(X && Q && scale, GMAGNUS_ERROR_INVALID_VALUE, "NULL X, Q or scale");
        GM_REQUIRE(block_rows == 1 || block_rows == SB, GMAGNUS_ERROR_INVALID_VALUE, "block_rows must be 1 or 128");
        const int64_t n = X->n_rows, k = X->n_cols;
        GM_REQUIRE(n >= 0 && n_stack >= 0, GMAGNUS_ERROR_INVALID_VALUE, "negative rows or stack");
        check_side(k, "columns of X");
        GM_REQUIRE(n < INT32_MAX && n_stack < INT32_MAX, GMAGNUS_ERROR_UNSUPPORTED, "rows or stack beyond 2^31 - 2");
        check_dense(X, "X", n, k, n_stack);
        check_dense(Q, "Q", n, k, n_stack);
        check_dense(scale, "scale", (n + block_rows - 1) / block_rows, (k + SB - 1) / SB, n_stack);
        GM_REQUIRE(X->data_type != GMAGNUS_DATA_FP8_E4M3 && Q->data_type == GMAGNUS_DATA_FP8_E4M3 &&
                       scale->data_type == GMAGNUS_DATA_FP32,
                   GMAGNUS_ERROR_INVALID_VALUE, "X must be fp32, bf16 or fp16, Q E4M3, scale fp32");
        if (n == 0 || n_stack == 0) return;
        for (const gmagnus_dense_t *m : {Q, scale})
            GM_REQUIRE(n_stack == 1 || m->stack_stride >= (m->n_rows - 1) * m->row_stride + m->n_cols,
                       GMAGNUS_ERROR_INVALID_VALUE, "matrices of Q or of scale overlap");
        const QuantArgs a{X->data, (uint8_t *)Q->data, (float *)scale->data, n, k, X->row_stride, X->stack_stride,
                          Q->row_stride, Q->stack_stride, scale->row_stride, scale->stack_stride, n_stack};
        hipStream_t s = (hipStream_t)hip_stream;
        auto launch = [&](auto v) {
            using T = decltype(v);
            if (block_rows == 1) {
                const int per = scale->n_cols < 16 ? (int)(16 / scale->n_cols) : 1;
                hipLaunchKernelGGL(k_quantise_rows<T>, dim3(grid_for(n_stack * n, per, MAX_GRID)), dim3(256), 0, s, a);
            } else {
                hipLaunchKernelGGL(k_quantise_tiles<T>, dim3(grid_for(n_stack * scale->n_rows * scale->n_cols, 1, MAX_GRID)),
                                   dim3(256), 0, s, a);
            }
        };
        if (X->data_type == GMAGNUS_DATA_BF16)
            launch(__bf16{});
        else if (X->data_type == GMAGNUS_DATA_FP16)
            launch(_Float16{});
        else
            launch(float{});
        GM_CHECK_LAUNCH();
    });
}

extern "C" gmagnus_status_t gmagnus_group_product_fp8(const gmagnus_groups_t *groups, const gmagnus_dense_t *X,
                                                      const gmagnus_dense_t *X_scale, const gmagnus_dense_t *W,
                                                      const gmagnus_dense_t *W_scale, const gmagnus_dense_t *Y,
                                                      void *hip_stream) {
    return guarded([&] {
        check_groups(groups);
        GM_REQUIRE(X && W && Y && X_scale && W_scale, GMAGNUS_ERROR_INVALID_VALUE, "NULL X, W, Y or scale");
        const int64_t k = X->n_cols, n = Y->n_cols;
        check_side(k, "columns of X");
        check_side(n, "columns of Y");
        const int64_t n_x = x_rows(*groups, *X), kb = (k + SB - 1) / SB;
        check_dense(X, "X", n_x, k);
        check_dense(X_scale, "X_scale", n_x, kb);
        check_dense(Y, "Y", groups->n_rows, n);
        check_dense(W, "W", n, k, groups->n_groups);
        check_dense(W_scale, "W_scale", (n + SB - 1) / SB, kb, groups->n_groups);
        GM_REQUIRE(n_x >= 0 && n_x < INT32_MAX, GMAGNUS_ERROR_UNSUPPORTED, "rows of X beyond 2^31 - 2");
        GM_REQUIRE(X->data_type == GMAGNUS_DATA_FP8_E4M3 && W->data_type == GMAGNUS_DATA_FP8_E4M3 &&
                       X_scale->data_type == GMAGNUS_DATA_FP32 && W_scale->data_type == GMAGNUS_DATA_FP32 &&
                       Y->data_type != GMAGNUS_DATA_FP8_E4M3,
                   GMAGNUS_ERROR_INVALID_VALUE, "X and W must be E4M3, their scales fp32, Y fp32, bf16 or fp16");
        if (groups->n_rows == 0) return;
        const Fp8Args a{groups->group_ptr, groups->index, groups->n_groups, groups->n_rows, n_x, n, k,
                        (const uint8_t *)X->data, (const uint8_t *)W->data, (const float *)X_scale->data,
                        (const float *)W_scale->data, Y->data, X->row_stride, X_scale->row_stride, W->row_stride,
                        W->stack_stride, W_scale->row_stride, W_scale->stack_stride, Y->row_stride, 0};
        hipStream_t s = (hipStream_t)hip_stream;
        auto launch = [&](auto o) {
            using O = decltype(o);
            auto go = [&](auto kernel, int bp, int bq, int threads, int lds) {
                Fp8Args f = a;
                f.max_row_tiles = row_tiles_bound(a.n_groups, a.n_rows, bp);
                launch_fast(kernel, f.max_row_tiles * ((n + bq - 1) / bq), threads, lds, f, s);
            };
            switch (fp8_shape(a)) {
            case Shape::FEW16: return go(k_group_product_fp8_few<O, 1, 4>, 16, 16, 256, 0);
            case Shape::FEW64: return go(k_group_product_fp8_few<O, 4, 4>, 16, 64, 256, 0);
            case Shape::ANY: return go(k_group_product_fp8_any<O>, GEN_B, GEN_B, GEN_T, 0);
            case Shape::T32: return go(k_group_product_fp8_fast<O, 32, 128, 1, 4>, 32, 128, 256, fast_lds<32, 128>());
            case Shape::T64: return go(k_group_product_fp8_fast<O, 64, 128, 2, 2>, 64, 128, 256, fast_lds<64, 128>());
            case Shape::T256: return go(k_group_product_fp8_fast<O, 256, 256, 2, 4>, 256, 256, 512, fast_lds<256, 256>());
            }
        };
        if (Y->data_type == GMAGNUS_DATA_BF16)
            launch(__bf16{});
        else if (Y->data_type == GMAGNUS_DATA_FP16)
            launch(_Float16{});
        else
            launch(float{});
        GM_CHECK_LAUNCH();
    });
}
