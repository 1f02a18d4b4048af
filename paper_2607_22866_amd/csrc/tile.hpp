// Operand tiles of a matrix product in LDS: their layout, how they get there
// straight from memory, and how a wave reads its fragments.
#pragma once

#include <type_traits>

#include "dense.hpp"

namespace gm {

constexpr int BK = 64;  // reduction elements of 16 bits a step (8 bits: twice as many)

// LDS layout of an operand tile, in 16-byte chunks (8 elements).
// k contiguous: 128-byte rows; chunk c of row r sits at c ^ swz(r).
// k as rows: rows of B elements; 32-byte unit u of row k sits at u ^ swz(k).
// Either swizzle spreads the chunks that a wave reads at once over the banks.
template <bool KROWS>
GM_DEV int swz(int r) {
    return KROWS ? (r & 3) | ((r >> 3) & 1) << 2 : (r >> 1) & 7;
}

// ---------------------------------------------------------------- fast layout
// Tiles brought straight from memory into LDS, 16 bytes a lane, for operands
// whose rows are 16-byte aligned and whose contiguous axis is a multiple of 8.
// LDS positions follow the lane order, so the swizzle is applied to what a lane
// fetches. Two buffers: while the matrix units work on one step's tile the next
// one is on its way.
struct Dma {
    const char *base;   // of the tile
    uint32_t records;   // bytes that may be read from base (k as rows without an index: of one row)
    int64_t stride;     // bytes between rows
    const int32_t *index;
    int64_t n_mem;
    int valid;
};

constexpr uint32_t NOWHERE = 0x80000000u;  // beyond any operand's bytes: reads as zeros

// Bytes from the first of `rows` rows to the last one's end.
GM_DEV uint32_t span(int64_t rows, int64_t stride, int64_t row) { return rows > 0 ? (uint32_t)((rows - 1) * stride + row) : 0u; }

// Lane l's BYTES (16 or 4) at base + v go to LDS at `to` + BYTES l; zeros where v is not
// below `records`, and nothing is read there. The instruction's scalar offset is
// always 0: it does not take part in that check as v does. An instruction without
// results: the compiler, which would wait for it before every transposing read
// of LDS, counts no load, and wait_and_barrier() is what waits. (M0 is set and
// used inside; the compiler, which reserves it, does the same for each of its
// own uses.)
template <int BYTES = 16>
GM_DEV void load_to_lds(const void *base, uint32_t records, uint32_t v, void *to) {
    typedef __attribute__((address_space(3))) char lds_char;
    const uint64_t b = (uint64_t)base;
    const u32x4 rsrc = {(uint32_t)b, (uint32_t)(b >> 32) & 0xffffu, records, 0x00027000u};
    const uint32_t m0 = (uint32_t)(uintptr_t)(lds_char *)to;
    if constexpr (BYTES == 16)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     :
                     : "s"(m0), "v"(v), "s"(rsrc)
                     : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                     :
                     : "s"(m0), "v"(v), "s"(rsrc)
                     : "memory");
}

// IDX: k as rows, their numbers by an index (k contiguous: the index is read once, at init).
template <bool KROWS, bool IDX, int B, int THREADS>
struct Feed {
    static_assert(!KROWS || B >= 128, "a row holds the 8 units that the swizzle permutes");
    static constexpr int W = THREADS / 64, L = B * BK * 2 / 1024 / W;  // loads of a wave a step
    static constexpr int PITCH = KROWS ? B * 2 : BK * 2;               // bytes of an LDS row
    static constexpr int SLOTS = PITCH / 16, ROWS = 1024 / PITCH;      // of one load
    uint32_t at[L];
    int32_t ids[KROWS && IDX ? L : 1];

    GM_DEV static int wave() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64)); }
    GM_DEV static int row_of(int i) { return (wave() * L + i) * ROWS + (threadIdx.x & 63) / SLOTS; }
    // first element on the contiguous axis that this lane fetches in load i
    GM_DEV static int elem_of(int i) {
        const int r = row_of(i), s = (threadIdx.x & 63) % SLOTS;
        if constexpr (KROWS) return (((s >> 1) ^ swz<true>(r)) << 1 | (s & 1)) * 8;
        return (s ^ swz<false>(r)) * 8;
    }
    GM_DEV void init(const Dma &d) {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int r = row_of(i), x = elem_of(i);
            if constexpr (KROWS) {
                at[i] = x < d.valid ? (IDX ? 0u : (uint32_t)(r * d.stride)) + x * 2 : NOWHERE;
            } else {
                int64_t m = r;
                bool ok = r < d.valid;
                if (IDX && d.index && ok) {
                    m = d.index[r];
                    ok = m >= 0 && m < d.n_mem;
                }
                at[i] = ok ? (uint32_t)(m * d.stride) + x * 2 : NOWHERE;
            }
        }
    }
    // the rows' numbers of step k0
    GM_DEV void fetch_ids(const Dma &d, int k0, int n_k) {
        if constexpr (KROWS && IDX) {
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const int k = k0 + row_of(i);
                ids[i] = k < n_k ? d.index[k] : -1;
            }
        }
    }
    // load i of step k0 (past n_k: zeros)
    GM_DEV void issue(const Dma &d, char *lds, int k0, int n_k, int i) {
        const char *base = d.base;
        uint32_t records = d.records, v = at[i];
        if constexpr (KROWS && IDX) {
            const bool ok = ids[i] >= 0 && ids[i] < (int)d.n_mem && v != NOWHERE;
            v = ok ? v + (uint32_t)ids[i] * (uint32_t)d.stride : NOWHERE;
        } else if constexpr (KROWS) {
            // the rows below n_k: what lies past them reads as zeros
            const int rows = n_k - k0 < BK ? n_k - k0 : BK;
            base += k0 * d.stride;
            records = rows > 0 ? (uint32_t)((rows - 1) * d.stride) + d.records : 0u;
        } else {
            v = elem_of(i) < n_k - k0 ? v + (uint32_t)k0 * 2 : NOWHERE;
        }
        load_to_lds(base, records, v, lds + (wave() * L + i) * 1024);
    }
};

// Every wave's loads into LDS have landed and its reads are done, for all waves.
// (Loads into LDS count as memory operations that a barrier alone does not wait
// for.)
GM_DEV void wait_and_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// What a wave reads of an operand's tile: its fragments from row (column) x0 on.
template <bool KROWS, int B>
struct Reader {
    typedef __attribute__((address_space(3))) const char lds_char;
    uint32_t at[KROWS ? 1 : 2];  // byte offset in a tile, for each half of the step (k contiguous)
    GM_DEV Reader(int x0) {
        const int lane = threadIdx.x & 63, i = lane % 16, g = lane / 16;
        if constexpr (KROWS) {
            // row 8g + i/4 of the step's half; unit x0/16 + t (t below 8) sits at (x0/16 + t) ^ swz
            const int k = g * 8 + i / 4;
            at[0] = k * (B * 2) + ((x0 / 16) ^ swz<true>(k)) * 32 + (i % 4) * 8;
        } else {
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) at[kk] = (x0 + i) * 128 + ((kk * 4 + g) ^ swz<false>(i)) * 16;
        }
    }
    // fragment t (16 rows) of half kk of the tile at `tile`
    GM_DEV u32x4 get(const char *tile, int kk, int t) const {
        lds_char *p = (lds_char *)tile;
        if constexpr (KROWS) {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            p += (at[0] ^ (uint32_t)(t * 32)) + kk * 32 * (B * 2);
            const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p));
            const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + 4 * (B * 2))));
            return u32x4{lo[0], lo[1], hi[0], hi[1]};
        } else {
            typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
            return *(lds_u32x4 *)(p + at[kk] + t * 16 * 128);
        }
    }
};

// Eight 16-bit neighbours of an output row, from `first` on as many as there are, at any alignment.
template <typename OUT>
GM_DEV void store8(OUT *p, u32x4 v, int left, int first) {
    if (left >= 8 && first <= 0) {
        *reinterpret_cast<Bytes16<2> *>(p) = Bytes16<2>{{v[0], v[1], v[2], v[3]}};
    } else {
        uint16_t *q = reinterpret_cast<uint16_t *>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i >= first && i < left) q[i] = (uint16_t)(v[i >> 1] >> (16 * (i & 1)));
    }
}

// Writes a work group's BP x BQ results, of which rows x cols are there and the
// first skip_p rows and skip_q columns another tile's. A lane
// holds four neighbours of a row (acc(i, j): row p0 + 16 i + lane % 16, columns from
// q0 + 16 j + 4 (lane / 16) on): 16-bit results go through LDS, so that whole lines
// leave the CU instead of quarters of them (gradient of 2048 x 2048 weights, 64
// groups of 64 rows: 226 -> 160 us). No wave may be reading LDS any more.
template <typename OUT, int BP, int BQ, int NP, int NQ, int THREADS, class ACC>
GM_DEV void store_tile(OUT *out, int64_t stride, int rows, int cols, int p0, int q0, char *lds, ACC &&acc, int skip_p = 0,
                       int skip_q = 0) {
    const int lane = threadIdx.x & 63;
    if constexpr (sizeof(OUT) == 2) {
        // 8-byte unit u of row r sits at u ^ 2 (r % 8)
        u32x2 *put = reinterpret_cast<u32x2 *>(lds);
        const u32x4 *get = reinterpret_cast<const u32x4 *>(lds);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int r = p0 + 16 * i + lane % 16;
#pragma unroll
            for (int j = 0; j < NQ; ++j) {
                const f32x4 v = acc(i, j);
                put[r * (BQ / 4) + (((q0 + 16 * j) / 4 + lane / 16) ^ (r % 8) * 2)] =
                    u32x2{pack2<OUT>(v[0], v[1]), pack2<OUT>(v[2], v[3])};
            }
        }
        wait_and_barrier();
#pragma unroll 4
        for (int x = threadIdx.x; x < BP * (BQ / 8); x += THREADS) {
            const int r = x / (BQ / 8), c = x % (BQ / 8);
            if (r >= skip_p && r < rows)
                store8(out + r * stride + c * 8, get[r * (BQ / 8) + (c ^ (r % 8))], cols - c * 8, skip_q - c * 8);
        }
    } else {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int r = p0 + 16 * i + lane % 16;
            if (r >= skip_p && r < rows) {
#pragma unroll
                for (int j = 0; j < NQ; ++j) {
                    const int c = q0 + 16 * j + lane / 16 * 4;
                    store4(out + r * stride + c, acc(i, j), cols - c, skip_q - c);
                }
            }
        }
    }
}

// Products of 16-bit fragments.
template <typename T>
struct Mul16 {
    typedef f32x4 sums;
    GM_DEV static f32x4 mul(u32x4 a, u32x4 b, f32x4 c) { return mfma_16x16x32(a, b, c, T{}); }
};
struct AsTheyAre {
    GM_DEV AsTheyAre operator()() const { return {}; }
    GM_DEV f32x4 operator()(int, int, f32x4 v) const { return v; }
};

// A tile by WP x WQ waves; bound by the matrix units' power and, in small groups,
// by the weights' bytes. One group of 8192 x 8192 x 8192, bf16: 1265-1440 TFLOP/s from
// card to card (weights n x k), 1357-1460 (k x n), gradient 1345-1465, on operands of
// zeros, which draw less power, 1655, 1700 and 1810; 32 groups of 1024 rows, 2048 x
// 4096, 1090-1130 (with one matrix of weights for all 1360), gradient 845-965. 256 x 256 tiles move the fewest bytes a product
// that registers hold sums for (128 a lane). A wave's share of a step is four units of (32
// reduction elements, half of its p rows); a unit's fragments are read from LDS
// while the one before is multiplied. The barrier stands before a step's last
// unit, whose fragments are in registers by then, so that the buffer can be
// filled again and the next step's first fragments read behind it. The loads
// into LDS are spread over two units: issued together they hold every wave up
// at the memory pipeline while the matrix units idle.
//
// MUL: what two fragments of 16 bytes a lane are multiplied as (a step is 128 bytes
// of a row, n_k and BK count pairs of them). finish(): called when the sums are whole, gives
// what makes a lane's four results of (i, j, its sums).
template <class MUL, typename OUT, bool PK, bool QK, bool PI, bool QI, int BP, int BQ, int WP, int WQ, class F>
GM_DEV void tile_fast(const Dma &p, const Dma &q, int n_k, OUT *out, int64_t out_stride, char *lds, F &&finish) {
    typedef typename MUL::sums sums;
    constexpr int THREADS = 64 * WP * WQ, MP = BP / WP, MQ = BQ / WQ, NP = MP / 32, NQ = MQ / 16;
    constexpr int PB = BP * BK * 2, QB = BQ * BK * 2;
    char *lp = lds, *lq = lds + 2 * PB;
    const int w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64));
    const int p0 = w / WQ * MP, q0 = w % WQ * MQ;
    Feed<PK, PI, BP, THREADS> fp;
    Feed<QK, QI, BQ, THREADS> fq;
    fp.init(p);
    fq.init(q);
    const Reader<PK, BP> rp(p0);
    const Reader<QK, BQ> rq(q0);
    sums acc[2][NP][NQ] = {};
    u32x4 a0[NP], a1[NP], b0[NQ], b1[NQ];
    const int steps = (n_k + BK - 1) / BK;
    auto feed_p = [&](int s, int i) { fp.issue(p, lp + (s & 1) * PB, s * BK, n_k, i); };
    auto feed_q = [&](int s, int i) { fq.issue(q, lq + (s & 1) * QB, s * BK, n_k, i); };
    auto read_p = [&](int s, int kk, int half, int i) { return rp.get(lp + (s & 1) * PB, kk, half * NP + i); };
    auto read_q = [&](int s, int kk, int j) { return rq.get(lq + (s & 1) * QB, kk, j); };
    constexpr int LP = decltype(fp)::L, LQ = decltype(fq)::L;
    // a unit's products, row by row, with a part of what else has to be issued before each
    auto unit = [&](int half, const u32x4(&a)[NP], const u32x4(&b)[NQ], auto &&before) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            before(i);
#pragma unroll
            for (int j = 0; j < NQ; ++j) acc[half][i][j] = MUL::mul(b[j], a[i], acc[half][i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // f(x) for the i-th of NP parts of 0 .. n
    auto part = [&](int n, int i, auto &&f) {
#pragma unroll
        for (int x = 0; x < 16; ++x)
            if (x < n && x * NP / n == i) f(x);
    };
    wait_and_barrier();  // (the last tile's reads of LDS)
    fp.fetch_ids(p, 0, n_k);
    fq.fetch_ids(q, 0, n_k);
#pragma unroll
    for (int x = 0; x < LP; ++x) feed_p(0, x);
#pragma unroll
    for (int x = 0; x < LQ; ++x) feed_q(0, x);
    fp.fetch_ids(p, BK, n_k);
    fq.fetch_ids(q, BK, n_k);
    wait_and_barrier();
#pragma unroll
    for (int x = 0; x < LP; ++x) feed_p(1, x);
    fp.fetch_ids(p, 2 * BK, n_k);
#pragma unroll
    for (int j = 0; j < NQ; ++j) b0[j] = read_q(0, 0, j);
#pragma unroll
    for (int i = 0; i < NP; ++i) a0[i] = read_p(0, 0, 0, i);
    // Steps past the last are fed as zeros and their fragments never used: one body for all steps.
    for (int s = 0; s < steps; ++s) {
        unit(0, a0, b0, [&](int i) {
            a1[i] = read_p(s, 0, 1, i);
            part(LQ, i, [&](int x) { feed_q(s + 1, x); });
        });
        fq.fetch_ids(q, (s + 2) * BK, n_k);
        unit(1, a1, b0, [&](int i) {
            a0[i] = read_p(s, 1, 0, i);
            part(NQ, i, [&](int x) { b1[x] = read_q(s, 1, x); });
        });
        unit(0, a0, b1, [&](int i) { a1[i] = read_p(s, 1, 1, i); });
        wait_and_barrier();
        unit(1, a1, b1, [&](int i) {
            a0[i] = read_p(s + 1, 0, 0, i);
            part(NQ, i, [&](int x) { b0[x] = read_q(s + 1, 0, x); });
            part(LP, i, [&](int x) { feed_p(s + 2, x); });
        });
        fp.fetch_ids(p, (s + 3) * BK, n_k);
    }
    wait_and_barrier();  // (no load may be on its way to LDS when the work group ends)
    const auto result = finish();
    store_tile<OUT, BP, BQ, 2 * NP, NQ, THREADS>(out, out_stride, p.valid, q.valid, p0, q0, lds,
                                                 [&](int i, int j) { return result(i, j, acc[i / NP][i % NP][j]); });
}

// Whether an operand's rows can be brought in by 16-byte pieces, with 32-bit
// offsets over `rows` rows.
inline bool fast_side(const void *p, int64_t stride, int64_t stack, int64_t axis, int64_t rows, int size = 2) {
    return aligned16(p, stride, stack, size) && axis * size % 16 == 0 && (rows * stride + axis) * size < (int64_t)NOWHERE;
}

// Whether a product of `groups` groups of `mean` rows and n columns takes 256 x
// 256 tiles (one work group a CU, the fewest bytes a product) rather than 64 x 128
// (three a CU). 64 groups, 2048 x 2048, bf16, sizes as chance deals them: of 128
// rows on the average 150 against 177 us, 192 rows 153 / 207, 512 rows 332 / 415, and
// already of 96 rows 142 / 152 (of 64 rows, equal groups, 139 against 133 with 32 x
// 128); all rows in one of the groups: mean 128 55 / 79, 256 104 / 156. Where they
// leave CUs without one: 8 groups of 512 rows, 1024 x 1024 (64 tiles), 24.5 / 17.7, of
// 1024 rows (128 tiles) 26.5 / 30.2; and not where the columns' padding grows by more
// than a third.
inline bool big_product_tiles(int64_t mean, int64_t n, int64_t groups) {
    const int64_t cols = (n + 255) / 256;
    return mean >= 128 && (mean + 255) / 256 * cols * groups >= 128 && 3 * 2 * cols <= 4 * ((n + 127) / 128);
}

// LDS of two buffers of tiles of bp and bq rows.
constexpr int fast_bytes(int bp, int bq) { return 2 * (bp + bq) * BK * 2; }

template <typename K, typename A>
void launch_fast(K kernel, int64_t tiles, int threads, int lds, const A &a, hipStream_t s) {
    GM_REQUIRE(tiles < INT32_MAX, GMAGNUS_ERROR_UNSUPPORTED, "2^31 tiles or more");
    if (lds > 0) allow_dynamic_lds(reinterpret_cast<const void *>(kernel), lds);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(tiles < MAX_GRID ? tiles : MAX_GRID)), dim3(threads), lds, s, a);
}

}  // namespace gm
