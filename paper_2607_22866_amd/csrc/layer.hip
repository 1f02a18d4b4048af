// A whole layer of gated experts for a few tokens, from the router's logits to the tokens' sums:
//   out[t] = sum over the experts e of t of R[t,e] * W2_e (silu(G_e x_t) . (U_e x_t)),   W1_e = [G_e; U_e]
// R as route gives it. The weights of the experts that are reached are read once and
// are all there is to it, so they go straight from memory into the matrix units'
// registers, and all else is kept small: two kernels, the products of W1 with the gate,
// then those of W2 with the sums. Every work group of the first finds the routing by
// itself (a few logits) and holds it in LDS; the first one leaves it to the second
// kernel. (Above 16 tokens that costs more than a kernel of its own for it.) Rows are
// grouped by expert, tokens ascending, as the grouped products have them.
#include "quant.hpp"
#include "route.hpp"

namespace gm {
namespace {

constexpr int MAX_TOKENS = 64;   // one bit each in an expert's mask
constexpr int MAX_ENTRIES = 1024;

struct LayerArgs {
    const void *x, *logits;
    const uint8_t *w1, *w2;
    const float *s1, *s2;  // of 8-bit weights
    void *out;
    int64_t xs, ls, w1s, w1g, s1s, s1g, w2s, w2g, s2s, s2g, os;  // (weights': in bytes)
    int n_tokens, n_experts, top_k, normalise, logit_type;
    int d, f, n;  // columns of x, of the gate's result, of out
    int splits;
    // workspace
    int32_t *arrived;  // of each column tile of the second kernel, how many of its splits are there
    int32_t *table;
    void *act;         // [2][entries][act_stride]: results and what is left of them, act_part elements between the two
    float *share;      // [column tiles][splits][n_tokens][32]
    int64_t act_stride, act_part;
};

// The routing: the experts that tokens have chosen, ascending, with their first rows, and the rows' tokens and weights.
struct Table {
    int32_t *n, *expert, *first, *token;
    float *weight;
    GM_DEV Table(int32_t *p, int entries) {
        n = p;
        expert = n + 1;
        first = expert + entries;
        token = first + entries + 1;
        weight = reinterpret_cast<float *>(token + entries);
    }
};
constexpr int table_words(int entries) { return 4 * entries + 2; }

// LDS of the routing: the table and what it is made from.
__host__ GM_DEV constexpr int route_words(int entries, int experts) { return (table_words(entries) + 1) / 2 * 2 + 2 * experts + 2 * entries + experts; }

// The choice of tokens first, first + step, ..., the next one's logits on their way while one is chosen from.
template <int V>
GM_DEV void choose_few(const LayerArgs &a, int first, int step, uint64_t *mask, int32_t *list_e, float *list_w) {
    const int lane = threadIdx.x & 63;
    float l[V], next[V], p[V];
    auto fetch = [&](int t, float(&v)[V]) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int e = j * 64 + lane;
            const int64_t at = t * a.ls + (e < a.n_experts ? e : 0);
            v[j] = a.logit_type == GMAGNUS_DATA_FP32   ? static_cast<const float *>(a.logits)[at]
                   : a.logit_type == GMAGNUS_DATA_BF16 ? (float)static_cast<const __bf16 *>(a.logits)[at]
                                                       : (float)static_cast<const _Float16 *>(a.logits)[at];
        }
    };
    if (first < a.n_tokens) fetch(first, l);
    for (int t = first; t < a.n_tokens; t += step) {
        if (t + step < a.n_tokens) fetch(t + step, next);
        uint64_t chosen[V];
        int n, before = t * a.top_k;
        const float scale = choose<float, V>(l, a.n_experts, a.top_k, a.normalise, chosen, p, n);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (chosen[j] >> lane & 1) {
                const int at = before + __popcll(chosen[j] & lanemask_lt());
                list_e[at] = j * 64 + lane;
                list_w[at] = p[j] * scale;
                atomicOr(reinterpret_cast<unsigned long long *>(&mask[j * 64 + lane]), 1ull << t);
            }
            before += __popcll(chosen[j]);
            l[j] = next[j];
        }
        for (int i = before + lane; i < (t + 1) * a.top_k; i += 64) list_e[i] = -1;
    }
}

// Fills the table in LDS; all threads of a work group.
GM_DEV void route_few(const LayerArgs &a, int32_t *lds, int waves) {
    const int entries = a.n_tokens * a.top_k, lane = threadIdx.x & 63, w = threadIdx.x / 64;
    const Table t(lds, entries);
    uint64_t *mask = reinterpret_cast<uint64_t *>(lds + (table_words(entries) + 1) / 2 * 2);
    int32_t *list_e = reinterpret_cast<int32_t *>(mask + a.n_experts);
    float *list_w = reinterpret_cast<float *>(list_e + entries);
    int32_t *row_of = reinterpret_cast<int32_t *>(list_w + entries);
    for (int e = threadIdx.x; e < a.n_experts; e += 64 * waves) mask[e] = 0;
    __syncthreads();
    if (a.n_experts <= 64)
        choose_few<1>(a, w, waves, mask, list_e, list_w);
    else if (a.n_experts <= 256)
        choose_few<4>(a, w, waves, mask, list_e, list_w);
    else
        choose_few<16>(a, w, waves, mask, list_e, list_w);
    __syncthreads();
    if (w == 0) {
        int used = 0, rows = 0;
        for (int e0 = 0; e0 < a.n_experts; e0 += 64) {
            const int e = e0 + lane, n = e < a.n_experts ? __popcll(mask[e]) : 0;
            const uint64_t some = ballot(n > 0);
            const int upto = wave_incl_scan<int32_t>(n);
            if (n > 0) {
                const int at = used + __popcll(some & lanemask_lt());
                t.expert[at] = e;
                t.first[at] = row_of[e] = rows + upto - n;
            }
            used += __popcll(some);
            rows += __builtin_amdgcn_readlane(upto, 63);
        }
        if (lane == 0) {
            t.first[used] = rows;
            *t.n = used;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < entries; i += 64 * waves) {
        const int e = list_e[i], token = i / a.top_k;
        if (e < 0) continue;
        const int row = row_of[e] + __popcll(mask[e] & ((1ull << token) - 1));
        t.token[row] = token;
        t.weight[row] = list_w[i];
    }
    __syncthreads();
}

__host__ GM_DEV constexpr int up_words(bool route, int entries, int experts) { return route ? route_words(entries, experts) : table_words(entries); }

// What the second kernel begins with: the routing, and no split counted.
GM_DEV void begin_second(const LayerArgs &a, const int32_t *table) {
    for (int i = threadIdx.x; i < table_words(a.n_tokens * a.top_k); i += blockDim.x) a.table[i] = table[i];
    for (int i = threadIdx.x; i < (a.n + 31) / 32; i += blockDim.x) a.arrived[i] = 0;
}

// More than 16 tokens: the routing by one work group, four tokens a wave. (In every work group of the next
// kernel it would take up to 16 a wave.)
constexpr int ROUTE_WAVES = 16;
__global__ __launch_bounds__(64 * ROUTE_WAVES) void k_layer_route(LayerArgs a) {
    extern __shared__ __align__(16) int32_t lds_layer[];
    route_few(a, lds_layer, ROUTE_WAVES);
    begin_second(a, lds_layer);
}

// ------------------------------------------------------------------- fragments
// A block of the reduction is 128 bytes of a row of weights: 64 values of 16 bits or
// 128 of 8. A lane has 16 bytes at g and 16 at g + 4 of a row's eight pieces, S
// fragments of 8 values each. Values of 8 bits are widened, exactly, to the rows' type.

// A gate's result is kept as two values of the rows' type, itself and what its rounding left: rounded once it would add
// as much error to the layer's result as that has from its own rounding. What is left is taken REST times, as many as fit:
// fp16 has 2^-25 for its least half step, and small results would be no better for their second value (of 1e-6, 3 %).
template <typename T>
constexpr float REST = std::is_same<T, _Float16>::value ? 2048.f : 1.f;

enum Kind { SAME, FP8, INT8 };  // weights: of the rows' type, E4M3 with block scales, integers with a scale a row

template <Kind KIND, typename T>
struct Block {
    static constexpr bool EIGHT = KIND != SAME;
    static constexpr int S = EIGHT ? 2 : 1, VALUES = EIGHT ? 128 : 64, BYTES = EIGHT ? 1 : 2;
    static_assert(VALUES * BYTES == 128, "");

    GM_DEV static int first(int h, int g) { return (h * 64 + g * 16) / BYTES; }
    GM_DEV static u32x4 load(const uint8_t *p) {
        if constexpr (EIGHT)
            return load16(p, 16);
        else
            return load8(reinterpret_cast<const T *>(p), 8);
    }
    GM_DEV static void widen(u32x4 v, u32x4 (&f)[S]) {
        if constexpr (!EIGHT) {
            f[0] = v;
        } else if constexpr (KIND == INT8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t u = v[i] ^ 0x80808080u;  // value + 128
                if constexpr (std::is_same<T, __bf16>::value) {
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        f[i / 2][i % 2 * 2 + k] = pack2<T>((float)(u >> (16 * k) & 0xff) - 128.f, (float)(u >> (16 * k + 8) & 0xff) - 128.f);
                } else {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {  // 1024 + u as fp16 has u in its low byte
                        const f16x2 h = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(u, 0x64006400u, k ? 0x01070106u : 0x01050104u));
                        f[i / 2][i % 2 * 2 + k] = __builtin_bit_cast(uint32_t, h - f16x2{(_Float16)1152.f, (_Float16)1152.f});
                    }
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (std::is_same<T, __bf16>::value) {
                    f[i / 2][i % 2 * 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)v[i], 1.f, false));
                    f[i / 2][i % 2 * 2 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)v[i], 1.f, true));
                } else {
                    f[i / 2][i % 2 * 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)v[i], 1.f, false));
                    f[i / 2][i % 2 * 2 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)v[i], 1.f, true));
                }
            }
        }
    }
    // the rows' fragments of a block at p
    GM_DEV static void load_rows(const T *p, int g, u32x4 (&f)[2 * S]) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int s = 0; s < S; ++s) f[h * S + s] = load8(p + first(h, g) + s * 8, 8);
    }
    // a row of weights' and the rows' fragments of the block at value k of n, which may end inside it
    GM_DEV static void load_cut(const uint8_t *row, int k, int n, int g, u32x4 (&f)[2]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) f[h] = cut_piece(row, (int64_t)(k + first(h, g)) * BYTES, (int64_t)n * BYTES);
    }
    GM_DEV static void load_rows_cut(const T *row, int k, int n, int g, u32x4 (&f)[2 * S]) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int s = 0; s < S; ++s)
                f[h * S + s] = cut_piece(reinterpret_cast<const uint8_t *>(row), (int64_t)(k + first(h, g) + s * 8) * 2, (int64_t)n * 2);
    }
    // acc += weights' fragments times the rows' (of P parts, the second REST times), by `scale` where blocks have one
    template <int P>
    GM_DEV static void multiply(const u32x4 (&w)[2], const u32x4 (&r)[P][2 * S], f32x4 scale, f32x4 &acc) {
        constexpr bool APART = P == 2 && REST<T> != 1.f;
        f32x4 sum = KIND == FP8 ? f32x4{0, 0, 0, 0} : acc, rest = {0, 0, 0, 0};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u32x4 f[S];
            widen(w[h], f);
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    f32x4 &to = APART && p == 1 ? rest : sum;
                    to = mfma_16x16x32(f[s], r[p][h * S + s], to, T{});
                }
        }
        if constexpr (APART)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += rest[e] * (1.f / REST<T>);
        if constexpr (KIND != FP8)
            acc = sum;
        else
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += scale[e] * sum[e];
    }
};

constexpr int WAVES = 4;
constexpr int PITCH = 32 + 4;  // of 32 fp32 results in LDS

// ---------------------------------------------------------------- W1 and gate
// An item is 16 columns of an expert's gate: 16 rows of G_e and 16 of U_e. The waves of a
// work group take turns at the blocks of the rows, U blocks' loads in flight each, and
// their sums are joined in LDS in the waves' order. RT: how many times 16 rows of an
// expert are multiplied while the weights are in registers; more than those read them
// again. ROUTE: the work group finds the routing (up to 16 tokens, four a wave).
// Bound by the weights' bytes: 16 tokens to 4 of 64 experts, 2048 to 1024 (344 MB), 60 us,
// 5.7 TB/s; 64 tokens to 6 of 64 (537 MB) 99; 48 tokens to 6 of 55, E4M3, 2048 to 1000 (224 MB) 54.
// One token to 2 of 16, 1024 to 2048 (17 MB), 7.8 us: latency of the routing and of one
// round of loads. (A wave with whole rows to itself, when the kernel took 65: 82 us.)
template <Kind KIND, typename T, int RT, bool ROUTE>
__global__ __launch_bounds__(64 * WAVES) void k_layer_up(LayerArgs a) {
    using B = Block<KIND, T>;
    constexpr int U = RT > 1 || B::EIGHT ? 2 : 4;
    extern __shared__ __align__(16) int32_t lds_layer[];
    const int entries = a.n_tokens * a.top_k;
    const int lane = threadIdx.x & 63, i16 = lane % 16, g = lane / 16;
    const int w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64));
    float *part = reinterpret_cast<float *>(lds_layer + (up_words(ROUTE, entries, a.n_experts) + 3) / 4 * 4);
    if constexpr (ROUTE) {
        route_few(a, lds_layer, WAVES);
        if (blockIdx.x == 0) begin_second(a, lds_layer);
    } else {
        for (int i = threadIdx.x; i < table_words(entries); i += 64 * WAVES) lds_layer[i] = a.table[i];
        __syncthreads();
    }
    const Table t(lds_layer, entries);
    const int tiles = (a.f + 15) / 16, n_used = __builtin_amdgcn_readfirstlane(*t.n);
    const int full = a.d / B::VALUES;
    for (int64_t it = blockIdx.x; it < (int64_t)n_used * tiles; it += gridDim.x) {
        const int u = (int)(it / tiles), f0 = (int)(it - (int64_t)u * tiles) * 16;
        const int e = __builtin_amdgcn_readfirstlane(t.expert[u]), base = __builtin_amdgcn_readfirstlane(t.first[u]);
        const int rows = __builtin_amdgcn_readfirstlane(t.first[u + 1]) - base;
        // (rows and columns that are not there read the last ones: their results are not used)
        const int c = min(f0 + i16, a.f - 1);
        const uint8_t *wr[2] = {a.w1 + e * a.w1g + c * a.w1s, a.w1 + e * a.w1g + ((int64_t)a.f + c) * a.w1s};
        // a tile of U_e's rows may lie in two blocks of scales
        const float *sg = nullptr, *su = nullptr, *sv = nullptr;
        bool second[4] = {};
        if constexpr (KIND == FP8) {
            const int64_t r0 = (int64_t)a.f + f0, last = min(r0 + 15, 2 * (int64_t)a.f - 1);
            sg = a.s1 + e * a.s1g + f0 / SB * a.s1s;
            su = a.s1 + e * a.s1g + r0 / SB * a.s1s;
            sv = a.s1 + e * a.s1g + last / SB * a.s1s;
#pragma unroll
            for (int i = 0; i < 4; ++i) second[i] = (r0 + 4 * g + i) / SB != r0 / SB;
        }
        auto scales = [&](int kb, f32x4(&s)[2]) {
            if constexpr (KIND == FP8) {
                const float x = sg[kb], y = su[kb], z = sv[kb];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[0][i] = x;
                    s[1][i] = second[i] ? z : y;
                }
            }
        };
        // (at most 16 tokens: one pass)
        for (int r0 = 0; RT == 1 ? r0 == 0 : r0 < rows; r0 += 16 * RT) {
            const T *xr[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r) xr[r] = static_cast<const T *>(a.x) + t.token[base + min(r0 + 16 * r + i16, rows - 1)] * a.xs;
            f32x4 acc[RT][2] = {};
            for (int k0 = w; k0 < full; k0 += WAVES * U) {
                u32x4 fw[U][2][2], fx[U][1][2 * B::S];
                f32x4 s[U][2];
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const int kb = min(k0 + i * WAVES, full - 1);
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int h = 0; h < 2; ++h) fw[i][j][h] = B::load(wr[j] + (int64_t)kb * 128 + h * 64 + g * 16);
                    B::load_rows(xr[0] + kb * B::VALUES, g, fx[i][0]);
                    scales(kb, s[i]);
                }
#pragma unroll
                for (int i = 0; i < U; ++i)
                    if (k0 + i * WAVES < full)
#pragma unroll
                        for (int j = 0; j < 2; ++j) B::multiply(fw[i][j], fx[i], s[i][j], acc[0][j]);
#pragma unroll
                for (int r = 1; r < RT; ++r)
                    if (r0 + 16 * r < rows) {
#pragma unroll
                        for (int i = 0; i < U; ++i) B::load_rows(xr[r] + min(k0 + i * WAVES, full - 1) * B::VALUES, g, fx[i][0]);
#pragma unroll
                        for (int i = 0; i < U; ++i)
                            if (k0 + i * WAVES < full)
#pragma unroll
                                for (int j = 0; j < 2; ++j) B::multiply(fw[i][j], fx[i], s[i][j], acc[r][j]);
                    }
            }
            if (full * B::VALUES < a.d && w == full % WAVES) {  // what is left of the last block
                u32x4 fw[2][2];
                f32x4 s[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) B::load_cut(wr[j], full * B::VALUES, a.d, g, fw[j]);
                scales(full, s);
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    if (r0 + 16 * r < rows) {
                        u32x4 fx[1][2 * B::S];
                        B::load_rows_cut(xr[r], full * B::VALUES, a.d, g, fx[0]);
#pragma unroll
                        for (int j = 0; j < 2; ++j) B::multiply(fw[j], fx, s[j], acc[r][j]);
                    }
            }
            T *out = static_cast<T *>(a.act) + (base + r0) * a.act_stride + f0;
            __syncthreads();  // (the last item's sums)
#pragma unroll
            for (int r = 0; r < RT; ++r)
                if (r0 + 16 * r < rows)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        *reinterpret_cast<f32x4 *>(&part[((w * RT + r) * 16 + i16) * PITCH + 16 * j + 4 * g]) = acc[r][j];
            __syncthreads();
            for (int i = threadIdx.x; i < min(rows - r0, RT * 16) * 16; i += 64 * WAVES) {
                const int r = i / 16, col = i % 16;
                float x = 0.f, y = 0.f;
#pragma unroll
                for (int v = 0; v < WAVES; ++v) {
                    x += part[(v * RT * 16 + r) * PITCH + col];
                    y += part[(v * RT * 16 + r) * PITCH + 16 + col];
                }
                if (f0 + col < a.f) {
                    if constexpr (KIND == INT8) {
                        x *= a.s1[e * a.s1g + f0 + col];
                        y *= a.s1[e * a.s1g + a.f + f0 + col];
                    }
                    const float v = gated(x, y);
                    const T top = (T)v;
                    out[r * a.act_stride + col] = top;
                    // (an infinite one leaves nothing)
                    out[a.act_part + r * a.act_stride + col] = fabsf((float)top) < INFINITY ? (T)((v - (float)top) * REST<T>) : (T)0.f;
                }
            }
        }
    }
}

// ----------------------------------------------------------------- W2 and sums
// A work group takes 32 columns of the result and every splits-th run of units; a
// wave's unit is U blocks of one expert's rows of W2, whose products go, times
// the tokens' weights, into the wave's own sums in LDS. The waves' sums are added in
// their order, and the splits' by the last of them to arrive, in theirs. The sizes above:
// 31 us (5.5 TB/s), 52-55, 44 (2.5: rows of 1000 bytes lie across lines, 135 MB come for 112),
// one token 6.4.
// (Waves a SIMD: integers in fp16, left alone, took registers for two: 48 tokens, 2048 x 1000, 145 us a layer, here 123.)
template <Kind KIND, typename T, typename OUT>
__global__ __launch_bounds__(64 * WAVES, KIND == SAME ? 4 : 3) void k_layer_down(LayerArgs a) {
    using B = Block<KIND, T>;
    constexpr int U = B::EIGHT ? 1 : 2;
    extern __shared__ __align__(16) int32_t lds_layer[];
    const int entries = a.n_tokens * a.top_k;
    const int lane = threadIdx.x & 63, i16 = lane % 16, g = lane / 16;
    const int w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64));
    const int tile = blockIdx.x / a.splits, split = blockIdx.x - tile * a.splits, q0 = tile * 32;
    float *sums = reinterpret_cast<float *>(lds_layer + (table_words(entries) + 3) / 4 * 4), *mine = sums + w * a.n_tokens * PITCH;
    for (int i = threadIdx.x; i < table_words(entries); i += 64 * WAVES) lds_layer[i] = a.table[i];
    for (int i = threadIdx.x; i < WAVES * a.n_tokens * PITCH; i += 64 * WAVES) sums[i] = 0.f;
    __syncthreads();
    const Table t(lds_layer, entries);
    const int n_used = __builtin_amdgcn_readfirstlane(*t.n);
    constexpr int CHUNK = U * B::VALUES;
    const int per = (a.f + CHUNK - 1) / CHUNK;
    // (an expert's units begin elsewhere with each turn: the last ones of rows that end inside a unit take longer)
    const int turns = max(1, a.splits * WAVES / per);
    for (int unit = split * WAVES + w; unit < n_used * per; unit += a.splits * WAVES) {
        const int u = unit / per, k0 = (unit - u * per + u / turns) % per * CHUNK;
        const int e = __builtin_amdgcn_readfirstlane(t.expert[u]), base = __builtin_amdgcn_readfirstlane(t.first[u]);
        const int rows = __builtin_amdgcn_readfirstlane(t.first[u + 1]) - base;
        const uint8_t *wr[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) wr[j] = a.w2 + e * a.w2g + min(q0 + 16 * j + i16, a.n - 1) * a.w2s;
        const float *sc = KIND == FP8 ? a.s2 + e * a.s2g + q0 / SB * a.s2s : nullptr;
        f32x4 sr[2];  // of the rows of W2 that a lane has results of
        if constexpr (KIND == INT8)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) sr[j][i] = a.s2[e * a.s2g + min(q0 + 16 * j + 4 * g + i, a.n - 1)];
        auto row_at = [&](int r) { return static_cast<const T *>(a.act) + (base + min(r + i16, rows - 1)) * a.act_stride; };
        auto add = [&](int r, const f32x4(&acc)[2]) {
            if (r + i16 < rows) {
                const int token = t.token[base + r + i16];
                const float weight = t.weight[base + r + i16];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    f32x4 *p = reinterpret_cast<f32x4 *>(&mine[token * PITCH + 16 * j + 4 * g]);
                    f32x4 v = *p;
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] += weight * (KIND == INT8 ? acc[j][i] * sr[j][i] : acc[j][i]);
                    *p = v;
                }
            }
        };
        auto scale = [&](int i) {
            const float x = KIND == FP8 ? sc[k0 / B::VALUES + i] : 0.f;
            return f32x4{x, x, x, x};
        };
        if (a.f - k0 >= CHUNK) {
            u32x4 fw[U][2][2], fr[U][2][2 * B::S];
            f32x4 s[U];
            const T *row = row_at(0);
#pragma unroll
            for (int i = 0; i < U; ++i) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h) fw[i][j][h] = B::load(wr[j] + k0 * B::BYTES + i * 128 + h * 64 + g * 16);
#pragma unroll
                for (int p = 0; p < 2; ++p) B::load_rows(row + p * a.act_part + k0 + i * B::VALUES, g, fr[i][p]);
                s[i] = scale(i);
            }
            for (int r = 0;;) {
                f32x4 acc[2] = {};
#pragma unroll
                for (int i = 0; i < U; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) B::multiply(fw[i][j], fr[i], s[i], acc[j]);
                add(r, acc);
                r += 16;
                if (r >= rows) break;
                row = row_at(r);
#pragma unroll
                for (int i = 0; i < U; ++i)
#pragma unroll
                    for (int p = 0; p < 2; ++p) B::load_rows(row + p * a.act_part + k0 + i * B::VALUES, g, fr[i][p]);
            }
        } else {
            for (int r = 0; r < rows; r += 16) {
                f32x4 acc[2] = {};
                const T *row = row_at(r);
                for (int i = 0; k0 + i * B::VALUES < a.f; ++i) {
                    u32x4 fw[2][2], fr[2][2 * B::S];
#pragma unroll
                    for (int j = 0; j < 2; ++j) B::load_cut(wr[j], k0 + i * B::VALUES, a.f, g, fw[j]);
#pragma unroll
                    for (int p = 0; p < 2; ++p) B::load_rows_cut(row + p * a.act_part, k0 + i * B::VALUES, a.f, g, fr[p]);
#pragma unroll
                    for (int j = 0; j < 2; ++j) B::multiply(fw[j], fr, scale(i), acc[j]);
                }
                add(r, acc);
            }
        }
    }
    __syncthreads();
    const int cols = a.n - q0;
    auto joined = [&](int i) {
        const int at = i / 8 * PITCH + i % 8 * 4;
        f32x4 v = *reinterpret_cast<const f32x4 *>(&sums[at]);
#pragma unroll
        for (int x = 1; x < WAVES; ++x) v += *reinterpret_cast<const f32x4 *>(&sums[x * a.n_tokens * PITCH + at]);
        return v;
    };
    auto result = [&](int i, f32x4 v) { store4(static_cast<OUT *>(a.out) + i / 8 * a.os + q0 + i % 8 * 4, v, cols - i % 8 * 4); };
    if (a.splits == 1) {
        for (int i = threadIdx.x; i < a.n_tokens * 8; i += 64 * WAVES) result(i, joined(i));
        return;
    }
    // Shares go past the caches of this XCD and are read past those of the last one's: agent
    // scope for each access, where a fence would write back and drop whole caches, once a
    // work group (16 tokens to 4 of 64 experts of 1024 x 2048: this kernel 300 us with fences).
    // What orders them is the wait for the stores' end before the barrier and the count.
    uint64_t *share = reinterpret_cast<uint64_t *>(a.share) + (int64_t)tile * a.splits * a.n_tokens * 16;
    for (int i = threadIdx.x; i < a.n_tokens * 16; i += 64 * WAVES) {
        const int at = i / 16 * PITCH + i % 16 * 2;
        float x = sums[at], y = sums[at + 1];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) {
            x += sums[v * a.n_tokens * PITCH + at];
            y += sums[v * a.n_tokens * PITCH + at + 1];
        }
        __hip_atomic_store(&share[split * a.n_tokens * 16 + i], __builtin_bit_cast(uint64_t, u32x2{__float_as_uint(x), __float_as_uint(y)}),
                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __shared__ int arrived;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) arrived = __hip_atomic_fetch_add(&a.arrived[tile], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (arrived != a.splits - 1) return;
    for (int i = threadIdx.x; i < a.n_tokens * 16; i += 64 * WAVES) {
        float x = 0.f, y = 0.f;
        for (int s0 = 0; s0 < a.splits; s0 += 16) {  // (16 loads in flight)
            uint64_t v[16];
#pragma unroll
            for (int s = 0; s < 16; ++s)
                v[s] = __hip_atomic_load(&share[min(s0 + s, a.splits - 1) * a.n_tokens * 16 + i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
            for (int s = 0; s < 16; ++s)
                if (s0 + s < a.splits) {
                    const u32x2 p = __builtin_bit_cast(u32x2, v[s]);
                    x += __uint_as_float(p[0]);
                    y += __uint_as_float(p[1]);
                }
        }
        OUT *p = static_cast<OUT *>(a.out) + i / 16 * a.os + q0 + i % 16 * 2;
        if (i % 16 * 2 < cols) p[0] = (OUT)x;
        if (i % 16 * 2 + 1 < cols) p[1] = (OUT)y;
    }
}

// ------------------------------------------------------------------- host side
struct LayerLayout {
    int64_t arrived, table, act, share, bytes, act_stride;
    int splits;
    LayerLayout(int64_t t, int64_t e, int64_t k, int64_t f, int64_t n, bool eight) {
        int64_t at = 0;
        auto take = [&](int64_t bytes) {
            const int64_t here = at;
            at += (bytes + 255) / 256 * 256;
            return here;
        };
        // Splits for two work groups a CU, of 8-bit weights for three, as many at most as there can be waves' units. The
        // second kernel, 2048 x 1024 (outputs x inner), 16 tokens to 4 of 64 experts: 256 work groups 31 us, 512 30, 768 31,
        // 1024 35, 2048 48; 64 tokens to 6 of 64 53, 52, 55, 72, 92; E4M3, 16 tokens 23, 17, 17, 20, 30, 48 tokens to 6 of 64,
        // 2048 x 1000, 94, 58, 50, 50, 71. The whole layer with integers, 16 tokens: 256 work groups 64 us, 512 59, 768 54,
        // 1024 64, 48 tokens 150, 126, 125, 138 (in fp16 141, 119, 121, 135).
        const int64_t tiles = (n + 31) / 32, used = e < t * k ? e : t * k, units = used * ((f + 127) / 128);
        int64_t s = ((eight ? 768 : 512) + tiles - 1) / tiles;
        if (s > (units + WAVES - 1) / WAVES) s = (units + WAVES - 1) / WAVES;
        splits = (int)s;
        act_stride = (f + 7) / 8 * 8;
        arrived = take(tiles * 4);
        table = take(table_words((int)(t * k)) * 4);
        act = take(2 * t * k * act_stride * 2);
        share = take(s > 1 ? tiles * s * t * 32 * 4 : 0);
        bytes = at;
    }
};

// A launch's LDS stays below the 64 KB that need no leave.
static_assert(4 * (route_words(MAX_ENTRIES, MAX_EXPERTS) + 4 + WAVES * 16 * PITCH) < 64 << 10 &&
                  4 * (table_words(MAX_ENTRIES) + 4 + WAVES * MAX_TOKENS * PITCH) + 16 < 64 << 10,
              "");

// A launch has less than 2^32 threads, and the second kernel a work group for every 32 columns.
constexpr int64_t MAX_OUT = (((int64_t(1) << 32) - 1) / (64 * WAVES)) * 32;

bool layer_sizes_ok(int64_t t, int64_t e, int64_t k, int64_t f, int64_t n) {
    return t >= 0 && t <= MAX_TOKENS && e >= 1 && e <= MAX_EXPERTS && k >= 1 && k <= e && t * k <= MAX_ENTRIES && f >= 1 &&
           2 * f <= MAX_SIDE && n >= 1 && n <= MAX_OUT;
}

}  // namespace
}  // namespace gm

using namespace gm;

extern "C" int64_t gmagnus_expert_layer_workspace_bytes(int64_t n_tokens, int64_t n_experts, int64_t top_k, int64_t inner,
                                                        int64_t n_cols) {
    // (8-bit weights have as many splits or more)
    return layer_sizes_ok(n_tokens, n_experts, top_k, inner, n_cols) ? LayerLayout(n_tokens, n_experts, top_k, inner, n_cols, true).bytes : 0;
}

extern "C" gmagnus_status_t gmagnus_expert_layer(const gmagnus_dense_t *X, const gmagnus_dense_t *logits, int64_t top_k,
                                                 int32_t normalise, const gmagnus_dense_t *W1, const gmagnus_dense_t *W1_scale,
                                                 const gmagnus_dense_t *W2, const gmagnus_dense_t *W2_scale,
                                                 const gmagnus_dense_t *OUT, void *workspace, int64_t workspace_bytes,
                                                 void *hip_stream) {
    return guarded([&] {
        GM_REQUIRE(X && logits && W1 && W2 && OUT, GMAGNUS_ERROR_INVALID_VALUE, "NULL X, logits, W1, W2 or OUT");
        const int64_t t = X->n_rows, d = X->n_cols, e = logits->n_cols, f = W2->n_cols, n = OUT->n_cols;
        GM_REQUIRE(t >= 0 && e >= 1 && top_k >= 1 && top_k <= e, GMAGNUS_ERROR_INVALID_VALUE,
                   "top_k must lie in 1 .. number of experts");
        GM_REQUIRE(normalise == 0 || normalise == 1, GMAGNUS_ERROR_INVALID_VALUE, "normalise must be 0 or 1");
        check_side(d, "columns of X");
        check_side(n, "columns of OUT");
        GM_REQUIRE(n <= MAX_OUT, GMAGNUS_ERROR_UNSUPPORTED, "columns of OUT beyond 2^29 - 32");
        check_side(f, "columns of W2");
        check_side(2 * f, "rows of W1");
        GM_REQUIRE(t <= MAX_TOKENS, GMAGNUS_ERROR_UNSUPPORTED, "more than 64 tokens: call the routing and the grouped products");
        GM_REQUIRE(e <= MAX_EXPERTS && t * top_k <= MAX_ENTRIES, GMAGNUS_ERROR_UNSUPPORTED, "more than 1024 experts or entries");
        check_dense(X, "X", t, d);
        check_dense(logits, "logits", t, e);
        check_dense(W1, "W1", 2 * f, d, e, GMAGNUS_DATA_INT8);
        check_dense(W2, "W2", n, f, e, GMAGNUS_DATA_INT8);
        check_dense(OUT, "OUT", t, n);
        GM_REQUIRE(X->data_type == GMAGNUS_DATA_BF16 || X->data_type == GMAGNUS_DATA_FP16, GMAGNUS_ERROR_INVALID_VALUE,
                   "X must be bf16 or fp16");
        GM_REQUIRE(is_float(logits->data_type), GMAGNUS_ERROR_INVALID_VALUE, "logits must be fp32, bf16 or fp16");
        GM_REQUIRE(OUT->data_type == X->data_type || OUT->data_type == GMAGNUS_DATA_FP32, GMAGNUS_ERROR_INVALID_VALUE,
                   "OUT must have the type of X, or fp32");
        const Kind kind = W1->data_type == GMAGNUS_DATA_FP8_E4M3 ? FP8 : W1->data_type == GMAGNUS_DATA_INT8 ? INT8 : SAME;
        GM_REQUIRE(W1->data_type == W2->data_type && (kind != SAME || W1->data_type == X->data_type), GMAGNUS_ERROR_INVALID_VALUE,
                   "W1 and W2 must both have the type of X, both be E4M3 or both int8");
        GM_REQUIRE(!W1_scale == (kind == SAME) && !W2_scale == (kind == SAME), GMAGNUS_ERROR_INVALID_VALUE,
                   "8-bit weights have scales, others none");
        if (kind == FP8) {
            check_dense(W1_scale, "W1_scale", (2 * f + SB - 1) / SB, (d + SB - 1) / SB, e);
            check_dense(W2_scale, "W2_scale", (n + SB - 1) / SB, (f + SB - 1) / SB, e);
        } else if (kind == INT8) {
            check_dense(W1_scale, "W1_scale", e, 2 * f);
            check_dense(W2_scale, "W2_scale", e, n);
        }
        GM_REQUIRE(kind == SAME || (W1_scale->data_type == GMAGNUS_DATA_FP32 && W2_scale->data_type == GMAGNUS_DATA_FP32),
                   GMAGNUS_ERROR_INVALID_VALUE, "scales must be fp32");
        if (t == 0) return;
        const LayerLayout l(t, e, top_k, f, n, kind != SAME);
        GM_REQUIRE(workspace && workspace_bytes >= l.bytes, GMAGNUS_ERROR_INVALID_VALUE,
                   "workspace below gmagnus_expert_layer_workspace_bytes");
        GM_REQUIRE((uintptr_t)workspace % 16 == 0, GMAGNUS_ERROR_INVALID_VALUE, "workspace is not 16-byte aligned");
        const int64_t tiles = (n + 31) / 32, entries = t * top_k, used = e < entries ? e : entries;
        GM_REQUIRE(used * ((f + 127) / 128) < INT32_MAX / 2, GMAGNUS_ERROR_UNSUPPORTED, "2^30 units of the reduction or more");
        char *ws = static_cast<char *>(workspace);
        const int size = kind == SAME ? 2 : 1;
        // (integers' scales: a row an expert)
        auto rows_of = [&](const gmagnus_dense_t *m) { return kind == FP8 ? m->row_stride : 0; };
        auto stack_of = [&](const gmagnus_dense_t *m) { return kind == FP8 ? m->stack_stride : kind == INT8 ? m->row_stride : 0; };
        const LayerArgs a{X->data, logits->data, (const uint8_t *)W1->data, (const uint8_t *)W2->data,
                          kind == SAME ? nullptr : (const float *)W1_scale->data, kind == SAME ? nullptr : (const float *)W2_scale->data,
                          OUT->data, X->row_stride, logits->row_stride, W1->row_stride * size, W1->stack_stride * size,
                          rows_of(W1_scale), stack_of(W1_scale), W2->row_stride * size, W2->stack_stride * size, rows_of(W2_scale),
                          stack_of(W2_scale), OUT->row_stride, (int)t, (int)e, (int)top_k, normalise, logits->data_type, (int)d,
                          (int)f, (int)n, l.splits, (int32_t *)(ws + l.arrived), (int32_t *)(ws + l.table), ws + l.act,
                          (float *)(ws + l.share), l.act_stride, entries * l.act_stride};
        hipStream_t s = (hipStream_t)hip_stream;
        const int64_t items = used * ((f + 15) / 16);
        auto go = [&](auto kernel, int64_t grid, int threads, int words) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(threads), words * 4, s, a);
            GM_CHECK_LAUNCH();
        };
        const int route = (route_words((int)entries, (int)e) + 3) / 4 * 4, table = (table_words((int)entries) + 3) / 4 * 4;
        auto both = [&](auto v, auto w) {
            using T = decltype(v);
            constexpr Kind KIND = decltype(w)::value;
            const int64_t grid = items < 1024 ? items : 1024;
            if (t <= 16) {
                go(k_layer_up<KIND, T, 1, true>, grid, 64 * WAVES, route + WAVES * 16 * PITCH);
            } else {
                go(k_layer_route, 1, 64 * ROUTE_WAVES, route);
                go(k_layer_up<KIND, T, 2, false>, grid, 64 * WAVES, table + WAVES * 32 * PITCH);
            }
            if (OUT->data_type == GMAGNUS_DATA_FP32)
                go(k_layer_down<KIND, T, float>, tiles * l.splits, 64 * WAVES, table + WAVES * (int)t * PITCH);
            else
                go(k_layer_down<KIND, T, T>, tiles * l.splits, 64 * WAVES, table + WAVES * (int)t * PITCH);
        };
        auto any = [&](auto v) {
            if (kind == FP8)
                both(v, std::integral_constant<Kind, FP8>{});
            else if (kind == INT8)
                both(v, std::integral_constant<Kind, INT8>{});
            else
                both(v, std::integral_constant<Kind, SAME>{});
        };
        if (X->data_type == GMAGNUS_DATA_BF16)
            any(__bf16{});
        else
            any(_Float16{});
    });
}
