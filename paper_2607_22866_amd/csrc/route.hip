// The routing matrix of a layer of experts: the top_k of each token's logits
// with their softmax weights, as CSR by token and by expert; its gradient; and
// the products of that matrix with a tall dense one (a token's weighted sum of
// its results) with theirs.
#include <type_traits>

#include "dense.hpp"

namespace gm {
namespace {

constexpr int MAX_EXPERTS = 1024;
constexpr int TOK = 32;            // tokens a work group of the routing takes: one bit each in an expert's mask
constexpr int ROUTE_T = 1024;      // its threads
constexpr int ROUTE_W = ROUTE_T / GM_WAVE;

// ---------------------------------------------------------------- selection
// A logit as an unsigned number of the same order, in as many bits as its type
// has (KEY_BITS); 0 for what is masked (-inf, NaN). -0 counts as +0.
template <typename T>
constexpr int KEY_BITS = 8 * (int)sizeof(T);

template <typename T>
GM_DEV uint32_t order_key(T v) {
    const float x = to_f32(v);
    if constexpr (sizeof(T) == 4) {
        const uint32_t u = __float_as_uint(x + 0.0f);
        return x > -INFINITY ? (u >> 31 ? ~u : u | 0x80000000u) : 0u;
    } else {
        const uint32_t u = x == 0.f ? 0u : __builtin_bit_cast(uint16_t, v);
        return x > -INFINITY ? (u >> 15 ? ~u & 0xffffu : u | 0x8000u) : 0u;
    }
}
template <typename T>
GM_DEV float key_value(uint32_t k) {
    if constexpr (sizeof(T) == 4)
        return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k);
    else
        return to_f32(__builtin_bit_cast(T, (uint16_t)(k >> 15 ? k & 0x7fffu : ~k)));
}

// e^x for x <= 0, by the hardware's power of two: what x log2(e) loses when it is
// rounded (|x| units of 2^-24 of the result) is multiplied in afterwards, so that a few
// units are off at any x. (From -200 on down the result is zero, for NaN too: an
// infinite logit, whose difference to itself that is, has a sum of zero and NaN weights.)
GM_DEV float exp_neg(float x) {
    constexpr float L = 0x1.715476p+0f, L_REST = 0x1.4ae0cp-26f, LN2 = 0x1.62e43p-1f;
    const float y = __builtin_amdgcn_fmed3f(x, -200.f, 0.f), t = y * L;
    const float rest = __builtin_fmaf(y, L_REST, __builtin_fmaf(y, L, -t));
    const float r = __builtin_amdgcn_exp2f(t);
    return __builtin_fmaf(r * LN2, rest, r);
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

struct RouteArgs {
    const void *logits;
    int64_t n_tokens, stride;
    int n_experts, top_k, normalise;
    int64_t n_blocks;
    gmagnus_routing_t out;
    // workspace
    uint32_t *mask;     // [n_blocks][n_experts]: the tokens of the block that chose the expert
    int32_t *base;      // [n_blocks][n_experts]: entries of the expert in earlier blocks
    int32_t *total;     // [n_experts]
    int32_t *block_n;   // [n_blocks]: entries
    int64_t *block_at;  // [n_blocks + 1]: entries before the block
    int32_t *count;     // [n_tokens]
    uint16_t *list_e;   // [n_tokens][top_k]: chosen experts, ascending
    float *list_w;      // their weights
};

// One token by one wave: marks its bit in the chosen experts' masks (LDS) and
// writes its list. Lane l holds experts l, l + 64, ... (V of them). The top_k-th
// largest key is found bit by bit from the top: a bit stays if at least top_k
// keys reach it, and once just top_k do, those are the choice (16384 tokens, 256
// experts, top_k 8: 20 us; taking the maximum over the wave top_k times: 37).
// Keys equal to the last one are taken from the lowest expert on.
template <typename T, int V>
GM_DEV int select_token(const RouteArgs &a, int64_t t, int bit, const T (&l)[V], uint32_t *mask) {
    const int lane = threadIdx.x & 63;
    uint32_t key[V], best = 0;
    uint64_t chosen[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        key[j] = j * 64 + lane < a.n_experts ? order_key(l[j]) : 0u;
        best = best > key[j] ? best : key[j];
    }
    best = wave_max(best);
    const float top = key_value<T>(best);
    auto reach = [&](uint32_t least) {  // keys of at least `least` (above 0)
        int n = 0;
#pragma unroll
        for (int j = 0; j < V; ++j) n += __popcll(ballot(key[j] >= least));
        return n;
    };
    int n = reach(1);
    uint32_t least = 1;
    if (n > a.top_k) {
        least = 0;
        for (uint32_t b = 1u << (KEY_BITS<T> - 1); b; b >>= 1) {
            const int m = reach(least | b);
            if (m >= a.top_k) {
                least |= b;
                n = m;
                if (m == a.top_k) break;
            }
        }
    }
    // n keys reach `least`; more than top_k only where several equal it
    int spare = n > a.top_k ? n - a.top_k : 0;
#pragma unroll
    for (int j = V - 1; j >= 0; --j) {
        chosen[j] = ballot(key[j] >= least);
        if (spare > 0) {
            uint64_t last = ballot(key[j] == least);
            while (spare > 0 && last) {
                const uint64_t high = uint64_t(1) << (63 - __clzll((long long)last));
                last ^= high;
                chosen[j] ^= high;
                --spare;
            }
        }
    }
    n = n < a.top_k ? n : a.top_k;
    float p[V], sum = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        p[j] = key[j] ? exp_neg(key_value<T>(key[j]) - top) : 0.f;
        if (!a.normalise || (chosen[j] >> lane & 1)) sum += p[j];
    }
    const float scale = 1.f / wave_sum(sum);
    int before = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if (chosen[j] >> lane & 1) {
            const int e = j * 64 + lane;
            const int64_t at = t * a.top_k + before + __popcll(chosen[j] & lanemask_lt());
            a.list_e[at] = (uint16_t)e;
            a.list_w[at] = p[j] * scale;
            atomicOr(&mask[e], 1u << bit);
        }
        before += __popcll(chosen[j]);
    }
    if (lane == 0) a.count[t] = n;
    return n;
}

// The tokens of a wave, the next one's logits on their way while one is chosen from.
template <typename T, int V>
GM_DEV int select_tokens(const RouteArgs &a, int64_t t0, int tokens, uint32_t *mask) {
    const int lane = threadIdx.x & 63;
    T l[V], next[V];
    auto fetch = [&](int i, T(&v)[V]) {
        const T *row = static_cast<const T *>(a.logits) + (t0 + i) * a.stride;
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = row[j * 64 + lane < a.n_experts ? j * 64 + lane : 0];
    };
    int n = 0, i = threadIdx.x / 64;
    if (i < tokens) fetch(i, l);
    for (; i < tokens; i += ROUTE_W) {
        if (i + ROUTE_W < tokens) fetch(i + ROUTE_W, next);
        n += select_token<T, V>(a, t0 + i, i, l, mask);
#pragma unroll
        for (int j = 0; j < V; ++j) l[j] = next[j];
    }
    return n;
}

template <typename T, int V>
GM_DEV void select_block(const RouteArgs &a, int64_t blk, uint32_t *mask, int *block_n) {
    const int64_t t0 = blk * TOK;
    const int tokens = (int)(a.n_tokens - t0 < TOK ? a.n_tokens - t0 : TOK);
    for (int e = threadIdx.x; e < a.n_experts; e += ROUTE_T) mask[e] = 0;
    if (threadIdx.x == 0) *block_n = 0;
    __syncthreads();
    const int n = select_tokens<T, V>(a, t0, tokens, mask);
    if ((threadIdx.x & 63) == 0 && n) atomicAdd(block_n, n);
    __syncthreads();
}

// Writes a block's entries in both orders. start[e]: the expert's first grouped
// row that is this block's; first: the block's first entry.
GM_DEV void place_block(const RouteArgs &a, int64_t blk, const uint32_t *mask, const int32_t *start, int64_t first,
                        int64_t n_entries, int *upto) {
    const int64_t t0 = blk * TOK;
    const int tokens = (int)(a.n_tokens - t0 < TOK ? a.n_tokens - t0 : TOK);
    if (threadIdx.x < GM_WAVE) {
        const int c = (int)threadIdx.x < tokens ? a.count[t0 + threadIdx.x] : 0;
        const int inc = wave_incl_scan<int32_t>(c);
        if (threadIdx.x < TOK) upto[threadIdx.x] = inc - c;
        if ((int)threadIdx.x < tokens) a.out.row_ptr[t0 + threadIdx.x] = first + inc - c;
    }
    __syncthreads();
    const int64_t cap = (int64_t)a.n_tokens * a.top_k;
    for (int i = threadIdx.x; i < tokens * a.top_k; i += ROUTE_T) {
        const int t = i / a.top_k, j = i - t * a.top_k;
        const int64_t src = (t0 + t) * a.top_k + j;
        if (j < a.count[t0 + t]) {
            const int e = a.list_e[src];
            const float w = a.list_w[src];
            const int64_t at = first + upto[t] + j;
            const int32_t row = start[e] + __popc(mask[e] & ((1u << t) - 1));
            a.out.expert[at] = e;
            a.out.weight[at] = w;
            a.out.slot[at] = row;
            a.out.token[row] = (int32_t)(t0 + t);
            a.out.group_weight[row] = w;
        }
        if (src >= n_entries && src < cap) {
            a.out.expert[src] = a.out.slot[src] = a.out.token[src] = -1;
            a.out.weight[src] = a.out.group_weight[src] = 0.f;
        }
    }
}

// At most 32 tokens: one work group does it all.
template <typename T, int V>
__global__ __launch_bounds__(ROUTE_T) void k_route_small(RouteArgs a) {
    __shared__ uint32_t mask[MAX_EXPERTS];
    __shared__ int32_t start[MAX_EXPERTS], scan[ROUTE_W], upto[TOK];
    __shared__ int block_n;
    select_block<T, V>(a, 0, mask, &block_n);
    const int e = threadIdx.x;
    const int n = e < a.n_experts ? __popc(mask[e]) : 0;
    const int at = block_excl_scan<ROUTE_T, int32_t>(n, scan);
    if (e < a.n_experts) {
        start[e] = at;
        a.out.group_ptr[e] = at;
    }
    if (e == 0) a.out.row_ptr[a.n_tokens] = a.out.group_ptr[a.n_experts] = block_n;
    __syncthreads();
    place_block(a, 0, mask, start, 0, block_n, upto);
}

template <typename T, int V>
__global__ __launch_bounds__(ROUTE_T) void k_route_select(RouteArgs a) {
    __shared__ uint32_t mask[MAX_EXPERTS];
    __shared__ int block_n;
    for (int64_t blk = blockIdx.x; blk < a.n_blocks; blk += gridDim.x) {
        select_block<T, V>(a, blk, mask, &block_n);
        for (int e = threadIdx.x; e < a.n_experts; e += ROUTE_T) a.mask[blk * a.n_experts + e] = mask[e];
        if (threadIdx.x == 0) a.block_n[blk] = block_n;
        __syncthreads();
    }
}

// Work group g < n_experts / 16: 16 experts' entries over the blocks, 64 runs of
// blocks side by side. The last work group: entries before each block.
constexpr int SCAN_E = 16, SCAN_RUNS = ROUTE_T / SCAN_E;
__global__ __launch_bounds__(ROUTE_T) void k_route_scan(RouteArgs a) {
    __shared__ int32_t part[SCAN_RUNS][SCAN_E];
    if (blockIdx.x == gridDim.x - 1) {
        int64_t *scan = reinterpret_cast<int64_t *>(part);
        int64_t carry = 0;
        for (int64_t b0 = 0; b0 < a.n_blocks; b0 += ROUTE_T) {
            const int64_t b = b0 + threadIdx.x, n = b < a.n_blocks ? a.block_n[b] : 0;
            int64_t all;
            const int64_t at = block_excl_scan<ROUTE_T, int64_t>(n, scan, &all);
            if (b < a.n_blocks) a.block_at[b] = carry + at;
            carry += all;
        }
        if (threadIdx.x == 0) a.block_at[a.n_blocks] = carry;
        return;
    }
    const int x = threadIdx.x % SCAN_E, run = threadIdx.x / SCAN_E;
    const int e = blockIdx.x * SCAN_E + x;
    const int64_t per = (a.n_blocks + SCAN_RUNS - 1) / SCAN_RUNS;
    const int64_t b0 = run * per, b1 = b0 + per < a.n_blocks ? b0 + per : a.n_blocks;
    int32_t n = 0;
    if (e < a.n_experts)
        for (int64_t b = b0; b < b1; ++b) n += __popc(a.mask[b * a.n_experts + e]);
    part[run][x] = n;
    __syncthreads();
    int32_t at = 0;
    for (int r = 0; r < run; ++r) at += part[r][x];
    if (e < a.n_experts) {
        if (run == SCAN_RUNS - 1) a.total[e] = at + n;
        for (int64_t b = b0; b < b1; ++b) {
            a.base[b * a.n_experts + e] = at;
            at += __popc(a.mask[b * a.n_experts + e]);
        }
    }
}

__global__ __launch_bounds__(ROUTE_T) void k_route_place(RouteArgs a) {
    __shared__ uint32_t mask[MAX_EXPERTS];
    __shared__ int32_t start[MAX_EXPERTS], scan[ROUTE_W], upto[TOK];
    const int e = threadIdx.x;
    const int32_t at = block_excl_scan<ROUTE_T, int32_t>(e < a.n_experts ? a.total[e] : 0, scan);
    const int64_t n_entries = a.block_at[a.n_blocks];
    if (blockIdx.x == 0) {
        if (e < a.n_experts) a.out.group_ptr[e] = at;
        if (e == 0) a.out.row_ptr[a.n_tokens] = a.out.group_ptr[a.n_experts] = n_entries;
    }
    for (int64_t blk = blockIdx.x; blk < a.n_blocks; blk += gridDim.x) {
        if (e < a.n_experts) {
            mask[e] = a.mask[blk * a.n_experts + e];
            start[e] = at + a.base[blk * a.n_experts + e];
        }
        __syncthreads();
        place_block(a, blk, mask, start, a.block_at[blk], n_entries, upto);
        __syncthreads();
    }
}

// -------------------------------------------------------- logits' gradient
struct RouteBackArgs {
    const void *logits;
    void *d_logits;
    int64_t n_tokens, stride, d_stride, cap;
    int n_experts, normalise;
    const int64_t *row_ptr;
    const int32_t *expert;
    const float *weight, *d_weight;
};

constexpr uint32_t NOT_CHOSEN = 0xffffffffu;  // as a weight: a NaN that no arithmetic gives

// A wave a token. Lane l holds experts l, l + 64, ...; the entries' gradients (and
// weights) reach their lanes through LDS. Bound by the latency of three dependent
// loads: 16384 tokens, 256 experts, top_k 8, bf16 10 us (17 MB).
template <typename T, int V>
__global__ __launch_bounds__(256) void k_route_backward(RouteBackArgs a) {
    __shared__ float grad[4][V * 64], prob[4][V * 64];
    const int lane = threadIdx.x & 63, w = threadIdx.x / 64;
    for (int64_t t = blockIdx.x * 4ll + w; t < a.n_tokens; t += gridDim.x * 4ll) {
        T l[V];  // (on their way while the row's entries are looked up)
        if (!a.normalise) {
            const T *row = static_cast<const T *>(a.logits) + t * a.stride;
#pragma unroll
            for (int j = 0; j < V; ++j) l[j] = row[j * 64 + lane < a.n_experts ? j * 64 + lane : 0];
        }
        int64_t b = a.row_ptr[t], f = a.row_ptr[t + 1];
        b = b < 0 ? 0 : b > a.cap ? a.cap : b;
        f = f < b ? b : f > a.cap ? a.cap : f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            grad[w][j * 64 + lane] = 0.f;
            if (a.normalise) prob[w][j * 64 + lane] = __uint_as_float(NOT_CHOSEN);
        }
        wave_lds_fence();
        float dot = 0.f;
        for (int64_t i = b + lane; i < f; i += 64) {
            const uint32_t e = (uint32_t)a.expert[i];
            const float p = a.weight[i], g = a.d_weight[i];
            if (e < (uint32_t)a.n_experts) {
                grad[w][e] = g;
                if (a.normalise) prob[w][e] = p;
                dot += p * g;
            }
        }
        wave_lds_fence();
        dot = wave_sum(dot);
        float p[V];
        bool there[V];  // the logit has a part in the softmax: the others' gradient is zero whatever the sum holds
        if (a.normalise) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                p[j] = prob[w][j * 64 + lane];
                there[j] = __float_as_uint(p[j]) != NOT_CHOSEN;
            }
        } else {
            uint32_t key[V], m = 0;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                key[j] = j * 64 + lane < a.n_experts ? order_key(l[j]) : 0u;
                m = m > key[j] ? m : key[j];
            }
            const float top = key_value<T>(wave_max(m));
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                p[j] = key[j] ? exp_neg(key_value<T>(key[j]) - top) : 0.f;
                sum += p[j];
            }
            const float scale = 1.f / wave_sum(sum);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                p[j] *= scale;
                there[j] = key[j] != 0;
            }
        }
        T *out = static_cast<T *>(a.d_logits) + t * a.d_stride;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int e = j * 64 + lane;
            if (e < a.n_experts) out[e] = there[j] ? (T)(p[j] * (grad[w][e] - dot)) : (T)0.f;
        }
        wave_lds_fence();
    }
}

// ------------------------------------------------------------------ combine
struct CombineArgs {
    const int64_t *row_ptr;
    const int32_t *slot;
    const float *weight;
    int64_t n_tokens, n_entries, n_y, n;
    const void *y, *out;  // (out: the sum, or its gradient)
    int64_t ys, os;
    void *result;         // the sum, or the gradient of y
    int64_t rs;
    float *d_weight;
    int64_t per;          // entries a row is expected to have
};

constexpr int LANE_N = 8, CHUNK = LANE_N * GM_WAVE;  // columns of a lane, of a wave's step

template <typename T>
GM_DEV void store_f32(T *p, int valid, const float (&v)[LANE_N]) {
    if (valid >= LANE_N) {
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
        for (int i = 0; i < LANE_N; ++i)
            if (i < valid) p[i] = (T)v[i];
    }
}

GM_DEV void entry_range(const CombineArgs &a, int64_t t, int64_t &b, int64_t &f) {
    b = a.row_ptr[t];
    f = a.row_ptr[t + 1];
    b = b < 0 ? 0 : b > a.n_entries ? a.n_entries : b;
    f = f < b ? b : f > a.n_entries ? a.n_entries : f;
}

GM_DEV int64_t wave_number() {
    return __builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64)) + (int64_t)blockIdx.x * (blockDim.x / 64);
}

// A wave: one token's CHUNK columns. Bound by its bytes: 8192 tokens of 4 rows of
// 4096 bf16 78 us, 4.3 TB/s (two entries' rows at once gained nothing: 83 us).
template <typename T>
__global__ __launch_bounds__(256) void k_combine(CombineArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t chunks = (a.n + CHUNK - 1) / CHUNK;
    for (int64_t u = wave_number(); u < a.n_tokens * chunks; u += (int64_t)gridDim.x * 4) {
        const int64_t t = u / chunks, c0 = (u - t * chunks) * CHUNK + lane * LANE_N;
        const int valid = a.n - c0 >= LANE_N ? LANE_N : a.n > c0 ? (int)(a.n - c0) : 0;
        int64_t b, f;
        entry_range(a, t, b, f);
        float s[LANE_N] = {};
        for (int64_t i = b; i < f; ++i) {
            const int64_t r = a.slot[i];
            if (r < 0 || r >= a.n_y) continue;
            const float w = a.weight ? a.weight[i] : 1.f;
            float v[LANE_N];
            load_f32x8(static_cast<const T *>(a.y) + r * a.ys + c0, valid, v);
#pragma unroll
            for (int k = 0; k < LANE_N; ++k) s[k] += w * v[k];
        }
        store_f32(static_cast<T *>(a.result) + t * a.rs + c0, valid, s);
    }
}

// A wave: one entry's row of Y with its token's row of the sum's gradient, read
// once from memory and top_k - 1 times from L2. The same sizes: 115-120 us, 5.1 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void k_combine_backward(CombineArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t first = wave_number(), step = (int64_t)gridDim.x * 4;
    for (int64_t u = first; u < a.n_tokens * a.per; u += step) {
        const int64_t t = u / a.per;
        int64_t b, f;
        entry_range(a, t, b, f);
        const T *d_out = static_cast<const T *>(a.out) + t * a.os;
        for (int64_t i = b + (u - t * a.per); i < f; i += a.per) {
            const int64_t r = a.slot[i];
            const bool there = r >= 0 && r < a.n_y;
            const float w = a.weight ? a.weight[i] : 1.f;
            float dot = 0.f;
            for (int64_t c0 = lane * LANE_N; there && c0 < a.n; c0 += CHUNK) {
                const int valid = a.n - c0 >= LANE_N ? LANE_N : (int)(a.n - c0);
                float d[LANE_N], v[LANE_N];
                load_f32x8(d_out + c0, valid, d);
                if (a.d_weight) {
                    load_f32x8(static_cast<const T *>(a.y) + r * a.ys + c0, valid, v);
#pragma unroll
                    for (int k = 0; k < LANE_N; ++k) dot += v[k] * d[k];
                }
                if (a.result) {
#pragma unroll
                    for (int k = 0; k < LANE_N; ++k) v[k] = w * d[k];
                    store_f32(static_cast<T *>(a.result) + r * a.rs + c0, valid, v);
                }
            }
            if (a.d_weight) {
                dot = wave_sum(dot);
                if (lane == 0) a.d_weight[i] = dot;
            }
        }
    }
    int64_t n = a.row_ptr[a.n_tokens];
    n = n < 0 ? 0 : n;
    if (a.d_weight)
        for (int64_t i = n + first * 64 + lane; i < a.n_entries; i += step * 64) a.d_weight[i] = 0.f;
    if (a.result) {
        const float z[LANE_N] = {};
        for (int64_t r = n + first; r < a.n_y; r += step)
            for (int64_t c0 = lane * LANE_N; c0 < a.n; c0 += CHUNK)
                store_f32(static_cast<T *>(a.result) + r * a.rs + c0, a.n - c0 >= LANE_N ? LANE_N : (int)(a.n - c0), z);
    }
}

// ------------------------------------------------------------------ host side
template <class F>
void with_float(int32_t type, F &&f) {
    if (type == GMAGNUS_DATA_BF16)
        f(__bf16{});
    else if (type == GMAGNUS_DATA_FP16)
        f(_Float16{});
    else
        f(float{});
}

// f(T{}, V{}): the logits' type, and how many of a row's e experts a lane holds.
template <class F>
void with_logits(int32_t type, int64_t e, F &&f) {
    with_float(type, [&](auto v) {
        if (e <= 64)
            f(v, std::integral_constant<int, 1>{});
        else if (e <= 128)
            f(v, std::integral_constant<int, 2>{});
        else if (e <= 256)
            f(v, std::integral_constant<int, 4>{});
        else if (e <= 512)
            f(v, std::integral_constant<int, 8>{});
        else
            f(v, std::integral_constant<int, 16>{});
    });
}

struct RouteLayout {
    int64_t n_blocks, mask, base, total, block_n, block_at, count, list_e, list_w, bytes;
    RouteLayout(int64_t t, int64_t e, int64_t k) {
        int64_t at = 0;
        auto take = [&](int64_t n) {
            const int64_t here = at;
            at += (n + 255) / 256 * 256;
            return here;
        };
        n_blocks = (t + TOK - 1) / TOK;
        const bool small = t <= TOK;  // one work group: lists only
        mask = take(small ? 0 : n_blocks * e * 4);
        base = take(small ? 0 : n_blocks * e * 4);
        total = take(small ? 0 : e * 4);
        block_n = take(small ? 0 : n_blocks * 4);
        block_at = take(small ? 0 : (n_blocks + 1) * 8);
        count = take(t * 4);
        list_e = take(t * k * 2);
        list_w = take(t * k * 4);
        bytes = at;
    }
};

bool route_sizes_ok(int64_t t, int64_t e, int64_t k) {
    return t >= 0 && e >= 1 && e <= MAX_EXPERTS && k >= 1 && k <= e && t < INT32_MAX / k;
}

void check_route(const gmagnus_dense_t *logits, int64_t top_k, int32_t normalise, const gmagnus_routing_t *r) {
    GM_REQUIRE(logits && r, GMAGNUS_ERROR_INVALID_VALUE, "NULL logits or routing");
    const int64_t t = logits->n_rows, e = logits->n_cols;
    GM_REQUIRE(t >= 0 && e >= 1 && top_k >= 1 && top_k <= e, GMAGNUS_ERROR_INVALID_VALUE,
               "top_k must lie in 1 .. number of experts");
    GM_REQUIRE(normalise == 0 || normalise == 1, GMAGNUS_ERROR_INVALID_VALUE, "normalise must be 0 or 1");
    GM_REQUIRE(e <= MAX_EXPERTS, GMAGNUS_ERROR_UNSUPPORTED, "more than 1024 experts");
    GM_REQUIRE(route_sizes_ok(t, e, top_k), GMAGNUS_ERROR_UNSUPPORTED, "2^31 - 1 entries or more");
    check_dense(logits, "logits", t, e);
    GM_REQUIRE(logits->data_type != GMAGNUS_DATA_FP8_E4M3, GMAGNUS_ERROR_INVALID_VALUE, "logits must be fp32, bf16 or fp16");
}

}  // namespace
}  // namespace gm

using namespace gm;

extern "C" int64_t gmagnus_route_workspace_bytes(int64_t n_tokens, int64_t n_experts, int64_t top_k) {
    return route_sizes_ok(n_tokens, n_experts, top_k) ? RouteLayout(n_tokens, n_experts, top_k).bytes : 0;
}

extern "C" gmagnus_status_t gmagnus_route(const gmagnus_dense_t *logits, int64_t top_k, int32_t normalise,
                                          const gmagnus_routing_t *out, void *workspace, int64_t workspace_bytes,
                                          void *hip_stream) {
    return guarded([&] {
        check_route(logits, top_k, normalise, out);
        const int64_t t = logits->n_rows, e = logits->n_cols;
        GM_REQUIRE(out->row_ptr && out->group_ptr, GMAGNUS_ERROR_INVALID_VALUE, "routing: NULL row_ptr or group_ptr");
        GM_REQUIRE(t == 0 || (out->expert && out->weight && out->token && out->slot && out->group_weight),
                   GMAGNUS_ERROR_INVALID_VALUE, "routing: NULL array");
        hipStream_t s = (hipStream_t)hip_stream;
        if (t == 0) {
            fill<int64_t>(out->row_ptr, 0, 1, s);
            fill<int64_t>(out->group_ptr, 0, e + 1, s);
            return;
        }
        const RouteLayout l(t, e, top_k);
        GM_REQUIRE(workspace && workspace_bytes >= l.bytes, GMAGNUS_ERROR_INVALID_VALUE,
                   "workspace below gmagnus_route_workspace_bytes");
        GM_REQUIRE((uintptr_t)workspace % 16 == 0, GMAGNUS_ERROR_INVALID_VALUE, "workspace is not 16-byte aligned");
        char *w = static_cast<char *>(workspace);
        const RouteArgs a{logits->data, t, logits->row_stride, (int)e, (int)top_k, normalise, l.n_blocks, *out,
                          (uint32_t *)(w + l.mask), (int32_t *)(w + l.base), (int32_t *)(w + l.total),
                          (int32_t *)(w + l.block_n), (int64_t *)(w + l.block_at), (int32_t *)(w + l.count),
                          (uint16_t *)(w + l.list_e), (float *)(w + l.list_w)};
        with_logits(logits->data_type, e, [&](auto v, auto per_lane) {
            using T = decltype(v);
            constexpr int V = decltype(per_lane)::value;
            if (l.n_blocks == 1) {
                hipLaunchKernelGGL((k_route_small<T, V>), dim3(1), dim3(ROUTE_T), 0, s, a);
                return;
            }
            const dim3 grid(grid_for(l.n_blocks, 1, 1 << 20));
            hipLaunchKernelGGL((k_route_select<T, V>), grid, dim3(ROUTE_T), 0, s, a);
            hipLaunchKernelGGL(k_route_scan, dim3((unsigned)((e + SCAN_E - 1) / SCAN_E + 1)), dim3(ROUTE_T), 0, s, a);
            hipLaunchKernelGGL(k_route_place, grid, dim3(ROUTE_T), 0, s, a);
        });
        GM_CHECK_LAUNCH();
    });
}

extern "C" gmagnus_status_t gmagnus_route_backward(const gmagnus_dense_t *logits, int64_t top_k, int32_t normalise,
                                                   const gmagnus_routing_t *routing, const float *d_weight,
                                                   const gmagnus_dense_t *d_logits, void *hip_stream) {
    return guarded([&] {
        check_route(logits, top_k, normalise, routing);
        const int64_t t = logits->n_rows, e = logits->n_cols;
        check_dense(d_logits, "d_logits", t, e);
        GM_REQUIRE(d_logits->data_type == logits->data_type, GMAGNUS_ERROR_INVALID_VALUE,
                   "d_logits must have the type of logits");
        if (t == 0) return;
        GM_REQUIRE(routing->row_ptr && routing->expert && routing->weight && d_weight, GMAGNUS_ERROR_INVALID_VALUE,
                   "routing: NULL row_ptr, expert, weight or d_weight");
        const RouteBackArgs a{logits->data, d_logits->data, t, logits->row_stride, d_logits->row_stride, t * top_k,
                              (int)e, normalise, routing->row_ptr, routing->expert, routing->weight, d_weight};
        hipStream_t s = (hipStream_t)hip_stream;
        const dim3 grid(grid_for(t, 4, 1 << 16));
        with_logits(logits->data_type, e, [&](auto v, auto per_lane) {
            hipLaunchKernelGGL((k_route_backward<decltype(v), decltype(per_lane)::value>), grid, dim3(256), 0, s, a);
        });
        GM_CHECK_LAUNCH();
    });
}

namespace {

// Checks shared by the sum and its gradients; OUT is the sum or its gradient.
void check_combine(const int64_t *row_ptr, const int32_t *slot, int64_t n_entries, const gmagnus_dense_t *OUT,
                   const char *name) {
    GM_REQUIRE(OUT != nullptr, GMAGNUS_ERROR_INVALID_VALUE, std::string("NULL ") + name);
    GM_REQUIRE(OUT->n_rows >= 0 && OUT->n_cols >= 1 && n_entries >= 0, GMAGNUS_ERROR_INVALID_VALUE,
               "negative rows or entries, or no columns");
    GM_REQUIRE(OUT->n_rows < INT32_MAX && OUT->n_cols < INT32_MAX && n_entries < INT32_MAX, GMAGNUS_ERROR_UNSUPPORTED,
               "rows, columns or entries beyond 2^31 - 2");
    check_dense(OUT, name, OUT->n_rows, OUT->n_cols);
    GM_REQUIRE(OUT->data_type != GMAGNUS_DATA_FP8_E4M3, GMAGNUS_ERROR_INVALID_VALUE,
               std::string(name) + " must be fp32, bf16 or fp16");
    GM_REQUIRE(row_ptr != nullptr, GMAGNUS_ERROR_INVALID_VALUE, "NULL row_ptr");
    GM_REQUIRE(slot != nullptr || n_entries == 0, GMAGNUS_ERROR_INVALID_VALUE, "NULL slot");
}

// Y, or the gradient of it: rows of its own, columns and type of `like`.
void check_rows(const gmagnus_dense_t *Y, const char *name, const gmagnus_dense_t *like) {
    GM_REQUIRE(Y != nullptr, GMAGNUS_ERROR_INVALID_VALUE, std::string("NULL ") + name);
    GM_REQUIRE(Y->n_rows >= 0 && Y->n_rows < INT32_MAX, GMAGNUS_ERROR_UNSUPPORTED, std::string(name) + ": rows beyond 2^31 - 2");
    check_dense(Y, name, Y->n_rows, like->n_cols);
    GM_REQUIRE(Y->data_type == like->data_type, GMAGNUS_ERROR_INVALID_VALUE, std::string(name) + " has another type");
}

}  // namespace

extern "C" gmagnus_status_t gmagnus_combine(const int64_t *row_ptr, const int32_t *slot, const float *weight,
                                            int64_t n_entries, const gmagnus_dense_t *Y, const gmagnus_dense_t *OUT,
                                            void *hip_stream) {
    return guarded([&] {
        check_combine(row_ptr, slot, n_entries, OUT, "OUT");
        check_rows(Y, "Y", OUT);
        if (OUT->n_rows == 0) return;
        const CombineArgs a{row_ptr, slot, weight, OUT->n_rows, n_entries, Y->n_rows, OUT->n_cols, Y->data, nullptr,
                            Y->row_stride, 0, OUT->data, OUT->row_stride, nullptr, 0};
        const int64_t waves = a.n_tokens * ((a.n + CHUNK - 1) / CHUNK);
        with_float(OUT->data_type, [&](auto v) {
            hipLaunchKernelGGL(k_combine<decltype(v)>, dim3(grid_for(waves, 4, 1 << 22)), dim3(256), 0,
                               (hipStream_t)hip_stream, a);
        });
        GM_CHECK_LAUNCH();
    });
}

extern "C" gmagnus_status_t gmagnus_combine_backward(const int64_t *row_ptr, const int32_t *slot, const float *weight,
                                                     int64_t n_entries, const gmagnus_dense_t *Y,
                                                     const gmagnus_dense_t *D_OUT, const gmagnus_dense_t *D_Y,
                                                     float *d_weight, void *hip_stream) {
    return guarded([&] {
        check_combine(row_ptr, slot, n_entries, D_OUT, "D_OUT");
        GM_REQUIRE(D_Y || d_weight, GMAGNUS_ERROR_INVALID_VALUE, "neither D_Y nor d_weight is wanted");
        if (d_weight) check_rows(Y, "Y", D_OUT);
        if (D_Y) check_rows(D_Y, "D_Y", D_OUT);
        GM_REQUIRE(!d_weight || !D_Y || Y->n_rows == D_Y->n_rows, GMAGNUS_ERROR_INVALID_VALUE, "Y and D_Y differ in rows");
        const int64_t n_y = D_Y ? D_Y->n_rows : Y->n_rows;
        const int64_t t = D_OUT->n_rows, per = t > 0 ? (n_entries + t - 1) / t : 1;
        const CombineArgs a{row_ptr, slot, weight, t, n_entries, n_y, D_OUT->n_cols, d_weight ? Y->data : nullptr,
                            D_OUT->data, d_weight ? Y->row_stride : 0, D_OUT->row_stride, D_Y ? D_Y->data : nullptr,
                            D_Y ? D_Y->row_stride : 0, d_weight, per > 1 ? per : 1};
        const int64_t waves = t * a.per > n_y ? t * a.per : n_y;
        with_float(D_OUT->data_type, [&](auto v) {
            hipLaunchKernelGGL(k_combine_backward<decltype(v)>, dim3(grid_for(waves, 4, 1 << 22)), dim3(256), 0,
                               (hipStream_t)hip_stream, a);
        });
        GM_CHECK_LAUNCH();
    });
}
