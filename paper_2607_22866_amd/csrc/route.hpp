// The choice of a token's experts from its logits, by one wave.
#pragma once

#include "dense.hpp"

namespace gm {

constexpr int MAX_EXPERTS = 1024;

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

// The choice of one token by one wave: lane l holds experts l, l + 64, ... (V of
// them). chosen[j]: the lanes whose expert is taken, p[j] times the returned scale:
// their weights; n: how many are taken. The top_k-th largest key is found bit by
// bit from the top: a bit stays if at least top_k keys reach it, and once just top_k
// do, those are the choice (16384 tokens, 256 experts, top_k 8: 20 us; taking the
// maximum over the wave top_k times: 37). Keys equal to the last one are taken from
// the lowest expert on. (The whole call for 16384 tokens, bf16, top_k 8, of 256, 512 and
// 1024 experts 29, 42 and 68 us; with the taken experts written in here rather than by the
// caller, which changes how registers are given out, 31.5, 42 and 66.)
template <typename T, int V>
GM_DEV float choose(const T (&l)[V], int n_experts, int top_k, bool normalise, uint64_t (&chosen)[V], float (&p)[V], int &n) {
    const int lane = threadIdx.x & 63;
    uint32_t key[V], best = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        key[j] = j * 64 + lane < n_experts ? order_key(l[j]) : 0u;
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
    n = reach(1);
    uint32_t least = 1;
    if (n > top_k) {
        least = 0;
        for (uint32_t b = 1u << (KEY_BITS<T> - 1); b; b >>= 1) {
            const int m = reach(least | b);
            if (m >= top_k) {
                least |= b;
                n = m;
                if (m == top_k) break;
            }
        }
    }
    // n keys reach `least`; more than top_k only where several equal it
    int spare = n > top_k ? n - top_k : 0;
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
    n = n < top_k ? n : top_k;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        p[j] = key[j] ? exp_neg(key_value<T>(key[j]) - top) : 0.f;
        if (!normalise || (chosen[j] >> lane & 1)) sum += p[j];
    }
    return 1.f / wave_sum(sum);
}

}  // namespace gm
