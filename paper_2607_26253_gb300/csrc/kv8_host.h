// What the entry points over the 8-bit cache check, and how they pick kernels by its shape.
#pragma once
#include <cstdint>
#include <type_traits>

#include "kv8.cuh"

namespace sara {

inline bool misaligned(const void *p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

// (a batch of no sequences has no table)
inline bool cache_ok(const sara_kv8_cache *c, int n_seq) {
    return c && c->codes && c->scales && (c->table || n_seq == 0) && c->n_blocks >= 1 && c->max_blocks >= 1 &&
           c->max_blocks <= INT32_MAX / SARA_KV8_PAGE && c->table_stride >= c->max_blocks && c->n_kv_heads >= 1 &&
           c->n_kv_heads <= 65536 && (c->head_dim == 32 || c->head_dim == 64 || c->head_dim == 128) &&
           (c->format == SARA_KV8_E4M3 || c->format == SARA_KV8_INT8) && !misaligned(c->codes, 16) && !misaligned(c->scales, 4);
}

inline Kv8Cache device_cache(const sara_kv8_cache *c) {
    return {c->codes, c->scales, c->table, c->table_stride, c->n_blocks, c->max_blocks, c->n_kv_heads};
}

// f.template operator()<head_dim, format>()
template <typename F>
void by_shape(const sara_kv8_cache *c, F f) {
    auto with = [&](auto hd) {
        if (c->format == SARA_KV8_E4M3) f(hd, std::integral_constant<int, SARA_KV8_E4M3>());
        else f(hd, std::integral_constant<int, SARA_KV8_INT8>());
    };
    if (c->head_dim == 32) with(std::integral_constant<int, 32>());
    else if (c->head_dim == 64) with(std::integral_constant<int, 64>());
    else with(std::integral_constant<int, 128>());
}

}  // namespace sara
