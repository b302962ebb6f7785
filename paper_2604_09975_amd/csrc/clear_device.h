// Types, wide loads and checks of arguments of the steps in the clear (clear_*.hip).
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/ckks_clear.h"
#include "ckks_internal.h"
#include "clear_extent.h"

namespace ckks {

typedef int64_t i64;
typedef _Float16 f16;
typedef __bf16 bf16;

// N values in one access.  A row of an odd width starts wherever its type allows; global memory takes such an address at
// full width, so there is no second code path for it.
template <class T, int N>
struct Pack {
    T v[N];
};
template <int N, class T>
__device__ __forceinline__ Pack<T, N> load_pack(const T *p) {
    Pack<T, N> r;
    __builtin_memcpy(&r, p, sizeof(r));
    return r;
}
template <int N, class T>
__device__ __forceinline__ void store_pack(T *p, const Pack<T, N> &x) {
    __builtin_memcpy(p, &x, sizeof(x));
}
// The first `n` of N values, zeros behind them.
template <int N, class T>
__device__ __forceinline__ Pack<T, N> load_part(const T *p, int n) {
    if (n >= N) return load_pack<N>(p);
    Pack<T, N> r;
#pragma unroll
    for (int i = 0; i < N; ++i) r.v[i] = i < n ? p[i] : (T)0.0f;
    return r;
}
template <int N, class T>
__device__ __forceinline__ void store_part(T *p, const Pack<T, N> &x, int n) {
    if (n >= N) {
        store_pack<N>(p, x);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < n) p[i] = x.v[i];
}

// ---- host ----
inline bool clear_dtype_ok(u32 d) { return d <= CKKS_CLEAR_BF16; }
inline u32 clear_dtype_bytes(u32 d) { return d == CKKS_CLEAR_F32 ? 4 : 2; }

// What append and attend ask of the pages and the batch alike.
inline int check_cache(const char *who, const ckks_clear_pages_t &g, const ckks_clear_batch_t &b) {
    if (!clear_dtype_ok(g.dtype) || !g.head_dim || g.head_dim % 8 || g.head_dim > 256 || !g.kv_heads || g.kv_heads > 1u << 16 || !g.page_size) {
        set_error("%s: pages of type %u, %u rows, %u heads of %u entries", who, g.dtype, g.page_size, g.kv_heads, g.head_dim);
        return CKKS_E_INVAL;
    }
    const auto near = [&](const i64 *st) { return st[0] >= 0 && st[0] < 1ll << 32 && st[1] >= 0 && st[2] >= 0 && st[2] < 1ll << 31 && (u64)st[2] * g.page_size < 1u << 31; };
    if (!near(g.k_stride) || !near(g.v_stride)) {
        set_error("%s: strides of the pages (a page's below 2^32 entries, a page itself below 2^31)", who);
        return CKKS_E_INVAL;
    }
    if (b.n_tokens >= 1u << 31 || b.n_seq >= 1u << 31 || (u64)b.table_width * g.page_size >= 1u << 31) {
        set_error("%s: %u tokens, %u sequences of up to %u pages of %u", who, b.n_tokens, b.n_seq, b.table_width, g.page_size);
        return CKKS_E_INVAL;
    }
    if (b.n_tokens && !b.n_seq) {
        set_error("%s: %u tokens of no sequence", who, b.n_tokens);
        return CKKS_E_INVAL;
    }
    if (b.n_tokens && (!b.d_q_start || !b.d_kv_len || (b.table_width && !b.d_page_table) || (g.n_pages && (!g.d_k || !g.d_v)))) {
        set_error("%s: null argument", who);
        return CKKS_E_INVAL;
    }
    return CKKS_OK;
}

}  // namespace ckks
