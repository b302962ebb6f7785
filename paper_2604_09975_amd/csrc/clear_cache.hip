// New keys and values into their pages, keys and queries rotated on the way.  Every array is read and written once: bound by
// memory, by the launch for a few tokens.  A thread moves V entries (rotated by halves: V of each half), a head's threads lie side
// by side, and all three arrays are moved by one launch.  About 23000 tokens of 32 query and 8 kv heads of 128, bf16, rotated:
// 568 MB in 116 to 125 us, 4.5 to 4.9 TB/s, what a large copy reaches (pairs side by side 139); 32 single tokens of 12 heads 3.7 us.
#include <algorithm>
#include <numeric>

#include "clear_device.h"

namespace ckks {

struct AppendArgs {
    const void *k, *v, *q;
    void *pk, *pv, *qo;
    i64 ks[2], vs[2], qs[2], qos[2], pks[3], pvs[3], ts;
    const float *cos, *sin;
    const int32_t *positions, *q_start, *kv_len, *table;
    u32 n_seq, n_tokens, t0, t1, n_pages, page_size, table_width, kv_heads, heads, head_dim, rot, n_pos;  // a launch moves tokens t0 .. t1-1
    u32 rot_items, items, per_token;  // items of a head that are rotated, all of them, those of a token
};

constexpr u32 STARTS = 1024;  // sequences whose starts fit the block's copy

// Sequence of a token: the largest b < n_seq with start(b) <= t.
template <class F>
__device__ __forceinline__ u32 find_seq(u32 t, u32 n_seq, F start) {
    u32 lo = 0, hi = n_seq;
    while (hi - lo > 1) {
        const u32 mid = (lo + hi) >> 1;
        if (start(mid) <= (int64_t)t)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

template <class T, int V, bool INTERLEAVED>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
    __shared__ int32_t starts[STARTS];
    const bool staged = a.n_seq <= STARTS;
    if (staged) {
        for (u32 i = threadIdx.x; i < a.n_seq; i += 256) starts[i] = a.q_start[i];
        __syncthreads();
    }
    const u32 at = blockIdx.x * 256 + threadIdx.x, t = a.t0 + at / a.per_token, rest = at % a.per_token;
    if (t >= a.t1) return;
    const u32 head = rest / a.items, item = rest % a.items;  // keys, values, queries
    const u32 b = staged ? find_seq(t, a.n_seq, [&](u32 i) { return (int64_t)starts[i]; })
                         : find_seq(t, a.n_seq, [&](u32 i) { return (int64_t)a.q_start[i]; });
    const i64 end = min((i64)a.q_start[b + 1], (i64)a.n_tokens);
    const i64 kv = min((i64)a.kv_len[b], (i64)a.table_width * a.page_size);
    // a token outside the sequences' rows has no position
    const i64 pos = (i64)t >= (i64)a.q_start[b] && (i64)t < end ? kv - (end - (i64)t) : -1;
    const T *src;
    T *dst;
    bool turn = item < a.rot_items;
    if (head < 2 * a.kv_heads) {
        if (pos < 0) return;
        const int32_t page = a.table[(i64)b * a.ts + (u32)pos / a.page_size];
        if ((u32)page >= a.n_pages) return;
        const u32 row = (u32)pos % a.page_size;
        if (head < a.kv_heads) {
            src = (const T *)a.k + (i64)t * a.ks[0] + head * a.ks[1];
            dst = (T *)a.pk + page * a.pks[0] + head * a.pks[1] + row * a.pks[2];
        } else {
            const u32 h = head - a.kv_heads;
            src = (const T *)a.v + (i64)t * a.vs[0] + h * a.vs[1];
            dst = (T *)a.pv + page * a.pvs[0] + h * a.pvs[1] + row * a.pvs[2];
            turn = false;
        }
    } else {
        const u32 h = head - 2 * a.kv_heads;
        src = (const T *)a.q + (i64)t * a.qs[0] + h * a.qs[1];
        dst = (T *)a.qo + (i64)t * a.qos[0] + h * a.qos[1];
    }
    const u32 half = a.rot / 2;
    // the items of a head: rotated ones first (by halves: V entries of each half), then the others; values keep to the
    // same places
    if (INTERLEAVED || item >= a.rot_items) {
        const u32 c = INTERLEAVED || item < a.rot_items ? item * V : a.rot + (item - a.rot_items) * V;
        Pack<T, V> x = load_pack<V>(src + c);
        if (INTERLEAVED && turn) {
            const i64 p = a.positions ? (i64)a.positions[t] : pos;
            if (p < 0 || p >= a.n_pos) {
#pragma unroll
                for (int i = 0; i < V; ++i) x.v[i] = (T)__builtin_nanf("");
            } else {
#pragma unroll
                for (int i = 0; i + 1 < V; i += 2) {
                    const float cs = a.cos[p * half + (c + i) / 2], sn = a.sin[p * half + (c + i) / 2];
                    const float x1 = (float)x.v[i], x2 = (float)x.v[i + 1];
                    x.v[i] = (T)(x1 * cs - x2 * sn);
                    x.v[i + 1] = (T)(x2 * cs + x1 * sn);
                }
            }
        }
        store_pack<V>(dst + c, x);
        return;
    }
    const u32 c = item * V;
    Pack<T, V> x1 = load_pack<V>(src + c), x2 = load_pack<V>(src + half + c);
    if (turn) {
        const i64 p = a.positions ? (i64)a.positions[t] : pos;
        if (p < 0 || p >= a.n_pos) {
#pragma unroll
            for (int i = 0; i < V; ++i) x1.v[i] = x2.v[i] = (T)__builtin_nanf("");
        } else {
            const Pack<float, V> cs = load_pack<V>(a.cos + p * half + c), sn = load_pack<V>(a.sin + p * half + c);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float u = (float)x1.v[i], w = (float)x2.v[i];
                x1.v[i] = (T)(u * cs.v[i] - w * sn.v[i]);
                x2.v[i] = (T)(w * cs.v[i] + u * sn.v[i]);
            }
        }
    }
    store_pack<V>(dst + c, x1);
    store_pack<V>(dst + half + c, x2);
}

template <class T, int V, bool INTERLEAVED>
static int launch_append(AppendArgs a, hipStream_t st) {
    a.rot_items = INTERLEAVED ? a.rot / V : a.rot / 2 / V;
    a.items = a.rot_items + (a.head_dim - a.rot) / V;
    a.per_token = (2 * a.kv_heads + (a.q ? a.heads : 0)) * a.items;
    const u32 most = std::max<u32>((1u << 30) / a.per_token, 1);  // tokens of a launch
    for (a.t0 = 0; a.t0 < a.n_tokens;) {
        const u32 n = std::min(a.n_tokens - a.t0, most);
        a.t1 = a.t0 + n;
        const dim3 grid((u32)(((u64)n * a.per_token + 255) / 256));
        hipLaunchKernelGGL((append_kernel<T, V, INTERLEAVED>), grid, dim3(256), 0, st, a);
        CKKS_LAUNCH_CHECK("append_kernel");
        a.t0 = a.t1;
    }
    return CKKS_OK;
}

// The widest access (16 bytes at most) that divides what a thread moves.
template <class T>
static int launch_append(const AppendArgs &a, bool interleaved, hipStream_t st) {
    const u32 g = std::gcd(std::gcd(interleaved ? a.rot : a.rot / 2, a.head_dim - a.rot), 16 / (u32)sizeof(T));
    if (interleaved) {  // rot and head_dim are even
        if constexpr (sizeof(T) == 2)
            if (g == 8) return launch_append<T, 8, true>(a, st);
        return g == 4 ? launch_append<T, 4, true>(a, st) : launch_append<T, 2, true>(a, st);
    }
    if constexpr (sizeof(T) == 2)
        if (g == 8) return launch_append<T, 8, false>(a, st);
    return g == 4 ? launch_append<T, 4, false>(a, st) : g == 2 ? launch_append<T, 2, false>(a, st) : launch_append<T, 1, false>(a, st);
}

}  // namespace ckks

using namespace ckks;

extern "C" int ckks_clear_cache_append(const ckks_clear_append_t *p, void *stream) {
    const char *who = "ckks_clear_cache_append";
    if (!p) {
        set_error("%s: null argument", who);
        return CKKS_E_INVAL;
    }
    const ckks_clear_pages_t &g = p->pages;
    const ckks_clear_batch_t &b = p->batch;
    if (int rc = check_cache(who, g, b)) return rc;
    if (!b.n_tokens || !b.n_seq) return CKKS_OK;
    if (!p->d_new_k || !p->d_new_v || (p->d_q && (!p->d_q_out || !p->heads))) {
        set_error("%s: null argument", who);
        return CKKS_E_INVAL;
    }
    if (p->rot % 2 || p->rot > g.head_dim || (p->rot && (!p->d_cos || !p->d_sin)) || (p->flags & ~CKKS_CLEAR_INTERLEAVED)) {
        set_error("%s: rotation of %u of %u entries (flags %u)", who, p->rot, g.head_dim, p->flags);
        return CKKS_E_INVAL;
    }
    const u32 heads = p->d_q ? p->heads : 0;
    if (heads > 1u << 16) {
        set_error("%s: %u heads", who, heads);
        return CKKS_E_INVAL;
    }
    const u32 e = clear_dtype_bytes(g.dtype);
    const Extent out[3] = {extent(g.d_k, e, {{g.n_pages, g.k_stride[0]}, {g.kv_heads, g.k_stride[1]}, {g.page_size, g.k_stride[2]}, {g.head_dim, 1}}),
                           extent(g.d_v, e, {{g.n_pages, g.v_stride[0]}, {g.kv_heads, g.v_stride[1]}, {g.page_size, g.v_stride[2]}, {g.head_dim, 1}}),
                           extent(p->d_q_out, e, {{heads ? b.n_tokens : 0, p->q_out_stride[0]}, {heads, p->q_out_stride[1]}, {g.head_dim, 1}})};
    const Extent in[8] = {extent(p->d_new_k, e, {{b.n_tokens, p->new_k_stride[0]}, {g.kv_heads, p->new_k_stride[1]}, {g.head_dim, 1}}),
                          extent(p->d_new_v, e, {{b.n_tokens, p->new_v_stride[0]}, {g.kv_heads, p->new_v_stride[1]}, {g.head_dim, 1}}),
                          extent(p->d_cos, 4, {{p->rot ? p->n_pos : 0, p->rot / 2}, {p->rot / 2, 1}}),
                          extent(p->d_sin, 4, {{p->rot ? p->n_pos : 0, p->rot / 2}, {p->rot / 2, 1}}),
                          extent(b.d_q_start, 4, {{b.n_seq + 1, 1}}),
                          extent(b.d_kv_len, 4, {{b.n_seq, 1}}),
                          extent(b.d_page_table, 4, {{b.n_seq, b.table_stride}, {b.table_width, 1}}),
                          extent(p->d_q, e, {{heads ? b.n_tokens : 0, p->q_stride[0]}, {heads, p->q_stride[1]}, {g.head_dim, 1}})};
    const Extent places = extent(p->d_positions, 4, {{p->d_positions ? b.n_tokens : 0, 1}});
    const auto runs = [&](const void *at, u32 n, const int64_t *st) { return Runs{at, g.head_dim * e, 2, {{b.n_tokens, st[0] * e}, {n, st[1] * e}}}; };
    const Runs rows[3] = {runs(p->d_new_k, g.kv_heads, p->new_k_stride), runs(p->d_new_v, g.kv_heads, p->new_v_stride), runs(p->d_q_out, heads, p->q_out_stride)};
    const bool in_place = p->d_q == p->d_q_out && p->q_stride[0] == p->q_out_stride[0] && p->q_stride[1] == p->q_out_stride[1];
    const auto cells = [&](const void *at, const int64_t *st) {
        return Runs{at, g.head_dim * e, 3, {{g.n_pages, st[0] * e}, {g.kv_heads, st[1] * e}, {g.page_size, st[2] * e}}};
    };
    bool bad = overlap(out[2], out[0]) || overlap(out[2], out[1]);
    // keys and values may lie in one array, page by page, but not in the same places of it
    const Runs keys = cells(g.d_k, g.k_stride), values = cells(g.d_v, g.v_stride);
    if (overlap(out[0], out[1])) bad |= share(keys, values);
    for (int o = 0; o < 3; ++o) {
        bad |= overlap(out[o], places);
        // the extents of new keys, values and queries interleave where they are columns of one array: with q_out in place of q
        // keys and values are asked for entries that they share with it
        for (int i = 0; i < 8; ++i)
            if (overlap(out[o], in[i])) bad |= !(o == 2 && in_place) || (i < 2 ? share(rows[2], rows[i]) : i != 7);
    }
    if (bad) {
        set_error("%s: an output overlaps another array", who);
        return CKKS_E_INVAL;
    }
    if (share_within(keys) || share_within(values) || (heads && share_within(rows[2]))) {
        set_error("%s: rows of an output overlap", who);
        return CKKS_E_INVAL;
    }
    AppendArgs a{};
    a.k = p->d_new_k, a.v = p->d_new_v, a.q = p->d_q, a.pk = g.d_k, a.pv = g.d_v, a.qo = p->d_q_out;
    for (int i = 0; i < 2; ++i)
        a.ks[i] = p->new_k_stride[i], a.vs[i] = p->new_v_stride[i], a.qs[i] = p->q_stride[i], a.qos[i] = p->q_out_stride[i];
    for (int i = 0; i < 3; ++i) a.pks[i] = g.k_stride[i], a.pvs[i] = g.v_stride[i];
    a.ts = b.table_stride, a.cos = p->d_cos, a.sin = p->d_sin, a.positions = p->d_positions;
    a.q_start = b.d_q_start, a.kv_len = b.d_kv_len, a.table = b.d_page_table;
    a.n_seq = b.n_seq, a.n_tokens = b.n_tokens, a.n_pages = g.n_pages, a.page_size = g.page_size, a.table_width = b.table_width;
    a.kv_heads = g.kv_heads, a.heads = heads, a.head_dim = g.head_dim, a.rot = p->rot, a.n_pos = p->n_pos;
    const bool il = p->flags & CKKS_CLEAR_INTERLEAVED;
    hipStream_t st = (hipStream_t)stream;
    return g.dtype == CKKS_CLEAR_F32   ? launch_append<float>(a, il, st)
           : g.dtype == CKKS_CLEAR_F16 ? launch_append<f16>(a, il, st)
                                       : launch_append<bf16>(a, il, st);
}
