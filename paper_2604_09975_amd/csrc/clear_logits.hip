// Rules on logits: history penalties, biases, mask.  A block takes a stretch of one row's vocabulary.  It tallies in LDS what the
// row's history and bias list say about the tokens of that stretch, works out the few logits that they change, streams the stretch
// through the mask, and then writes the changed ones over it.  The tallies are whole numbers, and of several biases the largest
// index counts: no order shows in a result.
// Bound by memory where there is no history (256 x 131072 bf16 with a mask 29 us, 4.8 TB/s); with one by the chain of its lookups,
// which a second block on the CU hides in part (the same with 4000 tokens a row 52 us, with up to 4000 and 100 biases 54 to 56), and by the launch for a
// row (50257 f32, 5.4 us).  Measured and dropped: a launch for the masked copy and one that tallies a row's history by hashing
// (64.9 us with 4000 tokens a row, 41.8 with 1000, where this takes 51.2 and 43.9; 256 x 131072 f32 110 and 71.6 against 75 and 60).
#include <algorithm>

#include "clear_device.h"

namespace ckks {

// Tally of a token: it is in the prompt; below this how often it was generated.
constexpr u32 SEEN = 1u << 31, COUNT = SEEN - 1;
constexpr u32 LISTED = 512, PLACES = 2 * LISTED;  // biases of a stretch that a table in LDS holds, in twice as many places

struct LogitsArgs {
    const void *logits;
    void *out;
    const int32_t *tokens, *token_start, *n_prompt;
    const float *repetition, *frequency, *presence;
    const int32_t *bias_ids, *bias_start;
    const float *bias;
    const int32_t *mask;
    i64 ls, os, ms;
    u32 vocab, n_tokens, n_biases, tiles;
};

__device__ __forceinline__ u32 clamp_at(int32_t v, u32 top) { return v < 0 ? 0u : min((u32)v, top); }

// Up to four ids, zeros behind the last.
__device__ __forceinline__ Pack<int32_t, 4> load_ids(const int32_t *p, u32 n) {
    if (n >= 4) return load_pack<4>(p);
    Pack<int32_t, 4> t{};
#pragma unroll
    for (u32 k = 0; k < 3; ++k)
        if (k < n) t.v[k] = p[k];
    return t;
}

// use(token - first, index, k) for the thread's part of the history, ids within the stretch only; `t` holds its first four, which
// come with k = 0 .. 3, the others with k = 4.
template <class F>
__device__ __forceinline__ void each_token(const LogitsArgs &a, u32 h0, u32 h1, Pack<int32_t, 4> t, u32 threads, u32 first, u32 span, F use) {
    u32 i = h0 + 4 * threadIdx.x;
#pragma unroll
    for (u32 k = 0; k < 4; ++k) {
        const u32 c = (u32)t.v[k] - first;
        if (i + k < h1 && c < span) use(c, i + k, k);
    }
    for (i += 4 * threads; i < h1; i += 4 * threads) {
        t = load_ids(a.tokens + i, h1 - i);
#pragma unroll
        for (u32 k = 0; k < 4; ++k) {
            const u32 c = (u32)t.v[k] - first;
            if (i + k < h1 && c < span) use(c, i + k, 4u);
        }
    }
}

// The place of token `c` of the stretch in the table of tokens + 1, found by hashing; the table is at most half full.  (A search of
// the stretch's list by each token took 22 us for 10 rows of 2228 with 83 biases, this takes 6; beyond the table, a row of 50257 with
// a bias for each token takes 270.)
__device__ __forceinline__ u32 bias_place(u32 *table, u32 c) {
    static_assert(PLACES == 1u << (32 - 22), "bits of the hash");
    u32 at = c * 2654435769u >> 22;
    for (;;) {
        const u32 was = atomicCAS(&table[at], 0u, c + 1);
        if (was == 0 || was == c + 1) return at;
        at = (at + 1) % PLACES;
    }
}
// use(token - first, index, k) for the thread's part of the bias list, ids within the stretch only; `id` is the thread's first, which
// comes with k = 0, the others with k = 1.
template <class F>
__device__ __forceinline__ void each_bias(const LogitsArgs &a, u32 b0, u32 b1, int32_t id, u32 threads, u32 first, u32 span, F use) {
    u32 b = b0 + threadIdx.x;
    if (b < b1 && (u32)id - first < span) use((u32)id - first, b, 0u);
    for (b += threads; b < b1; b += threads) {
        const u32 c = (u32)a.bias_ids[b] - first;
        if (c < span) use(c, b, 1u);
    }
}

// THREADS x V x R entries per block.  RULES: there is a history or a bias list.
template <class T, class TO, int THREADS, int R, bool RULES>
__global__ __launch_bounds__(THREADS) void logits_kernel(LogitsArgs a) {
    constexpr int V = 8, SPAN = THREADS * V * R;
    __shared__ __attribute__((aligned(16))) u32 tally[RULES ? SPAN : 4];   // then the changed logits
    __shared__ u32 taken[RULES ? SPAN / 32 : 1], biased[RULES ? SPAN / 32 : 1];  // a bit for each token: worked out; in the bias list
    __shared__ u32 bias_token[RULES ? PLACES : 1], bias_last[RULES ? PLACES : 1];  // the table; largest index in the bias list + 1
    __shared__ u32 n_listed;
    const u32 row = blockIdx.x / a.tiles, first = (blockIdx.x % a.tiles) * SPAN, span = min(a.vocab - first, (u32)SPAN);
    const T *in = (const T *)a.logits + (i64)row * a.ls + first;
    TO *out = (TO *)a.out + (i64)row * a.os + first;
    const int32_t *mask = a.mask ? a.mask + (i64)row * a.ms : nullptr;
    // the stretch is under way while the rules are worked out
    Pack<T, V> x[R];
    u32 bits[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const u32 c = (r * THREADS + threadIdx.x) * V;
        x[r] = load_part<V>(in + c, c < span ? (int)min(span - c, (u32)V) : 0);
        // `first` and c are multiples of 8: a thread's eight bits lie in one byte of the mask
        bits[r] = mask && c < span ? (u32)mask[(first + c) >> 5] >> ((first + c) & 31) : 0xffu;
    }
    u32 h0 = 0, h1 = 0, b0 = 0, b1 = 0;
    Pack<int32_t, 4> t0{};
    int32_t bias_id = 0;
    if (RULES) {
        u32 made = 0;
        if (a.tokens) {
            h0 = clamp_at(a.token_start[row], a.n_tokens);
            h1 = clamp_at(a.token_start[row + 1], a.n_tokens);
            made = a.n_prompt ? h0 + clamp_at(a.n_prompt[row], a.n_tokens) : h0;
        }
        if (a.bias) {
            b0 = clamp_at(a.bias_start[row], a.n_biases);
            b1 = clamp_at(a.bias_start[row + 1], a.n_biases);
        }
        const u32 i0 = h0 + 4 * threadIdx.x;
        if (i0 < h1) t0 = load_ids(a.tokens + i0, h1 - i0);
        const float rep = a.repetition ? a.repetition[row] : 1.0f, freq = a.frequency ? a.frequency[row] : 0.0f,
                    pres = a.presence ? a.presence[row] : 0.0f;
        // ... and so are the first bias and the logits of those tokens
        float bias0 = 0.0f;
        if (b0 + threadIdx.x < b1) {
            bias_id = a.bias_ids[b0 + threadIdx.x];
            bias0 = a.bias[b0 + threadIdx.x];
        }
        // (only those within the stretch, one in eight of a long row: the loads of the others would cost more than the branches)
        float l0[4] = {0, 0, 0, 0}, bias_l = 0.0f;
        u32 m0[4] = {0, 0, 0, 0}, bias_m = 0;
#pragma unroll
        for (u32 k = 0; k < 4; ++k) {
            const u32 c = (u32)t0.v[k] - first;
            if (i0 + k < h1 && c < span) {
                l0[k] = (float)in[c];
                m0[k] = mask ? (u32)mask[(first + c) >> 5] : ~0u;
            }
        }
        if (b0 + threadIdx.x < b1 && (u32)bias_id - first < span) {
            bias_l = (float)in[(u32)bias_id - first];
            bias_m = mask ? (u32)mask[(u32)bias_id >> 5] : ~0u;
        }
        for (u32 k = threadIdx.x; k < SPAN / 4; k += THREADS) ((uint4 *)tally)[k] = make_uint4(0, 0, 0, 0);
        for (u32 k = threadIdx.x; k < SPAN / 32; k += THREADS) taken[k] = biased[k] = 0;
        if (b0 < b1)
            for (u32 k = threadIdx.x; k < PLACES; k += THREADS) bias_token[k] = bias_last[k] = 0;
        if (threadIdx.x == 0) n_listed = 0;
        __syncthreads();
        each_token(a, h0, h1, t0, THREADS, first, span, [&](u32 c, u32 i, u32) {
            if (i < made)
                atomicOr(&tally[c], SEEN);
            else
                atomicAdd(&tally[c], 1u);
        });
        each_bias(a, b0, b1, bias_id, THREADS, first, span, [&](u32 c, u32 b, u32) {
            atomicOr(&biased[c >> 5], 1u << (c & 31));
            if (atomicAdd(&n_listed, 1u) < LISTED) atomicMax(&bias_last[bias_place(bias_token, c)], b + 1);
        });
        __syncthreads();
        // A token with biases is worked out by the thread of its last bias, one without by whoever comes first; the result takes the
        // place of the tally.
        auto take = [&](u32 c) { return !(atomicOr(&taken[c >> 5], 1u << (c & 31)) >> (c & 31) & 1); };
        auto change = [&](u32 c, bool known, float l, u32 m, float bias) {
            if (!known) {
                l = (float)in[c];
                m = mask ? (u32)mask[(first + c) >> 5] : ~0u;
            }
            const u32 t = tally[c], n = t & COUNT;
            if (t) l = l > 0.0f ? l / rep : l * rep;
            l = l - freq * (float)n;
            l = l - (n ? pres : 0.0f);
            l += bias;
            if (!(m >> ((first + c) & 31) & 1)) l = -__builtin_inff();
            tally[c] = __float_as_uint(l);
        };
        each_token(a, h0, h1, t0, THREADS, first, span, [&](u32 c, u32, u32 k) {
            if (!(biased[c >> 5] >> (c & 31) & 1) && take(c)) change(c, k < 4, l0[k & 3], m0[k & 3], -0.0f);
        });
        auto last = [&](u32 c, u32 b, u32 k) {
            take(c);
            change(c, !k, bias_l, bias_m, k ? a.bias[b] : bias0);
        };
        if (n_listed <= LISTED) {
            each_bias(a, b0, b1, bias_id, THREADS, first, span, [&](u32 c, u32 b, u32 k) {
                if (bias_last[bias_place(bias_token, c)] == b + 1) last(c, b, k);
            });
        } else {
            // too many for the table: for PLACES tokens at a time, a place for each
            for (u32 sub = 0; sub < span; sub += PLACES) {
                __syncthreads();
                for (u32 k = threadIdx.x; k < PLACES; k += THREADS) bias_last[k] = 0;
                __syncthreads();
                each_bias(a, b0, b1, bias_id, THREADS, first, span, [&](u32 c, u32 b, u32) {
                    if (c - sub < PLACES) atomicMax(&bias_last[c - sub], b + 1);
                });
                __syncthreads();
                each_bias(a, b0, b1, bias_id, THREADS, first, span, [&](u32 c, u32 b, u32 k) {
                    if (c - sub < PLACES && bias_last[c - sub] == b + 1) last(c, b, k);
                });
            }
        }
        __syncthreads();  // d_out may be d_logits: all that is changed has been read
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const u32 c = (r * THREADS + threadIdx.x) * V;
        if (c >= span) break;
        Pack<TO, V> y;
#pragma unroll
        for (int i = 0; i < V; ++i) y.v[i] = (TO)((bits[r] >> i) & 1 ? (float)x[r].v[i] : -__builtin_inff());
        store_part<V>(out + c, y, (int)min(span - c, (u32)V));
    }
    if (RULES) {
        __threadfence_block();
        __syncthreads();  // the stretch is written: now the changed logits
        auto write = [&](u32 c) {
            if (atomicAnd(&taken[c >> 5], ~(1u << (c & 31))) >> (c & 31) & 1) out[c] = (TO)__uint_as_float(tally[c]);
        };
        each_token(a, h0, h1, t0, THREADS, first, span, [&](u32 c, u32, u32) { write(c); });
        each_bias(a, b0, b1, bias_id, THREADS, first, span, [&](u32 c, u32, u32) { write(c); });
    }
}

template <class T, class TO, int THREADS, int R, bool RULES>
static void launch_logits(LogitsArgs a, u32 rows, hipStream_t st) {
    constexpr u32 span = THREADS * 8 * R;
    a.tiles = (a.vocab + span - 1) / span;
    hipLaunchKernelGGL((logits_kernel<T, TO, THREADS, R, RULES>), dim3(rows * a.tiles), dim3(THREADS), 0, st, a);
}
// Stretches: each block goes through the row's whole history, so long ones go through it less often, short ones put more CUs to
// work.  Measured on one card, history of h tokens a row, us:
//    8 rows of 50257, bf16:    2048 entries  4.8 (h = 100)   5.4 (1000)   7.6 (2000)  25.7 (10000)
//                              8192          5.6             5.9          6.0         11.4
//  256 rows of 131072, f32:    8192         60.6            59.9         63.9        129
//                             16384         72.7            78.1         82.6        129
//  256 rows of 131072, bf16:   8192         49.0            52.3         55.0        114
//                             16384         41.5            43.6         45.8         84.5
// So: 2048 where 8192 would leave CUs without a block, unless the threads of such a block need more than one load each for a
// history; 16384 for 16-bit logits where that fills the CUs (32 bytes a thread either way).  The mask alone: 8192 where it fills the
// CUs (256 x 131072 f32 49.5 us, bf16 29.3; with 2048 50.5 and 29.5, with 16384 62.0 and 29.4), else 2048 (8 x 50257 2.9 us,
// with 8192 3.3).
template <class T, class TO>
static void launch_logits(const LogitsArgs &a, u32 rows, hipStream_t st) {
    const auto blocks = [&](u32 span) { return (u64)rows * ((a.vocab + span - 1) / span); };
    if (!a.tokens && !a.bias) {
        if (blocks(8192) < 256)
            launch_logits<T, TO, 256, 1, false>(a, rows, st);
        else
            launch_logits<T, TO, 1024, 1, false>(a, rows, st);
        return;
    }
    if constexpr (sizeof(T) == 2)
        if (blocks(16384) >= 256) return launch_logits<T, TO, 1024, 2, true>(a, rows, st);
    if (blocks(8192) < 256 && a.n_tokens / rows <= 4 * 256)
        launch_logits<T, TO, 256, 1, true>(a, rows, st);
    else
        launch_logits<T, TO, 1024, 1, true>(a, rows, st);
}

}  // namespace ckks

using namespace ckks;

extern "C" int ckks_clear_logits(const ckks_clear_logits_t *p, void *stream) {
    if (!p || (p->rows && p->vocab && (!p->d_logits || !p->d_out))) {
        set_error("ckks_clear_logits: null argument");
        return CKKS_E_INVAL;
    }
    if (!clear_dtype_ok(p->dtype) || (p->out_dtype != p->dtype && p->out_dtype != CKKS_CLEAR_F32)) {
        set_error("ckks_clear_logits: types %u and %u (out): the output has the logits' type or f32", p->dtype, p->out_dtype);
        return CKKS_E_INVAL;
    }
    if ((p->n_tokens && !p->d_tokens) || (p->n_biases && (!p->d_bias_ids || !p->d_bias))) {
        set_error("ckks_clear_logits: null argument");
        return CKKS_E_INVAL;
    }
    if ((!p->d_token_start && (p->d_tokens || p->d_repetition || p->d_frequency || p->d_presence || p->d_n_prompt)) ||
        (!p->d_bias_start && (p->d_bias || p->d_bias_ids))) {
        set_error("ckks_clear_logits: tokens and penalties need d_token_start, biases d_bias_start");
        return CKKS_E_INVAL;
    }
    if (p->n_tokens >= 1u << 30 || p->n_biases >= 1u << 30 || p->vocab >= 1u << 31 || (u64)p->rows * ((p->vocab + 2047) / 2048) >= 1u << 31) {
        set_error("ckks_clear_logits: %u rows of %u, %u tokens, %u biases exceed one launch", p->rows, p->vocab, p->n_tokens, p->n_biases);
        return CKKS_E_INVAL;
    }
    if (!p->rows || !p->vocab) return CKKS_OK;
    const u32 e = clear_dtype_bytes(p->dtype), oe = clear_dtype_bytes(p->out_dtype);
    const Extent out = extent(p->d_out, oe, {{p->rows, p->out_stride}, {p->vocab, 1}});
    const u32 nt = p->n_tokens, nb = p->n_biases;
    const Extent in[] = {extent(p->d_logits, e, {{p->rows, p->logits_stride}, {p->vocab, 1}}),
                         extent(p->d_tokens, 4, {{nt, 1}}),
                         extent(p->d_token_start, 4, {{p->d_token_start ? p->rows + 1 : 0, 1}}),
                         extent(p->d_n_prompt, 4, {{p->d_n_prompt ? p->rows : 0, 1}}),
                         extent(p->d_repetition, 4, {{p->d_repetition ? p->rows : 0, 1}}),
                         extent(p->d_frequency, 4, {{p->d_frequency ? p->rows : 0, 1}}),
                         extent(p->d_presence, 4, {{p->d_presence ? p->rows : 0, 1}}),
                         extent(p->d_bias_ids, 4, {{nb, 1}}),
                         extent(p->d_bias, 4, {{nb, 1}}),
                         extent(p->d_bias_start, 4, {{p->d_bias_start ? p->rows + 1 : 0, 1}}),
                         extent(p->d_mask, 4, {{p->d_mask ? p->rows : 0, p->mask_stride}, {(p->vocab + 31) / 32, 1}})};
    const bool in_place = p->d_logits == p->d_out && e == oe && (p->rows == 1 || p->logits_stride == p->out_stride);
    for (size_t i = 0; i < sizeof(in) / sizeof(in[0]); ++i)
        if (!(i == 0 && in_place) && overlap(out, in[i])) {
            set_error("ckks_clear_logits: d_out overlaps an input");
            return CKKS_E_INVAL;
        }
    if (p->rows > 1 && (p->out_stride < 0 ? -p->out_stride : p->out_stride) < (i64)p->vocab) {
        set_error("ckks_clear_logits: output rows overlap (stride %lld)", (long long)p->out_stride);
        return CKKS_E_INVAL;
    }
    LogitsArgs a{};
    a.logits = p->d_logits, a.out = p->d_out, a.tokens = nt ? p->d_tokens : nullptr, a.token_start = p->d_token_start, a.n_prompt = p->d_n_prompt;
    a.repetition = p->d_repetition, a.frequency = p->d_frequency, a.presence = p->d_presence;
    a.bias_ids = p->d_bias_ids, a.bias_start = p->d_bias_start, a.bias = nb ? p->d_bias : nullptr, a.mask = p->d_mask;
    a.ls = p->logits_stride, a.os = p->out_stride, a.ms = p->mask_stride;
    a.vocab = p->vocab, a.n_tokens = nt, a.n_biases = nb;
    hipStream_t st = (hipStream_t)stream;
    const bool wide = p->out_dtype == CKKS_CLEAR_F32;
    if (p->dtype == CKKS_CLEAR_F32)
        launch_logits<float, float>(a, p->rows, st);
    else if (p->dtype == CKKS_CLEAR_F16)
        wide ? launch_logits<f16, float>(a, p->rows, st) : launch_logits<f16, f16>(a, p->rows, st);
    else
        wide ? launch_logits<bf16, float>(a, p->rows, st) : launch_logits<bf16, bf16>(a, p->rows, st);
    CKKS_LAUNCH_CHECK("logits_kernel");
    return CKKS_OK;
}
