// Rules on logits: history penalties, biases, mask.  A block takes a stretch of one row's vocabulary, tallies in LDS what the
// row's history and bias list say about the tokens of that stretch, and then streams the logits through it once.  The tallies
// are whole numbers (counts, and the largest list index of a bias), so their order cannot show in a result.
#include <algorithm>

#include "clear_device.h"

namespace ckks {

constexpr u32 SEEN = 1u << 31;  // tally: in the prompt; the bits below count the generated ones

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

// THREADS x V x R entries per block.
template <class T, class TO, int THREADS, int R, bool HISTORY, bool BIAS>
__global__ __launch_bounds__(THREADS) void logits_kernel(LogitsArgs a) {
    constexpr int V = 8, SPAN = THREADS * V * R;
    __shared__ __attribute__((aligned(16))) u32 tally[HISTORY ? SPAN : 4];
    __shared__ __attribute__((aligned(16))) u32 which[BIAS ? SPAN : 4];
    const u32 row = blockIdx.x / a.tiles, first = (blockIdx.x % a.tiles) * SPAN, span = min(a.vocab - first, (u32)SPAN);
    const T *in = (const T *)a.logits + (i64)row * a.ls + first;
    TO *out = (TO *)a.out + (i64)row * a.os + first;
    Pack<T, V> x[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const u32 c = (r * THREADS + threadIdx.x) * V;
        x[r] = load_part<V>(in + c, c < span ? (int)min(span - c, (u32)V) : 0);
    }
    if (HISTORY || BIAS) {
        if (HISTORY)
            for (u32 i = threadIdx.x; i < SPAN / 4; i += THREADS) ((uint4 *)tally)[i] = make_uint4(0, 0, 0, 0);
        if (BIAS)
            for (u32 i = threadIdx.x; i < SPAN / 4; i += THREADS) ((uint4 *)which)[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        if (HISTORY) {
            const u32 h0 = clamp_at(a.token_start[row], a.n_tokens), h1 = clamp_at(a.token_start[row + 1], a.n_tokens);
            const u32 made = a.n_prompt ? h0 + clamp_at(a.n_prompt[row], a.n_tokens) : h0;
            for (u32 i = h0 + threadIdx.x; i < h1; i += THREADS) {
                const u32 c = (u32)a.tokens[i] - first;
                if (c < span) {
                    if (i < made)
                        atomicOr(&tally[c], SEEN);
                    else
                        atomicAdd(&tally[c], 1u);
                }
            }
        }
        if (BIAS) {
            const u32 b0 = clamp_at(a.bias_start[row], a.n_biases), b1 = clamp_at(a.bias_start[row + 1], a.n_biases);
            for (u32 i = b0 + threadIdx.x; i < b1; i += THREADS) {
                const u32 c = (u32)a.bias_ids[i] - first;
                if (c < span) atomicMax(&which[c], i + 1);
            }
        }
        __syncthreads();
    }
    const float rep = HISTORY && a.repetition ? a.repetition[row] : 1.0f, freq = HISTORY && a.frequency ? a.frequency[row] : 0.0f,
                pres = HISTORY && a.presence ? a.presence[row] : 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const u32 c = (r * THREADS + threadIdx.x) * V;
        if (c >= span) break;
        // `first` and c are multiples of 8: a thread's eight bits lie in one byte of the mask
        const u32 bits = a.mask ? (u32)a.mask[(i64)row * a.ms + ((first + c) >> 5)] >> ((first + c) & 31) : 0xffu;
        Pack<TO, V> y;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float l = (float)x[r].v[i];
            if (HISTORY) {
                const u32 t = tally[c + i], n = t & (SEEN - 1);
                if (t) {
                    l = l > 0.0f ? l / rep : l * rep;
                    l = l - freq * (float)n;
                    l = l - (n ? pres : 0.0f);
                }
            }
            if (BIAS) {
                const u32 b = which[c + i];
                if (b) l += a.bias[b - 1];
            }
            y.v[i] = (TO)((bits >> i) & 1 ? l : -__builtin_inff());
        }
        store_part<V>(out + c, y, (int)min(span - c, (u32)V));
    }
}

template <class T, class TO>
static void launch_logits(LogitsArgs a, u32 rows, hipStream_t st) {
    const bool h = a.tokens, b = a.bias;
    // 8192 entries a block: each block reads the row's whole history, so a long stretch reads it less often; 2048 where that
    // leaves most of the 256 CUs without a block
    const bool small = (u64)rows * ((a.vocab + 8191) / 8192) < 256;
    const u32 span = small ? 2048 : 8192;
    a.tiles = (a.vocab + span - 1) / span;
    const dim3 grid(rows * a.tiles);
#define CKKS_LOGITS(H, B)                                                                                          \
    if (h == H && b == B) {                                                                                        \
        if (small)                                                                                                 \
            hipLaunchKernelGGL((logits_kernel<T, TO, 256, 1, H, B>), grid, dim3(256), 0, st, a);                   \
        else                                                                                                       \
            hipLaunchKernelGGL((logits_kernel<T, TO, 512, 2, H, B>), grid, dim3(512), 0, st, a);                   \
    }
    CKKS_LOGITS(false, false)
    CKKS_LOGITS(false, true)
    CKKS_LOGITS(true, false)
    CKKS_LOGITS(true, true)
#undef CKKS_LOGITS
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
    if (p->n_tokens >= 1u << 31 || p->n_biases >= 1u << 31 || p->vocab >= 1u << 31 || (u64)p->rows * ((p->vocab + 2047) / 2048) >= 1u << 31) {
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
