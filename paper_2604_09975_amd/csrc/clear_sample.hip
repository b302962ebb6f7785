// Draw of the next token: temperature, top-k, top-p, min-p and a given uniform number.  A block takes a row.
//
// What is drawn depends on sums of up to a million weights compared with each other, so a weight is computed in 64 bits and added as a
// whole number of 2^-bits: such sums do not depend on their order, and a token next to the border of two is off by 2^-40 of the sum at
// most.  w = exp((l - max) / T) = 2^(n / 64) 2^f with n whole, |f| <= 1/128: a table of 64 and a polynomial of degree 4 (r^5 / 120
// < 4e-14 for r = f ln 2).  Weights below 2^-64 are none.
//
// The order by logits is not needed, only where the kept tokens end in it.  One pass sums counts and weights into bins of
// n / 2 (2^-1/32 apart).  The bin in which the top_k-th token, or the one that fills top_p, lies is then resolved: tokens of one
// value by their count, few by their ranks, many by bins of their values again.  The draw sums the kept weights by stretches of ids and
// looks into the one that holds u.
#include <algorithm>

#include "clear_device.h"

namespace ckks {

constexpr u32 THREADS = 1024, WAVES = THREADS / 64, BINS = 2048, LIST = 256, CHUNKS = 4096;
constexpr u32 MAX_VOCAB = 1u << 20;

struct SampleArgs {
    const void *logits;
    int32_t *token;
    float *prob;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    i64 stride;
    u32 vocab, bits;
};

__device__ __forceinline__ u32 low32(u64 x) { return (u32)x; }
__device__ __forceinline__ u64 shfl_up64(u64 x, int by) {
    return (u64)(u32)__shfl_up((u32)(x >> 32), by) << 32 | (u32)__shfl_up((u32)x, by);
}
// Inclusive sums over the lanes of a wave.
__device__ __forceinline__ u64 scan_wave(u64 x) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const u64 up = shfl_up64(x, o);
        if ((threadIdx.x & 63) >= (u32)o) x += up;
    }
    return x;
}
// Inclusive sums over the block's threads; `wave_sums` is scratch of WAVES.
__device__ __forceinline__ u64 scan_block(u64 x, u64 *wave_sums) {
    x = scan_wave(x);
    const u32 lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    __syncthreads();
    if (lane == 63) wave_sums[wave] = x;
    __syncthreads();
    u64 before = 0;
    for (u32 w = 0; w < WAVES; ++w) before += w < wave ? wave_sums[w] : 0;
    return x + before;
}
// The order of floats as that of whole numbers (-0 as 0).
__device__ __forceinline__ u32 key_of(float x) {
    const u32 b = __float_as_uint(x + 0.0f);
    return b >> 31 ? ~b : b | 1u << 31;
}

template <class T>
__global__ __launch_bounds__(THREADS) void sample_kernel(SampleArgs a) {
    constexpr int V = 16 / sizeof(T);
    constexpr u32 SPAN = THREADS * V;  // ids of a round
    __shared__ u64 mass[CHUNKS];       // of the bins; of stretches of ids
    __shared__ u32 count[BINS];
    __shared__ double power[64];       // 2^(j / 64)
    __shared__ u64 wave_sums[WAVES];
    __shared__ u32 list_key[LIST], list_id[LIST];
    __shared__ u64 list_w[LIST];
    __shared__ u32 n_list, key_min, key_max;
    __shared__ u32 found[4];
    __shared__ u64 found64[2];
    __shared__ float wave_top[WAVES];
    u64 *const chunk = mass;

    const u32 row = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const T *in = (const T *)a.logits + (i64)row * a.stride;
    const u32 rounds = (a.vocab + SPAN - 1) / SPAN;
    auto fetch = [&](u32 r) {
        const u32 c = r * SPAN + threadIdx.x * V;
        Pack<T, V> x;
        if (c + V <= a.vocab) return load_pack<V>(in + c);
#pragma unroll
        for (int i = 0; i < V; ++i) x.v[i] = c + i < a.vocab ? in[c + i] : (T)-__builtin_inff();
        return x;
    };
    // use(round, pack) for the thread's part of the row, the next round's under way
    auto each = [&](auto use) {
        Pack<T, V> next = fetch(0);
#pragma unroll 1
        for (u32 r = 0; r < rounds; ++r) {
            const Pack<T, V> x = next;
            next = fetch(r + 1);
            use(r, x);
        }
    };

    float top = -__builtin_inff();
    each([&](u32, const Pack<T, V> &x) {
#pragma unroll
        for (int i = 0; i < V; ++i) top = fmaxf(top, (float)x.v[i]);
    });
#pragma unroll
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    if (lane == 0) wave_top[wave] = top;
    if (threadIdx.x < 64) power[threadIdx.x] = exp2(threadIdx.x / 64.0);
    __syncthreads();
#pragma unroll
    for (u32 w = 0; w < WAVES; ++w) top = fmaxf(top, wave_top[w]);
    if (top == -__builtin_inff()) {
        if (threadIdx.x == 0) {
            a.token[row] = -1;
            if (a.prob) a.prob[row] = 0.0f;
        }
        return;
    }
    // logits as they count: NaN as -infinity; beside +infinity only such
    const bool endless = top == __builtin_inff();
    if (endless) top = 0.0f;
    auto logit = [&](T x) {
        const float l = fmaxf((float)x, -__builtin_inff());
        return endless ? (l == __builtin_inff() ? 0.0f : -__builtin_inff()) : l;
    };

    float temperature = a.temperature ? a.temperature[row] : 1.0f;
    const bool greedy = temperature <= 0.0f;
    if (!(temperature > 0.0f)) temperature = 1.0f;
    const double c64 = 64.0 * 1.4426950408889634074 / (double)temperature, top64 = top;
    const double magic = __longlong_as_double((long long)(1023 + 52 - a.bits) << 52);
    constexpr double STEP = 0.69314718055994530942 / 64;
    // 64 d and the weight of a logit, d = log2 of its inverse; none from 2^-64
    struct Weight {
        u32 n;
        double w;
        __device__ bool some() const { return n < 2 * BINS; }
    };
    auto place = [&](float l, double &f) {
        const double t = fmax(((double)l - top64) * c64, -8192.0), n = __builtin_rint(t);
        f = t - n;
        return (u32)-(int)n;
    };
    auto weigh = [&](float l) {
        Weight r;
        double f;
        r.n = place(l, f);
        f *= STEP;
        const double e = __builtin_fma(f, __builtin_fma(f, __builtin_fma(f, __builtin_fma(f, 1.0 / 24, 1.0 / 6), 0.5), 1.0), 1.0);
        const int n = -(int)r.n;
        r.w = r.some() ? __builtin_ldexp(e * power[n & 63], n >> 6) : 0.0;
        return r;
    };
    auto whole = [&](double w) { return (u64)__double_as_longlong(w + magic) & ((1ull << 52) - 1); };

    // The lowest id with sum over ids up to it of amount(id, logit) above `target`; `all` becomes the sum over all ids.
    auto by_id = [&](auto amount, auto target, u64 &all, u64 &own) -> u32 {
        __syncthreads();
        each([&](u32 r, const Pack<T, V> &x) {
            u64 sum = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) sum += amount(r * SPAN + threadIdx.x * V + i, logit(x.v[i]));
            if (__any(sum != 0)) sum = scan_wave(sum);
            if (lane == 63) chunk[r * WAVES + wave] = sum;
        });
        __syncthreads();
        // four chunks a thread
        const u32 n = rounds * WAVES;
        u64 part[CHUNKS / THREADS], sum = 0;
#pragma unroll
        for (u32 k = 0; k < CHUNKS / THREADS; ++k) {
            const u32 at = threadIdx.x * (CHUNKS / THREADS) + k;
            part[k] = at < n ? chunk[at] : 0;
            sum += part[k];
        }
        const u64 upto = scan_block(sum, wave_sums);
        if (threadIdx.x == THREADS - 1) found64[0] = upto;
        __syncthreads();
        all = found64[0];
        const u64 goal = target(all);
        u64 before = upto - sum;
#pragma unroll
        for (u32 k = 0; k < CHUNKS / THREADS; ++k) {
            if (before <= goal && goal < before + part[k]) {
                found[0] = threadIdx.x * (CHUNKS / THREADS) + k;
                found64[1] = before;
            }
            before += part[k];
        }
        __syncthreads();
        const u32 at = min(found[0], n - 1);
        if (wave == at % WAVES) {
            const u32 r = at / WAVES;
            const Pack<T, V> x = fetch(r);
            u64 part[V], sum = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) sum += part[i] = amount(r * SPAN + threadIdx.x * V + i, logit(x.v[i]));
            u64 before = found64[1] + scan_wave(sum) - sum;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (before <= goal && goal < before + part[i]) {
                    found[1] = r * SPAN + threadIdx.x * V + i;
                    found64[0] = part[i];
                }
                before += part[i];
            }
        }
        __syncthreads();
        own = found64[0];
        return found[1];
    };

    // The last token kept in the order of logits: larger ones are, of equal ones those up to its id.
    float last = -__builtin_inff();
    u32 last_id = ~0u;
    auto kept = [&](float l, u32 id) { return l > last || (l == last && id <= last_id); };
    u64 all, own;
    const int32_t top_k = a.top_k ? a.top_k[row] : 0;
    const float top_p = a.top_p ? a.top_p[row] : 1.0f, min_p = a.min_p ? a.min_p[row] : 0.0f;
    const bool limit_k = top_k > 0 && (u32)top_k < a.vocab, limit_p = top_p < 1.0f;
    if (greedy || (limit_k && top_k == 1)) {
        last = top;
        last_id = by_id([&](u32, float l) { return l == top ? 1ull : 0ull; }, [](u64) { return 0ull; }, all, own);
        if (threadIdx.x == 0) {
            a.token[row] = (int32_t)last_id;
            if (a.prob) a.prob[row] = 1.0f;
        }
        return;
    }
    if (limit_k || limit_p) {
        // counts and weights by bins
        for (u32 i = threadIdx.x; i < BINS; i += THREADS) mass[i] = 0, count[i] = 0;
        __syncthreads();
        each([&](u32, const Pack<T, V> &x) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const Weight w = weigh(logit(x.v[i]));
                if (w.some()) {
                    atomicAdd((unsigned long long *)&mass[w.n >> 1], (unsigned long long)whole(w.w));
                    atomicAdd(&count[w.n >> 1], 1u);
                }
            }
        });
        __syncthreads();
        u64 bin_mass[2], upto_mass[2];
        u32 bin_count[2], upto_count[2];
        {
            const u32 b = 2 * threadIdx.x;
#pragma unroll
            for (int k = 0; k < 2; ++k) bin_mass[k] = mass[b + k], bin_count[k] = count[b + k];
            upto_mass[1] = scan_block(bin_mass[0] + bin_mass[1], wave_sums);
            upto_mass[0] = upto_mass[1] - bin_mass[1];
            upto_count[1] = (u32)scan_block(bin_count[0] + bin_count[1], wave_sums);
            upto_count[0] = upto_count[1] - bin_count[1];
        }
        if (threadIdx.x == THREADS - 1) {
            found64[0] = upto_mass[1];
            found[0] = upto_count[1];
        }
        __syncthreads();
        u64 total = found64[0];
        const u32 tokens = found[0];
        // Narrows to the last token that counts: with `by_count` the goal_count-th, else the one before which weights sum to less than
        // goal_mass and with which they do not.  Sets last, last_id; returns the weights up to and with it.
        auto resolve = [&](bool by_count, u64 goal_count, double goal_mass) -> u64 {
            const auto reached = [&](u64 c, u64 m) { return by_count ? c >= goal_count : (double)m >= goal_mass; };
            __syncthreads();
            if (threadIdx.x == 0) found[0] = ~0u;
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (reached(upto_count[k], upto_mass[k]) && !reached(upto_count[k] - bin_count[k], upto_mass[k] - bin_mass[k])) {
                    found[0] = 2 * threadIdx.x + k;
                    found[1] = upto_count[k] - bin_count[k];
                    found64[0] = upto_mass[k] - bin_mass[k];
                }
            __syncthreads();
            const u32 bin = found[0];
            u64 above_count = found[1], above_mass = found64[0];
            if (bin == ~0u) {  // all of them count
                last = -__builtin_inff();
                last_id = ~0u;
                return total;
            }
            u32 lo = 0, hi = ~0u;  // keys that are looked at
            for (;;) {
                __syncthreads();
                if (threadIdx.x == 0) n_list = 0, key_min = ~0u, key_max = 0;
                __syncthreads();
                each([&](u32 r, const Pack<T, V> &x) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float l = logit(x.v[i]);
                        double f;
                        const u32 key = key_of(l);
                        if (place(l, f) >> 1 == bin && key >= lo && key <= hi) {
                            atomicMin(&key_min, key);
                            atomicMax(&key_max, key);
                            const u32 at = atomicAdd(&n_list, 1u);
                            if (at < LIST) {
                                list_key[at] = key;
                                list_id[at] = r * SPAN + threadIdx.x * V + i;
                                list_w[at] = whole(weigh(l).w);
                            }
                        }
                    }
                });
                __syncthreads();
                const u32 n = n_list, from = key_min, to = key_max;
                const auto value = [](u32 key) { return __uint_as_float(key >> 31 ? key & ~(1u << 31) : ~key); };
                if (from == to) {  // equal ones: by their ids
                    last = value(from);
                    const u64 w = whole(weigh(last).w);
                    u64 m;
                    if (by_count) {
                        m = goal_count - above_count;
                    } else {  // the smallest m with above + m w >= goal
                        m = w ? (u64)((goal_mass - (double)above_mass) / (double)w) : 1;
                        while (m > 1 && (double)(above_mass + (m - 1) * w) >= goal_mass) --m;
                        while (m < n && (double)(above_mass + m * w) < goal_mass) ++m;
                    }
                    m = min(max(m, 1ull), (u64)n);
                    u64 sum, one;
                    const float at = last;
                    last_id = by_id([&](u32, float l) { return l == at ? 1ull : 0ull; }, [&](u64) { return m - 1; }, sum, one);
                    return above_mass + m * w;
                }
                if (n <= LIST) {  // by their ranks
                    if (threadIdx.x < n) {
                        const u32 key = list_key[threadIdx.x], id = list_id[threadIdx.x];
                        const u64 w = list_w[threadIdx.x];
                        u64 c = above_count, m = above_mass;
                        for (u32 j = 0; j < n; ++j)
                            if (list_key[j] > key || (list_key[j] == key && list_id[j] < id)) {
                                ++c;
                                m += list_w[j];
                            }
                        if (!reached(c, m) && reached(c + 1, m + w)) {
                            found[2] = key;
                            found[3] = id;
                            found64[1] = m + w;
                        }
                    }
                    __syncthreads();
                    last = value(found[2]);
                    last_id = found[3];
                    return found64[1];
                }
                // by bins of their keys
                u32 shift = 0;
                while ((to - from) >> shift >= BINS) ++shift;
                for (u32 i = threadIdx.x; i < BINS; i += THREADS) mass[i] = 0, count[i] = 0;
                __syncthreads();
                each([&](u32, const Pack<T, V> &x) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float l = logit(x.v[i]);
                        double f;
                        const u32 key = key_of(l);
                        if (place(l, f) >> 1 == bin && key >= from && key <= to) {
                            atomicAdd((unsigned long long *)&mass[(to - key) >> shift], (unsigned long long)whole(weigh(l).w));
                            atomicAdd(&count[(to - key) >> shift], 1u);
                        }
                    }
                });
                __syncthreads();
                const u64 m0 = mass[2 * threadIdx.x], m1 = mass[2 * threadIdx.x + 1];
                const u32 c0 = count[2 * threadIdx.x], c1 = count[2 * threadIdx.x + 1];
                const u64 um = above_mass + scan_block(m0 + m1, wave_sums), uc = above_count + scan_block(c0 + c1, wave_sums);
                auto take = [&](u32 b, u64 c, u64 m, u64 dc, u64 dm) {
                    if (reached(c, m) && !reached(c - dc, m - dm)) {
                        found[0] = b;
                        found[1] = (u32)(c - dc);
                        found64[0] = m - dm;
                    }
                };
                take(2 * threadIdx.x, uc - c1, um - m1, c0, m0);
                take(2 * threadIdx.x + 1, uc, um, c1, m1);
                __syncthreads();
                above_count = found[1];
                above_mass = found64[0];
                hi = to - (found[0] << shift);
                const u32 width = (1u << shift) - 1;
                lo = hi - from > width ? hi - width : from;
            }
        };
        if (limit_k && (u32)top_k < tokens) total = resolve(true, (u64)top_k, 0.0);
        if (limit_p) {
            const float l = last;
            const u32 id = last_id;
            resolve(false, 0, fmax((double)top_p * (double)total, 0.5));
            // (within the top_k already, but for a goal that rounds to all of them)
            if (l > last || (l == last && id < last_id)) last = l, last_id = id;
        }
    }
    const double least = min_p > 0.0f ? fmin((double)min_p, 1.0) : 0.0;
    const float u = a.u[row];
    const u32 id = by_id(
        [&](u32 i, float l) -> u64 {
            if (!kept(l, i)) return 0;
            const Weight w = weigh(l);
            return w.w >= least ? whole(w.w) : 0ull;
        },
        [&](u64 sum) -> u64 { return u < 1.0f ? min((u64)(fmax((double)u, 0.0) * (double)sum), sum - 1) : u >= 1.0f ? sum - 1 : 0ull; }, all, own);
    if (threadIdx.x == 0) {
        a.token[row] = (int32_t)id;
        if (a.prob) a.prob[row] = (float)((double)own / (double)all);
    }
}

template <class T>
static void launch_sample(const SampleArgs &a, u32 rows, hipStream_t st) {
    hipLaunchKernelGGL((sample_kernel<T>), dim3(rows), dim3(THREADS), 0, st, a);
}

}  // namespace ckks

using namespace ckks;

extern "C" int ckks_clear_sample(const ckks_clear_sample_t *p, void *stream) {
    const char *who = "ckks_clear_sample";
    if (!p || (p->rows && (!p->d_token || !p->d_u || (p->vocab && !p->d_logits)))) {
        set_error("%s: null argument", who);
        return CKKS_E_INVAL;
    }
    if (!clear_dtype_ok(p->dtype) || !p->vocab || p->vocab > MAX_VOCAB || p->rows >= 1u << 31) {
        set_error("%s: %u rows of %u logits of type %u (a row has 1 to %u)", who, p->rows, p->vocab, p->dtype, MAX_VOCAB);
        return CKKS_E_INVAL;
    }
    if (!p->rows) return CKKS_OK;
    const u32 n = p->rows;
    const Extent out[2] = {extent(p->d_token, 4, {{n, 1}}), extent(p->d_prob, 4, {{p->d_prob ? n : 0, 1}})};
    const Extent in[6] = {extent(p->d_logits, clear_dtype_bytes(p->dtype), {{n, p->logits_stride}, {p->vocab, 1}}),
                          extent(p->d_u, 4, {{n, 1}}),
                          extent(p->d_temperature, 4, {{p->d_temperature ? n : 0, 1}}),
                          extent(p->d_top_p, 4, {{p->d_top_p ? n : 0, 1}}),
                          extent(p->d_min_p, 4, {{p->d_min_p ? n : 0, 1}}),
                          extent(p->d_top_k, 4, {{p->d_top_k ? n : 0, 1}})};
    bool bad = overlap(out[0], out[1]);
    for (const Extent &o : out)
        for (const Extent &i : in) bad |= overlap(o, i);
    if (bad) {
        set_error("%s: an output overlaps another array", who);
        return CKKS_E_INVAL;
    }
    SampleArgs a{};
    a.logits = p->d_logits, a.token = p->d_token, a.prob = p->d_prob, a.u = p->d_u, a.temperature = p->d_temperature;
    a.top_p = p->d_top_p, a.min_p = p->d_min_p, a.top_k = p->d_top_k, a.stride = p->logits_stride, a.vocab = p->vocab;
    // sums of all weights, 1 at most each, below 2^62; the magic number needs fewer than 52 bits
    a.bits = 62;
    while ((1u << (62 - a.bits)) < p->vocab) --a.bits;
    a.bits = std::min(a.bits, 51u);
    hipStream_t st = (hipStream_t)stream;
    if (p->dtype == CKKS_CLEAR_F32)
        launch_sample<float>(a, n, st);
    else if (p->dtype == CKKS_CLEAR_F16)
        launch_sample<f16>(a, n, st);
    else
        launch_sample<bf16>(a, n, st);
    CKKS_LAUNCH_CHECK("sample_kernel");
    return CKKS_OK;
}
