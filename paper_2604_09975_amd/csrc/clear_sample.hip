// Draw of the next token: temperature, top-k, top-p, min-p and a given uniform number.  A block takes a row.
//
// What is drawn depends on sums of up to a million weights compared with each other, so a weight is computed in 64 bits.
// w = exp((l - max) / T) = 2^(-n / 256) 2^(f / 256) with n whole, |f| <= 1/2: a table of 256 and a polynomial of degree 3
// (r^4 / 24 < 1.4e-13 < 2^-42 for r = f ln 2 / 256).  Weights below 2^-64 are none.  Sums are of 64-bit floats in a fixed order, and
// where atomics add, of whole numbers, which do not depend on theirs:
//   by bins: of 2^-bits of the octave that the bin lies in, 2^-42 of each weight for 2^20 tokens, 2^-45 for 131072;
//   of up to 8192 tokens set apart: of 2^-54 for weights from 2^-13 on, of 2^-66 for those below: 2^-41 of the sum.
// So a token next to the border of two is off by 2^-40 of the sum at most, however many small weights make up the sum.
//
// The order by logits is not needed, only where the kept tokens end in it: at a value, and after so many of the tokens that have it.
//   top_k of up to 256: the logits are counted by bins of their distance from the largest, those of the bins that hold the top_k are
//     put into a list, and all the rest goes by the list.
//   else: one pass sums counts and weights into bins (2^-1/32 apart).  The bin in which the top_k-th token, or the one that fills
//     top_p, lies is then resolved: tokens of one value by their count, others by sorting them, very many by bins of their values first.
// The draw sums the kept weights by stretches of ids and looks into the one that holds u.
//
// Bound by a weight's 25 instructions or so in 64 bits where each row has a CU, not by the logits' bytes: 256 rows of 131072 bf16 (67 MB,
// 14 us by the bytes) take 44 us with no limit, 29 with top_k 50, which needs no weights but the list's, 116 with top_p 0.9, which needs
// all of them and a border resolved.  A single row has one CU: 50257 logits 14 us with a list, 42 with top_p 0.9 alone.
// 1024 threads leave 128 registers each: of F32 rows 10 lie in scratch, at the edges of the steps, of 16-bit ones none.
#include <algorithm>
#include <type_traits>

#include "clear_device.h"

namespace ckks {

constexpr u32 BINS = 2048, CHUNKS = 4096;
constexpr u32 LIST_K = 256, LISTED = 2048;  // the largest top_k that goes by a list, and the list's room
constexpr u32 MAX_VOCAB = 1u << 20;
constexpr u32 GRAIN = 256, GRAINS = 64 * GRAIN;  // steps of n: 2^-1/256; weights below 2^-64 are none
constexpr double FAR = 512 * GRAIN;              // ... as they are computed: 2^-512, nothing beside a weight
constexpr double TINY = 0x1p-100;                // more than what many such sum to, less than a weight

struct SampleArgs {
    const void *logits;
    int32_t *token;
    float *prob;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    i64 stride;
    u32 vocab, bits, row0;
};

// Inclusive sums over the lanes of a wave: by DPP within rows of 16, then from row to row.
template <int CTRL, int ROWS>
__device__ __forceinline__ u32 add_dpp(u32 x) {
    return x + (u32)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double add_dpp(double x) {
    const u64 b = (u64)__double_as_longlong(x);
    const u32 lo = (u32)__builtin_amdgcn_update_dpp(0, (int)(u32)b, CTRL, ROWS, 0xf, false);
    const u32 hi = (u32)__builtin_amdgcn_update_dpp(0, (int)(u32)(b >> 32), CTRL, ROWS, 0xf, false);
    return x + __longlong_as_double((long long)((u64)hi << 32 | lo));
}
template <class X>
__device__ __forceinline__ X scan_wave(X x) {
    x = add_dpp<0x111, 0xf>(x);  // row_shr 1, 2, 4, 8
    x = add_dpp<0x112, 0xf>(x);
    x = add_dpp<0x114, 0xf>(x);
    x = add_dpp<0x118, 0xf>(x);
    x = add_dpp<0x142, 0xa>(x);  // row_bcast 15, 31
    return add_dpp<0x143, 0xc>(x);
}
__device__ __forceinline__ u32 lane_of(u32 x, u32 lane) { return (u32)__builtin_amdgcn_readlane((int)x, lane); }
__device__ __forceinline__ double lane_of(double x, u32 lane) {
    const u64 b = (u64)__double_as_longlong(x);
    return __longlong_as_double((long long)((u64)lane_of((u32)(b >> 32), lane) << 32 | lane_of((u32)b, lane)));
}
// The order of floats as that of whole numbers (-0 as 0), and back.
__device__ __forceinline__ u32 key_of(float x) {
    const u32 b = __float_as_uint(x + 0.0f);
    return b >> 31 ? ~b : b | 1u << 31;
}
__device__ __forceinline__ float value_of(u32 key) { return __uint_as_float(key >> 31 ? key & ~(1u << 31) : ~key); }

// V: logits of an access, which a row has at least.
template <class T, int THREADS, int V>
__global__ __launch_bounds__(THREADS) void sample_kernel(SampleArgs a) {
    constexpr int PER = BINS / THREADS;
    constexpr u32 APART = THREADS == 1024 ? 8192 : 2048;
    constexpr u32 SPAN = THREADS * V, WAVES = THREADS / 64;    // SPAN: ids of a round
    __shared__ __attribute__((aligned(16))) u64 mass[CHUNKS];  // weights of the bins, as whole numbers; of stretches of ids; lists
    __shared__ u32 count[CHUNKS];                              // tokens of the bins; of stretches of ids that have the last value
    __shared__ u64 apart[APART];                               // tokens set apart, those that all later passes are about
    __shared__ double power[GRAIN];                            // 2^(j / 256)
    __shared__ u32 wave_counts[WAVES];
    __shared__ double wave_sums[WAVES];
    __shared__ u32 n_list, n_bin, key_min, key_max;
    __shared__ u32 found[3], found_count;
    __shared__ double found_sum;
    __shared__ float wave_top[WAVES];

    const u32 row = a.row0 + blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const T *in = (const T *)a.logits + (i64)row * a.stride;
    const u32 rounds = (a.vocab + SPAN - 1) / SPAN;
    // First id of the thread's part of a round; the last ones of a row begin before their place, and what lies there is left out.
    auto at_of = [&](u32 r) { return min(r * SPAN + threadIdx.x * V, a.vocab - V); };
    auto fetch = [&](u32 r) { return load_pack<V>(in + at_of(r)); };
    auto cut = [&](u32 r, Pack<T, V> &x) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (at_of(r) + i < r * SPAN + threadIdx.x * V) x.v[i] = (T)-__builtin_inff();
    };
    // use(first id, pack, round) for the thread's part of the row, `ahead` rounds under way.  (They keep their registers: moving a
    // pack from one to another would be a wait for it.)
    auto each = [&](auto ahead, auto use) {
        constexpr u32 AHEAD = decltype(ahead)::value;
        Pack<T, V> next[AHEAD];
#pragma unroll
        for (u32 k = 0; k < AHEAD; ++k) next[k] = fetch(k);
#pragma unroll 1
        for (u32 r = 0; r < rounds; r += AHEAD)
#pragma unroll
            for (u32 k = 0; k < AHEAD; ++k) {
                Pack<T, V> x = next[k];
                next[k] = fetch(r + k + AHEAD);
                if (r + k >= rounds) break;
                if (r + k + 1 == rounds) cut(r + k, x);
                use(at_of(r + k), x, r + k);
            }
    };
    constexpr std::integral_constant<u32, 4> LIGHT;  // for passes that do little with a logit, and for the others
    constexpr std::integral_constant<u32, 2> HEAVY;
    // use(i, logit) for those few of a pack that `some` holds for: as many turns as the lane with the most of them has
    // (then end(lanes that had one), by all lanes of the wave)
    auto few_of = [&](const Pack<T, V> &x, auto some, auto use, auto end) {
        u32 bits = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) bits |= some((float)x.v[i]) ? 1u << i : 0u;
        u32 w[8] = {};
        __builtin_memcpy(w, &x, sizeof(x));
        for (u64 active; (active = __ballot(bits != 0)); end(active)) {
            if (!bits) continue;
            const u32 i = __ffs(bits) - 1, at = i * sizeof(T) / 4;
            bits &= bits - 1;
            const u32 a0 = at & 1 ? w[1] : w[0], a1 = at & 1 ? w[3] : w[2], a2 = at & 1 ? w[5] : w[4], a3 = at & 1 ? w[7] : w[6];
            const u32 word = at & 4 ? (at & 2 ? a3 : a2) : (at & 2 ? a1 : a0), cell = word >> (i * sizeof(T) % 4 * 8);
            T v;
            __builtin_memcpy(&v, &cell, sizeof(T));
            use(i, (float)v);
        }
    };
    auto nothing = [](u64) {};
    bool set_apart = false, many = false;  // many: too many to be set apart
    u32 own_apart = 0;                     // tokens that the wave has set apart, in its own stretch of `apart`
    constexpr u32 OWN = APART / WAVES;
    auto each_of = [&](auto some, auto use) {
        if (set_apart) {
            for (u32 i = lane; i < own_apart; i += 64) {
                const u64 x = apart[wave * OWN + i];
                const float l = value_of((u32)(x >> 32));
                if (some(l)) use((u32)~x, l);
            }
            return;
        }
        each(LIGHT, [&](u32 at, const Pack<T, V> &x, u32) { few_of(x, some, [&](u32 i, float l) { use(at + i, l); }, nothing); });
    };
    // Inclusive sums over the threads, and over all of them, in two steps with a barrier between them.
    auto scan_begin = [&](auto x, auto *of_wave) {
        x = scan_wave(x);
        if (lane == 63) of_wave[wave] = x;
        return x;
    };
    auto scan_end = [&](auto x, const auto *of_wave, auto &all) {
        const auto upto = scan_wave(lane < WAVES ? of_wave[lane] : decltype(x)(0));
        all = lane_of(upto, WAVES - 1);
        return wave ? x + lane_of(upto, wave - 1) : x;
    };
    auto scan_sums = [&](double x, double &all) {
        __syncthreads();
        x = scan_begin(x, wave_sums);
        __syncthreads();
        return scan_end(x, wave_sums, all);
    };
    auto scan_counts = [&](u32 x, u32 &all) {
        __syncthreads();
        x = scan_begin(x, wave_counts);
        __syncthreads();
        return scan_end(x, wave_counts, all);
    };
    auto scan_both = [&](double &x, double &all, u32 &n, u32 &count) {
        __syncthreads();
        x = scan_begin(x, wave_sums);
        n = scan_begin(n, wave_counts);
        __syncthreads();
        x = scan_end(x, wave_sums, all);
        n = scan_end(n, wave_counts, count);
    };
    // Atomics of single lanes go to an address of their own: one that the compiler knows to be the same for all lanes it goes through lane by
    // lane, which takes ten times as long.
    u32 zero = 0;
    asm volatile("" : "+v"(zero));
    // The least `first` and the largest `end` of all threads, in `found`; ~0 and 0 are none.  (Both rise from thread to thread.)
    auto find_ends = [&](u32 first, u32 end) {
        const u64 firsts = __ballot(first != ~0u), ends = __ballot(end != 0);
        if (firsts) first = lane_of(first, (u32)__ffsll((unsigned long long)firsts) - 1);
        if (ends) end = lane_of(end, 63 - (u32)__clzll((long long)ends));
        if (lane == 0 && firsts) atomicMin(&found[0] + zero, first);
        if (lane == 0 && ends) atomicMax(&found[1] + zero, end);
    };
    auto finish = [&](u32 token, double prob) {
        if (threadIdx.x == 0) {
            a.token[row] = (int32_t)token;
            if (a.prob) a.prob[row] = (float)prob;
        }
    };

    float top = -__builtin_inff();
    each(LIGHT, [&](u32, const Pack<T, V> &x, u32) {
#pragma unroll
        for (int i = 0; i < V; ++i) top = fmaxf(top, (float)x.v[i]);
    });
    const float own_top = top;
#pragma unroll
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    if (lane == 0) wave_top[wave] = top;
    for (u32 j = threadIdx.x; j < GRAIN; j += THREADS) power[j] = exp2(j / (double)GRAIN);
    for (u32 i = threadIdx.x; i < BINS; i += THREADS) mass[i] = 0, count[i] = 0;
    if (threadIdx.x == 0) n_list = 0;
    __syncthreads();
#pragma unroll
    for (u32 w = 0; w < WAVES; ++w) top = fmaxf(top, wave_top[w]);
    if (top == -__builtin_inff()) return finish(~0u, 0.0);

    const float temperature = a.temperature && a.temperature[row] == a.temperature[row] ? a.temperature[row] : 1.0f;
    const float top_p = a.top_p ? a.top_p[row] : 1.0f, min_p = a.min_p ? a.min_p[row] : 0.0f, u = a.u[row];
    const int32_t top_k = a.top_k ? a.top_k[row] : 0;
    const bool limit_k = top_k > 0 && (u32)top_k < a.vocab, limit_p = top_p < 1.0f;
    const double least = min_p > 0.0f ? fmin((double)min_p, 1.0) : 0.0;
    const double c = GRAIN * 1.4426950408889634074 / (double)temperature, top64 = top;
    const double magic = __longlong_as_double((long long)(1023 + 52 - a.bits) << 52);
    // Logits that have a weight, of 2^-64 or more; false for NaN and -infinity.
    const double least_l = top64 - GRAINS / c;
    float floor_l = fmaxf((float)least_l, -3.402823466e38f);
    if ((double)floor_l < least_l) floor_l = value_of(key_of(floor_l) + 1);
    auto may = [&](float l) { return l >= floor_l; };
    const float reach = 1e-6f * fabsf(top);  // more than bounds that are worked out in 32 bits are off by
    // n: steps down from the largest; w = 2^(-n / 256) 2^(f / 256).  (NaN and all that is far below: n = FAR.)
    struct Weight {
        u32 n;
        double w;
    };
    auto weigh = [&](float l) {
        constexpr double ROUND = 6755399441055744.0, STEP = 0.69314718055994530942 / GRAIN;  // 1.5 * 2^52: n in the lower word of the sum
        const double t = fmax(((double)l - top64) * c, -FAR), s = t + ROUND, f = t - (s - ROUND);
        const double q = f * __builtin_fma(f, __builtin_fma(f, STEP * STEP * STEP / 6, STEP * STEP / 2), STEP);
        const int n = (int)(u32)__double_as_longlong(s);
        const u64 e = (u64)__double_as_longlong(power[n & (GRAIN - 1)]) + ((u64)(u32)((n >> 8) << 20) << 32);
        const double p = __longlong_as_double((long long)e);
        return Weight{(u32)-n, __builtin_fma(p, q, p)};
    };
    static_assert(GRAIN == 256, "n >> 8");
    auto bin_of = [&](u32 n) { return min(n / (GRAINS / BINS), BINS - 1); };
    // A bin's weights as whole numbers of 2^-bits of its octave (a half to one of it, so none becomes 0), and a sum of them.
    constexpr u32 OCTAVE = GRAIN / (GRAINS / BINS);  // bins of an octave
    auto whole = [&](double w, u32 bin) {
        const double x = __longlong_as_double(__double_as_longlong(w) + ((long long)(bin / OCTAVE) << 52));
        return (u64)__double_as_longlong(x + magic) & ((1ull << 52) - 1);
    };
    auto sum_of = [&](u64 sum, u32 bin) { return (double)sum * __longlong_as_double((long long)(1023 - a.bits - bin / OCTAVE) << 52); };
    // What u asks for of a sum: the token is the first with which the sum is above it, or the last.
    auto share = [&](double sum) { return u < 1.0f ? fmax((double)u, 0.0) * sum : u >= 1.0f ? __builtin_inf() : 0.0; };
    // Logits that may reach min_p, and a little below.  (The logarithm of the hardware takes a subnormal as 0; and no weight is below 2^-64.)
    const float least_log = __log2f(fmaxf((float)least, 0x1p-64f));
    const float enough = least > 0.0 ? (float)(top64 + (least_log * GRAIN - 1.0) / c) - reach : floor_l;

    // Kept are the tokens above `last`, and of those that have it the `ties` with the lowest ids.
    float last = floor_l;
    u32 ties = ~0u;

    // The lowest id up to which amounts sum to more than goal(all of them), or the last that has one: amount(logit) where `some` holds, and
    // `one` for each of the first `ties` tokens of value `last` (for which `some` need not hold).  `dense`: how many logits have an
    // amount.  prob: the token's share.
    auto draw = [&](auto dense, auto some, auto amount, double one, auto goal, double &prob) -> u32 {
        constexpr bool DENSE = decltype(dense)::value > 0, TIES = decltype(dense)::value < 2;
        auto value = [&](double sum, u32 n) { return TIES ? sum + (double)min(n, ties) * one : sum; };
        // whether there is something among tokens of this sum, `same` of them of value `last` after `before` others
        auto any_of = [&](double sum, u32 same, u32 before) { return sum > TINY || (TIES && same && before < ties && one > 0.0); };
        const u32 n = rounds * WAVES;  // a chunk: what a wave takes in a round, 64 V ids; 2048 at most
        const bool by_atomics = !DENSE && set_apart;
        constexpr double LARGE = 0x1p54, SMALL = 0x1p66;  // grids: sums of a chunk's 512 weights stay below 2^64
        u64 *const small = mass + CHUNKS / 2;
        __syncthreads();
        if (by_atomics) {
            for (u32 i = threadIdx.x; i < n; i += THREADS) mass[i] = 0, small[i] = 0, count[i] = 0;
            __syncthreads();
            each_of([&](float l) { return l >= last && some(l); }, [&](u32 id, float l) {
                if (l > last) {
                    const double w = amount(l);
                    if (w >= 0x1p-13)
                        atomicAdd((unsigned long long *)&mass[id / (64 * V)], (unsigned long long)(w * LARGE));
                    else
                        atomicAdd((unsigned long long *)&small[id / (64 * V)], (unsigned long long)(w * SMALL));
                } else {
                    atomicAdd(&count[id / (64 * V)], 1u);
                }
            });
        } else each(std::integral_constant<u32, DENSE ? 2 : 4>(), [&](u32, const Pack<T, V> &x, u32 r) {
            double sum = 0.0;
            u32 same = 0;
            if (DENSE) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float l = (float)x.v[i];
                    sum += amount((TIES ? l > last : may(l)) ? l : -__builtin_inff());
                    if (TIES) same += l == last;
                    if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                }
            } else {
                few_of(x, [&](float l) { return l >= last && some(l); }, [&](u32, float l) {
                    if (l > last)
                        sum += amount(l);
                    else
                        ++same;
                }, nothing);
            }
            if (DENSE || __any(sum != 0.0)) sum = scan_wave(sum);
            if (TIES && __any(same != 0)) same = scan_wave(same);
            if (lane == 63) {
                mass[r * WAVES + wave] = (u64)__double_as_longlong(sum);
                count[r * WAVES + wave] = same;
            }
        });
        __syncthreads();
        if (threadIdx.x == 0) found[0] = ~0u, found[1] = 0;
        constexpr u32 EACH = THREADS == 1024 ? CHUNKS / 2 / THREADS : 1;  // chunks a thread
        double part[EACH], sum = 0.0;
        u32 same[EACH], sames = 0;
#pragma unroll
        for (u32 k = 0; k < EACH; ++k) {
            const u32 at = threadIdx.x * EACH + k;
            part[k] = 0.0;
            if (at < n) part[k] = by_atomics ? (double)mass[at] * (1 / LARGE) + (double)small[at] * (1 / SMALL) : __longlong_as_double((long long)mass[at]);
            same[k] = at < n ? count[at] : 0;
            sum += part[k];
            sames += same[k];
        }
        double sum0 = sum, all;
        u32 same0 = sames, all_same = 0;
        if constexpr (TIES)
            scan_both(sum0, all, same0, all_same);
        else
            sum0 = scan_sums(sum0, all);
        all = value(all, all_same);
        const double wanted = goal(all);
        sum0 -= sum;
        same0 -= sames;
        u32 first = ~0u, end = 0;  // the first of the thread's chunks with which the sum is above it; behind the last that adds to it
        {
            double s = sum0;
            u32 m = same0;
#pragma unroll
            for (u32 k = 0; k < EACH; ++k) {
                if (any_of(part[k], same[k], m)) {
                    end = threadIdx.x * EACH + k + 1;
                    if (first == ~0u && value(s + part[k], m + same[k]) > wanted) first = end - 1;
                }
                s += part[k];
                m += same[k];
            }
        }
        find_ends(first, end);
        __syncthreads();
        const u32 at = min(min(found[0], found[1] - 1), n - 1);
        if (threadIdx.x == at / EACH) {
#pragma unroll
            for (u32 k = 0; k < EACH; ++k)
                if (k < at % EACH) sum0 += part[k], same0 += same[k];
            found_sum = sum0;
            found_count = same0;
        }
        __syncthreads();
        const double sum1 = found_sum;
        const u32 same1 = found_count;
        __syncthreads();
        if (wave == at % WAVES) {
            const u32 r = at / WAVES;
            Pack<T, V> x = fetch(r);
            cut(r, x);
            double part[V], sum = 0.0;
            u32 same[V], sames = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float l = (float)x.v[i];
                const bool in = l >= last && some(l);
                part[i] = in && (!TIES || l > last) ? amount(l) : 0.0;
                same[i] = TIES && in && l == last;
                sum += part[i];
                sames += same[i];
            }
            double s = sum1 + (scan_wave(sum) - sum);
            u32 m = TIES ? same1 + scan_wave(sames) - sames : 0;
            int hit = -1, latest = -1;
            double hit_amount = 0.0, latest_amount = 0.0;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (any_of(part[i], same[i], m)) {
                    latest = i;
                    latest_amount = same[i] ? one : part[i];
                    if (hit < 0 && value(s + part[i], m + same[i]) > wanted) hit = i, hit_amount = latest_amount;
                }
                s += part[i];
                m += same[i];
            }
            const u64 hits = __ballot(hit >= 0), some_here = __ballot(latest >= 0);
            const u32 chosen = hits ? (u32)__ffsll((unsigned long long)hits) - 1 : 63 - (u32)__clzll((long long)(some_here | 1));
            if (lane == chosen) {
                found[2] = at_of(r) + (hits ? hit : max(latest, 0));
                found_sum = hits ? hit_amount : latest_amount;
            }
        }
        __syncthreads();
        prob = found_sum / all;
        return found[2];
    };
    constexpr std::integral_constant<int, 0> SPARSE;
    constexpr std::integral_constant<int, 1> MOST;
    constexpr std::integral_constant<int, 2> ALL;  // there is no last one

    u64 *const list = mass, *const weight = mass + LISTED;  // tokens by their order: key, then the lower id; weights by rank
    auto entry = [](u32 id, float l) { return (u64)key_of(l) << 32 | (u32)~id; };
    auto enlist = [&](u32 id, float l) {
        const u32 at = atomicAdd(&n_list + zero, 1u);
        if (at < LISTED) list[at] = entry(id, l);
    };
    // Sorts `size` (a power of two) numbers, largest first.
    auto sort = [&](u32 size) {
        if (size <= 256) {  // by counting the larger ones, several threads to a number; they all differ but for the zeros behind them
            const u32 parts = THREADS / size, at = threadIdx.x / parts, part = threadIdx.x % parts;
            const u64 x = list[at];
            u32 rank = 0;
            for (u32 i = part; i < size; i += parts) rank += list[i] > x || (list[i] == x && i < at);
            for (u32 o = 1; o < parts; o *= 2) rank += __shfl_xor(rank, o);
            __syncthreads();
            if (!part) list[rank] = x;
            __syncthreads();
            return;
        }
        // by exchanges; those less than 128 apart stay within what a wave does, in its order
        for (u32 k = 2; k <= size; k *= 2)
            for (u32 j = k / 2; j; j /= 2) {
                if (j >= 128) __syncthreads();
                for (u32 i = threadIdx.x; i < size / 2; i += THREADS) {
                    const u32 p = 2 * i - (i & (j - 1)), q = p + j;
                    const u64 x = list[p], y = list[q];
                    if ((x < y) == !(p & k)) list[p] = y, list[q] = x;
                }
                if (j >= 128) {
                    __syncthreads();
                } else {
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    __builtin_amdgcn_wave_barrier();
                }
            }
        __syncthreads();
    };
    // Fills the list up with what comes last and sorts it.
    auto sort_list = [&](u32 n) {
        u32 size = 64;
        while (size < n) size *= 2;
        for (u32 i = n + threadIdx.x; i < size; i += THREADS) list[i] = 0;
        __syncthreads();
        sort(size);
    };

    double prob;
    const bool endless = top == __builtin_inff();  // beside +infinity nothing else counts
    if (temperature <= 0.0f || (limit_k && top_k == 1) || endless) {
        // the largest ones have the same weight: the first of them, or one of the first that the limits leave
        last = top;
        const bool first = temperature <= 0.0f;
        const u32 id = draw(
            SPARSE, [&](float) { return true; }, [&](float) { return 0.0; }, 1.0,
            [&](double n) {
                if (limit_k) n = fmin(n, (double)top_k);
                if (limit_p) n = fmax(ceil((double)top_p * n), 1.0);
                ties = first ? 1 : (u32)n;
                return share((double)ties);
            },
            prob);
        return finish(id, 1.0 / (double)ties);
    }

    if (limit_k && (u32)top_k <= LIST_K) {
        const float inv = (float)(c * (1.0 / (GRAINS / BINS)));
        auto slot = [&](float l) { return (u32)fminf((top - l) * inv, (float)(BINS - 1)); };  // (NaN: the last)
        u32 listed = 0;
        // As many threads as top_k have a logit at or above the top_k-th of the threads' largest, so the top_k are among those: mostly
        // not many more.  If there are, all logits are counted.
        for (u32 attempt = 0; attempt < 2; ++attempt) {
            if (attempt) {
                for (u32 i = threadIdx.x; i < BINS; i += THREADS) count[i] = 0;
                __syncthreads();
                each(LIGHT, [&](u32, const Pack<T, V> &x, u32) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float l = (float)x.v[i];
                        if (may(l)) atomicAdd(&count[slot(l)], 1u);
                    }
                });
            } else if (may(own_top)) {
                atomicAdd(&count[slot(own_top)], 1u);
            }
            __syncthreads();
            u32 n[PER], sum = 0;
#pragma unroll
            for (int k = 0; k < PER; ++k) sum += n[k] = count[PER * threadIdx.x + k];
            u32 all, upto = scan_counts(sum, all) - sum;
            if (threadIdx.x == 0) found[0] = BINS - 1, n_list = 0;
            __syncthreads();
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                if (upto < (u32)top_k && (u32)top_k <= upto + n[k]) found[0] = PER * threadIdx.x + k;
                upto += n[k];
            }
            __syncthreads();
            const u32 bin = found[0];
            const float lo = bin == BINS - 1 ? floor_l : fmaxf(top - (float)(bin + 1) / inv * 1.000001f - reach, floor_l);
            each_of([&](float l) { return l >= lo; },
                    [&](u32 id, float l) {
                        if (slot(l) <= bin) enlist(id, l);
                    });
            __syncthreads();
            listed = n_list;
            if (listed <= LISTED) break;
        }
        if (listed <= LISTED) {
            sort_list(listed);
            // a rank a thread
            const u32 kept = min((u32)top_k, listed), rank = threadIdx.x;
            const u64 own = rank < kept ? list[rank] : 0;
            const float l = value_of((u32)(own >> 32));
            const double w = rank < kept ? weigh(l).w : 0.0;
            // top_p goes by all of them, whatever min_p leaves
            double all, before = scan_sums(w, all) - w;
            const double limit = limit_p ? fmax((double)top_p * all, TINY) : __builtin_inf();
            if (rank < kept) weight[rank] = (u64)__double_as_longlong(before < limit && w >= least ? w : 0.0);
            // by ids
            u32 many = 64;
            while (many < kept) many *= 2;
            __syncthreads();
            if (rank < many) list[rank] = rank < kept ? (u64)(u32)own << 32 | rank : 0;
            if (threadIdx.x == 0) found[0] = ~0u, found[1] = 0;
            __syncthreads();
            sort(many);
            const u64 at = rank < kept ? list[rank] : 0;
            const double part = rank < kept ? __longlong_as_double((long long)weight[(u32)at]) : 0.0;
            const double upto = scan_sums(part, all), wanted = share(all);
            find_ends(part > 0.0 && upto > wanted ? rank : ~0u, part > 0.0 ? rank + 1 : 0);
            __syncthreads();
            if (rank == min(found[0], found[1] - 1)) {
                a.token[row] = (int32_t)~(u32)(at >> 32);
                if (a.prob) a.prob[row] = (float)(part / all);
            }
            return;
        }
        // too many near the border of the top_k
        for (u32 i = threadIdx.x; i < BINS; i += THREADS) mass[i] = 0, count[i] = 0;
        __syncthreads();
    }

    if (limit_k || limit_p) {
        // counts and weights by bins
        each(HEAVY, [&](u32, const Pack<T, V> &x, u32) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float l = (float)x.v[i];
                if (may(l)) {
                    const Weight w = weigh(l);
                    const u32 bin = bin_of(w.n);
                    atomicAdd((unsigned long long *)&mass[bin], (unsigned long long)whole(w.w, bin));
                    if (limit_k) atomicAdd(&count[bin], 1u);
                }
                if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            }
        });
        __syncthreads();
        struct Bins {  // the thread's: what is in each, and in all before each and behind the last
            u64 mass[PER];
            u32 count[PER];
            double upto_mass[PER + 1];
            u32 upto_count[PER + 1];
        };
        double total;
        u32 tokens;
        // m0, c0: what lies above them; bin: that which they are parts of, or ~0.  (A thread's lie in one octave: their sums are exact.)
        static_assert(OCTAVE % PER == 0, "scan_bins");
        auto scan_bins = [&](double m0, u32 c0, u32 bin, double &all, u32 &all_count) {
            Bins b;
            u64 m = 0;
            u32 n = 0;
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                b.mass[k] = mass[PER * threadIdx.x + k], b.count[k] = count[PER * threadIdx.x + k];
                m += b.mass[k], n += b.count[k];
            }
            const u32 octave = bin == ~0u ? PER * threadIdx.x : bin;
            const double own = sum_of(m, octave);
            double before = own;
            u32 before_count = n;
            scan_both(before, all, before_count, all_count);
            before = m0 + (before - own), before_count = c0 + before_count - n;
            m = 0, n = 0;
#pragma unroll
            for (int k = 0; k <= PER; ++k) {
                b.upto_mass[k] = before + sum_of(m, octave), b.upto_count[k] = before_count + n;
                if (k < PER) m += b.mass[k], n += b.count[k];
            }
            return b;
        };
        const Bins bins = scan_bins(0.0, 0, ~0u, total, tokens);
        // Narrows to the last token that counts: with `by_count` the goal_count-th, else the one before which weights sum to less than
        // goal_mass and with which they do not.  Lowers the tokens kept to those up to it; returns the weights up to and with it.
        auto resolve = [&](bool by_count, u32 goal_count, double goal_mass) -> double {
            const auto reached = [&](u32 n, double m) { return by_count ? n >= goal_count : m >= goal_mass; };
            const auto lower = [&](float l, u32 n) {
                if (l > last)
                    last = l, ties = n;
                else if (l == last)
                    ties = min(ties, n);
            };
            // The first bin with which it is reached, and what lies above it; if none is: ~0, or with `inner` (parts of a bin with which
            // it is, but for a rounding) the last that holds something.
            auto find = [&](const Bins &b, bool inner) {
                __syncthreads();
                if (threadIdx.x == 0) found[0] = ~0u, found[1] = 0;
                __syncthreads();
                u32 first = ~0u, end = 0;
#pragma unroll
                for (int k = 0; k < PER; ++k)
                    if (by_count ? b.count[k] != 0 : b.mass[k] != 0) {
                        end = PER * threadIdx.x + k + 1;
                        if (first == ~0u && reached(b.upto_count[k + 1], b.upto_mass[k + 1])) first = end - 1;
                    }
                find_ends(first, inner ? end : 0);
                __syncthreads();
                const u32 bin = inner ? min(found[0], found[1] - 1) : found[0];
#pragma unroll
                for (int k = 0; k < PER; ++k)
                    if (PER * threadIdx.x + k == bin) {
                        found_count = b.upto_count[k];
                        found_sum = b.upto_mass[k];
                    }
                __syncthreads();
                return bin;
            };
            const u32 bin = find(bins, false);
            if (bin == ~0u) return total;  // all of them count
            u32 above_count = found_count;
            double above_mass = found_sum;
            // logits of the bin, and a little beside it
            float lo = fmaxf((float)(top64 - ((bin + 1) * (GRAINS / BINS) + 0.5) / c) - reach, floor_l), hi = (float)(top64 - (bin * (GRAINS / BINS) - 1.0) / c) + reach;
            if (!(c > 0.0)) lo = floor_l, hi = top;
            if (!set_apart && !many) {  // what is kept lies in this bin and above it
                each(LIGHT, [&](u32 at, const Pack<T, V> &x, u32) {
                    if (own_apart > OWN) return;
                    few_of(
                        x, [&](float l) { return l >= lo; },
                        [&](u32 i, float l) {
                            const u64 active = __ballot(true);
                            const u32 place = own_apart + __builtin_amdgcn_mbcnt_hi((u32)(active >> 32), __builtin_amdgcn_mbcnt_lo((u32)active, 0));
                            if (place < OWN) apart[wave * OWN + place] = entry(at + i, l);
                        },
                        [&](u64 active) { own_apart += __popcll(active); });
                });
                set_apart = !__syncthreads_or(own_apart > OWN);
                many = !set_apart;
            }
            auto near_bin = [&](float l) { return __builtin_amdgcn_fmed3f(l, lo, hi) == l; };
            u32 from = 0, to = ~0u;  // keys that are looked at
            for (;;) {
                __syncthreads();
                if (threadIdx.x == 0) n_list = n_bin = 0, key_min = ~0u, key_max = 0;
                __syncthreads();
                const bool again = from || ~to;
                each_of(near_bin, [&](u32 id, float l) {
                    const u32 key = key_of(l);
                    if (!again || (key >= from && key <= to)) enlist(id, l);
                });
                __syncthreads();
                // those that are indeed of the bin, their number and the range of their keys
                u32 n = n_list, low = ~0u, high = 0, mine = 0;
                const bool fits = n <= LISTED;
                auto look = [&](u32 key) {
                    if (bin_of(weigh(value_of(key)).n) != bin) return false;
                    low = min(low, key), high = max(high, key), ++mine;
                    return true;
                };
                if (fits) {
                    for (u32 i = threadIdx.x; i < n; i += THREADS)
                        if (!look((u32)(list[i] >> 32))) list[i] = 0;
                } else {
                    each_of(near_bin, [&](u32, float l) {
                        const u32 key = key_of(l);
                        if (key >= from && key <= to) look(key);
                    });
                }
                if (mine) {
                    atomicMin(&key_min + zero, low);
                    atomicMax(&key_max + zero, high);
                    atomicAdd(&n_bin + zero, mine);
                }
                __syncthreads();
                const u32 members = n_bin;
                from = key_min, to = key_max;
                if (from == to) {  // equal ones: so many of them
                    const float l = value_of(from);
                    const double w = weigh(l).w;
                    // the smallest m with above + m w >= goal
                    const double m = by_count ? (double)(goal_count - above_count) : ceil((goal_mass - above_mass) / w);
                    const u32 n = (u32)fmin(fmax(m, 1.0), (double)members);
                    lower(l, n);
                    return above_mass + n * w;
                }
                if (fits) {  // in their order
                    if (threadIdx.x == 0) found[0] = ~0u;
                    sort_list(n);
                    constexpr u32 EACH = LISTED / THREADS;
                    double w[EACH], m = 0.0;
#pragma unroll
                    for (u32 k = 0; k < EACH; ++k) {
                        const u32 rank = threadIdx.x * EACH + k;
                        m += w[k] = rank < members ? weigh(value_of((u32)(list[rank] >> 32))).w : 0.0;
                    }
                    double all, upto[EACH], sum = above_mass + (scan_sums(m, all) - m);
                    u32 hit = ~0u;
#pragma unroll
                    for (u32 k = 0; k < EACH; ++k) {
                        const u32 rank = threadIdx.x * EACH + k;
                        upto[k] = sum += w[k];
                        if (hit == ~0u && rank < members && reached(above_count + rank + 1, sum)) hit = rank;
                    }
                    find_ends(hit, 0);
                    __syncthreads();
                    const u32 rank = min(found[0], members - 1), key = (u32)(list[rank] >> 32);
#pragma unroll
                    for (u32 k = 0; k < EACH; ++k)
                        if (threadIdx.x * EACH + k == rank) found_sum = upto[k];
                    __syncthreads();
                    // its place among its equals: the first of them by halves
                    u32 first = 0, end = rank;
                    while (first < end) {
                        const u32 mid = (first + end) / 2;
                        if ((u32)(list[mid] >> 32) > key)
                            first = mid + 1;
                        else
                            end = mid;
                    }
                    lower(value_of(key), rank - first + 1);
                    return found_sum;
                }
                // by bins of their keys
                u32 shift = 0;
                while ((to - from) >> shift >= BINS) ++shift;
                for (u32 i = threadIdx.x; i < BINS; i += THREADS) mass[i] = 0, count[i] = 0;
                __syncthreads();
                each_of(near_bin, [&](u32, float l) {
                    const u32 key = key_of(l);
                    const Weight w = weigh(l);
                    if (bin_of(w.n) != bin || key < from || key > to) return;
                    atomicAdd((unsigned long long *)&mass[(to - key) >> shift], (unsigned long long)whole(w.w, bin));
                    atomicAdd(&count[(to - key) >> shift], 1u);
                });
                __syncthreads();
                double all;
                u32 all_count;
                const u32 part = min(find(scan_bins(above_mass, above_count, bin, all, all_count), true), BINS - 1);
                above_count = found_count;
                above_mass = found_sum;
                to -= part << shift;
                const u32 width = (1u << shift) - 1;
                from = to - from > width ? to - width : from;
            }
        };
        // No more tokens and weights than these reach min_p: a limit that they keep to leaves them all.
        double likely_mass = __builtin_inf();
        u32 likely = ~0u;
        if (least > 0.0) {
            const u32 bin = bin_of((u32)(-least_log * GRAIN) + 3);
            __syncthreads();
#pragma unroll
            for (int k = 0; k < PER; ++k)
                if (PER * threadIdx.x + k == bin) found_sum = bins.upto_mass[k + 1], found[0] = bins.upto_count[k + 1];
            __syncthreads();
            likely_mass = found_sum;
            likely = found[0];
        }
        // (Where top_p follows, it goes by the sum of the top_k.)
        if (limit_k && (u32)top_k < (limit_p ? tokens : min(tokens, likely))) total = resolve(true, (u32)top_k, 0.0);
        const double goal = fmax((double)top_p * total, TINY);
        if (limit_p && !(likely_mass <= goal)) resolve(false, 0, goal);
    }
    const double w_last = weigh(last).w, one = w_last >= least ? w_last : 0.0;
    const auto weight_of = [&](float l) { return weigh(l).w; };
    u32 id;
    if (least > 0.0 || (!many && (last > floor_l || ties != ~0u))) {
        id = draw(
            SPARSE, [&](float l) { return l >= enough; },
            [&](float l) {
                const double w = weigh(l).w;
                return w >= least ? w : 0.0;
            },
            one, share, prob);
    } else if (last > floor_l || ties != ~0u) {
        id = draw(MOST, may, weight_of, one, share, prob);
    } else {
        id = draw(ALL, may, weight_of, 0.0, share, prob);
    }
    finish(id, prob);
}

template <class T>
static int launch_sample(SampleArgs a, u32 rows, hipStream_t st) {
    constexpr u32 V = 8, ROWS = 1u << 21;  // rows of a launch, which has fewer than 2^32 threads
    for (; a.row0 < rows; a.row0 += ROWS) {
        const u32 n = std::min(rows - a.row0, ROWS);
        if (a.vocab < V)
            hipLaunchKernelGGL((sample_kernel<T, 256, 1>), dim3(n), dim3(256), 0, st, a);
        else if (a.vocab <= 256 * V * 4)
            hipLaunchKernelGGL((sample_kernel<T, 256, V>), dim3(n), dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((sample_kernel<T, 1024, V>), dim3(n), dim3(1024), 0, st, a);
        CKKS_LAUNCH_CHECK("sample_kernel");
    }
    return CKKS_OK;
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
    return p->dtype == CKKS_CLEAR_F32   ? launch_sample<float>(a, n, st)
           : p->dtype == CKKS_CLEAR_F16 ? launch_sample<f16>(a, n, st)
                                        : launch_sample<bf16>(a, n, st);
}
