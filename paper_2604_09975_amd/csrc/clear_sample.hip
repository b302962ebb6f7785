// Draw of the next token: temperature, top-k, top-p, min-p and a given uniform number.  A block takes a row.
//
// What is drawn depends on sums of up to a million weights compared with each other, so a weight is computed in 64 bits and added as a
// whole number of 2^-bits: such sums do not depend on their order, and a token next to the border of two is off by 2^-40 of the sum at
// most.  w = exp((l - max) / T) = 2^(-n / 256) 2^(f / 256) with n whole, |f| <= 1/2: a table of 256 and a polynomial of degree 3
// (r^4 / 24 < 1.4e-13 for r = f ln 2 / 256).  Weights below 2^-64 are none.
//
// The order by logits is not needed, only where the kept tokens end in it: at a value, and after so many of the tokens that have it.
//   top_k of up to 256: the logits are counted by bins of their distance from the largest, those of the bins that hold the top_k are
//     put into a list, and all the rest goes by the list.
//   else: one pass sums counts and weights into bins (2^-1/32 apart).  The bin in which the top_k-th token, or the one that fills
//     top_p, lies is then resolved: tokens of one value by their count, others by sorting them, very many by bins of their values first.
// The draw sums the kept weights by stretches of ids and looks into the one that holds u.
//
// Bound by a weight's 25 instructions or so in 64 bits where each row has a CU, not by the logits' bytes: 256 rows of 131072 bf16 (67 MB,
// 14 us by the bytes) take 37 us with no limit, 33 with top_k 50, which needs no weights but the list's, 129 with top_p 0.9, which needs
// all of them and a border resolved.  A single row has one CU: 50257 logits 13.8 us with a list, 40 with top_p 0.9 alone.
#include <algorithm>
#include <type_traits>

#include "clear_device.h"

namespace ckks {

constexpr u32 BINS = 2048, CHUNKS = 4096;
constexpr u32 LIST_K = 256, LISTED = 2048;  // the largest top_k that goes by a list, and the list's room
constexpr u32 MAX_VOCAB = 1u << 20;
constexpr u32 GRAIN = 256, GRAINS = 64 * GRAIN;  // steps of n: 2^-1/256; weights below 2^-64 are none

struct SampleArgs {
    const void *logits;
    int32_t *token;
    float *prob;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    i64 stride;
    u32 vocab, bits;
};

// Inclusive sums over the lanes of a wave: by DPP within rows of 16, then from row to row.
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 add_dpp(u64 x) {
    const u32 lo = (u32)__builtin_amdgcn_update_dpp(0, (int)(u32)x, CTRL, ROWS, 0xf, false);
    const u32 hi = (u32)__builtin_amdgcn_update_dpp(0, (int)(u32)(x >> 32), CTRL, ROWS, 0xf, false);
    return x + ((u64)hi << 32 | lo);
}
__device__ __forceinline__ u64 scan_wave(u64 x) {
    x = add_dpp<0x111, 0xf>(x);  // row_shr 1, 2, 4, 8
    x = add_dpp<0x112, 0xf>(x);
    x = add_dpp<0x114, 0xf>(x);
    x = add_dpp<0x118, 0xf>(x);
    x = add_dpp<0x142, 0xa>(x);  // row_bcast 15, 31
    return add_dpp<0x143, 0xc>(x);
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
    __shared__ __attribute__((aligned(16))) u64 mass[CHUNKS];  // weights of the bins; of stretches of ids; lists
    __shared__ u32 count[CHUNKS];                              // tokens of the bins; of stretches of ids that have the last value
    __shared__ u64 apart[APART];                               // tokens set apart, those that all later passes are about
    __shared__ double power[GRAIN];                            // 2^(j / 256)
    __shared__ u64 wave_sums[WAVES];
    __shared__ u32 n_list, n_bin, key_min, key_max;
    __shared__ u32 found[4];
    __shared__ u64 found64[2];
    __shared__ float wave_top[WAVES];

    const u32 row = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
    // Inclusive sums over the threads.
    auto scan_block = [&](u64 x) {
        x = scan_wave(x);
        __syncthreads();
        if (lane == 63) wave_sums[wave] = x;
        __syncthreads();
        u64 before = 0;
#pragma unroll
        for (u32 w = 0; w < WAVES; ++w) before += w < wave ? wave_sums[w] : 0;
        return x + before;
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
    // Logits that may have a weight; false for NaN and -infinity.  (A little below, so that it does not cut off what `weigh` counts.)
    const float floor_l = fmaxf((float)(top64 - (GRAINS + 8.0) / c * (1 + 1e-6)), -3.402823466e38f);
    auto may = [&](float l) { return l >= floor_l; };
    const float reach = 1e-6f * fabsf(top);  // more than bounds that are worked out in 32 bits are off by
    // n: steps down from the largest; w = 2^(-n / 256) 2^(f / 256).  NaN and all that is far below: n = GRAINS + 64.
    struct Weight {
        u32 n;
        double w;
    };
    auto weigh = [&](float l) {
        constexpr double ROUND = 6755399441055744.0, STEP = 0.69314718055994530942 / GRAIN;  // 1.5 * 2^52: n in the lower word of the sum
        const double t = fmax(((double)l - top64) * c, -(double)(GRAINS + 64)), s = t + ROUND, f = t - (s - ROUND);
        const double q = f * __builtin_fma(f, __builtin_fma(f, STEP * STEP * STEP / 6, STEP * STEP / 2), STEP);
        const int n = (int)(u32)__double_as_longlong(s);
        const u64 e = (u64)__double_as_longlong(power[n & (GRAIN - 1)]) + ((u64)(u32)((n >> 8) << 20) << 32);
        const double p = __longlong_as_double((long long)e);
        return Weight{(u32)-n, __builtin_fma(p, q, p)};
    };
    static_assert(GRAIN == 256, "n >> 8");
    auto bin_of = [&](u32 n) { return n / (GRAINS / BINS); };
    // (0 from 2^-52 on, as `bits` is 51 at most)
    auto whole = [&](double w) { return (u64)__double_as_longlong(w + magic) & ((1ull << 52) - 1); };
    // What u asks for of a sum.
    auto share = [&](u64 sum) -> u64 { return u < 1.0f ? min((u64)(fmax((double)u, 0.0) * (double)sum), sum - 1) : u >= 1.0f ? sum - 1 : 0ull; };

    // Kept are the tokens above `last`, and of those that have it the `ties` with the lowest ids.
    float last = floor_l;
    u64 ties = ~0ull;

    // The lowest id up to which amounts sum to more than goal(all of them): amount(logit) where `some` holds, and `one` for each of the
    // first `ties` tokens of value `last` (for which `some` need not hold).  `dense`: how many logits have an amount.  prob: the
    // token's share.
    auto draw = [&](auto dense, auto some, auto amount, u64 one, auto goal, double &prob) -> u32 {
        constexpr bool DENSE = decltype(dense)::value > 0, TIES = decltype(dense)::value < 2;
        auto value = [&](u64 sum, u64 n) { return sum + min(n, ties) * one; };
        const u32 n = rounds * WAVES;  // a chunk: what a wave takes in a round, 64 V ids
        __syncthreads();
        if (!DENSE && set_apart) {
            for (u32 i = threadIdx.x; i < n; i += THREADS) mass[i] = 0, count[i] = 0;
            __syncthreads();
            each_of([&](float l) { return l >= last && some(l); }, [&](u32 id, float l) {
                if (l > last)
                    atomicAdd((unsigned long long *)&mass[id / (64 * V)], (unsigned long long)amount(l));
                else
                    atomicAdd(&count[id / (64 * V)], 1u);
            });
        } else each(std::integral_constant<u32, DENSE ? 2 : 4>(), [&](u32, const Pack<T, V> &x, u32 r) {
            u64 sum = 0;
            u32 same = 0;
            if (DENSE) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float l = (float)x.v[i];
                    const u64 w = amount(l);
                    sum += !TIES || l > last ? w : 0;
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
            if (DENSE || __any(sum != 0)) sum = scan_wave(sum);
            if (TIES && __any(same != 0)) same = (u32)scan_wave(same);
            if (lane == 63) {
                mass[r * WAVES + wave] = sum;
                count[r * WAVES + wave] = same;
            }
        });
        __syncthreads();
        constexpr u32 EACH = THREADS == 1024 ? CHUNKS / THREADS : 1;  // chunks a thread
        u64 part[EACH], sum = 0;
        u32 same[EACH], sames = 0;
#pragma unroll
        for (u32 k = 0; k < EACH; ++k) {
            const u32 at = threadIdx.x * EACH + k;
            part[k] = at < n ? mass[at] : 0;
            same[k] = at < n ? count[at] : 0;
            sum += part[k];
            sames += same[k];
        }
        u64 sum0 = scan_block(sum);
        u64 same0 = scan_block(sames);
        if (threadIdx.x == THREADS - 1) found64[0] = value(sum0, same0);
        sum0 -= sum;
        same0 -= sames;
        __syncthreads();
        const u64 all = found64[0], wanted = goal(all);
        __syncthreads();
#pragma unroll
        for (u32 k = 0; k < EACH; ++k) {
            if (value(sum0, same0) <= wanted && wanted < value(sum0 + part[k], same0 + same[k])) {
                found[0] = threadIdx.x * EACH + k;
                found64[0] = sum0;
                found64[1] = same0;
            }
            sum0 += part[k];
            same0 += same[k];
        }
        __syncthreads();
        const u32 at = min(found[0], n - 1);
        const u64 sum1 = found64[0], same1 = found64[1];
        __syncthreads();
        if (wave == at % WAVES) {
            const u32 r = at / WAVES;
            Pack<T, V> x = fetch(r);
            cut(r, x);
            u64 part[V], sum = 0;
            u32 same[V], sames = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float l = (float)x.v[i];
                const bool in = l >= last && some(l);
                part[i] = in && (!TIES || l > last) ? amount(l) : 0;
                same[i] = TIES && in && l == last;
                sum += part[i];
                sames += same[i];
            }
            u64 s = sum1 + scan_wave(sum) - sum, m = same1 + scan_wave(sames) - sames;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const u64 before = value(s, m), after = value(s + part[i], m + same[i]);
                if (before <= wanted && wanted < after) {
                    found[1] = at_of(r) + i;
                    found64[0] = after - before;
                }
                s += part[i];
                m += same[i];
            }
        }
        __syncthreads();
        prob = (double)found64[0] / (double)all;
        return found[1];
    };
    constexpr std::integral_constant<int, 0> SPARSE;
    constexpr std::integral_constant<int, 1> MOST;
    constexpr std::integral_constant<int, 2> ALL;  // there is no last one

    u64 *const list = mass, *const weight = mass + LISTED;  // tokens by their order: key, then the lower id; weights by rank
    auto entry = [](u32 id, float l) { return (u64)key_of(l) << 32 | (u32)~id; };
    // Few lanes at a time have a token for the list: each adds 1 for itself.  (An address that the compiler knows to be one for all
    // lanes makes it sum over the wave first, which takes ten times as long.)
    u32 zero = 0;
    asm volatile("" : "+v"(zero));
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
            SPARSE, [&](float) { return true; }, [&](float) { return 0ull; }, 1,
            [&](u64 n) {
                if (limit_k) n = min(n, (u64)top_k);
                if (limit_p) n = (u64)fmax(ceil((double)top_p * (double)n), 1.0);
                ties = first ? 1 : n;
                return share(ties);
            },
            prob);
        return finish(id, ties == ~0ull ? 1.0 : 1.0 / (double)ties);
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
            u32 upto = (u32)scan_block(sum) - sum;
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
            // consecutive ranks a thread
            constexpr u32 EACH = 1;
            const u32 kept = min((u32)top_k, listed);
            u64 w[EACH], sum = 0;
            u32 id[EACH];
#pragma unroll
            for (u32 k = 0; k < EACH; ++k) {
                const u32 rank = threadIdx.x * EACH + k;
                const u64 at = rank < kept ? list[rank] : 0;
                id[k] = ~(u32)at;
                const Weight x = weigh(value_of((u32)(at >> 32)));
                w[k] = rank < kept && x.w >= least ? whole(x.w) : 0;
                // top_p goes by all of them, whatever min_p leaves
                sum += rank < kept ? whole(x.w) : 0;
            }
            u64 before = scan_block(sum);
            if (threadIdx.x == THREADS - 1) found64[0] = before;
            before -= sum;
            __syncthreads();
            const double limit = limit_p ? fmax((double)top_p * (double)found64[0], 0.5) : __builtin_inf();
            sum = 0;
#pragma unroll
            for (u32 k = 0; k < EACH; ++k) {
                const u32 rank = threadIdx.x * EACH + k;
                const u64 own = rank < kept ? whole(weigh(value_of((u32)(list[rank] >> 32))).w) : 0;
                if (!((double)before < limit)) w[k] = 0;
                before += own;
                sum += w[k];
                if (rank < kept) weight[rank] = w[k];
            }
            __syncthreads();
            // by ids
            u32 many = 64;
            while (many < kept) many *= 2;
#pragma unroll
            for (u32 k = 0; k < EACH; ++k) {
                const u32 rank = threadIdx.x * EACH + k;
                if (rank < many) list[rank] = rank < kept ? (u64)(u32)~id[k] << 32 | rank : 0;
            }
            __syncthreads();
            sort(many);
            sum = 0;
#pragma unroll
            for (u32 k = 0; k < EACH; ++k) {
                const u32 rank = threadIdx.x * EACH + k;
                const u64 at = rank < kept ? list[rank] : 0;
                id[k] = ~(u32)(at >> 32);
                w[k] = rank < kept ? weight[(u32)at] : 0;
                sum += w[k];
            }
            before = scan_block(sum);
            if (threadIdx.x == THREADS - 1) found64[0] = before;
            before -= sum;
            __syncthreads();
            const u64 all = found64[0], wanted = share(all);
#pragma unroll
            for (u32 k = 0; k < EACH; ++k) {
                if (before <= wanted && wanted < before + w[k]) {
                    a.token[row] = (int32_t)id[k];
                    if (a.prob) a.prob[row] = (float)((double)w[k] / (double)all);
                }
                before += w[k];
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
                    if (w.n < GRAINS) {
                        atomicAdd((unsigned long long *)&mass[bin_of(w.n)], (unsigned long long)whole(w.w));
                        if (limit_k) atomicAdd(&count[bin_of(w.n)], 1u);
                    }
                }
                if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            }
        });
        __syncthreads();
        struct Bins {  // the thread's: what is in each, and in all up to each
            u64 mass[PER], upto_mass[PER];
            u32 count[PER], upto_count[PER];
        };
        auto scan_bins = [&](u64 m0, u32 c0) {  // m0, c0: what lies above them
            Bins b;
            u64 m = 0;
            u32 n = 0;
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                b.mass[k] = mass[PER * threadIdx.x + k], b.count[k] = count[PER * threadIdx.x + k];
                m += b.mass[k], n += b.count[k];
            }
            m = m0 + scan_block(m) - m;
            n = c0 + (u32)scan_block(n) - n;
#pragma unroll
            for (int k = 0; k < PER; ++k) b.upto_mass[k] = m += b.mass[k], b.upto_count[k] = n += b.count[k];
            return b;
        };
        const Bins bins = scan_bins(0, 0);
        if (threadIdx.x == THREADS - 1) {
            found64[0] = bins.upto_mass[PER - 1];
            found[0] = bins.upto_count[PER - 1];
        }
        __syncthreads();
        u64 total = found64[0];
        const u32 tokens = found[0];
        // Narrows to the last token that counts: with `by_count` the goal_count-th, else the one before which weights sum to less than
        // goal_mass and with which they do not.  Lowers the tokens kept to those up to it; returns the weights up to and with it.
        auto resolve = [&](bool by_count, u64 goal_count, double goal_mass) -> u64 {
            const auto reached = [&](u64 n, u64 m) { return by_count ? n >= goal_count : (double)m >= goal_mass; };
            const auto lower = [&](float l, u64 n) {
                if (l > last)
                    last = l, ties = n;
                else if (l == last)
                    ties = min(ties, n);
            };
            auto find = [&](const Bins &b) {
                __syncthreads();
                if (threadIdx.x == 0) found[0] = ~0u;
                __syncthreads();
#pragma unroll
                for (int k = 0; k < PER; ++k) {
                    const u32 n = b.upto_count[k] - b.count[k];
                    const u64 m = b.upto_mass[k] - b.mass[k];
                    if (reached(b.upto_count[k], b.upto_mass[k]) && !reached(n, m)) {
                        found[0] = PER * threadIdx.x + k;
                        found[1] = n;
                        found64[0] = m;
                    }
                }
                __syncthreads();
            };
            find(bins);
            const u32 bin = found[0];
            u64 above_count = found[1], above_mass = found64[0];
            if (bin == ~0u) return total;  // all of them count
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
                    atomicMin(&key_min, low);
                    atomicMax(&key_max, high);
                    atomicAdd(&n_bin, mine);
                }
                __syncthreads();
                const u32 members = n_bin;
                from = key_min, to = key_max;
                if (from == to) {  // equal ones: so many of them
                    const float l = value_of(from);
                    const u64 w = whole(weigh(l).w);
                    u64 m;
                    if (by_count) {
                        m = goal_count - above_count;
                    } else {  // the smallest m with above + m w >= goal
                        m = w ? (u64)((goal_mass - (double)above_mass) / (double)w) : 1;
                        while (m > 1 && (double)(above_mass + (m - 1) * w) >= goal_mass) --m;
                        while (m < members && (double)(above_mass + m * w) < goal_mass) ++m;
                    }
                    m = min(max(m, 1ull), (u64)members);
                    lower(l, m);
                    return above_mass + m * w;
                }
                if (fits) {  // in their order
                    sort_list(n);
                    constexpr u32 EACH = LISTED / THREADS;
                    u64 w[EACH], m = 0;
#pragma unroll
                    for (u32 k = 0; k < EACH; ++k) {
                        const u32 rank = threadIdx.x * EACH + k;
                        m += w[k] = rank < members ? whole(weigh(value_of((u32)(list[rank] >> 32))).w) : 0;
                    }
                    u64 before = above_mass + scan_block(m) - m;
#pragma unroll
                    for (u32 k = 0; k < EACH; ++k) {
                        const u32 rank = threadIdx.x * EACH + k;
                        const u64 at = above_count + rank;
                        if (rank < members && !reached(at, before) && reached(at + 1, before + w[k])) {
                            found[2] = rank;
                            found64[1] = before + w[k];
                        }
                        before += w[k];
                    }
                    __syncthreads();
                    // its place among its equals: the first of them by halves
                    const u32 rank = min(found[2], members - 1), key = (u32)(list[rank] >> 32);
                    u32 first = 0, end = rank;
                    while (first < end) {
                        const u32 mid = (first + end) / 2;
                        if ((u32)(list[mid] >> 32) > key)
                            first = mid + 1;
                        else
                            end = mid;
                    }
                    lower(value_of(key), rank - first + 1);
                    return found64[1];
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
                    atomicAdd((unsigned long long *)&mass[(to - key) >> shift], (unsigned long long)whole(w.w));
                    atomicAdd(&count[(to - key) >> shift], 1u);
                });
                __syncthreads();
                find(scan_bins(above_mass, (u32)above_count));
                above_count = found[1];
                above_mass = found64[0];
                to -= min(found[0], BINS - 1) << shift;
                const u32 width = (1u << shift) - 1;
                from = to - from > width ? to - width : from;
            }
        };
        // No more tokens and weights than these reach min_p: a limit that they keep to leaves them all.
        u64 likely_mass = ~0ull;
        u32 likely = ~0u;
        if (least > 0.0) {
            // (the logarithm of the hardware takes a subnormal as 0; and no weight is below 2^-64)
            const u32 bin = min(bin_of((u32)(-__log2f(fmaxf((float)least, 0x1p-64f)) * GRAIN) + 3), BINS - 1);
            __syncthreads();
#pragma unroll
            for (int k = 0; k < PER; ++k)
                if (PER * threadIdx.x + k == bin) found64[0] = bins.upto_mass[k], found[0] = bins.upto_count[k];
            __syncthreads();
            likely_mass = found64[0];
            likely = found[0];
        }
        // (Where top_p follows, it goes by the sum of the top_k.)
        if (limit_k && (u32)top_k < (limit_p ? tokens : min(tokens, likely))) total = resolve(true, (u64)top_k, 0.0);
        const double goal = fmax((double)top_p * (double)total, 0.5);
        if (limit_p && !((double)likely_mass <= goal)) resolve(false, 0, goal);
    }
    u32 id;
    const double w_last = weigh(last).w;
    const u64 one = w_last >= least ? whole(w_last) : 0ull;
    if (least > 0.0 || (!many && (last > floor_l || ties != ~0ull))) {
        // logits that may reach min_p, and a little below
        const float enough = least > 0.0 ? (float)(top64 + (__log2f(fmaxf((float)least, 0x1p-64f)) * GRAIN - 1.0) / c) - reach : last;
        id = draw(
            SPARSE, [&](float l) { return !(l < enough); },
            [&](float l) -> u64 {
                const double w = weigh(l).w;
                return w >= least ? whole(w) : 0ull;
            },
            one, share, prob);
    } else if (last > floor_l || ties != ~0ull) {
        id = draw(MOST, may, [&](float l) { return whole(weigh(l).w); }, one, share, prob);
    } else {
        id = draw(ALL, may, [&](float l) { return whole(weigh(l).w); }, 0, share, prob);
    }
    finish(id, prob);
}

template <class T>
static void launch_sample(const SampleArgs &a, u32 rows, hipStream_t st) {
    constexpr u32 V = 8;
    if (a.vocab < V)
        hipLaunchKernelGGL((sample_kernel<T, 256, 1>), dim3(rows), dim3(256), 0, st, a);
    else if (a.vocab <= 256 * V * 4)
        hipLaunchKernelGGL((sample_kernel<T, 256, V>), dim3(rows), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((sample_kernel<T, 1024, V>), dim3(rows), dim3(1024), 0, st, a);
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
