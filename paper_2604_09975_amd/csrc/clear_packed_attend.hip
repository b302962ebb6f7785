// Attention over pages of 8 bits.  Chunks go through the kernels of clear_attend.hip: codes are brought to the queries' type, exactly, on
// their way into LDS, and from there on nothing differs.  Few rows over heads of up to 128 have a kernel of their own.
// Chunks are bound by the matrix products and, between them, by what a weight costs: 2 x 4096 tokens of 32 heads of 128 over up to 12301
// keys take 1370 to 1490 us with E4M3 (0.96 to 0.89 PFLOP/s), 1540 to 1655 with I8, 1300 over a plain bf16 cache.  Their weights are rounded to the type
// before the second product, as there and for the same reason: the error against 64 bits is 0.0021 of the result where one rounding of
// it alone gives 0.0017.
#include "clear_attend_device.h"

namespace ckks {

typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// What codes become in the matrix products over few rows: F16 for F16, else BF16, which holds every code times a power of two down to 2^-133.  A 32-bit
// number goes into them as three of 8 bits, a softmax weight of the 16-bit types as two.
template <class T>
struct Thin {
    typedef bf16 type;
    static constexpr int Q = 1, W = 2;
};
template <>
struct Thin<f16> {
    typedef f16 type;
    static constexpr int Q = 1, W = 2;
};
template <>
struct Thin<float> {
    typedef bf16 type;
    static constexpr int Q = 3, W = 3;
};

// The largest (the sum) over the four lanes that hold a row, all 16 apart.
__device__ __forceinline__ float row_max(float x) {
    const auto far = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(far[0]), __uint_as_float(far[1]));
    const auto near = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(near[0]), __uint_as_float(near[1]));
}
__device__ __forceinline__ float row_sum(float x) {
    const auto far = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(far[0]) + __uint_as_float(far[1]);
    const auto near = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(near[0]) + __uint_as_float(near[1]);
}

// Few rows (16: the query heads of a kv head, of one token or a few) over pages of 8 bits; each of KW waves takes every KW-th tile of
// 32 keys by itself, as in attend_kernel.  S^T = K Q^T and O^T = V^T P^T as there, by products of 16 x 16 with depth 32:
//   keys: lane l holds a quarter of key l % 16's codes, quarter l / 16, side by side as they lie in the page.  The depth is taken in that
//     order (step s: bytes 8 s .. of each quarter), so codes go from the page to registers to the product, without LDS;
//   scores: lane l has row l % 16, keys 4 (l / 16) + i and 16 more;
//   values: expanded with their powers on the way into LDS, read back by columns for the very keys that the lane has weights of.
// Bound by memory.  64 tokens over up to 8192 keys of 8 heads of 128 (617 MB) take 131 us, 4.7 TB/s, and no less without any of the
// arithmetic; I8, whose codes take two instructions each to expand, 162.  attend_kernel's waves-apart form took 231 over a plain cache, of
// twice the bytes.  One tile a wave is in flight at 3 waves a SIMD: with two at 2 waves 156 us where this took 146, at 4 waves
// registers spill (169).  One sequence of 131001 keys (2 heads of 128, 69 MB) is bound by its start, the joining launch and the
// waves' last tiles: 24 us and 5 where the bytes take 14.  (One wave on a SIMD waits for each of its eight tiles; two tiles under way have not been
// measured there.)
// WHOLE: pages hold whole tiles.
template <class T, int FORM, int DP, bool WHOLE, int KW, int OCC>
__global__ __launch_bounds__(64 * KW, OCC) void attend_thin_kernel(PackedAttendArgs a) {
    typedef typename Thin<T>::type C;
    typedef typename Frag<C>::type frag;
    constexpr float LIFT = Frag<C>::LIFT, LAG = Frag<C>::LAG;
    constexpr int NQ = Thin<T>::Q, NW = Thin<T>::W, TK = 32, ROWS = 16, STEPS = DP / 32, DT = DP / 16;
    constexpr int QUARTER = DP / 4;                      // bytes of a key that a lane holds
    constexpr int VS = DP + 32;                          // entries between rows of values in LDS
    constexpr int LANES = DP / 16, PASS = 64 / LANES, PASSES = TK / PASS;  // values: lanes to a row, 16 bytes each; rows at a time
    constexpr size_t STAGE = (size_t)KW * TK * VS * 2, JOIN = (size_t)KW * ROWS * (DP + 2) * 4;
    __shared__ __attribute__((aligned(16))) unsigned char lds[STAGE > JOIN ? STAGE : JOIN];

    const u32 lane = threadIdx.x & 63, kw = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4;
    const u32 kv_head = blockIdx.x % a.kv_heads, split = blockIdx.x / a.kv_heads % a.splits;
    RowTile r;
    if (!find_tile<ROWS>(a, a.tiles - 1 - blockIdx.x / a.kv_heads / a.splits, r)) return;
    key_range<ROWS, TK>(a, a.kv_len[r.seq], r);
    r.kv = __builtin_amdgcn_readfirstlane(r.kv);
    r.t0 = __builtin_amdgcn_readfirstlane(r.t0);
    r.tile0 = __builtin_amdgcn_readfirstlane(r.tile0);
    r.n_tiles = __builtin_amdgcn_readfirstlane(r.n_tiles);
    r.per = __builtin_amdgcn_readfirstlane(r.per);
    r.n_splits = __builtin_amdgcn_readfirstlane(r.n_splits);
    if (split >= r.n_splits) return;
    const u32 first = split * r.per, last = min(first + r.per, r.n_tiles);

    const u32 row = min(r.first_row + (lane & 15), r.rows - 1), token = row / a.group, head = kv_head * a.group + row % a.group;
    const int pos = max(r.t0 + (int)token, -1);
    // keys lo <= j < hi are seen; all_lo, all_hi: by all rows
    const int hi = a.causal ? min(r.kv, pos + 1) : r.kv, lo = a.window ? max(pos - a.window + 1, 0) : 0;
    const int p_first = row_pos(a, r, r.first_row), p_last = row_pos(a, r, min(r.first_row + ROWS, r.rows) - 1);
    const int all_hi = a.causal ? min(r.kv, p_first + 1) : r.kv, all_lo = a.window ? max(p_last - a.window + 1, 0) : 0;

    frag qf[NQ][STEPS];
    {
        const T *q = (const T *)a.q + (i64)(r.start + token) * a.qs[0] + head * a.qs[1];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const u32 d = quarter * QUARTER + 8 * s;
            Pack<T, 8> x{};
            if (d < a.head_dim) x = load_pack<8>(q + d);
            if constexpr (NQ == 1) {
                __builtin_memcpy(&qf[0][s], &x, 16);
            } else {
                // cut, not rounded: the parts are exact, and none is infinite where the number is not
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float x0 = x.v[i], x1 = __uint_as_float(__float_as_uint(x0) & 0xffff0000u), y = is_finite(x0) ? x0 - x1 : 0.0f;
                    const float x2 = __uint_as_float(__float_as_uint(y) & 0xffff0000u);
                    qf[0][s][i] = (C)x1;
                    qf[1][s][i] = (C)x2;
                    qf[2][s][i] = (C)(y - x2);
                }
            }
        }
    }

    // Where a lane's keys (two, 16 apart) and its pieces of the values' rows lie.
    const u32 key_row = lane & 15, fetch_row = lane / LANES, piece = lane % LANES;
    const bool piece_ok = piece * 16 < a.head_dim;
    constexpr int KP = QUARTER / 16;  // 16-byte pieces of a quarter
    bool k_ok[KP];
#pragma unroll
    for (int h = 0; h < KP; ++h) k_ok[h] = quarter * QUARTER + h * 16 < a.head_dim;
    const u32 k_block = min(quarter * QUARTER, a.head_dim - 1) / PACK_BLOCK, v_block = piece_ok ? piece * 16 / PACK_BLOCK : 0;
    const unsigned char *kp = (const unsigned char *)a.k + (i64)kv_head * a.ks[1], *vp = (const unsigned char *)a.v + (i64)kv_head * a.vs[1];
    const unsigned char *kzp = a.kz + (i64)kv_head * a.kzs[1] + k_block, *vzp = a.vz + (i64)kv_head * a.vzs[1] + v_block;
    const int32_t *table = a.table + (i64)r.seq * a.ts;
    // (a page lies within 2^31 bytes: check_cache)
    const u32 ks2 = (u32)a.ks[2], vs2 = (u32)a.vs[2], kzs2 = (u32)a.kzs[2], vzs2 = (u32)a.vzs[2];
    const u32 k_lane = key_row * ks2 + quarter * QUARTER, v_lane = fetch_row * vs2 + (piece_ok ? piece * 16 : 0), kz_lane = key_row * kzs2, vz_lane = fetch_row * vzs2;
    const bool full = a.head_dim == DP;
    constexpr int NK = WHOLE ? 1 : 2, NV = WHOLE ? 1 : PASSES;
    struct Place {
        u32 k_page[NK], k_row[NK], v_page[NV], v_row[NV];  // of each row; of the tile, where pages hold whole tiles
    };
    auto look_up = [&](u32 tile) {
        Place at;
        const u32 j0 = (r.tile0 + tile) * TK;
        auto one = [&](u32 j, u32 &page, u32 &row) {
            const u32 n = __umulhi(2 * j, a.page_mul) >> a.page_shift;
            page = (u32)table[n];
            row = j - n * a.page_size;
        };
        if constexpr (WHOLE) {
            one(min(j0, ((u32)r.kv - 1) / TK * TK), at.k_page[0], at.k_row[0]);
        } else {
#pragma unroll
            for (int u = 0; u < 2; ++u) one(min(j0 + 16 * u + key_row, (u32)r.kv - 1), at.k_page[u], at.k_row[u]);
#pragma unroll
            for (int p = 0; p < PASSES; ++p) one(min(j0 + p * PASS + fetch_row, (u32)r.kv - 1), at.v_page[p], at.v_row[p]);
        }
        return at;
    };
    // A tile under way: codes, powers, and a bit for each row that is not there (fetched from page 0, and taken as zeros).
    struct Tile {
        uint4 k[2][KP], v[PASSES];
        u32 kz[2], vz[PASSES], none;
    };
    auto fetch = [&](u32 tile, const Place &at) {
        Tile x;
        x.none = 0;
        const u32 j0 = (r.tile0 + tile) * TK;
        // from a base and the lane's place
        auto k_from = [&](int u, const unsigned char *k, u32 lane, const unsigned char *kz, u32 z_lane) {
#pragma unroll
            for (int h = 0; h < KP; ++h) __builtin_memcpy(&x.k[u][h], k + (lane + (full || k_ok[h] ? h * 16 : 0u - quarter * QUARTER)), 16);
            x.kz[u] = kz[z_lane];
        };
        auto v_from = [&](int p, const unsigned char *v, u32 lane, const unsigned char *vz, u32 z_lane) {
            __builtin_memcpy(&x.v[p], v + lane, 16);
            x.vz[p] = vz[z_lane];
        };
        if constexpr (WHOLE) {
            const u32 page = at.k_page[0] < a.n_pages ? at.k_page[0] : 0, row = at.k_row[0];
            if (at.k_page[0] >= a.n_pages) x.none = ~0u;
            const unsigned char *k = kp + ((u64)page * (u32)a.ks[0] + row * ks2), *kz = kzp + ((u64)page * (u32)a.kzs[0] + row * kzs2);
            const unsigned char *v = vp + ((u64)page * (u32)a.vs[0] + row * vs2), *vz = vzp + ((u64)page * (u32)a.vzs[0] + row * vzs2);
#pragma unroll
            for (int u = 0; u < 2; ++u) k_from(u, k + 16 * u * ks2, k_lane, kz + 16 * u * kzs2, kz_lane);
#pragma unroll
            for (int p = 0; p < PASSES; ++p) v_from(p, v + p * PASS * vs2, v_lane, vz + p * PASS * vzs2, vz_lane);
        } else {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const u32 page = at.k_page[u] < a.n_pages ? at.k_page[u] : 0, row = at.k_row[u];
                if (at.k_page[u] >= a.n_pages) x.none |= 1u << u;
                k_from(u, kp + (u64)page * (u32)a.ks[0], row * ks2 + quarter * QUARTER, kzp + (u64)page * (u32)a.kzs[0], row * kzs2);
            }
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                const u32 page = at.v_page[p] < a.n_pages ? at.v_page[p] : 0, row = at.v_row[p];
                if (at.v_page[p] >= a.n_pages) x.none |= 4u << p;
                v_from(p, vp + (u64)page * (u32)a.vs[0], row * vs2 + (piece_ok ? piece * 16 : 0), vzp + (u64)page * (u32)a.vzs[0], row * vzs2);
            }
        }
        if (j0 + TK > (u32)r.kv) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if (j0 + 16 * u + key_row >= (u32)r.kv) x.none |= 1u << u;
#pragma unroll
            for (int p = 0; p < PASSES; ++p)
                if (j0 + p * PASS + fetch_row >= (u32)r.kv) x.none |= 4u << p;
        }
        return x;
    };

    f32x4 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[d][i] = 0.0f;
    float m = -__builtin_inff(), l = 0.0f;
    f32x4 s[2];
    frag w[NW];
    u32 odd = 0;
    C *vb = (C *)lds + kw * TK * VS;

    // The largest power with which every code that is a number is finite.
    constexpr u32 LARGE = std::is_same<C, f16>::value ? (FORM == E4M3 ? 127 + 7 : 127 + 8) : (FORM == E4M3 ? 127 + 119 : 127 + 120);
    auto k_power = [&](float power, int h) { return full || k_ok[h] ? power : 1.0f; };
    auto score = [&](Tile &x) {
        if (!full)  // what a lane has beyond the head
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int h = 0; h < KP; ++h)
                    if (!k_ok[h]) x.k[u][h] = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (__any(x.none & 3u))
                if (x.none >> u & 1) {
#pragma unroll
                    for (int h = 0; h < KP; ++h) x.k[u][h] = make_uint4(0, 0, 0, 0);
                    x.kz[u] = 0;
                }
        auto products = [&](auto finite) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const float power = power_of<FORM>(x.kz[u]);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[u][i] = 0.0f;
#pragma unroll
                for (int d = 0; d < STEPS; ++d) {
                    C k[8];
                    const uint4 y = x.k[u][d / 2];
                    unpack4<C, FORM>(d % 2 ? y.z : y.x, k_power(power, d / 2), k);
                    unpack4<C, FORM>(d % 2 ? y.w : y.y, k_power(power, d / 2), k + 4);
                    frag f;
                    __builtin_memcpy(&f, k, 16);
                    s[u] = mma16(f, qf[0][d], s[u]);
                    if (decltype(finite)::value) {
                        uint4 z;
                        u32 odd_key = 0;
                        __builtin_memcpy(&z, k, 16);
                        z = finite_part<C>(z, odd_key);
                        __builtin_memcpy(&f, &z, 16);
                    }
#pragma unroll
                    for (int n = 1; n < NQ; ++n) s[u] = mma16(f, qf[n][d], s[u]);
                }
            }
        };
        products(std::false_type());
        // an infinite key is for the query's first part alone: the others may be 0
        if (NQ > 1 && __any(max(x.kz[0], x.kz[1]) > LARGE)) products(std::true_type());
    };
    // An infinity or NaN among the values would meet weights of 0, and here also the rest of a weight, which may be: such values are taken as
    // zeros and come back at the end.  Only large powers give one (and codes that are no number, which matter where some row does not
    // see the tile in full).
    auto put_v = [&](u32 tile, Tile &x) {
        const int j0 = (int)((r.tile0 + tile) * TK);
        u32 large = 0;
        if (__any(x.none >> 2))
#pragma unroll
            for (int p = 0; p < PASSES; ++p)
                if (x.none >> (p + 2) & 1) {
                    x.v[p] = make_uint4(0, 0, 0, 0);
                    x.vz[p] = 0;
                }
#pragma unroll
        for (int p = 0; p < PASSES; ++p) large = max(large, x.vz[p]);
        const bool clean = all_hi - j0 < TK || j0 < all_lo || __any(large > LARGE);
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            C v[16];
            const float power = power_of<FORM>(x.vz[p]);
            unpack4<C, FORM>(x.v[p].x, power, v);
            unpack4<C, FORM>(x.v[p].y, power, v + 4);
            unpack4<C, FORM>(x.v[p].z, power, v + 8);
            unpack4<C, FORM>(x.v[p].w, power, v + 12);
            uint4 y[2];
            __builtin_memcpy(y, v, 32);
            if (clean) y[0] = finite_part<C>(y[0], odd), y[1] = finite_part<C>(y[1], odd);
            uint4 *to = (uint4 *)(vb + (p * PASS + fetch_row) * VS + piece * 16);
            to[0] = y[0];
            to[1] = y[1];
        }
    };
    auto soften = [&](u32 tile) {
        const int j0 = (int)((r.tile0 + tile) * TK);
        if (all_hi - j0 < TK || j0 < all_lo) {
            const int from = lo - j0 - 4 * (int)quarter, to = hi - j0 - 4 * (int)quarter;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (16 * u + i < from || 16 * u + i >= to) s[u][i] = -__builtin_inff();
        }
        const float top = row_max(fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3]))));
        if (__any((top - m) * a.c > LAG)) {
            const float mn = fmaxf(m, top);
            const float f = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((m - mn) * a.c);
            m = mn;
            l *= f;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[d][i] *= f;
        }
        const float mc = (m == -__builtin_inff() ? 0.0f : m * a.c) - LIFT;
        f32x8 x;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * u + i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], a.c, -mc));
        l += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
#pragma unroll
        for (int n = 0; n < NW; ++n) {
            w[n] = __builtin_convertvector(x, frag);
            x -= __builtin_convertvector(w[n], f32x8);
        }
    };
    auto gather = [&] {
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const C *p = vb + (4 * quarter + ((lane & 15) >> 2)) * VS + 4 * (lane & 3);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const s16x4 a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + d * 16));
            const s16x4 a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + d * 16 + 16 * VS));
            const s16x8 both = __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7);
            frag v;
            __builtin_memcpy(&v, &both, 16);
#pragma unroll
            for (int n = 0; n < NW; ++n) o[d] = mma16(v, w[n], o[d]);
        }
    };

    // AHEAD tiles of the wave are under way, the place of the one behind them looked up.  It is one tile, but the inner loop stays:
    // without it the compiler schedules the long sequence above into 27.5 us instead of 24 (other shapes alike).
    constexpr int AHEAD = 1;
    if (first + kw < last) {
        Tile x[AHEAD];
        Place at = look_up(first + kw);
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) {
            x[n] = fetch(first + kw + n * KW, at);
            at = look_up(first + kw + (n + 1) * KW);
        }
        for (u32 i = first + kw; i < last; i += AHEAD * KW) {
#pragma unroll
            for (int n = 0; n < AHEAD; ++n) {
                const u32 tile = i + n * KW;
                if (tile >= last) break;
                put_v(tile, x[n]);
                score(x[n]);
                if (tile + AHEAD * KW < last) {
                    x[n] = fetch(tile + AHEAD * KW, at);
                    at = look_up(tile + (AHEAD + 1) * KW);
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
                soften(tile);
                gather();
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
            }
        }
    }
    l = row_sum(l);

    // What put_v left out, added to the rows that see it: their sums take nothing else that could undo it any more.
    if (__any(odd != 0)) {
#pragma unroll 1
        for (u32 i = first + kw; i < last; i += KW) {
#pragma unroll 1
            for (int key = 0; key < TK; ++key) {
                const int j = (int)((r.tile0 + i) * TK) + key;
                if (j >= r.kv) break;
                const u32 pg = (u32)table[(u32)j / a.page_size], at = (u32)j % a.page_size;
                if (pg >= a.n_pages) continue;
                const unsigned char *v = vp + (i64)pg * a.vs[0] + (i64)at * a.vs[2];
                const unsigned char *z = a.vz + (i64)kv_head * a.vzs[1] + (i64)pg * a.vzs[0] + (i64)at * a.vzs[2];
#pragma unroll 1
                for (u32 e0 = 0; e0 < a.head_dim; e0 += 64) {
                    const float x = e0 + lane < a.head_dim ? (float)(C)unpack<FORM>(v[e0 + lane], z[(e0 + lane) / PACK_BLOCK]) : 0.0f;
                    for (unsigned long long bad = __ballot(!is_finite(x)); bad; bad &= bad - 1) {
                        const int b = __ffsll(bad) - 1;
                        const float add = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), b));
                        if (j >= lo && j < hi)
#pragma unroll
                            for (int d = 0; d < DT; ++d)
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    if (d * 16 + 4 * (int)quarter + k == (int)e0 + b) o[d][k] += add;
                    }
                }
            }
        }
    }

    // join the waves' results: [KW][16][DP] sums, then [KW][16] maxima and sums
    const bool split_up = r.n_splits > 1;
    float *jo = (float *)lds, *jm = jo + KW * ROWS * DP, *jl = jm + KW * ROWS;
    __syncthreads();
#pragma unroll
    for (int d = 0; d < DT; ++d) *(f32x4 *)(jo + (kw * ROWS + (lane & 15)) * DP + d * 16 + 4 * quarter) = o[d];
    if (quarter == 0) {
        jm[kw * ROWS + lane] = m;
        jl[kw * ROWS + lane] = l;
    }
    __syncthreads();
    const u32 n_rows = min((u32)ROWS, r.rows - r.first_row), quads = a.head_dim / 4;
    for (u32 x = threadIdx.x; x < n_rows * quads; x += 64 * KW) {
        const u32 jr = x / quads, e = x % quads * 4;
        float top = -__builtin_inff(), sum = 0.0f;
#pragma unroll
        for (int w = 0; w < KW; ++w) top = fmaxf(top, jm[w * ROWS + jr]);
        f32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < KW; ++w) {
            const float mw = jm[w * ROWS + jr], lw = jl[w * ROWS + jr];
            float f = mw == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((mw - top) * a.c);
            // a wave that saw no key has nothing to add; one whose sum is NaN has
            if (mw == -__builtin_inff() && lw == lw) continue;
            if (lw != lw) f = 1.0f;
            sum = __builtin_fmaf(f, lw, sum);
            const f32x4 y = *(const f32x4 *)(jo + (w * ROWS + jr) * DP + e);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] = __builtin_fmaf(f, y[i], acc[i]);
        }
        const bool some = sum > 0.0f || sum != sum;
        const float inv = some ? 1.0f / sum : 0.0f;
        const float lse2 = some ? __builtin_fmaf(top, a.c, __log2f(sum) - LIFT) : -__builtin_inff();
        const u32 jrow = r.first_row + jr, jt = r.start + jrow / a.group, jh = kv_head * a.group + jrow % a.group;
        const u64 at = (u64)jt * a.heads + jh;
        Pack<float, 4> res;
#pragma unroll
        for (int i = 0; i < 4; ++i) res.v[i] = some ? acc[i] * inv : 0.0f;
        if (split_up) {
            if (e == 0) a.part_lse[at * a.splits + split] = lse2;
            store_pack<4>(a.part + (at * a.splits + split) * a.head_dim + e, res);
        } else {
            if (e == 0 && a.lse) a.lse[at] = lse2 * 0.693147180559945309f;
            Pack<T, 4> y;
#pragma unroll
            for (int i = 0; i < 4; ++i) y.v[i] = (T)res.v[i];
            store_pack<4>((T *)a.out + (i64)jt * a.os[0] + jh * a.os[1] + e, y);
        }
    }
}

}  // namespace ckks

using namespace ckks;

// attend_thin_kernel, as a form of plan_attend: by its costs few rows of 16-entry pieces and every F32 head come here, chunks of the
// 16-bit types go to the forms whose waves share tiles.  F32, 2 x 1024 tokens over 2000 more keys, 32 / 8 heads of 128: 340 us here with E4M3, 456
// with I8, 787 over a plain cache.
constexpr AttendForm THIN_64 = {0, 16, 32, 128, 5, 0.8f, 1.2f, 3}, THIN_128 = {0, 16, 32, 128, 5, 1.0f, 2.0f, 3};

static AttendSizes sizes(const ckks_clear_packed_attend_t &p) {
    const ckks_clear_packed_t &g = p.pages;
    const AttendForm *thin = g.head_dim % 16 || g.head_dim > 128 ? nullptr : g.head_dim <= 64 ? &THIN_64 : &THIN_128;
    return {p.batch, p.heads, g.kv_heads, g.head_dim, g.page_size, g.dtype, p.flags, p.window, 2.0 * (g.head_dim + packed_blocks(g.head_dim)), thin};
}
template <class T, int FORM, int DP>
static int launch_thin(const PackedAttendArgs &a, hipStream_t st) {
    constexpr int OCC = sizeof(T) == 4 && DP == 128 ? 2 : 3;
    const dim3 grid(a.kv_heads * a.splits * a.tiles);
    if (a.page_size % 32)
        hipLaunchKernelGGL((attend_thin_kernel<T, FORM, DP, false, 4, OCC>), grid, dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((attend_thin_kernel<T, FORM, DP, true, 4, OCC>), grid, dim3(256), 0, st, a);
    CKKS_LAUNCH_CHECK("attend_thin_kernel");
    return launch_join<T, 16, 32>(a, DP / 4, st);
}
template <class T, int FORM>
static int launch_packed(const PackedAttendArgs &a, const AttendPlan &n, hipStream_t st) {
    if (n.form.waves_rows) return launch_attend<T, FORM>(a, n, st);
    return n.dp == 64 ? launch_thin<T, FORM, 64>(a, st) : launch_thin<T, FORM, 128>(a, st);
}
template <class T>
static int launch_packed(const PackedAttendArgs &a, const AttendPlan &n, u32 format, hipStream_t st) {
    return format == CKKS_CLEAR_E4M3 ? launch_packed<T, E4M3>(a, n, st) : launch_packed<T, I8>(a, n, st);
}

extern "C" {

uint64_t ckks_clear_packed_attend_work_bytes(const ckks_clear_packed_attend_t *p) {
    AttendPlan n;
    return p && plan_attend(sizes(*p), n) ? n.work_bytes : 0;
}

int ckks_clear_packed_attend(const ckks_clear_packed_attend_t *p, void *stream) {
    const char *who = "ckks_clear_packed_attend";
    if (!p) {
        set_error("%s: null argument", who);
        return CKKS_E_INVAL;
    }
    const ckks_clear_packed_t &g = p->pages;
    if (int rc = check_packed(who, g, p->batch)) return rc;
    const PackedPlaces places = packed_places(g);
    AttendPlan n;
    PackedAttendArgs a{};
    const ckks_clear_pages_t codes = as_pages(g, false);
    const AttendCall call{codes, p->d_q, p->d_out, p->d_lse, p->d_work, p->work_bytes, p->q_stride, p->out_stride, p->scale, places.at, 4};
    if (int rc = prepare_attend(who, sizes(*p), call, n, a)) return rc;
    if (!n.splits) return CKKS_OK;
    a.kz = g.d_k_power, a.vz = g.d_v_power;
    for (int i = 0; i < 3; ++i) a.kzs[i] = g.k_power_stride[i], a.vzs[i] = g.v_power_stride[i];
    if (!g.n_pages) {  // as the codes
        a.kz = a.vz = (const unsigned char *)p->d_q;
        for (int i = 0; i < 3; ++i) a.kzs[i] = a.vzs[i] = 0;
    }
    hipStream_t st = (hipStream_t)stream;
    return g.dtype == CKKS_CLEAR_F32   ? launch_packed<float>(a, n, g.format, st)
           : g.dtype == CKKS_CLEAR_F16 ? launch_packed<f16>(a, n, g.format, st)
                                       : launch_packed<bf16>(a, n, g.format, st);
}

}  // extern "C"
