// Attention of a chunk of new tokens over the paged cache.
//
// The query heads that share a kv head are rows of one problem: row i * group + g of (sequence, kv head) is new token i, head
// kv_head * group + g.  A wave takes 32 rows.  It computes the scores transposed, S^T = K Q^T, so that a lane holds scores of
// one row only (row lane % 32; the two halves of the wave hold different keys): maximum and sum of the softmax stay in the
// lane but for one exchange between the halves, and the weights come out in the order in which the next product,
// O^T = V^T P^T, wants them.  Neither scores nor weights pass through LDS.
//
//   RW = 4, 8: waves of 32 rows share each tile of keys and values (chunks of a prompt).
//   KW > 1: one set of 32 rows, each wave takes every KW-th tile through its own stretch of LDS, without barriers, and the
//           waves' results are joined at the end (single tokens: the time is that of reading the cache).
// Either may split the keys over several blocks; a second kernel then joins the blocks' results in order.
//
// Measured (heads of 128, 32 query and 8 kv heads, 16 bits, unless said):
//   prompts, 2 chunks of up to 4096 tokens over 12301 more keys, RW = 8: 1265 to 1315 us, 1.00 to 1.04 PFLOP/s, where a library product of 8192^3
//     reaches 1.13; the matrix units are fed half the cycles and the softmax's arithmetic takes nearly as many, at a clock that
//     the power limit holds down;
//   64 single tokens over up to 8192 keys each, KW = 4: 225 us for 1.2 GB, 5.3 TB/s;
//   1 token over 131002 keys, 16 and 2 heads, KW = 4, split: 26 to 30 us and 5 us to join (134 MB, 27 us at a copy's rate);
//   1 token over 128 keys, 12 heads of 64: 6.9 us; 128 tokens of 32 bits: 10.7 us: the chain of lookup, load, product, join.
//   Heads of 136 to 256 do not fit the registers: 172 of a lane lie in scratch with KW = 4 (64 tokens over 8192 keys, 8 heads of 256, bf16
//     1.5 ms, 2.9 TB/s; one token 41 us), 38 with RW = 4 in 32 bits (88 TFLOP/s); RW = 4 in 16 bits reaches 590 TFLOP/s.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "clear_device.h"

namespace ckks {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

struct AttendArgs {
    const void *q, *k, *v;
    void *out;
    float *lse, *part, *part_lse;
    i64 qs[2], os[2], ks[3], vs[3], ts;
    const int32_t *q_start, *kv_len, *table;
    u32 n_seq, n_tokens, n_pages, page_size, table_width, kv_heads, heads, group, head_dim, causal;
    int window;
    u32 page_mul, page_shift;  // position / page_size = (2 * position * page_mul >> 32) >> page_shift
    u32 alike;                 // keys and values have the same strides
    u32 tiles, splits, min_tiles;
    float c;             // scale * log2(e)
};

// One 16-deep step of a 32 x 32 product.  A lane holds 8 entries of row (column) lane % 32 of A (B), those of depth
// 8 * (lane / 32) ..; the sum over the depth does not care in which order the entries are taken, so with 32-bit types the eight
// steps of depth 2 pair entry j of the halves.
__device__ __forceinline__ f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma(f32x8 a, f32x8 b, f32x16 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
}
// What the softmax's weights are held at, as powers of two: LIFT times exp2(score - maximum), where the maximum may lag by LAG.
// In 16 bits a weight below 2^-14 loses bits and one below 2^-25 is gone, while the sum, in 32, counts it: beside one key that takes
// most of a row, 1e5 others at 2^-24 of it came out as 0.0078 where they make up 0.0054.  F16 weights are therefore lifted
// as far as the type goes, 2^15 with the lag (the lift cancels in out and is taken off lse): a weight keeps all its bits down to
// 2^-25 of the largest and is gone from 2^-36.  BF16 has the range of 32 bits.
template <class T>
struct Frag;
template <>
struct Frag<float> {
    typedef f32x8 type;
    static constexpr float LIFT = 0.0f, LAG = 8.0f;
};
template <>
struct Frag<f16> {
    typedef f16x8 type;
    static constexpr float LIFT = 11.0f, LAG = 4.0f, BELOW = 1.0f - 0x1p-10f;
};
template <>
struct Frag<bf16> {
    typedef bf16x8 type;
    static constexpr float LIFT = 0.0f, LAG = 8.0f, BELOW = 1.0f - 0x1p-7f;
};

template <class T>
__device__ __forceinline__ typename Frag<T>::type row_frag(const T *p) {
    typename Frag<T>::type r;
    __builtin_memcpy(&r, __builtin_assume_aligned(p, 16), sizeof(r));
    return r;
}

// Entries of column `lane % 32` of the values, keys 4h .. 4h+3 and 8 + 4h .. 8 + 4h + 3 of the 16 that begin at `v` (h = lane / 32):
// the order in which the scores' accumulators hold a row's weights.  For 16-bit types the transposing LDS read: 16 lanes
// read 4 rows of 16 entries, and each gets a column.
template <class T, int STRIDE>
__device__ __forceinline__ typename Frag<T>::type col_frag(const T *v, u32 lane) {
    typename Frag<T>::type r;
    if constexpr (sizeof(T) == 2) {
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const T *p = v + (4 * (lane >> 5) + ((lane & 15) >> 2)) * STRIDE + (lane & 16) + 4 * (lane & 3);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + 8 * STRIDE));
        const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        __builtin_memcpy(&r, &both, 16);
    } else {
        const T *p = v + 4 * (lane >> 5) * STRIDE + (lane & 31);
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] = p[(j < 4 ? j : j + 4) * STRIDE];
    }
    return r;
}

// The larger of x and its value in the other half of the wave (NaN gives way), without LDS.
__device__ __forceinline__ float other_half_max(float x) {
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
}

// What a tile of rows works on.
struct RowTile {
    u32 seq, start, n, first_row, rows;  // first token and tokens of the sequence; first row of the tile, rows in all
    int kv, t0;                          // keys, position of the sequence's first new token
    u32 tile0, n_tiles, per, n_splits;   // first key tile, key tiles, key tiles of a split, splits
};

// Position of a row; those before the cache are all alike.
__device__ __forceinline__ int row_pos(const AttendArgs &a, const RowTile &r, u32 row) { return max(r.t0 + (int)(row / a.group), -1); }

// Key tiles that the rows first_row .. first_row + ROWS - 1 see between them.
template <int ROWS, int TK>
__device__ __forceinline__ void key_range(const AttendArgs &a, int kv_len, RowTile &r) {
    const int kv = min(kv_len, (int)(a.table_width * a.page_size));
    r.kv = max(0, kv);
    r.t0 = max(kv, 0) - (int)r.n;
    const u32 last = min(r.first_row + ROWS, r.rows) - 1;
    const int hi = a.causal ? min(r.kv, row_pos(a, r, last) + 1) : r.kv;
    const int lo = a.window ? max(0, row_pos(a, r, r.first_row) - a.window + 1) : 0;
    r.tile0 = (u32)lo / TK;
    r.n_tiles = hi > lo ? ((u32)hi + TK - 1) / TK - r.tile0 : 0;
    r.per = max(a.min_tiles, (r.n_tiles + a.splits - 1) / a.splits);
    r.n_splits = max(1u, (r.n_tiles + r.per - 1) / r.per);
}

// The sequence that holds tile `tile` of all sequences' tiles.  Called by whole waves.
template <int ROWS>
__device__ __forceinline__ bool find_tile(const AttendArgs &a, u32 tile, RowTile &r) {
    const u32 lane = threadIdx.x & 63;
    u32 before = 0;
    for (u32 base = 0; base < a.n_seq; base += 64) {
        const u32 b = base + lane;
        int s = 0, e = 0;
        if (b < a.n_seq) {
            s = min(max(a.q_start[b], 0), (int)a.n_tokens);
            e = max(min(a.q_start[b + 1], (int)a.n_tokens), s);
        }
        const u32 tiles = ((u32)(e - s) * a.group + ROWS - 1) / ROWS;
        u32 sum = tiles;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const u32 up = __shfl_up(sum, o);
            if (lane >= (u32)o) sum += up;
        }
        const u32 total = __builtin_amdgcn_readlane(sum, 63);
        if (tile - before < total) {
            const int at = __ffsll((unsigned long long)__ballot(sum > tile - before)) - 1;
            r.seq = base + at;
            r.start = __builtin_amdgcn_readlane(s, at);
            r.n = __builtin_amdgcn_readlane(e, at) - r.start;
            r.first_row = (tile - before - (__builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(tiles, at))) * ROWS;
            r.rows = r.n * a.group;
            return true;
        }
        before += total;
    }
    return false;
}

__device__ __forceinline__ bool is_finite(float x) { return __builtin_fabsf(x) <= 3.402823466e38f; }
// 16 bytes of T with zeros in place of infinities and NaN, whose exponents are all ones; `odd` becomes nonzero if there was one.
template <class T>
__device__ __forceinline__ uint4 finite_part(uint4 x, u32 &odd) {
    auto clean = [&](u32 w) {
        if constexpr (sizeof(T) == 4) {
            const u32 bad = (w & 0x7f800000u) == 0x7f800000u ? ~0u : 0u;
            odd |= bad;
            return w & ~bad;
        } else {
            constexpr u32 EXP = std::is_same<T, f16>::value ? 0x7c007c00u : 0x7f807f80u, ONE = EXP & (0u - EXP) & 0xffffu;
            const u32 top = (w & EXP) + ONE * 0x10001u & 0x80008000u;  // both halves at once: the sum of a half stays in it
            odd |= top;
            return w & ~(top | (top - (top >> 15)));
        }
    };
    return make_uint4(clean(x.x), clean(x.y), clean(x.z), clean(x.w));
}

template <class T, int DP, int RW, int KW, int TK>
struct AttendShape {
    static constexpr int KS = DP + 16 / (int)sizeof(T);               // row strides in LDS: keys are read 16 bytes from each
    static constexpr int VS = DP + (sizeof(T) == 2 ? 32 : 8);         // of 32 rows, values 64 bytes (32 entries) from each of 4:
                                                                      // these pads spread either over the banks
    static constexpr int TILE = TK * (KS + VS);                       // entries of a tile
    static constexpr int BUFFERS = RW > 1 ? 2 : KW;
    static constexpr size_t STAGE_BYTES = (size_t)TILE * BUFFERS * sizeof(T);
    static constexpr size_t JOIN_BYTES = KW > 1 ? (size_t)KW * 32 * (DP + 2) * 4 : 0;
    static constexpr size_t LDS = STAGE_BYTES > JOIN_BYTES ? STAGE_BYTES : JOIN_BYTES;
};

template <class T, int DP, int RW, int KW, int TK, int OCC>
__global__ __launch_bounds__(64 * RW * KW, OCC) void attend_kernel(AttendArgs a) {
    typedef AttendShape<T, DP, RW, KW, TK> Shape;
    typedef typename Frag<T>::type frag;
    constexpr float LIFT = Frag<T>::LIFT, LAG = Frag<T>::LAG;
    // Weights of 16 bits: where each wave goes through the cache by itself the matrix units have time for a second product, with
    // what the weights lack (`low`), and results are as good as with weights of 32 bits; 64 single tokens over up to 8192 keys take
    // 231 us with it, 229 without.  The high part is rounded from a little less than the weight, so that both are above 0 and an
    // infinite value stays one (F16: down to 2^-24 of the largest weight).  Where waves share tiles the products bound the kernel, and
    // the weights' rounding stays: the error against 64 bits is 1.25 to 1.4 times that of weights of 32 bits (bf16 0.0023 against
    // 0.0017), where 2 x 4096 tokens over 12301 would take 1957 us instead of 1274, heads of 64 over 4000 531 instead of 413.
    constexpr bool LOW = KW > 1 && sizeof(T) == 2;
    constexpr int KS = Shape::KS, VS = Shape::VS, ROWS = 32 * RW, SUB = TK / 32, DT = DP / 32;
    constexpr int E = 16 / sizeof(T);                  // entries of a 16-byte piece
    constexpr int PIECES = DP / E;                     // pieces of a row
    constexpr int STAGERS = 64 * RW;                   // threads that fetch a tile
    constexpr int PASS = STAGERS / PIECES;             // rows that they fetch at a time
    constexpr int PASSES = TK / PASS;
    __shared__ __attribute__((aligned(16))) unsigned char lds[Shape::LDS];

    const u32 lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const u32 kv_head = blockIdx.x % a.kv_heads, split = blockIdx.x / a.kv_heads % a.splits;
    RowTile r;
    // the last tiles of a causal chunk see the most keys: they start first
    if (!find_tile<ROWS>(a, a.tiles - 1 - blockIdx.x / a.kv_heads / a.splits, r)) return;
    key_range<ROWS, TK>(a, a.kv_len[r.seq], r);
    // the same in every lane: scalars from here on
    r.kv = __builtin_amdgcn_readfirstlane(r.kv);
    r.t0 = __builtin_amdgcn_readfirstlane(r.t0);
    r.tile0 = __builtin_amdgcn_readfirstlane(r.tile0);
    r.n_tiles = __builtin_amdgcn_readfirstlane(r.n_tiles);
    r.per = __builtin_amdgcn_readfirstlane(r.per);
    r.n_splits = __builtin_amdgcn_readfirstlane(r.n_splits);
    if (split >= r.n_splits) return;
    const u32 first = split * r.per, last = min(first + r.per, r.n_tiles);

    const u32 rw = RW > 1 ? wave : 0, kw = KW > 1 ? wave : 0;
    const u32 row0 = r.first_row + 32 * rw;
    const bool idle = row0 >= r.rows;                  // no row of this wave exists
    const u32 row = min(row0 + (lane & 31), r.rows - 1), token = row / a.group, head = kv_head * a.group + row % a.group;
    const int pos = max(r.t0 + (int)token, -1);
    // keys lo <= j < hi are seen, and none of these bounds is below 0: their differences with a key's place stay in 32 bits
    const int hi = a.causal ? min(r.kv, pos + 1) : r.kv, lo = a.window ? max(pos - a.window + 1, 0) : 0;
    // bounds over the wave's rows: keys that all of them see, keys that any of them sees
    const int p_first = row_pos(a, r, min(row0, r.rows - 1)), p_last = row_pos(a, r, min(row0 + 31, r.rows - 1));
    const int all_hi = a.causal ? min(r.kv, p_first + 1) : r.kv, any_hi = a.causal ? min(r.kv, p_last + 1) : r.kv;
    // ... of the block's rows
    const int block_hi = a.causal ? min(r.kv, row_pos(a, r, r.first_row) + 1) : r.kv,
              block_lo = a.window ? max(row_pos(a, r, min(r.first_row + ROWS, r.rows) - 1) - a.window + 1, 0) : 0;
    const int all_lo = a.window ? max(p_last - a.window + 1, 0) : 0, any_lo = a.window ? max(p_first - a.window + 1, 0) : 0;

    frag qf[DP / 16];
    {
        const T *q = (const T *)a.q + (i64)(r.start + token) * a.qs[0] + head * a.qs[1];
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
            const u32 d = s * 16 + half * 8;
            if (d < a.head_dim) {
                __builtin_memcpy(&qf[s], q + d, 8 * sizeof(T));
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) qf[s][j] = (T)0.0f;
            }
        }
    }

    // a lane's piece of each row that it fetches
    const u32 stager = RW > 1 ? threadIdx.x : lane, piece = stager % PIECES, fetch_row = stager / PIECES;
    const bool piece_ok = piece * E < a.head_dim;
    const T *kp = (const T *)a.k + (i64)kv_head * a.ks[1], *vp = (const T *)a.v + (i64)kv_head * a.vs[1];
    const int32_t *table = a.table + (i64)r.seq * a.ts;
    typedef uint4 piece_t;
    piece_t kr[PASSES], vr[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) kr[p] = vr[p] = make_uint4(0, 0, 0, 0);
    // Where the rows that this thread fetches lie.  The table's answer is looked at only when it is needed, a tile later: a wait
    // or a branch here would be a wait for all loads under way.
    struct Place {
        u32 page[PASSES], row[PASSES];  // of each row
        u32 tile_page, tile_row;        // of the tile, where pages hold whole tiles
    };
    const bool whole = a.page_size % TK == 0;
    auto look_up = [&](u32 tile) {
        Place at;
        if (whole) {
            const u32 j = min(r.tile0 + tile, ((u32)r.kv - 1) / TK) * TK, n = __umulhi(2 * j, a.page_mul) >> a.page_shift;
            at.tile_page = (u32)table[n];
            at.tile_row = j - n * a.page_size;
        } else {
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                const u32 j = min((r.tile0 + tile) * TK + p * PASS + fetch_row, (u32)r.kv - 1);
                const u32 n = __umulhi(2 * j, a.page_mul) >> a.page_shift;
                at.page[p] = (u32)table[n];
                at.row[p] = j - n * a.page_size;
            }
        }
        return at;
    };
    // Rows and pieces that are not there are fetched from page 0 and become zeros when they are put into LDS (`none`: a bit
    // for each pass): a branch around a load would have its result copied, and so waited for, at once.
    const u32 lane_piece = piece_ok ? piece * E : 0;
    const u32 k_lane = fetch_row * (u32)a.ks[2] + lane_piece, v_lane = fetch_row * (u32)a.vs[2] + lane_piece;
    struct Sources {
        u64 k[PASSES], v[PASSES];
        u32 none;
    };
    auto locate = [&](u32 tile, const Place &at) {
        Sources s;
        s.none = piece_ok ? 0 : ~0u;
        // check_cache: a page's stride fits 32 bits, and so does every offset within a page
        if (whole) {
            const u32 pg = at.tile_page < a.n_pages ? at.tile_page : 0;
            if (at.tile_page >= a.n_pages) s.none = ~0u;
            const u64 k0 = (u64)pg * (u32)a.ks[0] + at.tile_row * (u32)a.ks[2], v0 = (u64)pg * (u32)a.vs[0] + at.tile_row * (u32)a.vs[2];
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                s.k[p] = k0 + p * PASS * (u32)a.ks[2] + k_lane;
                s.v[p] = v0 + p * PASS * (u32)a.vs[2] + v_lane;
            }
        } else {
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                u32 pg = at.page[p];
                if (pg >= a.n_pages) {
                    pg = 0;
                    s.none |= 1u << p;
                }
                s.k[p] = (u64)pg * (u32)a.ks[0] + (at.row[p] * (u32)a.ks[2] + lane_piece);
                s.v[p] = a.alike ? s.k[p] : (u64)pg * (u32)a.vs[0] + (at.row[p] * (u32)a.vs[2] + lane_piece);
            }
        }
        if ((r.tile0 + tile + 1) * TK > (u32)r.kv)
#pragma unroll
            for (int p = 0; p < PASSES; ++p)
                if ((r.tile0 + tile) * TK + p * PASS + fetch_row >= (u32)r.kv) s.none |= 1u << p;
        return s;
    };
    u32 k_none = 0, v_none = 0;
    auto fetch_k = [&](const Sources &from) {
#pragma unroll
        for (int p = 0; p < PASSES; ++p) __builtin_memcpy(&kr[p], kp + from.k[p], 16);
        k_none = from.none;
    };
    auto fetch_v = [&](const Sources &from) {
#pragma unroll
        for (int p = 0; p < PASSES; ++p) __builtin_memcpy(&vr[p], vp + from.v[p], 16);
        v_none = from.none;
    };
    auto fetch = [&](u32 tile, const Place &at) {
        const Sources from = locate(tile, at);
        fetch_k(from);
        fetch_v(from);
    };
    auto blank = [&](piece_t *x, u32 none) {
        if (__any(none != 0))
#pragma unroll
            for (int p = 0; p < PASSES; ++p)
                if (none >> p & 1) x[p] = make_uint4(0, 0, 0, 0);
    };
    auto put_k = [&](T *buf) {
        blank(kr, k_none);
#pragma unroll
        for (int p = 0; p < PASSES; ++p) *(piece_t *)(buf + (p * PASS + fetch_row) * KS + piece * E) = kr[p];
    };
    // A weight of 0 does not keep an infinity or NaN of an unseen value out of a sum.  In a tile that some row of the block does
    // not see in full such values are taken as zeros; whether there were any decides about the pass at the end.
    u32 odd = 0;
    auto partial = [&](u32 tile) {
        const int j0 = (int)((r.tile0 + tile) * TK);
        return block_hi - j0 < TK || j0 < block_lo;
    };
    auto put_v = [&](u32 tile, T *buf) {
        blank(vr, v_none);
        if (tile < last && partial(tile))
#pragma unroll
            for (int p = 0; p < PASSES; ++p) vr[p] = finite_part<T>(vr[p], odd);
#pragma unroll
        for (int p = 0; p < PASSES; ++p) *(piece_t *)(buf + (p * PASS + fetch_row) * VS + piece * E) = vr[p];
    };

    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    float m = -__builtin_inff(), l = 0.0f;  // maximum of the row's scores (it may lag, below), the lane's part of the sum

    f32x16 s[SUB];       // scores of a tile; accumulator i of a lane: key 8 (i / 4) + 4 half + i % 4 of its 32
    frag w[2 * SUB];     // weights, 16 keys each
    frag low[LOW ? 2 * SUB : 1];  // what they lack
    // whether any row of the wave sees the tile, and whether some row does not see all of it
    auto seen = [&](u32 tile) {
        const int j0 = (int)((r.tile0 + tile) * TK);
        return !idle && j0 < any_hi && any_lo - j0 < TK;
    };
    auto masked = [&](u32 tile) {
        const int j0 = (int)((r.tile0 + tile) * TK);
        return all_hi - j0 < TK || j0 < all_lo;
    };
    auto see_lo = [&](u32 tile) { return lo - (int)((r.tile0 + tile) * TK) - 4 * (int)half; };
    auto see_hi = [&](u32 tile) { return hi - (int)((r.tile0 + tile) * TK) - 4 * (int)half; };

    auto score = [&](const T *kb) {
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[u][i] = 0.0f;
#pragma unroll
        for (int d = 0; d < DP / 16; ++d)
#pragma unroll
            for (int u = 0; u < SUB; ++u) s[u] = mma(row_frag(kb + (u * 32 + (lane & 31)) * KS + d * 16 + half * 8), qf[d], s[u]);
    };
    auto soften = [&](u32 tile) {
        if (!seen(tile)) {
#pragma unroll
            for (int k = 0; k < 2 * SUB; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) w[k][j] = (T)0.0f;
            return;
        }
        if (masked(tile)) {
            const int from = see_lo(tile), to = see_hi(tile);
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = u * 32 + 8 * (i / 4) + i % 4;
                    if (key < from || key >= to) s[u][i] = -__builtin_inff();
                }
        }
        // four chains each for maximum and sum: nothing else runs on the wave meanwhile
        float tops[4] = {s[0][0], s[0][1], s[0][2], s[0][3]};
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int i = u ? 0 : 4; i < 16; ++i) tops[i % 4] = fmaxf(tops[i % 4], s[u][i]);
        const float top = other_half_max(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])));
        // The maximum only has to keep the weights in range: it moves when a score passes it by LAG powers of two, and then all
        // that was summed is scaled.
        if (__any((top - m) * a.c > LAG)) {
            const float mn = fmaxf(m, top);
            const float f = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((m - mn) * a.c);
            m = mn;
            l *= f;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= f;
        }
        const float mc = (m == -__builtin_inff() ? 0.0f : m * a.c) - LIFT;
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[u][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], a.c, -mc));
                sum[i % 4] += s[u][i];
            }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                f32x8 x;
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = s[u][8 * kk + j];
                if constexpr (LOW) {
                    w[2 * u + kk] = __builtin_convertvector(x * Frag<T>::BELOW, frag);
                    low[2 * u + kk] = __builtin_convertvector(x - __builtin_convertvector(w[2 * u + kk], f32x8), frag);
                } else {
                    w[2 * u + kk] = __builtin_convertvector(x, frag);
                }
            }
    };
    auto gather = [&](const T *vb) {
#pragma unroll
        for (int k = 0; k < 2 * SUB; ++k)
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const frag v = col_frag<T, VS>(vb + k * 16 * VS + d * 32, lane);
                o[d] = mma(v, w[k], o[d]);
                if constexpr (LOW) o[d] = mma(v, low[k], o[d]);
            }
    };
    auto work = [&](u32 tile, const T *buf) {
        if (!seen(tile)) return;
        score(buf);
        soften(tile);
        gather(buf + TK * KS);
    };

    T *buf = (T *)lds;
    if (first >= last) {  // no key is seen: nothing may be looked up either
    } else if constexpr (RW == 8) {
        // Two sets of four waves, one of each on every SIMD, work half a tile apart: while one set keeps the matrix units busy
        // (scores of tile i, sum of tile i - 1), the other does the softmax of its tile and moves the next one in.  A barrier
        // ends each half.  Keys of tile i + 1 and values of tile i are written while those before them are read: two
        // buffers of each.
        const u32 set = wave >> 2, n = last - first;
        T *kb = buf, *vb = buf + 2 * TK * KS;
        auto half_done = [] {
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
            __builtin_amdgcn_sched_barrier(0);
        };
        Place at = look_up(first);
        fetch(first, at);
        at = look_up(first + 1);
        put_k(kb);
        Sources next = locate(first + 1, at);
        fetch_k(next);
        at = look_up(first + 2);
        // Past the last tile these move what nobody reads.
        auto put = [&](u32 i) {
            put_k(kb + (i + 1 & 1) * TK * KS);
            put_v(first + i, vb + (i & 1) * TK * VS);
        };
        auto move = [&](u32 i) {
            const Sources after = locate(first + i + 2, at);
            at = look_up(first + i + 3);
            fetch_v(next);
            fetch_k(after);
            next = after;
        };
        // the first sum has weights 0 and no values yet
        for (u32 x = threadIdx.x; x < TK * VS / E; x += 64 * RW) *(piece_t *)(vb + TK * VS + x * E) = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int k = 0; k < 2 * SUB; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) w[k][j] = (T)0.0f;
        // The order of the products and the LDS reads that feed them: AHEAD fragments are under way before the first product,
        // and one more (keys: one read, values: two) follows each product.
        auto interleave = [] {
            constexpr int MFMA = 0x8, READ = 0x100, AHEAD = 6, NK = SUB * DP / 16, NV = 2 * SUB * DT;
            __builtin_amdgcn_sched_group_barrier(READ, AHEAD, 0);
#pragma unroll
            for (int x = 0; x < NK - AHEAD; ++x) {
                __builtin_amdgcn_sched_group_barrier(MFMA, 1, 0);
                __builtin_amdgcn_sched_group_barrier(READ, 1, 0);
            }
#pragma unroll
            for (int x = 0; x < NV; ++x) {
                __builtin_amdgcn_sched_group_barrier(MFMA, 1, 0);
                __builtin_amdgcn_sched_group_barrier(READ, 2, 0);
            }
            __builtin_amdgcn_sched_group_barrier(MFMA, AHEAD, 0);
        };
        half_done();
        if (set) {
            put(0);
            move(0);
            half_done();
        }
        for (u32 i = 0; i <= n; ++i) {
            __builtin_amdgcn_s_setprio(1);
            if (i) move(i + set - 1);
            score(kb + (i & 1) * TK * KS);
            gather(vb + (i + 1 & 1) * TK * VS);
            interleave();
            __builtin_amdgcn_s_setprio(0);
            half_done();
            if (i < n) soften(first + i);
            put(i + set);
            half_done();
        }
        if (!set) half_done();
    } else if constexpr (RW > 1) {
        Place at = look_up(first);
        fetch(first, at);
        at = look_up(first + 1);
        put_k(buf);
        put_v(first, buf + TK * KS);
        for (u32 i = first; i < last; ++i) {
            __syncthreads();
            if (i + 1 < last) {
                fetch(i + 1, at);
                at = look_up(i + 2);
            }
            work(i, buf + (i - first & 1) * Shape::TILE);
            // the other buffer was read before this barrier
            put_k(buf + (i + 1 - first & 1) * Shape::TILE);
            put_v(i + 1, buf + (i + 1 - first & 1) * Shape::TILE + TK * KS);
        }
    } else {
        buf += kw * Shape::TILE;
        Place at = look_up(first + kw);
        fetch(first + kw, at);
        at = look_up(first + kw + KW);
        for (u32 i = first + kw; i < last; i += KW) {
            put_k(buf);
            put_v(i, buf + TK * KS);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (i + KW < last) {
                fetch(i + KW, at);
                at = look_up(i + 2 * KW);
            }
            work(i, buf);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
    l += __shfl_xor(l, 32);

    // What put_v left out, added to the rows that see it: their sums take nothing else that could undo it any more.
    const bool left_out = RW > 1 ? __syncthreads_or(odd != 0) : __any(odd != 0);
    if (left_out) {
#pragma unroll 1
        for (u32 i = RW > 1 ? first : first + kw; i < last; i += KW) {
            if (!partial(i)) continue;
#pragma unroll 1
            for (int key = 0; key < TK; ++key) {
                const int j = (int)((r.tile0 + i) * TK) + key;
                if (j >= r.kv) break;
                const u32 pg = (u32)table[(u32)j / a.page_size];
                if (pg >= a.n_pages) continue;
                const T *v = vp + (i64)pg * a.vs[0] + (i64)((u32)j % a.page_size) * a.vs[2];
#pragma unroll 1
                for (u32 e0 = 0; e0 < a.head_dim; e0 += 64) {
                    const float x = e0 + lane < a.head_dim ? (float)v[e0 + lane] : 0.0f;
                    for (unsigned long long bad = __ballot(!is_finite(x)); bad; bad &= bad - 1) {
                        const int b = __ffsll(bad) - 1;
                        const float add = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), b));
                        if (j >= lo && j < hi)
#pragma unroll
                            for (int d = 0; d < DT; ++d)
#pragma unroll
                                for (int k = 0; k < 16; ++k)
                                    if (d * 32 + 8 * (k / 4) + 4 * (int)half + k % 4 == (int)e0 + b) o[d][k] += add;
                    }
                }
            }
        }
    }

    // Result of rows in this wave (or of the block's 32 rows): O^T holds entry 32 d + 8 (i / 4) + 4 half + i % 4 of its row.
    const bool split_up = r.n_splits > 1;
    if (KW == 1) {
        if (row0 + (lane & 31) >= r.rows) return;
        const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
        const float lse2 = l > 0.0f || l != l ? __builtin_fmaf(m, a.c, __log2f(l) - LIFT) : -__builtin_inff();
        const u64 at = (u64)(r.start + token) * a.heads + head;
        if (half == 0) {
            if (split_up)
                a.part_lse[at * a.splits + split] = lse2;
            else if (a.lse)
                a.lse[at] = lse2 * 0.693147180559945309f;
        }
        float *part = a.part + (at * a.splits + split) * a.head_dim;
        T *out = (T *)a.out + (i64)(r.start + token) * a.os[0] + head * a.os[1];
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const u32 e = d * 32 + g * 8 + half * 4;
                if (e >= a.head_dim) continue;
                Pack<float, 4> x;
                Pack<T, 4> y;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x.v[i] = l > 0.0f || l != l ? o[d][g * 4 + i] * inv : 0.0f;
                    y.v[i] = (T)x.v[i];
                }
                if (split_up)
                    store_pack<4>(part + e, x);
                else
                    store_pack<4>(out + e, y);
            }
        return;
    }
    // join the waves' results: [KW][32][DP] sums, then [KW][32] maxima and sums
    float *jo = (float *)lds, *jm = jo + KW * 32 * DP, *jl = jm + KW * 32;
    __syncthreads();
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            Pack<float, 4> x;
#pragma unroll
            for (int i = 0; i < 4; ++i) x.v[i] = o[d][g * 4 + i];
            *(float4 *)(jo + (kw * 32 + (lane & 31)) * DP + d * 32 + g * 8 + half * 4) = make_float4(x.v[0], x.v[1], x.v[2], x.v[3]);
        }
    if (half == 0) {
        jm[kw * 32 + lane] = m;
        jl[kw * 32 + lane] = l;
    }
    __syncthreads();
    const u32 n_rows = min(32u, r.rows - r.first_row), quads = a.head_dim / 4;
    for (u32 x = threadIdx.x; x < n_rows * quads; x += 64 * KW) {
        const u32 jr = x / quads, e = x % quads * 4;
        float top = -__builtin_inff(), sum = 0.0f, f[KW];
#pragma unroll
        for (int w = 0; w < KW; ++w) top = fmaxf(top, jm[w * 32 + jr]);
        float4 acc = make_float4(0, 0, 0, 0);
#pragma unroll
        for (int w = 0; w < KW; ++w) {
            const float mw = jm[w * 32 + jr];
            f[w] = mw == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((mw - top) * a.c);
            const float lw = jl[w * 32 + jr];
            // a wave that saw no key has nothing to add; one whose sum is NaN has
            if (mw == -__builtin_inff() && lw == lw) continue;
            if (lw != lw) f[w] = 1.0f;
            sum = __builtin_fmaf(f[w], lw, sum);
            const float4 y = *(const float4 *)(jo + (w * 32 + jr) * DP + e);
            acc.x = __builtin_fmaf(f[w], y.x, acc.x);
            acc.y = __builtin_fmaf(f[w], y.y, acc.y);
            acc.z = __builtin_fmaf(f[w], y.z, acc.z);
            acc.w = __builtin_fmaf(f[w], y.w, acc.w);
        }
        const bool some = sum > 0.0f || sum != sum;
        const float inv = some ? 1.0f / sum : 0.0f;
        const float lse2 = some ? __builtin_fmaf(top, a.c, __log2f(sum) - LIFT) : -__builtin_inff();
        const u32 jrow = r.first_row + jr, jt = r.start + jrow / a.group, jh = kv_head * a.group + jrow % a.group;
        const u64 at = (u64)jt * a.heads + jh;
        Pack<float, 4> res = {{some ? acc.x * inv : 0.0f, some ? acc.y * inv : 0.0f, some ? acc.z * inv : 0.0f, some ? acc.w * inv : 0.0f}};
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

// Joins the splits of a row (token, head): WAVES waves for each, a group of `lanes` lanes (four entries each) takes every
// so-manieth split, and the groups' sums are added in their order.  Bound by latency.  us of 2048 rows of 6 splits: one wave a
// row 5.0, four 7.3, sixteen 20; of 16 rows of 128 splits: 20, 7.8, 5.0.
template <class T, int ROWS, int TK, int WAVES>
__global__ __launch_bounds__(WAVES < 4 ? 256 : 64 * WAVES) void attend_join_kernel(AttendArgs a, u32 lanes) {
    constexpr int PER = WAVES < 4 ? 4 / WAVES : 1;  // rows of a block
    __shared__ __attribute__((aligned(16))) float4 acc_of[64 * WAVES * PER];
    __shared__ float sum_of[4 * WAVES * PER];
    const u64 at = (u64)blockIdx.x * PER + threadIdx.x / (64 * WAVES);
    const u32 in_row = threadIdx.x % (64 * WAVES), lane = threadIdx.x & 63;
    const u32 token = (u32)(at / a.heads), head = (u32)(at % a.heads);
    const u32 groups = 64 * WAVES / lanes, group = in_row / lanes, e = in_row % lanes * 4;
    const float *lse = a.part_lse + at * a.splits, *part = a.part + at * a.splits * a.head_dim + (e < a.head_dim ? e : 0);
    const bool row_ok = token < a.n_tokens;
    // The first splits' results and the sequences' lengths are under way before it is known which of them count.
    constexpr int EARLY = 4;
    float z0 = 0.0f, z[EARLY];
    float4 x[EARLY];
    if (row_ok) {
        z0 = lse[min(lane, a.splits - 1)];
#pragma unroll
        for (int k = 0; k < EARLY; ++k) {
            const u32 i = min(group + k * groups, a.splits - 1);
            z[k] = lse[i];
            x[k] = *(const float4 *)(part + (u64)i * a.head_dim);
        }
    }
    RowTile r;
    r.n_splits = 1;
    if (row_ok) {
        // the last sequence that starts at the token or before it: down to 64 by halves, then a lane for each
        u32 first = 0, count = a.n_seq;
        while (count > 64) {
            const u32 mid = first + count / 2;
            const bool up = (i64)a.q_start[mid] <= (i64)token;
            count = up ? count - count / 2 : count / 2;
            first = up ? mid : first;
        }
        const u32 b = first + min(lane, count - 1);
        const int start = a.q_start[b], next = a.q_start[b + 1], kv_len = a.kv_len[b];
        const u64 before = __ballot(lane < count && start <= (int)token);
        const int own = before ? 63 - __clzll(before) : 0;
        const int s = min(max(__shfl(start, own), 0), (int)a.n_tokens), end = max(min(__shfl(next, own), (int)a.n_tokens), s);
        const int kv = __shfl(kv_len, own);
        if ((int)token >= s && (int)token < end) {
            r.seq = first + own;
            r.start = s;
            r.n = end - s;
            r.rows = r.n * a.group;
            r.first_row = ((token - s) * a.group + head % a.group) / ROWS * ROWS;
            key_range<ROWS, TK>(a, kv, r);
        }
    }
    // one split: the row has been written already
    const u32 n = r.n_splits > 1 ? r.n_splits : 0;
    float top = lane < n ? z0 : -__builtin_inff();
    for (u32 i = lane + 64; i < n; i += 64) top = fmaxf(top, lse[i]);
#pragma unroll
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    float sum = 0.0f;
    float4 acc = make_float4(0, 0, 0, 0);
    auto add = [&](float zi, float4 xi) {
        // a split that saw no key has nothing to add; one whose sum is not a number has
        const float f = zi == -__builtin_inff() ? 0.0f : zi != zi ? zi : __builtin_amdgcn_exp2f(zi - top);
        sum += f;
        acc.x = __builtin_fmaf(f, xi.x, acc.x);
        acc.y = __builtin_fmaf(f, xi.y, acc.y);
        acc.z = __builtin_fmaf(f, xi.z, acc.z);
        acc.w = __builtin_fmaf(f, xi.w, acc.w);
    };
    if (e < a.head_dim) {
#pragma unroll
        for (int k = 0; k < EARLY; ++k)
            if (group + k * groups < n) add(z[k], x[k]);
#pragma unroll 4
        for (u32 i = group + EARLY * groups; i < n; i += groups) add(lse[i], *(const float4 *)(part + (u64)i * a.head_dim));
    }
    acc_of[threadIdx.x] = acc;
    if (e == 0) sum_of[threadIdx.x / lanes] = sum;
    __syncthreads();
    if (!n || group || e >= a.head_dim) return;
    for (u32 g = 1; g < groups; ++g) {
        const float4 x = acc_of[threadIdx.x + g * lanes];
        acc.x += x.x;
        acc.y += x.y;
        acc.z += x.z;
        acc.w += x.w;
    }
    sum = 0.0f;
    for (u32 g = 0; g < groups; ++g) sum += sum_of[threadIdx.x / lanes + g];
    const bool some = sum > 0.0f || sum != sum;
    const float inv = some ? 1.0f / sum : 0.0f;
    if (a.lse && e == 0) a.lse[at] = some ? (top + __log2f(sum)) * 0.693147180559945309f : -__builtin_inff();
    Pack<T, 4> y = {{(T)(some ? acc.x * inv : 0.0f), (T)(some ? acc.y * inv : 0.0f), (T)(some ? acc.z * inv : 0.0f), (T)(some ? acc.w * inv : 0.0f)}};
    store_pack<4>((T *)a.out + (i64)token * a.os[0] + head * a.os[1] + e, y);
}

// ---- host ----
// The forms of the kernel and what they cost, measured on prompts and single tokens with many and with few blocks: a block does
// `rows` rows, a step of `keys` keys takes step_us where it has its CU for itself and full_us where `fit` blocks share it, and
// begin_us goes into finding its rows, its first keys and its output.
struct AttendForm {
    u32 waves_rows, rows, tk, keys;  // RW; rows of a block; keys of a tile and of a step
    float begin_us, step_us, full_us;
    u32 fit;
};
constexpr AttendForm FORMS_64[] = {{1, 32, 32, 128, 6, 1.1f, 1.8f, 2}, {4, 128, 64, 64, 7, 1.3f, 2.3f, 3}};
constexpr AttendForm FORMS_128[] = {{1, 32, 32, 128, 6, 1.7f, 3.1f, 2}, {4, 128, 64, 64, 8, 1.8f, 2.6f, 2}, {8, 256, 64, 64, 10, 1.9f, 1.9f, 1}};
constexpr AttendForm FORMS_256[] = {{1, 32, 32, 128, 8, 4, 4, 1}, {4, 128, 32, 32, 10, 2.2f, 2.2f, 1}};
// 32-bit products are slow enough for each wave to read its keys by itself: with rows of 64 the form of shared tiles gains nothing
// (32 heads, 2 x 1024 tokens over 3024 keys: 439 us, apart 447); with rows of 128, where only one block of waves apart fits a CU,
// two with shared tiles do (963 -> 802 us).  Rows of 256 fit no other way.  The full costs of 16-bit single tokens are those with low parts of
// their weights (heads of 64 1.6, of 128 2.8 without).
constexpr AttendForm FORMS_F32_64[] = {{1, 32, 32, 128, 6, 4, 4, 1}};
constexpr AttendForm FORMS_F32_128[] = {{1, 32, 32, 128, 6, 8, 8, 1}, {4, 128, 32, 32, 10, 4.9f, 8.4f, 2}};
constexpr AttendForm FORMS_F32_256[] = {{4, 128, 32, 32, 10, 14, 14, 1}};

struct AttendPlan {
    AttendForm form;
    u32 dp, tiles, splits, min_tiles;
    u64 work_bytes;
};

// The form and the number of splits that the measured costs promise the least time for.  Lengths are on the device: the table's
// width bounds them, and sequences are taken to be of equal shares of the new tokens.
static bool plan_attend(const ckks_clear_attend_t &p, AttendPlan &n) {
    const ckks_clear_pages_t &g = p.pages;
    const ckks_clear_batch_t &b = p.batch;
    if (!clear_dtype_ok(g.dtype) || !g.head_dim || g.head_dim % 8 || g.head_dim > 256 || !g.kv_heads || !p.heads || p.heads % g.kv_heads ||
        p.heads > 1u << 16)
        return false;
    const u64 group = p.heads / g.kv_heads, rows = (u64)b.n_tokens * group, seqs = std::min(b.n_seq, b.n_tokens);
    const u64 width = (u64)b.table_width * g.page_size;
    if (rows >= 1u << 31 || width >= 1u << 31 || b.n_seq >= 1u << 31) return false;
    n.dp = g.head_dim <= 64 ? 64 : g.head_dim <= 128 ? 128 : 256;
    const bool f32 = g.dtype == CKKS_CLEAR_F32;
    const AttendForm *forms = f32 ? (n.dp == 64 ? FORMS_F32_64 : n.dp == 128 ? FORMS_F32_128 : FORMS_F32_256)
                                  : (n.dp == 64 ? FORMS_64 : n.dp == 128 ? FORMS_128 : FORMS_256);
    const u32 count = f32 ? (n.dp == 128 ? 2 : 1) : n.dp == 128 ? 3 : 2;
    constexpr double CUS = 256, READ = 4.9e6, JOIN = 1.5e6;  // bytes a microsecond
    const double per_seq = seqs ? (double)rows / seqs : 0, causal = p.flags & CKKS_CLEAR_CAUSAL;
    double keys = (double)width - (causal ? per_seq / group / 2 : 0);  // that a row sees, about
    if (p.window && p.window < width) keys = std::min<double>(keys, p.window + per_seq / group);
    keys = std::max(keys, 1.0);
    const double key_bytes = 2.0 * g.head_dim * clear_dtype_bytes(g.dtype), all = seqs * g.kv_heads * keys * key_bytes;
    double best = 0;
    n.splits = 0;
    for (u32 f = 0; f < count; ++f) {
        const AttendForm &form = forms[f];
        const double blocks = (seqs ? seqs * std::ceil(per_seq / form.rows) : 1) * g.kv_heads;
        const bool may_split = (u64)b.n_tokens * p.heads < 1u << 31;  // the joining kernel's grid
        const double most = !may_split ? 1.0 : std::max(1.0, std::min(1024.0, keys / form.keys / (form.waves_rows > 1 ? 4 : 1)));
        auto consider = [&](u32 splits) {
            if (splits < 1 || splits > most) return;
            const double load = blocks * splits / CUS, steps = std::ceil(keys / splits / form.keys);
            const double share = form.fit > 1 ? std::min(1.0, std::max(0.0, (load - 1) / (form.fit - 1))) : 0.0;
            const double step = form.step_us + share * (form.full_us - form.step_us), rounds = load / form.fit;
            const double work = (rounds <= 1 ? 1 : rounds < 3 ? std::ceil(rounds) : rounds + 0.5) * (form.begin_us + steps * step);
            // Reading the cache: slower with fewer CUs at it, or with one block on some and two on others; where sequences differ
            // in length, part of a block is left at the end.
            double read = all / READ / std::min(1.0, 1.3 * load);
            if (load > 1) read *= 0.5 + 0.5 * std::ceil(load) / load;
            if (seqs > 1) read += 0.15 * steps * form.keys * key_bytes * CUS * form.fit / READ;
            const double join = splits > 1 ? 5 + (double)b.n_tokens * p.heads * g.head_dim * 8 * splits / JOIN : 0;
            const double us = std::max(work, form.begin_us + read) + join;
            if (!n.splits || us < best) {
                best = us;
                n.form = form;
                n.splits = splits;
            }
        };
        for (u32 splits = 1; splits <= most; splits += std::max(1u, splits / 2)) consider(splits);
        for (u32 k = 1; k <= 2; ++k) consider((u32)std::min(1024.0, k * CUS / blocks));  // as many blocks as CUs, or twice that
    }
    const u64 tiles = rows / n.form.rows + seqs;  // at most
    if (tiles * g.kv_heads * n.splits >= 1u << 31) return false;
    n.tiles = (u32)tiles;
    n.min_tiles = 4;
    n.work_bytes = n.splits > 1 ? (u64)n.splits * b.n_tokens * p.heads * (g.head_dim + 1) * 4 : 0;
    return true;
}

template <class T, int DP, int RW, int KW, int TK, int OCC>
static int launch_attend(const AttendArgs &a, hipStream_t st) {
    hipLaunchKernelGGL((attend_kernel<T, DP, RW, KW, TK, OCC>), dim3(a.kv_heads * a.splits * a.tiles), dim3(64 * RW * KW), 0, st, a);
    CKKS_LAUNCH_CHECK("attend_kernel");
    if (a.splits > 1) {
        const u64 rows = (u64)a.n_tokens * a.heads;
        const u32 lanes = DP / 4;
        if (a.splits <= 8)
            hipLaunchKernelGGL((attend_join_kernel<T, 32 * RW, TK, 1>), dim3((u32)((rows + 3) / 4)), dim3(256), 0, st, a, lanes);
        else if (a.splits <= 32)
            hipLaunchKernelGGL((attend_join_kernel<T, 32 * RW, TK, 4>), dim3((u32)rows), dim3(256), 0, st, a, lanes);
        else
            hipLaunchKernelGGL((attend_join_kernel<T, 32 * RW, TK, 16>), dim3((u32)rows), dim3(1024), 0, st, a, lanes);
        CKKS_LAUNCH_CHECK("attend_join_kernel");
    }
    return CKKS_OK;
}
template <class T>
static int launch_attend(const AttendArgs &a, const AttendPlan &n, hipStream_t st) {
    if constexpr (sizeof(T) == 4) {
        if (n.dp == 64) return launch_attend<T, 64, 1, 4, 32, 1>(a, st);
        if (n.dp == 128) return n.form.waves_rows == 1 ? launch_attend<T, 128, 1, 4, 32, 1>(a, st) : launch_attend<T, 128, 4, 1, 32, 2>(a, st);
        return launch_attend<T, 256, 4, 1, 32, 1>(a, st);
    } else {
        if (n.dp == 64) return n.form.waves_rows == 1 ? launch_attend<T, 64, 1, 4, 32, 2>(a, st) : launch_attend<T, 64, 4, 1, 64, 2>(a, st);
        if (n.dp == 256) return n.form.waves_rows == 1 ? launch_attend<T, 256, 1, 4, 32, 1>(a, st) : launch_attend<T, 256, 4, 1, 32, 1>(a, st);
        return n.form.waves_rows == 1   ? launch_attend<T, 128, 1, 4, 32, 2>(a, st)
               : n.form.waves_rows == 4 ? launch_attend<T, 128, 4, 1, 64, 2>(a, st)
                                        : launch_attend<T, 128, 8, 1, 64, 2>(a, st);
    }
}

}  // namespace ckks

using namespace ckks;

extern "C" {

uint64_t ckks_clear_attend_work_bytes(const ckks_clear_attend_t *p) {
    AttendPlan n;
    return p && plan_attend(*p, n) ? n.work_bytes : 0;
}

int ckks_clear_attend(const ckks_clear_attend_t *p, void *stream) {
    const char *who = "ckks_clear_attend";
    if (!p) {
        set_error("%s: null argument", who);
        return CKKS_E_INVAL;
    }
    const ckks_clear_pages_t &g = p->pages;
    const ckks_clear_batch_t &b = p->batch;
    if (int rc = check_cache(who, g, b)) return rc;
    AttendPlan n;
    if (!plan_attend(*p, n)) {
        set_error("%s: %u heads over %u kv heads, %u tokens", who, p->heads, g.kv_heads, b.n_tokens);
        return CKKS_E_INVAL;
    }
    if ((p->flags & ~CKKS_CLEAR_CAUSAL) || (p->window && !(p->flags & CKKS_CLEAR_CAUSAL)) || !(p->scale > 0.0f) || !std::isfinite(p->scale)) {
        set_error("%s: flags %u, window %u (causal only), scale %g", who, p->flags, p->window, (double)p->scale);
        return CKKS_E_INVAL;
    }
    if (!b.n_tokens || !b.n_seq) return CKKS_OK;
    if (!p->d_q || !p->d_out) {
        set_error("%s: null argument", who);
        return CKKS_E_INVAL;
    }
    if (n.work_bytes > p->work_bytes || (n.work_bytes && (!p->d_work || (uintptr_t)p->d_work % 16))) {
        set_error("%s: workspace of %llu bytes, needs %llu (16-byte aligned)", who, (unsigned long long)p->work_bytes, (unsigned long long)n.work_bytes);
        return CKKS_E_INVAL;
    }
    const u32 e = clear_dtype_bytes(g.dtype);
    const Extent out[3] = {extent(p->d_out, e, {{b.n_tokens, p->out_stride[0]}, {p->heads, p->out_stride[1]}, {g.head_dim, 1}}),
                           extent(p->d_lse, 4, {{p->d_lse ? b.n_tokens : 0, p->heads}, {p->heads, 1}}), extent(p->d_work, 1, {{n.work_bytes, 1}})};
    const Extent in[6] = {extent(p->d_q, e, {{b.n_tokens, p->q_stride[0]}, {p->heads, p->q_stride[1]}, {g.head_dim, 1}}),
                          extent(g.d_k, e, {{g.n_pages, g.k_stride[0]}, {g.kv_heads, g.k_stride[1]}, {g.page_size, g.k_stride[2]}, {g.head_dim, 1}}),
                          extent(g.d_v, e, {{g.n_pages, g.v_stride[0]}, {g.kv_heads, g.v_stride[1]}, {g.page_size, g.v_stride[2]}, {g.head_dim, 1}}),
                          extent(b.d_q_start, 4, {{b.n_seq + 1, 1}}),
                          extent(b.d_kv_len, 4, {{b.n_seq, 1}}),
                          extent(b.d_page_table, 4, {{b.n_seq, b.table_stride}, {b.table_width, 1}})};
    bool bad = overlap(out[0], out[1]) || overlap(out[0], out[2]) || overlap(out[1], out[2]);
    for (const Extent &o : out)
        for (const Extent &i : in) bad |= overlap(o, i);
    if (bad) {
        set_error("%s: an output overlaps another array", who);
        return CKKS_E_INVAL;
    }
    if (share_within({p->d_out, g.head_dim * e, 2, {{b.n_tokens, p->out_stride[0] * e}, {p->heads, p->out_stride[1] * e}}})) {
        set_error("%s: rows of the output overlap", who);
        return CKKS_E_INVAL;
    }
    AttendArgs a{};
    a.q = p->d_q, a.k = g.d_k, a.v = g.d_v, a.out = p->d_out, a.lse = p->d_lse;
    a.part_lse = (float *)p->d_work;
    a.part = a.part_lse;
    if (n.splits > 1) {  // partial results first: 16-byte rows where head_dim is a multiple of 4
        a.part = (float *)p->d_work;
        a.part_lse = a.part + (u64)n.splits * b.n_tokens * p->heads * g.head_dim;
    }
    for (int i = 0; i < 2; ++i) a.qs[i] = p->q_stride[i], a.os[i] = p->out_stride[i];
    for (int i = 0; i < 3; ++i) a.ks[i] = g.k_stride[i], a.vs[i] = g.v_stride[i];
    a.ts = b.table_stride, a.q_start = b.d_q_start, a.kv_len = b.d_kv_len, a.table = b.d_page_table;
    if (!g.n_pages) {  // nothing is a page: what is fetched in its place, and not used, comes from the queries
        a.k = a.v = p->d_q;
        for (int i = 0; i < 3; ++i) a.ks[i] = a.vs[i] = 0;
    }
    a.n_seq = b.n_seq, a.n_tokens = b.n_tokens, a.n_pages = g.n_pages, a.page_size = g.page_size, a.table_width = b.table_width;
    a.kv_heads = g.kv_heads, a.heads = p->heads, a.group = p->heads / g.kv_heads, a.head_dim = g.head_dim;
    // a window of all positions is none
    a.window = p->window < (u64)b.table_width * g.page_size ? (int)p->window : 0, a.causal = p->flags & CKKS_CLEAR_CAUSAL;
    // positions are below 2^31: with l = ceil(log2(page_size)) the quotient by ceil(2^(31+l) / page_size) / 2^(31+l) is exact
    while (a.page_shift < 31 && (1u << a.page_shift) < g.page_size) ++a.page_shift;
    a.page_mul = (u32)((((u64)1 << (31 + a.page_shift)) + g.page_size - 1) / g.page_size);
    a.alike = a.ks[0] == a.vs[0] && a.ks[2] == a.vs[2];
    a.tiles = n.tiles, a.splits = n.splits, a.min_tiles = n.min_tiles;
    a.c = p->scale * 1.44269504088896340736f;
    hipStream_t st = (hipStream_t)stream;
    return g.dtype == CKKS_CLEAR_F32   ? launch_attend<float>(a, n, st)
           : g.dtype == CKKS_CLEAR_F16 ? launch_attend<f16>(a, n, st)
                                       : launch_attend<bf16>(a, n, st);
}

}  // extern "C"
