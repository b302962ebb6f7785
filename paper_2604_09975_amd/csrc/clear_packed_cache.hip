// New keys and values into pages of 8 bits, keys and queries normed and rotated on the way, and rows read back.
//
// A head's entries lie eight to a lane in a group of G lanes, so that four lanes hold a block of 32 and the group a head.  A wave
// takes a token, its groups the token's heads one after the other, values, keys, queries: place, angles and weights are looked up once.
//
// Rounding to 8 bits is the only rounding that may show, so what leads there is exact or in 64 bits, which the vector units do at
// the rate of 32: with weight w, angle (c, s) and partner x' (weight w') an entry is r (x w c +- x' w' s), where w c and w' s are
// exact products, worked out once for all heads of the token, and r = 1/sqrt(mean(x^2) + eps).  Of the 53 bits the upper 21 go on,
// the last of them set if anything below is (round to odd): rounding that to a type of 19 bits or fewer rounds once.
//
// Many tokens are bound by memory: 22600 tokens of 32 heads and 8 kv heads of 128 in bf16, normed and rotated, take 128 us (512 MB, 4.0
// TB/s), 111 without norm and rotation (4.6), F32 into I8 195 (5.0).  A few tokens are bound by one wave's way through place, angles
// and sum (3.7 us), so there each turn of a token's work has a wave of its own.  Weights go through LDS (the block's tokens share them)
// and the first rows are loaded after them: with those loads ahead of the weights 143 us instead of 128, in scalar loads 158.
#include <algorithm>

#include "clear_packed.h"

namespace ckks {

struct PackedAppendArgs {
    const void *k, *v, *q;
    unsigned char *pk, *pv, *zk, *zv;
    void *qo;
    i64 ks[2], vs[2], qs[2], qos[2], pks[3], pvs[3], zks[3], zvs[3], ts;
    const void *k_norm, *q_norm;
    const float *cos, *sin;
    const int32_t *positions, *q_start, *kv_len, *table;
    u32 n_seq, n_tokens, n_pages, page_size, table_width, kv_heads, heads, head_dim, rot, n_pos, interleaved, norm_f32, slices, kinds, t0;
    double eps, inv_dim;
};

// Sequence of a token: the last b < n_seq with start[b] <= t, by the 64 lanes of a wave together.
__device__ __forceinline__ u32 find_seq_wave(const int32_t *start, u32 n_seq, u32 t) {
    const u32 lane = threadIdx.x & 63;
    u32 lo = 0, n = n_seq;  // it is lo or within the n from there
    while (n > 1) {
        const u32 step = (n + 63) / 64, at = lane * step;
        const bool up = at < n && (i64)start[lo + at] <= (i64)t;
        const u64 all = __ballot(up);
        const u32 k = all ? 63 - __clzll(all) : 0;
        lo += k * step;
        n = min(step, n - k * step);
    }
    return lo;
}

struct TokenPlace {
    u32 b;
    i64 pos, page;  // < 0: none
    u32 row;
};
// Where token t (the same in all lanes) lies.
template <class A>
__device__ __forceinline__ TokenPlace place_of(const A &a, u32 t) {
    TokenPlace p;
    p.b = find_seq_wave(a.q_start, a.n_seq, t);
    const i64 end = min((i64)a.q_start[p.b + 1], (i64)a.n_tokens);
    const i64 kv = min((i64)a.kv_len[p.b], (i64)a.table_width * a.page_size);
    const bool in = (i64)t >= (i64)a.q_start[p.b] && (i64)t < end;
    p.pos = in ? kv - (end - (i64)t) : -1;
    p.page = -1;
    p.row = 0;
    if (p.pos >= 0) {
        const u32 page = (u32)a.table[(i64)p.b * a.ts + (u32)p.pos / a.page_size];
        p.page = page < a.n_pages ? (i64)page : -1;
        p.row = (u32)p.pos % a.page_size;
    } else {
        p.pos = in ? -1 : -2;  // -2: in no sequence
    }
    return p;
}

// Neighbours' values without LDS: DPP within 16 lanes.
template <int CTRL>
__device__ __forceinline__ u32 dpp(u32 x) {
    return (u32)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ __forceinline__ double dpp(double x) {
    const u64 b = (u64)__double_as_longlong(x);
    return __longlong_as_double((long long)((u64)dpp<CTRL>((u32)(b >> 32)) << 32 | dpp<CTRL>((u32)b)));
}
constexpr int XOR1 = 0xb1, XOR2 = 0x4e, MIRROR8 = 0x141, MIRROR16 = 0x140;
// Over the four lanes of a block.
__device__ __forceinline__ u32 max_of_block(u32 x) {
    x = max(x, dpp<XOR1>(x));
    return max(x, dpp<XOR2>(x));
}
// Over the G lanes of a head, the same sum in all of them.
template <int G>
__device__ __forceinline__ double sum_of_head(double x) {
    x += dpp<XOR1>(x);
    x += dpp<XOR2>(x);
    if (G > 4) x += dpp<MIRROR8>(x);
    if (G > 8) x += dpp<MIRROR16>(x);
    if (G > 16) x += __shfl_xor(x, 16);
    return x;
}

// The upper 21 bits of a double as a float, the last one set where a bit below is.
__device__ __forceinline__ float to_odd(double x) {
    const u64 b = (u64)__double_as_longlong(x);
    const u32 hi = (u32)(b >> 32) | min((u32)b, 1u);
    return (float)__longlong_as_double((long long)((u64)hi << 32));
}
// 1 / sqrt(x) to the last bits of a double: the hardware's value and a step of third order.
__device__ __forceinline__ double rsqrt_of(double x) {
    const double y = __builtin_amdgcn_rsq(x);
    const double e = __builtin_fma(-x * y, y, 1.0);
    const double r = __builtin_fma(y * e, __builtin_fma(e, 0.375, 0.5), y);
    return x < __builtin_inf() ? r : y;  // infinity: 0
}

// Blocks whose entries T holds end below TOP (as T rounds, where that is still to be done).  Of those above HIGH, with their last power, a code
// of 256 or 64 stands for 2^16 (F16) or 2^128, which T does not hold; the one before it is right.
template <class T, int FORM>
struct Range {
    static constexpr bool F = std::is_same<T, f16>::value;
    static constexpr float TOP = F ? 65520.0f : __builtin_inff();
    static constexpr float HIGH = FORM == E4M3 ? (F ? 448 * 0x1p7f : 448 * 0x1p119f) : (F ? 127 * 0x1p9f : 127 * 0x1p121f);
};

// Eight entries of a block of 32 spread over four lanes, as codes; `power` is the block's.
template <class T, int FORM>
__device__ __forceinline__ uint2 pack8(const float *x, u32 &power) {
    typedef Range<T, FORM> range;
    u32 top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    top = max_of_block(top);
    // M is 1.75 * 2^8 or 1.984375 * 2^6
    constexpr u32 SHIFT = FORM == E4M3 ? 8 : 6, MANTISSA = FORM == E4M3 ? 0x600000u : 0x7e0000u, LEAST = 127 - 100;
    const u32 e = (top >> 23) + ((top & 0x7fffffu) > MANTISSA);
    power = top >= 0x7f800000u ? 255u : max(e, LEAST + SHIFT) - SHIFT;
    const float f = __uint_as_float((254 - min(power, 253u)) << 23);
    const bool high = top > __builtin_bit_cast(u32, range::HIGH) && top < __builtin_bit_cast(u32, range::TOP);
    uint2 r;
    if (FORM == E4M3) {
        int lo = 0, hi = 0;
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * f, x[1] * f, lo, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * f, x[3] * f, lo, true);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[4] * f, x[5] * f, hi, false);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[6] * f, x[7] * f, hi, true);
        r = make_uint2((u32)lo, (u32)hi);
        if (__any(high))
            if (high) {
                // 0x78 is the last code that such a block has; bit 7 of a byte of y is set where it is
                auto before = [](u32 w) {
                    const u32 y = 0x80808080u - ((w & 0x7f7f7f7fu) ^ 0x78787878u);
                    return w - ((y & 0x80808080u) >> 7);
                };
                r = make_uint2(before(r.x), before(r.y));
            }
    } else {
        // x 2^-e is exact, and its sum with 1.5 2^23 is rounded to a whole number, whose lowest bits are the code
        const float end = high ? 63.0f : 127.0f;
        u32 c[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = __float_as_uint(__builtin_amdgcn_fmed3f(x[i] * f, -end, end) + 12582912.0f) & 0xffu;
        r = make_uint2(c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24);
    }
    if (power == 255) r = make_uint2(0, 0);
    return r;
}

// The arguments, read anew: held all at once they would take more scalar registers than there are, and go through vector registers
// lane by lane.
typedef const __attribute__((address_space(4))) PackedAppendArgs LateArgs;
__device__ __forceinline__ LateArgs *late_args() {
    LateArgs *p = (LateArgs *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return p;
}

// A job: a token, and of its values (kind 0), keys (1) and queries (2) all or, where there are few tokens, one.
template <class T, int FORM, int G>
__global__ __launch_bounds__(256, 4) void packed_append_kernel(PackedAppendArgs a) {
    constexpr u32 GROUPS = 64 / G;
    __shared__ __attribute__((aligned(16))) float lds[256 * 8];
    __shared__ __attribute__((aligned(16))) float weights[2][G * 8];  // of keys, of queries
    const u32 lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (u32 k = 0; k < 2; ++k) {
        const void *norm = k ? a.q_norm : a.k_norm;
        for (u32 i = threadIdx.x; i < G * 8; i += 256)
            weights[k][i] = !norm || i >= a.head_dim ? 1.0f : a.norm_f32 ? ((const float *)norm)[i] : (float)((const T *)norm)[i];
    }
    __syncthreads();
    const u32 t = a.t0 + blockIdx.x * 4 + wave, kinds = a.kinds, only = blockIdx.y % kinds, slice = blockIdx.y / kinds;
    if (t >= a.n_tokens) return;
    const u32 first = slice * GROUPS + lane / G, step = a.slices * GROUPS;  // heads of the group
    const u32 c = lane % G * 8, dim = a.head_dim, rot = a.rot, half = rot / 2;
    const bool live = c < dim, interleaved = a.interleaved;
    const u32 at_c = live ? c : 0;
    const TokenPlace at = place_of(a, t);
    float *own = lds + (threadIdx.x - lane % G) * 8;  // the head's entries

    // use(head, entries) for the group's heads, the next one's entries under way
    auto each_head = [&](const void *rows, i64 stride0, i64 stride1, u32 heads, auto use) {
        const T *src = (const T *)rows + (i64)t * stride0 + at_c;
        Pack<T, 8> next{};
        if (first < heads) next = load_pack<8>(src + first * stride1);
        for (u32 h = first; h < heads; h += step) {
            const Pack<T, 8> in = next;
            next = load_pack<8>(src + min(h + step, heads - 1) * stride1);
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = live ? (float)in.v[i] : 0.0f;
            use(h, x);
        }
    };
    auto store_codes = [&](const float *x, unsigned char *codes, unsigned char *powers) {
        u32 power;
        const uint2 packed = pack8<T, FORM>(x, power);
        if (live) {
            __builtin_memcpy(codes + c, &packed, 8);
            if (c % PACK_BLOCK == 0) powers[c / PACK_BLOCK] = (unsigned char)power;
        }
    };
    if (at.page >= 0 && (kinds == 1 || only == 0)) {
        LateArgs *p = late_args();
        unsigned char *codes = p->pv + at.page * p->pvs[0] + (i64)at.row * p->pvs[2], *powers = p->zv + at.page * p->zvs[0] + (i64)at.row * p->zvs[2];
        const i64 sc = p->pvs[1], sz = p->zvs[1];
        each_head(p->v, p->vs[0], p->vs[1], p->kv_heads, [&](u32 h, const float *x) { store_codes(x, codes + h * sc, powers + h * sz); });
    }
    if (kinds > 1 && only == 0) return;

    // Keys and queries: A of an entry is its weight times the cosine, B its partner's weight times +-sine.
    const bool by_four = !interleaved && half % 4 == 0, part = rot < dim;
    auto partner = [&](u32 j) { return j >= rot ? j : interleaved ? j ^ 1 : j < half ? j + half : j - half; };
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) cs[i] = 1.0f, sn[i] = 0.0f;
    if (rot) {
        LateArgs *p = late_args();
        const i64 angle_at = p->positions ? (i64)p->positions[t] : at.pos;
        const bool angle = angle_at >= 0 && angle_at < (i64)p->n_pos;
        const float *cos = p->cos + (angle ? angle_at * half : 0), *sin = p->sin + (angle ? angle_at * half : 0);
        const u32 f = interleaved ? c / 2 : c < half ? c : c - half;
        if (angle && rot % 8 == 0 && (interleaved || half % 8 == 0)) {  // all of a lane's entries are rotated, or none
            if (c >= rot) {
            } else if (interleaved) {
                const Pack<float, 4> u = load_pack<4>(cos + f), v = load_pack<4>(sin + f);
#pragma unroll
                for (int i = 0; i < 8; ++i) cs[i] = u.v[i / 2], sn[i] = i % 2 ? v.v[i / 2] : -v.v[i / 2];
            } else {
                const Pack<float, 8> u = load_pack<8>(cos + f), v = load_pack<8>(sin + f);
#pragma unroll
                for (int i = 0; i < 8; ++i) cs[i] = u.v[i], sn[i] = c < half ? -v.v[i] : v.v[i];
            }
        } else if (p->n_pos) {
            // every lane loads, some for nothing: a branch around a load would be a wait for it
            float u[8], v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const u32 j = c + i, f = j >= rot ? 0 : interleaved ? j / 2 : j < half ? j : j - half;
                u[i] = cos[f];
                v[i] = sin[f];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const u32 j = c + i;
                const bool minus = interleaved ? !(j & 1) : j < half;
                if (j < rot) {
                    cs[i] = angle ? u[i] : __builtin_nanf("");
                    sn[i] = angle ? (minus ? -v[i] : v[i]) : 0.0f;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) cs[i] = c + i < rot ? __builtin_nanf("") : 1.0f;
        }
    }
    // where the partners of a head's entries stand in LDS
    const u32 pa = live ? partner(c) : c, pb = live ? partner(c + 4) : c + 4;
    auto partners_of = [&](const float *x, float *p) {
        if (by_four) {
            const float4 u = *(const float4 *)(x + pa), v = *(const float4 *)(x + pb);
            p[0] = u.x, p[1] = u.y, p[2] = u.z, p[3] = u.w;
            p[4] = v.x, p[5] = v.y, p[6] = v.z, p[7] = v.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = x[live ? partner(c + i) : c];
        }
    };
    auto partners = [&](const float *x, float *p) {
        if (interleaved) {
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = x[i ^ 1];
        } else {
            *(float4 *)(own + c) = make_float4(x[0], x[1], x[2], x[3]);
            *(float4 *)(own + c + 4) = make_float4(x[4], x[5], x[6], x[7]);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            partners_of(own, p);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        if (part)  // those that are not rotated have none, whatever stands in their place
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = c + i < rot ? p[i] : 0.0f;
    };
    auto factors = [&](const float *w, double *A, double *B) {
        float wp[8];
        partners_of(w, wp);
#pragma unroll
        for (int i = 0; i < 8; ++i) A[i] = (double)cs[i] * (double)w[c + i], B[i] = (double)sn[i] * (double)wp[i];
    };
    const double eps = a.eps, inv_dim = a.inv_dim;
    auto turned = [&](bool norm, const double *A, const double *B, const float *x, double *y) {
        double r = 1.0;
        if (norm) {
            double ss = 0.0;
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = __builtin_fma((double)x[i], (double)x[i], ss);
            r = rsqrt_of(__builtin_fma(sum_of_head<G>(ss), inv_dim, eps));
        }
        if (rot) {
            float p[8];
            partners(x, p);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = __builtin_fma((double)p[i], B[i], (double)x[i] * A[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = (double)x[i] * A[i];
        }
        if (norm)
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] *= r;
    };
    double A[8], B[8];
    if (at.page >= 0 && (kinds == 1 || only == 1)) {
        LateArgs *p = late_args();
        const bool norm = p->k_norm, plain = !norm && !rot;
        factors(weights[0], A, B);
        unsigned char *codes = p->pk + at.page * p->pks[0] + (i64)at.row * p->pks[2], *powers = p->zk + at.page * p->zks[0] + (i64)at.row * p->zks[2];
        const i64 sc = p->pks[1], sz = p->zks[1];
        each_head(p->k, p->ks[0], p->ks[1], p->kv_heads, [&](u32 h, float *x) {
            if (!plain) {
                double y[8];
                turned(norm, A, B, x, y);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = to_odd(y[i]);
            }
            store_codes(x, codes + h * sc, powers + h * sz);
        });
    }
    if (kinds == 1 || only == 2) {
        LateArgs *p = late_args();
        const bool norm = p->q_norm, plain = !norm && !rot;
        factors(weights[1], A, B);
        T *out = (T *)p->qo + (i64)t * p->qos[0] + c;
        const i64 so = p->qos[1];
        each_head(p->q, p->qs[0], p->qs[1], p->heads, [&](u32 h, float *x) {
            Pack<T, 8> y8;
            if (!plain) {
                double y[8];
                turned(norm, A, B, x, y);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = (float)y[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) y8.v[i] = (T)x[i];
            if (live) store_pack<8>(out + h * so, y8);
        });
    }
}

struct PackedReadArgs {
    const unsigned char *pk, *pv, *zk, *zv;
    void *ko, *vo;
    i64 pks[3], pvs[3], zks[3], zvs[3], kos[2], vos[2], ts;
    const int32_t *q_start, *kv_len, *table;
    u32 n_seq, n_tokens, n_pages, page_size, table_width, kv_heads, head_dim, slices, t0;
};

// A wave takes a token, a lane eight entries.  Bound by memory: 101 thousand tokens of 8 heads of 128 (214 MB) as bf16
// rows (415 MB) take 129 us, 4.9 TB/s.
template <class T, int FORM>
__global__ __launch_bounds__(256) void packed_read_kernel(PackedReadArgs a) {
    const u32 lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const u64 job = (u64)blockIdx.x * 4 + wave;
    const u32 t = a.t0 + (u32)(job / a.slices), slice = (u32)(job % a.slices);
    if (t >= a.n_tokens) return;
    const TokenPlace at = place_of(a, t);
    if (at.pos == -2) return;
    const u32 per = a.head_dim / 8, n = a.kv_heads * per;
    for (u32 i = slice * 64 + lane; i < 2 * n; i += a.slices * 64) {
        const bool is_k = i < n;
        if (!(is_k ? a.ko : a.vo)) continue;
        const u32 j = is_k ? i : i - n, head = j / per, c = j % per * 8;
        uint2 codes = make_uint2(0, 0);
        u32 power = 0;
        if (at.page >= 0) {
            const unsigned char *src = is_k ? a.pk + at.page * a.pks[0] + head * a.pks[1] + (i64)at.row * a.pks[2]
                                            : a.pv + at.page * a.pvs[0] + head * a.pvs[1] + (i64)at.row * a.pvs[2];
            const unsigned char *z = is_k ? a.zk + at.page * a.zks[0] + head * a.zks[1] + (i64)at.row * a.zks[2]
                                          : a.zv + at.page * a.zvs[0] + head * a.zvs[1] + (i64)at.row * a.zvs[2];
            __builtin_memcpy(&codes, src + c, 8);
            power = z[c / PACK_BLOCK];
        }
        Pack<T, 8> out;
        unpack4<T, FORM>(codes.x, power_of<FORM>(power), out.v);
        unpack4<T, FORM>(codes.y, power_of<FORM>(power), out.v + 4);
        T *dst = is_k ? (T *)a.ko + (i64)t * a.kos[0] + head * a.kos[1] : (T *)a.vo + (i64)t * a.vos[0] + head * a.vos[1];
        store_pack<8>(dst + c, out);
    }
}

// Waves of a token: enough to fill the CUs where there are few tokens, at most one for each turn of its work.
// (a launch has fewer than 2^32 threads: tokens of one)
constexpr u32 TOKENS = 1u << 25;
static u32 slices_of(u32 n_tokens, u32 turns) { return std::max(1u, std::min(turns, 4096 / std::max(n_tokens, 1u))); }

template <class T, int FORM, int G>
static int launch_packed_append(PackedAppendArgs a, hipStream_t st) {
    a.slices = slices_of(a.n_tokens, (std::max(a.kv_heads, a.heads) + 64 / G - 1) / (64 / G));
    a.kinds = a.n_tokens * a.slices <= 2048 ? 3 : 1;
    for (; a.t0 < a.n_tokens; a.t0 += TOKENS) {
        hipLaunchKernelGGL((packed_append_kernel<T, FORM, G>), dim3((std::min(a.n_tokens - a.t0, TOKENS) + 3) / 4, a.slices * a.kinds), dim3(256), 0, st, a);
        CKKS_LAUNCH_CHECK("packed_append_kernel");
    }
    return CKKS_OK;
}
template <class T, int FORM>
static int launch_packed_append(const PackedAppendArgs &a, hipStream_t st) {
    return a.head_dim <= 32    ? launch_packed_append<T, FORM, 4>(a, st)
           : a.head_dim <= 64  ? launch_packed_append<T, FORM, 8>(a, st)
           : a.head_dim <= 128 ? launch_packed_append<T, FORM, 16>(a, st)
                               : launch_packed_append<T, FORM, 32>(a, st);
}
template <class T>
static int launch_packed_append(const PackedAppendArgs &a, u32 format, hipStream_t st) {
    return format == CKKS_CLEAR_E4M3 ? launch_packed_append<T, E4M3>(a, st) : launch_packed_append<T, I8>(a, st);
}
template <class T>
static int launch_packed_read(PackedReadArgs a, u32 format, hipStream_t st) {
    a.slices = slices_of(a.n_tokens, (2 * a.kv_heads * (a.head_dim / 8) + 63) / 64);
    for (; a.t0 < a.n_tokens; a.t0 += TOKENS) {
        const u32 blocks = (std::min(a.n_tokens - a.t0, TOKENS) * a.slices + 3) / 4;
        if (format == CKKS_CLEAR_E4M3)
            hipLaunchKernelGGL((packed_read_kernel<T, E4M3>), dim3(blocks), dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((packed_read_kernel<T, I8>), dim3(blocks), dim3(256), 0, st, a);
        CKKS_LAUNCH_CHECK("packed_read_kernel");
    }
    return CKKS_OK;
}

}  // namespace ckks

using namespace ckks;

extern "C" {

int ckks_clear_packed_append(const ckks_clear_packed_append_t *p, void *stream) {
    const char *who = "ckks_clear_packed_append";
    if (!p) {
        set_error("%s: null argument", who);
        return CKKS_E_INVAL;
    }
    const ckks_clear_packed_t &g = p->pages;
    const ckks_clear_batch_t &b = p->batch;
    if (int rc = check_packed(who, g, b)) return rc;
    if (!b.n_tokens || !b.n_seq) return CKKS_OK;
    if (!p->d_new_k || !p->d_new_v || (p->d_q && (!p->d_q_out || !p->heads)) || (p->d_q_norm && !p->d_q)) {
        set_error("%s: null argument", who);
        return CKKS_E_INVAL;
    }
    if (p->rot % 2 || p->rot > g.head_dim || (p->rot && (!p->d_cos || !p->d_sin)) || (p->flags & ~CKKS_CLEAR_INTERLEAVED)) {
        set_error("%s: rotation of %u of %u entries (flags %u)", who, p->rot, g.head_dim, p->flags);
        return CKKS_E_INVAL;
    }
    const bool norms = p->d_k_norm || p->d_q_norm;
    if (norms && ((p->norm_dtype != CKKS_CLEAR_F32 && p->norm_dtype != g.dtype) || !(p->eps >= 0.0f) || p->eps > 3.4e38f)) {
        set_error("%s: norms by weights of type %u, eps %g", who, p->norm_dtype, (double)p->eps);
        return CKKS_E_INVAL;
    }
    const u32 heads = p->d_q ? p->heads : 0;
    if (heads > 1u << 16) {
        set_error("%s: %u heads", who, heads);
        return CKKS_E_INVAL;
    }
    const u32 e = clear_dtype_bytes(g.dtype), ne = norms ? clear_dtype_bytes(p->norm_dtype) : 0;
    const PackedPlaces pages = packed_places(g);
    const Extent q_out = extent(p->d_q_out, e, {{heads ? b.n_tokens : 0, p->q_out_stride[0]}, {heads, p->q_out_stride[1]}, {g.head_dim, 1}});
    // the last three may lie between the rows of queries that are rotated in place
    const Extent in[11] = {extent(p->d_cos, 4, {{p->rot ? p->n_pos : 0, p->rot / 2}, {p->rot / 2, 1}}),
                           extent(p->d_sin, 4, {{p->rot ? p->n_pos : 0, p->rot / 2}, {p->rot / 2, 1}}),
                           extent(b.d_q_start, 4, {{b.n_seq + 1, 1}}),
                           extent(b.d_kv_len, 4, {{b.n_seq, 1}}),
                           extent(b.d_page_table, 4, {{b.n_seq, b.table_stride}, {b.table_width, 1}}),
                           extent(p->d_positions, 4, {{p->d_positions ? b.n_tokens : 0, 1}}),
                           extent(p->d_k_norm, ne, {{p->d_k_norm ? g.head_dim : 0, 1}}),
                           extent(p->d_q_norm, ne, {{p->d_q_norm ? g.head_dim : 0, 1}}),
                           extent(p->d_new_k, e, {{b.n_tokens, p->new_k_stride[0]}, {g.kv_heads, p->new_k_stride[1]}, {g.head_dim, 1}}),
                           extent(p->d_new_v, e, {{b.n_tokens, p->new_v_stride[0]}, {g.kv_heads, p->new_v_stride[1]}, {g.head_dim, 1}}),
                           extent(p->d_q, e, {{heads ? b.n_tokens : 0, p->q_stride[0]}, {heads, p->q_stride[1]}, {g.head_dim, 1}})};
    const auto runs = [&](const void *at, u32 n, const int64_t *st) { return Runs{at, g.head_dim * e, 2, {{b.n_tokens, st[0] * e}, {n, st[1] * e}}}; };
    const Runs q_rows = runs(p->d_q_out, heads, p->q_out_stride);
    const bool in_place = p->d_q == p->d_q_out && p->q_stride[0] == p->q_out_stride[0] && p->q_stride[1] == p->q_out_stride[1];
    bool bad = false;
    for (int i = 0; i < 4; ++i) {
        bad |= overlap(pages.at[i], q_out);
        for (const Extent &x : in) bad |= overlap(pages.at[i], x);
        // codes and powers may lie in one array, but not in the same places of it
        for (int j = 0; j < i; ++j)
            if (overlap(pages.at[i], pages.at[j])) bad |= share_any(pages.cells[i], pages.cells[j]);
    }
    for (int i = 0; i < 11; ++i)
        if (overlap(q_out, in[i])) {
            if (i < 8 || !in_place)
                bad = true;
            else if (i < 10)
                bad |= share(q_rows, i == 8 ? runs(p->d_new_k, g.kv_heads, p->new_k_stride) : runs(p->d_new_v, g.kv_heads, p->new_v_stride));
        }
    if (bad) {
        set_error("%s: an output overlaps another array", who);
        return CKKS_E_INVAL;
    }
    bool folded = heads && share_within(q_rows);
    for (int i = 0; i < 4; ++i) folded |= share_within(pages.cells[i]);
    if (folded) {
        set_error("%s: rows of an output overlap", who);
        return CKKS_E_INVAL;
    }
    PackedAppendArgs a{};
    a.k = p->d_new_k, a.v = p->d_new_v, a.q = p->d_q, a.qo = p->d_q_out;
    a.pk = g.d_k, a.pv = g.d_v, a.zk = g.d_k_power, a.zv = g.d_v_power;
    for (int i = 0; i < 2; ++i)
        a.ks[i] = p->new_k_stride[i], a.vs[i] = p->new_v_stride[i], a.qs[i] = p->q_stride[i], a.qos[i] = p->q_out_stride[i];
    for (int i = 0; i < 3; ++i)
        a.pks[i] = g.k_stride[i], a.pvs[i] = g.v_stride[i], a.zks[i] = g.k_power_stride[i], a.zvs[i] = g.v_power_stride[i];
    a.ts = b.table_stride, a.k_norm = p->d_k_norm, a.q_norm = p->d_q_norm, a.cos = p->d_cos, a.sin = p->d_sin, a.positions = p->d_positions;
    a.q_start = b.d_q_start, a.kv_len = b.d_kv_len, a.table = b.d_page_table;
    a.n_seq = b.n_seq, a.n_tokens = b.n_tokens, a.n_pages = g.n_pages, a.page_size = g.page_size, a.table_width = b.table_width;
    a.kv_heads = g.kv_heads, a.heads = heads, a.head_dim = g.head_dim, a.rot = p->rot, a.n_pos = p->n_pos;
    a.interleaved = p->flags & CKKS_CLEAR_INTERLEAVED, a.norm_f32 = p->norm_dtype == CKKS_CLEAR_F32;
    a.eps = p->eps, a.inv_dim = 1.0 / g.head_dim;
    hipStream_t st = (hipStream_t)stream;
    return g.dtype == CKKS_CLEAR_F32   ? launch_packed_append<float>(a, g.format, st)
           : g.dtype == CKKS_CLEAR_F16 ? launch_packed_append<f16>(a, g.format, st)
                                       : launch_packed_append<bf16>(a, g.format, st);
}

int ckks_clear_packed_read(const ckks_clear_packed_read_t *p, void *stream) {
    const char *who = "ckks_clear_packed_read";
    if (!p) {
        set_error("%s: null argument", who);
        return CKKS_E_INVAL;
    }
    const ckks_clear_packed_t &g = p->pages;
    const ckks_clear_batch_t &b = p->batch;
    if (int rc = check_packed(who, g, b)) return rc;
    if (!b.n_tokens || !b.n_seq || (!p->d_k_out && !p->d_v_out)) return CKKS_OK;
    const u32 e = clear_dtype_bytes(g.dtype);
    const PackedPlaces pages = packed_places(g);
    void *outs[2] = {p->d_k_out, p->d_v_out};
    const int64_t *st[2] = {p->k_out_stride, p->v_out_stride};
    Extent out[2];
    Runs rows[2];
    bool bad = false, folded = false;
    for (int o = 0; o < 2; ++o) {
        const u32 n = outs[o] ? b.n_tokens : 0;
        out[o] = extent(outs[o], e, {{n, st[o][0]}, {g.kv_heads, st[o][1]}, {g.head_dim, 1}});
        rows[o] = Runs{outs[o], g.head_dim * e, 2, {{n, st[o][0] * e}, {g.kv_heads, st[o][1] * e}}};
        for (const Extent &x : pages.at) bad |= overlap(out[o], x);
        bad |= overlap(out[o], extent(b.d_q_start, 4, {{b.n_seq + 1, 1}})) || overlap(out[o], extent(b.d_kv_len, 4, {{b.n_seq, 1}})) ||
               overlap(out[o], extent(b.d_page_table, 4, {{b.n_seq, b.table_stride}, {b.table_width, 1}}));
        folded |= n && share_within(rows[o]);
    }
    if (bad || (overlap(out[0], out[1]) && share(rows[0], rows[1]))) {
        set_error("%s: an output overlaps another array", who);
        return CKKS_E_INVAL;
    }
    if (folded) {
        set_error("%s: rows of an output overlap", who);
        return CKKS_E_INVAL;
    }
    PackedReadArgs a{};
    a.pk = g.d_k, a.pv = g.d_v, a.zk = g.d_k_power, a.zv = g.d_v_power, a.ko = p->d_k_out, a.vo = p->d_v_out;
    for (int i = 0; i < 2; ++i) a.kos[i] = p->k_out_stride[i], a.vos[i] = p->v_out_stride[i];
    for (int i = 0; i < 3; ++i)
        a.pks[i] = g.k_stride[i], a.pvs[i] = g.v_stride[i], a.zks[i] = g.k_power_stride[i], a.zvs[i] = g.v_power_stride[i];
    a.ts = b.table_stride, a.q_start = b.d_q_start, a.kv_len = b.d_kv_len, a.table = b.d_page_table;
    a.n_seq = b.n_seq, a.n_tokens = b.n_tokens, a.n_pages = g.n_pages, a.page_size = g.page_size, a.table_width = b.table_width;
    a.kv_heads = g.kv_heads, a.head_dim = g.head_dim;
    hipStream_t s = (hipStream_t)stream;
    return g.dtype == CKKS_CLEAR_F32   ? launch_packed_read<float>(a, g.format, s)
           : g.dtype == CKKS_CLEAR_F16 ? launch_packed_read<f16>(a, g.format, s)
                                       : launch_packed_read<bf16>(a, g.format, s);
}

}  // extern "C"
