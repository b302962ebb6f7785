// Cache pages of 8 bits (ckks_clear_packed_t): codes to values and back, and the checks of such pages.
#pragma once
#include <type_traits>

#include "clear_device.h"

namespace ckks {

constexpr int PLAIN = 0, E4M3 = CKKS_CLEAR_E4M3, I8 = CKKS_CLEAR_I8;  // forms of a page
constexpr u32 PACK_BLOCK = 32;                                        // entries that share a power of two

// 2^(z - 127), NaN for 255, as the conversions below take it: those of the hardware, exact for every code and power, read the exponent
// field of a float, 255 of which is their NaN; to multiply by, 0 is the denormal 2^-127.
template <int FORM>
__device__ __forceinline__ float power_of(u32 z) {
    if (FORM == E4M3) return __uint_as_float(z << 23);
    return __uint_as_float(z == 0 ? 0x00400000u : z == 255 ? 0x7fc00000u : z << 23);
}

// The value of one code.
template <int FORM>
__device__ __forceinline__ float unpack(u32 code, u32 z) {
    if constexpr (FORM == E4M3)
        return __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(code, power_of<FORM>(z), false)[0];
    else
        return (float)(signed char)code * power_of<FORM>(z);
}

// Four codes of one block as T.
template <class T, int FORM>
__device__ __forceinline__ void unpack4(u32 codes, float power, T *out) {
    if constexpr (FORM == E4M3) {
        if constexpr (std::is_same<T, bf16>::value) {
            const auto lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, power, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, power, true);
            out[0] = lo[0], out[1] = lo[1], out[2] = hi[0], out[3] = hi[1];
        } else if constexpr (std::is_same<T, f16>::value) {
            const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, power, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, power, true);
            out[0] = lo[0], out[1] = lo[1], out[2] = hi[0], out[3] = hi[1];
        } else {
            const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, power, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, power, true);
            out[0] = lo[0], out[1] = lo[1], out[2] = hi[0], out[3] = hi[1];
        }
    } else {
        // (as a vector: number by number the compiler converts each alone and joins pairs by shifts; prompts of I8 1776 -> 1655 us)
        typedef float f32s __attribute__((ext_vector_type(4)));
        typedef T cells __attribute__((ext_vector_type(4)));
        f32s x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (float)(signed char)(codes >> 8 * i);
        const cells y = __builtin_convertvector(x * power, cells);
        __builtin_memcpy(out, &y, sizeof(y));
    }
}
// 16 bytes of T out of a piece of their codes.
template <class T, int FORM, class P>
__device__ __forceinline__ uint4 unpack_piece(const P &x, u32 z) {
    T v[16 / sizeof(T)];
    const float power = power_of<FORM>(z);
    if constexpr (sizeof(P) == 8) {
        unpack4<T, FORM>(x.x, power, v);
        unpack4<T, FORM>(x.y, power, v + 4);
    } else {
        unpack4<T, FORM>(x, power, v);
    }
    uint4 r;
    __builtin_memcpy(&r, v, 16);
    return r;
}

// ---- host ----
inline u32 packed_blocks(u32 head_dim) { return (head_dim + PACK_BLOCK - 1) / PACK_BLOCK; }
// The pages as check_cache takes them, with codes or with powers for their entries.
inline ckks_clear_pages_t as_pages(const ckks_clear_packed_t &g, bool power) {
    ckks_clear_pages_t p{};
    p.d_k = power ? g.d_k_power : g.d_k, p.d_v = power ? g.d_v_power : g.d_v;
    for (int i = 0; i < 3; ++i) {
        p.k_stride[i] = power ? g.k_power_stride[i] : g.k_stride[i];
        p.v_stride[i] = power ? g.v_power_stride[i] : g.v_stride[i];
    }
    p.n_pages = g.n_pages, p.page_size = g.page_size, p.kv_heads = g.kv_heads, p.head_dim = g.head_dim, p.dtype = g.dtype;
    return p;
}
inline int check_packed(const char *who, const ckks_clear_packed_t &g, const ckks_clear_batch_t &b) {
    if (g.format != CKKS_CLEAR_E4M3 && g.format != CKKS_CLEAR_I8) {
        set_error("%s: pages of format %u", who, g.format);
        return CKKS_E_INVAL;
    }
    if (int rc = check_cache(who, as_pages(g, false), b)) return rc;
    return check_cache(who, as_pages(g, true), b);
}
// Where codes and powers of keys and values lie: extents and runs, keys, values, powers of keys, powers of values.
struct PackedPlaces {
    Extent at[4];
    Runs cells[4];
};
inline PackedPlaces packed_places(const ckks_clear_packed_t &g) {
    const void *p[4] = {g.d_k, g.d_v, g.d_k_power, g.d_v_power};
    const int64_t *st[4] = {g.k_stride, g.v_stride, g.k_power_stride, g.v_power_stride};
    PackedPlaces r;
    for (int i = 0; i < 4; ++i) {
        const u32 run = i < 2 ? g.head_dim : packed_blocks(g.head_dim);
        r.at[i] = extent(p[i], 1, {{g.n_pages, st[i][0]}, {g.kv_heads, st[i][1]}, {g.page_size, st[i][2]}, {run, 1}});
        r.cells[i] = Runs{p[i], run, 3, {{g.n_pages, st[i][0]}, {g.kv_heads, st[i][1]}, {g.page_size, st[i][2]}}};
    }
    return r;
}

}  // namespace ckks
