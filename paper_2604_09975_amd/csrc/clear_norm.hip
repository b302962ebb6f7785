// Layer norm and its gradient.  A group of threads holds a row in registers, so every array is read once: both calls are
// bound by memory.  The weight's and bias's gradients are column sums: each group keeps them for the columns that it holds
// over all its rows, writes them once, and a second kernel adds the groups' sums in their order.
#include <algorithm>
#include <type_traits>

#include "clear_device.h"

namespace ckks {

struct NormArgs {
    const void *x, *dy, *w, *b;
    void *y;                    // forward: y, gradient: dx
    float *mean, *rstd;
    float *part;                // gradient: [blocks][2][cols] sums of dy*xh and dy, or null
    i64 xs, dys, ys;
    u32 rows, cols;
    float eps;
};

// Sums of two values (of p alone without BOTH) over the TPR threads of a group.  `slot` alternates between two halves of the exchange area, so one
// barrier per call is enough: a wave can be at most one call ahead.
template <int TPR, bool BOTH = true>
__device__ __forceinline__ void group_sum2(float &p, float &q, float (*ex)[2][2], u32 &slot) {
#pragma unroll
    for (int o = TPR < 64 ? TPR / 2 : 32; o; o >>= 1) {
        p += __shfl_xor(p, o);
        if (BOTH) q += __shfl_xor(q, o);
    }
    if (TPR > 64) {
        const u32 wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
            ex[wave][slot][0] = p;
            if (BOTH) ex[wave][slot][1] = q;
        }
        __syncthreads();
        p = 0.0f;
        if (BOTH) q = 0.0f;
#pragma unroll
        for (int i = 0; i < TPR / 64; ++i) {
            p += ex[i][slot][0];
            if (BOTH) q += ex[i][slot][1];
        }
        slot ^= 1;
    }
}

// 1 / sqrt(variance + eps) from the mean square of differences whose own mean is `off`, small beside them or all there is of them.
__device__ __forceinline__ float row_rstd(float square, float off, float eps) {
    const float var = __builtin_fmaf(-off, off, square);
    return 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps);
}

// A thread's E entries of a row: chunks of 16 bytes, TPR chunks apart.  A chunk that would pass the end of the row is moved back
// to end with it, and its first `skip` entries belong to others (all of it: the thread has no such chunk).  So every load is one
// of full width without a branch around it -- a branch would have the result waited for at once -- and what is stored twice is
// stored with the same bits.  Rows have at least one chunk.
template <int V, int K, int TPR>
struct Columns {
    u32 col[K];
    int skip[K];
    bool ragged;  // some thread skips something
    __device__ __forceinline__ Columns(u32 cols, u32 t) {
        ragged = cols != (u32)(V * K * TPR);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const u32 c = (k * TPR + t) * V;
            col[k] = min(c, cols - V);
            skip[k] = (int)min(c - col[k], (u32)V);
        }
    }
};

// TPR threads hold a row, E entries each: a first mean, then the sums of the differences from it and of their squares, then the
// scaled row.  The first mean is off by what its sum and 1/cols were rounded by, a few last places of the row's offset, which
// rstd would multiply; the mean of the differences is that error, and is taken off them: 119 entries of 1e4 have no deviation.
// Bound by memory: 16384 x 8192 bf16 in 93 us, 5.8 TB/s of the 4.9 that a large copy reaches (part of it lies in the last cache);
// 4099 x 1280 f16 7.9 us; 128 x 768 f32 3.7 us, a launch.  Weight and bias stay in registers over a block's rows.
template <class T, class TW, int TPR, int E>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_kernel(NormArgs a) {
    constexpr int V = 16 / sizeof(T), K = E / V, THREADS = TPR < 256 ? 256 : TPR;
    __shared__ float ex[TPR < 64 ? 1 : TPR / 64][2][2];
    u32 slot = 0;
    const u32 t = threadIdx.x % TPR, groups = gridDim.x * (THREADS / TPR);
    const Columns<V, K, TPR> at(a.cols, t);
    u32 row = blockIdx.x * (THREADS / TPR) + threadIdx.x / TPR;
    Pack<T, V> next[K];
    auto fetch = [&](u32 r) {
        const T *x = (const T *)a.x + (i64)min(r, a.rows - 1) * a.xs;
#pragma unroll
        for (int k = 0; k < K; ++k) next[k] = load_pack<V>(x + at.col[k]);
    };
    fetch(row);
    float w[K][V], b[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const Pack<TW, V> pw = a.w ? load_pack<V>((const TW *)a.w + at.col[k]) : Pack<TW, V>{};
        const Pack<TW, V> pb = a.b ? load_pack<V>((const TW *)a.b + at.col[k]) : Pack<TW, V>{};
#pragma unroll
        for (int i = 0; i < V; ++i) {
            w[k][i] = a.w ? (float)pw.v[i] : 1.0f;
            b[k][i] = (float)pb.v[i];
        }
    }
    const float inv = 1.0f / (float)a.cols;
    for (; row < a.rows; row += groups) {
        float v[K][V], s = 0.0f, q = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i] = (float)next[k].v[i];
        fetch(row + groups);  // the next row is under way while this one is worked on
        if (at.ragged) {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) s += i >= at.skip[k] ? v[k][i] : 0.0f;
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) s += v[k][i];
        }
        group_sum2<TPR, false>(s, q, ex, slot);
        const float first = s * inv;
        s = q = 0.0f;
        if (at.ragged) {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    v[k][i] -= first;
                    const float d = i >= at.skip[k] ? v[k][i] : 0.0f;
                    s += d;
                    q = __builtin_fmaf(d, v[k][i], q);
                }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    v[k][i] -= first;
                    s += v[k][i];
                    q = __builtin_fmaf(v[k][i], v[k][i], q);
                }
        }
        group_sum2<TPR>(s, q, ex, slot);
        const float off = s * inv, r = row_rstd(q * inv, off, a.eps), shift = -off * r;
        if (t == 0 && a.mean) {
            a.mean[row] = first + off;
            a.rstd[row] = r;
        }
        T *y = (T *)a.y + (i64)row * a.ys;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            Pack<T, V> p;
#pragma unroll
            for (int i = 0; i < V; ++i) p.v[i] = (T)__builtin_fmaf(__builtin_fmaf(v[k][i], r, shift), w[k][i], b[k][i]);
            if (at.skip[k] < V) store_pack<V>(y + at.col[k], p);
        }
    }
}

// As norm_kernel with rows of x and dy.  The weight lies in LDS: registers hold the sums of the columns and the row that comes
// next.  Bound by memory: 16384 x 8192 bf16 183 us, 4.6 TB/s with the sums that it writes (256 us with loads behind branches and
// no row ahead); 4099 x 1280 f16 14.0 us, by the latency of four to five rows one after the other in each group, one wave on a SIMD.
// f32 rows of 8193 to 16384 leave 31 registers of a thread in scratch: 4096 x 12000 173 us with the second kernel, 120 at a copy's rate.
template <class T, class TW, int TPR, int E>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_grad_kernel(NormArgs a) {
    constexpr int V = 16 / sizeof(T), K = E / V, THREADS = TPR < 256 ? 256 : TPR, GROUPS = THREADS / TPR;
    __shared__ float ex[TPR < 64 ? 1 : TPR / 64][2][2];
    __shared__ __attribute__((aligned(16))) float weight[K][TPR][V];
    u32 slot = 0;
    const u32 t = threadIdx.x % TPR, groups = gridDim.x * GROUPS;
    const Columns<V, K, TPR> at(a.cols, t);
    u32 row = blockIdx.x * GROUPS + threadIdx.x / TPR;
    Pack<T, V> next_x[K], next_d[K];
    float next_mean, next_r;
    auto fetch = [&](u32 r) {
        r = min(r, a.rows - 1);
        const T *x = (const T *)a.x + (i64)r * a.xs, *dy = (const T *)a.dy + (i64)r * a.dys;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            next_x[k] = load_pack<V>(x + at.col[k]);
            next_d[k] = load_pack<V>(dy + at.col[k]);
        }
        next_mean = a.mean[r];
        next_r = a.rstd[r];
    };
    fetch(row);
    float dw[K][V], db[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const Pack<TW, V> pw = a.w ? load_pack<V>((const TW *)a.w + at.col[k]) : Pack<TW, V>{};
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (threadIdx.x < TPR) weight[k][t][i] = a.w ? (float)pw.v[i] : 1.0f;
            dw[k][i] = db[k][i] = 0.0f;
        }
    }
    __syncthreads();
    const float inv = 1.0f / (float)a.cols;
    for (; row < a.rows; row += groups) {
        Pack<T, V> px[K], pd[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            px[k] = next_x[k];
            pd[k] = next_d[k];
        }
        const float mean = next_mean, r = next_r;
        fetch(row + groups);
        float s1 = 0.0f, s2 = 0.0f;
        auto sums = [&](auto ragged) {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float d = !ragged.value || i >= at.skip[k] ? (float)pd[k].v[i] : 0.0f, h = ((float)px[k].v[i] - mean) * r;
                    const float g = d * weight[k][t][i];
                    dw[k][i] = __builtin_fmaf(d, h, dw[k][i]);
                    db[k][i] += d;
                    s1 += g;
                    s2 = __builtin_fmaf(g, h, s2);
                }
        };
        if (at.ragged)
            sums(std::true_type());
        else
            sums(std::false_type());
        if (!a.y) continue;
        group_sum2<TPR>(s1, s2, ex, slot);
        s1 *= inv;
        s2 *= inv;
        T *dx = (T *)a.y + (i64)row * a.ys;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            Pack<T, V> p;
#pragma unroll
            for (int i = 0; i < V; ++i)
                p.v[i] = (T)(r * ((float)pd[k].v[i] * weight[k][t][i] - s1 - ((float)px[k].v[i] - mean) * r * s2));
            if (at.skip[k] < V) store_pack<V>(dx + at.col[k], p);
        }
    }
    if (!a.part) return;
    float *part = a.part + (size_t)blockIdx.x * 2 * a.cols;
    if (GROUPS == 1) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i >= at.skip[k]) {
                    part[at.col[k] + i] = dw[k][i];
                    part[a.cols + at.col[k] + i] = db[k][i];
                }
        return;
    }
    // the block's groups hold the same columns: joined here, a quarter as many sums reach memory
    __shared__ float join[GROUPS][2][TPR * V];
    const u32 gr = threadIdx.x / TPR;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) {
            join[gr][0][t * V + i] = dw[k][i];
            join[gr][1][t * V + i] = db[k][i];
        }
        __syncthreads();
        for (u32 c = threadIdx.x; c < 2 * TPR * V; c += THREADS) {
            const u32 which = c / (TPR * V), j = c % (TPR * V), begin = (k * TPR + j / V) * V, col = min(begin, a.cols - V) + j % V;
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < GROUPS; ++i) s += join[i][which][j];
            if (col >= begin) part[which * (size_t)a.cols + col] = s;
        }
    }
}

// Rows wider than the registers of a block, or shorter than an access: the same sums in loops over the row, which comes from the
// caches again, an entry at a time: 4096 x 16400 bf16 164 us, gradient 267, where 4096 x 16384 in registers takes 54 and 102; 65000 x 5
// 390 and 490.
template <class T, class TW>
__global__ __launch_bounds__(1024) void norm_wide_kernel(NormArgs a) {
    __shared__ float ex[16][2][2];
    u32 slot = 0;
    const float inv = 1.0f / (float)a.cols;
    for (u32 row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = (const T *)a.x + (i64)row * a.xs;
        T *y = (T *)a.y + (i64)row * a.ys;
        float s = 0.0f, q = 0.0f;
        for (u64 c = threadIdx.x; c < a.cols; c += 1024) s += (float)x[c];
        group_sum2<1024, false>(s, q, ex, slot);
        const float first = s * inv;
        s = q = 0.0f;
        for (u64 c = threadIdx.x; c < a.cols; c += 1024) {
            const float d = (float)x[c] - first;
            s += d;
            q = __builtin_fmaf(d, d, q);
        }
        group_sum2<1024>(s, q, ex, slot);
        const float off = s * inv, r = row_rstd(q * inv, off, a.eps);
        if (threadIdx.x == 0 && a.mean) {
            a.mean[row] = first + off;
            a.rstd[row] = r;
        }
        for (u64 c = threadIdx.x; c < a.cols; c += 1024) {
            const float w = a.w ? (float)((const TW *)a.w)[c] : 1.0f, b = a.b ? (float)((const TW *)a.b)[c] : 0.0f;
            y[c] = (T)__builtin_fmaf(((float)x[c] - first - off) * r, w, b);
        }
    }
}

// Column sums first (dx may take the place of dy), then dx.
template <class T>
__global__ __launch_bounds__(256) void norm_grad_wide_cols_kernel(NormArgs a, u32 parts) {
    const u64 c = (u64)blockIdx.x * 256 + threadIdx.x;
    if (c >= a.cols) return;
    float dw = 0.0f, db = 0.0f;
    for (u32 row = blockIdx.y; row < a.rows; row += parts) {
        const float d = (float)((const T *)a.dy)[(i64)row * a.dys + c];
        dw = __builtin_fmaf(d, ((float)((const T *)a.x)[(i64)row * a.xs + c] - a.mean[row]) * a.rstd[row], dw);
        db += d;
    }
    float *part = a.part + (size_t)blockIdx.y * 2 * a.cols;
    part[c] = dw;
    part[a.cols + c] = db;
}
template <class T, class TW>
__global__ __launch_bounds__(1024) void norm_grad_wide_kernel(NormArgs a) {
    __shared__ float ex[16][2][2];
    u32 slot = 0;
    const float inv = 1.0f / (float)a.cols;
    for (u32 row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = (const T *)a.x + (i64)row * a.xs, *dy = (const T *)a.dy + (i64)row * a.dys;
        T *dx = (T *)a.y + (i64)row * a.ys;
        const float mean = a.mean[row], r = a.rstd[row];
        float s1 = 0.0f, s2 = 0.0f;
        for (u64 c = threadIdx.x; c < a.cols; c += 1024) {
            const float g = (float)dy[c] * (a.w ? (float)((const TW *)a.w)[c] : 1.0f);
            s1 += g;
            s2 = __builtin_fmaf(g, ((float)x[c] - mean) * r, s2);
        }
        group_sum2<1024>(s1, s2, ex, slot);
        s1 *= inv;
        s2 *= inv;
        for (u64 c = threadIdx.x; c < a.cols; c += 1024) {
            const float g = (float)dy[c] * (a.w ? (float)((const TW *)a.w)[c] : 1.0f);
            dx[c] = (T)(r * (g - s1 - ((float)x[c] - mean) * r * s2));
        }
    }
}

// dw[c], db[c] = the sums of all parts, always in the same order.  64 columns per block, so that whole lines are read, and 16 threads
// to share a column's parts: 512 parts of 8192 columns 6.7 us, bound by memory; 256 of 1280 3.8, by the loads' latency.
template <class TW>
__global__ __launch_bounds__(1024) void norm_parts_kernel(const float *__restrict__ part, u32 parts, u32 cols, TW *dw, TW *db) {
    __shared__ float join[16][64];
    const u32 c = threadIdx.x % 64, q = threadIdx.x / 64;
    const u64 col = (u64)blockIdx.x * 64 + c;
    TW *out = blockIdx.y ? db : dw;
    if (!out) return;
    float s = 0.0f;
    if (col < cols)
#pragma unroll 8
        for (u32 p = q; p < parts; p += 16) s += part[((size_t)p * 2 + blockIdx.y) * cols + col];
    join[q][c] = s;
    __syncthreads();
    if (q == 0 && col < cols) {
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += join[i][c];
        out[col] = (TW)s;
    }
}
template <class TW>
static void launch_parts(const float *part, u32 parts, u32 cols, void *dw, void *db, hipStream_t st) {
    hipLaunchKernelGGL((norm_parts_kernel<TW>), dim3((u32)(((u64)cols + 63) / 64), 2), dim3(1024), 0, st, part, parts, cols, (TW *)dw, (TW *)db);
}

// Threads per row and entries per thread: the smallest group whose registers hold the row at up to 32 entries a thread
// (16 where 1024 threads share the register file).  0: none does, or the row is shorter than an access.  A larger group waits for
// more exchanges and has fewer bytes under way.  us forward (calls back to back in a graph), gradient (bf16):
//   16384 x 2048: 64 threads 27.0, 45.9; 256 threads 33.6, 60.2      8192 x 8192: 256 threads 51.8, 99.8; 1024 threads 91.6, 115
//   32768 x 1536: 64 threads 40.2, 61.8; 256 threads 58.8, 88.8      64 x 2048: 3.4, 9.8 and 3.1, 7.9: not worth a second rule
// Rows of up to 256 leave most of a wave idle: 65000 x 64 bf16 16 threads 7.1, 14.5 (64: 20.7, 29.8), 56383 x 203 32 threads 11.8, 22.7
// (64: 19.7, 33.0).  24 entries where they do rather than 32: 16384 x 1280 15.3, 31.6 (32: 17.1, 34.7), 4000 x 4800 f32 33.2, 51.0 (36.0, 60.2).
struct NormShape {
    u32 tpr, e;
};
static NormShape norm_shape(u32 cols) {
    if (cols < 8) return {0, 0};
    if (cols <= 16 * 8) return {16, 8};
    if (cols <= 32 * 8) return {32, 8};
    if (cols <= 64 * 32) return {64, cols <= 64 * 8 ? 8u : cols <= 64 * 16 ? 16u : cols <= 64 * 24 ? 24u : 32u};
    if (cols <= 256 * 32) return {256, cols <= 256 * 16 ? 16u : cols <= 256 * 24 ? 24u : 32u};
    if (cols <= 1024 * 16) return {1024, 16};
    return {0, 0};
}
// Blocks: as many as the registers let run at once on 256 CUs, each with every so-manieth row.  Each block of the gradient leaves
// one pair of column sums, so it has fewer: two or three a CU (16384 x 4000 bf16 88.6 us, with four 98.5; 60000 x 300 33.1, with six
// 36.9), and beyond one a CU its groups have four rows at least (1000 x 5000 bf16 23.7 us, with a row each 29.4; 4099 x 1280 f16 17.6,
// 18.5; 2000 x 768 f32 11.4, 13.8).
static u32 norm_blocks(u32 rows, const NormShape &s, bool grad) {
    const u32 per = s.tpr <= 64 ? 256 / s.tpr : 1, most = (rows + per - 1) / per;
    if (!grad) return std::min<u32>(most, 256 * (s.tpr == 1024 ? 1 : s.e == 32 ? 3 : s.e == 24 ? 4 : 6));
    const u32 cu = s.tpr == 1024 ? 1 : s.e >= 16 ? 2 : 3;
    return std::min(most, std::max<u32>(256, std::min(256 * cu, rows / (4 * per))));
}
static u32 norm_grad_blocks(u32 rows, u32 cols) {
    const NormShape s = norm_shape(cols);
    return s.tpr ? norm_blocks(rows, s, true) : std::min<u32>(rows, 64);
}

template <class T, class TW>
static void launch_norm(const NormArgs &a, hipStream_t st) {
    const NormShape s = norm_shape(a.cols);
    const u32 blocks = s.tpr ? norm_blocks(a.rows, s, false) : 0;
#define CKKS_NORM(TPR, E) \
    if (s.tpr == TPR && s.e == E) {                                                                                      \
        hipLaunchKernelGGL((norm_kernel<T, TW, TPR, E>), dim3(blocks), dim3(TPR < 256 ? 256 : TPR), 0, st, a);         \
        return;                                                                                                           \
    }
    CKKS_NORM(16, 8)
    CKKS_NORM(32, 8)
    CKKS_NORM(64, 8)
    CKKS_NORM(64, 16)
    CKKS_NORM(64, 24)
    CKKS_NORM(64, 32)
    CKKS_NORM(256, 16)
    CKKS_NORM(256, 24)
    CKKS_NORM(256, 32)
    CKKS_NORM(1024, 16)
#undef CKKS_NORM
    hipLaunchKernelGGL((norm_wide_kernel<T, TW>), dim3(std::min<u32>(a.rows, 1024)), dim3(1024), 0, st, a);
}

template <class T, class TW>
static void launch_norm_grad(const NormArgs &a, u32 blocks, hipStream_t st) {
    const NormShape s = norm_shape(a.cols);
#define CKKS_NORM(TPR, E) \
    if (s.tpr == TPR && s.e == E) {                                                                                      \
        hipLaunchKernelGGL((norm_grad_kernel<T, TW, TPR, E>), dim3(blocks), dim3(TPR < 256 ? 256 : TPR), 0, st, a);    \
        return;                                                                                                           \
    }
    CKKS_NORM(16, 8)
    CKKS_NORM(32, 8)
    CKKS_NORM(64, 8)
    CKKS_NORM(64, 16)
    CKKS_NORM(64, 24)
    CKKS_NORM(64, 32)
    CKKS_NORM(256, 16)
    CKKS_NORM(256, 24)
    CKKS_NORM(256, 32)
    CKKS_NORM(1024, 16)
#undef CKKS_NORM
    if (a.part)
        hipLaunchKernelGGL((norm_grad_wide_cols_kernel<T>), dim3((u32)(((u64)a.cols + 255) / 256), blocks), dim3(256), 0, st, a, blocks);
    if (a.y)
        hipLaunchKernelGGL((norm_grad_wide_kernel<T, TW>), dim3(std::min<u32>(a.rows, 1024)), dim3(1024), 0, st, a);
}

}  // namespace ckks

using namespace ckks;

// (T, TW) of a pair of types that the calls take
#define CKKS_NORM_TYPES(F, ...)                                                     \
    (dtype == CKKS_CLEAR_F32   ? F<float, float>(__VA_ARGS__)                       \
     : dtype == CKKS_CLEAR_F16 ? (wtype == CKKS_CLEAR_F32 ? F<f16, float>(__VA_ARGS__) : F<f16, f16>(__VA_ARGS__)) \
                               : (wtype == CKKS_CLEAR_F32 ? F<bf16, float>(__VA_ARGS__) : F<bf16, bf16>(__VA_ARGS__)))

static int check_norm(const char *who, u32 rows, u32 cols, u32 dtype, u32 wtype) {
    if (!clear_dtype_ok(dtype) || (wtype != CKKS_CLEAR_F32 && wtype != dtype)) {
        set_error("%s: types %u and %u (weight): the weight has the rows' type or f32", who, dtype, wtype);
        return CKKS_E_INVAL;
    }
    if (!cols || rows >= 1u << 31 || cols >= 1u << 31) {
        set_error("%s: %u rows of %u entries", who, rows, cols);
        return CKKS_E_INVAL;
    }
    return CKKS_OK;
}

extern "C" {

int ckks_clear_layer_norm(const ckks_clear_norm_t *p, void *stream) {
    if (!p || (p->rows && (!p->d_x || !p->d_y))) {
        set_error("ckks_clear_layer_norm: null argument");
        return CKKS_E_INVAL;
    }
    if (int rc = check_norm("ckks_clear_layer_norm", p->rows, p->cols, p->dtype, p->weight_dtype)) return rc;
    if (!(p->eps >= 0.0f) || !p->d_mean != !p->d_rstd) {
        set_error("ckks_clear_layer_norm: eps %g, or only one of d_mean and d_rstd", (double)p->eps);
        return CKKS_E_INVAL;
    }
    if (!p->rows) return CKKS_OK;
    const u32 dtype = p->dtype, wtype = p->weight_dtype, e = clear_dtype_bytes(dtype), we = clear_dtype_bytes(wtype);
    const Extent x = extent(p->d_x, e, {{p->rows, p->x_stride}, {p->cols, 1}}), y = extent(p->d_y, e, {{p->rows, p->y_stride}, {p->cols, 1}});
    const Extent w = extent(p->d_weight, we, {{p->d_weight ? p->cols : 0, 1}}), b = extent(p->d_bias, we, {{p->d_bias ? p->cols : 0, 1}});
    const Extent m = extent(p->d_mean, 4, {{p->d_mean ? p->rows : 0, 1}}), r = extent(p->d_rstd, 4, {{p->d_rstd ? p->rows : 0, 1}});
    const bool in_place = p->d_x == p->d_y && (p->x_stride == p->y_stride || p->rows == 1);
    if ((!in_place && overlap(x, y)) || overlap(y, w) || overlap(y, b) || overlap(y, m) || overlap(y, r) || overlap(m, x) ||
        overlap(r, x) || overlap(m, r) || overlap(m, w) || overlap(m, b) || overlap(r, w) || overlap(r, b)) {
        set_error("ckks_clear_layer_norm: an output overlaps another array");
        return CKKS_E_INVAL;
    }
    if (p->rows > 1 && (p->y_stride < 0 ? -p->y_stride : p->y_stride) < (i64)p->cols) {
        set_error("ckks_clear_layer_norm: output rows overlap (stride %lld)", (long long)p->y_stride);
        return CKKS_E_INVAL;
    }
    NormArgs a{};
    a.x = p->d_x, a.w = p->d_weight, a.b = p->d_bias, a.y = p->d_y, a.mean = p->d_mean, a.rstd = p->d_rstd;
    a.xs = p->x_stride, a.ys = p->y_stride, a.rows = p->rows, a.cols = p->cols, a.eps = p->eps;
    CKKS_NORM_TYPES(launch_norm, a, (hipStream_t)stream);
    CKKS_LAUNCH_CHECK("norm_kernel");
    return CKKS_OK;
}

uint64_t ckks_clear_layer_norm_grad_work_bytes(uint32_t rows, uint32_t cols, uint32_t) {
    return (u64)norm_grad_blocks(rows, cols) * 2 * cols * sizeof(float);
}

int ckks_clear_layer_norm_grad(const ckks_clear_norm_grad_t *p, void *stream) {
    if (!p || (p->rows && (!p->d_x || !p->d_dy || !p->d_mean || !p->d_rstd))) {
        set_error("ckks_clear_layer_norm_grad: null argument");
        return CKKS_E_INVAL;
    }
    if (int rc = check_norm("ckks_clear_layer_norm_grad", p->rows, p->cols, p->dtype, p->weight_dtype)) return rc;
    const u32 dtype = p->dtype, wtype = p->weight_dtype, e = clear_dtype_bytes(dtype), we = clear_dtype_bytes(wtype);
    const bool params = p->d_dweight || p->d_dbias;
    if (params && p->cols >= 1u << 28) {  // 16 threads to a column where row sums are joined, and fewer than 2^32 in a launch
        set_error("ckks_clear_layer_norm_grad: gradients of %u weights exceed one launch", p->cols);
        return CKKS_E_INVAL;
    }
    const u64 need = params ? ckks_clear_layer_norm_grad_work_bytes(p->rows, p->cols, dtype) : 0;
    if (need > p->work_bytes || (need && (!p->d_work || (uintptr_t)p->d_work % 4))) {
        set_error("ckks_clear_layer_norm_grad: workspace of %llu bytes, needs %llu (4-byte aligned)", (unsigned long long)p->work_bytes,
                  (unsigned long long)need);
        return CKKS_E_INVAL;
    }
    const Extent in[5] = {extent(p->d_x, e, {{p->rows, p->x_stride}, {p->cols, 1}}), extent(p->d_weight, we, {{p->d_weight ? p->cols : 0, 1}}),
                          extent(p->d_mean, 4, {{p->rows, 1}}), extent(p->d_rstd, 4, {{p->rows, 1}}),
                          extent(p->d_dy, e, {{p->rows, p->dy_stride}, {p->cols, 1}})};
    const Extent out[4] = {extent(p->d_dx, e, {{p->d_dx ? p->rows : 0, p->dx_stride}, {p->cols, 1}}),
                           extent(p->d_dweight, we, {{p->d_dweight ? p->cols : 0, 1}}), extent(p->d_dbias, we, {{p->d_dbias ? p->cols : 0, 1}}),
                           extent(p->d_work, 1, {{need, 1}})};
    const bool in_place = p->d_dx == p->d_dy && (p->dx_stride == p->dy_stride || p->rows == 1);
    bool bad = false;
    for (int o = 0; o < 4; ++o) {
        for (int i = 0; i < 5; ++i) bad |= !(o == 0 && i == 4 && in_place) && overlap(out[o], in[i]);
        for (int i = 0; i < o; ++i) bad |= overlap(out[o], out[i]);
    }
    if (bad) {
        set_error("ckks_clear_layer_norm_grad: an output overlaps another array");
        return CKKS_E_INVAL;
    }
    if (p->d_dx && p->rows > 1 && (p->dx_stride < 0 ? -p->dx_stride : p->dx_stride) < (i64)p->cols) {
        set_error("ckks_clear_layer_norm_grad: output rows overlap (stride %lld)", (long long)p->dx_stride);
        return CKKS_E_INVAL;
    }
    NormArgs a{};
    a.x = p->d_x, a.dy = p->d_dy, a.w = p->d_weight, a.y = p->d_dx;
    a.mean = (float *)p->d_mean, a.rstd = (float *)p->d_rstd, a.part = params ? (float *)p->d_work : nullptr;
    a.xs = p->x_stride, a.dys = p->dy_stride, a.ys = p->dx_stride, a.rows = p->rows, a.cols = p->cols;
    const u32 blocks = norm_grad_blocks(p->rows, p->cols);
    hipStream_t st = (hipStream_t)stream;
    if (p->rows && (a.y || params)) {
        CKKS_NORM_TYPES(launch_norm_grad, a, blocks, st);
        CKKS_LAUNCH_CHECK("norm_grad_kernel");
    }
    if (params) {
        if (wtype == CKKS_CLEAR_F32)
            launch_parts<float>(a.part, blocks, p->cols, p->d_dweight, p->d_dbias, st);
        else if (wtype == CKKS_CLEAR_F16)
            launch_parts<f16>(a.part, blocks, p->cols, p->d_dweight, p->d_dbias, st);
        else
            launch_parts<bf16>(a.part, blocks, p->cols, p->d_dweight, p->d_dbias, st);
        CKKS_LAUNCH_CHECK("norm_parts_kernel");
    }
    return CKKS_OK;
}

}  // extern "C"
