// Layer norm over rows (see include/nb_norm.h for the arithmetic).  A row is held in the registers of a group of threads: 4 to 32
// lanes of a warp (short rows, several to a warp) or a whole block (long rows); statistics take two passes over the registers.
// Rows too long for that, of any alignment, are read again from the caches (the *_loop kernels).
#pragma once
#include "common.cuh"

namespace nbcbs {

constexpr int LN_THREADS = 256;   // of a block whose groups are lanes of a warp
constexpr int LN_MAX_BLOCK = 1024;
constexpr int LN_BWD_MAX_BLOCK = 512;

// V consecutive elements: a 16-byte vector, or a single element where rows are not whole vectors.
template <typename T, int V> struct LnVec {
    T v[V];
};
template <typename T, int V> __device__ __forceinline__ LnVec<T, V> ln_ld(const T* p) {
    LnVec<T, V> r;
    if constexpr (V == 1) {
        r.v[0] = *p;
    } else {
        static_assert(V * sizeof(T) == 16, "16-byte vectors");
        *reinterpret_cast<uint4*>(&r) = *reinterpret_cast<const uint4*>(p);
    }
    return r;
}
template <typename T, int V> __device__ __forceinline__ void ln_st(T* p, const LnVec<T, V>& r) {
    if constexpr (V == 1) *p = r.v[0]; else *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(&r);
}
// The same as packed fp32 pairs (fma / mul / add .f32x2, see common.cuh); a single element is a pair whose second half is zero.
template <typename T, int V> struct LnPairs {
    static constexpr int N = (V + 1) / 2;
    float2 p[N];
    __device__ __forceinline__ LnPairs() {}
    __device__ __forceinline__ explicit LnPairs(const LnVec<T, V>& v) {
        if constexpr (V == 1) {
            p[0] = make_float2(to_f32<T>(v.v[0]), 0.f);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) p[j] = pair_to_f32<T>(v.v + 2 * j);
        }
    }
    __device__ __forceinline__ LnVec<T, V> rounded() const {
        LnVec<T, V> o;
        if constexpr (V == 1) {
            o.v[0] = from_f32<T>(p[0].x);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) pair_from_f32<T>(o.v + 2 * j, p[j]);
        }
        return o;
    }
};
template <int V> __device__ __forceinline__ void ln_ldf(const float* p, float2 (&o)[(V + 1) / 2], float without) {
    if (!p) {
#pragma unroll
        for (int j = 0; j < (V + 1) / 2; ++j) o[j] = make_float2(without, without);
    } else if constexpr (V == 1) {
        o[0] = make_float2(__ldg(p), 0.f);
    } else {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            const float4 f = __ldg(reinterpret_cast<const float4*>(p + j));
            o[j / 2] = make_float2(f.x, f.y);
            o[j / 2 + 1] = make_float2(f.z, f.w);
        }
    }
}

// Sums over a group of L lanes (L <= 32), or over the block (L = 0; `red` holds two floats a warp, and consecutive calls alternate
// between two such arrays so that one barrier a call is enough).
template <int L> __device__ __forceinline__ float2 ln_sum2(float2 s, float2* red) {
    constexpr int W = L == 0 ? 32 : L;
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) {
        s.x += __shfl_xor_sync(0xffffffffu, s.x, o);
        s.y += __shfl_xor_sync(0xffffffffu, s.y, o);
    }
    if constexpr (L == 0) {
        const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0) red[threadIdx.x >> 5] = s;
        __syncthreads();
        s = lane < warps ? red[lane] : make_float2(0.f, 0.f);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            s.x += __shfl_xor_sync(0xffffffffu, s.x, o);
            s.y += __shfl_xor_sync(0xffffffffu, s.y, o);
        }
    }
    return s;
}
template <int L> __device__ __forceinline__ float ln_sum(float s, float2* red) { return ln_sum2<L>(make_float2(s, 0.f), red).x; }
// s / c by the rounded reciprocal of c and one correction of the quotient: exact where the quotient is a number of fp32, so that a constant row's
// mean is its constant (half a unit off, x - mean would be an error of 1000 * 2^-24 / sqrt(eps) in a row of 1000s).
__device__ __forceinline__ float ln_mean(float s, float c, float inv_c) {
    const float q = s * inv_c;
    return fabsf(q) < __int_as_float(0x7f800000) ? fmaf(fmaf(-q, c, s), inv_c, q) : q;
}

struct LnFwd {
    const void* x;
    void* y;
    const float *gamma, *beta;
    float *mean, *rstd;
    long long rows, ld_x, ld_y;
    int c, nvec;  // channels, vectors of a row
    float eps;
};

// Bound: memory (x once, y once).  gamma and beta are read behind the statistics, from L1.
template <typename T, int V, int L, int VPL> __global__ void __launch_bounds__(L == 0 ? LN_MAX_BLOCK : LN_THREADS) layer_norm_fwd_kernel(LnFwd P) {
    pdl_launch_dependents();
    pdl_wait();
    __shared__ float2 red[2][32];
    const int W = L == 0 ? (int)blockDim.x : L;                        // threads of a group
    const int lane = L == 0 ? (int)threadIdx.x : (int)threadIdx.x % L;  // this thread's place in it
    const int groups = L == 0 ? 1 : LN_THREADS / L, group = L == 0 ? 0 : (int)threadIdx.x / L;
    const float inv_c = 1.f / (float)P.c;
    for (long long r0 = (long long)blockIdx.x * groups; r0 < P.rows; r0 += (long long)gridDim.x * groups) {
        const long long row = r0 + group;
        const bool live = row < P.rows;
        const T* x = static_cast<const T*>(P.x) + (live ? row : 0) * P.ld_x;
        constexpr int N = (V + 1) / 2;
        LnPairs<T, V> f[VPL];
        LnVec<T, V> raw[VPL];
#pragma unroll
        for (int k = 0; k < VPL; ++k) {
            const int i = lane + k * W;
            if (live && i < P.nvec) {
                raw[k] = ln_ld<T, V>(x + (long long)i * V);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) raw[k].v[j] = from_f32<T>(0.f);
            }
        }
        float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < VPL; ++k) {
            f[k] = LnPairs<T, V>(raw[k]);
#pragma unroll
            for (int j = 0; j < N; ++j) s2 = add2(s2, f[k].p[j]);
        }
        const float mean = ln_mean(ln_sum<L>(s2.x + s2.y, red[0]), (float)P.c, inv_c);
        s2 = make_float2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < VPL; ++k)
            if (lane + k * W < P.nvec)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    f[k].p[j] = add2(f[k].p[j], make_float2(-mean, V == 1 ? 0.f : -mean));
                    s2 = fma2(f[k].p[j], f[k].p[j], s2);
                }
        const float rstd = 1.f / sqrtf(ln_sum<L>(s2.x + s2.y, red[1]) * inv_c + P.eps);
        if (!live) continue;
        T* y = static_cast<T*>(P.y) + row * P.ld_y;
#pragma unroll
        for (int k = 0; k < VPL; ++k) {
            const int i = lane + k * W;
            if (i < P.nvec) {
                float2 ga[N], be[N];
                ln_ldf<V>(P.gamma ? P.gamma + i * V : nullptr, ga, 1.f);
                ln_ldf<V>(P.beta ? P.beta + i * V : nullptr, be, 0.f);
#pragma unroll
                for (int j = 0; j < N; ++j) f[k].p[j] = fma2(mul2(f[k].p[j], splat2(rstd)), ga[j], be[j]);
                ln_st<T, V>(y + (long long)i * V, f[k].rounded());
            }
        }
        if (P.mean && lane == 0) {
            P.mean[row] = mean;
            P.rstd[row] = rstd;
        }
    }
}

// Dense rows of a channel count that no vector divides: eight of 16-bit elements (four of fp32) are whole 16-byte vectors together,
// so a block takes that many at a time through shared memory, with vectors from and to global memory.  Warps have the rows for
// the statistics, threads the columns for the rest.  5003 x 1001 fp16, forward and backward with the sums: 72 us element by element,
// 39 in this form.
constexpr int LN_TILE_THREADS = 256;
constexpr int LN_TILE_COLS = 8;  // columns of the sums that a thread of the backward pass may own
template <typename T> __host__ __device__ constexpr int ln_tile_rows() { return 16 / (int)sizeof(T); }
// n elements (whole vectors), of which `left` exist in memory; the others become zeros
template <typename T> __device__ __forceinline__ void ln_tile_in(T* dst, const T* src, long long left, int n) {
    constexpr int V = 16 / (int)sizeof(T);
    for (int i = threadIdx.x; i < n / V; i += LN_TILE_THREADS) {
        if ((long long)(i + 1) * V <= left) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((unsigned)__cvta_generic_to_shared(dst + i * V)), "l"(src + (long long)i * V) : "memory");
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) dst[i * V + j] = (long long)i * V + j < left ? src[(long long)i * V + j] : from_f32<T>(0.f);
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
}
template <typename T> __device__ __forceinline__ void ln_tile_out(T* dst, const T* src, long long left, int n) {
    constexpr int V = 16 / (int)sizeof(T);
    for (int i = threadIdx.x; i < n / V; i += LN_TILE_THREADS) {
        if ((long long)(i + 1) * V <= left) {
            *reinterpret_cast<uint4*>(dst + (long long)i * V) = *reinterpret_cast<const uint4*>(src + i * V);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if ((long long)i * V + j < left) dst[(long long)i * V + j] = src[i * V + j];
        }
    }
}

template <typename T> __global__ void __launch_bounds__(LN_TILE_THREADS) layer_norm_fwd_tile_kernel(LnFwd P) {
    pdl_launch_dependents();
    pdl_wait();
    extern __shared__ __align__(16) uint8_t ln_smem[];
    constexpr int R = ln_tile_rows<T>();
    T* t = reinterpret_cast<T*>(ln_smem);
    const int n = R * P.c, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float inv_c = 1.f / (float)P.c;
    const long long total = P.rows * P.c;
    for (long long r0 = (long long)blockIdx.x * R; r0 < P.rows; r0 += (long long)gridDim.x * R) {
        const T* x = static_cast<const T*>(P.x) + r0 * P.c;
        ln_tile_in(t, x, total - r0 * P.c, n);
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
        if (warp < R) {
            T* row = t + warp * P.c;
            float s = 0.f;
#pragma unroll 8
            for (int i = lane; i < P.c; i += 32) s += to_f32<T>(row[i]);
            const float mean = ln_mean(ln_sum<32>(s, nullptr), (float)P.c, inv_c);
            s = 0.f;
#pragma unroll 8
            for (int i = lane; i < P.c; i += 32) {
                const float d = to_f32<T>(row[i]) - mean;
                s = fmaf(d, d, s);
            }
            const float rstd = 1.f / sqrtf(ln_sum<32>(s, nullptr) * inv_c + P.eps);
#pragma unroll 8
            for (int i = lane; i < P.c; i += 32)
                row[i] = from_f32<T>(fmaf((to_f32<T>(row[i]) - mean) * rstd, P.gamma ? __ldg(P.gamma + i) : 1.f, P.beta ? __ldg(P.beta + i) : 0.f));
            if (P.mean && lane == 0 && r0 + warp < P.rows) {
                P.mean[r0 + warp] = mean;
                P.rstd[r0 + warp] = rstd;
            }
        }
        __syncthreads();
        ln_tile_out(static_cast<T*>(P.y) + r0 * P.c, t, total - r0 * P.c, n);
        __syncthreads();
    }
}

// The sum over a row of what `f` gives for its elements, by a whole block: eight at a time in fp32, those in fp64, since a thread may have
// thousands (`red`: as in ln_sum2).
template <typename F> __device__ __forceinline__ double ln_row_sum(int c, double* red, F f) {
    double s = 0.0;
    for (int i0 = threadIdx.x; i0 < c; i0 += 8 * blockDim.x) {
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = i0 + u * (int)blockDim.x < c ? f(i0 + u * (int)blockDim.x) : 0.f;
        s += (double)(((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])));
    }
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) red[threadIdx.x >> 5] = s;
    __syncthreads();
    s = lane < warps ? red[lane] : 0.0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
}

// Any channel count: a block a row, the row read three times (the second and third time from the caches).
template <typename T> __global__ void __launch_bounds__(LN_MAX_BLOCK) layer_norm_fwd_loop_kernel(LnFwd P) {
    pdl_launch_dependents();
    pdl_wait();
    __shared__ double red[2][32];
    for (long long row = blockIdx.x; row < P.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(P.x) + row * P.ld_x;
        T* y = static_cast<T*>(P.y) + row * P.ld_y;
        const float mean = (float)(ln_row_sum(P.c, red[0], [&](int i) { return to_f32<T>(x[i]); }) / P.c);
        const float var = (float)(ln_row_sum(P.c, red[1], [&](int i) {
            const float d = to_f32<T>(x[i]) - mean;
            return d * d;
        }) / P.c);
        const float rstd = 1.f / sqrtf(var + P.eps);
        for (int i = threadIdx.x; i < P.c; i += blockDim.x)
            y[i] = from_f32<T>(fmaf((to_f32<T>(x[i]) - mean) * rstd, P.gamma ? P.gamma[i] : 1.f, P.beta ? P.beta[i] : 0.f));
        if (P.mean && threadIdx.x == 0) {
            P.mean[row] = mean;
            P.rstd[row] = rstd;
        }
    }
}

struct LnBwd {
    const void *g, *x, *add;
    void* dx;
    const float *gamma, *mean, *rstd;
    float* partials;  // [blocks][2][c]: sums of g*xhat and of g over the rows of a block; NULL: not wanted
    long long rows, ld_g, ld_x, ld_add, ld_dx;
    int c, nvec;
};

// Bound: memory (g and x once, dx once).  A block walks over rows; a thread keeps the sums of its own columns in registers, and the
// next row's g and x are requested before this row's sums are formed.
template <typename T, int V, int L, int VPL, bool ADD, bool SUMS>
__global__ void __launch_bounds__(L == 0 ? LN_BWD_MAX_BLOCK : LN_THREADS, L != 0 && VPL * V <= 8 ? 3 : 1) layer_norm_bwd_kernel(LnBwd P) {
    pdl_launch_dependents();
    pdl_wait();
    __shared__ float2 red[2][32];
    const int W = L == 0 ? (int)blockDim.x : L;
    const int lane = L == 0 ? (int)threadIdx.x : (int)threadIdx.x % L;
    const int groups = L == 0 ? 1 : LN_THREADS / L, group = L == 0 ? 0 : (int)threadIdx.x / L;
    const float inv_c = 1.f / (float)P.c;
    const long long step = (long long)gridDim.x * groups;
    constexpr int N = (V + 1) / 2;
    float2 sg[SUMS ? VPL : 1][N], sb[SUMS ? VPL : 1][N], ga[VPL][N];
    if (SUMS)
#pragma unroll
        for (int k = 0; k < VPL; ++k)
#pragma unroll
            for (int j = 0; j < N; ++j) sg[k][j] = sb[k][j] = make_float2(0.f, 0.f);
#pragma unroll
    for (int k = 0; k < VPL; ++k) {
        const int i = lane + k * W;
        ln_ldf<V>(P.gamma && i < P.nvec ? P.gamma + i * V : nullptr, ga[k], 1.f);
    }
    LnVec<T, V> gn[VPL], xn[VPL];
    float mn = 0.f, rn = 0.f;
    auto fetch = [&](long long row) {
        const bool live = row < P.rows;
        const T* g = static_cast<const T*>(P.g) + (live ? row : 0) * P.ld_g;
        const T* x = static_cast<const T*>(P.x) + (live ? row : 0) * P.ld_x;
#pragma unroll
        for (int k = 0; k < VPL; ++k) {
            const int i = lane + k * W;
            if (live && i < P.nvec) {
                gn[k] = ln_ld<T, V>(g + (long long)i * V);
                xn[k] = ln_ld<T, V>(x + (long long)i * V);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) gn[k].v[j] = xn[k].v[j] = from_f32<T>(0.f);
            }
        }
        mn = live ? P.mean[row] : 0.f;
        rn = live ? P.rstd[row] : 0.f;
    };
    int turn = 0;
    long long row = (long long)blockIdx.x * groups + group;
    fetch(row);
    for (long long r0 = (long long)blockIdx.x * groups; r0 < P.rows; r0 += step, row += step) {
        LnPairs<T, V> d[VPL], xh[VPL];  // g, from there g*gamma; x, from there xhat
#pragma unroll
        for (int k = 0; k < VPL; ++k) {
            d[k] = LnPairs<T, V>(gn[k]);
            xh[k] = LnPairs<T, V>(xn[k]);
        }
        const float mean = mn, rstd = rn;
        if (r0 + step < P.rows) fetch(row + step);
        float2 sa = make_float2(0.f, 0.f), sx = sa;
#pragma unroll
        for (int k = 0; k < VPL; ++k) {
            const float rk = lane + k * W < P.nvec ? rstd : 0.f;
            const float2 rs = make_float2(rk, V == 1 ? 0.f : rk);
#pragma unroll
            for (int j = 0; j < N; ++j) {  // (columns past the end have g = 0, and xhat = 0 where mean * rstd would be inf)
                const float2 g = d[k].p[j], h = mul2(add2(xh[k].p[j], splat2(-mean)), rs), t = mul2(g, ga[k][j]);
                sa = add2(sa, t);
                sx = fma2(t, h, sx);
                if (SUMS) {
                    sg[k][j] = fma2(g, h, sg[k][j]);
                    sb[k][j] = add2(sb[k][j], g);
                }
                d[k].p[j] = t;
                xh[k].p[j] = h;
            }
        }
        const float2 s = ln_sum2<L>(make_float2(sa.x + sa.y, sx.x + sx.y), red[turn]);
        turn ^= 1;
        const float2 r = splat2(rstd), a = splat2(-s.x * inv_c * rstd), b = splat2(-s.y * inv_c * rstd);
        if (row < P.rows) {
            T* dx = static_cast<T*>(P.dx) + row * P.ld_dx;
            const T* add = ADD ? static_cast<const T*>(P.add) + row * P.ld_add : nullptr;
#pragma unroll
            for (int k = 0; k < VPL; ++k) {
                const int i = lane + k * W;
                if (i < P.nvec) {
                    LnPairs<T, V> ad;
                    if (ADD) ad = LnPairs<T, V>(ln_ld<T, V>(add + (long long)i * V));
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        d[k].p[j] = fma2(xh[k].p[j], b, fma2(d[k].p[j], r, a));
                        if (ADD) d[k].p[j] = add2(d[k].p[j], ad.p[j]);
                    }
                    ln_st<T, V>(dx + (long long)i * V, d[k].rounded());
                }
            }
        }
    }
    if constexpr (SUMS) {
        float* out = P.partials + (size_t)blockIdx.x * 2 * P.c;
        if constexpr (L == 0) {
#pragma unroll
            for (int k = 0; k < VPL; ++k) {
                const int i = lane + k * W;
                if (i < P.nvec)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        out[i * V + j] = j & 1 ? sg[k][j / 2].y : sg[k][j / 2].x;
                        out[P.c + i * V + j] = j & 1 ? sb[k][j / 2].y : sb[k][j / 2].x;
                    }
            }
        } else {
            // the groups of a warp, then the warps one after the other
            extern __shared__ float ln_cols[];  // [2][c]
#pragma unroll
            for (int k = 0; k < VPL; ++k)
#pragma unroll
                for (int j = 0; j < N; ++j)
#pragma unroll
                    for (int o = L; o < 32; o <<= 1) {
                        sg[k][j].x += __shfl_xor_sync(0xffffffffu, sg[k][j].x, o);
                        sg[k][j].y += __shfl_xor_sync(0xffffffffu, sg[k][j].y, o);
                        sb[k][j].x += __shfl_xor_sync(0xffffffffu, sb[k][j].x, o);
                        sb[k][j].y += __shfl_xor_sync(0xffffffffu, sb[k][j].y, o);
                    }
            for (int w = 0; w < LN_THREADS / 32; ++w) {
                if ((int)(threadIdx.x >> 5) == w && (threadIdx.x & 31) < L) {
#pragma unroll
                    for (int k = 0; k < VPL; ++k) {
                        const int i = lane + k * W;
                        if (i < P.nvec)
#pragma unroll
                            for (int j = 0; j < V; ++j) {
                                const int at = i * V + j;
                                ln_cols[at] = (w ? ln_cols[at] : 0.f) + (j & 1 ? sg[k][j / 2].y : sg[k][j / 2].x);
                                ln_cols[P.c + at] = (w ? ln_cols[P.c + at] : 0.f) + (j & 1 ? sb[k][j / 2].y : sb[k][j / 2].x);
                            }
                    }
                }
                __syncthreads();
            }
            for (int i = threadIdx.x; i < 2 * P.c; i += LN_THREADS) out[i] = ln_cols[i];
        }
    }
}

// The backward pass on such tiles: g and x (and `add`) of R rows in shared memory; a thread owns columns of the sums.
template <typename T, bool SUMS> __global__ void __launch_bounds__(LN_TILE_THREADS) layer_norm_bwd_tile_kernel(LnBwd P) {
    pdl_launch_dependents();
    pdl_wait();
    extern __shared__ __align__(16) uint8_t ln_smem[];
    constexpr int R = ln_tile_rows<T>();
    const int n = R * P.c, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    T* g = reinterpret_cast<T*>(ln_smem);
    T* x = g + n;
    T* ad = x + n;
    __shared__ float4 stat[R];  // mean, rstd, rstd*avg(d), rstd*avg(d*xhat) of a row
    const float inv_c = 1.f / (float)P.c;
    const long long total = P.rows * P.c;
    float sg[LN_TILE_COLS], sb[LN_TILE_COLS];
#pragma unroll
    for (int k = 0; k < LN_TILE_COLS; ++k) sg[k] = sb[k] = 0.f;
    for (long long r0 = (long long)blockIdx.x * R; r0 < P.rows; r0 += (long long)gridDim.x * R) {
        const long long at = r0 * P.c, left = total - at;
        ln_tile_in(g, static_cast<const T*>(P.g) + at, left, n);
        ln_tile_in(x, static_cast<const T*>(P.x) + at, left, n);
        if (P.add) ln_tile_in(ad, static_cast<const T*>(P.add) + at, left, n);
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
        if (warp < R) {
            const bool live = r0 + warp < P.rows;
            const float mean = live ? P.mean[r0 + warp] : 0.f, rstd = live ? P.rstd[r0 + warp] : 0.f;
            float2 s = make_float2(0.f, 0.f);
#pragma unroll 8
            for (int i = lane; i < P.c; i += 32) {
                const float d = to_f32<T>(g[warp * P.c + i]) * (P.gamma ? __ldg(P.gamma + i) : 1.f);
                s.x += d;
                s.y = fmaf(d, (to_f32<T>(x[warp * P.c + i]) - mean) * rstd, s.y);
            }
            s = ln_sum2<32>(s, nullptr);
            if (lane == 0) stat[warp] = make_float4(mean, rstd, s.x * inv_c * rstd, s.y * inv_c * rstd);
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < LN_TILE_COLS; ++k) {
            const int i = threadIdx.x + k * LN_TILE_THREADS;
            if (i >= P.c) break;
            const float ga = P.gamma ? __ldg(P.gamma + i) : 1.f;
#pragma unroll
            for (int r = 0; r < R; ++r) {  // (rows behind the last: g and rstd are zero)
                const float4 q = stat[r];
                const float gj = to_f32<T>(g[r * P.c + i]), xh = (to_f32<T>(x[r * P.c + i]) - q.x) * q.y;
                if (SUMS) {
                    sg[k] = fmaf(gj, xh, sg[k]);
                    sb[k] += gj;
                }
                float v = fmaf(gj * ga, q.y, -q.z) - xh * q.w;
                if (P.add) v += to_f32<T>(ad[r * P.c + i]);
                g[r * P.c + i] = from_f32<T>(v);
            }
        }
        __syncthreads();
        ln_tile_out(static_cast<T*>(P.dx) + at, g, left, n);
        __syncthreads();
    }
    if (SUMS) {
        float* out = P.partials + (size_t)blockIdx.x * 2 * P.c;
#pragma unroll
        for (int k = 0; k < LN_TILE_COLS; ++k) {
            const int i = threadIdx.x + k * LN_TILE_THREADS;
            if (i < P.c) {
                out[i] = sg[k];
                out[P.c + i] = sb[k];
            }
        }
    }
}

// Any channel count: dx of a row by a block that reads the row twice, ...
template <typename T> __global__ void __launch_bounds__(LN_MAX_BLOCK) layer_norm_bwd_loop_kernel(LnBwd P) {
    pdl_launch_dependents();
    pdl_wait();
    __shared__ float2 red[2][32];
    const float inv_c = 1.f / (float)P.c;
    int turn = 0;
    for (long long row = blockIdx.x; row < P.rows; row += gridDim.x) {
        const T* g = static_cast<const T*>(P.g) + row * P.ld_g;
        const T* x = static_cast<const T*>(P.x) + row * P.ld_x;
        const T* add = P.add ? static_cast<const T*>(P.add) + row * P.ld_add : nullptr;
        T* dx = static_cast<T*>(P.dx) + row * P.ld_dx;
        const float mean = P.mean[row], rstd = P.rstd[row];
        float2 s = make_float2(0.f, 0.f);
        for (int i = threadIdx.x; i < P.c; i += blockDim.x) {
            const float d = to_f32<T>(g[i]) * (P.gamma ? P.gamma[i] : 1.f);
            s.x += d;
            s.y = fmaf(d, (to_f32<T>(x[i]) - mean) * rstd, s.y);
        }
        s = ln_sum2<0>(s, red[turn]);
        turn ^= 1;
        for (int i = threadIdx.x; i < P.c; i += blockDim.x) {
            const float d = to_f32<T>(g[i]) * (P.gamma ? P.gamma[i] : 1.f), xh = (to_f32<T>(x[i]) - mean) * rstd;
            float v = rstd * (d - s.x * inv_c - xh * (s.y * inv_c));
            if (add) v += to_f32<T>(add[i]);
            dx[i] = from_f32<T>(v);
        }
    }
}
// ... and the columns' sums by blocks of 128 columns (x) and a range of rows (y), before dx may overwrite g.
template <typename T> __global__ void __launch_bounds__(128) layer_norm_cols_kernel(LnBwd P, long long rows_per_block) {
    pdl_launch_dependents();
    pdl_wait();
    const int i = blockIdx.x * 128 + threadIdx.x;
    if (i >= P.c) return;
    const long long r0 = (long long)blockIdx.y * rows_per_block, r1 = r0 + rows_per_block < P.rows ? r0 + rows_per_block : P.rows;
    float sg = 0.f, sb = 0.f;
    for (long long r = r0; r < r1; ++r) {
        const float g = to_f32<T>(static_cast<const T*>(P.g)[r * P.ld_g + i]);
        sg = fmaf(g, (to_f32<T>(static_cast<const T*>(P.x)[r * P.ld_x + i]) - P.mean[r]) * P.rstd[r], sg);
        sb += g;
    }
    float* out = P.partials + (size_t)blockIdx.y * 2 * P.c;
    out[i] = sg;
    out[P.c + i] = sb;
}

// dgamma and dbeta from `parts` blocks' sums: 8 columns (a 32-byte sector) by 128 threads each, in fp64 and a fixed order.
constexpr int LN_RED_COLS = 8, LN_RED_ROWS = 128;
static __global__ void __launch_bounds__(LN_RED_COLS * LN_RED_ROWS) layer_norm_reduce_kernel(const float* __restrict__ partials, int parts, int c, float* __restrict__ dgamma, float* __restrict__ dbeta) {
    pdl_launch_dependents();
    pdl_wait();
    __shared__ double red[LN_RED_ROWS / 4][LN_RED_COLS];
    const int j = threadIdx.x % LN_RED_COLS, w = threadIdx.x / LN_RED_COLS, col = blockIdx.x * LN_RED_COLS + j;
    double s = 0.0;
    if (col < 2 * c) {
        const float* p = partials + col;
        const size_t ld = 2 * (size_t)c;
#pragma unroll 8
        for (int b = w; b < parts; b += LN_RED_ROWS) s += (double)p[(size_t)b * ld];
    }
    s += __shfl_xor_sync(0xffffffffu, s, 8);  // a warp holds four rows of the eight columns
    s += __shfl_xor_sync(0xffffffffu, s, 16);
    if ((threadIdx.x & 31) < LN_RED_COLS) red[w / 4][j] = s;
    __syncthreads();
    if (threadIdx.x < 32) {  // four threads a column
        s = 0.0;
        for (int b = threadIdx.x / LN_RED_COLS; b < LN_RED_ROWS / 4; b += 4) s += red[b][j];
        s += __shfl_xor_sync(0xffffffffu, s, 8);
        s += __shfl_xor_sync(0xffffffffu, s, 16);
        if (threadIdx.x < LN_RED_COLS && col < 2 * c) (col < c ? dgamma[col] : dbeta[col - c]) = (float)s;
    }
}

}  // namespace nbcbs
