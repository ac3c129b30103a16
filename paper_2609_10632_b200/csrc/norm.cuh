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
template <int V> __device__ __forceinline__ void ln_ldf(const float* p, float (&o)[V], float without) {
    if (!p) {
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = without;
    } else if constexpr (V == 1) {
        o[0] = __ldg(p);
    } else {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            const float4 f = __ldg(reinterpret_cast<const float4*>(p + j));
            o[j] = f.x; o[j + 1] = f.y; o[j + 2] = f.z; o[j + 3] = f.w;
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
        float f[VPL][V];
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < VPL; ++k) {
            const int i = lane + k * W;
            if (live && i < P.nvec) {
                const LnVec<T, V> v = ln_ld<T, V>(x + (long long)i * V);
#pragma unroll
                for (int j = 0; j < V; ++j) f[k][j] = to_f32<T>(v.v[j]);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) f[k][j] = 0.f;
            }
        }
#pragma unroll
        for (int k = 0; k < VPL; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) s += f[k][j];
        const float mean = ln_sum<L>(s, red[0]) * inv_c;
        s = 0.f;
#pragma unroll
        for (int k = 0; k < VPL; ++k)
            if (lane + k * W < P.nvec)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    f[k][j] -= mean;
                    s = fmaf(f[k][j], f[k][j], s);
                }
        const float rstd = 1.f / sqrtf(ln_sum<L>(s, red[1]) * inv_c + P.eps);
        if (!live) continue;
        T* y = static_cast<T*>(P.y) + row * P.ld_y;
#pragma unroll
        for (int k = 0; k < VPL; ++k) {
            const int i = lane + k * W;
            if (i < P.nvec) {
                float ga[V], be[V];
                ln_ldf<V>(P.gamma ? P.gamma + i * V : nullptr, ga, 1.f);
                ln_ldf<V>(P.beta ? P.beta + i * V : nullptr, be, 0.f);
                LnVec<T, V> o;
#pragma unroll
                for (int j = 0; j < V; ++j) o.v[j] = from_f32<T>(fmaf(f[k][j] * rstd, ga[j], be[j]));
                ln_st<T, V>(y + (long long)i * V, o);
            }
        }
        if (P.mean && lane == 0) {
            P.mean[row] = mean;
            P.rstd[row] = rstd;
        }
    }
}

// Any channel count: a block a row, the row read three times (the second and third time from the caches).
template <typename T> __global__ void __launch_bounds__(LN_MAX_BLOCK) layer_norm_fwd_loop_kernel(LnFwd P) {
    pdl_launch_dependents();
    pdl_wait();
    __shared__ float2 red[2][32];
    const float inv_c = 1.f / (float)P.c;
    for (long long row = blockIdx.x; row < P.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(P.x) + row * P.ld_x;
        T* y = static_cast<T*>(P.y) + row * P.ld_y;
        float s = 0.f;
        for (int i = threadIdx.x; i < P.c; i += blockDim.x) s += to_f32<T>(x[i]);
        const float mean = ln_sum<0>(s, red[0]) * inv_c;
        s = 0.f;
        for (int i = threadIdx.x; i < P.c; i += blockDim.x) {
            const float d = to_f32<T>(x[i]) - mean;
            s = fmaf(d, d, s);
        }
        const float rstd = 1.f / sqrtf(ln_sum<0>(s, red[1]) * inv_c + P.eps);
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
__global__ void __launch_bounds__(L == 0 ? LN_BWD_MAX_BLOCK : LN_THREADS) layer_norm_bwd_kernel(LnBwd P) {
    pdl_launch_dependents();
    pdl_wait();
    __shared__ float2 red[2][32];
    const int W = L == 0 ? (int)blockDim.x : L;
    const int lane = L == 0 ? (int)threadIdx.x : (int)threadIdx.x % L;
    const int groups = L == 0 ? 1 : LN_THREADS / L, group = L == 0 ? 0 : (int)threadIdx.x / L;
    const float inv_c = 1.f / (float)P.c;
    const long long step = (long long)gridDim.x * groups;
    float sg[SUMS ? VPL : 1][V], sb[SUMS ? VPL : 1][V];
    if (SUMS)
#pragma unroll
        for (int k = 0; k < VPL; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) sg[k][j] = sb[k][j] = 0.f;
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
        LnVec<T, V> gv[VPL], xv[VPL];
#pragma unroll
        for (int k = 0; k < VPL; ++k) {
            gv[k] = gn[k];
            xv[k] = xn[k];
        }
        const float mean = mn, rstd = rn;
        if (r0 + step < P.rows) fetch(row + step);
        float2 s = make_float2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < VPL; ++k) {
            const int i = lane + k * W;
            if (i < P.nvec) {
                float ga[V];
                ln_ldf<V>(P.gamma ? P.gamma + i * V : nullptr, ga, 1.f);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float gj = to_f32<T>(gv[k].v[j]), xh = (to_f32<T>(xv[k].v[j]) - mean) * rstd, d = gj * ga[j];
                    s.x += d;
                    s.y = fmaf(d, xh, s.y);
                    if (SUMS) {
                        sg[k][j] = fmaf(gj, xh, sg[k][j]);
                        sb[k][j] += gj;
                    }
                }
            }
        }
        s = ln_sum2<L>(s, red[turn]);
        turn ^= 1;
        const float a = s.x * inv_c, b = s.y * inv_c;
        if (row < P.rows) {
            T* dx = static_cast<T*>(P.dx) + row * P.ld_dx;
            const T* add = ADD ? static_cast<const T*>(P.add) + row * P.ld_add : nullptr;
#pragma unroll
            for (int k = 0; k < VPL; ++k) {
                const int i = lane + k * W;
                if (i < P.nvec) {
                    float ga[V];
                    ln_ldf<V>(P.gamma ? P.gamma + i * V : nullptr, ga, 1.f);
                    LnVec<T, V> o, ad;
                    if (ADD) ad = ln_ld<T, V>(add + (long long)i * V);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float xh = (to_f32<T>(xv[k].v[j]) - mean) * rstd, d = to_f32<T>(gv[k].v[j]) * ga[j];
                        float v = rstd * (d - a - xh * b);
                        if (ADD) v += to_f32<T>(ad.v[j]);
                        o.v[j] = from_f32<T>(v);
                    }
                    ln_st<T, V>(dx + (long long)i * V, o);
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
                        out[i * V + j] = sg[k][j];
                        out[P.c + i * V + j] = sb[k][j];
                    }
            }
        } else {
            // the groups of a warp, then the warps one after the other
            extern __shared__ float ln_cols[];  // [2][c]
#pragma unroll
            for (int k = 0; k < VPL; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j)
#pragma unroll
                    for (int o = L; o < 32; o <<= 1) {
                        sg[k][j] += __shfl_xor_sync(0xffffffffu, sg[k][j], o);
                        sb[k][j] += __shfl_xor_sync(0xffffffffu, sb[k][j], o);
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
                                ln_cols[at] = (w ? ln_cols[at] : 0.f) + sg[k][j];
                                ln_cols[P.c + at] = (w ? ln_cols[P.c + at] : 0.f) + sb[k][j];
                            }
                    }
                }
                __syncthreads();
            }
            for (int i = threadIdx.x; i < 2 * P.c; i += LN_THREADS) out[i] = ln_cols[i];
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

// dgamma and dbeta from `parts` blocks' sums: 32 columns by 32 threads each, in fp64 and a fixed order.
static __global__ void __launch_bounds__(1024) layer_norm_reduce_kernel(const float* __restrict__ partials, int parts, int c, float* __restrict__ dgamma, float* __restrict__ dbeta) {
    pdl_launch_dependents();
    pdl_wait();
    __shared__ double red[32][33];
    const int col = blockIdx.x * 32 + (threadIdx.x & 31), w = threadIdx.x >> 5;
    double s = 0.0;
    if (col < 2 * c) {
        const float* p = partials + col;
        const size_t ld = 2 * (size_t)c;
#pragma unroll 8
        for (int b = w; b < parts; b += 32) s += (double)p[(size_t)b * ld];
    }
    red[w][threadIdx.x & 31] = s;
    __syncthreads();
    s = red[threadIdx.x & 31][w];  // column w of the 32, summed by this warp
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const int out = blockIdx.x * 32 + w;
    if ((threadIdx.x & 31) == 0 && out < 2 * c) (out < c ? dgamma[out] : dbeta[out - c]) = (float)s;
}

}  // namespace nbcbs
