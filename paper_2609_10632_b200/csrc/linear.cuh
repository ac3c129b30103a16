// Matrix products of MLP layers on the CUDA cores, their activations, and the sums of split products (see include/nb_linear.h
// for the arithmetic; the tensor-core kernel is tc_linear.cuh).
#pragma once
#include <type_traits>

#include "../../include/nb_linear.h"
#include "common.cuh"

namespace nbcbs {

enum { LIN_FWD = 0, LIN_DATA = 1, LIN_WEIGHT = 2 };

// ------------------------------------------------------------------------------------------ activations, fp32
// (An infinite z has the limit's value, not the NaN of inf * 0: where z is a factor it counts as the largest finite number.  A NaN stays
// in the other factor.)
__device__ __forceinline__ float lin_finite(float z) { return fminf(fmaxf(z, -3.4028235e38f), 3.4028235e38f); }
__device__ __forceinline__ float lin_act(float z, int act) {
    if (act == NB_ACT_SILU) return z < 0.f ? lin_finite(z) / (1.f + expf(-z)) : z / (1.f + expf(-z));
    if (act == NB_ACT_GELU) return z < 0.f ? 0.5f * lin_finite(z) * erfcf(-0.70710678f * z) : 0.5f * z * erfcf(-0.70710678f * z);
    return z;
}
__device__ __forceinline__ float lin_act_grad(float z, int act) {
    if (act == NB_ACT_SILU) {
        const float s = 1.f / (1.f + expf(-z));
        return s * (1.f + lin_finite(z) * (1.f - s));
    }
    if (act == NB_ACT_GELU) return fmaf(lin_finite(z) * 0.39894228f, expf(-0.5f * z * z), 0.5f * erfcf(-0.70710678f * z));
    return 1.f;
}

// ------------------------------------------------------------------------------------------ the same for 16-bit results
// Errors relative to the VALUE, in the tails too: GELU and SiLU of a negative z are far smaller than z, and an absolute error that
// rounding hides at z = 1 is the whole value at z = -5 (SiLU by the hardware's tanh, which was here, is 10 % off at -6).  So nothing
// is formed as a difference of nearly equal numbers.  With t = |z|:
//   E = e^(-t^2/2),  q = Phi(-t) = E * P(1 / (1 + 0.36 t)):  P a polynomial of degree 5 (Hastings' form of the tail), fitted here to
//   Phi(-t) e^(t^2/2) on [0, 14] for the least relative error, 1.3e-5; with the roundings of E's exponent 2^-15 as far as t = 8
//   (beyond, E is the error: its exponent's rounding grows as t^2, and 2^-126 is reached at 13.2).
// t counts as 64 at most, so that 0 * inf is not formed; a NaN stays in E.
struct LinTail {
    float2 t, E, minus_P;
};
__device__ __forceinline__ float lin_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float lin_rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ LinTail lin_tail2(float2 z) {
    LinTail o;
    const float2 e = mul2(mul2(z, z), splat2(-0.72134752f));  // -z^2/2 in base 2
    o.E = make_float2(lin_ex2(e.x), lin_ex2(e.y));
    o.t = make_float2(fminf(fabsf(z.x), 64.f), fminf(fabsf(z.y), 64.f));
    const float2 d = fma2(o.t, splat2(0.36f), splat2(1.f));
    const float r = lin_rcp(d.x * d.y);  // (one reciprocal for both: the special-function unit is what this takes most of)
    const float2 u = mul2(splat2(r), make_float2(d.y, d.x));
    float2 p = fma2(u, splat2(0.09851564340977417f), splat2(-0.25438743173341666f));
    p = fma2(p, u, splat2(-0.035116434501124935f));
    p = fma2(p, u, splat2(-0.16869575236171047f));
    p = fma2(p, u, splat2(-0.14012407751013303f));
    o.minus_P = fma2(p, u, splat2(-0.0001912892156621022f));
    return o;
}
// The logistic function 1 / (1 + e^-z): relative error 2^-19 or less from z = -8 on (the exponent's rounding grows as z; at -87 the sum
// leaves what the reciprocal takes and the result is zero).
__device__ __forceinline__ float2 lin_logistic2(float2 z) {
    const float2 e = mul2(z, splat2(-1.44269504f)), d = add2(make_float2(lin_ex2(e.x), lin_ex2(e.y)), splat2(1.f));
    return make_float2(lin_rcp(d.x), lin_rcp(d.y));
}
__device__ __forceinline__ float2 lin_act2(float2 z, int act) {
    if (act == NB_ACT_GELU) {  // z Phi(z) = max(z, 0) - t Phi(-t)
        const LinTail f = lin_tail2(z);
        return fma2(mul2(f.E, f.minus_P), f.t, make_float2(fmaxf(z.x, 0.f), fmaxf(z.y, 0.f)));
    }
    if (act == NB_ACT_SILU) return mul2(make_float2(fmaxf(z.x, -3.4028235e38f), fmaxf(z.y, -3.4028235e38f)), lin_logistic2(z));
    return z;
}
__device__ __forceinline__ float2 lin_act_grad2(float2 z, int act) {
    if (act == NB_ACT_GELU) {  // Phi(z) + z phi(z): with k = t phi(t) - Phi(-t), -k for a negative z and 1 + k else
        const LinTail f = lin_tail2(z);
        const float2 k = mul2(f.E, fma2(f.t, splat2(0.39894228f), f.minus_P)), r = add2(k, splat2(1.f));
        return make_float2(z.x < 0.f ? -k.x : r.x, z.y < 0.f ? -k.y : r.y);
    }
    if (act == NB_ACT_SILU) {
        const float2 s = lin_logistic2(z), q = fma2(s, splat2(-1.f), splat2(1.f));
        return mul2(s, fma2(make_float2(lin_finite(z.x), lin_finite(z.y)), q, splat2(1.f)));
    }
    return splat2(1.f);
}

// ------------------------------------------------------------------------------------------ products on plain FMA units
// C[m][n] = sum_k A(m,k) B(n,k):
//   LIN_FWD     m = row,   n = c_out, k = c_in   A = x [m][k], B = w [n][k]
//   LIN_DATA    m = row,   n = c_in,  k = c_out  A = dy [m][k], B = w [k][n]
//   LIN_WEIGHT  m = c_out, n = c_in,  k = row    A = dy [k][m], B = x [k][n]
struct LinArgs {
    const void *a, *b;
    long long lda, ldb;
    long long M, N, K, kslice;  // kslice: products of a slice (blockIdx.z), a multiple of LS_BK
    int slices;
    float* partial;  // slices > 1: [slices][M][N]
    // epilogue
    const float* bias;
    int act;
    const void *add, *zin;  // residual / other branch's gradient [M][N] with pitch ld_add; z_in [M][N]
    long long ld_add;
    void* z;                // [M][N]
    void* out;              // LIN_WEIGHT: fp32
    long long ld_out;
    int* status;            // of the plan
};

// One result, rounded; fp16: a saturated one is counted.
template <typename T> __device__ __forceinline__ T lin_rounded(const LinArgs& P, float v) {
    const T r = from_f32<T>(v);
    if constexpr (std::is_same<T, __half>::value) {
        if ((__half_as_ushort(r) & 0x7fffu) >= 0x7bffu) atomicAdd(P.status + ST_SAT, 1);
    }
    return r;
}

template <typename T, int KIND> __device__ __forceinline__ void lin_store(const LinArgs& P, long long m, long long n, float v) {
    if (KIND == LIN_WEIGHT) {
        static_cast<float*>(P.out)[m * P.ld_out + n] = v;
        return;
    }
    if (KIND == LIN_FWD) {
        if (P.bias) v += P.bias[n];
        if (P.z) static_cast<T*>(P.z)[m * P.N + n] = lin_rounded<T>(P, v);
        v = lin_act(v, P.act);
        if (P.add) v += to_f32<T>(static_cast<const T*>(P.add)[m * P.ld_add + n]);
    } else {
        if (P.add) v += to_f32<T>(static_cast<const T*>(P.add)[m * P.ld_add + n]);
        if (P.zin) v *= lin_act_grad(to_f32<T>(static_cast<const T*>(P.zin)[m * P.N + n]), P.act);
    }
    static_cast<T*>(P.out)[m * P.ld_out + n] = lin_rounded<T>(P, v);
}

// Bound: FMA issue.  A block of 256 threads has a [TILE x TILE] tile: 128 (a thread [8 x 8]: four 16-byte shared loads for 64 products) where
// there are enough of them, on their own or with long slices of k, else 64 ([4 x 4]), with slices that put four blocks on an SM.  Operand tiles of 16 k travel
// through registers into shared memory as fp32, k-major, double-buffered.  VEC: every operand row is whole vectors of four.
// 1600 x 384 x 384 forward: 43 us with one 64-tile block an SM, 37 with four; 8000 x 1024 x 1024 480 us (35 TFLOP/s; the library product 360).
// 1061 x 3520 -> 1000 forward: 369 us on tiles of 64, 213 on tiles of 128 in four slices; the weight gradient of 25600 x 384 -> 384 285 and 148.
constexpr int LS_BK = 16, LS_THREADS = 256;

// Four elements of an operand stored [outer][inner] at (outer, inner..inner+3) as fp32, zeros outside.
template <typename T, bool VEC> __device__ __forceinline__ float4 ls_load(const T* p, long long ld, long long outer, long long inner, long long outers, long long inners) {
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (outer >= outers) return v;
    const T* q = p + outer * ld + inner;
    if (VEC) {
        if (inner < inners) {
            if constexpr (sizeof(T) == 4) {
                v = *reinterpret_cast<const float4*>(q);
            } else {
                const uint2 r = *reinterpret_cast<const uint2*>(q);
                const float2 lo = pair_to_f32<T>(reinterpret_cast<const T*>(&r.x)), hi = pair_to_f32<T>(reinterpret_cast<const T*>(&r.y));
                v = make_float4(lo.x, lo.y, hi.x, hi.y);
            }
        }
    } else {
        if (inner < inners) v.x = to_f32<T>(q[0]);
        if (inner + 1 < inners) v.y = to_f32<T>(q[1]);
        if (inner + 2 < inners) v.z = to_f32<T>(q[2]);
        if (inner + 3 < inners) v.w = to_f32<T>(q[3]);
    }
    return v;
}

template <typename T, int KIND, bool VEC, int TILE> __global__ void __launch_bounds__(LS_THREADS, TILE == 128 ? 2 : 4) lin_simt_kernel(LinArgs P) {
    pdl_launch_dependents();
    pdl_wait();
    constexpr int G = TILE / 64;  // groups of four rows (columns) that a thread has, 64 apart
    constexpr int PITCH = TILE + 4;
    __shared__ __align__(16) float sA[2][LS_BK][PITCH], sB[2][LS_BK][PITCH];
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const long long tiles_n = (P.N + TILE - 1) / TILE;
    const long long m0 = blockIdx.x / tiles_n * TILE, n0 = blockIdx.x % tiles_n * TILE;
    const long long k0 = (long long)blockIdx.z * P.kslice, k1 = k0 + P.kslice < P.K ? k0 + P.kslice : P.K;
    const T* A = static_cast<const T*>(P.a);
    const T* B = static_cast<const T*>(P.b);
    constexpr bool A_K = KIND != LIN_WEIGHT, B_K = KIND == LIN_FWD;  // k is the contiguous index of the operand
    // an operand tile is 16 k x TILE outer: stored [outer][k] a thread takes 4 k of G.. of one outer index, stored [k][outer] 4 outer of G k
    const int ro = tid % TILE, rk = tid / TILE * (4 * G), co = tid % (TILE / 4) * 4, ck = tid / (TILE / 4);
    constexpr int CK = LS_THREADS / (TILE / 4);  // k between a thread's groups in the second case
    float4 ra[G], rb[G];
    auto fetch = [&](long long k) {
#pragma unroll
        for (int g = 0; g < G; ++g) {
            ra[g] = A_K ? ls_load<T, VEC>(A, P.lda, m0 + ro, k + rk + 4 * g, P.M, k1) : ls_load<T, VEC>(A, P.lda, k + ck + CK * g, m0 + co, k1, P.M);
            rb[g] = B_K ? ls_load<T, VEC>(B, P.ldb, n0 + ro, k + rk + 4 * g, P.N, k1) : ls_load<T, VEC>(B, P.ldb, k + ck + CK * g, n0 + co, k1, P.N);
        }
    };
    auto put = [&](int s) {
#pragma unroll
        for (int g = 0; g < G; ++g) {
            if (A_K) {
                sA[s][rk + 4 * g][ro] = ra[g].x; sA[s][rk + 4 * g + 1][ro] = ra[g].y; sA[s][rk + 4 * g + 2][ro] = ra[g].z; sA[s][rk + 4 * g + 3][ro] = ra[g].w;
            } else {
                *reinterpret_cast<float4*>(&sA[s][ck + CK * g][co]) = ra[g];
            }
            if (B_K) {
                sB[s][rk + 4 * g][ro] = rb[g].x; sB[s][rk + 4 * g + 1][ro] = rb[g].y; sB[s][rk + 4 * g + 2][ro] = rb[g].z; sB[s][rk + 4 * g + 3][ro] = rb[g].w;
            } else {
                *reinterpret_cast<float4*>(&sB[s][ck + CK * g][co]) = rb[g];
            }
        }
    };
    float2 acc[4 * G][2 * G];
#pragma unroll
    for (int i = 0; i < 4 * G; ++i)
#pragma unroll
        for (int j = 0; j < 2 * G; ++j) acc[i][j] = make_float2(0.f, 0.f);
    fetch(k0);
    put(0);
    __syncthreads();
    int s = 0;
    for (long long k = k0; k < k1; k += LS_BK) {
        const bool more = k + LS_BK < k1;
        if (more) fetch(k + LS_BK);
#pragma unroll
        for (int kk = 0; kk < LS_BK; ++kk) {
            float av[4 * G];
            float2 bv[2 * G];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const float4 a = *reinterpret_cast<const float4*>(&sA[s][kk][64 * g + ty * 4]), b = *reinterpret_cast<const float4*>(&sB[s][kk][64 * g + tx * 4]);
                av[4 * g] = a.x; av[4 * g + 1] = a.y; av[4 * g + 2] = a.z; av[4 * g + 3] = a.w;
                bv[2 * g] = make_float2(b.x, b.y);
                bv[2 * g + 1] = make_float2(b.z, b.w);
            }
#pragma unroll
            for (int i = 0; i < 4 * G; ++i)
#pragma unroll
                for (int j = 0; j < 2 * G; ++j) acc[i][j] = fma2(splat2(av[i]), bv[j], acc[i][j]);
        }
        if (more) {
            s ^= 1;
            put(s);  // (the other buffer: its readers passed the barrier of the round before)
            __syncthreads();
        }
    }
#pragma unroll
    for (int i = 0; i < 4 * G; ++i) {
        const long long m = m0 + 64 * (i / 4) + ty * 4 + i % 4;
        if (m >= P.M) continue;
#pragma unroll
        for (int j = 0; j < 4 * G; ++j) {
            const long long n = n0 + 64 * (j / 4) + tx * 4 + j % 4;
            if (n >= P.N) continue;
            const float v = j & 1 ? acc[i][j / 2].y : acc[i][j / 2].x;
            if (P.slices > 1) P.partial[((long long)blockIdx.z * P.M + m) * P.N + n] = v;
            else lin_store<T, KIND>(P, m, n, v);
        }
    }
}

// Adds the slices of a product (fp64, in their order) and finishes it.
template <typename T, int KIND> __global__ void __launch_bounds__(256) lin_slices_kernel(LinArgs P) {
    pdl_launch_dependents();
    pdl_wait();
    const long long n = P.M * P.N;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
        double s = 0.0;
        for (int z = 0; z < P.slices; ++z) s += (double)P.partial[z * n + i];
        lin_store<T, KIND>(P, i / P.N, i % P.N, (float)s);
    }
}

// Partial sums of dy over ranges of rows: [gridDim.y][c].  Bound: memory.  A block has 16 groups of V columns (V = 1 or a 16-byte
// vector) and 16 rows of them at a time.
template <typename T, int V> __global__ void __launch_bounds__(256) lin_colsum_kernel(const T* __restrict__ dy, long long ld, long long rows, int c, long long per, float* __restrict__ partial) {
    pdl_launch_dependents();
    pdl_wait();
    __shared__ float red[16][16 * V + 1];
    const int gx = threadIdx.x & 15, w = threadIdx.x >> 4, col = (blockIdx.x * 16 + gx) * V;
    const long long r0 = (long long)blockIdx.y * per, r1 = r0 + per < rows ? r0 + per : rows;
    float s[V];
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = 0.f;
    if (col < c) {
        const T* p = dy + col;
        long long r = r0 + w;
        for (; r + 48 < r1; r += 64) {  // four rows in flight
            T v[4][V];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if constexpr (V == 1) v[u][0] = p[(r + 16 * u) * ld];
                else *reinterpret_cast<uint4*>(v[u]) = *reinterpret_cast<const uint4*>(p + (r + 16 * u) * ld);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int j = 0; j < V; ++j) s[j] += to_f32<T>(v[u][j]);
        }
        for (; r < r1; r += 16)
#pragma unroll
            for (int j = 0; j < V; ++j) s[j] += to_f32<T>(p[r * ld + j]);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) red[w][gx * V + j] = s[j];
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * V; e += 256) {
        double t = 0.0;
#pragma unroll
        for (int k = 0; k < 16; ++k) t += (double)red[k][e];
        if (blockIdx.x * 16 * V + e < c) partial[(size_t)blockIdx.y * c + blockIdx.x * 16 * V + e] = (float)t;
    }
}
// dw (n1 elements, `s1` slices) and dbias (n2 elements, `s2` slices) from their slices, in one launch; a count of zero slices: nothing to add.
// `add1`: what dw holds is added as well.
static __global__ void __launch_bounds__(256) lin_weight_sums_kernel(const float* __restrict__ p1, int s1, long long n1, float* __restrict__ o1, const float* __restrict__ p2, int s2, int n2,
                                                                     float* __restrict__ o2, int add1) {
    pdl_launch_dependents();
    pdl_wait();
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x, step = (long long)gridDim.x * 256;
    if (s1 && (n1 & 3) == 0) {
        for (long long v = at; v < n1 / 4; v += step) {
            double s[4] = {0.0, 0.0, 0.0, 0.0};
            if (add1) {
                const float4 was = reinterpret_cast<const float4*>(o1)[v];
                s[0] = was.x; s[1] = was.y; s[2] = was.z; s[3] = was.w;
            }
            for (int z0 = 0; z0 < s1; z0 += 8) {  // eight slices in flight
                float4 a[8];
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (z0 + u < s1) a[u] = reinterpret_cast<const float4*>(p1 + (long long)(z0 + u) * n1)[v];
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (z0 + u < s1) {
                        s[0] += (double)a[u].x;
                        s[1] += (double)a[u].y;
                        s[2] += (double)a[u].z;
                        s[3] += (double)a[u].w;
                    }
            }
            reinterpret_cast<float4*>(o1)[v] = make_float4((float)s[0], (float)s[1], (float)s[2], (float)s[3]);
        }
    } else if (s1) {
        for (long long i = at; i < n1; i += step) {
            double s = add1 ? (double)o1[i] : 0.0;
            for (int z = 0; z < s1; ++z) s += (double)p1[z * n1 + i];
            o1[i] = (float)s;
        }
    }
    if (s2)
        for (long long i = at; i < n2; i += step) {
            double s = 0.0;
            for (int z = 0; z < s2; ++z) s += (double)p2[(long long)z * n2 + i];
            o2[i] = (float)s;
        }
}

// ------------------------------------------------------------------------------------------ a few rows: the weights are streamed once
// Forward product of R rows (1, 2, 4 or 8): bound by the bytes of w.  WPC warps share a column of the output (a row of w); a
// lane takes 16-byte pieces of it, several in flight, against the same pieces of every row of x, which L1 holds.
constexpr int LR_THREADS = 256;
template <typename T, int R> __global__ void __launch_bounds__(LR_THREADS) lin_rows_kernel(LinArgs P, int rows, int wpc) {
    pdl_launch_dependents();
    pdl_wait();
    constexpr int V = 16 / (int)sizeof(T);
    __shared__ float red[LR_THREADS / 32][R];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cols = LR_THREADS / 32 / wpc, part = warp % wpc;
    const long long n = (long long)blockIdx.x * cols + warp / wpc;
    const bool live = n < P.N;
    const int nvec = (int)(P.K / V);
    const T* x = static_cast<const T*>(P.a);
    const T* w = static_cast<const T*>(P.b) + (live ? n : 0) * P.ldb;
    float2 acc[R];
#pragma unroll
    for (int r = 0; r < R; ++r) acc[r] = make_float2(0.f, 0.f);
    constexpr int U = 4;
    const int stride = 32 * wpc;
    for (int i0 = part * 32 + lane; i0 < nvec; i0 += U * stride) {
        Vec16<T> wv[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (live && i0 + u * stride < nvec) wv[u] = ld16_stream(w + (long long)(i0 + u * stride) * V);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * stride;
            if (!live || i >= nvec) break;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (r >= rows) break;
                const Vec16<T> xv = ld16(x + (long long)r * P.lda + (long long)i * V);
#pragma unroll
                for (int j = 0; j < V; j += 2) acc[r] = fma2(pair_to_f32<T>(xv.v + j), pair_to_f32<T>(wv[u].v + j), acc[r]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float s = acc[r].x + acc[r].y;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0) red[warp][r] = s;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < cols * rows; e += LR_THREADS) {
        const int c = e % cols, r = e / cols;
        const long long nn = (long long)blockIdx.x * cols + c;
        float s = 0.f;
        for (int p = 0; p < wpc; ++p) s += red[c * wpc + p][r];
        if (nn < P.N) lin_store<T, LIN_FWD>(P, r, nn, s);
    }
}

// ------------------------------------------------------------------------------------------ odd channel counts on the tensor cores
// TMA wants rows of whole 16-byte vectors: operands of layers with other channel counts are copied into rows padded with zeros, and
// results out of such rows.  Eight elements of a padded row a thread; 16-bit elements as they are.
static __global__ void __launch_bounds__(256) lin_pad_kernel(const uint16_t* __restrict__ src, long long ld, long long rows, int cols, int cols8, uint16_t* __restrict__ dst) {
    pdl_launch_dependents();
    pdl_wait();
    const int nv = cols8 / 8;
    const long long n = rows * nv, step = (long long)gridDim.x * 256;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
        const long long r = i / nv;
        const int c = (int)(i - r * nv) * 8;
        const uint16_t* s = src + r * ld + c;
        uint16_t e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = c + j < cols ? s[j] : (uint16_t)0;
        uint4 v;
        v.x = e[0] | (uint32_t)e[1] << 16;
        v.y = e[2] | (uint32_t)e[3] << 16;
        v.z = e[4] | (uint32_t)e[5] << 16;
        v.w = e[6] | (uint32_t)e[7] << 16;
        *reinterpret_cast<uint4*>(dst + i * 8) = v;
    }
}
static __global__ void __launch_bounds__(256) lin_unpad_kernel(const uint16_t* __restrict__ src, int cols8, long long rows, int cols, uint16_t* __restrict__ dst, long long ld) {
    pdl_launch_dependents();
    pdl_wait();
    // a warp a row at a time: consecutive lanes, consecutive elements
    const long long warps = (long long)gridDim.x * 8;
    const int lane = threadIdx.x & 31;
    for (long long r = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); r < rows; r += warps) {
        const uint16_t* s = src + r * cols8;
        uint16_t* d = dst + r * ld;
        int c = lane;
        for (; c + 96 < cols; c += 128) {
            const uint16_t a = s[c], b = s[c + 32], e = s[c + 64], f = s[c + 96];
            d[c] = a;
            d[c + 32] = b;
            d[c + 64] = e;
            d[c + 96] = f;
        }
        for (; c < cols; c += 32) d[c] = s[c];
    }
}
// dw [co][ci] from `slices` matrices [co][ci8], in fp64 and their order.
static __global__ void __launch_bounds__(256) lin_weight_unpad_kernel(const float* __restrict__ part, int slices, long long co, int ci, int ci8, float* __restrict__ dw) {
    pdl_launch_dependents();
    pdl_wait();
    const long long n = co * ci, step = (long long)gridDim.x * 256, one = co * ci8;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
        const long long r = i / ci, at = r * ci8 + (i - r * ci);
        double s = 0.0;
        for (int z = 0; z < slices; ++z) s += (double)part[z * one + at];
        dw[i] = (float)s;
    }
}

// ------------------------------------------------------------------------------------------ dz = dy * act'(z)
template <typename T, bool VEC> __global__ void __launch_bounds__(256) lin_act_bwd_kernel(const T* dy, const T* z, T* dz, long long n, int act) {
    pdl_launch_dependents();
    pdl_wait();
    constexpr int V = VEC ? 16 / (int)sizeof(T) : 1;
    const long long nv = n / V, step = (long long)gridDim.x * 256;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < nv; i += step) {
        if constexpr (VEC) {
            const Vec16<T> g = ld16_stream(dy + i * V), x = ld16_stream(z + i * V);
            Vec16<T> o;
#pragma unroll
            for (int j = 0; j < V; ++j) o.v[j] = from_f32<T>(to_f32<T>(g.v[j]) * lin_act_grad(to_f32<T>(x.v[j]), act));
            st16(dz + i * V, o);
        } else {
            dz[i] = from_f32<T>(to_f32<T>(dy[i]) * lin_act_grad(to_f32<T>(z[i]), act));
        }
    }
    if (VEC && blockIdx.x == 0 && threadIdx.x < n - nv * V) {
        const long long i = nv * V + threadIdx.x;
        dz[i] = from_f32<T>(to_f32<T>(dy[i]) * lin_act_grad(to_f32<T>(z[i]), act));
    }
}

}  // namespace nbcbs
