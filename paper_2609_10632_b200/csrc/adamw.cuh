// Fused AdamW step over a list of tensors (see include/nb_adamw.h for the arithmetic): a kernel that sums the squares of all
// gradients and prepares the step's scalars, and one that clips and updates.  As in the SGD step the elements of all tensors
// are cut into chunks, chunk i belongs to block i % gridDim.x, and both kernels walk the same table.
#pragma once
#include <cuda_fp8.h>
#include <stddef.h>

#include "../../include/nb_adamw.h"
#include "common.cuh"

namespace nbcbs {

constexpr int AW_THREADS = 256;
constexpr int AW_VPT = 2;                          // groups of four elements per thread and chunk
constexpr int AW_CHUNK = 4 * AW_VPT * AW_THREADS;  // elements per chunk: whole blocks of the 8-bit form
constexpr int AW_AHEAD = 4;                        // chunks that a block of the norm kernel has in flight
constexpr int AW_BLOCKS_PER_SM = 4;                  // blocks of the norm kernel and of the update kernel that an SM holds
constexpr int AW_MAX_BLOCKS = 2048;
static_assert(AW_CHUNK * 2 == AW_THREADS * 16 && AW_CHUNK % NB_ADAMW_BLOCK == 0 && NB_ADAMW_BLOCK == 128, "a warp holds one block of the 8-bit form in four elements a lane");

struct __align__(64) AwChunk {  // everything a block needs to know about a chunk: addresses of its first element
    const void* grad;
    float* param;
    void* exp_avg;
    void* exp_avg_sq;
    float* exp_avg_scale;
    float* exp_avg_sq_scale;
    void* copy;
    uint16_t len;         // elements (<= AW_CHUNK)
    uint8_t group, grad_dtype, copy_dtype, reserved[3];
};
static_assert(sizeof(AwChunk) == 64, "four 16-byte copies");
struct AwHeader {  // at the start of the workspace
    int32_t nchunks, grid;
    int32_t eight, reserved;  // the first `eight` chunks are those of moments in 8 bits
    uint64_t off_chunks, off_partials, total_bytes;
};
struct AwStep {  // what the norm kernel leaves for the update kernel, behind the header
    int64_t t;           // number of this step, from 1
    float loss_scale;    // 1 without a scaler
    float inv_bc1;       // 1 / (1 - beta1^t)
    float inv_root_bc2;  // 1 / sqrt(1 - beta2^t)
    int32_t first;       // t == 1: the moments hold nothing yet
};
constexpr int AW_STEP_AT = 128;  // byte offset of AwStep

struct AwScalars {
    float eps, max_norm;
    float lr[NB_SGD_GROUPS], keep[NB_SGD_GROUPS];  // keep = 1 - lr*weight_decay
    float b1, c1, b2, c2;                          // beta1, 1-beta1, beta2, 1-beta2, each rounded once
    int64_t* step;
    nb_loss_scaler* scaler;
    float growth_factor, backoff_factor, floor_scale;
    int growth_interval;
};

// Four consecutive elements as fp32, zeros past `left` elements (left >= 4: one vector load).
__device__ __forceinline__ float4 aw_ld4_f32(const float* p, int left) {
    if (left >= 4) return *reinterpret_cast<const float4*>(p);
    return make_float4(left > 0 ? p[0] : 0.f, left > 1 ? p[1] : 0.f, left > 2 ? p[2] : 0.f, 0.f);
}
__device__ __forceinline__ float4 aw_ld4_f32_stream(const float* p, int left) {
    if (left >= 4) return __ldcs(reinterpret_cast<const float4*>(p));
    return aw_ld4_f32(p, left);
}
__device__ __forceinline__ uint2 aw_ld4_16(const void* base, int at, int left) {
    const uint16_t* p = static_cast<const uint16_t*>(base) + at;
    if (left >= 4) return *reinterpret_cast<const uint2*>(p);
    uint2 r = make_uint2(0u, 0u);
    if (left > 0) r.x = p[0];
    if (left > 1) r.x |= (uint32_t)p[1] << 16;
    if (left > 2) r.y = p[2];
    return r;
}
__device__ __forceinline__ uint32_t aw_ld4_8(const void* base, int at, int left) {
    const uint8_t* p = static_cast<const uint8_t*>(base) + at;
    if (left >= 4) return __ldcs(reinterpret_cast<const uint32_t*>(p));
    uint32_t r = 0;
    if (left > 0) r = p[0];
    if (left > 1) r |= (uint32_t)p[1] << 8;
    if (left > 2) r |= (uint32_t)p[2] << 16;
    return r;
}
// A gradient's four elements as they lie in memory (two words when they are 16 bits wide), and what they stand for.
__device__ __forceinline__ uint4 aw_ld4_grad(const void* base, int at, int left, int dtype) {
    if (dtype == NB_DTYPE_F32) {
        const float4 f = aw_ld4_f32(static_cast<const float*>(base) + at, left);
        return make_uint4(__float_as_uint(f.x), __float_as_uint(f.y), __float_as_uint(f.z), __float_as_uint(f.w));
    }
    const uint2 h = aw_ld4_16(base, at, left);
    return make_uint4(h.x, h.y, 0u, 0u);
}
__device__ __forceinline__ float4 aw_grad_f32(uint4 r, int dtype) {
    if (dtype == NB_DTYPE_F32) return make_float4(__uint_as_float(r.x), __uint_as_float(r.y), __uint_as_float(r.z), __uint_as_float(r.w));
    if (dtype == NB_DTYPE_BF16) return make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u), __uint_as_float(r.y << 16), __uint_as_float(r.y & 0xffff0000u));
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&r.x)), b = __half22float2(*reinterpret_cast<const __half2*>(&r.y));
    return make_float4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ float4 aw_e4m3_f32(uint32_t q) {
    const __half2_raw a = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(q & 0xffffu), __NV_E4M3);
    const __half2_raw b = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(q >> 16), __NV_E4M3);
    const float2 fa = __half22float2(__half2(a)), fb = __half22float2(__half2(b));
    return make_float4(fa.x, fa.y, fb.x, fb.y);
}
__device__ __forceinline__ uint32_t aw_f32_e4m3(float4 v) {
    const uint32_t a = __nv_cvt_float2_to_fp8x2(make_float2(v.x, v.y), __NV_SATFINITE, __NV_E4M3);
    const uint32_t b = __nv_cvt_float2_to_fp8x2(make_float2(v.z, v.w), __NV_SATFINITE, __NV_E4M3);
    return a | (b << 16);
}

__device__ __forceinline__ double aw_block_sum(double v, double* red /*[AW_THREADS/32]*/) {  // fixed order; valid in thread 0
    for (int o = 16; o > 0; o >>= 1) v += __shfl_down_sync(0xffffffffu, v, o);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) red[warp] = v;
    __syncthreads();
    double t = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < AW_THREADS / 32; ++w) t += red[w];
    return t;
}

__device__ __forceinline__ double aw_sq4(float4 g, double s) {
    s = fma((double)g.x, (double)g.x, s);
    s = fma((double)g.y, (double)g.y, s);
    s = fma((double)g.z, (double)g.z, s);
    return fma((double)g.w, (double)g.w, s);
}

// partials[b] = sum of g^2 over the chunks of block b, in fp64 throughout, so that the clip coefficient is the fp32 number nearest to
// the true one whatever the order of the sum (with fp32 sums of eight squares 2 of 60 gradient lists had another).  Block 0
// also derives the step's scalars from the count of steps.  want_norm = 0 (one block): the scalars only.
__global__ void __launch_bounds__(AW_THREADS, AW_BLOCKS_PER_SM) adamw_norm_kernel(uint8_t* __restrict__ ws, AwScalars hs, double beta1, double beta2, int want_norm) {
    pdl_launch_dependents();
    pdl_wait();
    if (blockIdx.x == 0 && threadIdx.x == AW_THREADS - 1) {
        AwStep s;
        s.t = *hs.step + 1;
        s.loss_scale = hs.scaler ? hs.scaler->scale : 1.f;
        s.inv_bc1 = (float)(1.0 / (1.0 - pow(beta1, (double)s.t)));
        s.inv_root_bc2 = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)s.t)));
        s.first = s.t == 1;
        *reinterpret_cast<AwStep*>(ws + AW_STEP_AT) = s;
    }
    if (!want_norm) return;
    const AwHeader& H = *reinterpret_cast<const AwHeader*>(ws);
    const AwChunk* C = reinterpret_cast<const AwChunk*>(ws + H.off_chunks);
    __shared__ double red[AW_THREADS / 32];
    double acc = 0.0, acc2 = 0.0;
    const int grid = (int)gridDim.x;
    const uint4* src[AW_AHEAD];
    uint32_t meta[AW_AHEAD];  // elements, type << 16
    auto records = [&](int c0) {  // (those of the next round travel behind this one's data)
#pragma unroll
        for (int j = 0; j < AW_AHEAD; ++j) {
            const int c = c0 + j * grid;
            src[j] = c < H.nchunks ? static_cast<const uint4*>(C[c].grad) + threadIdx.x : nullptr;
            meta[j] = c < H.nchunks ? (uint32_t)C[c].len | ((uint32_t)C[c].grad_dtype << 16) : 0u;
        }
    };
    records(blockIdx.x);
    for (int c0 = blockIdx.x; c0 < H.nchunks; c0 += AW_AHEAD * grid) {
        uint4 r[AW_AHEAD][2];  // a full chunk is one 16-byte vector a thread, two of fp32 gradients
        uint32_t was[AW_AHEAD];
        const uint4* from[AW_AHEAD];
#pragma unroll
        for (int j = 0; j < AW_AHEAD; ++j) {
            was[j] = meta[j];
            from[j] = src[j];
            const bool full = (meta[j] & 0xffffu) == AW_CHUNK;
            r[j][0] = full ? src[j][0] : make_uint4(0u, 0u, 0u, 0u);
            r[j][1] = full && meta[j] >> 16 == NB_DTYPE_F32 ? src[j][AW_THREADS] : make_uint4(0u, 0u, 0u, 0u);
        }
        records(c0 + AW_AHEAD * grid);
#pragma unroll
        for (int j = 0; j < AW_AHEAD; ++j) {
            const int dtype = (int)(was[j] >> 16), len = (int)(was[j] & 0xffffu);
            if (len == AW_CHUNK) {
                const uint4 second = dtype == NB_DTYPE_F32 ? r[j][1] : make_uint4(r[j][0].z, r[j][0].w, 0u, 0u);
                acc = aw_sq4(aw_grad_f32(r[j][0], dtype), acc);
                acc2 = aw_sq4(aw_grad_f32(second, dtype), acc2);
            } else if (len) {
#pragma unroll
                for (int k = 0; k < AW_VPT; ++k) {
                    const int i = 4 * (threadIdx.x + k * AW_THREADS);
                    acc = aw_sq4(aw_grad_f32(aw_ld4_grad(from[j] - threadIdx.x, i, len - i, dtype), dtype), acc);
                }
            }
        }
    }
    const double t = aw_block_sum(acc + acc2, red);
    if (threadIdx.x == 0) reinterpret_cast<double*>(ws + H.off_partials)[blockIdx.x] = t;
}

// sqrt(v) of two non-negative numbers: the hardware's approximate 1/sqrt, then one step of Newton's method on the residual
// v - r*r, which a fused multiply-add gives without rounding error.  1/sqrt is cut to 2^63, so that zero comes out as zero.  Not for a v
// between 0 and 2^-126, which the approximation takes for zero, nor for inf.
__device__ __forceinline__ float2 aw_root(float2 v) {
    float2 y, e;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(v.x));
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(v.y));
    y.x = fminf(y.x, 9.223372e18f);
    y.y = fminf(y.y, 9.223372e18f);
    const float2 r = mul2(v, y);
    e.x = fmaf(-r.x, r.x, v.x);
    e.y = fmaf(-r.y, r.y, v.y);
    return fma2(mul2(e, splat2(0.5f)), y, r);
}

// The update of such a v, over the whole range of fp32: approximations of 2^-23 that take subnormal numbers, zero and inf as they are.
__device__ __forceinline__ float aw_careful(float m, float v, float& root, float step_size, float inv_root_bc2, float eps) {
    float q;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(root) : "f"(v));
    asm("div.full.f32 %0, %1, %2;" : "=f"(q) : "f"(m * -step_size), "f"(fmaf(root, inv_root_bc2, eps)));
    return q;
}
__device__ __forceinline__ bool aw_not_normal(float v) { return __float_as_uint(v) - 0x00800000u >= 0x7f000000u; }

// Two elements: the moments in place (each operation rounded by itself), the new parameters returned.
__device__ __forceinline__ float2 aw_two(float2 g, float2 p, float2& m, float2& v, float2& root, float coef, float step_size, float inv_root_bc2, float keep, const AwScalars& hs) {
    g = mul2(g, splat2(coef));
    const float2 ma = mul2(splat2(hs.b1), m), mb = mul2(splat2(hs.c1), g), va = mul2(splat2(hs.b2), v), vb = mul2(mul2(splat2(hs.c2), g), g);
    // (a packed addition would be fused with the packed products in front of it: measured, a quarter of the sums had other bits)
    m = make_float2(__fadd_rn(ma.x, mb.x), __fadd_rn(ma.y, mb.y));
    v = make_float2(__fadd_rn(va.x, vb.x), __fadd_rn(va.y, vb.y));
    root = aw_root(v);
    const float2 den = fma2(root, splat2(inv_root_bc2), splat2(hs.eps));
    float2 rec;  // (within 2^-22, which moves a parameter by 2^-22 of one step)
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(rec.x) : "f"(den.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(rec.y) : "f"(den.y));
    // A v that is not a normal number (zero, underflown, overflown to inf, NaN) takes another way: the root's tricks do not cover it,
    // and with a tiny eps neither the reciprocal's.  With inf the update is m / inf = 0.
    float2 update = mul2(mul2(m, splat2(-step_size)), rec);
    if (aw_not_normal(v.x)) update.x = aw_careful(m.x, v.x, root.x, step_size, inv_root_bc2, hs.eps);
    if (aw_not_normal(v.y)) update.y = aw_careful(m.y, v.y, root.y, step_size, inv_root_bc2, hs.eps);
    return fma2(p, splat2(keep), update);
}

__device__ __forceinline__ float aw_max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float aw_warp_max(float4 x) {
    // (bits of non-negative floats order like the floats, with inf and NaN above all)
    const float a = aw_max_nan(aw_max_nan(fabsf(x.x), fabsf(x.y)), aw_max_nan(fabsf(x.z), fabsf(x.w)));
    return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(a)));
}
__device__ __forceinline__ uint32_t aw_times_e4m3(float4 x, float up) {
    const float2 q0 = mul2(make_float2(x.x, x.y), splat2(up)), q1 = mul2(make_float2(x.z, x.w), splat2(up));
    return aw_f32_e4m3(make_float4(q0.x, q0.y, q1.x, q1.y));
}
// Codes of the 128 first moments and of the 128 roots that a warp holds (four each a lane).  `scale` is that of the first moments
// in lanes 0-15 and that of the roots in lanes 16-31: each half of the warp takes one reciprocal for both.
__device__ __forceinline__ void aw_encode(float4 m, float4 r, uint32_t& mc, uint32_t& vc, float& scale) {
    const float mm = aw_warp_max(m), mr = aw_warp_max(r);
    const float most = (threadIdx.x & 16) ? mr : mm;
    const bool none = most < 7.888609e-31f;  // 2^-100
    const float up = none ? 0.f : __fmul_rn(__frcp_rn(most), 448.f);
    scale = none ? 0.f : __fmul_rn(most, 1.f / 448.f);
    const float up_r = __shfl_sync(0xffffffffu, up, 16);
    mc = aw_times_e4m3(m, __shfl_sync(0xffffffffu, up, 0));
    vc = aw_times_e4m3(r, up_r);
    if (((vc - 0x01010101u) & ~vc & 0x80808080u) && up_r != 0.f) {  // a zero byte: the smallest code where the root is not zero
        if (!(vc & 0x000000ffu) && r.x > 0.f) vc |= 0x00000001u;
        if (!(vc & 0x0000ff00u) && r.y > 0.f) vc |= 0x00000100u;
        if (!(vc & 0x00ff0000u) && r.z > 0.f) vc |= 0x00010000u;
        if (!(vc & 0xff000000u) && r.w > 0.f) vc |= 0x01000000u;
    }
}

// Four elements as they lie in memory: gradient, parameters, moments (8 bits: codes and scale).
template <bool EIGHT> struct AwRaw;
template <> struct AwRaw<false> {
    uint4 g;
    float4 p, m, v;
};
template <> struct AwRaw<true> {
    uint4 g;
    float4 p;
    uint32_t m, v;
    float ms, vs;
};
// FULL: the chunk has AW_CHUNK elements, nothing is guarded.
template <bool FULL> __device__ __forceinline__ void aw_load(const AwChunk& t, int i, bool first, AwRaw<false>& r) {
    const int left = FULL ? 4 : t.len - i;
    r.g = aw_ld4_grad(t.grad, i, left, t.grad_dtype);
    r.p = aw_ld4_f32_stream(t.param + i, left);
    r.m = r.v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (first) return;
    r.m = aw_ld4_f32_stream(static_cast<const float*>(t.exp_avg) + i, left);
    r.v = aw_ld4_f32_stream(static_cast<const float*>(t.exp_avg_sq) + i, left);
}
template <bool FULL> __device__ __forceinline__ void aw_load(const AwChunk& t, int i, bool first, AwRaw<true>& r) {
    const int left = FULL ? 4 : t.len - i;
    r.g = aw_ld4_grad(t.grad, i, left, t.grad_dtype);
    r.p = aw_ld4_f32_stream(t.param + i, left);
    r.m = r.v = 0u;
    r.ms = r.vs = 0.f;
    if (first || left <= 0) return;
    r.m = aw_ld4_8(t.exp_avg, i, left);
    r.v = aw_ld4_8(t.exp_avg_sq, i, left);
    r.ms = t.exp_avg_scale[i / NB_ADAMW_BLOCK];  // (one address per warp)
    r.vs = t.exp_avg_sq_scale[i / NB_ADAMW_BLOCK];
}
__device__ __forceinline__ void aw_moments(const AwRaw<false>& r, float2& m0, float2& m1, float2& v0, float2& v1) {
    m0 = make_float2(r.m.x, r.m.y);
    m1 = make_float2(r.m.z, r.m.w);
    v0 = make_float2(r.v.x, r.v.y);
    v1 = make_float2(r.v.z, r.v.w);
}
__device__ __forceinline__ void aw_moments(const AwRaw<true>& r, float2& m0, float2& m1, float2& v0, float2& v1) {
    const float4 mq = aw_e4m3_f32(r.m), vq = aw_e4m3_f32(r.v);
    const float2 sm = splat2(r.ms), sv = splat2(r.vs);
    m0 = mul2(make_float2(mq.x, mq.y), sm);
    m1 = mul2(make_float2(mq.z, mq.w), sm);
    v0 = mul2(make_float2(vq.x, vq.y), sv);
    v1 = mul2(make_float2(vq.z, vq.w), sv);
    v0 = mul2(v0, v0);
    v1 = mul2(v1, v1);
}

// What a thread's four elements become.
template <bool EIGHT> struct AwNew;
template <> struct AwNew<false> {
    float2 p0, p1, m0, m1, v0, v1;
};
template <> struct AwNew<true> {
    float2 p0, p1;
    uint32_t m, v;
    float scale;
};
template <bool EIGHT>
__device__ __forceinline__ AwNew<EIGHT> aw_update(const AwRaw<EIGHT>& raw, int grad_dtype, float coef, float step_size, float inv_root_bc2, float keep, const AwScalars& hs) {
    AwNew<EIGHT> o;
    float2 m0, m1, v0, v1, r0, r1;
    aw_moments(raw, m0, m1, v0, v1);
    const float4 g = aw_grad_f32(raw.g, grad_dtype);
    o.p0 = aw_two(make_float2(g.x, g.y), make_float2(raw.p.x, raw.p.y), m0, v0, r0, coef, step_size, inv_root_bc2, keep, hs);
    o.p1 = aw_two(make_float2(g.z, g.w), make_float2(raw.p.z, raw.p.w), m1, v1, r1, coef, step_size, inv_root_bc2, keep, hs);
    if constexpr (EIGHT) {  // (the whole warp takes part; what lies past the end is zero, which changes no maximum)
        aw_encode(make_float4(m0.x, m0.y, m1.x, m1.y), make_float4(r0.x, r0.y, r1.x, r1.y), o.m, o.v, o.scale);
    } else {
        o.m0 = m0;
        o.m1 = m1;
        o.v0 = v0;
        o.v1 = v1;
    }
    return o;
}

template <bool EIGHT, bool FULL> __device__ __forceinline__ void aw_store(const AwChunk& t, int i, const AwNew<EIGHT>& o) {
    const int left = FULL ? 4 : t.len - i;
    if constexpr (EIGHT) {
        // (lanes 0 and 16; the block has a first element)
        if ((threadIdx.x & 15) == 0 && (FULL || (i & ~(NB_ADAMW_BLOCK - 1)) < t.len))
            ((threadIdx.x & 16) ? t.exp_avg_sq_scale : t.exp_avg_scale)[i / NB_ADAMW_BLOCK] = o.scale;
    }
    if (left <= 0) return;
    uint16_t* copy = static_cast<uint16_t*>(t.copy);
    uint2 lo = make_uint2(0u, 0u);
    if (copy) {
        if (t.copy_dtype == NB_DTYPE_F16) {
            __half h[4];
            pair_from_f32(h, o.p0);
            pair_from_f32(h + 2, o.p1);
            lo = make_uint2(*reinterpret_cast<const uint32_t*>(h), *reinterpret_cast<const uint32_t*>(h + 2));
        } else {
            __nv_bfloat16 h[4];
            pair_from_f32(h, o.p0);
            pair_from_f32(h + 2, o.p1);
            lo = make_uint2(*reinterpret_cast<const uint32_t*>(h), *reinterpret_cast<const uint32_t*>(h + 2));
        }
    }
    if (left >= 4) {
        __stcs(reinterpret_cast<float4*>(t.param + i), make_float4(o.p0.x, o.p0.y, o.p1.x, o.p1.y));
        if constexpr (EIGHT) {
            __stcs(reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.exp_avg) + i), o.m);
            __stcs(reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.exp_avg_sq) + i), o.v);
        } else {
            __stcs(reinterpret_cast<float4*>(static_cast<float*>(t.exp_avg) + i), make_float4(o.m0.x, o.m0.y, o.m1.x, o.m1.y));
            __stcs(reinterpret_cast<float4*>(static_cast<float*>(t.exp_avg_sq) + i), make_float4(o.v0.x, o.v0.y, o.v1.x, o.v1.y));
        }
        if (copy) *reinterpret_cast<uint2*>(copy + i) = lo;
    } else {
        const float pe[3] = {o.p0.x, o.p0.y, o.p1.x};
#pragma unroll
        for (int e = 0; e < 3; ++e) {
            if (e >= left) break;
            t.param[i + e] = pe[e];
            if constexpr (EIGHT) {
                static_cast<uint8_t*>(t.exp_avg)[i + e] = (uint8_t)(o.m >> (8 * e));
                static_cast<uint8_t*>(t.exp_avg_sq)[i + e] = (uint8_t)(o.v >> (8 * e));
            } else {
                static_cast<float*>(t.exp_avg)[i + e] = e == 0 ? o.m0.x : e == 1 ? o.m0.y : o.m1.x;
                static_cast<float*>(t.exp_avg_sq)[i + e] = e == 0 ? o.v0.x : e == 1 ? o.v0.y : o.v1.x;
            }
            if (copy) copy[i + e] = (uint16_t)((e < 2 ? lo.x : lo.y) >> (16 * (e & 1)));
        }
    }
}

struct AwGroup {  // a group's scalars, picked by selects so that they stay in the parameter bank
    float step_size, keep;
    __device__ __forceinline__ AwGroup(int grp, const AwScalars& hs, const AwStep& S) {
        step_size = (grp == 0 ? hs.lr[0] : grp == 1 ? hs.lr[1] : hs.lr[2]) * S.inv_bc1;
        keep = grp == 0 ? hs.keep[0] : grp == 1 ? hs.keep[1] : hs.keep[2];
    }
};
__device__ __forceinline__ void aw_copy16(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void aw_copy4(uint32_t dst, const void* src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void aw_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void aw_arrived() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
    __syncwarp();
}

// A block's share of the chunks of 32-bit moments, last first.  14.2 million parameters in 83 us with the norm kernel (426 MB without the
// gradients' second reading, 65 us at the copy rate).  The next chunk's record travels behind this one's data, into a slot
// of each warp's own.
__device__ __forceinline__ void aw_walk32(const AwChunk* C, int from, int to, bool first, float coef, const AwStep& S, const AwScalars& hs) {
    __shared__ AwChunk slots[AW_THREADS / 32][2];
    AwChunk* slot = slots[threadIdx.x >> 5];
    const int lane = threadIdx.x & 31, grid = (int)gridDim.x;
    auto fetch = [&](int c, int s) {
        if (lane < 4 && c >= from) aw_copy16((uint32_t)__cvta_generic_to_shared(slot + s) + 16u * lane, reinterpret_cast<const char*>(C + c) + 16 * lane);
        aw_commit();
    };
    int c = to - 1 - (int)blockIdx.x, s = 0;
    if (c < from) return;
    fetch(c, 0);
    for (; c >= from; c -= grid) {
        aw_arrived<0>();  // (and every lane is done with the slot that is fetched into now)
        fetch(c - grid, s ^ 1);
        const AwChunk& ch = slot[s];
        s ^= 1;
        const bool full = ch.len == AW_CHUNK;
        AwRaw<false> raw[AW_VPT];
#pragma unroll
        for (int k = 0; k < AW_VPT; ++k) {
            const int i = 4 * (threadIdx.x + k * AW_THREADS);
            if (full) aw_load<true>(ch, i, first, raw[k]); else aw_load<false>(ch, i, first, raw[k]);
        }
        const AwGroup grp(ch.group, hs, S);
#pragma unroll
        for (int k = 0; k < AW_VPT; ++k) {
            const int i = 4 * (threadIdx.x + k * AW_THREADS);
            const AwNew<false> o = aw_update<false>(raw[k], ch.grad_dtype, coef, grp.step_size, S.inv_root_bc2, grp.keep, hs);
            if (full) aw_store<false, true>(ch, i, o); else aw_store<false, false>(ch, i, o);
        }
    }
    aw_arrived<0>();
}

// The chunks of 8-bit moments: a warp owns 256 consecutive elements of a chunk (two blocks of 128) and a ring in shared memory of
// its own, into which its share of the two chunks behind the current one travels by asynchronous copies.  Here the arithmetic
// takes nearly as many issue slots as the bytes take time, so loads and arithmetic have to overlap.  100.7 million parameters with bf16
// gradients, clipped (floor 248 us for 1.62 GB): 507 us with a thread's loads in front of its arithmetic, 432 without guards on full chunks,
// 400 with the ring, 390 with the two blocks' arithmetic interleaved, 384 with the norm kernel's next records on their way.
// Now 325 us here (16 bytes a parameter: 5.0 TB/s, 60 % of the issue slots) and 52 in the norm kernel (3.9 TB/s).
constexpr int AW_STAGES = 3, AW_RECORDS = 8;
// A stage of a warp's ring: 256 parameters, codes of both moments, their four scales, gradients.
constexpr int AW_AT_M = 1024, AW_AT_SCALE = AW_AT_M + 512, AW_AT_G = AW_AT_SCALE + 16;
constexpr int aw_stage_bytes(bool grads_f32) { return AW_AT_G + (grads_f32 ? 1024 : 512); }
constexpr int aw_ring_bytes(bool grads_f32) { return AW_THREADS / 32 * (AW_RECORDS * (int)sizeof(AwChunk) + AW_STAGES * aw_stage_bytes(grads_f32)); }
static_assert(AW_CHUNK == 256 * (AW_THREADS / 32) && AW_VPT == 2, "every warp has 256 elements of a chunk");

__device__ __forceinline__ void aw_walk8(const AwChunk* C, int to, uint8_t* smem, int stage_bytes, bool first, float coef, const AwStep& S, const AwScalars& hs) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grid = (int)gridDim.x;
    AwChunk* rec = reinterpret_cast<AwChunk*>(smem) + warp * AW_RECORDS;
    uint8_t* ring = smem + AW_THREADS / 32 * AW_RECORDS * sizeof(AwChunk) + warp * AW_STAGES * stage_bytes;
    const int base = 256 * warp;  // this warp's first element inside a chunk
    auto record = [&](int c, int n) {
        if (lane < 4 && c >= 0) aw_copy16((uint32_t)__cvta_generic_to_shared(rec + (n & (AW_RECORDS - 1))) + 16u * lane, reinterpret_cast<const char*>(C + c) + 16 * lane);
    };
    auto data = [&](int c, int n, int st) {  // (its record has arrived)
        if (c < 0) return;
        const AwChunk& ch = rec[n & (AW_RECORDS - 1)];
        if (ch.len != AW_CHUNK) return;  // a ragged chunk is loaded where it is updated
        const uint32_t d = (uint32_t)__cvta_generic_to_shared(ring) + (uint32_t)(st * stage_bytes) + 16u * lane;
        const char* p = reinterpret_cast<const char*>(ch.param + base) + 16 * lane;
        aw_copy16(d, p);
        aw_copy16(d + 512u, p + 512);
        if (ch.grad_dtype == NB_DTYPE_F32) {
            const char* g = static_cast<const char*>(ch.grad) + 4 * base + 16 * lane;
            aw_copy16(d + AW_AT_G, g);
            aw_copy16(d + AW_AT_G + 512u, g + 512);
        } else {
            aw_copy16(d + AW_AT_G, static_cast<const char*>(ch.grad) + 2 * base + 16 * lane);
        }
        if (first) return;
        aw_copy16(d + AW_AT_M, static_cast<const char*>(lane < 16 ? ch.exp_avg : ch.exp_avg_sq) + base + 16 * (lane & 15));  // (v lies behind m)
        if (lane < 4) aw_copy4(d + AW_AT_SCALE - 12u * lane, (lane < 2 ? ch.exp_avg_scale : ch.exp_avg_sq_scale) + base / NB_ADAMW_BLOCK + (lane & 1));
    };
    const int c0 = to - 1 - (int)blockIdx.x;
    if (c0 < 0) return;
    // groups of copies, one a round: that of round n brings the data of chunk n + 2 and the record of chunk n + 4
    for (int n = 0; n < 4; ++n) record(c0 - n * grid, n);
    aw_commit();
    aw_arrived<0>();
    data(c0, 0, 0);
    aw_commit();
    data(c0 - grid, 1, 1);
    aw_commit();
    int st = 0;
    for (int n = 0, c = c0; c >= 0; ++n, c -= grid) {
        aw_arrived<1>();  // (and every lane is done with the stage of the round before)
        data(c - 2 * grid, n + 2, st == 0 ? 2 : st - 1);
        record(c - 4 * grid, n + 4);
        aw_commit();
        const AwChunk ch = rec[n & (AW_RECORDS - 1)];  // (in registers: the stores below could alias it)
        const uint8_t* T = ring + st * stage_bytes;
        const AwGroup grp(ch.group, hs, S);
        const bool full = ch.len == AW_CHUNK;
        AwRaw<true> raw[AW_VPT];
#pragma unroll
        for (int k = 0; k < AW_VPT; ++k) {
            const int e = 128 * k + 4 * lane;
            if (full) {
                raw[k].p = *reinterpret_cast<const float4*>(T + 4 * e);
                if (ch.grad_dtype == NB_DTYPE_F32) {
                    raw[k].g = *reinterpret_cast<const uint4*>(T + AW_AT_G + 4 * e);
                } else {
                    const uint2 h = *reinterpret_cast<const uint2*>(T + AW_AT_G + 2 * e);
                    raw[k].g = make_uint4(h.x, h.y, 0u, 0u);
                }
                raw[k].m = raw[k].v = 0u;
                raw[k].ms = raw[k].vs = 0.f;
                if (!first) {
                    raw[k].m = *reinterpret_cast<const uint32_t*>(T + AW_AT_M + e);
                    raw[k].v = *reinterpret_cast<const uint32_t*>(T + AW_AT_M + 256 + e);
                    raw[k].ms = *reinterpret_cast<const float*>(T + AW_AT_SCALE + 4 * k);
                    raw[k].vs = *reinterpret_cast<const float*>(T + AW_AT_SCALE + 8 + 4 * k);
                }
            } else {
                aw_load<false>(ch, base + e, first, raw[k]);
            }
        }
        AwNew<true> o[AW_VPT];
#pragma unroll
        for (int k = 0; k < AW_VPT; ++k) o[k] = aw_update<true>(raw[k], ch.grad_dtype, coef, grp.step_size, S.inv_root_bc2, grp.keep, hs);
#pragma unroll
        for (int k = 0; k < AW_VPT; ++k) {
            const int i = base + 128 * k + 4 * lane;
            if (full) aw_store<true, true>(ch, i, o[k]); else aw_store<true, false>(ch, i, o[k]);
        }
        st = st == AW_STAGES - 1 ? 0 : st + 1;
    }
    aw_arrived<0>();
}

// Bound: memory.  Chunks are taken last first, because the end of the gradients is what the norm kernel has left in L2;
// parameters and moments pass through L2 as streams.  EIGHT: the chunks of 8-bit moments, else those of 32-bit ones; a list that
// has both takes two launches, of which the one with `leader` writes what the step leaves for its caller.
template <bool EIGHT>
__global__ void __launch_bounds__(AW_THREADS, AW_BLOCKS_PER_SM) adamw_update_kernel(uint8_t* __restrict__ ws, AwScalars hs, int want_norm, float* __restrict__ total_norm_out, int leader, int stage_bytes) {
    pdl_launch_dependents();
    pdl_wait();
    const AwHeader& H = *reinterpret_cast<const AwHeader*>(ws);
    const AwChunk* C = reinterpret_cast<const AwChunk*>(ws + H.off_chunks);
    const AwStep S = *reinterpret_cast<const AwStep*>(ws + AW_STEP_AT);
    __shared__ double red[AW_THREADS / 32];
    __shared__ float s_coef;
    __shared__ int s_skip;
    double t = 0.0;
    if (want_norm) {  // every block adds the norm kernel's partial sums itself, in one fixed order
        const double* partials = reinterpret_cast<const double*>(ws + H.off_partials);
        double acc = 0.0;
        for (int i = threadIdx.x; i < H.grid; i += AW_THREADS) acc += partials[i];
        t = aw_block_sum(acc, red);
    }
    if (threadIdx.x == 0) {
        const double inv = hs.scaler ? 1.0 / (double)S.loss_scale : 1.0;
        const double total = sqrt(t) * inv;  // inf or NaN if any gradient element is
        double c = 1.0;
        if (hs.max_norm > 0.f && hs.max_norm < __int_as_float(0x7f800000)) {
            c = (double)hs.max_norm / (total + 1e-6);
            c = c > 1.0 ? 1.0 : c;  // (a NaN norm stays NaN: no tensor takes an unclipped step)
        }
        const bool skip = hs.scaler && !isfinite(t);
        s_coef = (float)(c * inv);
        s_skip = skip;
        if (blockIdx.x == 0 && leader) {  // (no block of either launch reads what is written here)
            if (total_norm_out) *total_norm_out = (float)total;
            if (!skip) *hs.step = S.t;
            if (hs.scaler) {
                nb_loss_scaler s = *hs.scaler;
                if (skip) {
                    s.scale = fmaxf(s.scale * hs.backoff_factor, hs.floor_scale);
                    s.growth_tracker = 0;
                } else if (++s.growth_tracker >= hs.growth_interval) {
                    s.scale *= hs.growth_factor;
                    s.growth_tracker = 0;
                }
                hs.scaler->scale = s.scale;
                hs.scaler->growth_tracker = s.growth_tracker;
                hs.scaler->skipped = skip ? 1 : 0;
            }
        }
    }
    __syncthreads();
    if (s_skip) return;
    const float coef = s_coef;
    const bool first = S.first != 0;
    extern __shared__ __align__(64) uint8_t aw_smem[];
    if (EIGHT) aw_walk8(C, H.eight, aw_smem, stage_bytes, first, coef, S, hs);
    else aw_walk32(C, H.eight, H.nchunks, first, coef, S, hs);
}

}  // namespace nbcbs
