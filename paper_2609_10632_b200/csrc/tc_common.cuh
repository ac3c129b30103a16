// What the tensor-core kernels share: bounded waits on mbarriers, rounding of accumulator pairs, and on the host the driver's
// tensor-map encoders and the shared-memory limit.
#pragma once
#include <cuda.h>

#include <string>

#include "../../include/nb_cbs.h"
#include "common.cuh"
#include "ptx_sm100.cuh"

namespace nbcbs {

__device__ __forceinline__ uint64_t global_timer_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}

// A wait has run out: recorded (the first one wins), and the CTA's other roles stop waiting.
static __device__ __noinline__ void give_up(volatile int* abort_flag, int* status, int site) {
    *abort_flag = 1;
    report_timeout(status, site, (int)blockIdx.x);
}

// Bounded mbarrier wait: gives up after `limit_ns` (or as soon as another role has given up), records the site.
static __device__ __noinline__ bool wait_bar(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int* status, int site, uint64_t limit_ns = kWaitLimitNs) {
    uint64_t t0 = 0;
    for (uint32_t i = 0;; ++i) {
        if (ptx::mbar_try_wait_parked(bar, parity, 4000u)) return true;
        if ((i & 127u) == 127u) {
            if (*abort_flag) return false;
            const uint64_t now = global_timer_ns();
            if (t0 == 0) {
                t0 = now;
            } else if (now - t0 > limit_ns) {
                give_up(abort_flag, status, site);
                return false;
            }
        }
    }
}

// Fast path inline (the barrier is usually complete already), slow bounded path out of line.
// Called by all 32 lanes of a producer or MMA warp; the lanes leave together with the same answer.
__device__ __forceinline__ bool wait_bar_fast(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int* status, int site) {
    bool ok = ptx::mbar_try_wait(bar, parity);
    if (!ok) ok = wait_bar(bar, parity, abort_flag, status, site);
    return __all_sync(0xffffffffu, ok) != 0;
}

template <typename OutT> __device__ __forceinline__ uint32_t pack2(float a, float b, int* sat);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b, int*) {
    __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&v);
}
// fp16 stores saturate to the largest finite value; `sat` collects, per 16-bit half, a flag bit (bit 15 / 31) that is set
// when a stored magnitude is 65504 (0x7bff) or an exceptional pattern above it.
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b, int* sat) {
    uint32_t v;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(v) : "f"(b), "f"(a));
    if (sat) *sat |= (int)((v & 0x7fff7fffu) + 0x04010401u);  // (sat is a compile-time NULL where the caller tracks saturation otherwise)
    return v;
}

// ------------------------------------------------------------------------------------------ host side
namespace tcdetail {

inline std::string& err() {
    static thread_local std::string e;
    return e;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
typedef CUresult (*EncodeIm2colFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const int*, const int*,
                                   cuuint32_t, cuuint32_t, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                   CUtensorMapFloatOOBfill);

struct DriverFns {
    EncodeTiledFn tiled = nullptr;
    EncodeIm2colFn im2col = nullptr;
    DriverFns() {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess)
            tiled = reinterpret_cast<EncodeTiledFn>(f);
        f = nullptr;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeIm2col", &f, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess)
            im2col = reinterpret_cast<EncodeIm2colFn>(f);
    }
};
inline DriverFns& driver() {
    static DriverFns d;  // (looked up once, by the first caller)
    return d;
}

constexpr size_t kMaxSmem = 232448;  // 227 KB opt-in limit per CTA

}  // namespace tcdetail
}  // namespace nbcbs
