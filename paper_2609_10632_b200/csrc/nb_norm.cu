// C ABI of the layer norm (see include/nb_norm.h).  Everything runs on the current device; no memory is allocated.
#include <algorithm>
#include <atomic>
#include <cstring>

#include "../../include/nb_norm.h"
#include "api_common.cuh"
#include "norm.cuh"

using namespace nbcbs;
using namespace nbapi;

namespace {

int sm_count() {
    int dev = 0, sms = 148;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    return std::max(sms, 1);
}

bool known(int32_t dtype) { return dtype == NB_DTYPE_F32 || dtype == NB_DTYPE_BF16 || dtype == NB_DTYPE_F16; }
size_t size_of(int32_t dtype) { return dtype == NB_DTYPE_F32 ? 4 : 2; }

// The group that holds a row of `nvec` vectors: `lanes` of a warp, or a block of `threads` (lanes = 0), each with `vpl` vectors.
struct Group {
    int lanes, vpl, threads;
};
// Least idle lanes; among equals the smaller group with more vectors a lane (fewer steps of the reductions) or, `wide`, the larger
// (fewer registers a thread, more blocks an SM: the backward pass over 409600 x 96 bf16 64 -> 60 us).  `most` vectors a lane.
Group choose_group(int nvec, int most, bool wide) {
    Group best = {0, 0, 0};
    int waste = 1 << 30;
    for (int lanes = 4; lanes <= 32; lanes *= 2)
        for (int vpl = 1; vpl <= most; ++vpl)
            if (lanes * vpl >= nvec && lanes * vpl - nvec < waste + (wide ? 1 : 0)) {
                waste = lanes * vpl - nvec;
                best = {lanes, vpl, LN_THREADS};
            }
    if (best.lanes) return best;
    const int threads = [&](int vpl) { return ((nvec + vpl - 1) / vpl + 31) / 32 * 32; }(most);
    return {0, most, threads};
}

unsigned blocks_for(long long rows, int per_block) { return (unsigned)std::min<long long>((rows + per_block - 1) / per_block, 0x7fffffffLL); }

template <typename T, int V, int VPL> void launch_fwd_lanes(const Group& G, const LnFwd& P, cudaStream_t st) {
    const unsigned grid = blocks_for(P.rows, G.lanes ? LN_THREADS / G.lanes : 1);
    if (G.lanes == 4) launch_k(layer_norm_fwd_kernel<T, V, 4, VPL>, dim3(grid), dim3(LN_THREADS), 0, st, 1, P);
    else if (G.lanes == 8) launch_k(layer_norm_fwd_kernel<T, V, 8, VPL>, dim3(grid), dim3(LN_THREADS), 0, st, 1, P);
    else if (G.lanes == 16) launch_k(layer_norm_fwd_kernel<T, V, 16, VPL>, dim3(grid), dim3(LN_THREADS), 0, st, 1, P);
    else if (G.lanes == 32) launch_k(layer_norm_fwd_kernel<T, V, 32, VPL>, dim3(grid), dim3(LN_THREADS), 0, st, 1, P);
    else launch_k(layer_norm_fwd_kernel<T, V, 0, VPL>, dim3(grid), dim3(G.threads), 0, st, 1, P);
}

// Rows that are whole vectors only several at a time: dense, from 16-byte aligned pointers, as wide as the tiles' shared memory and a
// thread's columns allow.
constexpr size_t LN_TILE_SMEM = 98304;
template <typename T> bool tile_rows(bool dense, int c, int tiles, size_t* smem) {
    *smem = (size_t)tiles * ln_tile_rows<T>() * c * sizeof(T);
    return dense && c >= 64 && c <= LN_TILE_COLS * LN_TILE_THREADS && *smem <= LN_TILE_SMEM;
}
// The tiles may be more shared memory than a kernel has by default: asked for once per kernel and device.
template <typename... A> nb_status allow_smem(void (*kernel)(A...), std::atomic<unsigned long long>& done) {
    int dev = 0;
    cudaGetDevice(&dev);
    const unsigned long long bit = 1ull << (dev & 63);
    if (done.load(std::memory_order_acquire) & bit) return NB_OK;
    NB_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)LN_TILE_SMEM));
    done.fetch_or(bit, std::memory_order_release);
    return NB_OK;
}

template <typename T> nb_status run_fwd(LnFwd P, bool vec, bool dense, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T);
    P.nvec = vec ? P.c / V : P.c;
    size_t smem = 0;
    if (!vec && tile_rows<T>(dense, P.c, 1, &smem)) {
        static std::atomic<unsigned long long> done{0};
        NB_TRY(allow_smem(layer_norm_fwd_tile_kernel<T>, done));
        launch_k(layer_norm_fwd_tile_kernel<T>, dim3(blocks_for(P.rows, ln_tile_rows<T>())), dim3(LN_TILE_THREADS), smem, st, 1, P);
        return launch_ok("layer_norm_fwd (tiles)");
    }
    if (vec && P.nvec <= 4 * 512) {
        const Group G = choose_group(P.nvec, 4, false);
        if (G.vpl == 1) launch_fwd_lanes<T, V, 1>(G, P, st);
        else if (G.vpl == 2) launch_fwd_lanes<T, V, 2>(G, P, st);
        else if (G.vpl == 3) launch_fwd_lanes<T, V, 3>(G, P, st);
        else launch_fwd_lanes<T, V, 4>(G, P, st);
    } else if (!vec && P.c <= 32) {
        launch_k(layer_norm_fwd_kernel<T, 1, 32, 1>, dim3(blocks_for(P.rows, LN_THREADS / 32)), dim3(LN_THREADS), 0, st, 1, P);
    } else if (!vec && P.c <= 1024) {
        const unsigned grid = blocks_for(P.rows, LN_THREADS / 32);
        if (P.c <= 256) launch_k(layer_norm_fwd_kernel<T, 1, 32, 8>, dim3(grid), dim3(LN_THREADS), 0, st, 1, P);
        else launch_k(layer_norm_fwd_kernel<T, 1, 32, 32>, dim3(grid), dim3(LN_THREADS), 0, st, 1, P);
    } else if (!vec && P.c <= 8 * LN_MAX_BLOCK) {
        launch_k(layer_norm_fwd_kernel<T, 1, 0, 8>, dim3(blocks_for(P.rows, 1)), dim3((P.c + 255) / 256 * 32), 0, st, 1, P);
    } else {
        launch_k(layer_norm_fwd_loop_kernel<T>, dim3(blocks_for(P.rows, 1)), dim3(LN_MAX_BLOCK), 0, st, 1, P);
    }
    return launch_ok("layer_norm_fwd");
}

// Blocks of the backward call, each of which leaves a row of partial sums: as many as are resident, fewer where rows are long and
// the partial sums would be read and written for longer than they help.
int bwd_blocks(long long rows, int c, int sms) {
    const long long most = (long long)sms * (c <= 1024 ? 6 : c <= 2048 ? 4 : 2);
    return (int)std::max<long long>(1, std::min(rows, most));
}

template <typename T, int V, int L, int VPL> void launch_bwd_group(const LnBwd& P, unsigned grid, int threads, cudaStream_t st) {
    const size_t smem = L && P.partials ? 2 * (size_t)P.c * sizeof(float) : 0;
    if (P.add) {
        if (P.partials) launch_k(layer_norm_bwd_kernel<T, V, L, VPL, true, true>, dim3(grid), dim3(threads), smem, st, 1, P);
        else launch_k(layer_norm_bwd_kernel<T, V, L, VPL, true, false>, dim3(grid), dim3(threads), smem, st, 1, P);
    } else {
        if (P.partials) launch_k(layer_norm_bwd_kernel<T, V, L, VPL, false, true>, dim3(grid), dim3(threads), smem, st, 1, P);
        else launch_k(layer_norm_bwd_kernel<T, V, L, VPL, false, false>, dim3(grid), dim3(threads), smem, st, 1, P);
    }
}
template <typename T, int V, int VPL> void launch_bwd_lanes(const Group& G, const LnBwd& P, unsigned grid, cudaStream_t st) {
    if (G.lanes == 4) launch_bwd_group<T, V, 4, VPL>(P, grid, LN_THREADS, st);
    else if (G.lanes == 8) launch_bwd_group<T, V, 8, VPL>(P, grid, LN_THREADS, st);
    else if (G.lanes == 16) launch_bwd_group<T, V, 16, VPL>(P, grid, LN_THREADS, st);
    else if (G.lanes == 32) launch_bwd_group<T, V, 32, VPL>(P, grid, LN_THREADS, st);
    else launch_bwd_group<T, V, 0, VPL>(P, grid, G.threads, st);
}

template <typename T> nb_status run_bwd(LnBwd P, bool vec, bool dense, int blocks, float* dgamma, float* dbeta, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T);
    P.nvec = vec ? P.c / V : P.c;
    int parts = blocks;
    size_t smem = 0;
    constexpr int most = 16 / V;  // 16 columns a thread: their sums, this row's and the next row's values fit 128 registers
    if (!vec && tile_rows<T>(dense, P.c, P.add ? 3 : 2, &smem)) {
        parts = (int)std::min<long long>(blocks, (P.rows + ln_tile_rows<T>() - 1) / ln_tile_rows<T>());
        static std::atomic<unsigned long long> done{0}, done_sums{0};
        if (P.partials) {
            NB_TRY(allow_smem(layer_norm_bwd_tile_kernel<T, true>, done_sums));
            launch_k(layer_norm_bwd_tile_kernel<T, true>, dim3((unsigned)parts), dim3(LN_TILE_THREADS), smem, st, 1, P);
        } else {
            NB_TRY(allow_smem(layer_norm_bwd_tile_kernel<T, false>, done));
            launch_k(layer_norm_bwd_tile_kernel<T, false>, dim3((unsigned)parts), dim3(LN_TILE_THREADS), smem, st, 1, P);
        }
    } else if (vec && P.nvec <= most * LN_BWD_MAX_BLOCK) {
        const Group G = choose_group(P.nvec, most, true);
        const int groups = G.lanes ? LN_THREADS / G.lanes : 1;
        parts = (int)std::min<long long>(blocks, (P.rows + groups - 1) / groups);
        if (G.vpl == 1) launch_bwd_lanes<T, V, 1>(G, P, (unsigned)parts, st);
        else if (G.vpl == 2) launch_bwd_lanes<T, V, 2>(G, P, (unsigned)parts, st);
        else if constexpr (most == 4) {
            if (G.vpl == 3) launch_bwd_lanes<T, V, 3>(G, P, (unsigned)parts, st);
            else launch_bwd_lanes<T, V, 4>(G, P, (unsigned)parts, st);
        }
    } else if (!vec && P.c <= 8 * LN_BWD_MAX_BLOCK) {
        launch_bwd_group<T, 1, 0, 8>(P, (unsigned)parts, (P.c + 255) / 256 * 32, st);
    } else {
        if (P.partials) {
            const long long per = (P.rows + parts - 1) / parts;
            parts = (int)((P.rows + per - 1) / per);
            launch_k(layer_norm_cols_kernel<T>, dim3((unsigned)((P.c + 127) / 128), (unsigned)parts), dim3(128), 0, st, 1, P, per);
            NB_LAUNCH_OK("layer_norm_cols");
        }
        launch_k(layer_norm_bwd_loop_kernel<T>, dim3(blocks_for(P.rows, 1)), dim3(LN_MAX_BLOCK), 0, st, 1, P);
    }
    NB_LAUNCH_OK("layer_norm_bwd");
    if (P.partials) {
        launch_k(layer_norm_reduce_kernel, dim3((unsigned)((2 * (long long)P.c + LN_RED_COLS - 1) / LN_RED_COLS)), dim3(LN_RED_COLS * LN_RED_ROWS), 0, st, 1, (const float*)P.partials, parts, P.c, dgamma, dbeta);
        NB_LAUNCH_OK("layer_norm_reduce");
    }
    return NB_OK;
}

nb_status check_rows(int32_t dtype, int64_t rows, int32_t c) {
    if (!known(dtype)) return fail(NB_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (rows <= 0 || c <= 0) return fail(NB_ERR_INVALID_ARG, "rows and c must be positive");
    if (c > (1 << 24)) return fail(NB_ERR_INVALID_ARG, "c must not be above 2^24");
    return NB_OK;
}
// A matrix operand: pitch (0 = dense) and alignment; `vec` stays true while every row is whole 16-byte vectors, `dense` while
// rows follow one another from a 16-byte boundary.
nb_status check_matrix(const char* name, const void* p, int64_t* ld, int32_t c, size_t es, bool* vec, bool* dense) {
    if (*ld == 0) *ld = c;
    if (*ld < c) return fail(NB_ERR_INVALID_ARG, "ld_%s is smaller than c", name);
    if (reinterpret_cast<uintptr_t>(p) & (es - 1)) return fail(NB_ERR_ALIGNMENT, "%s is not aligned to its element size", name);
    if ((reinterpret_cast<uintptr_t>(p) & 15u) || ((uint64_t)*ld * es) % 16 || ((uint64_t)c * es) % 16) *vec = false;
    if ((reinterpret_cast<uintptr_t>(p) & 15u) || *ld != c) *dense = false;
    return NB_OK;
}
nb_status check_floats(const char* name, const float* p, bool* vec) {
    if (reinterpret_cast<uintptr_t>(p) & 3u) return fail(NB_ERR_ALIGNMENT, "%s is not 4-byte aligned", name);
    if (vec && (reinterpret_cast<uintptr_t>(p) & 15u)) *vec = false;
    return NB_OK;
}

}  // namespace

extern "C" {

nb_status nb_layer_norm_fwd(int32_t dtype, int64_t rows, int32_t c, const void* x, int64_t ld_x, const float* gamma, const float* beta, float eps, void* y, int64_t ld_y,
                            float* mean, float* rstd, void* stream) {
    g_err.clear();
    NB_TRY(check_rows(dtype, rows, c));
    if (!x || !y) return fail(NB_ERR_INVALID_ARG, "x and y must not be NULL");
    if (!mean != !rstd) return fail(NB_ERR_INVALID_ARG, "mean and rstd must be given together");
    if (!(eps > 0.f)) return fail(NB_ERR_INVALID_ARG, "eps must be positive");
    const size_t es = size_of(dtype);
    bool vec = true, dense = true;
    NB_TRY(check_matrix("x", x, &ld_x, c, es, &vec, &dense));
    NB_TRY(check_matrix("y", y, &ld_y, c, es, &vec, &dense));
    NB_TRY(check_floats("gamma", gamma, &vec));
    NB_TRY(check_floats("beta", beta, &vec));
    NB_TRY(check_floats("mean", mean, nullptr));
    NB_TRY(check_floats("rstd", rstd, nullptr));
    LnFwd P = {x, y, gamma, beta, mean, rstd, rows, ld_x, ld_y, c, 0, eps};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == NB_DTYPE_F32) return run_fwd<float>(P, vec, dense, st);
    if (dtype == NB_DTYPE_BF16) return run_fwd<__nv_bfloat16>(P, vec, dense, st);
    return run_fwd<__half>(P, vec, dense, st);
}

nb_status nb_layer_norm_workspace_bytes(int64_t rows, int32_t c, size_t* bytes) {
    g_err.clear();
    if (!bytes) return fail(NB_ERR_INVALID_ARG, "bytes is NULL");
    NB_TRY(check_rows(NB_DTYPE_F32, rows, c));
    *bytes = align_up((size_t)bwd_blocks(rows, c, sm_count()) * 2 * (size_t)c * sizeof(float), 256);
    return NB_OK;
}

nb_status nb_layer_norm_bwd(int32_t dtype, int64_t rows, int32_t c, const void* g, int64_t ld_g, const void* x, int64_t ld_x, const float* gamma, const float* mean,
                            const float* rstd, const void* add, int64_t ld_add, void* dx, int64_t ld_dx, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes,
                            void* stream) {
    g_err.clear();
    NB_TRY(check_rows(dtype, rows, c));
    if (!g || !x || !mean || !rstd || !dx) return fail(NB_ERR_INVALID_ARG, "g, x, mean, rstd and dx must not be NULL");
    if (!dgamma != !dbeta) return fail(NB_ERR_INVALID_ARG, "dgamma and dbeta must be given together");
    const size_t es = size_of(dtype);
    bool vec = true, dense = true;
    NB_TRY(check_matrix("g", g, &ld_g, c, es, &vec, &dense));
    NB_TRY(check_matrix("x", x, &ld_x, c, es, &vec, &dense));
    if (add) NB_TRY(check_matrix("add", add, &ld_add, c, es, &vec, &dense));
    NB_TRY(check_matrix("dx", dx, &ld_dx, c, es, &vec, &dense));
    NB_TRY(check_floats("gamma", gamma, &vec));
    NB_TRY(check_floats("mean", mean, nullptr));
    NB_TRY(check_floats("rstd", rstd, nullptr));
    NB_TRY(check_floats("dgamma", dgamma, nullptr));
    NB_TRY(check_floats("dbeta", dbeta, nullptr));
    const int blocks = bwd_blocks(rows, c, sm_count());
    if (dgamma) NB_TRY(check_ws(workspace, workspace_bytes, align_up((size_t)blocks * 2 * (size_t)c * sizeof(float), 256)));
    LnBwd P = {g, x, add, dx, gamma, mean, rstd, dgamma ? static_cast<float*>(workspace) : nullptr, rows, ld_g, ld_x, ld_add, ld_dx, c, 0};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == NB_DTYPE_F32) return run_bwd<float>(P, vec, dense, blocks, dgamma, dbeta, st);
    if (dtype == NB_DTYPE_BF16) return run_bwd<__nv_bfloat16>(P, vec, dense, blocks, dgamma, dbeta, st);
    return run_bwd<__half>(P, vec, dense, blocks, dgamma, dbeta, st);
}

}  // extern "C"
