// C ABI of the fused AdamW step (see include/nb_adamw.h): tensor-list plans, the step and its loss-scaled form.  Host memory
// only; the workspace is the caller's.
#include <algorithm>
#include <atomic>
#include <cstddef>
#include <cstring>
#include <memory>
#include <new>
#include <vector>

#include "adamw.cuh"
#include "api_common.cuh"
#include "common.cuh"

using namespace nbcbs;
using namespace nbapi;

struct nb_adamw_plan_s {
    int device = 0, sms = 0;
    bool grads_f32 = false;  // of a tensor whose moments are held in 8 bits
    AwHeader h;
    std::vector<uint8_t> image;  // header + tensor list + chunk table, as they sit at the start of the workspace
};

namespace {
struct Range {
    uintptr_t lo, hi;
    int tensor;
    bool written;
};

nb_status check_tensor(const nb_adamw_tensor& t, int i) {
    if (t.numel <= 0) return fail(NB_ERR_INVALID_ARG, "tensor %d: numel must be positive", i);
    if (t.numel >= (1LL << 43)) return fail(NB_ERR_UNSUPPORTED, "tensor %d: too many elements", i);
    if (t.group < 0 || t.group >= NB_SGD_GROUPS) return fail(NB_ERR_INVALID_ARG, "tensor %d: group %d out of range", i, t.group);
    if (!t.grad || !t.param || !t.exp_avg || !t.exp_avg_sq) return fail(NB_ERR_INVALID_ARG, "tensor %d: grad, param, exp_avg and exp_avg_sq must not be NULL", i);
    if (t.grad_dtype != NB_DTYPE_F32 && t.grad_dtype != NB_DTYPE_BF16 && t.grad_dtype != NB_DTYPE_F16)
        return fail(NB_ERR_INVALID_ARG, "tensor %d: unknown grad_dtype %d", i, t.grad_dtype);
    if (t.copy_dtype != 0 && t.copy_dtype != NB_DTYPE_BF16 && t.copy_dtype != NB_DTYPE_F16)
        return fail(NB_ERR_INVALID_ARG, "tensor %d: copy_dtype %d is neither bf16 nor fp16", i, t.copy_dtype);
    if (t.state_bits != 32 && t.state_bits != 8) return fail(NB_ERR_INVALID_ARG, "tensor %d: state_bits is %d, must be 32 or 8", i, t.state_bits);
    if (t.state_bits == 8 ? (!t.exp_avg_scale || !t.exp_avg_sq_scale) : (t.exp_avg_scale || t.exp_avg_sq_scale))
        return fail(NB_ERR_INVALID_ARG, "tensor %d: moments in 8 bits take two scale arrays, moments in 32 bits none", i);
    const uintptr_t bits = reinterpret_cast<uintptr_t>(t.grad) | reinterpret_cast<uintptr_t>(t.param) | reinterpret_cast<uintptr_t>(t.exp_avg) |
                           reinterpret_cast<uintptr_t>(t.exp_avg_sq) | reinterpret_cast<uintptr_t>(t.param_copy);
    if (bits & 15u) return fail(NB_ERR_ALIGNMENT, "tensor %d: a pointer is not 16-byte aligned", i);
    if ((reinterpret_cast<uintptr_t>(t.exp_avg_scale) | reinterpret_cast<uintptr_t>(t.exp_avg_sq_scale)) & 3u)
        return fail(NB_ERR_ALIGNMENT, "tensor %d: a scale pointer is not 4-byte aligned", i);
    return NB_OK;
}

// What a step writes must not overlap anything else that it reads or writes: blocks work on all tensors at once.
nb_status check_overlap(const nb_adamw_tensor* t, int count) {
    std::vector<Range> r;
    r.reserve((size_t)count * 7);
    for (int i = 0; i < count; ++i) {
        const uintptr_t n = (uintptr_t)t[i].numel, blocks = (n + NB_ADAMW_BLOCK - 1) / NB_ADAMW_BLOCK, state = t[i].state_bits == 8 ? 1 : 4;
        auto add = [&](const void* p, uintptr_t bytes, bool written) {
            const uintptr_t a = reinterpret_cast<uintptr_t>(p);
            if (p) r.push_back({a, a + bytes, i, written});
        };
        add(t[i].grad, n * (t[i].grad_dtype == NB_DTYPE_F32 ? 4 : 2), false);
        add(t[i].param, n * 4, true);
        add(t[i].exp_avg, n * state, true);
        add(t[i].exp_avg_sq, n * state, true);
        add(t[i].exp_avg_scale, blocks * 4, true);
        add(t[i].exp_avg_sq_scale, blocks * 4, true);
        add(t[i].param_copy, n * 2, true);
    }
    std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
    uintptr_t any_end = 0, written_end = 0;  // furthest end so far, of any range and of the written ones
    int any_of = -1, written_of = -1;
    for (const Range& x : r) {
        const uintptr_t end = x.written ? any_end : written_end;
        if (x.lo < end) return fail(NB_ERR_INVALID_ARG, "tensors %d and %d: a range that the step writes overlaps another", x.written ? any_of : written_of, x.tensor);
        if (x.hi > any_end) { any_end = x.hi; any_of = x.tensor; }
        if (x.written && x.hi > written_end) { written_end = x.hi; written_of = x.tensor; }
    }
    return NB_OK;
}

// The ring of the 8-bit form is more shared memory than a kernel has by default: asked for once per device.
nb_status allow_ring(int device) {
    static std::atomic<unsigned long long> done{0};
    const unsigned long long bit = 1ull << (device & 63);
    if (done.load(std::memory_order_acquire) & bit) return NB_OK;
    NB_CUDA_CHECK(cudaFuncSetAttribute(adamw_update_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, aw_ring_bytes(true)));
    done.fetch_or(bit, std::memory_order_release);
    return NB_OK;
}

nb_status adamw_step_impl(nb_adamw_plan p, void* workspace, size_t workspace_bytes, const nb_adamw_hyper* hyper, const nb_scaler_hyper* sc, nb_loss_scaler* state,
                          int64_t* step, float* total_norm, void* stream) {
    if (!p) return fail(NB_ERR_INVALID_ARG, "plan is NULL");
    if (!hyper) return fail(NB_ERR_INVALID_ARG, "hyper is NULL");
    if (hyper->struct_size != sizeof(nb_adamw_hyper)) return fail(NB_ERR_INVALID_ARG, "nb_adamw_hyper.struct_size is %u, expected %zu", hyper->struct_size, sizeof(nb_adamw_hyper));
    if (!(hyper->beta1 >= 0.0 && hyper->beta1 < 1.0) || !(hyper->beta2 >= 0.0 && hyper->beta2 < 1.0)) return fail(NB_ERR_INVALID_ARG, "beta1 and beta2 must be in [0, 1)");
    if (!(hyper->eps >= 0.f)) return fail(NB_ERR_INVALID_ARG, "eps must not be negative");
    if (!step) return fail(NB_ERR_INVALID_ARG, "step is NULL");
    if (reinterpret_cast<uintptr_t>(step) & 7u) return fail(NB_ERR_ALIGNMENT, "step is not 8-byte aligned");
    if (reinterpret_cast<uintptr_t>(total_norm) & 3u) return fail(NB_ERR_ALIGNMENT, "total_norm is not 4-byte aligned");
    NB_TRY(check_ws(workspace, workspace_bytes, (size_t)p->h.total_bytes));
    DeviceGuard on_device(p->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    AwScalars s;
    s.eps = hyper->eps;
    s.max_norm = hyper->max_norm;
    for (int i = 0; i < NB_SGD_GROUPS; ++i) {
        s.lr[i] = hyper->lr[i];
        s.keep[i] = (float)(1.0 - (double)hyper->lr[i] * (double)hyper->weight_decay[i]);
    }
    s.b1 = (float)hyper->beta1;
    s.c1 = (float)(1.0 - hyper->beta1);
    s.b2 = (float)hyper->beta2;
    s.c2 = (float)(1.0 - hyper->beta2);
    s.step = step;
    s.scaler = state;
    s.growth_factor = s.backoff_factor = 1.f;
    s.floor_scale = 0.f;
    s.growth_interval = 1;
    if (sc) {
        s.growth_factor = sc->growth_factor;
        s.backoff_factor = sc->backoff_factor;
        s.floor_scale = sc->floor_scale;
        s.growth_interval = sc->growth_interval;
    }
    // (the norm is not needed when nothing depends on it: no clipping, no scaler that looks for inf and NaN, nobody asks for it)
    const int want_norm = (hyper->max_norm > 0.f && hyper->max_norm < __builtin_inff()) || state || total_norm;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    launch_k(adamw_norm_kernel, dim3(want_norm ? (unsigned)p->h.grid : 1u), dim3(AW_THREADS), 0, st, 1, ws, s, hyper->beta1, hyper->beta2, want_norm);
    NB_LAUNCH_OK("adamw_norm");
    const int n8 = p->h.eight, n32 = p->h.nchunks - n8;
    if (n8) {
        NB_TRY(allow_ring(p->device));
        // (resident blocks of an SM: four by registers, three where fp32 gradients make the ring larger)
        launch_k(adamw_update_kernel<true>, dim3((unsigned)std::min(n8, p->sms * (p->grads_f32 ? 3 : AW_BLOCKS_PER_SM))), dim3(AW_THREADS), (size_t)aw_ring_bytes(p->grads_f32), st, 1, ws, s, want_norm,
                 total_norm, n32 ? 0 : 1, aw_stage_bytes(p->grads_f32));
        NB_LAUNCH_OK("adamw_update (8 bits)");
    }
    if (n32) {
        launch_k(adamw_update_kernel<false>, dim3((unsigned)std::min(n32, p->h.grid)), dim3(AW_THREADS), 0, st, 1, ws, s, want_norm, total_norm, 1, 0);
        NB_LAUNCH_OK("adamw_update");
    }
    return NB_OK;
}
}  // namespace

extern "C" {

nb_status nb_adamw_plan_create(const nb_adamw_tensor* t, int32_t count, int device, nb_adamw_plan* out) {
    g_err.clear();
    if (!out) return fail(NB_ERR_INVALID_ARG, "out_plan is NULL");
    *out = nullptr;
    if (!t) return fail(NB_ERR_INVALID_ARG, "host_tensors is NULL");
    if (count <= 0) return fail(NB_ERR_INVALID_ARG, "count must be positive, got %d", count);
    try {
        long long nchunks = 0, eight = 0;
        bool grads_f32 = false;
        for (int i = 0; i < count; ++i) {
            NB_TRY(check_tensor(t[i], i));
            const long long n = (t[i].numel + AW_CHUNK - 1) / AW_CHUNK;
            nchunks += n;
            if (t[i].state_bits == 8) {
                eight += n;
                grads_f32 |= t[i].grad_dtype == NB_DTYPE_F32;
            }
        }
        if (nchunks > 0x7fffffffLL) return fail(NB_ERR_UNSUPPORTED, "too many elements for one tensor list");
        NB_TRY(check_overlap(t, count));
        int sms = 0;
        if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) {
            cudaGetLastError();
            return fail(NB_ERR_CUDA, "cannot query device %d", device);
        }
        std::unique_ptr<nb_adamw_plan_s> p(new nb_adamw_plan_s);
        p->device = device;
        p->sms = std::max(sms, 1);
        p->grads_f32 = grads_f32;
        AwHeader& h = p->h;
        memset(&h, 0, sizeof h);
        h.nchunks = (int32_t)nchunks;
        h.eight = (int32_t)eight;
        h.grid = (int32_t)std::min<long long>(nchunks, std::min<long long>(AW_MAX_BLOCKS, (long long)std::max(sms, 1) * AW_BLOCKS_PER_SM));
        size_t off = 256;
        h.off_chunks = off; off = align_up(off + (size_t)nchunks * sizeof(AwChunk), 256);
        h.off_partials = off; off = align_up(off + (size_t)AW_MAX_BLOCKS * sizeof(double), 256);
        h.total_bytes = off;
        p->image.assign((size_t)h.off_partials, 0);
        memcpy(p->image.data(), &h, sizeof h);
        AwChunk* c = reinterpret_cast<AwChunk*>(p->image.data() + h.off_chunks);
        for (int pass = 0; pass < 2 * count; ++pass) {  // first the tensors with moments in 8 bits, then the others
            const int i = pass % count;
            const bool eight = t[i].state_bits == 8;
            if (eight != (pass < count)) continue;
            for (int64_t s = 0; s < t[i].numel; s += AW_CHUNK, ++c) {
                const int64_t se = eight ? 1 : 4, ge = t[i].grad_dtype == NB_DTYPE_F32 ? 4 : 2;
                c->grad = static_cast<const char*>(t[i].grad) + s * ge;
                c->param = t[i].param + s;
                c->exp_avg = static_cast<char*>(t[i].exp_avg) + s * se;
                c->exp_avg_sq = static_cast<char*>(t[i].exp_avg_sq) + s * se;
                c->exp_avg_scale = eight ? t[i].exp_avg_scale + s / NB_ADAMW_BLOCK : nullptr;
                c->exp_avg_sq_scale = eight ? t[i].exp_avg_sq_scale + s / NB_ADAMW_BLOCK : nullptr;
                c->copy = t[i].param_copy ? static_cast<char*>(t[i].param_copy) + s * 2 : nullptr;
                c->len = (uint16_t)std::min<int64_t>(AW_CHUNK, t[i].numel - s);
                c->group = (uint8_t)t[i].group;
                c->grad_dtype = (uint8_t)t[i].grad_dtype;
                c->copy_dtype = (uint8_t)t[i].copy_dtype;
            }
        }
        *out = p.release();
        return NB_OK;
    } catch (const std::bad_alloc&) {
        return fail(NB_ERR_INTERNAL, "out of host memory");
    }
}

nb_status nb_adamw_plan_destroy(nb_adamw_plan p) {
    g_err.clear();
    delete p;
    return NB_OK;
}

nb_status nb_adamw_workspace_bytes(nb_adamw_plan p, size_t* bytes) {
    g_err.clear();
    if (!p || !bytes) return fail(NB_ERR_INVALID_ARG, "NULL argument");
    *bytes = (size_t)p->h.total_bytes;
    return NB_OK;
}

nb_status nb_adamw_upload(nb_adamw_plan p, void* workspace, size_t workspace_bytes, void* stream) {
    g_err.clear();
    if (!p) return fail(NB_ERR_INVALID_ARG, "plan is NULL");
    NB_TRY(check_ws(workspace, workspace_bytes, (size_t)p->h.total_bytes));
    DeviceGuard on_device(p->device);
    // the source is the plan's own host image, which lives as long as the plan
    NB_CUDA_CHECK(cudaMemcpyAsync(workspace, p->image.data(), p->image.size(), cudaMemcpyHostToDevice, static_cast<cudaStream_t>(stream)));
    return NB_OK;
}

nb_status nb_adamw_step(nb_adamw_plan p, void* workspace, size_t workspace_bytes, const nb_adamw_hyper* hyper, int64_t* step, float* total_norm, void* stream) {
    g_err.clear();
    return adamw_step_impl(p, workspace, workspace_bytes, hyper, nullptr, nullptr, step, total_norm, stream);
}

nb_status nb_adamw_step_scaled(nb_adamw_plan p, void* workspace, size_t workspace_bytes, const nb_adamw_hyper* hyper, const nb_scaler_hyper* sc, nb_loss_scaler* state,
                               int64_t* step, float* total_norm, void* stream) {
    g_err.clear();
    if (!sc || !state) return fail(NB_ERR_INVALID_ARG, "scaler and state must not be NULL");
    if (sc->struct_size != sizeof(nb_scaler_hyper)) return fail(NB_ERR_INVALID_ARG, "nb_scaler_hyper.struct_size is %u, expected %zu", sc->struct_size, sizeof(nb_scaler_hyper));
    if (reinterpret_cast<uintptr_t>(state) & 15u) return fail(NB_ERR_ALIGNMENT, "state is not 16-byte aligned");
    if (!(sc->growth_factor > 0.f) || !(sc->backoff_factor > 0.f) || sc->growth_interval < 1) return fail(NB_ERR_INVALID_ARG, "scaler factors must be positive, growth_interval >= 1");
    return adamw_step_impl(p, workspace, workspace_bytes, hyper, sc, state, step, total_norm, stream);
}

}  // extern "C"
