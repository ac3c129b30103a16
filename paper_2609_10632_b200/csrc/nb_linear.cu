// C ABI of the MLP products (see include/nb_linear.h): plans, the choice of kernels and tiles, the three calls.  The only
// allocation is a plan's status block; the workspace is the caller's.
#include <algorithm>
#include <atomic>
#include <cstring>
#include <memory>
#include <new>

#include "api_common.cuh"
#include "linear.cuh"
#include "tc_common.cuh"
#include "tc_linear.cuh"

using namespace nbcbs;
using namespace nbapi;

struct nb_linear_plan_s {
    nb_linear_desc d;
    int device = 0, sms = 148;
    int* status = nullptr;
};

namespace {

size_t size_of(int32_t dtype) { return dtype == NB_DTYPE_F32 ? 4 : 2; }
long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// ---------------------------------------------------------------- tensor cores: tiles
struct TlCfg {
    bool cg2 = false;
    int bn = 0, m_tiles = 0, n_tiles = 0, kblocks = 0, splits = 1, kb_per_split = 0;
    double cost = 0;
};

// Cycles of a stage (128 rows a CTA, BN columns, 64 k): the products, or the operand bytes from L2 at what an SM gets of them
// (measured on products of 1024 to 4096 terms: 700 a stage of 256 columns in a pair, 62 bytes a cycle; the weight gradient, whose
// operands come in twice as many boxes, follows the second pair of figures better: 8192 x 1024 x 1024 24 against 30 us).
double stage_cycles(bool cg2, int bn, bool weight) {
    const double bytes = 16384.0 + (cg2 ? bn / 2 : bn) * 128.0;
    return weight ? std::max(2.0 * bn, bytes / 55.0) : std::max(2.75 * bn, bytes / 62.0);
}

// Tiles of a forward product or data gradient: the least time of the persistent loop over what the candidates give.  A tile takes its
// products or its epilogue, whichever is longer; the epilogue has a part of its own (handing the accumulators over, twice as long
// between the CTAs of a pair) and `per_col` cycles for each column, `narrow` times as many in a forward product whose passes have 32
// columns (tiles of 64 and 192), and `wait` for a residual's tile.  us, the same buffers again and again, tiles of 256, 192 and 128 columns:
//   25600 x 384 -> 1536 with GELU and z   pairs 58.7, 65.0, 67.9   single CTAs 53.3, 58.6, 57.2
//   the same with a residual, without z   pairs 68.1, 69.1, 77.8   single CTAs 60.8, 61.3, 70.7
//   25600 x 384 -> 768 with GELU          pairs 30.8, 33.6, 35.8   single CTAs 29.2, 30.7, 28.7
//   8192 x 1024 -> 4096 with GELU and z   pairs 63.1, 70.5, 72.0   single CTAs 67.1, 74.3, 75.3
//   data gradient of 25600 x 1536 -> 384 through GELU   pairs 75.1, 68.1, 81.7   single CTAs 63.5, 59.0, 71.5
//   25600 x 1536 -> 384 with bias         pairs 34.9, 29.5, 33.9   single CTAs 37.3, 34.1, 36.8
// Products of more than `chunk` k-blocks take the kernel whose sums leave the tensor cores in between, on tiles of 128 columns: what that
// exactness costs is 4096 x 32768 -> 1024 in fp16 203 -> 243 us, 2048 x 151936 -> 2048 in bf16 908 -> 1036.
TlCfg choose_rows(long long M, long long N, long long K, int sms, double per_col, double narrow, double wait, int chunk) {
    TlCfg best;
    for (int cg2 = 1; cg2 >= 0; --cg2)
        for (int bn = 256; bn >= 64; bn -= 64) {
            if (K > (long long)chunk * TL_KC && bn != 128) continue;
            TlCfg c;
            c.cg2 = cg2 != 0;
            c.bn = bn;
            c.m_tiles = (int)ceil_div(M, cg2 ? 256 : 128);
            c.n_tiles = (int)ceil_div(N, bn);
            c.kblocks = (int)ceil_div(K, TL_KC);
            const long long workers = cg2 ? sms / 2 : sms, tiles = (long long)c.m_tiles * c.n_tiles;
            const double main = c.kblocks * stage_cycles(cg2, bn, false), epi = (cg2 ? 2800.0 : 1450.0) + wait + bn * per_col * (bn % 128 ? narrow : 1.0);
            c.cost = (double)ceil_div(tiles, workers) * std::max(main, epi) + std::min(main, epi) + 1000.0;
            if (!best.bn || c.cost < best.cost) best = c;
        }
    return best;
}

// Tiles and row slices of a weight gradient: every item is a CTA (or pair) of its own.
// Tiles of at most 192 columns have room in TMEM for the bias's column of sums; wider ones leave it to a pass over dy.
bool db_in_tile(const TlCfg& c) { return c.bn + 32 <= 256; }
TlCfg choose_weight(long long M, long long N, long long K, int sms) {
    TlCfg best;
    for (int cg2 = 1; cg2 >= 0; --cg2)
        for (int bn = 256; bn >= 64; bn -= 64) {
            TlCfg c;
            c.cg2 = cg2 != 0;
            c.bn = bn;
            c.m_tiles = (int)ceil_div(M, cg2 ? 256 : 128);
            c.n_tiles = (int)ceil_div(N, bn);
            c.kblocks = (int)ceil_div(K, TL_KC);
            const long long workers = cg2 ? sms / 2 : sms, tiles = (long long)c.m_tiles * c.n_tiles;
            const long long most = std::max<long long>(1, std::min<long long>({64, c.kblocks, ceil_div(4 * workers, tiles)}));
            // (from one length of a slice to the next shorter one: counts that give the same length give the same slices, and every call asks)
            for (long long s = 1; s <= most; s = c.kb_per_split > 1 ? ceil_div(c.kblocks, c.kb_per_split - 1) : most + 1) {
                c.kb_per_split = (int)ceil_div(c.kblocks, s);
                c.splits = (int)ceil_div(c.kblocks, c.kb_per_split);
                const double item = c.kb_per_split * stage_cycles(cg2, bn, true) + bn * 8.0 + 1500.0;
                // (slices: written, read back and added at about 2.5 KB a cycle, and another launch)
                const double sums = c.splits > 1 ? 3000.0 + 2.0 * c.splits * (double)M * N * 4 / 2500.0 : 0.0;
                const double db = db_in_tile(c) ? 0.0 : 3000.0 + 2.0 * M * K / 3400.0;
                c.cost = (double)ceil_div(tiles * c.splits, workers) * item + sums + db;
                if (!best.bn || c.cost < best.cost) best = c;
            }
        }
    return best;
}

// ---------------------------------------------------------------- CUDA cores: slices of k
struct SimtCfg {
    int tile = 64;
    long long tiles = 0, kslice = 0;
    int slices = 1;
};
SimtCfg simt_cfg(long long M, long long N, long long K, int sms, bool weight) {
    SimtCfg c;
    c.tiles = ceil_div(M, 128) * ceil_div(N, 128);
    long long s = 1;
    const long long small = ceil_div(M, 64) * ceil_div(N, 64), s128 = c.tiles < 2 * sms ? 2 * sms / c.tiles : 1;
    // Tiles of 128 while they, with slices of 256 products or more each, are two on most SMs, and their edges no large part of them.
    if (2 * c.tiles * s128 >= 3 * sms && (s128 == 1 || (K / s128 >= 256 && 8 * c.tiles <= 3 * small))) {
        c.tile = 128;
        s = s128;
    } else {
        c.tiles = small;
        // as many slices as give an SM four blocks, of 64 products or more each
        if (c.tiles < 4 * sms) s = std::min<long long>(ceil_div(4 * sms, c.tiles), std::max<long long>(1, K / 64));
    }
    if (weight) s = std::max(s, ceil_div(K, 4096));  // which bounds the rounding errors of an fp32 sum over rows
    s = std::min<long long>(s, 1024);
    c.kslice = ceil_div(ceil_div(K, s), LS_BK) * LS_BK;
    c.slices = (int)ceil_div(K, c.kslice);
    return c;
}
// Slices of a weight gradient on the CUDA cores that are in memory at once: at most 128 MB of them (or one).  The others follow, group by
// group, added to dw.  All at once (4096 rows each) they were 236 MB for 409600 rows of 384 -> 1536 and 16 GB for a million of 4096 -> 4096,
// in the workspace of tensor-core layers too, whose misaligned calls end up here.  Of the counts that fit, the one whose blocks leave the
// fewest places empty (two blocks of 128-tiles an SM, four of 64): 409600 rows of 384 -> 1536 in fp32 8.8 ms as all at once, 11.1 in the
// groups of 14 that 32 MB hold.
int weight_group(const SimtCfg& c, long long M, long long N, int sms) {
    const long long fit = std::max<long long>(1, (128ll << 20) / (M * N * 4)), places = (c.tile == 128 ? 2ll : 4ll) * sms;
    if (c.slices <= fit) return c.slices;
    int best = 1;
    long long least = -1;
    for (int g = (int)std::min<long long>(fit, c.slices); g >= 1; --g) {
        const long long cost = c.slices / g * ceil_div(c.tiles * g, places) + ceil_div(c.tiles * (c.slices % g), places);
        if (least < 0 || cost < least) {
            least = cost;
            best = g;
        }
    }
    return best;
}
constexpr int COLSUM_PARTS = 128;
// Ranges of rows of a column-sum pass over c columns, `v` a vector: about four blocks an SM.
int colsum_parts(long long rows, long long c, int v, int sms) {
    const long long wide = ceil_div(c, 16 * v);
    return (int)std::max<long long>(1, std::min<long long>({COLSUM_PARTS, rows / 64, ceil_div(4 * sms, wide)}));
}

// ---------------------------------------------------------------- choice of kernels
bool tc_layer(const nb_linear_plan_s* p) {
    return p->d.dtype != NB_DTYPE_F32 && !(p->d.flags & NB_LINEAR_FLAG_FORCE_SIMT) && p->d.c_in % 8 == 0 && p->d.c_out % 8 == 0;
}
// Layers whose channel counts are not multiples of 8 run on padded copies of their operands (bandwidth against the tensor cores' rate);
// below this many products the copies and launches take longer than the CUDA cores.
int round8(int c) { return (c + 7) / 8 * 8; }
bool tc_padded(const nb_linear_plan_s* p, long long rows) {
    return p->d.dtype != NB_DTYPE_F32 && !(p->d.flags & NB_LINEAR_FLAG_FORCE_SIMT) && (p->d.c_in % 8 || p->d.c_out % 8) &&
           (double)rows * p->d.c_in * p->d.c_out >= 134217728.0;
}
bool few_rows(const nb_linear_plan_s* p, long long rows) { return rows <= 8 && ((size_t)p->d.c_in * size_of(p->d.dtype)) % 16 == 0; }
bool whole16(const void* q, long long ld, size_t es) { return !(reinterpret_cast<uintptr_t>(q) & 15u) && ((size_t)ld * es) % 16 == 0; }

size_t simt_ws(const nb_linear_plan_s* p, long long rows, int kind) {
    const long long ci = p->d.c_in, co = p->d.c_out;
    const long long M = kind == LIN_WEIGHT ? co : rows, N = kind == LIN_FWD ? co : ci, K = kind == LIN_FWD ? ci : kind == LIN_DATA ? co : rows;
    const SimtCfg c = simt_cfg(M, N, K, p->sms, kind == LIN_WEIGHT);
    const int slices = kind == LIN_WEIGHT ? weight_group(c, M, N, p->sms) : c.slices;
    size_t b = c.slices > 1 ? align_up((size_t)slices * M * N * 4, 256) : 0;
    if (kind == LIN_WEIGHT) b += align_up((size_t)COLSUM_PARTS * co * 4, 256);
    return b;
}
size_t tc_weight_ws(const nb_linear_plan_s* p, const TlCfg& c) {
    const size_t M = p->d.c_out, N = p->d.c_in;
    return (c.splits > 1 ? align_up((size_t)c.splits * M * N * 4, 256) : 0) + align_up((size_t)std::max(c.splits * c.n_tiles, COLSUM_PARTS) * M * 4, 256);
}
size_t rows_bytes(long long rows, int cols) { return align_up((size_t)rows * round8(cols) * 2, 256); }
size_t padded_ws(const nb_linear_plan_s* p, long long rows) {
    const int ci = p->d.c_in, co = p->d.c_out;
    const size_t a = rows_bytes(rows, ci), b = rows_bytes(rows, co), w = rows_bytes(co, ci);
    const TlCfg c = choose_weight(co, round8(ci), rows, p->sms);
    const size_t part = align_up((size_t)c.splits * co * round8(ci) * 4, 256) + align_up((size_t)std::max(c.splits * c.n_tiles, COLSUM_PARTS) * co * 4, 256);
    return std::max({w + a + 3 * b, w + b + 3 * a, a + b + part});  // forward: x; out, z, res.  data: dy; dx, z_in, add.  weight
}
size_t workspace_for(const nb_linear_plan_s* p, long long rows) {
    size_t b = 256;
    for (int kind = 0; kind < 3; ++kind) b = std::max(b, simt_ws(p, rows, kind));
    if (tc_layer(p)) b = std::max(b, tc_weight_ws(p, choose_weight(p->d.c_out, p->d.c_in, rows, p->sms)));
    if (tc_padded(p, rows)) b = std::max(b, padded_ws(p, rows));
    return b;
}

// k-blocks that a 16-bit result's sum may stay in the tensor cores.
int long_sum(const nb_linear_plan_s* p) { return p->d.dtype == NB_DTYPE_F16 ? TL_LONG_F16 : TL_LONG_BF16; }
// Columns of an epilogue pass: a warp has half of a tile's.
int pass_cols(const TlCfg& c) { return c.bn % 128 == 0 ? 64 : 32; }

// ---------------------------------------------------------------- tensor cores: launch
bool encode(CUtensorMap* m, int32_t dtype, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box, CUtensorMapSwizzle sw, bool load) {
    tcdetail::DriverFns& d = tcdetail::driver();
    if (!d.tiled) return false;
    const CUtensorMapDataType t = dtype == NB_DTYPE_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : dtype == NB_DTYPE_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    const cuuint32_t one[3] = {1, 1, 1};
    return d.tiled(m, t, (cuuint32_t)rank, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, sw,
                   load ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// a matrix [rows][cols] of 16-bit elements, boxes of box_cols (64: 128-byte swizzle, 32: 64-byte swizzle) by box_rows
bool encode2(CUtensorMap* m, int32_t dtype, const void* base, long long rows, long long cols, long long ld, int box_cols, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows};
    return encode(m, dtype, base, 2, dims, strides, box, box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, true);
}

template <typename T, int KIND, bool CG2, int NP, bool LONG> nb_status launch_tc(const nb_linear_plan_s* plan, const TcLinParams& P, unsigned grid, size_t smem, cudaStream_t st) {
    static std::atomic<unsigned long long> attr_set{0};  // one bit per device ordinal
    const unsigned long long bit = 1ull << (plan->device & 63);
    if (!(attr_set.load(std::memory_order_acquire) & bit)) {
        NB_CUDA_CHECK(cudaFuncSetAttribute(tc_linear_kernel<T, KIND, CG2, NP, LONG>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)tcdetail::kMaxSmem));
        attr_set.fetch_or(bit, std::memory_order_release);
    }
    launch_k(tc_linear_kernel<T, KIND, CG2, NP, LONG>, dim3(grid), dim3(TL_THREADS), smem, st, CG2 ? 2 : 1, P);
    return launch_ok("tc_linear");
}

template <int KIND> nb_status run_tc(const nb_linear_plan_s* plan, const TlCfg& c, TcLinParams& P, cudaStream_t st) {
    const bool f16 = plan->d.dtype == NB_DTYPE_F16;
    P.kblocks = c.kblocks;
    P.chunk = long_sum(plan);
    P.BN = c.bn;
    P.m_tiles = c.m_tiles;
    P.n_tiles = c.n_tiles;
    P.group_m = 8;
    P.acc_stride = 256;
    P.splits = c.splits;
    P.kb_per_split = c.kb_per_split;
    P.status = plan->status;
    const int own = c.cg2 ? c.bn / 2 : c.bn;
    P.nblkB = (own + 63) / 64;
    P.b_bytes = KIND == LIN_FWD ? (uint32_t)own * 128u : (uint32_t)P.nblkB * TL_BLK;
    const int tm = c.cg2 ? 256 : 128;
    P.idesc = ptx::make_idesc_bf16(tm, c.bn, KIND == LIN_WEIGHT, KIND != LIN_FWD, f16);
    P.idesc_ones = ptx::make_idesc_bf16(tm, c.cg2 ? 32 : 16, 1, 1, f16);
    const size_t fixed = 1024 + (size_t)16 * TL_STG + (KIND == LIN_WEIGHT ? (int)TL_ONES_BYTES : KIND == LIN_FWD ? 8 * 512 : 0) + 512;
    P.stages = (int)std::min<size_t>(6, (tcdetail::kMaxSmem - fixed) / (TL_A_BYTES + P.b_bytes));
    const size_t smem = fixed + (size_t)P.stages * (TL_A_BYTES + P.b_bytes);
    const long long tiles = (long long)c.m_tiles * c.n_tiles * (KIND == LIN_WEIGHT ? c.splits : 1);
    if (tiles > 0x3fffffffLL) return fail(NB_ERR_UNSUPPORTED, "too many tiles");
    const long long workers = c.cg2 ? plan->sms / 2 : plan->sms;
    const unsigned grid = (unsigned)((KIND == LIN_WEIGHT ? tiles : std::min(tiles, workers)) * (c.cg2 ? 2 : 1));
#define NB_TL(T, NP, LONG) (c.cg2 ? launch_tc<T, KIND, true, NP, LONG>(plan, P, grid, smem, st) : launch_tc<T, KIND, false, NP, LONG>(plan, P, grid, smem, st))
    if constexpr (KIND != LIN_WEIGHT) {
        if (c.kblocks > P.chunk) return f16 ? NB_TL(__half, 64, true) : NB_TL(__nv_bfloat16, 64, true);
        if (pass_cols(c) == 64) return f16 ? NB_TL(__half, 64, false) : NB_TL(__nv_bfloat16, 64, false);
    }
    return f16 ? NB_TL(__half, 32, false) : NB_TL(__nv_bfloat16, 32, false);
#undef NB_TL
}

// ---------------------------------------------------------------- CUDA cores: launch
template <typename T, int KIND> nb_status run_simt(const nb_linear_plan_s* plan, LinArgs& P, const SimtCfg& c, bool vec, void* workspace, cudaStream_t st) {
    if (c.tiles > 0x7fffffffLL) return fail(NB_ERR_UNSUPPORTED, "too many tiles");
    P.kslice = c.kslice;
    P.slices = c.slices;
    P.partial = static_cast<float*>(workspace);
    const dim3 grid((unsigned)c.tiles, 1, (unsigned)c.slices);
    if (c.tile == 128) {
        if (vec) launch_k(lin_simt_kernel<T, KIND, true, 128>, grid, dim3(LS_THREADS), 0, st, 1, P);
        else launch_k(lin_simt_kernel<T, KIND, false, 128>, grid, dim3(LS_THREADS), 0, st, 1, P);
    } else {
        if (vec) launch_k(lin_simt_kernel<T, KIND, true, 64>, grid, dim3(LS_THREADS), 0, st, 1, P);
        else launch_k(lin_simt_kernel<T, KIND, false, 64>, grid, dim3(LS_THREADS), 0, st, 1, P);
    }
    NB_LAUNCH_OK("lin_simt");
    if (KIND != LIN_WEIGHT && c.slices > 1) {
        launch_k(lin_slices_kernel<T, KIND>, dim3((unsigned)std::min<long long>(ceil_div(P.M * P.N, 256), plan->sms * 8)), dim3(256), 0, st, 1, P);
        NB_LAUNCH_OK("lin_slices");
    }
    return NB_OK;
}
template <int KIND> nb_status run_simt_any(const nb_linear_plan_s* plan, LinArgs& P, const SimtCfg& c, bool vec, void* workspace, cudaStream_t st) {
    if (plan->d.dtype == NB_DTYPE_F32) return run_simt<float, KIND>(plan, P, c, vec, workspace, st);
    if (plan->d.dtype == NB_DTYPE_BF16) return run_simt<__nv_bfloat16, KIND>(plan, P, c, vec, workspace, st);
    return run_simt<__half, KIND>(plan, P, c, vec, workspace, st);
}

// Sums of dy's columns over ranges of rows into `partial`; returns the number of ranges in *parts.
template <typename T> nb_status run_colsum(const nb_linear_plan_s* plan, const void* dy, long long ld, long long rows, float* partial, int* parts, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T);
    const int c = plan->d.c_out;
    const bool vec = !(reinterpret_cast<uintptr_t>(dy) & 15u) && ld % V == 0 && c % V == 0;
    const long long per = ceil_div(rows, colsum_parts(rows, c, vec ? V : 1, plan->sms));
    *parts = (int)ceil_div(rows, per);
    if (vec) launch_k(lin_colsum_kernel<T, V>, dim3((unsigned)ceil_div(c, 16 * V), (unsigned)*parts), dim3(256), 0, st, 1, static_cast<const T*>(dy), ld, rows, c, per, partial);
    else launch_k(lin_colsum_kernel<T, 1>, dim3((unsigned)ceil_div(c, 16), (unsigned)*parts), dim3(256), 0, st, 1, static_cast<const T*>(dy), ld, rows, c, per, partial);
    return launch_ok("lin_colsum");
}
nb_status run_colsum_any(const nb_linear_plan_s* plan, const void* dy, long long ld, long long rows, float* partial, int* parts, cudaStream_t st) {
    if (plan->d.dtype == NB_DTYPE_F32) return run_colsum<float>(plan, dy, ld, rows, partial, parts, st);
    if (plan->d.dtype == NB_DTYPE_BF16) return run_colsum<__nv_bfloat16>(plan, dy, ld, rows, partial, parts, st);
    return run_colsum<__half>(plan, dy, ld, rows, partial, parts, st);
}

template <typename T> nb_status run_rows(const nb_linear_plan_s* plan, LinArgs& P, int rows, cudaStream_t st) {
    // warps that share a column: enough warps for the GPU, but at least two 16-byte pieces a lane
    int wpc = 1;
    while (wpc < 8 && P.N * wpc < plan->sms * 16LL && P.K / (16 / (int)sizeof(T)) >= 64LL * 2 * wpc) wpc *= 2;
    P.slices = 1;
    const unsigned grid = (unsigned)ceil_div(P.N, LR_THREADS / 32 / wpc);
    if (rows == 1) launch_k(lin_rows_kernel<T, 1>, dim3(grid), dim3(LR_THREADS), 0, st, 1, P, rows, wpc);
    else if (rows == 2) launch_k(lin_rows_kernel<T, 2>, dim3(grid), dim3(LR_THREADS), 0, st, 1, P, rows, wpc);
    else if (rows <= 4) launch_k(lin_rows_kernel<T, 4>, dim3(grid), dim3(LR_THREADS), 0, st, 1, P, rows, wpc);
    else launch_k(lin_rows_kernel<T, 8>, dim3(grid), dim3(LR_THREADS), 0, st, 1, P, rows, wpc);
    return launch_ok("lin_rows");
}

// ---------------------------------------------------------------- tensor cores: the forward product and the data gradient
// on operands whose rows are whole vectors; N and K may be padded counts (w has c_out rows all the same)
nb_status tc_fwd(const nb_linear_plan_s* p, long long rows, const void* x, long long ld_x, const void* w, const float* bias, int act, const void* res, long long ld_res, void* z,
                 void* out, long long ld_out, int ci, int co, cudaStream_t st) {
    const TlCfg c = choose_rows(rows, co, ci, p->sms, 15.0 + (bias ? 3.0 : 0.0) + (act == NB_ACT_GELU ? 8.0 : act ? 4.5 : 0.0) + (z ? 4.0 : 0.0) + (res ? 4.0 : 0.0), 1.2, res ? 1000.0 : 0.0,
                                long_sum(p));
    TcLinParams P;
    memset(&P, 0, sizeof P);
    P.M = (int)rows; P.N = co; P.n_bias = p->d.c_out;
    P.bias = bias; P.act = act; P.has_in = res != nullptr; P.want_z = z != nullptr; P.res = res; P.ld_res = ld_res;
    const int np = pass_cols(c);
    if (!encode2(&P.tmA, p->d.dtype, x, rows, ci, ld_x, 64, 128) || !encode2(&P.tmB, p->d.dtype, w, p->d.c_out, ci, ci, 64, c.cg2 ? c.bn / 2 : c.bn) ||
        !encode2(&P.tmOut, p->d.dtype, out, rows, co, ld_out, np, 32) || (z && !encode2(&P.tmZ, p->d.dtype, z, rows, co, co, np, 32)) ||
        (res && !encode2(&P.tmIn, p->d.dtype, res, rows, co, ld_res, np, 32)))
        return fail(NB_ERR_CUDA, "cuTensorMapEncodeTiled failed");
    return run_tc<LIN_FWD>(p, c, P, st);
}
nb_status tc_data(const nb_linear_plan_s* p, long long rows, const void* dy, long long ld_dy, const void* w, const void* z_in, int act_in, const void* add, long long ld_add, void* dx,
                  long long ld_dx, int ci, int co, cudaStream_t st) {
    const TlCfg c = choose_rows(rows, ci, co, p->sms, 15.0 + (act_in == NB_ACT_GELU ? 24.0 : z_in ? 14.0 : 0.0) + (add ? 10.0 : 0.0), 1.0, 0.0, long_sum(p));
    TcLinParams P;
    memset(&P, 0, sizeof P);
    P.M = (int)rows; P.N = ci;
    P.act = act_in; P.add = add; P.ld_add = ld_add; P.has_in = z_in != nullptr;
    const int np = pass_cols(c);
    if (!encode2(&P.tmA, p->d.dtype, dy, rows, co, ld_dy, 64, 128) || !encode2(&P.tmB, p->d.dtype, w, co, ci, ci, 64, TL_KC) ||
        !encode2(&P.tmOut, p->d.dtype, dx, rows, ci, ld_dx, np, 32) || (z_in && !encode2(&P.tmIn, p->d.dtype, z_in, rows, ci, ci, np, 32)))
        return fail(NB_ERR_CUDA, "cuTensorMapEncodeTiled failed");
    return run_tc<LIN_DATA>(p, c, P, st);
}

// Padded copies in the workspace, one behind the other.
struct Padded {
    const nb_linear_plan_s* p;
    uint8_t* at;
    cudaStream_t stream;
    nb_status st = NB_OK;
    Padded(const nb_linear_plan_s* plan, long long, void* workspace, cudaStream_t s) : p(plan), at(static_cast<uint8_t*>(workspace)), stream(s) {}
    void* take(long long rows, int cols) {
        void* d = at;
        at += rows_bytes(rows, cols);
        return d;
    }
    const void* in(const void* src, long long ld, long long rows, int cols) {
        void* d = take(rows, cols);
        const long long n = rows * (round8(cols) / 8);
        launch_k(lin_pad_kernel, dim3((unsigned)std::min<long long>(ceil_div(n, 256), p->sms * 16)), dim3(256), 0, stream, 1, static_cast<const uint16_t*>(src), ld, rows, cols, round8(cols),
                 static_cast<uint16_t*>(d));
        if (st == NB_OK) st = launch_ok("lin_pad");
        return d;
    }
    nb_status out(const void* src, long long rows, int cols, void* dst, long long ld) {
        launch_k(lin_unpad_kernel, dim3((unsigned)std::min<long long>(ceil_div(rows, 8), p->sms * 16)), dim3(256), 0, stream, 1, static_cast<const uint16_t*>(src), round8(cols), rows, cols,
                 static_cast<uint16_t*>(dst), ld);
        return launch_ok("lin_unpad");
    }
};

nb_status check_call(const nb_linear_plan_s* plan, int64_t rows) {
    if (!plan) return fail(NB_ERR_INVALID_ARG, "plan is NULL");
    if (rows <= 0) return fail(NB_ERR_INVALID_ARG, "rows must be positive");
    if (rows >= 0x7fff0000LL) return fail(NB_ERR_UNSUPPORTED, "too many rows");
    return NB_OK;
}
nb_status check_matrix(const char* name, const void* p, int64_t* ld, int64_t cols, size_t es) {
    if (*ld == 0) *ld = cols;
    if (*ld < cols) return fail(NB_ERR_INVALID_ARG, "the pitch of %s is smaller than its row", name);
    if (reinterpret_cast<uintptr_t>(p) & (es - 1)) return fail(NB_ERR_ALIGNMENT, "%s is not aligned to its element size", name);
    return NB_OK;
}
nb_status check16(const char* name, const void* p) {
    if (reinterpret_cast<uintptr_t>(p) & 15u) return fail(NB_ERR_ALIGNMENT, "%s is not 16-byte aligned", name);
    return NB_OK;
}
bool vec4(const void* q, long long ld, long long cols, size_t es) { return !(reinterpret_cast<uintptr_t>(q) & (4 * es - 1)) && ld % 4 == 0 && cols % 4 == 0; }

}  // namespace

extern "C" {

nb_status nb_linear_plan_create(const nb_linear_desc* desc, int device, nb_linear_plan* out) {
    g_err.clear();
    if (!out) return fail(NB_ERR_INVALID_ARG, "out_plan is NULL");
    *out = nullptr;
    if (!desc) return fail(NB_ERR_INVALID_ARG, "desc is NULL");
    if (desc->struct_size != sizeof(nb_linear_desc)) return fail(NB_ERR_INVALID_ARG, "nb_linear_desc.struct_size is %u, expected %zu", desc->struct_size, sizeof(nb_linear_desc));
    if (desc->c_in <= 0 || desc->c_out <= 0 || desc->c_in > (1 << 24) || desc->c_out > (1 << 24)) return fail(NB_ERR_INVALID_ARG, "c_in and c_out must be in 1 .. 2^24");
    if (desc->dtype != NB_DTYPE_F32 && desc->dtype != NB_DTYPE_BF16 && desc->dtype != NB_DTYPE_F16) return fail(NB_ERR_INVALID_ARG, "unknown dtype %d", desc->dtype);
    if (desc->flags & ~NB_LINEAR_FLAG_FORCE_SIMT) return fail(NB_ERR_INVALID_ARG, "unknown flags %u", desc->flags);
    int sms = 0, major = 0;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess ||
        cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, device) != cudaSuccess) {
        cudaGetLastError();
        return fail(NB_ERR_CUDA, "cannot query device %d", device);
    }
    if (major != 10) return fail(NB_ERR_ARCH, "device %d is not compute capability 10.x", device);
    std::unique_ptr<nb_linear_plan_s> p(new (std::nothrow) nb_linear_plan_s);
    if (!p) return fail(NB_ERR_INTERNAL, "out of host memory");
    p->d = *desc;
    p->device = device;
    p->sms = std::max(sms, 2);
    DeviceGuard on_device(device);
    NB_CUDA_CHECK(cudaMalloc(&p->status, ST_WORDS * sizeof(int)));
    const cudaError_t e = cudaMemset(p->status, 0, ST_WORDS * sizeof(int));
    if (e != cudaSuccess) {
        cudaFree(p->status);
        return fail(NB_ERR_CUDA, "cudaMemset failed: %s", cudaGetErrorString(e));
    }
    *out = p.release();
    return NB_OK;
}

nb_status nb_linear_plan_destroy(nb_linear_plan p) {
    g_err.clear();
    if (!p) return NB_OK;
    {
        DeviceGuard on_device(p->device);
        if (p->status) cudaFree(p->status);
    }
    delete p;
    return NB_OK;
}

nb_status nb_linear_workspace_bytes(nb_linear_plan p, int64_t rows, size_t* bytes) {
    g_err.clear();
    NB_TRY(check_call(p, rows));
    if (!bytes) return fail(NB_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = workspace_for(p, rows);
    return NB_OK;
}

nb_status nb_linear_paths(nb_linear_plan p, int64_t rows, int32_t* paths3) {
    g_err.clear();
    NB_TRY(check_call(p, rows));
    if (!paths3) return fail(NB_ERR_INVALID_ARG, "paths3 is NULL");
    const int tc = tc_layer(p) || tc_padded(p, rows) ? 1 : 0;
    paths3[0] = few_rows(p, rows) ? 2 : tc;
    paths3[1] = paths3[2] = tc;
    return NB_OK;
}

nb_status nb_linear_poll_status(nb_linear_plan p, void* stream) {
    g_err.clear();
    if (!p) return fail(NB_ERR_INVALID_ARG, "plan is NULL");
    DeviceGuard on_device(p->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int host[ST_WORDS] = {0};
    NB_CUDA_CHECK(cudaMemcpyAsync(host, p->status, sizeof host, cudaMemcpyDeviceToHost, st));
    NB_CUDA_CHECK(cudaStreamSynchronize(st));
    if (host[ST_ERR] || host[ST_SAT]) {
        NB_CUDA_CHECK(cudaMemsetAsync(p->status, 0, sizeof host, st));
        NB_CUDA_CHECK(cudaStreamSynchronize(st));
    }
    if (host[ST_ERR]) return fail((nb_status)host[ST_ERR], "a kernel gave up a bounded wait (site %d, block %d)", host[ST_WHERE], host[ST_DETAIL]);
    if (host[ST_SAT]) fail(NB_OK, "%d fp16 stores of the products' results saturated or held a NaN", host[ST_SAT]);
    return NB_OK;
}

nb_status nb_linear_fwd(nb_linear_plan p, int64_t rows, const void* x, int64_t ld_x, const void* w, const float* bias, int32_t act, const void* res, int64_t ld_res, void* z,
                        void* out, int64_t ld_out, void* workspace, size_t workspace_bytes, void* stream) {
    g_err.clear();
    NB_TRY(check_call(p, rows));
    if (!x || !w || !out) return fail(NB_ERR_INVALID_ARG, "x, w and out must not be NULL");
    if (act < NB_ACT_NONE || act > NB_ACT_GELU) return fail(NB_ERR_INVALID_ARG, "unknown act %d", act);
    const size_t es = size_of(p->d.dtype);
    const int64_t ci = p->d.c_in, co = p->d.c_out;
    NB_TRY(check_matrix("x", x, &ld_x, ci, es));
    NB_TRY(check_matrix("out", out, &ld_out, co, es));
    if (res) NB_TRY(check_matrix("res", res, &ld_res, co, es));
    NB_TRY(check16("w", w));
    NB_TRY(check16("bias", bias));
    if (reinterpret_cast<uintptr_t>(z) & (es - 1)) return fail(NB_ERR_ALIGNMENT, "z is not aligned to its element size");
    NB_TRY(check_ws(workspace, workspace_bytes, workspace_for(p, rows)));
    DeviceGuard on_device(p->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    LinArgs A;
    memset(&A, 0, sizeof A);
    A.a = x; A.lda = ld_x; A.b = w; A.ldb = ci;
    A.M = rows; A.N = co; A.K = ci;
    A.status = p->status; A.bias = bias; A.act = act; A.add = res; A.ld_add = ld_res; A.z = z; A.out = out; A.ld_out = ld_out;
    if (few_rows(p, rows) && whole16(x, ld_x, es)) {
        if (p->d.dtype == NB_DTYPE_F32) return run_rows<float>(p, A, (int)rows, st);
        if (p->d.dtype == NB_DTYPE_BF16) return run_rows<__nv_bfloat16>(p, A, (int)rows, st);
        return run_rows<__half>(p, A, (int)rows, st);
    }
    if (tc_layer(p) && whole16(x, ld_x, es) && whole16(out, ld_out, es) && (!res || whole16(res, ld_res, es)) && whole16(z, co, es))
        return tc_fwd(p, rows, x, ld_x, w, bias, act, res, ld_res, z, out, ld_out, (int)ci, (int)co, st);
    if (tc_padded(p, rows)) {
        Padded S(p, rows, workspace, st);
        const int ci8 = round8((int)ci), co8 = round8((int)co);
        const void* xs = S.in(x, ld_x, rows, (int)ci);
        const void* wp = S.in(w, ci, co, (int)ci);
        const void* rs = res ? S.in(res, ld_res, rows, (int)co) : nullptr;
        void *os = S.take(rows, (int)co), *zs = z ? S.take(rows, (int)co) : nullptr;
        NB_TRY(S.st);
        NB_TRY(tc_fwd(p, rows, xs, ci8, wp, bias, act, rs, co8, zs, os, co8, ci8, co8, st));
        if (z) NB_TRY(S.out(zs, rows, (int)co, z, co));
        return S.out(os, rows, (int)co, out, ld_out);
    }
    return run_simt_any<LIN_FWD>(p, A, simt_cfg(A.M, A.N, A.K, p->sms, false), vec4(x, ld_x, ci, es) && vec4(w, ci, ci, es), workspace, st);
}

nb_status nb_linear_bwd_data(nb_linear_plan p, int64_t rows, const void* dy, int64_t ld_dy, const void* w, const void* z_in, int32_t act_in, const void* add, int64_t ld_add,
                             void* dx, int64_t ld_dx, void* workspace, size_t workspace_bytes, void* stream) {
    g_err.clear();
    NB_TRY(check_call(p, rows));
    if (!dy || !w || !dx) return fail(NB_ERR_INVALID_ARG, "dy, w and dx must not be NULL");
    if (act_in < NB_ACT_NONE || act_in > NB_ACT_GELU) return fail(NB_ERR_INVALID_ARG, "unknown act_in %d", act_in);
    if ((act_in == NB_ACT_NONE) != !z_in) return fail(NB_ERR_INVALID_ARG, "z_in must be NULL exactly when act_in is NB_ACT_NONE");
    const size_t es = size_of(p->d.dtype);
    const int64_t ci = p->d.c_in, co = p->d.c_out;
    NB_TRY(check_matrix("dy", dy, &ld_dy, co, es));
    NB_TRY(check_matrix("dx", dx, &ld_dx, ci, es));
    if (add) NB_TRY(check_matrix("add", add, &ld_add, ci, es));
    NB_TRY(check16("w", w));
    if (reinterpret_cast<uintptr_t>(z_in) & (es - 1)) return fail(NB_ERR_ALIGNMENT, "z_in is not aligned to its element size");
    NB_TRY(check_ws(workspace, workspace_bytes, workspace_for(p, rows)));
    DeviceGuard on_device(p->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (tc_layer(p) && whole16(dy, ld_dy, es) && whole16(dx, ld_dx, es) && (!add || whole16(add, ld_add, es)) && whole16(z_in, ci, es))
        return tc_data(p, rows, dy, ld_dy, w, z_in, act_in, add, ld_add, dx, ld_dx, (int)ci, (int)co, st);
    if (tc_padded(p, rows)) {
        Padded S(p, rows, workspace, st);
        const int ci8 = round8((int)ci), co8 = round8((int)co);
        const void* ds = S.in(dy, ld_dy, rows, (int)co);
        const void* wp = S.in(w, ci, co, (int)ci);
        const void* zs = z_in ? S.in(z_in, ci, rows, (int)ci) : nullptr;
        const void* as = add ? S.in(add, ld_add, rows, (int)ci) : nullptr;
        void* xs = S.take(rows, (int)ci);
        NB_TRY(S.st);
        NB_TRY(tc_data(p, rows, ds, co8, wp, zs, act_in, as, ci8, xs, ci8, ci8, (int)co, st));
        return S.out(xs, rows, (int)ci, dx, ld_dx);
    }
    LinArgs A;
    memset(&A, 0, sizeof A);
    A.a = dy; A.lda = ld_dy; A.b = w; A.ldb = ci;
    A.M = rows; A.N = ci; A.K = co;
    A.status = p->status; A.act = act_in; A.zin = z_in; A.add = add; A.ld_add = ld_add; A.out = dx; A.ld_out = ld_dx;
    return run_simt_any<LIN_DATA>(p, A, simt_cfg(A.M, A.N, A.K, p->sms, false), vec4(dy, ld_dy, co, es) && vec4(w, ci, ci, es), workspace, st);
}

nb_status nb_linear_bwd_weight(nb_linear_plan p, int64_t rows, const void* x, int64_t ld_x, const void* dy, int64_t ld_dy, float* dw, float* dbias, void* workspace,
                               size_t workspace_bytes, void* stream) {
    g_err.clear();
    NB_TRY(check_call(p, rows));
    if (!x || !dy || !dw) return fail(NB_ERR_INVALID_ARG, "x, dy and dw must not be NULL");
    const size_t es = size_of(p->d.dtype);
    const int64_t ci = p->d.c_in, co = p->d.c_out;
    NB_TRY(check_matrix("x", x, &ld_x, ci, es));
    NB_TRY(check_matrix("dy", dy, &ld_dy, co, es));
    NB_TRY(check16("dw", dw));
    NB_TRY(check16("dbias", dbias));
    NB_TRY(check_ws(workspace, workspace_bytes, workspace_for(p, rows)));
    DeviceGuard on_device(p->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    const long long n1 = co * ci;
    auto sums = [&](const float* p1, int s1, const float* p2, int s2, bool more = false) -> nb_status {
        const long long work = std::max(s1 ? ceil_div(n1, n1 % 4 ? 1 : 4) : 0LL, s2 ? (long long)co : 0LL);
        launch_k(lin_weight_sums_kernel, dim3((unsigned)std::min<long long>(ceil_div(work, 256), p->sms * 8)), dim3(256), 0, st, 1, p1, s1, n1, dw, p2, s2, (int)co, dbias, (int)more);
        return launch_ok("lin_weight_sums");
    };
    const bool whole = tc_layer(p) && whole16(x, ld_x, es) && whole16(dy, ld_dy, es), padded = !whole && tc_padded(p, rows);
    if (whole || padded) {
        Padded S(p, rows, workspace, st);
        const int ci8 = round8((int)ci);
        const void *xs = x, *ds = dy;
        int64_t lx = ld_x, ld = ld_dy;
        if (padded) {
            xs = S.in(x, ld_x, rows, (int)ci);
            ds = S.in(dy, ld_dy, rows, (int)co);
            NB_TRY(S.st);
            lx = ci8;
            ld = round8((int)co);
        }
        const TlCfg c = choose_weight(co, ci8, rows, p->sms);
        TcLinParams P;
        memset(&P, 0, sizeof P);
        P.M = (int)co; P.N = ci8;
        const bool sliced = c.splits > 1 || padded;
        const size_t one = (size_t)co * ci8;
        float* part = sliced ? reinterpret_cast<float*>(S.at) : dw;
        float* db = reinterpret_cast<float*>(S.at + (sliced ? align_up(c.splits * one * 4, 256) : 0));
        int db_parts = c.splits * c.n_tiles;
        if (dbias && !db_in_tile(c)) NB_TRY(run_colsum_any(p, ds, ld, rows, db, &db_parts, st));  // (first: what it reads may wait in L2)
        else if (dbias && db_parts == 1) db = dbias;
        P.db = dbias && db_in_tile(c) ? db : nullptr;
        const cuuint64_t dims[3] = {(cuuint64_t)ci8, (cuuint64_t)co, (cuuint64_t)c.splits}, strides[2] = {(cuuint64_t)ci8 * 4, (cuuint64_t)one * 4};
        const cuuint32_t box[3] = {32, 32, 1};
        if (!encode2(&P.tmA, p->d.dtype, ds, rows, padded ? ld : co, ld, 64, TL_KC) || !encode2(&P.tmB, p->d.dtype, xs, rows, ci8, lx, 64, TL_KC) ||
            !encode(&P.tmOut, NB_DTYPE_F32, part, 3, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B, false))
            return fail(NB_ERR_CUDA, "cuTensorMapEncodeTiled failed");
        NB_TRY(run_tc<LIN_WEIGHT>(p, c, P, st));
        const bool add_db = dbias && db != dbias;
        if (padded) {
            launch_k(lin_weight_unpad_kernel, dim3((unsigned)std::min<long long>(ceil_div(n1, 256), p->sms * 8)), dim3(256), 0, st, 1, (const float*)part, c.splits, (long long)co, (int)ci, ci8,
                     dw);
            NB_LAUNCH_OK("lin_weight_unpad");
            return add_db ? sums(nullptr, 0, db, db_parts) : NB_OK;
        }
        return c.splits > 1 || add_db ? sums(part, c.splits > 1 ? c.splits : 0, db, add_db ? db_parts : 0) : NB_OK;
    }
    LinArgs A;
    memset(&A, 0, sizeof A);
    A.a = dy; A.lda = ld_dy; A.b = x; A.ldb = ld_x;
    A.M = co; A.N = ci; A.K = rows;
    A.ld_out = ci;
    const SimtCfg c = simt_cfg(co, ci, rows, p->sms, true);
    const bool vec = vec4(dy, ld_dy, co, es) && vec4(x, ld_x, ci, es);
    const int group = weight_group(c, co, ci, p->sms);
    float* part = static_cast<float*>(workspace);
    float* db = reinterpret_cast<float*>(ws + (c.slices > 1 ? align_up((size_t)group * n1 * 4, 256) : 0));
    int parts = 0;
    for (int s0 = 0; s0 < c.slices; s0 += group) {
        SimtCfg g = c;
        g.slices = std::min(group, c.slices - s0);
        const long long k0 = s0 * c.kslice;
        A.a = static_cast<const char*>(dy) + k0 * ld_dy * (long long)es;
        A.b = static_cast<const char*>(x) + k0 * ld_x * (long long)es;
        A.K = std::min<long long>(rows - k0, g.slices * c.kslice);
        A.out = c.slices > 1 ? part : dw;  // (where a group is one slice; more go to `part` by themselves)
        NB_TRY(run_simt_any<LIN_WEIGHT>(p, A, g, vec, workspace, st));
        if (s0 == 0 && dbias) NB_TRY(run_colsum_any(p, dy, ld_dy, rows, db, &parts, st));
        if (c.slices > 1 || parts) NB_TRY(sums(part, c.slices > 1 ? g.slices : 0, db, s0 ? 0 : parts, s0 > 0));
    }
    return NB_OK;
}

nb_status nb_act_bwd(int32_t dtype, int64_t n, int32_t act, const void* dy, const void* z, void* dz, void* stream) {
    g_err.clear();
    if (dtype != NB_DTYPE_F32 && dtype != NB_DTYPE_BF16 && dtype != NB_DTYPE_F16) return fail(NB_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (n <= 0) return fail(NB_ERR_INVALID_ARG, "n must be positive");
    if (act != NB_ACT_SILU && act != NB_ACT_GELU) return fail(NB_ERR_INVALID_ARG, "act %d has no gradient pass", act);
    if (!dy || !z || !dz) return fail(NB_ERR_INVALID_ARG, "dy, z and dz must not be NULL");
    const uintptr_t bits = reinterpret_cast<uintptr_t>(dy) | reinterpret_cast<uintptr_t>(z) | reinterpret_cast<uintptr_t>(dz);
    if (bits & (size_of(dtype) - 1)) return fail(NB_ERR_ALIGNMENT, "a pointer is not aligned to its element size");
    const bool vec = !(bits & 15u);
    int dev = 0, sms = 148;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const long long items = vec ? ceil_div(n, 16 / (long long)size_of(dtype)) : n;
    const dim3 grid((unsigned)std::min<long long>(ceil_div(items, 256), sms * 16LL));
#define NB_ACTB(T)                                                                                                                                           \
    if (vec) launch_k(lin_act_bwd_kernel<T, true>, grid, dim3(256), 0, st, 1, static_cast<const T*>(dy), static_cast<const T*>(z), static_cast<T*>(dz), (long long)n, (int)act); \
    else launch_k(lin_act_bwd_kernel<T, false>, grid, dim3(256), 0, st, 1, static_cast<const T*>(dy), static_cast<const T*>(z), static_cast<T*>(dz), (long long)n, (int)act);
    if (dtype == NB_DTYPE_F32) { NB_ACTB(float) }
    else if (dtype == NB_DTYPE_BF16) { NB_ACTB(__nv_bfloat16) }
    else { NB_ACTB(__half) }
#undef NB_ACTB
    return launch_ok("lin_act_bwd");
}

}  // extern "C"
