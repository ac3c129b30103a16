// Matrix products of MLP layers on the tensor cores (see include/nb_linear.h): D[m][n] = sum_k A(m,k) B(n,k) with 16-bit operands,
// fetched by TMA in the 128-byte swizzle, multiplied by tcgen05.mma into fp32 accumulators in TMEM and finished by eight
// epilogue warps.
//   LIN_FWD     m = row,   n = c_out, k = c_in    A = x  (k contiguous: K-major),  B = w (K-major)
//   LIN_DATA    m = row,   n = c_in,  k = c_out   A = dy (K-major),                B = w (n contiguous: MN-major)
//   LIN_WEIGHT  m = c_out, n = c_in,  k = row     A = dy (m contiguous: MN-major), B = x (MN-major)
// No operand is rearranged in memory.  Tiles are 128 x BN a CTA or, with CG2, 256 x BN a pair of CTAs (cta_group::2: each has 128
// rows and fetches its own rows of A and half of B); the forward and data-gradient kernels are persistent, with two accumulator
// sets so that the epilogue of a tile runs beside the products of the next; the weight gradient gives every tile a slice of the
// rows and adds the slices in a second kernel.  No multicast; every wait on an mbarrier is bounded.
#pragma once
#include "linear.cuh"
#include "tc_common.cuh"

namespace nbcbs {

constexpr int TL_THREADS = 320;  // warp 0: TMA producer, warp 1: MMA issuer and owner of TMEM, warps 2-9: epilogue
constexpr int TL_KC = 64;        // k of a stage: 128 bytes of a 16-bit K-major operand
constexpr uint32_t TL_BLK = 64 * 128;         // an MN-major block: 64 m (or n) by 64 k
constexpr uint32_t TL_A_BYTES = 128 * 128;    // A rows of a CTA by 64 k
constexpr int TL_STG = 4096;     // staging buffer of an epilogue warp: 32 rows of 128 bytes; it has two
constexpr int TL_CHUNK = 16;                    // k-blocks after which a weight gradient's sums leave the tensor cores
// ... of a forward product or data gradient: 1024 additions are off by 9e-5 at most, 8192 by 7e-4, both 0.18 of half a step of the type.
constexpr int TL_LONG_F16 = 256, TL_LONG_BF16 = 2048;
constexpr uint32_t TL_ONES_BYTES = 4096;

struct TcLinParams {
    CUtensorMap tmA, tmB, tmOut, tmZ, tmIn;  // tmIn: the residual (forward), z_in (data gradient)
    int M, N, kblocks;  // k-blocks of TL_KC
    int chunk;          // LONG: k-blocks after which the sums leave the tensor cores
    int n_bias;         // columns that have a bias (N may be padded)
    int BN, m_tiles, n_tiles, group_m;
    int stages, acc_stride;
    int nblkB;                     // MN-major: 64-column blocks of this CTA's part of B
    uint32_t b_bytes, idesc;
    // epilogue
    const float* bias;
    int act;
    int has_in, want_z;
    const void* res;  // forward with z: the residual
    long long ld_res;
    const void* add;  // data gradient: the other branch's gradient
    long long ld_add;
    // weight gradient
    int splits, kb_per_split;
    float* db;  // partial sums of dbias [splits * n_tiles][M], or NULL
    uint32_t idesc_ones;
    int* status;
};

// Order of the tiles: group_m row tiles by all column tiles at a time, so that what is in flight at once shares both operands in L2.
__device__ __forceinline__ void tl_tile(const TcLinParams& p, int tile, int& mt, int& nt) {
    const int per = p.group_m * p.n_tiles, g = tile / per, r = tile - g * per;
    const int first = g * p.group_m, rows = min(p.group_m, p.m_tiles - first);
    nt = r / rows;
    mt = first + r - nt * rows;
}

// Eight consecutive 16-bit elements as four pairs.
template <typename T> __device__ __forceinline__ float2 tl_pair(const uint4& v, int j) {
    const uint32_t w = j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w;
    return pair_to_f32<T>(reinterpret_cast<const T*>(&w));
}

// One pass of the epilogue by a warp: NP (64 or 32) accumulator columns of its 32 rows become results.  A lane has one row's.  They go
// through one of the warp's staging buffers (rows of 2*NP bytes in the swizzle of that width) and leave as a TMA store; a residual or
// z_in has come into the same buffer by a TMA load.  Both run beside the arithmetic.
template <typename T, int KIND, int NP, bool LONG> struct TlPass {
    static __device__ __forceinline__ uint4* piece(uint8_t* stg, int lane, int j) {
        return reinterpret_cast<uint4*>(stg + lane * (NP * 2) + (NP == 64 ? (j ^ (lane & 7)) : (j ^ ((lane >> 1) & 3))) * 16);
    }
    // (fp16: a lane whose part of a row of the matrix holds a saturated value counts it)
    static __device__ __forceinline__ void stage(const TcLinParams& p, uint8_t* stg, int lane, int row0, const float2 (&v)[NP / 2]) {
        int sat = 0;
#pragma unroll
        for (int j = 0; j < NP / 8; ++j)
            *piece(stg, lane, j) = make_uint4(pack2<T>(v[4 * j].x, v[4 * j].y, &sat), pack2<T>(v[4 * j + 1].x, v[4 * j + 1].y, &sat),
                                              pack2<T>(v[4 * j + 2].x, v[4 * j + 2].y, &sat), pack2<T>(v[4 * j + 3].x, v[4 * j + 3].y, &sat));
        if ((sat & (int)0x80008000u) && row0 + lane < p.M) atomicAdd(p.status + ST_SAT, 1);
    }
    // this row's pieces of a matrix [M][N], straight from memory
    static __device__ __forceinline__ void direct(const TcLinParams& p, uint4 (&d)[NP / 8], const void* base, long long ld, long long row, int col) {
        const T* q = static_cast<const T*>(base) + row * ld + col;
#pragma unroll
        for (int j = 0; j < NP / 8; ++j) d[j] = row < p.M && col + 8 * j < p.N ? *reinterpret_cast<const uint4*>(q + 8 * j) : make_uint4(0u, 0u, 0u, 0u);
    }
    static __device__ __forceinline__ void send(const CUtensorMap* tm, uint8_t* stg, int lane, int col, int row0) {
        ptx::fence_async_smem();
        __syncwarp();
        if (lane == 0) {
            ptx::tma_store_2d(tm, stg, col, row0);
            ptx::tma_store_commit();
        }
    }
    // `in_here`: the pass's input lies in buffer `stg`; `other` gives z a buffer; `sum`: LONG, what earlier chunks of k have given
    template <class Release, class Other>
    static __device__ __forceinline__ void run(const TcLinParams& p, uint32_t taddr, int lane, int row0, int col, const float* bias, uint8_t* stg, bool in_here, const float2* sum, Release release, Other other) {
        uint32_t r[NP];
#pragma unroll
        for (int h = 0; h < NP / 32; ++h) ptx::tmem_ld_32x32b_x32(taddr + 32u * h, r + 32 * h);
        uint4 in[NP / 8];
        if (in_here) {
#pragma unroll
            for (int j = 0; j < NP / 8; ++j) in[j] = *piece(stg, lane, j);
        } else if (KIND == LIN_FWD && p.has_in) {
            direct(p, in, p.res, p.ld_res, (long long)row0 + lane, col);
        }
        ptx::tmem_ld_wait();
        release();
        float2 v[NP / 2];
#pragma unroll
        for (int j = 0; j < NP / 2; ++j) {
            v[j] = make_float2(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
            if (LONG) v[j] = add2(sum[j], v[j]);
        }
        if (KIND == LIN_FWD) {
            if (p.bias) {
#pragma unroll
                for (int j = 0; j < NP / 4; ++j) {
                    const float4 b = *reinterpret_cast<const float4*>(bias + 4 * j);  // (shared memory, one address a warp)
                    v[2 * j] = add2(v[2 * j], make_float2(b.x, b.y));
                    v[2 * j + 1] = add2(v[2 * j + 1], make_float2(b.z, b.w));
                }
            }
            if (p.want_z) {
                uint8_t* zs = other();
                stage(p, zs, lane, row0, v);
                send(&p.tmZ, zs, lane, col, row0);
            }
            if (p.act == NB_ACT_GELU) {
#pragma unroll
                for (int j = 0; j < NP / 2; ++j) v[j] = lin_act2(v[j], NB_ACT_GELU);
            } else if (p.act == NB_ACT_SILU) {
#pragma unroll
                for (int j = 0; j < NP / 2; ++j) v[j] = lin_act2(v[j], NB_ACT_SILU);
            }
            if (p.has_in) {
#pragma unroll
                for (int j = 0; j < NP / 2; ++j) v[j] = add2(v[j], tl_pair<T>(in[j / 4], j & 3));
            }
        } else {
            if (p.add) {
                uint4 ad[NP / 8];
                direct(p, ad, p.add, p.ld_add, (long long)row0 + lane, col);
#pragma unroll
                for (int j = 0; j < NP / 2; ++j) v[j] = add2(v[j], tl_pair<T>(ad[j / 4], j & 3));
            }
            if (p.has_in) {
                if (p.act == NB_ACT_GELU) {
#pragma unroll
                    for (int j = 0; j < NP / 2; ++j) v[j] = mul2(v[j], lin_act_grad2(tl_pair<T>(in[j / 4], j & 3), NB_ACT_GELU));
                } else {
#pragma unroll
                    for (int j = 0; j < NP / 2; ++j) v[j] = mul2(v[j], lin_act_grad2(tl_pair<T>(in[j / 4], j & 3), NB_ACT_SILU));
                }
            }
        }
        if (KIND == LIN_FWD && p.want_z) {
            if (lane == 0) ptx::tma_store_wait_read<1>();
            __syncwarp();
        }
        stage(p, stg, lane, row0, v);
        send(&p.tmOut, stg, lane, col, row0);
        __syncwarp();  // (the next accumulator load wants the whole warp)
    }
};

template <typename T, int KIND, bool CG2, int NP, bool LONG> __global__ void __launch_bounds__(TL_THREADS, 1) tc_linear_kernel(const __grid_constant__ TcLinParams p) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* sA = smem;
    uint8_t* sB = sA + (size_t)p.stages * TL_A_BYTES;
    uint8_t* stg = sB + (size_t)p.stages * p.b_bytes;     // [8 warps][2]
    uint8_t* ones = stg + (size_t)16 * TL_STG;            // weight gradient with dbias
    float* sbias = reinterpret_cast<float*>(ones);        // forward: a warp's 128 columns of the bias
    uint64_t* bars = reinterpret_cast<uint64_t*>(ones + (KIND == LIN_WEIGHT ? (int)TL_ONES_BYTES : KIND == LIN_FWD ? 8 * 512 : 0));
    uint64_t* full = bars;
    uint64_t* empty = full + p.stages;
    uint64_t* tfull = empty + p.stages;  // [2]
    uint64_t* tempty = tfull + 2;        // [2]
    uint64_t* infull = tempty + 2;       // [8 warps][2]
    uint64_t* drain = infull + 16;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    constexpr bool A_MN = KIND == LIN_WEIGHT, B_MN = KIND != LIN_FWD;

    pdl_launch_dependents();
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t rank = CG2 ? (blockIdx.x & 1u) : 0u;
    const int worker = CG2 ? (int)(blockIdx.x >> 1) : (int)blockIdx.x, nworkers = CG2 ? (int)(gridDim.x >> 1) : (int)gridDim.x;
    const int tiles = p.m_tiles * p.n_tiles * (KIND == LIN_WEIGHT ? p.splits : 1);
    constexpr int TM = CG2 ? 256 : 128;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            ptx::mbar_init(full + s, 1);
            ptx::mbar_init(empty + s, 1);
        }
        for (int i = 0; i < 2; ++i) {
            ptx::mbar_init(tfull + i, 1);
            ptx::mbar_init(tempty + i, CG2 ? 16 : 8);  // one arrival per epilogue warp (of both CTAs)
        }
        for (int i = 0; i < 16; ++i) ptx::mbar_init(infull + i, 1);
        ptx::mbar_init(drain, 1);
        *abort_flag = 0;
        ptx::fence_mbar_init();
    }
    if (lane == 0 && warp == 0) {
        ptx::prefetch_tmap(&p.tmA);
        ptx::prefetch_tmap(&p.tmB);
    }
    if (lane == 0 && warp == 2) {
        ptx::prefetch_tmap(&p.tmOut);
        if (p.want_z) ptx::prefetch_tmap(&p.tmZ);
        if (p.has_in) ptx::prefetch_tmap(&p.tmIn);
    }
    if (KIND == LIN_WEIGHT && p.db && warp >= 2) {
        // 16 columns of ones as an operand: the same whatever the layout
        const uint32_t w = (p.idesc >> 7) & 1u ? 0x3f803f80u : 0x3c003c00u;  // (bf16 or fp16, as the descriptor says)
        for (uint32_t i = threadIdx.x - 64; i < TL_ONES_BYTES / 4; i += TL_THREADS - 64) reinterpret_cast<uint32_t*>(ones)[i] = w;
        ptx::fence_async_smem();
    }
    if (warp == 1) {
        if (CG2) {
            ptx::tmem_alloc_cg2(tmem_slot, 512);
            ptx::tmem_relinquish_cg2();
        } else {
            ptx::tmem_alloc(tmem_slot, 512);
            ptx::tmem_relinquish();
        }
    }
    ptx::tc_fence_before();
    if (CG2) ptx::cluster_sync_all(); else __syncthreads();  // barriers of both CTAs are initialised before any remote arrive
    ptx::tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    // The tensor cores add to their accumulator with truncation: 1024 additions (16384 rows) left a weight gradient 1.9e-5 off, relative
    // to its norm, always towards zero.  So a weight gradient's sums leave them every TL_CHUNK k-blocks (64 additions) and are added in
    // fp32 registers, beside the next chunk's products in the other accumulator set; 1e-6 is left.  Sums of positive terms lose most, 8.5e-8
    // of the sum at every addition; a 16-bit result sees that when there are thousands, and LONG products do the same every p.chunk k-blocks.
    const int chunk = KIND == LIN_WEIGHT ? TL_CHUNK : LONG ? p.chunk : p.kblocks;
    // a work item: a tile and, for the weight gradient, a slice of the rows
    auto item = [&](int i, int& mt, int& nt, int& split, int& kb0, int& kb1) {
        split = 0;
        if (KIND == LIN_WEIGHT) {  // slices fastest: what runs at once reads different rows of all channels
            split = i % p.splits;
            i /= p.splits;
        }
        tl_tile(p, i, mt, nt);
        kb0 = KIND == LIN_WEIGHT ? split * p.kb_per_split : 0;
        kb1 = KIND == LIN_WEIGHT ? min(p.kblocks, kb0 + p.kb_per_split) : p.kblocks;
    };

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer (the warp runs converged, `leader` issues)
        const uint32_t leader = ptx::elect_one() ? 1u : 0u;
        int s = 0;
        uint32_t ph = 0;
        long long issued = 0;
        bool ok = true;
        const int bn_own = CG2 ? p.BN / 2 : p.BN;
        const uint32_t a_u32 = ptx::smem_u32(sA), b_u32 = ptx::smem_u32(sB);
        const uint32_t full_u32 = CG2 ? ptx::mapa_u32(ptx::smem_u32(full), 0u) : ptx::smem_u32(full);  // pairs: counted at rank 0
        const uint32_t tx = TL_A_BYTES + (B_MN ? (uint32_t)p.nblkB * TL_BLK : (uint32_t)bn_own * 128u);
        auto load = [&](uint32_t dst, const CUtensorMap* tm, uint32_t bar, int c0, int c1) {
            if (CG2) ptx::tma_load_2d_cg2_if(leader, dst, tm, bar, c0, c1); else ptx::tma_load_2d_u32_if(leader, dst, tm, bar, c0, c1);
        };
        pdl_wait();
        for (int i = worker; ok && i < tiles; i += nworkers) {
            int mt, nt, split, kb0, kb1;
            item(i, mt, nt, split, kb0, kb1);
            const int m0 = mt * TM + (int)rank * 128, n0 = nt * p.BN + (int)rank * bn_own;
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!wait_bar_fast(empty + s, ph ^ 1u, abort_flag, p.status, 21)) {
                    ok = false;
                    break;
                }
                const uint32_t bar = full_u32 + 8u * (uint32_t)s, a = a_u32 + (uint32_t)s * TL_A_BYTES, b = b_u32 + (uint32_t)s * p.b_bytes;
                if (!CG2) ptx::mbar_expect_tx_u32_if(leader, bar, tx);
                else if (rank == 0) ptx::mbar_expect_tx_u32_if(leader, ptx::smem_u32(full) + 8u * (uint32_t)s, 2u * tx);
                const int k = kb * TL_KC;
                if (A_MN) {
                    load(a, &p.tmA, bar, m0, k);
                    load(a + TL_BLK, &p.tmA, bar, m0 + 64, k);
                } else {
                    load(a, &p.tmA, bar, k, m0);
                }
                if (B_MN) {
                    for (int j = 0; j < p.nblkB; ++j) load(b + (uint32_t)j * TL_BLK, &p.tmB, bar, n0 + 64 * j, k);
                } else {
                    load(b, &p.tmB, bar, k, n0);
                }
                ++issued;
                if (++s == p.stages) {
                    s = 0;
                    ph ^= 1u;
                }
            }
        }
        if (!ok) {
            // Gave up: wait (bounded) for the loads still in flight so that nothing lands after the CTA has exited.
            const int back = issued < (long long)p.stages ? (int)issued : p.stages;
            for (int b = 0; b < back; ++b) {
                s = (s == 0) ? p.stages - 1 : s - 1;
                if (s == p.stages - 1) ph ^= 1u;
                for (int j = 0; j < 100000 && !ptx::mbar_try_wait(full + s, ph); ++j) {
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer (in a pair that of rank 0)
        const uint32_t leader = ptx::elect_one() ? 1u : 0u;
        if (rank == 0) {
            int s = 0, acc = 0;
            uint32_t ph = 0, acc_ph = 0;
            bool ok = true;
            // K-major: rows of 128 bytes, 8 rows a group (SBO 1024), a K = 16 step is 32 bytes.  MN-major: 8 k rows of 128 bytes a group
            // (SBO 1024), the next 64 m (n) one block behind (LBO), a K = 16 step is two groups.
            const uint64_t da0 = ptx::make_smem_desc(ptx::smem_u32(sA), A_MN ? TL_BLK : 16u, 1024, ptx::kSwizzle128);
            const uint64_t db0 = ptx::make_smem_desc(ptx::smem_u32(sB), B_MN ? TL_BLK : 16u, 1024, ptx::kSwizzle128);
            const uint64_t d1 = KIND == LIN_WEIGHT ? ptx::make_smem_desc(ptx::smem_u32(ones), TL_BLK, 1024, ptx::kSwizzle128) : 0ull;
            constexpr uint64_t ka = A_MN ? 128 : 2, kb_ = B_MN ? 128 : 2;
            const uint64_t a_stage = TL_A_BYTES >> 4, b_stage = p.b_bytes >> 4;
            const uint32_t empty_u32 = ptx::smem_u32(empty), tfull_u32 = ptx::smem_u32(tfull);
            auto mma = [&](uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
                if (CG2) ptx::umma_f16_cg2_if(leader, d, a, b, idesc, accumulate); else ptx::umma_f16_if(leader, d, a, b, idesc, accumulate);
            };
            uint64_t da = da0, db = db0;
            for (int i = worker; ok && i < tiles; i += nworkers) {
                int mt, nt, split, kb0, kb1;
                item(i, mt, nt, split, kb0, kb1);
                for (int c0 = kb0; ok && c0 < kb1; c0 += chunk) {
                    const int c1 = min(kb1, c0 + chunk);
                    if (!wait_bar_fast(tempty + acc, acc_ph ^ 1u, abort_flag, p.status, 22)) {
                        ok = false;
                        break;
                    }
                    ptx::tc_fence_after();
                    const uint32_t dt = tmem_base + (uint32_t)(acc * p.acc_stride);
                    uint32_t accumulate = 0, accumulate1 = 0;
                    for (int kb = c0; kb < c1; ++kb) {
                        if (!wait_bar_fast(full + s, ph, abort_flag, p.status, 23)) {
                            ok = false;
                            break;
                        }
                        ptx::tc_fence_after();
                        mma(dt, da, db, p.idesc, accumulate);
                        mma(dt, da + ka, db + kb_, p.idesc, 1u);
                        mma(dt, da + 2 * ka, db + 2 * kb_, p.idesc, 1u);
                        mma(dt, da + 3 * ka, db + 3 * kb_, p.idesc, 1u);
                        accumulate = 1u;
                        if (KIND == LIN_WEIGHT && p.db && kb % p.n_tiles == nt) {
                            // sums of A over k: a product with columns of ones, whose share each column tile takes of the k-blocks in turn
                            mma(dt + (uint32_t)p.BN, da, d1, p.idesc_ones, accumulate1);
                            mma(dt + (uint32_t)p.BN, da + ka, d1, p.idesc_ones, 1u);
                            mma(dt + (uint32_t)p.BN, da + 2 * ka, d1, p.idesc_ones, 1u);
                            mma(dt + (uint32_t)p.BN, da + 3 * ka, d1, p.idesc_ones, 1u);
                            accumulate1 = 1u;
                        }
                        if (CG2) ptx::umma_commit_cg2_mc_if(leader, empty_u32 + 8u * (uint32_t)s, 3); else ptx::umma_commit_u32_if(leader, empty_u32 + 8u * (uint32_t)s);
                        da += a_stage;
                        db += b_stage;
                        if (++s == p.stages) {
                            s = 0;
                            ph ^= 1u;
                            da = da0;
                            db = db0;
                        }
                    }
                    if (!ok) break;
                    if (CG2) ptx::umma_commit_cg2_mc_if(leader, tfull_u32 + 8u * (uint32_t)acc, 3); else ptx::umma_commit_u32_if(leader, tfull_u32 + 8u * (uint32_t)acc);
                    acc ^= 1;
                    if (acc == 0) acc_ph ^= 1u;
                }
            }
            // Make sure every MMA issued by this thread has retired before TMEM is released.
            if (CG2) ptx::umma_commit_cg2_if(leader, ptx::smem_u32(drain)); else ptx::umma_commit_u32_if(leader, ptx::smem_u32(drain));
            for (int j = 0; j < 4000000 && !ptx::mbar_try_wait(drain, 0); ++j) {
            }
        }
    } else {
        // ------------------------------------------------------------------ epilogue: two teams of four warps, each half of a tile's columns
        // Every warp goes its own way through its 32 rows.  25600 x 384 -> 1536 with GELU and z takes 53 us (the same buffers again and
        // again) on the tiles chosen now; the forms were compared on pairs of CTAs with a shorter GELU: this one 56, lanes that store
        // themselves (64-byte pieces of eight rows an instruction) 71, sixteen warps in teams with a buffer and barriers for each four 63
        // to 78, and their polling costs the long products 5 %.
        const int ew = warp - 2, team = ew >> 2, lane_group = warp & 3;  // TMEM lanes [32*lane_group, +32)
        const int ncol = p.BN / 2, c_lo = team * ncol;
        uint8_t* const my_stg = stg + (size_t)ew * 2 * TL_STG;
        uint64_t* const my_in = infull + 2 * ew;
        float* const my_bias = sbias + ew * 128;
        const uint32_t tempty_u32 = CG2 ? ptx::mapa_u32(ptx::smem_u32(tempty), 0u) : ptx::smem_u32(tempty);
        int acc = 0, buf = 0;
        uint32_t acc_ph = 0, in_ph = 0;  // in_ph: a bit for each buffer
        auto wait_acc = [&]() {
            bool ok = true;
            if (lane == 0) ok = wait_bar(tfull + acc, acc_ph, abort_flag, p.status, 24);  // one poller a warp
            ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
            if (ok) ptx::tc_fence_after();
            return ok;
        };
        auto release_acc = [&]() {  // this warp is done reading the accumulator set
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (CG2) ptx::mbar_arrive_cluster(tempty_u32 + 8u * (uint32_t)acc); else ptx::mbar_arrive(tempty + acc);
            }
        };
        auto next_acc = [&]() {
            acc ^= 1;
            if (acc == 0) acc_ph ^= 1u;
        };
        pdl_wait();
        for (int i = worker; i < tiles; i += nworkers) {
            int mt, nt, split, kb0, kb1;
            item(i, mt, nt, split, kb0, kb1);
            const int row0 = mt * TM + (int)rank * 128 + lane_group * 32;
            const uint32_t lanes = tmem_base + ((uint32_t)(lane_group * 32) << 16);
            if constexpr (KIND == LIN_WEIGHT) {
                float2 sum[4][16];  // 32 columns each
                float dbs = 0.f;
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[q][j] = make_float2(0.f, 0.f);
                bool ok = true;
                for (int c0 = kb0; c0 < kb1; c0 += chunk) {
                    ok = wait_acc();
                    if (!ok) break;
                    const uint32_t taddr = lanes + (uint32_t)(acc * p.acc_stride);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        if (32 * q >= ncol) break;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {  // (16 columns at a time: registers)
                            uint32_t r[16];
                            ptx::tmem_ld_32x32b_x16(taddr + (uint32_t)(c_lo + 32 * q + 16 * h), r);
                            ptx::tmem_ld_wait();
#pragma unroll
                            for (int j = 0; j < 8; ++j) sum[q][8 * h + j] = add2(sum[q][8 * h + j], make_float2(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1])));
                        }
                    }
                    if (p.db && team == 1) {
                        uint32_t r[16];
                        ptx::tmem_ld_32x32b_x16(taddr + (uint32_t)p.BN, r);
                        ptx::tmem_ld_wait();
                        // (a chunk without a k-block of this column tile's share has left nothing in these columns)
                        const int first = c0 + (nt - c0 % p.n_tiles + p.n_tiles) % p.n_tiles;
                        if (first < min(kb1, c0 + chunk)) dbs += __uint_as_float(r[0]);
                        __syncwarp();
                    }
                    release_acc();
                    next_acc();
                }
                if (!ok) break;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int col = nt * p.BN + c_lo + 32 * q;
                    if (32 * q >= ncol || col >= p.N) break;
                    uint8_t* b = my_stg + (q & 1) * TL_STG;
                    if (lane == 0) ptx::tma_store_wait_read<1>();  // (what went out of it before has been read)
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        *reinterpret_cast<float4*>(b + lane * 128 + ((j ^ (lane & 7)) * 16)) = make_float4(sum[q][2 * j].x, sum[q][2 * j].y, sum[q][2 * j + 1].x, sum[q][2 * j + 1].y);
                    ptx::fence_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        ptx::tma_store_3d(&p.tmOut, b, col, row0, split);
                        ptx::tma_store_commit();
                    }
                }
                if (p.db && team == 1 && row0 + lane < p.M) p.db[((size_t)split * p.n_tiles + nt) * p.M + row0 + lane] = dbs;
                __syncwarp();
            } else {
                // the passes of this warp that have columns; pass k uses buffer (buf + k) & 1
                const int col0 = nt * p.BN + c_lo, passes = max(0, (min(ncol, p.N - col0) + NP - 1) / NP);
                const bool in_tma = p.has_in && !p.want_z;  // (with z both buffers are at work when the residual would have to come)
                auto request = [&](int b, int k) {  // pass k's input into buffer b, by lane 0, with the buffer free
                    ptx::mbar_expect_tx(my_in + b, 32 * NP * 2);
                    ptx::tma_load_2d(my_stg + b * TL_STG, &p.tmIn, my_in + b, col0 + k * NP, row0);
                };
                if (KIND == LIN_FWD && p.bias) {
                    __syncwarp();
                    for (int e = lane; e < ncol; e += 32) my_bias[e] = col0 + e < p.n_bias ? p.bias[col0 + e] : 0.f;
                    __syncwarp();
                }
                if (in_tma && lane == 0) {
                    if (passes > 0) {
                        ptx::tma_store_wait_read<1>();
                        request(buf, 0);
                    }
                    if (passes > 1) {
                        ptx::tma_store_wait_read<0>();
                        request(buf ^ 1, 1);
                    }
                }
                bool ok = true;
                float2 sum[LONG ? NP / 2 : 1];
                if constexpr (LONG) {  // (tiles of 2 * NP columns: a warp has one pass)
#pragma unroll
                    for (int j = 0; j < NP / 2; ++j) sum[j] = make_float2(0.f, 0.f);
                    for (int c0 = kb0; c0 + chunk < kb1; c0 += chunk) {
                        ok = wait_acc();
                        if (!ok) break;
#pragma unroll
                        for (int h = 0; h < NP / 32; ++h) {
                            uint32_t r[32];
                            ptx::tmem_ld_32x32b_x32(lanes + (uint32_t)(acc * p.acc_stride + c_lo + 32 * h), r);
                            ptx::tmem_ld_wait();
#pragma unroll
                            for (int j = 0; j < 16; ++j) sum[16 * h + j] = add2(sum[16 * h + j], make_float2(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1])));
                        }
                        release_acc();
                        next_acc();
                    }
                }
                if (ok) ok = wait_acc();
                const uint32_t taddr = lanes + (uint32_t)(acc * p.acc_stride + c_lo);
                if (ok && passes == 0) release_acc();
                for (int k = 0; k < passes; ++k) {
                    uint8_t* b = my_stg + buf * TL_STG;
                    if (in_tma) {  // (waited for whatever has failed: nothing may land after the CTA has exited)
                        __syncwarp();
                        bool there = false;
                        for (int j = 0; j < 400000 && !(there = ptx::mbar_try_wait(my_in + buf, (in_ph >> buf) & 1u)); ++j) {
                        }
                        if (!there) give_up(abort_flag, p.status, 25);
                        ok = __all_sync(0xffffffffu, ok && there) != 0;
                        in_ph ^= 1u << buf;
                        if (!ok && k < 2) {  // (those requested so far)
                            buf ^= 1;
                            continue;
                        }
                    }
                    if (!ok) break;
                    auto release = [&]() {
                        if (k == passes - 1) release_acc();
                    };
                    auto other = [&]() {  // z goes first and takes this pass's buffer, the result the next one
                        if (lane == 0) ptx::tma_store_wait_read<1>();
                        __syncwarp();
                        uint8_t* zs = my_stg + buf * TL_STG;
                        buf ^= 1;
                        return zs;
                    };
                    if (!in_tma && !p.want_z) {
                        if (lane == 0) ptx::tma_store_wait_read<1>();
                        __syncwarp();
                    }
                    TlPass<T, KIND, NP, LONG>::run(p, taddr + (uint32_t)(k * NP), lane, row0, col0 + k * NP, my_bias + k * NP, p.want_z ? my_stg + (buf ^ 1) * TL_STG : b, in_tma, sum, release, other);
                    buf ^= 1;
                    if (in_tma && k + 2 < passes && lane == 0) {
                        ptx::tma_store_wait_read<0>();
                        request(buf ^ 1, k + 2);  // (the buffer of pass k)
                    }
                }
                if (!ok) break;
                next_acc();
            }
        }
        // the staging rows must have been read before this CTA's shared memory is released
        if (lane == 0) ptx::tma_store_wait_read<0>();
        __syncwarp();
    }
    __syncwarp();  // (the cluster barrier and the release of TMEM want whole warps)
    ptx::tc_fence_before();
    if (CG2) ptx::cluster_sync_all(); else __syncthreads();  // pairs: neither CTA may leave while the other still uses its memory
    if (warp == 1) {
        ptx::tc_fence_after();
        if (CG2) ptx::tmem_dealloc_cg2(tmem_base, 512); else ptx::tmem_dealloc(tmem_base, 512);
    }
}

}  // namespace nbcbs
