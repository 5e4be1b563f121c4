// Backward of a token loss with at most 128 rows: dHidden's parts and dW in one sweep over W.
//
//   dHidden[r, h] = sum_v G[r, v] W[v, h]          dW[v, h] = sum_r G[r, v] hidden[r, h]
//
// With so few rows both products take less time than their bytes: W is read and dW written, each V x H values.  As two launches
// they read at 5.9 and write at 4.1 TB/s, the most that either direction gives alone; reads and writes at the same time share
// more (a copy: 6.5 TB/s).  So a CTA walks a range of the vocabulary in chunks of 128 entries for 128 columns of H: a chunk's
// tile of W and its 128 x 128 block of G (32 KiB each) land by TMA, and one thread issues
//   dHidden (128 rows x 128 columns, tensor-memory columns 0..127)  +=  G     W        G K-major, W MN-major
//   dW      (128 entries x 128 columns, one of two stages behind)    =  G^T   hidden   both MN-major, G being the same bytes
// as 16 MMAs.  The columns' hidden rows (32 KiB) stay in shared memory throughout.  Four epilogue warps round a dW tile to bf16
// into the place of the chunk's W, whose MMAs have completed, and a warp of its own sends it off as bulk stores (a thread per
// entry storing its own 256 bytes touches 32 lines at a time and took 10 % longer); fp32 tiles go out by plain stores.  W comes
// from HBM and its place is taken until the tile has left: a ring of four stages and a producer of its own.  G comes from L2 and
// is done with after the MMAs: two stages.  (Three stages of both: 652 us for the step of 96 rows x 3584 x 152064, now 605.)
// At the end the epilogue writes the CTA's part of dHidden.  The vocabulary is cut into as many ranges as fill the SMs once.
// Measured (training step, this kernel against two GEMMs): 40 rows x 896 x 151936 204 / 248 us, x 1536 304 / 339, 60 rows x
// 2560 x 100000 318 / 363, 96 rows x 3584 x 152064 610 / 659, 40 rows x 256 x 4096 44 / 53; the kernel alone moves W and dW
// at 5.1 to 5.4 TB/s.  Bound: HBM, beside shared memory, which the MMAs' operands, the loads and the stores pass through
// (256 KiB and 2.0 k clocks per chunk, of 3.2 k).
// Every mbarrier wait is bounded as in gemm_tcgen05.cu.
#include <cstring>

#include "internal.h"
#include "ptx.cuh"

namespace unity {

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 128;                              // vocabulary entries per stage
constexpr int kCols = 128;                               // columns of H per CTA
constexpr int kRows = 128;
constexpr int kBox = kRows * 128;                        // 64 bf16 columns x 128 rows
constexpr int kHiddenBytes = 2 * kBox;
constexpr int kGBytes = 2 * kBox, kWBytes = 2 * kBox;
constexpr int kGStages = 2, kWStages = 4;
constexpr int kSmemBytes = 1024 + kHiddenBytes + kGStages * kGBytes + kWStages * kWBytes + 256;
constexpr int kTmemCols = 512;                           // 128 + 2 x 128, rounded up to a power of two

__device__ __forceinline__ void store_row(float* dst, const uint32_t (&r)[32], bool wide) {
    if (wide) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            ptx::st_global_v8(dst + 8 * q, r[8 * q], r[8 * q + 1], r[8 * q + 2], r[8 * q + 3], r[8 * q + 4], r[8 * q + 5], r[8 * q + 6], r[8 * q + 7]);
    } else {
#pragma unroll
        for (int q = 0; q < 8; ++q)
            *reinterpret_cast<uint4*>(dst + 4 * q) = make_uint4(r[4 * q], r[4 * q + 1], r[4 * q + 2], r[4 * q + 3]);
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 1)
k_few_rows_bwd(const __grid_constant__ CUtensorMap tmG, const __grid_constant__ CUtensorMap tmH,
               const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmO, const FewRowsArgs a) {
    constexpr bool kStaged = sizeof(T) == 2;     // bf16 dW leaves through shared memory
    extern __shared__ uint8_t smem_raw[];
    uint8_t* hidden = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* ring_g = hidden + kHiddenBytes;
    uint8_t* ring_w = ring_g + kGStages * kGBytes;
    uint64_t* g_full = reinterpret_cast<uint64_t*>(ring_w + kWStages * kWBytes);   // [kGStages] a stage's bytes have landed
    uint64_t* g_empty = g_full + kGStages;       // [kGStages] the MMAs that read it have completed
    uint64_t* w_full = g_empty + kGStages;       // [kWStages]
    uint64_t* w_empty = w_full + kWStages;       // [kWStages] the MMAs that read it have completed; bf16 dW: its tile has left
    uint64_t* staged = w_empty + kWStages;       // [kWStages] a bf16 dW tile lies where the stage's W was
    uint64_t* acc_full = staged + kWStages;      // [2] a dW tile is complete
    uint64_t* acc_empty = acc_full + 2;          // [2] ... and drained
    uint64_t* hid_full = acc_empty + 2;
    uint64_t* dh_full = hid_full + 1;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(dh_full + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kGStages; ++s) { ptx::mbar_init(&g_full[s], 1); ptx::mbar_init(&g_empty[s], 1); }
        for (int s = 0; s < kWStages; ++s) { ptx::mbar_init(&w_full[s], 1); ptx::mbar_init(&w_empty[s], 1); ptx::mbar_init(&staged[s], 4); }
        for (int b = 0; b < 2; ++b) { ptx::mbar_init(&acc_full[b], 1); ptx::mbar_init(&acc_empty[b], 4); }
        ptx::mbar_init(hid_full, 1);
        ptx::mbar_init(dh_full, 1);
        *abort_flag = 0;
        ptx::fence_barrier_init();
        ptx::prefetch_tensormap(&tmG);
        ptx::prefetch_tensormap(&tmH);
        ptx::prefetch_tensormap(&tmW);
    }
    if (warp == 1) { ptx::tmem_alloc(tmem_slot, kTmemCols); ptx::tmem_relinquish(); }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    // (the set-up overlaps the launch before this one: nothing in global memory is touched until that is complete)
    ptx::grid_launch_dependents();
    ptx::grid_wait();

    const int first = a.plan->off[a.model], valid = a.plan->counts[a.model];
    const int h0 = blockIdx.x % a.n_col_blocks * kCols, part = blockIdx.x / a.n_col_blocks;
    const int n_cols = min(kCols, a.H - h0);                          // 64 or 128
    const int c0 = part * a.per_part, c1 = min(c0 + a.per_part, (a.V + kChunk - 1) / kChunk);
    T* dW = static_cast<T*>(a.dW);

    if (valid == 0) {
        // a model without rows: its dW reads zero
        constexpr int kUnit = 16 / sizeof(T);
        const int per_row = n_cols / kUnit, rows = min(c1 * kChunk, a.V) - c0 * kChunk;
        for (int i = threadIdx.x; i < rows * per_row; i += kThreads) {
            const int v = c0 * kChunk + i / per_row, h = h0 + i % per_row * kUnit;
            *reinterpret_cast<uint4*>(dW + static_cast<long long>(v) * a.H + h) = make_uint4(0, 0, 0, 0);
        }
    } else if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer of W, as far ahead as its ring allows
        if (lane == 0) {
            const uint64_t once = ptx::l2_policy(1);
            int s = 0;
            uint32_t phase = 0;
            for (int c = c0; c < c1; ++c) {
                if (!ptx::mbar_wait(&w_empty[s], phase ^ 1, a.wait_budget) || *abort_flag) {
                    *abort_flag = 1;
                    atomicOr(a.status, kStatusTimeout);
                    break;
                }
                const uint32_t bar = ptx::smem_u32(&w_full[s]);
                ptx::mbar_arrive_expect_tx(&w_full[s], kWBytes);
                for (int k = 0; k < 2; ++k)                          // 64 entries each: a box of 64 columns, then the next
                    for (int j = 0; j < 2; ++j)
                        ptx::tma_load_2d_hint_on<1>(ring_w + s * kWBytes + (2 * k + j) * (kBox / 2), &tmW, bar, h0 + 64 * j, c * kChunk + 64 * k, once);
                if (++s == kWStages) { s = 0; phase ^= 1; }
            }
        }
    } else if (warp == 7) {
        // ------------------------------------------------------------------ ... of the hidden rows and G
        if (lane == 0) {
            const uint64_t keep = ptx::l2_policy(0);
            ptx::mbar_arrive_expect_tx(hid_full, kHiddenBytes);
            for (int j = 0; j < 2; ++j)
                ptx::tma_load_2d_hint_on<1>(hidden + j * kBox, &tmH, ptx::smem_u32(hid_full), h0 + 64 * j, first, keep);
            int s = 0;
            uint32_t phase = 0;
            for (int c = c0; c < c1; ++c) {
                if (!ptx::mbar_wait(&g_empty[s], phase ^ 1, a.wait_budget) || *abort_flag) {
                    *abort_flag = 1;
                    atomicOr(a.status, kStatusTimeout);
                    break;
                }
                const uint32_t bar = ptx::smem_u32(&g_full[s]);
                ptx::mbar_arrive_expect_tx(&g_full[s], kGBytes);
                for (int j = 0; j < 2; ++j) ptx::tma_load_2d_hint_on<1>(ring_g + s * kGBytes + j * kBox, &tmG, bar, c * kChunk + 64 * j, first, keep);
                if (++s == kGStages) { s = 0; phase ^= 1; }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        if (lane == 0) {
            const uint32_t id_dh = ptx::idesc_bf16_f32(kRows, kCols) | (1u << 16);
            const uint32_t id_dw = ptx::idesc_bf16_f32(kChunk, kCols) | (1u << 15) | (1u << 16);
            // rows that hold tokens, or (low halves) all 128, in steps of 16; the rows behind them are not gradients
            const int k_rows = valid <= a.low_rows ? kRows / 16 : (valid + kTileK - 1) / kTileK * (kTileK / 16);
            bool ok = ptx::mbar_wait(hid_full, 0, a.wait_budget);
            int s = 0, t = 0;
            uint32_t phase = 0, phase_w = 0;
            for (int c = c0; ok && c < c1; ++c) {
                const int b = (c - c0) & 1;
                const uint32_t acc_phase = ((c - c0) >> 1) & 1;
                ok = ptx::mbar_wait(&acc_empty[b], acc_phase ^ 1, a.wait_budget) && ptx::mbar_wait(&w_full[t], phase_w, a.wait_budget) &&
                     ptx::mbar_wait(&g_full[s], phase, a.wait_budget) && !*abort_flag;
                if (!ok) break;
                ptx::tc_fence_after();
                const uint32_t g = ptx::smem_u32(ring_g + s * kGBytes), w = ptx::smem_u32(ring_w + t * kWBytes);
                for (int k = 0; k < kChunk / 16; ++k) {              // 16 entries each: inside a swizzle row of G, 16 rows of W
                    const uint64_t da = ptx::smem_desc_k_sw128(g + (k >> 2) * kBox) + 2 * (k & 3);
                    const uint64_t db = ptx::smem_desc_mn_sw128(w + (k >> 2) * kBox, kBox / 2) + 128 * (k & 3);
                    ptx::mma_bf16_ss(tmem, da, db, id_dh, c > c0 || k > 0 ? 1u : 0u);
                }
                const uint64_t da = ptx::smem_desc_mn_sw128(g, kBox), db = ptx::smem_desc_mn_sw128(ptx::smem_u32(hidden), kBox);
                for (int k = 0; k < k_rows; ++k) ptx::mma_bf16_ss(tmem + kCols * (1 + b), da + 128 * k, db + 128 * k, id_dw, k > 0 ? 1u : 0u);
                ptx::tc_commit(&g_empty[s]);
                if (!kStaged) ptx::tc_commit(&w_empty[t]);
                ptx::tc_commit(&acc_full[b]);
                if (++s == kGStages) { s = 0; phase ^= 1; }
                if (++t == kWStages) { t = 0; phase_w ^= 1; }
            }
            if (ok) ptx::tc_commit(dh_full);
            else { *abort_flag = 1; atomicOr(a.status, kStatusTimeout); }
        }
    } else if (warp == 6) {
        // ------------------------------------------------------------------ dW writer: a tile leaves as one or two bulk stores
        if (kStaged && lane == 0) {
            int s = 0;
            uint32_t phase = 0;
            for (int c = c0; c < c1; ++c) {
                if (!ptx::mbar_wait(&staged[s], phase, a.wait_budget) || *abort_flag) {
                    *abort_flag = 1;
                    atomicOr(a.status, kStatusTimeout);
                    break;
                }
                for (int j = 0; 64 * j < n_cols; ++j)                // (rows behind the vocabulary are left out by the map)
                    ptx::tma_store_2d(&tmO, ring_w + s * kWBytes + j * kBox, h0 + 64 * j, c * kChunk);
                ptx::tma_store_commit();
                ptx::tma_store_wait_read();
                ptx::mbar_arrive(&w_empty[s]);
                if (++s == kWStages) { s = 0; phase ^= 1; }
            }
            ptx::tma_store_wait();
        }
    } else {
        // ------------------------------------------------------------------ epilogue: thread = one vocabulary entry, then one row
        const int quarter = warp & 3, at = quarter * 32 + lane;
        const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
        const float alpha = a.alpha[a.model];
        bool ok = true;
        uint32_t r[32], next[32];
        int s = 0;
        for (int c = c0; c < c1; ++c) {
            const int b = (c - c0) & 1;
            // (all lanes go on or none: the loads from tensor memory are the whole warp's)
            ok = __all_sync(0xffffffffu, ptx::mbar_wait(&acc_full[b], ((c - c0) >> 1) & 1, a.wait_budget) && !*abort_flag);
            if (!ok) break;
            ptx::tc_fence_after();
            const int v = c * kChunk + at;
            const uint32_t acc = tmem + lanes + kCols * (1 + b);
            // the stage's MMAs have completed: its W gives way to the dW tile, in the layout of a store's boxes (rows of 128
            // bytes whose 16-byte units are exchanged by row, which also keeps these writes free of bank conflicts)
            uint8_t* out = ring_w + s * kWBytes + at * 128;
            ptx::tmem_ld_32x32(acc, r);
            ptx::tmem_ld_wait_for(r);
#pragma unroll 1
            for (int q = 0; q * 32 < n_cols; ++q) {
                const bool more = (q + 1) * 32 < n_cols;
                if (more) ptx::tmem_ld_32x32(acc + 32 * (q + 1), next);
#pragma unroll
                for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(alpha * __uint_as_float(r[j]));
                if (kStaged) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        unsigned o[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(r[8 * i + 2 * j]), __uint_as_float(r[8 * i + 2 * j + 1]));
                            o[j] = *reinterpret_cast<const unsigned*>(&h);
                        }
                        *reinterpret_cast<uint4*>(out + (q >> 1) * kBox + ((((q & 1) * 4 + i) ^ (at & 7)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
                    }
                } else if (v < a.V) {
                    store_row(reinterpret_cast<float*>(a.dW) + static_cast<long long>(v) * a.H + h0 + 32 * q, r, a.wide != 0);
                }
                __syncwarp();
                if (!more) break;
                ptx::tmem_ld_wait_for(next);
#pragma unroll
                for (int j = 0; j < 32; ++j) r[j] = next[j];
            }
            if (kStaged) ptx::fence_proxy_async();
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (kStaged) ptx::mbar_arrive(&staged[s]);
                ptx::mbar_arrive(&acc_empty[b]);
            }
            if (++s == kWStages) s = 0;
        }
        if (ok) ok = __all_sync(0xffffffffu, ptx::mbar_wait(dh_full, 0, a.wait_budget) && !*abort_flag);
        if (ok) {
            ptx::tc_fence_after();
            float* dst = a.parts + (static_cast<long long>(part) * kRows + at) * a.H + h0;
#pragma unroll 1
            for (int q = 0; q * 32 < n_cols; ++q) {
                ptx::tmem_ld_32x32(tmem + lanes + 32 * q, r);
                ptx::tmem_ld_wait_for(r);
                store_row(dst + 32 * q, r, true);
                __syncwarp();
            }
        } else {
            *abort_flag = 1;
            atomicOr(a.status, kStatusTimeout);
        }
    }

    // ---------------------------------------------------------------------- teardown
    __syncwarp();
    if (*abort_flag) {
        // copies issued before the abort may still be landing in shared memory: give them time
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000) { }
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, kTmemCols);
    }
}

template <typename T>
cudaError_t launch(const CUtensorMap& tmG, const CUtensorMap& tmH, const CUtensorMap& tmW, const CUtensorMap& tmO, const FewRowsArgs& a,
                   cudaStream_t stream) {
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3(a.n_col_blocks * a.parts_n);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmemBytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_few_rows_bwd<T>, tmG, tmH, tmW, tmO, a);
}

}  // namespace

cudaError_t few_rows_set_attributes() {
    const cudaError_t e = cudaFuncSetAttribute(k_few_rows_bwd<float>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(k_few_rows_bwd<__nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
}

// Where the ranges of all column blocks fill three quarters of the SMs, or the vocabulary has no more chunks than SMs to go
// round.  A training step of 120 rows against two GEMMs: 4608 columns (97 % of the SMs) x 60000 330 / 385 us, 4096 (86 %)
// 308 / 332, 5120 (81 %) x 152064 882 / 941, 7168 (76 %) x 60000 548 / 565; below that (9600: 51 %) the rest idles.
bool few_rows_pays(int H, int V, int sm_count) {
    const int blocks = (H + kCols - 1) / kCols, parts = sm_count / blocks;
    return parts >= (V + kChunk - 1) / kChunk || 4 * blocks * parts >= 3 * sm_count;
}

void few_rows_plan(int H, int V, int sm_count, long long part_capacity, FewRowsArgs* a) {
    const int chunks = (V + kChunk - 1) / kChunk;
    a->n_col_blocks = (H + kCols - 1) / kCols;
    long long parts = sm_count / a->n_col_blocks;
    if (parts > part_capacity / (static_cast<long long>(kRows) * H)) parts = part_capacity / (static_cast<long long>(kRows) * H);
    if (parts > chunks) parts = chunks;
    if (parts < 1) parts = 1;
    a->per_part = static_cast<int>((chunks + parts - 1) / parts);
    a->parts_n = (chunks + a->per_part - 1) / a->per_part;
}

cudaError_t launch_few_rows_bwd(const CUtensorMap& tmG, const CUtensorMap& tmH, const CUtensorMap& tmW, const CUtensorMap* tmO,
                                const FewRowsArgs& a, cudaStream_t stream) {
    return tmO ? launch<__nv_bfloat16>(tmG, tmH, tmW, *tmO, a, stream) : launch<float>(tmG, tmH, tmW, tmW, a, stream);
}

}  // namespace unity
