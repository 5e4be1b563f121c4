// RMS norm of token rows with one weight vector per model, and its backward (unity_rms_norm_fwd, unity_rms_norm_bwd).
// A row is held in the registers of the warps that share it: one read of its inputs, one write of its outputs, the sums over
// the columns in fp32.  dgamma is summed per block in registers over the block's rows, then over the blocks, both in a fixed
// order: no atomics.
#include "internal.h"
#include "ptx.cuh"

namespace unity {

namespace {

constexpr unsigned kFull = 0xffffffffu;

// Every kernel here calls this before its first access to global memory: it may be in place when the kernel before it ends, and waits
// for that one to complete.
__device__ __forceinline__ void begin() {
    ptx::grid_launch_dependents();
    ptx::grid_wait();
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}

// Invocation of token `tok` by the whole warp: 32 places of the offsets are looked at per step (one of 8192 invocations takes three
// dependent loads instead of thirteen).
__device__ __forceinline__ int token_invocation(const NormArgs& a, long long tok, int lane) {
    int lo = 0, hi = a.n_inv;                                   // the number of ends cu[1..n_inv] that are <= tok lies in [lo, hi]
    while (lo < hi) {
        const int step = (hi - lo + 31) / 32;
        const int at = lo + (lane + 1) * step - 1;
        const unsigned below = __ballot_sync(kFull, at < hi && a.cu_seqlens[at + 1] <= tok);
        const int n = __popc(below);
        const int next = lo + (n + 1) * step - 1;
        lo += n * step;
        hi = n == 32 ? hi : min(hi, next);
        lo = min(lo, hi);
    }
    return min(lo, a.n_inv - 1);
}
// Its model, -1 for a role out of range.
__device__ __forceinline__ int invocation_model(const NormArgs& a, int s) {
    const int role = a.inv_role[s];
    return role >= 0 && role < a.n_roles ? a.role_model[role] : -1;
}

// Eight consecutive elements.  Plain loads, not the read-only path: an output may be the input's own memory.
struct Raw16 { uint4 v; };
struct Raw32 { float4 a, b; };
__device__ __forceinline__ void load8(const __nv_bfloat16* p, Raw16& r) { r.v = *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void load8(const float* p, Raw32& r) {
    r.a = *reinterpret_cast<const float4*>(p);
    r.b = *reinterpret_cast<const float4*>(p + 4);
}
__device__ __forceinline__ void widen(const Raw16& r, float (&f)[8]) {
    const unsigned w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void widen(const Raw32& r, float (&f)[8]) {
    f[0] = r.a.x; f[1] = r.a.y; f[2] = r.a.z; f[3] = r.a.w; f[4] = r.b.x; f[5] = r.b.y; f[6] = r.b.z; f[7] = r.b.w;
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&f)[8]) {
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const unsigned*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float* p, const float (&f)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void load_gamma(const NormArgs& a, int model, int col, float (&g)[8]) {
    if (a.gamma_bf16) {
        Raw16 r;
        load8(static_cast<const __nv_bfloat16*>(a.gamma[model]) + col, r);
        widen(r, g);
    } else {
        Raw32 r;
        load8(static_cast<const float*>(a.gamma[model]) + col, r);
        widen(r, g);
    }
}

// The same as four packed pairs, for arithmetic on two lanes at once.
typedef uint64_t Pairs[4];
__device__ __forceinline__ void pairs_of(const float (&f)[8], Pairs& p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = ptx::pack2(f[2 * i], f[2 * i + 1]);
}
__device__ __forceinline__ void floats_of(const Pairs& p, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) ptx::unpack2(p[i], f[2 * i], f[2 * i + 1]);
}

template <typename T> struct RawOf;
template <> struct RawOf<__nv_bfloat16> { typedef Raw16 type; };
template <> struct RawOf<float> { typedef Raw32 type; };

// Copies to shared memory; both sides and the size in multiples of 16 bytes.
__device__ __forceinline__ void bulk_load(void* to, const void* from, unsigned bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(ptx::smem_u32(to)), "l"(from),
                 "r"(bytes), "r"(ptx::smem_u32(bar)) : "memory");
}

// Sum of a pair over the WPR warps of a row; `slots` holds two of them in turn, so that one barrier per call is enough.  What the row's
// threads read of shared memory before it has been read behind it, for one warp too: shuffles alone do not order memory.
template <int WPR>
__device__ __forceinline__ float2 row_sum(float2 v, float2 (&slots)[2][WPR], int turn) {
    v.x = warp_sum(v.x);
    v.y = warp_sum(v.y);
    if (WPR == 1) {
        __syncwarp();
        return v;
    }
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) slots[turn][warp] = v;
    __syncthreads();
    float2 s = slots[turn][0];
#pragma unroll
    for (int w = 1; w < WPR; ++w) { s.x += slots[turn][w].x; s.y += slots[turn][w].y; }
    return s;
}

// ------------------------------------------------------------------------------------------------
// y = gamma r s, r = x + residual, s = 1 / sqrt(mean r^2 + eps).  A row belongs to WPR warps, each lane holding NV vectors of
// eight columns, 256 WPR columns apart: at most eight, so that all of a row's loads are in flight at once and a dozen rows fit an SM.
// The norm is taken of the fp32 sum; r is rounded only where it is written.  HBM bounds it (20001 x 3584 bf16 82 us, 98 % of the copy
// rate; 32768 x 5120 with fp32 residual 291 us), one row takes 4.4 us from launch to launch.
// ------------------------------------------------------------------------------------------------
constexpr int kFwdRowsOfWarps = 4;          // rows of a block whose rows belong to one warp each
template <int WPR, int NV, typename R, bool HAS_R>
__global__ void __launch_bounds__(WPR == 1 ? 32 * kFwdRowsOfWarps : 32 * WPR) k_norm_fwd(const __grid_constant__ NormArgs a) {
    begin();
    __shared__ float2 slots[2][WPR];
    const int lane = threadIdx.x & 31;
    const int t = WPR == 1 ? lane : threadIdx.x;
    const long long row = WPR == 1 ? static_cast<long long>(blockIdx.x) * kFwdRowsOfWarps + (threadIdx.x >> 5) : blockIdx.x;
    if (row >= a.n_tok) return;                                  // (a whole warp, or a whole block)
    const int H = a.H;
    const long long base = row * H;
    // (the search for the model needs nothing of the mask: the loads of both are on their way together)
    const uint8_t mask = a.tok_mask == nullptr ? 1 : a.tok_mask[row];
    const int inv = token_invocation(a, row, lane);
    bool on = mask != 0;
    int model = -1;
    Raw16 x[NV];
    typename RawOf<R>::type res[NV];
    if (on) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = (j * WPR * 32 + t) * 8;
            if (col < H) {
                load8(a.x + base + col, x[j]);
                if (HAS_R) load8(static_cast<const R*>(a.residual) + base + col, res[j]);
            }
        }
        model = invocation_model(a, inv);
        on = model >= 0;
        if (!on && lane == 0) atomicOr(a.status, kStatusBadIndex);
    }
    if (!on) {                                                   // (the same for every warp of the row)
        const float zero[8] = {};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = (j * WPR * 32 + t) * 8;
            if (col < H) {
                store8(a.y + base + col, zero);
                if (HAS_R && a.res_out) store8(static_cast<R*>(a.res_out) + base + col, zero);
            }
        }
        return;
    }
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int col = (j * WPR * 32 + t) * 8;
        if (col < H) {
            float f[8], g[8];
            widen(x[j], f);
            if (HAS_R) {
                widen(res[j], g);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] += g[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(f[i], f[i], sum);
        }
    }
    const float2 total = row_sum<WPR>(make_float2(sum, 0.f), slots, 0);
    const float s = 1.f / sqrtf(total.x / static_cast<float>(H) + a.eps);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int col = (j * WPR * 32 + t) * 8;
        if (col < H) {
            float f[8], g[8];
            widen(x[j], f);
            if (HAS_R) {
                widen(res[j], g);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] += g[i];
                if (a.res_out) store8(static_cast<R*>(a.res_out) + base + col, f);
            }
            load_gamma(a, model, col, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = g[i] * (f[i] * s);
            store8(a.y + base + col, f);
        }
    }
}

// ------------------------------------------------------------------------------------------------
// dr = s (g - r s mean(g r s)) + dres with g = dy gamma; dgamma += dy r s.  A block takes a run of consecutive rows, so that its
// dgamma stays in registers; where the model changes it goes to the block's slice of that model and the next one begins.  The rows
// come through a ring in shared memory, by asynchronous copies that run ahead of the row that is worked on: registers hold the
// columns' sums and weights only, and HBM is asked for rows without a pause (40001 x 3584 fp32 with dres: 285 to 300 us, 0.9 of the
// copy rate; rows in registers, without the ring, 378).  5000 x 1536 bf16: 22 us with the sums of the slices, most of it latency.  A block of
// 32 warps (H above 8192) has no registers for its row and its dgamma: they go to local memory (8000 x 16384 bf16 610 us with dgamma and
// 231 without, where 8192 columns take 100 and 96).
// ------------------------------------------------------------------------------------------------
constexpr int kMaxStages = 4;
template <int WPR, int NV, typename R, bool DG>
__global__ void __launch_bounds__(32 * WPR) k_norm_bwd(const __grid_constant__ NormArgs a, int stages, int ring_dres) {
    __shared__ float2 slots[2][WPR];
    __shared__ uint64_t full[kMaxStages];
    extern __shared__ __align__(16) unsigned char ring[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = threadIdx.x, H = a.H;
    const long long first = a.n_tok * blockIdx.x / gridDim.x, last = a.n_tok * (blockIdx.x + 1) / gridDim.x;
    const unsigned res_bytes = H * sizeof(R), dy_bytes = H * 2, stage_bytes = res_bytes + dy_bytes + (ring_dres ? res_bytes : 0);
    if (t == 0) {
        for (int i = 0; i < stages; ++i) ptx::mbar_init(&full[i], 1);
        ptx::fence_barrier_init();
    }
    __syncthreads();
    begin();
    // mask bits of the 32 rows from `base`
    auto bits_of = [&](long long base) {
        return __ballot_sync(kFull, base + lane < last && (a.tok_mask == nullptr || a.tok_mask[base + lane] != 0));
    };
    // The first warp asks for the unmasked rows in order, `stages` of them ahead.
    long long ask_base = first;
    unsigned ask_bits = warp == 0 && first < last ? bits_of(first) : 0;
    int asked = 0;
    auto ask = [&]() {
        while (ask_bits == 0) {
            if (ask_base + 32 >= last) return;
            ask_base += 32;
            ask_bits = bits_of(ask_base);
        }
        const long long at = (ask_base + __ffs(ask_bits) - 1) * H;
        ask_bits &= ask_bits - 1;
        if (lane == 0) {
            const int stage = asked % stages;
            unsigned char* to = ring + static_cast<size_t>(stage) * stage_bytes;
            ptx::mbar_arrive_expect_tx(&full[stage], stage_bytes);
            bulk_load(to, static_cast<const R*>(a.res) + at, res_bytes, &full[stage]);
            bulk_load(to + res_bytes, a.dy + at, dy_bytes, &full[stage]);
            if (ring_dres) bulk_load(to + res_bytes + dy_bytes, static_cast<const R*>(a.dres) + at, res_bytes, &full[stage]);
        }
        ++asked;
    };
    if (warp == 0)
        for (int i = 0; i < stages; ++i) ask();

    Pairs acc[NV], gamma[NV];
    int model = -1, found = -1, done = 0;
    long long found_end = first;
    unsigned touched = 0;
    auto flush = [&]() {
        if (!DG || model < 0) return;
        float* slice = a.parts + (static_cast<long long>(blockIdx.x) * a.K + model) * H;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = (j * WPR * 32 + t) * 8;
            if (col < H) {
                float f[8];
                floats_of(acc[j], f);
                if (touched >> model & 1) {
                    Raw32 r;
                    float old[8];
                    load8(slice + col, r);
                    widen(r, old);
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] += old[i];
                }
                store8(slice + col, f);
            }
        }
        touched |= 1u << model;
    };
    unsigned bits = 0;
    for (long long row = first; row < last; ++row) {
        const int place = static_cast<int>(row - first) & 31;
        if (place == 0) bits = bits_of(row);
        const long long base = row * H;
        R* dx = static_cast<R*>(a.dx) + base;
        const float zero[8] = {};
        if (!(bits >> place & 1)) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int col = (j * WPR * 32 + t) * 8;
                if (col < H) store8(dx + col, zero);
            }
            continue;
        }
        if (row >= found_end) {
            const int inv = token_invocation(a, row, lane);
            found = invocation_model(a, inv);
            found_end = a.cu_seqlens[inv + 1];
            if (found < 0 && lane == 0) atomicOr(a.status, kStatusBadIndex);
        }
        const int m = found;
        if (m >= 0 && m != model) {
            flush();
            model = m;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int col = (j * WPR * 32 + t) * 8;
                if (col < H) {
                    float g[8];
                    load_gamma(a, m, col, g);
                    pairs_of(g, gamma[j]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[j][i] = 0;
            }
        }
        const int stage = done % stages;
        const unsigned char* in = ring + static_cast<size_t>(stage) * stage_bytes;
        const R* res = reinterpret_cast<const R*>(in);
        const __nv_bfloat16* dy = reinterpret_cast<const __nv_bfloat16*>(in + res_bytes);
        const R* dres = ring_dres ? reinterpret_cast<const R*>(in + res_bytes + dy_bytes) : a.dres ? static_cast<const R*>(a.dres) + base : nullptr;
        if (!ptx::mbar_wait(&full[stage], done / stages & 1, kWaitBudgetCycles) && lane == 0) atomicOr(a.status, kStatusTimeout);
        // r and dy stay in registers; sums of two columns side by side
        Pairs r[NV], d[NV];
        uint64_t squares = 0, dots = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = (j * WPR * 32 + t) * 8;
            if (col < H) {
                typename RawOf<R>::type raw_r;
                Raw16 raw_d;
                float f[8];
                load8(res + col, raw_r);
                load8(dy + col, raw_d);
                widen(raw_r, f);
                pairs_of(f, r[j]);
                widen(raw_d, f);
                pairs_of(f, d[j]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    squares = ptx::fma2(r[j][i], r[j][i], squares);
                    dots = ptx::fma2(ptx::mul2(d[j][i], gamma[j][i]), r[j][i], dots);
                }
            }
        }
        float lo, hi;
        float2 sum;
        ptx::unpack2(squares, lo, hi);
        sum.x = lo + hi;
        ptx::unpack2(dots, lo, hi);
        sum.y = lo + hi;
        // (a barrier: every thread is through with the row before, whose place in the ring takes the next one)
        sum = row_sum<WPR>(sum, slots, done & 1);
        if (warp == 0 && done > 0) ask();
        ++done;
        const float s = 1.f / sqrtf(sum.x / static_cast<float>(H) + a.eps);
        // With t = r s: dr = s (g - t mean(g t)) and dgamma's share is dy t.  Powers of s by themselves leave fp32 where rows are very
        // small or large: s^3 has no digits left from a root mean square of 4e12 on.
        const float c = -(sum.y / static_cast<float>(H)) * s;
        const uint64_t s2 = ptx::pack2(s, s), c2 = ptx::pack2(c, c);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = (j * WPR * 32 + t) * 8;
            if (col < H) {
                Pairs g;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint64_t t2 = ptx::mul2(r[j][i], s2);
                    if (DG && m >= 0) acc[j][i] = ptx::fma2(d[j][i], t2, acc[j][i]);
                    g[i] = ptx::mul2(ptx::fma2(t2, c2, ptx::mul2(d[j][i], gamma[j][i])), s2);
                }
                if (dres) {
                    typename RawOf<R>::type more;
                    float f[8];
                    Pairs p;
                    load8(dres + col, more);
                    widen(more, f);
                    pairs_of(f, p);
#pragma unroll
                    for (int i = 0; i < 4; ++i) g[i] = ptx::add2(g[i], p[i]);
                }
                float f[8];
                floats_of(g, f);
                if (m >= 0) store8(dx + col, f); else store8(dx + col, zero);
            }
        }
    }
    flush();
    if (DG && t == 0) a.touched[blockIdx.x] = touched;
}

// dgamma of 32 columns of one model: the block's 64 groups of eight lanes share the blocks' slices, each adds its own up in ascending
// order, then the groups in a fixed tree.
constexpr int kDgammaWarps = 16;
__global__ void __launch_bounds__(32 * kDgammaWarps) k_norm_dgamma(const __grid_constant__ NormArgs a, int slices) {
    begin();
    __shared__ float4 part[kDgammaWarps][8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k = blockIdx.y;
    const int col = blockIdx.x * 32 + (lane & 7) * 4, group = threadIdx.x >> 3;
    const float* from = a.parts + static_cast<long long>(k) * a.H + col;
    const long long pitch = static_cast<long long>(a.K) * a.H;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int b = group; b < slices; b += 4 * kDgammaWarps)
        if (a.touched[b] >> k & 1) {
            const float4 v = *reinterpret_cast<const float4*>(from + b * pitch);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
#pragma unroll
    for (int o = 8; o < 32; o <<= 1) {
        s.x += __shfl_xor_sync(kFull, s.x, o);
        s.y += __shfl_xor_sync(kFull, s.y, o);
        s.z += __shfl_xor_sync(kFull, s.z, o);
        s.w += __shfl_xor_sync(kFull, s.w, o);
    }
    if (lane < 8) part[warp][lane] = s;
    __syncthreads();
    if (threadIdx.x >= 8) return;
    s = part[0][lane];
    for (int w = 1; w < kDgammaWarps; ++w) {
        const float4 v = part[w][lane];
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    float4* out = reinterpret_cast<float4*>(a.dgamma[k] + col);
    if (a.accumulate) {
        const float4 v = *out;
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    *out = s;
}

template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, int bytes, cudaStream_t stream, const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int WPR, int NV>
cudaError_t fwd_rows(const NormArgs& a, cudaStream_t st) {
    const int rows = WPR == 1 ? kFwdRowsOfWarps : 1, threads = 32 * WPR * rows;
    const unsigned grid = static_cast<unsigned>((a.n_tok + rows - 1) / rows);
    if (a.residual == nullptr) return launch(k_norm_fwd<WPR, NV, __nv_bfloat16, false>, grid, threads, 0, st, a);
    if (a.res_bf16) return launch(k_norm_fwd<WPR, NV, __nv_bfloat16, true>, grid, threads, 0, st, a);
    return launch(k_norm_fwd<WPR, NV, float, true>, grid, threads, 0, st, a);
}
// The ring's depth and what it holds: as many rows as leave room for two blocks on an SM, or for one; a row's dres stays outside
// where two rows with it do not fit.
constexpr int kMaxRing = 220 * 1024;
static_assert(2 * UNITY_MAX_NORM_H * (4 + 2) <= kMaxRing, "two rows without dres");
struct Ring { int stages, dres, bytes; };
Ring ring_of(const NormArgs& a) {
    const int width = a.res_bf16 ? 2 : 4;
    Ring r;
    r.dres = a.dres != nullptr && 2 * a.H * (2 * width + 2) <= kMaxRing;
    const int stage = a.H * (width + 2 + (r.dres ? width : 0));
    r.stages = 110 * 1024 / stage;
    r.stages = r.stages < 2 ? 2 : r.stages > kMaxStages ? kMaxStages : r.stages;
    r.bytes = r.stages * stage;
    return r;
}
template <int WPR, int NV, typename R, bool DG>
cudaError_t bwd_launch(const NormArgs& a, int grid, cudaStream_t st) {
    const Ring r = ring_of(a);
    if (r.bytes > 47 * 1024) {                                    // (what a block has without asking)
        // The limit belongs to the function, whichever contexts and host threads launch it: always that of the largest ring, so that no
        // call takes away what another is about to use.
        const cudaError_t e = cudaFuncSetAttribute(k_norm_bwd<WPR, NV, R, DG>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxRing);
        if (e != cudaSuccess) return e;
    }
    return launch(k_norm_bwd<WPR, NV, R, DG>, grid, 32 * WPR, r.bytes, st, a, r.stages, r.dres);
}
template <int WPR, int NV>
cudaError_t bwd_rows(const NormArgs& a, int grid, cudaStream_t st) {
    if (a.res_bf16) return a.parts ? bwd_launch<WPR, NV, __nv_bfloat16, true>(a, grid, st) : bwd_launch<WPR, NV, __nv_bfloat16, false>(a, grid, st);
    return a.parts ? bwd_launch<WPR, NV, float, true>(a, grid, st) : bwd_launch<WPR, NV, float, false>(a, grid, st);
}

int vectors(int H, int wpr) { return (H / 8 + 32 * wpr - 1) / (32 * wpr); }   // of a lane

}  // namespace

cudaError_t launch_norm_fwd(const NormArgs& a, cudaStream_t st) {
    // the fewest warps per row with at most 8 vectors per lane
    int wpr = 1;
    while (vectors(a.H, wpr) > 8) wpr *= 2;
    switch (wpr * 16 + vectors(a.H, wpr)) {
#define UNITY_ROWS(W, N) case (W) * 16 + (N): return fwd_rows<W, N>(a, st);
        UNITY_ROWS(1, 1) UNITY_ROWS(1, 2) UNITY_ROWS(1, 3) UNITY_ROWS(1, 4) UNITY_ROWS(1, 5) UNITY_ROWS(1, 6) UNITY_ROWS(1, 7) UNITY_ROWS(1, 8)
        UNITY_ROWS(2, 5) UNITY_ROWS(2, 6) UNITY_ROWS(2, 7) UNITY_ROWS(2, 8)
        UNITY_ROWS(4, 5) UNITY_ROWS(4, 6) UNITY_ROWS(4, 7) UNITY_ROWS(4, 8)
        UNITY_ROWS(8, 5) UNITY_ROWS(8, 6) UNITY_ROWS(8, 7) UNITY_ROWS(8, 8)
    }
    return cudaErrorInvalidValue;
}

// Warps that share a row of the backward: the fewest with at most two vectors per lane.
static int bwd_warps(int H) {
    int wpr = 1;
    while (vectors(H, wpr) > 2) wpr *= 2;
    return wpr;
}
// Blocks of the backward, each with a slice of H floats per model for its share of dgamma: 16 warps on each of a B200's 148 SMs (a
// constant, since the workspace's size is asked for without a device), and four rows for a block at least where there are enough.
int norm_bwd_blocks(long long n_tok, int H) {
    const int wpr = bwd_warps(H), per_sm = wpr >= 16 ? 1 : 16 / wpr;
    const long long most = 148LL * per_sm, few = n_tok < 148 ? n_tok : n_tok < 4 * 148 ? 148 : (n_tok + 3) / 4;
    return static_cast<int>(few < most ? few : most);
}

cudaError_t launch_norm_bwd(const NormArgs& a, int blocks, cudaStream_t st, int* n_launches) {
    const int wpr = bwd_warps(a.H);
    cudaError_t e = cudaErrorInvalidValue;
    switch (wpr * 16 + vectors(a.H, wpr)) {
#undef UNITY_ROWS
#define UNITY_ROWS(W, N) case (W) * 16 + (N): e = bwd_rows<W, N>(a, blocks, st); break;
        UNITY_ROWS(1, 1) UNITY_ROWS(1, 2) UNITY_ROWS(2, 2) UNITY_ROWS(4, 2) UNITY_ROWS(8, 2) UNITY_ROWS(16, 2) UNITY_ROWS(32, 2)
    }
#undef UNITY_ROWS
    *n_launches += 1;
    if (e != cudaSuccess || a.parts == nullptr) return e;
    *n_launches += 1;
    return launch(k_norm_dgamma, dim3(a.H / 32, a.K), 32 * kDgammaWarps, 0, st, a, blocks);
}

}  // namespace unity
