// RMS norm of token rows with one weight vector per model, and its backward (unity_rms_norm_fwd, unity_rms_norm_bwd).
// A row is held in the registers of the warps that share it: one read of its inputs, one write of its outputs, the sums over
// the columns in fp32.  dgamma is summed per block in registers over the block's rows, then over the blocks, both in a fixed
// order: no atomics.
#include "internal.h"
#include "ptx.cuh"

namespace unity {

namespace {

constexpr unsigned kFull = 0xffffffffu;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}

// Model of token `tok` by the whole warp: 32 places of the offsets are looked at per step (a role in 8192 invocations takes
// three dependent loads instead of thirteen).  -1: an id out of range, which is flagged.
__device__ __forceinline__ int token_model(const NormArgs& a, long long tok, int lane) {
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
    const int role = a.inv_role[min(lo, a.n_inv - 1)];
    if (role >= 0 && role < a.n_roles) return a.role_model[role];
    if (lane == 0) atomicOr(a.status, kStatusBadIndex);
    return -1;
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

template <typename T> struct RawOf;
template <> struct RawOf<__nv_bfloat16> { typedef Raw16 type; };
template <> struct RawOf<float> { typedef Raw32 type; };

// Sum of a pair over the WPR warps of a row; `slots` holds two of them in turn, so that one barrier per call is enough.
template <int WPR>
__device__ __forceinline__ float2 row_sum(float2 v, float2 (&slots)[2][WPR], int turn) {
    v.x = warp_sum(v.x);
    v.y = warp_sum(v.y);
    if (WPR == 1) return v;
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
// eight columns, 256 WPR columns apart.  The norm is taken of the fp32 sum; r is rounded only where it is written.
// ------------------------------------------------------------------------------------------------
constexpr int kFwdRowsOfWarps = 4;          // rows of a block whose rows belong to one warp each
template <int WPR, int NV, typename R, bool HAS_R>
__global__ void __launch_bounds__(WPR == 1 ? 32 * kFwdRowsOfWarps : 32 * WPR) k_norm_fwd(const __grid_constant__ NormArgs a) {
    __shared__ float2 slots[2][WPR];
    const int lane = threadIdx.x & 31;
    const int t = WPR == 1 ? lane : threadIdx.x;
    const long long row = WPR == 1 ? static_cast<long long>(blockIdx.x) * kFwdRowsOfWarps + (threadIdx.x >> 5) : blockIdx.x;
    if (row >= a.n_tok) return;                                  // (a whole warp, or a whole block)
    const int H = a.H;
    const long long base = row * H;
    bool on = a.tok_mask == nullptr || a.tok_mask[row] != 0;
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
        model = token_model(a, row, lane);
        on = model >= 0;
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
// dr = s g - r s^3 mean(g r) + dres with g = dy gamma; dgamma += dy r s.  A block takes a run of consecutive rows, so that its
// dgamma stays in registers; where the model changes it goes to the block's slice of that model and the next one begins.
// ------------------------------------------------------------------------------------------------
template <int WPR, int NV, typename R, bool DG>
__global__ void __launch_bounds__(32 * WPR) k_norm_bwd(const __grid_constant__ NormArgs a) {
    __shared__ float2 slots[2][WPR];
    const int lane = threadIdx.x & 31, t = threadIdx.x, H = a.H;
    const long long first = a.n_tok * blockIdx.x / gridDim.x, last = a.n_tok * (blockIdx.x + 1) / gridDim.x;
    float acc[NV][8];
    int model = -1, turn = 0;
    unsigned touched = 0;
    auto flush = [&]() {
        if (!DG || model < 0) return;
        float* slice = a.parts + (static_cast<long long>(blockIdx.x) * a.K + model) * H;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = (j * WPR * 32 + t) * 8;
            if (col < H) {
                if (touched >> model & 1) {
                    Raw32 r;
                    float f[8];
                    load8(slice + col, r);
                    widen(r, f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[j][i] += f[i];
                }
                store8(slice + col, acc[j]);
            }
        }
        touched |= 1u << model;
    };
    for (long long row = first; row < last; ++row) {
        const long long base = row * H;
        const bool on = a.tok_mask == nullptr || a.tok_mask[row] != 0;
        const int m = on ? token_model(a, row, lane) : -1;
        R* dx = static_cast<R*>(a.dx) + base;
        if (m < 0) {
            const float zero[8] = {};
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int col = (j * WPR * 32 + t) * 8;
                if (col < H) store8(dx + col, zero);
            }
            continue;
        }
        if (m != model) {
            flush();
            model = m;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[j][i] = 0.f;
        }
        typename RawOf<R>::type res[NV];
        Raw16 dy[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = (j * WPR * 32 + t) * 8;
            if (col < H) {
                load8(static_cast<const R*>(a.res) + base + col, res[j]);
                load8(a.dy + base + col, dy[j]);
            }
        }
        float2 sum = make_float2(0.f, 0.f);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = (j * WPR * 32 + t) * 8;
            if (col < H) {
                float r[8], d[8], g[8];
                widen(res[j], r);
                widen(dy[j], d);
                load_gamma(a, m, col, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    sum.x = fmaf(r[i], r[i], sum.x);
                    sum.y = fmaf(d[i] * g[i], r[i], sum.y);
                }
            }
        }
        sum = row_sum<WPR>(sum, slots, turn);
        turn ^= 1;
        const float s = 1.f / sqrtf(sum.x / static_cast<float>(H) + a.eps);
        const float c = s * s * s * (sum.y / static_cast<float>(H));
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = (j * WPR * 32 + t) * 8;
            if (col < H) {
                float r[8], d[8], g[8];
                widen(res[j], r);
                widen(dy[j], d);
                load_gamma(a, m, col, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    g[i] = s * (d[i] * g[i]) - c * r[i];
                    if (DG) acc[j][i] = fmaf(d[i], r[i] * s, acc[j][i]);
                }
                if (a.dres) {
                    typename RawOf<R>::type more;
                    load8(static_cast<const R*>(a.dres) + base + col, more);
                    widen(more, r);
#pragma unroll
                    for (int i = 0; i < 8; ++i) g[i] += r[i];
                }
                store8(dx + col, g);
            }
        }
    }
    flush();
    if (DG && t == 0) a.touched[blockIdx.x] = touched;
}

// dgamma of 128 columns of one model: the warps share the blocks' slices, each in ascending order, then warp by warp.
constexpr int kDgammaWarps = 16;
__global__ void __launch_bounds__(32 * kDgammaWarps) k_norm_dgamma(const __grid_constant__ NormArgs a, int slices) {
    __shared__ float4 part[kDgammaWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k = blockIdx.y;
    const int col = blockIdx.x * 128 + lane * 4;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (col < a.H) {
#pragma unroll 4
        for (int b = warp; b < slices; b += kDgammaWarps) {
            if (!(a.touched[b] >> k & 1)) continue;
            const float4 v = *reinterpret_cast<const float4*>(a.parts + (static_cast<long long>(b) * a.K + k) * a.H + col);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
    }
    part[warp][lane] = s;
    __syncthreads();
    if (warp != 0 || col >= a.H) return;
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

template <int WPR, int NV>
cudaError_t fwd_rows(const NormArgs& a, cudaStream_t st) {
    const int rows = WPR == 1 ? kFwdRowsOfWarps : 1, threads = 32 * WPR * rows;
    const unsigned grid = static_cast<unsigned>((a.n_tok + rows - 1) / rows);
    if (a.residual == nullptr) k_norm_fwd<WPR, NV, __nv_bfloat16, false><<<grid, threads, 0, st>>>(a);
    else if (a.res_bf16) k_norm_fwd<WPR, NV, __nv_bfloat16, true><<<grid, threads, 0, st>>>(a);
    else k_norm_fwd<WPR, NV, float, true><<<grid, threads, 0, st>>>(a);
    return cudaGetLastError();
}
template <int WPR, int NV>
cudaError_t bwd_rows(const NormArgs& a, int grid, cudaStream_t st) {
    if (a.res_bf16) {
        if (a.parts) k_norm_bwd<WPR, NV, __nv_bfloat16, true><<<grid, 32 * WPR, 0, st>>>(a);
        else k_norm_bwd<WPR, NV, __nv_bfloat16, false><<<grid, 32 * WPR, 0, st>>>(a);
    } else {
        if (a.parts) k_norm_bwd<WPR, NV, float, true><<<grid, 32 * WPR, 0, st>>>(a);
        else k_norm_bwd<WPR, NV, float, false><<<grid, 32 * WPR, 0, st>>>(a);
    }
    return cudaGetLastError();
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

// Blocks of the backward, each with a slice of H floats per model for its share of dgamma.
int norm_bwd_blocks(long long n_tok) {
    const long long most = 148 * 4;
    return static_cast<int>(n_tok < most ? n_tok : most);
}

cudaError_t launch_norm_bwd(const NormArgs& a, int blocks, cudaStream_t st, int* n_launches) {
    int wpr = 1;
    while (vectors(a.H, wpr) > 4) wpr *= 2;
    cudaError_t e = cudaErrorInvalidValue;
    switch (wpr * 16 + vectors(a.H, wpr)) {
#undef UNITY_ROWS
#define UNITY_ROWS(W, N) case (W) * 16 + (N): e = bwd_rows<W, N>(a, blocks, st); break;
        UNITY_ROWS(1, 1) UNITY_ROWS(1, 2) UNITY_ROWS(1, 3) UNITY_ROWS(1, 4)
        UNITY_ROWS(2, 3) UNITY_ROWS(2, 4) UNITY_ROWS(4, 3) UNITY_ROWS(4, 4)
        UNITY_ROWS(8, 3) UNITY_ROWS(8, 4) UNITY_ROWS(16, 3) UNITY_ROWS(16, 4)
    }
#undef UNITY_ROWS
    *n_launches += 1;
    if (e != cudaSuccess || a.parts == nullptr) return e;
    k_norm_dgamma<<<dim3((a.H + 127) / 128, a.K), 32 * kDgammaWarps, 0, st>>>(a, blocks);
    *n_launches += 1;
    return cudaGetLastError();
}

}  // namespace unity
