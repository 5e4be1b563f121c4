// Global gradient norm of each model over a list of tensors, and the gradients scaled to a largest norm
// (unity_clip_grad_norm).  Two passes: squares, then norm, factor and scaling.  A block takes a run of consecutive chunks of the
// listed tensors and the second pass walks it from its end, where the first one left it in L2.  Sums are fp64 in a fixed order;
// every block of the second pass adds up the first one's partial sums by itself, so no block waits for another.
// HBM bounds it: two reads and a write, 1.76 ms for 1.09 G fp32 gradients to bf16 (10.9 GB at 6.2 TB/s), 0.97 ms for 919 M bf16 ones; 12 us
// for 1.6 M, where the launches count.  Holding gradients on chip between the passes would save at most what the caches have.
#include "internal.h"
#include "ptx.cuh"

namespace unity {

namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kThreads = 256;
// A chunk is 32 KB of what is read: 128 bytes in flight per thread, 128 KB on an SM with four blocks (half of that for bf16, as with
// chunks of as many elements, left 40 % of the rate).
__host__ __device__ constexpr int chunk_of(bool bf16) { return kThreads * 8 * (bf16 ? 8 : 4); }   // elements: vectors of eight

// Both kernels begin with this, before any access to global memory: they may be in place when the kernel before them ends, and wait
// for it to complete.
__device__ __forceinline__ void begin() {
    ptx::grid_launch_dependents();
    ptx::grid_wait();
}

template <int N>
struct ClipTable {
    int n;
    int launch;
    long long chunks;
    ClipEntry e[N];
};

// Elements before the first vector of eight (32 bytes of fp32, 16 of bf16).
__host__ __device__ inline long long head_of(const ClipEntry& e) {
    const uintptr_t width = e.src_bf16 ? 2 : 4, at = reinterpret_cast<uintptr_t>(e.src) / width % 8;
    const long long h = at ? 8 - static_cast<long long>(at) : 0;
    return h < e.n ? h : e.n;
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}
// The sum over the block, in every thread.
__device__ __forceinline__ double block_sum(double v, double (&slots)[kThreads / 32]) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = v;
    __syncthreads();
    v = slots[0];
#pragma unroll
    for (int w = 1; w < kThreads / 32; ++w) v += slots[w];
    return v;
}

__device__ __forceinline__ float element(const ClipEntry& e, long long i) {
    return e.src_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(e.src)[i]) : static_cast<const float*>(e.src)[i];
}
__device__ __forceinline__ void put(const ClipEntry& e, long long i, float v) {
    if (e.dst_bf16) static_cast<__nv_bfloat16*>(e.dst)[i] = __float2bfloat16_rn(v);
    else static_cast<float*>(e.dst)[i] = v;
}
// Eight elements from an aligned place (32 bytes of fp32 in one instruction).
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&f)[8]) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) { f[2 * k] = __uint_as_float(w[k] << 16); f[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u); }
}
__device__ __forceinline__ void load8(const float* p, float (&f)[8]) {
    asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]), "=f"(f[4]), "=f"(f[5]), "=f"(f[6]), "=f"(f[7]) : "l"(p) : "memory");
}
__device__ __forceinline__ void store8(const ClipEntry& e, long long i, const float (&f)[8], bool aligned) {
    if (!aligned) {
#pragma unroll
        for (int k = 0; k < 8; ++k) put(e, i + k, f[k]);
    } else if (e.dst_bf16) {
        unsigned w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * k], f[2 * k + 1]);
            w[k] = *reinterpret_cast<const unsigned*>(&b);
        }
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(e.dst) + i) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        ptx::st_global_v8(static_cast<float*>(e.dst) + i, __float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]),
                          __float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
    }
}

__device__ __forceinline__ double squares_in_64(const float (&f)[8]) {
    double s = 0.0;
    for (int k = 0; k < 8; ++k) s = fma(static_cast<double>(f[k]), static_cast<double>(f[k]), s);
    return s;
}
// Eight squares are added in fp32 where their sum lies far from both ends of the range (a square that underflows is then below 2^-30
// of it): eight roundings of one addition each, at most 8 2^-24 of the sum, 4 2^-24 of the norm, and all of one sign at worst.  Tiny,
// huge and zero vectors take 64 bits.
__device__ __forceinline__ double squares(const float (&f)[8]) {
    float q = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) q = fmaf(f[k], f[k], q);
    return q > 0x1p-90f && q < 0x1p120f ? static_cast<double>(q) : squares_in_64(f);
}

// The vectors of chunk `c` of the launch, which belongs to entry e: elements [i0, i1) of it, vectors in [v0, v1).
struct Span { long long i0, i1, v0, v1; };
__device__ __forceinline__ Span span_of(const ClipEntry& e, long long c) {
    const long long h = head_of(e), local = c - e.chunk0, chunk = chunk_of(e.src_bf16);
    Span s;
    s.v0 = h + local * chunk;
    s.i0 = local == 0 ? 0 : s.v0;
    s.i1 = s.v0 + chunk < e.n ? s.v0 + chunk : e.n;
    s.v1 = s.v0 + (s.i1 - s.v0) / 8 * 8;
    return s;
}
template <int N>
__device__ __forceinline__ int entry_of(const ClipTable<N>& t, long long c) {
    int lo = 0, hi = t.n - 1;                                   // the last entry with chunk0 <= c (empty tensors have none of their own)
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.e[mid].chunk0 <= c) lo = mid; else hi = mid - 1;
    }
    return lo;
}

template <typename T>
__device__ __forceinline__ double chunk_squares(const T* src, const Span& s) {
    constexpr int kEach = 16 / sizeof(T);
    double acc = 0.0;
    float f[kEach][8];
    if (s.v1 - s.v0 == kEach * kThreads * 8) {
        const T* p = src + s.v0 + threadIdx.x * 8;
#pragma unroll
        for (int j = 0; j < kEach; ++j) load8(p + j * kThreads * 8, f[j]);
#pragma unroll
        for (int j = 0; j < kEach; ++j) acc += squares(f[j]);
        return acc;
    }
    for (long long i = s.v0 + threadIdx.x * 8; i < s.v1; i += kThreads * 8) {
        load8(src + i, f[0]);
        acc += squares(f[0]);
    }
    return acc;
}

template <int N>
__global__ void __launch_bounds__(kThreads) k_grad_squares(const __grid_constant__ ClipArgs a, const __grid_constant__ ClipTable<N> t) {
    begin();
    __shared__ double slots[kThreads / 32], sums[UNITY_MAX_MODELS];
    const long long first = t.chunks * blockIdx.x / gridDim.x, last = t.chunks * (blockIdx.x + 1) / gridDim.x;
    if (threadIdx.x < UNITY_MAX_MODELS) sums[threadIdx.x] = 0.0;
    double acc = 0.0;
    int k = first < last ? entry_of(t, first) : 0, model = first < last ? t.e[k].model : -1;
    for (long long c = first; c < last; ++c) {
        while (k + 1 < t.n && t.e[k + 1].chunk0 <= c) ++k;
        const ClipEntry& e = t.e[k];
        if (e.model != model) {
            const double s = block_sum(acc, slots);
            if (threadIdx.x == 0) sums[model] += s;
            acc = 0.0;
            model = e.model;
        }
        const Span s = span_of(e, c);
        acc += e.src_bf16 ? chunk_squares(static_cast<const __nv_bfloat16*>(e.src), s) : chunk_squares(static_cast<const float*>(e.src), s);
        // up to seven elements before the vectors and seven behind them
        const long long i = s.i0 + threadIdx.x, tail = s.v1 + threadIdx.x;
        if (i < s.v0) { const double v = element(e, i); acc = fma(v, v, acc); }
        if (tail < s.i1) { const double v = element(e, tail); acc = fma(v, v, acc); }
    }
    if (model >= 0) {
        const double s = block_sum(acc, slots);
        if (threadIdx.x == 0) sums[model] += s;
    }
    __syncthreads();
    if (threadIdx.x < a.K) a.partial[(static_cast<long long>(t.launch) * kClipBlocks + blockIdx.x) * a.K + threadIdx.x] = sums[threadIdx.x];
}

// Norm of a model in fp64: the partial sums of all launches' blocks, shared among the threads in a fixed way.
__device__ __forceinline__ double model_norm(const ClipArgs& a, int model, double (&slots)[kThreads / 32]) {
    double s = 0.0;
    const long long n = a.n_launches == 1 ? a.blocks : static_cast<long long>(a.n_launches) * kClipBlocks;
    for (long long b = threadIdx.x; b < n; b += kThreads) s += a.partial[b * a.K + model];
    return sqrt(block_sum(s, slots));
}
// (a norm that is not a number gives a factor that is none)
__device__ __forceinline__ float factor_of(const ClipArgs& a, int model, double norm) {
    return !a.has_max || norm <= static_cast<double>(a.max_norm[model]) ? 1.f : static_cast<float>(static_cast<double>(a.max_norm[model]) / norm);
}

template <typename T>
__device__ __forceinline__ void chunk_scale(const ClipEntry& e, const Span& s, float coef, bool aligned) {
    constexpr int kEach = 16 / sizeof(T);
    const T* src = static_cast<const T*>(e.src);
    float f[kEach][8];
    if (s.v1 - s.v0 == kEach * kThreads * 8) {
        const long long i = s.v0 + threadIdx.x * 8;
#pragma unroll
        for (int j = 0; j < kEach; ++j) load8(src + i + j * kThreads * 8, f[j]);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
#pragma unroll
            for (int q = 0; q < 8; ++q) f[j][q] *= coef;
            store8(e, i + j * kThreads * 8, f[j], aligned);
        }
        return;
    }
    for (long long i = s.v0 + threadIdx.x * 8; i < s.v1; i += kThreads * 8) {
        load8(src + i, f[0]);
#pragma unroll
        for (int q = 0; q < 8; ++q) f[0][q] *= coef;
        store8(e, i, f[0], aligned);
    }
}

template <int N>
__global__ void __launch_bounds__(kThreads) k_grad_scale(const __grid_constant__ ClipArgs a, const __grid_constant__ ClipTable<N> t) {
    begin();
    __shared__ double slots[kThreads / 32];
    if (t.launch == 0 && blockIdx.x == 0) {
        for (int m = 0; m < a.K; ++m) {
            const double norm = model_norm(a, m, slots);
            if (threadIdx.x == 0) {
                a.norm[m] = static_cast<float>(norm);
                if (a.coef) a.coef[m] = factor_of(a, m, norm);
            }
        }
    }
    if (!a.write) return;
    const long long first = t.chunks * blockIdx.x / gridDim.x, last = t.chunks * (blockIdx.x + 1) / gridDim.x;
    int k = first < last ? entry_of(t, last - 1) : 0, model = -1;
    float coef = 1.f;
    for (long long c = last - 1; c >= first; --c) {
        while (t.e[k].chunk0 > c) --k;
        const ClipEntry& e = t.e[k];
        if (e.model != model) {
            model = e.model;
            coef = factor_of(a, model, model_norm(a, model, slots));
        }
        if (e.src == e.dst && coef == 1.f) continue;
        const Span s = span_of(e, c);
        const bool aligned = (reinterpret_cast<uintptr_t>(e.dst) / (e.dst_bf16 ? 2 : 4) + s.v0) % 8 == 0;
        if (e.src_bf16) chunk_scale<__nv_bfloat16>(e, s, coef, aligned);
        else chunk_scale<float>(e, s, coef, aligned);
        const long long i = s.i0 + threadIdx.x, tail = s.v1 + threadIdx.x;
        if (i < s.v0) put(e, i, element(e, i) * coef);
        if (tail < s.i1) put(e, tail, element(e, tail) * coef);
    }
}

template <int N, bool SCALE>
cudaError_t launch_table(const ClipArgs& a, const ClipEntry* entries, int n, long long chunks, int launch, cudaStream_t st) {
    ClipTable<N> t;
    t.n = n; t.launch = launch; t.chunks = chunks;
    for (int i = 0; i < n; ++i) t.e[i] = entries[i];
    cudaLaunchConfig_t cfg = {};
    // (with several launches the sums are over all blocks that each might have: those without a chunk write their zeros)
    cfg.gridDim = dim3(SCALE && !a.write ? 1 : SCALE || a.n_launches == 1 ? clip_blocks(chunks) : kClipBlocks);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return SCALE ? cudaLaunchKernelEx(&cfg, k_grad_scale<N>, a, t) : cudaLaunchKernelEx(&cfg, k_grad_squares<N>, a, t);
}

}  // namespace

long long clip_chunks(const ClipEntry& e) {
    const long long body = e.n - head_of(e);
    const long long chunk = chunk_of(e.src_bf16);
    return e.n == 0 ? 0 : (body <= chunk ? 1 : (body + chunk - 1) / chunk);
}
int clip_blocks(long long chunks) { return static_cast<int>(chunks < 1 ? 1 : (chunks < kClipBlocks ? chunks : kClipBlocks)); }

// Few tensors go with a small table: a launch's parameters are copied with it.
cudaError_t launch_grad_squares(const ClipArgs& a, const ClipEntry* entries, int n, long long chunks, int launch, cudaStream_t st) {
    return n <= 64 ? launch_table<64, false>(a, entries, n, chunks, launch, st) : launch_table<kClipEntries, false>(a, entries, n, chunks, launch, st);
}
cudaError_t launch_grad_scale(const ClipArgs& a, const ClipEntry* entries, int n, long long chunks, int launch, cudaStream_t st) {
    return n <= 64 ? launch_table<64, true>(a, entries, n, chunks, launch, st) : launch_table<kClipEntries, true>(a, entries, n, chunks, launch, st);
}

}  // namespace unity
