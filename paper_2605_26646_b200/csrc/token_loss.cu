// Streaming kernels of the token losses (unity_cross_entropy_fwd_bwd, unity_distill_fwd_bwd): the teacher's lists, the
// per-row losses and gradient coefficients, the loss sums, the listed entries' gradients and the cast of dW.
// Every sum has a fixed order and every output one writer: results are bitwise reproducible.
#include "internal.h"

namespace unity {

namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kMaxTop = UNITY_MAX_TOP;
constexpr int kNone = 0x7fffffff;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kFull, v, o));
    return v;
}

// One warp per packed row: the row's listed entries become ascending, distinct vocabulary indexes with their teacher
// probabilities q.  Entries with a negative id are empty places, an id >= V is reported and counts as one, and so do
// entries of probability zero (a logit of -inf); equal ids add up in list order.  With at most 128 entries a rank by
// counting (each entry is compared with all others, which sit in shared memory) needs no sorting network.
__global__ void __launch_bounds__(256) k_teacher_lists(TeacherArgs a) {
    __shared__ int sh_id[8][kMaxTop];
    __shared__ float sh_q[8][kMaxTop];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long slot = static_cast<long long>(blockIdx.x) * 8 + warp;
    if (slot >= a.plan->off[a.K]) return;                       // whole warps leave: only warp-wide barriers below
    const int tok = a.slot_tok[slot];
    if (tok < 0) {
        if (lane == 0) a.cnt_p[slot] = 0;
        return;
    }
    const int* ids = a.top_ids + static_cast<long long>(tok) * a.n_top;
    const float* vals = a.top_vals + static_cast<long long>(tok) * a.n_top;
    int id[kMaxTop / 32];
    float x[kMaxTop / 32];
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < kMaxTop / 32; ++u) {
        const int j = lane + 32 * u;
        id[u] = -1;
        x[u] = 0.f;
        if (j < a.n_top) {
            id[u] = ids[j];
            if (id[u] >= a.V) { atomicOr(a.status, kStatusBadIndex); id[u] = -1; }
            if (id[u] >= 0) {
                x[u] = a.logits ? vals[j] * a.scale : vals[j];
                m = fmaxf(m, x[u]);
            }
        }
    }
    float sum = 1.f;
    if (a.logits) {
        m = warp_max(m);
        float s = 0.f;
#pragma unroll
        for (int u = 0; u < kMaxTop / 32; ++u) {
            // a list without a finite or infinite-above entry (m = -inf) has no probabilities: its row is empty
            x[u] = id[u] >= 0 ? (x[u] == -INFINITY ? 0.f : expf(x[u] - m)) : 0.f;
            s += x[u];
        }
        sum = warp_sum(s);
    } else {
#pragma unroll
        for (int u = 0; u < kMaxTop / 32; ++u) x[u] = id[u] >= 0 ? expf(x[u]) : 0.f;
    }
#pragma unroll
    for (int u = 0; u < kMaxTop / 32; ++u) {
        const int j = lane + 32 * u;
        const float q = x[u] == 0.f ? 0.f : x[u] / sum;
        if (id[u] < 0 || q == 0.f) id[u] = kNone;
        if (j < a.n_top) { sh_id[warp][j] = id[u]; sh_q[warp][j] = q; }
    }
    __syncwarp();
    // pass 1: the first of several equal ids takes their sum
    bool lead[kMaxTop / 32];
    float q[kMaxTop / 32];
#pragma unroll
    for (int u = 0; u < kMaxTop / 32; ++u) {
        const int j = lane + 32 * u;
        lead[u] = j < a.n_top && id[u] != kNone;
        q[u] = 0.f;
        if (lead[u]) {
            for (int i = 0; i < a.n_top; ++i) {
                if (sh_id[warp][i] != id[u]) continue;
                if (i < j) { lead[u] = false; break; }
                q[u] += sh_q[warp][i];
            }
        }
    }
    __syncwarp();
#pragma unroll
    for (int u = 0; u < kMaxTop / 32; ++u) {
        const int j = lane + 32 * u;
        if (j < a.n_top && !lead[u]) sh_id[warp][j] = kNone;
    }
    __syncwarp();
    // pass 2: rank among the first ones
    int n = 0;
#pragma unroll
    for (int u = 0; u < kMaxTop / 32; ++u) {
        n += __popc(__ballot_sync(kFull, lead[u]));
        if (!lead[u]) continue;
        int rank = 0;
        for (int i = 0; i < a.n_top; ++i) rank += sh_id[warp][i] < id[u];
        a.ids_p[slot * a.n_top + rank] = id[u];
        a.q_p[slot * a.n_top + rank] = q[u];
    }
    if (lane == 0) a.cnt_p[slot] = n;
}

// One warp per packed row: merge the vocabulary splits' statistics (one lane per split), then the row's loss and what
// its gradient needs.  With d_v = lse - z_v (taken as scale*(max - acc_v) + log s, which keeps the digits of a sure
// token's small loss):
//   cross entropy : l = (1-eps) d_y + eps (lse - mean z) + lam lse^2
//   distillation  : l = kd sum_v q_v (log q_v + d_v) + hard d_y
// A block's eight losses times their weights are one entry of `partial`; a model's rows start at a multiple of 256, so
// no entry mixes two models.
__global__ void __launch_bounds__(256) k_loss_rows(LossRowArgs a) {
    __shared__ FwdShape sh_shape[UNITY_MAX_MODELS];
    __shared__ int sh_first[UNITY_MAX_MODELS], sh_rows[UNITY_MAX_MODELS];
    __shared__ long long sh_base[UNITY_MAX_MODELS];
    __shared__ int sh_lo, sh_hi;
    __shared__ float sh_wl[8];
    if (threadIdx.x < UNITY_MAX_MODELS) {
        const int k = threadIdx.x;
        int first = 0, rows = 0;
        long long base = 0;
        if (k < a.K) {
            if (a.block.model >= 0) {
                if (k == a.block.model) span_resolve(a.block, first, rows);
            } else {
                first = a.plan->off[k];
                rows = a.plan->off[k + 1] - first;
                base = a.plan->stats_base[k];
            }
        }
        sh_first[k] = first; sh_rows[k] = rows; sh_base[k] = base;
        if (rows > 0) sh_shape[k] = forward_shape(a.fwd, rows);
        if (k == 0) {
            if (a.block.model >= 0) { int f, r; span_resolve(a.block, f, r); sh_lo = f; sh_hi = f + r; }
            else { sh_lo = 0; sh_hi = a.plan->off[a.K]; }
        }
    }
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long idx = static_cast<long long>(blockIdx.x) * 8 + warp;
    if (static_cast<long long>(blockIdx.x) * 8 >= sh_hi - sh_lo) return;      // the whole block: spans are multiples of 128
    const int slot = sh_lo + static_cast<int>(idx);
    const int tok = a.slot_tok[slot];
    float wl = 0.f;
    if (tok < 0) {
        if (lane == 0 && a.with_grad) { a.row_lse[slot] = 0.f; a.coef_p[slot] = 0.f; a.coef_g[slot] = 0.f; a.target_g[slot] = 0.f; }
    } else {
        const int k = a.tok_model[tok];
        const FwdShape& fs = sh_shape[k];
        long long pitch = sh_rows[k];
        const int r = slot - sh_first[k];
        const float4* st = a.stats + sh_base[k] + r;
        int n_splits = fs.splits;
        const long long last_row0 = static_cast<long long>(fs.last_m0) * a.fwd.tile_rows;
        if (r >= last_row0) {                                 // swept in the launch's short last round
            st = a.stats + sh_base[k] + static_cast<long long>(fs.splits) * pitch + (r - last_row0);
            pitch -= last_row0;
            n_splits = fs.last_splits;
        }
        const float c = a.scale * 1.4426950408889634f;
        float m = -3.0e38f, s = 0.f, zsum = 0.f, zy = -3.0e38f;
        for (int j = lane; j < n_splits; j += 32) {
            const float4 p = st[j * pitch];
            const float mn = fmaxf(m, p.x);
            s = s * exp2f((m - mn) * c) + p.y * exp2f((p.x - mn) * c);
            m = mn;
            zsum += p.z;
            zy = fmaxf(zy, p.w);
        }
        const float m_all = warp_max(m);
        s = warp_sum(s * exp2f((m - m_all) * c));
        m = m_all;
        zsum = warp_sum(zsum);
        zy = warp_max(zy);
        const float log_s = logf(s);
        const float lse = a.scale * m + log_s;
        const float dy = a.scale * (m - zy) + log_s;          // lse - z_y (unused without a target)
        const float w = a.tok_weight ? a.tok_weight[tok] : 1.f;
        const float M = a.has_norm ? a.norm[k] : fmaxf(static_cast<float>(a.plan->counts[k]), 1.f);
        const float cg = a.scale * (w / M);
        float l, cp, gt;
        if (a.n_top == 0) {
            l = dy + a.z_loss * lse * lse;
            if (a.smoothing > 0.f) l = (1.f - a.smoothing) * dy + a.smoothing * (lse - a.scale * zsum / static_cast<float>(a.V)) + a.z_loss * lse * lse;
            const float twice = 2.f * a.z_loss * lse;
            cp = 1.f + twice;
            gt = expm1f(-dy) + twice * expf(-dy) + (a.smoothing - a.smoothing / static_cast<float>(a.V));
        } else {
            const long long base = static_cast<long long>(slot) * a.n_top;
            const int cnt = a.cnt_p[slot], tgt = a.target_p[slot];
            float kl = 0.f, Q = 0.f;
            for (int j = lane; j < cnt; j += 32) {
                const float q = a.q_p[base + j];
                kl += q * (logf(q) + (a.scale * (m - a.top_z[base + j]) + log_s));
                Q += q;
            }
            kl = warp_sum(kl);
            Q = warp_sum(Q);
            l = a.kd * kl + (a.hard > 0.f ? a.hard * dy : 0.f);
            cp = a.kd * Q + a.hard;
            gt = a.hard > 0.f ? cp * expf(-dy) - a.hard : 0.f;
            if (a.with_grad) {
                for (int j = lane; j < cnt; j += 32) {         // the logits give way to the entries' gradients
                    const float d = a.scale * (m - a.top_z[base + j]) + log_s;
                    const float own = a.kd * a.q_p[base + j] + (a.ids_p[base + j] == tgt ? a.hard : 0.f);
                    a.top_z[base + j] = cg * (cp * expf(-d) - own);
                }
            }
        }
        wl = w * l;
        if (lane == 0) {
            if (a.tok_loss) a.tok_loss[tok] = l;
            if (a.lse) a.lse[tok] = lse;
            if (a.with_grad) { a.row_lse[slot] = lse; a.coef_p[slot] = cg * cp; a.coef_g[slot] = cg; a.target_g[slot] = cg * gt; }
        }
    }
    if (lane == 0) sh_wl[warp] = wl;
    __syncthreads();
    if (threadIdx.x == 0) {
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) s += sh_wl[j];
        a.partial[slot >> 3] = s;
    }
}

// One block per model: its entries of `partial` in a fixed order.
__global__ void __launch_bounds__(256) k_loss_sum(LossRowArgs a) {
    __shared__ double sh[256];
    const int k = blockIdx.x;
    double s = 0.0;
    for (int j = (a.plan->off[k] >> 3) + threadIdx.x; j < (a.plan->off[k + 1] >> 3); j += 256) s += a.partial[j];
    sh[threadIdx.x] = s;
    __syncthreads();
    for (int o = 128; o > 0; o >>= 1) {
        if (threadIdx.x < o) sh[threadIdx.x] += sh[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        const float M = a.has_norm ? a.norm[k] : fmaxf(static_cast<float>(a.plan->counts[k]), 1.f);
        a.loss[k] = static_cast<float>(sh[0] / M);
    }
}

// One warp per row of the span: the gradients of its listed entries among columns [v0, v0 + cols) replace what the dense
// pass wrote there (which left out the teacher's part).
__global__ void __launch_bounds__(256) k_teacher_scatter(TeacherScatterArgs a) {
    const int lane = threadIdx.x & 31;
    int slot0, rows;
    span_resolve(a.span, slot0, rows);
    const int r = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (r >= rows) return;
    const long long base = static_cast<long long>(slot0 + r) * a.n_top;
    const int cnt = a.cnt_p[slot0 + r];
    for (int j = lane; j < cnt; j += 32) {
        const int c = a.ids_p[base + j] - a.v0;
        if (c >= 0 && c < a.cols) a.G[static_cast<long long>(r) * a.ld + c] = __float2bfloat16_rn(a.top_g[base + j]);
    }
}

// A block converts 8192 columns of a row: each thread issues four 128-bit loads 4 KiB apart, so a warp's access is the 256
// columns of one tile of the forward GEMM and has one reference.  2 B read and 2 B written per logit.
constexpr int kGradVecs = 4;
__global__ void __launch_bounds__(256) k_loss_grad_inplace(LossGradArgs a) {
    const int c_first = blockIdx.x * (256 * 8 * kGradVecs) + threadIdx.x * 8;
    int row0, rows;
    span_resolve(a.span, row0, rows);
    for (int r = blockIdx.y; r < rows; r += gridDim.y) {
        const int slot = row0 + r;
        uint4* row = reinterpret_cast<uint4*>(a.Z + static_cast<long long>(r) * a.ld);
        const float* tm = a.tile_max + static_cast<long long>(r) * a.n_tiles;
        uint4 raw[kGradVecs];
        float shift[kGradVecs];
#pragma unroll
        for (int u = 0; u < kGradVecs; ++u) {
            const int c0 = c_first + u * 2048;
            if (c0 < a.cols) { raw[u] = row[c0 >> 3]; shift[u] = tm[c0 / kTileN]; }
        }
        const float base = kRefRoom - a.row_lse[slot] * 1.4426950408889634f;
        const float cp = a.coef_p[slot], cu = a.coef_g[slot] * a.uniform, gt = a.target_g[slot];
        const int tgt = a.target_p[slot];
#pragma unroll
        for (int u = 0; u < kGradVecs; ++u) {
            const int c0 = c_first + u * 2048;
            if (c0 >= a.cols) continue;
            const float sh = fmaf(shift[u], a.c2, base);
            unsigned* w = reinterpret_cast<unsigned*>(&raw[u]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float u0 = __uint_as_float(__byte_perm(w[j], 0x4b000000u, 0x7610)) - 8388608.f;
                const float u1 = __uint_as_float(__byte_perm(w[j], 0x4b000000u, 0x7632)) - 8388608.f;
                float g0 = fmaf(cp, exp2f(fmaf(u0, -1.f / kStashSteps, sh)), -cu);
                float g1 = fmaf(cp, exp2f(fmaf(u1, -1.f / kStashSteps, sh)), -cu);
                if (c0 + 2 * j == tgt) g0 = gt;
                if (c0 + 2 * j + 1 == tgt) g1 = gt;
                const __nv_bfloat162 h = __floats2bfloat162_rn(g0, g1);
                w[j] = *reinterpret_cast<const unsigned*>(&h);
            }
            row[c0 >> 3] = raw[u];
        }
    }
}

// One block per row: four columns per thread and step, the parts added in their order, one rounding to bf16.
__global__ void __launch_bounds__(256) k_store_parts(StoreArgs a) {
    int slot0, rows;
    span_resolve(a.span, slot0, rows);
    const int r = blockIdx.x;
    if (r >= rows) return;
    const int tok = a.slot_tok[slot0 + r];
    if (tok < 0) return;
    __shared__ int sh_splits;
    if (threadIdx.x == 0)
        sh_splits = a.most != 0 ? split_shape(a.most, rows / a.tile_rows, a.n_tiles, a.k_iters, a.workers).splits : 1;
    __syncthreads();
    const int splits = sh_splits;
    const long long stride = static_cast<long long>(rows) * a.H;
    const float* src = a.parts + static_cast<long long>(r) * a.H;
    __nv_bfloat16* dst = a.dHidden + static_cast<long long>(tok) * a.H;
    for (int c = threadIdx.x * 4; c < a.H; c += 1024) {
        float4 v = *reinterpret_cast<const float4*>(src + c);
        for (int s = 1; s < splits; ++s) {
            const float4 o = *reinterpret_cast<const float4*>(src + s * stride + c);
            v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
        }
        const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
        *reinterpret_cast<uint2*>(dst + c) = make_uint2(*reinterpret_cast<const unsigned*>(&lo), *reinterpret_cast<const unsigned*>(&hi));
    }
}

// dst = bf16(src) (+ dst): one rounding of the fp32 sum over all row blocks.  Eight values per thread and step.
__global__ void __launch_bounds__(256) k_cast_dw(const float4* __restrict__ src, uint4* __restrict__ dst, long long n8, int add) {
    const long long stride = static_cast<long long>(gridDim.x) * blockDim.x;
    for (long long i = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x; i < n8; i += stride) {
        const float4 a = src[2 * i], b = src[2 * i + 1];
        float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        uint4 o;
        unsigned* ow = reinterpret_cast<unsigned*>(&o);
        if (add) {
            const uint4 old = dst[i];
            const unsigned* pw = reinterpret_cast<const unsigned*>(&old);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[2 * j] += __uint_as_float(pw[j] << 16);
                v[2 * j + 1] += __uint_as_float(pw[j] & 0xffff0000u);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
            ow[j] = *reinterpret_cast<const unsigned*>(&h);
        }
        dst[i] = o;
    }
}

}  // namespace

cudaError_t launch_teacher_lists(const TeacherArgs& a, long long max_slots, cudaStream_t stream) {
    k_teacher_lists<<<static_cast<unsigned>((max_slots + 7) / 8), 256, 0, stream>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_loss_rows(const LossRowArgs& a, cudaStream_t stream) {
    const long long n = a.block.model >= 0 ? a.block.row_cap : a.max_slots;
    if (n <= 0) return cudaSuccess;
    k_loss_rows<<<static_cast<unsigned>((n + 7) / 8), 256, 0, stream>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_loss_sum(const LossRowArgs& a, cudaStream_t stream) {
    k_loss_sum<<<a.K, 256, 0, stream>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_teacher_scatter(const TeacherScatterArgs& a, cudaStream_t stream) {
    k_teacher_scatter<<<static_cast<unsigned>((a.span.row_cap + 7) / 8), 256, 0, stream>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_loss_grad_inplace(const LossGradArgs& a, cudaStream_t stream) {
    const int gx = (a.cols + 256 * 8 * kGradVecs - 1) / (256 * 8 * kGradVecs);
    const int gy = a.span.row_cap < 32768 ? a.span.row_cap : 32768;
    if (gy <= 0) return cudaSuccess;
    k_loss_grad_inplace<<<dim3(gx, gy), 256, 0, stream>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_store_parts(const StoreArgs& a, cudaStream_t stream) {
    k_store_parts<<<a.span.row_cap, 256, 0, stream>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_cast_dw(const float* src, __nv_bfloat16* dst, long long n, bool add, cudaStream_t stream) {
    k_cast_dw<<<1184, 256, 0, stream>>>(reinterpret_cast<const float4*>(src), reinterpret_cast<uint4*>(dst), n >> 3, add ? 1 : 0);
    return cudaGetLastError();
}

}  // namespace unity
