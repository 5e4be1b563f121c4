// Streaming kernels of the token losses (unity_cross_entropy_fwd_bwd, unity_distill_fwd_bwd): routing, packing with the
// teacher's lists, the per-row losses and gradient coefficients with their sums, the kept logits' conversion to gradients,
// and the outputs' last sums and roundings.
// Every sum has a fixed order and every output one writer: results are bitwise reproducible.
#include "internal.h"
#include "ptx.cuh"

namespace unity {

namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kMaxTop = UNITY_MAX_TOP;
constexpr int kNone = 0x7fffffff;

// Every launch of a token loss may overlap the end of the one before it (programmatic stream serialisation): its blocks are
// in place when that one ends.  So every kernel here begins with this, before any access to global memory; since each waits
// for its predecessor to complete, order is that of the stream.
__device__ __forceinline__ void begin() {
    ptx::grid_launch_dependents();
    ptx::grid_wait();
}
template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, cudaStream_t stream, const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

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

__device__ __forceinline__ long long warp_min64(long long v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const long long u = __shfl_xor_sync(kFull, v, o);
        v = u < v ? u : v;
    }
    return v;
}

// One warp: the parts of a contraction, a candidate per lane.
__device__ __forceinline__ SplitShape warp_split(const SplitParams& p, int m_tiles) {
    SplitShape s;
    long long best = 0x7fffffffffffffffll;
    const int c = (threadIdx.x & 31) + 1;
    static_assert(kMaxKSplits <= 32, "one candidate per lane");
    if (split_allowed(p, m_tiles, c)) best = split_candidate(p, m_tiles, c, s) * 64 + c;
    best = warp_min64(best);
    split_candidate(p, m_tiles, static_cast<int>(best & 63), s);
    return s;
}
// ... and the schedules of `rows` packed rows, `valid` of which hold tokens (the forward's is forward_shape's choice).
__device__ __forceinline__ void warp_shapes(const LossRouteArgs& a, int rows, int valid, FwdShape* fwd, SplitShape* dh, SplitShape* dw) {
    const int lane = threadIdx.x & 31;
    const FwdPlanParams& p = a.route.fwd;
    FwdShape f;
    const int m = rows / p.tile_rows, cand_min = forward_cand_min(p, m);
    long long best = 0x7fffffffffffffffll;
    for (int cand = p.gmax - lane; cand >= cand_min; cand -= 32) {
        const long long key = forward_candidate(p, m, cand, f) * 4096 + (p.gmax - cand);
        best = key < best ? key : best;
    }
    best = warp_min64(best);
    if (lane == 0) {
        forward_candidate(p, m, p.gmax - static_cast<int>(best & 4095), f);
        forward_finish(p, rows, m, f);
        *fwd = f;
    }
    const SplitShape h = warp_split(a.split, rows / a.split.tile_rows);
    SplitParams pw = a.split_dw;
    pw.k_iters = (valid + kTileK - 1) / kTileK;
    const SplitShape w = warp_split(pw, 1);
    if (lane == 0) { *dh = h; *dw = w; }
}

// Model w / 2, its full block or its last one, for w over the block's warps; then the models' statistics bases.
__device__ __forceinline__ void write_shapes(const LossRouteArgs& a, const int* off, const int* counts) {
    __shared__ long long sh_stats[UNITY_MAX_MODELS][2];
    for (int w = threadIdx.x >> 5; w < 2 * a.route.K; w += blockDim.x >> 5) {
        const int k = w >> 1, rows = off[k + 1] - off[k];
        const bool full = (w & 1) == 0;
        if (full && rows < a.block_rows) continue;             // no full block, no schedule of one
        FwdShape f;
        SplitShape h, d;
        const int here = full ? a.block_rows : rows % a.block_rows, valid = full ? here : counts[k] - (rows - here);
        warp_shapes(a, here, valid < here ? valid : here, &f, &h, &d);
        if ((threadIdx.x & 31) == 0) {
            a.shapes->fwd[k][w & 1] = f;
            a.shapes->dh[k][w & 1] = h;
            a.shapes->dw[k][w & 1] = d;
            sh_stats[k][w & 1] = f.stats_rows;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        long long base = 0;
        for (int j = 0; j < a.route.K; ++j) {
            a.route.plan->stats_base[j] = base;
            // (read only where a model is one block)
            const int rows = off[j + 1] - off[j];
            base += rows == 0 ? 0 : sh_stats[j][rows >= a.block_rows ? 0 : 1];
        }
    }
}
__global__ void __launch_bounds__(1024) k_loss_shapes(LossRouteArgs a) {
    begin();
    write_shapes(a, a.route.plan->off, a.route.plan->counts);
}

// Routing of all tokens by one block: thread t takes the tokens [t*per, t*per + per), counts them by model, and a scan over
// the warps gives every token its rank within its model, tokens in order.
template <int kThreads>
struct RouteShared {
    static constexpr int kCu = 1024;
    int cu[kCu];
    int cnt[UNITY_MAX_MODELS][kThreads / 32];
    int off[UNITY_MAX_MODELS + 1];     // first slot of each model
    int tot[UNITY_MAX_MODELS];         // its tokens
};
template <int kThreads, int kPer>
__device__ __forceinline__ void route_tokens(const RouteArgs& r, bool report, RouteShared<kThreads>& sh, int (&model)[kPer],
                                             int (&rank)[kPer]) {
    constexpr int kCu = RouteShared<kThreads>::kCu, kWarps = kThreads / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = static_cast<int>(r.n_tok);
    const int per = (n + kThreads - 1) / kThreads, i0 = tid * per;
    const bool staged = r.n_inv < kCu;
    if (staged) for (int s = tid; s <= r.n_inv; s += kThreads) sh.cu[s] = static_cast<int>(r.cu_seqlens[s]);
    bool on[kPer];
    int tgt[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const bool in = j < per && i0 + j < n;
        on[j] = in && (r.tok_mask ? r.tok_mask[i0 + j] != 0 : true);
        tgt[j] = in && r.target ? r.target[i0 + j] : 0;
        model[j] = -1;
        rank[j] = 0;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        if (!on[j]) continue;
        int lo = 0, hi = r.n_inv;                             // entries cu[1 .. n_inv] that are <= the token
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            const long long c = staged ? sh.cu[mid + 1] : r.cu_seqlens[mid + 1];
            if (c <= i0 + j) lo = mid + 1; else hi = mid;
        }
        const int role = r.inv_role[min(lo, r.n_inv - 1)];
        if (role >= 0 && role < r.n_roles && tgt[j] >= 0 && tgt[j] < r.V) model[j] = r.role_model[role];
        else if (report) atomicOr(r.status, kStatusBadIndex);
    }
    for (int k = 0; k < r.K; ++k) {
        int c = 0;
#pragma unroll
        for (int j = 0; j < kPer; ++j) c += model[j] == k;
        int incl = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(kFull, incl, o);
            if (lane >= o) incl += u;
        }
        int at = incl - c;
#pragma unroll
        for (int j = 0; j < kPer; ++j) if (model[j] == k) rank[j] = at++;
        if (lane == 31) sh.cnt[k][warp] = incl;
    }
    __syncthreads();
    for (int k = warp; k < r.K; k += kWarps) {
        const int c = lane < kWarps ? sh.cnt[k][lane] : 0;
        int incl = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(kFull, incl, o);
            if (lane >= o) incl += u;
        }
        if (lane < kWarps) sh.cnt[k][lane] = incl - c;
        if (lane == 31) sh.tot[k] = incl;
    }
    __syncthreads();
    if (tid <= r.K) {
        int off = 0;
        for (int k = 0; k < tid; ++k) off += (sh.tot[k] + kTileM - 1) / kTileM * kTileM;
        sh.off[tid] = off;
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) if (model[j] >= 0) rank[j] += sh.cnt[model[j]][warp];
    __syncthreads();
}

// ... and its result for the later launches.
template <int kThreads, int kPer>
__device__ __forceinline__ void write_routes(const LossRouteArgs& a, const RouteShared<kThreads>& sh, const int (&model)[kPer],
                                             const int (&rank)[kPer]) {
    const RouteArgs& r = a.route;
    const int tid = threadIdx.x, n = static_cast<int>(r.n_tok), per = (n + kThreads - 1) / kThreads, i0 = tid * per;
    for (int j = tid; j < a.n_counters; j += kThreads) a.counters[j] = 0u;
    if (tid <= r.K) {
        r.plan->off[tid] = sh.off[tid];
        if (tid < r.K) r.plan->counts[tid] = sh.tot[tid];
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        if (j >= per || i0 + j >= n) continue;
        const int slot = model[j] >= 0 ? sh.off[model[j]] + rank[j] : -1;
        r.tok_slot[i0 + j] = slot;
        if (slot >= 0) { r.slot_tok[slot] = i0 + j; continue; }
        if (a.tok_loss) a.tok_loss[i0 + j] = 0.f;
        if (a.lse) a.lse[i0 + j] = 0.f;
    }
    for (int k = 0; k < r.K; ++k)
        for (int s = sh.off[k] + sh.tot[k] + tid; s < sh.off[k + 1]; s += kThreads) r.slot_tok[s] = -1;
    write_shapes(a, sh.off, sh.tot);
}

// One block routes a whole batch of up to kLossRouteTokens tokens, in place of four memsets and three routing launches.
__global__ void __launch_bounds__(1024) k_loss_route(LossRouteArgs a) {
    begin();
    __shared__ RouteShared<1024> sh;
    int model[kLossRouteTokens / 1024], rank[kLossRouteTokens / 1024];
    route_tokens(a.route, true, sh, model, rank);
    write_routes(a, sh, model, rank);
}

// One warp's list: ascending, distinct vocabulary indexes with their teacher probabilities q.  Entries with a negative id are
// empty places, an id >= V is reported and counts as one, and so do entries of probability zero (a logit of -inf); equal ids
// add up in list order.  With at most 128 entries, four to a lane, a rank by counting (each entry is compared with all others,
// which sit in shared memory and are read four at a time) needs no sorting network.  Without targets the likeliest entry (the first
// of equal ones) is the row's "target", the one that the forward sweep keeps apart: a model as sure as its teacher is sure of that.
__device__ __forceinline__ void warp_list(const LossGatherArgs& a, long long slot, int tok, int (*sh_ids)[kMaxTop], float (*sh_qs)[kMaxTop]) {
    constexpr int kPer = kMaxTop / 32;
    const int lane = threadIdx.x & 31;
    int* sh_id = sh_ids[threadIdx.x >> 5];
    float* sh_q = sh_qs[threadIdx.x >> 5];
    const int* ids = a.top_ids + static_cast<long long>(tok) * a.n_top;
    const float* vals = a.top_vals + static_cast<long long>(tok) * a.n_top;
    int id[kPer];
    float x[kPer];
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int j = lane + 32 * u;
        id[u] = -1;
        x[u] = 0.f;
        if (j < a.n_top) {
            id[u] = ids[j];
            x[u] = vals[j];
        }
    }
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        if (id[u] >= a.V) { atomicOr(a.status, kStatusBadIndex); id[u] = -1; }
        if (id[u] >= 0) {
            if (a.logits) x[u] *= a.scale;
            m = fmaxf(m, x[u]);
        }
    }
    float sum = 1.f;
    if (a.logits) {
        m = warp_max(m);
        float s = 0.f;
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            // a list without an entry above -inf has no probabilities: its row is empty
            x[u] = id[u] >= 0 ? (x[u] == -INFINITY ? 0.f : expf(x[u] - m)) : 0.f;
            s += x[u];
        }
        sum = warp_sum(s);
    } else {
#pragma unroll
        for (int u = 0; u < kPer; ++u) x[u] = id[u] >= 0 ? expf(x[u]) : 0.f;
    }
    int n = 0;
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        x[u] = x[u] == 0.f ? 0.f : x[u] / sum;
        if (id[u] < 0 || x[u] == 0.f) id[u] = kNone;
        sh_id[lane + 32 * u] = id[u];
        n += __popc(__ballot_sync(kFull, id[u] != kNone));
    }
    __syncwarp();
    int rank[kPer] = {};
    for (int i = 0; i < a.n_top; i += 4) {
        const int4 v = *reinterpret_cast<const int4*>(sh_id + i);
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            if (32 * u >= a.n_top) break;
            const int j = lane + 32 * u;
            rank[u] += (v.x < id[u] || (v.x == id[u] && i < j)) + (v.y < id[u] || (v.y == id[u] && i + 1 < j)) +
                       (v.z < id[u] || (v.z == id[u] && i + 2 < j)) + (v.w < id[u] || (v.w == id[u] && i + 3 < j));
        }
    }
    __syncwarp();
#pragma unroll
    for (int u = 0; u < kPer; ++u)
        if (id[u] != kNone) { sh_id[rank[u]] = id[u]; sh_q[rank[u]] = x[u]; }
    __syncwarp();
    // sorted: the first of several equal ids takes their sum
    int kept = 0, best = kNone;
    float best_q = 0.f;
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int r = lane + 32 * u;
        const int mine = r < n ? sh_id[r] : kNone;
        const bool lead = r < n && (r == 0 || sh_id[r - 1] != mine);
        const unsigned leads = __ballot_sync(kFull, lead);
        if (lead) {
            float q = sh_q[r];
            for (int i = r + 1; i < n && sh_id[i] == mine; ++i) q += sh_q[i];
            const long long at = slot * a.n_top + kept + __popc(leads & ((1u << lane) - 1u));
            a.ids_p[at] = mine;
            a.q_p[at] = q;
            if (q > best_q) { best_q = q; best = mine; }
        }
        kept += __popc(leads);
    }
    if (lane == 0) a.cnt_p[slot] = kept;
    if (a.target == nullptr) {
        best = __reduce_min_sync(kFull, best_q == warp_max(best_q) ? best : kNone);
        if (lane == 0) a.target_p[slot] = best == kNone ? -1 : best;
    }
}

// One warp per packed row and per token, w: 128-bit copies of the hidden row (zeros for padding slots) with its target, and
// zeros for a masked token's gradient row; with teacher's lists, every second warp takes a row's list.
// `twice`: the row is packed low_rows rows further on as well.
__device__ __forceinline__ void gather_row(const LossGatherArgs& a, long long w, bool list, int n_slots, int tok, bool masked,
                                           bool twice, int (*sh_id)[kMaxTop], float (*sh_q)[kMaxTop]) {
    const int lane = threadIdx.x & 31, n16 = a.H >> 3;
    if (list) {
        if (w >= n_slots) return;                              // whole warps leave: only warp-wide barriers below
        if (tok < 0) { if (lane == 0) a.cnt_p[w] = 0; return; }
        warp_list(a, w, tok, sh_id, sh_q);
        return;
    }
    if (a.dHidden != nullptr && masked) {
        uint4* dst = reinterpret_cast<uint4*>(a.dHidden + w * a.H);
        for (int j = lane; j < n16; j += 32) dst[j] = make_uint4(0, 0, 0, 0);
    }
    if (w >= n_slots) return;
    uint4* dst = reinterpret_cast<uint4*>(a.hp + w * a.H);
    uint4* low = dst + static_cast<long long>(a.low_rows) * n16;
    if (tok < 0) {
        for (int j = lane; j < n16; j += 32) {
            dst[j] = make_uint4(0, 0, 0, 0);
            if (twice) low[j] = make_uint4(0, 0, 0, 0);
        }
        if (lane == 0) a.target_p[w] = 0;
        return;
    }
    const uint4* src = reinterpret_cast<const uint4*>(a.hidden + static_cast<long long>(tok) * a.H);
    for (int j0 = lane; j0 < n16; j0 += 256) {                 // eight loads in flight
        uint4 v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) if (j0 + 32 * u < n16) v[u] = src[j0 + 32 * u];
#pragma unroll
        for (int u = 0; u < 8; ++u) if (j0 + 32 * u < n16) dst[j0 + 32 * u] = v[u];
        if (twice) {
#pragma unroll
            for (int u = 0; u < 8; ++u) if (j0 + 32 * u < n16) low[j0 + 32 * u] = v[u];
        }
    }
    if (lane == 0 && a.target != nullptr) a.target_p[w] = a.target[tok];
}

__global__ void __launch_bounds__(256) k_loss_gather(LossGatherArgs a) {
    begin();
    __shared__ __align__(16) int sh_id[8][kMaxTop];
    __shared__ float sh_q[8][kMaxTop];
    long long w = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    const bool list = a.n_top > 0 && (w & 1);
    if (a.n_top > 0) w >>= 1;
    const int tok = w < a.max_slots ? a.slot_tok[w] : -1;      // (not written beyond off[K]: not used there)
    const bool masked = a.dHidden != nullptr && w < a.n_tok && a.tok_slot[w] < 0;
    gather_row(a, w, list, a.plan->off[a.K], tok, masked, false, sh_id, sh_q);
}

// Up to kLossPackTokens tokens: routing and packing in one launch.  Every block routes all tokens for itself (a few memory
// latencies, no waiting for another block); block 0 writes the result down and weighs the schedules while the others pack.
__global__ void __launch_bounds__(256) k_loss_pack(LossRouteArgs r, LossGatherArgs a) {
    begin();
    __shared__ RouteShared<256> sh;
    __shared__ short sh_tok[kLossPackTokens];                  // tokens by model and rank
    __shared__ signed char sh_model[kLossPackTokens];
    __shared__ __align__(16) int sh_id[8][kMaxTop];
    __shared__ float sh_q[8][kMaxTop];
    constexpr int kPer = kLossPackTokens / 256;
    int model[kPer], rank[kPer];
    route_tokens(r.route, blockIdx.x == 0, sh, model, rank);
    if (blockIdx.x == 0) { write_routes(r, sh, model, rank); return; }
    const int n = static_cast<int>(r.route.n_tok), per = (n + 255) / 256, i0 = threadIdx.x * per;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        if (j >= per || i0 + j >= n) continue;
        sh_model[i0 + j] = static_cast<signed char>(model[j]);
        if (model[j] < 0) continue;
        int first = 0;
        for (int k = 0; k < model[j]; ++k) first += sh.tot[k];
        sh_tok[first + rank[j]] = static_cast<short>(i0 + j);
    }
    __syncthreads();
    long long w = static_cast<long long>(blockIdx.x - 1) * 8 + (threadIdx.x >> 5);
    const bool list = a.n_top > 0 && (w & 1);
    if (a.n_top > 0) w >>= 1;
    int tok = -1, first = 0, rel = 0;
    bool low = false;                                          // the row's model has its rows twice
    for (int k = 0; k < r.route.K; ++k) {
        if (w >= sh.off[k] && w < sh.off[k + 1]) {
            rel = static_cast<int>(w) - sh.off[k];
            if (rel < sh.tot[k]) tok = sh_tok[first + rel];
            low = sh.tot[k] <= a.low_rows;
        }
        first += sh.tot[k];
    }
    // (a row whose place the first rows' second copies take is left alone, but for its list and its token's zeros)
    int n_slots = sh.off[r.route.K];
    if (!list && low && rel >= a.low_rows && rel < 2 * a.low_rows) n_slots = 0;
    gather_row(a, w, list, n_slots, tok, w < n && sh_model[w] < 0, low && rel < a.low_rows, sh_id, sh_q);
}

// One warp per packed row: merge the vocabulary splits' statistics (one lane per split), then the row's loss and what
// its gradient needs.  With d_v = lse - z_v, which for the target is log(1 + s / e): e = exp(z_target - ref) and s the sum of all
// other columns' terms, kept apart since the sweep (the digits of a sure token's small loss are those of s).  Where e is a small
// share of the sum, and for the other listed entries, d_v = scale*(ref - acc_v) + log(s + e):
//   cross entropy : l = (1-eps) d_y + eps (lse - mean z) + lam lse^2
//   distillation  : l = kd sum_v q_v (log q_v + d_v) + hard d_y
// A block's eight losses times their weights are one entry of `partial`; a model's rows start at a multiple of 256, so
// no entry mixes two models.
__global__ void __launch_bounds__(256) k_loss_rows(LossRowArgs a) {
    begin();
    __shared__ float sh_wl[8];
    __shared__ double sh_sum[8];
    __shared__ bool sh_last;
    const bool whole = a.block.model < 0;
    int lo = 0, n_rows = 0;
    if (whole) n_rows = a.plan->off[a.K];
    else span_resolve(a.block, lo, n_rows);
    if (blockIdx.x == 0 && threadIdx.x < a.K) {               // models without a row (of a block: without a first one)
        const int k = threadIdx.x;
        if (a.plan->counts[k] == 0 && (whole || k == a.block.model)) a.loss[k] = 0.f;
        if (a.with_grad) a.alpha[k] = a.scale / (a.has_norm ? a.norm[k] : fmaxf(static_cast<float>(a.plan->counts[k]), 1.f));
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long idx = static_cast<long long>(blockIdx.x) * 8 + warp;
    if (static_cast<long long>(blockIdx.x) * 8 >= n_rows) return;             // the whole block: spans are multiples of 128
    const int slot = lo + static_cast<int>(idx);
    const int tok = a.slot_tok[slot];
    int k = whole ? 0 : a.block.model;
    while (whole && k + 1 < a.K && slot >= a.plan->off[k + 1]) ++k;
    float wl = 0.f;
    if (tok < 0) {
        if (lane == 0 && a.with_grad) { a.row_lse[slot] = 0.f; a.coef_p[slot] = 0.f; a.coef_g[slot] = 0.f; a.target_g[slot] = 0.f; }
    } else {
        const int first = whole ? a.plan->off[k] : lo;
        const int span = min(whole ? a.plan->off[k + 1] - first : n_rows, a.block.row_cap);   // rows of the forward launch
        const FwdShape& fs = a.shapes->fwd[k][span == a.block.row_cap ? 0 : 1];
        long long pitch = span;
        const int r = slot - first;
        const float4* st = a.stats + (whole ? a.plan->stats_base[k] : 0) + r;
        int n_splits = fs.splits;
        const long long last_row0 = static_cast<long long>(fs.last_m0) * a.tile_rows;
        if (r >= last_row0) {                                 // swept in the launch's short last round
            st += static_cast<long long>(fs.splits) * pitch - last_row0;
            pitch -= last_row0;
            n_splits = fs.last_splits;
        }
        const float c = a.scale * 1.4426950408889634f;
        float m = -3.0e38f, s = 0.f, zsum = 0.f, zy = -INFINITY;
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
        const float e = exp2f((zy - m) * c);                  // 0 without a target
        const float log_s = logf(s + e);
        const float lse = a.scale * m + log_s;
        const float dy = e >= s * 0x1p-10f ? log1pf(s / e) : a.scale * (m - zy) + log_s;      // lse - z_y (unused without a target)
        const float w = a.tok_weight ? a.tok_weight[tok] : 1.f;
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
                kl += q * (logf(q) + (a.ids_p[base + j] == tgt ? dy : a.scale * (m - a.top_z[base + j]) + log_s));
                Q += q;
            }
            kl = warp_sum(kl);
            Q = warp_sum(Q);
            l = a.kd * kl + (a.hard > 0.f ? a.hard * dy : 0.f);
            cp = a.kd * Q + a.hard;
            gt = a.hard > 0.f ? a.kd * Q * expf(-dy) + a.hard * expm1f(-dy) : 0.f;
            if (a.with_grad) {
                for (int j = lane; j < cnt; j += 32) {         // the logits give way to the entries' gradients
                    const bool at = a.ids_p[base + j] == tgt;
                    const float d = at ? dy : a.scale * (m - a.top_z[base + j]) + log_s, q = a.q_p[base + j];
                    // Q p - q, of the target as Q (p - 1) + (Q - q): both may be near 1
                    const float p = at ? expm1f(-d) : expf(-d);
                    a.top_z[base + j] = w * (a.kd * (at ? Q * p + (Q - q) : Q * p - q) + a.hard * p);
                }
            }
        }
        wl = w * l;
        if (lane == 0) {
            if (a.tok_loss) a.tok_loss[tok] = l;
            if (a.lse) a.lse[tok] = lse;
            if (a.with_grad) { a.row_lse[slot] = lse; a.coef_p[slot] = w * cp; a.coef_g[slot] = w; a.target_g[slot] = w * gt; }
        }
    }
    if (lane == 0) sh_wl[warp] = wl;
    __syncthreads();
    if (threadIdx.x == 0) {
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) s += sh_wl[j];
        a.partial[slot >> 3] = s;
        __threadfence();
        sh_last = atomicAdd(a.ticket, 1u) + 1u == static_cast<unsigned>((n_rows + 7) / 8);
    }
    __syncthreads();
    if (!sh_last) return;
    // The block that finishes last adds up the entries of its models, in a fixed order: of a block's model, those of the
    // blocks before it too, so that the last block's launch leaves the whole sum.
    __threadfence();
    for (int k = whole ? 0 : a.block.model; k < (whole ? a.K : a.block.model + 1); ++k) {
        const int j0 = a.plan->off[k] >> 3, j1 = (whole ? a.plan->off[k + 1] : lo + n_rows) >> 3;
        if (a.plan->counts[k] == 0) continue;
        double s = 0.0;
        for (int j = j0 + threadIdx.x; j < j1; j += 256) s += __ldcg(a.partial + j);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
        if (lane == 0) sh_sum[warp] = s;
        __syncthreads();
        s = 0.0;
        for (int j = 0; j < 8; ++j) s += sh_sum[j];
        if (threadIdx.x == 0) a.loss[k] = static_cast<float>(s / (a.has_norm ? a.norm[k] : fmaxf(static_cast<float>(a.plan->counts[k]), 1.f)));
        __syncthreads();
    }
}

// One warp per row of the span: the gradients of its listed entries among columns [v0, v0 + cols) replace what the dense
// pass wrote there (which left out the teacher's part).
__global__ void __launch_bounds__(256) k_teacher_scatter(TeacherScatterArgs a) {
    begin();
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
// columns of one tile of the forward GEMM and has one reference.  2 B read and 2 B written per logit; eight resident blocks
// per SM walk the items (1200 rows x 151936: 134 us, 5.4 TB/s of the copy's 6.5; five blocks with more registers: 163 us; eight
// hold a thread to 32 registers, of which a few go through local memory).
constexpr int kGradVecs = 4;
constexpr int kGradCols = 256 * 8 * kGradVecs;
template <bool LOW>
__global__ void __launch_bounds__(256, LOW ? 6 : 8) k_loss_grad_inplace(LossGradArgs a) {
    begin();
    // the rows that the contractions read: of a block, or of every model (their slabs end with the last token)
    __shared__ int sh_off[UNITY_MAX_MODELS], sh_rows[UNITY_MAX_MODELS], sh_valid[UNITY_MAX_MODELS];
    const bool joint = a.span.model < 0;
    int row0 = 0, rows = 0, valid = 0;
    if (joint) {
        if (threadIdx.x < a.K) {
            const int k = threadIdx.x;
            sh_off[k] = a.span.plan->off[k];
            sh_valid[k] = a.span.plan->counts[k];
            sh_rows[k] = (sh_valid[k] + kTileK - 1) / kTileK * kTileK;
        }
        __syncthreads();
        for (int k = 0; k < a.K; ++k) rows += sh_rows[k];
    } else {
        span_resolve(a.span, row0, rows);
        rows = span_slab_rows(a.span, rows);
        valid = a.span.plan->counts[a.span.model] - a.span.row_begin;
    }
    const int per_row = (a.cols + kGradCols - 1) / kGradCols;
    for (int item = blockIdx.x; item < rows * per_row; item += gridDim.x) {      // at most 18432 rows of 2^18 columns
        int r = item / per_row;
        const int c_lo = (item - r * per_row) * kGradCols, c_first = c_lo + threadIdx.x * 8;
        bool low = false;                                      // the row's model has low halves
        if (joint) {
            int k = 0;
            while (r >= sh_rows[k]) r -= sh_rows[k++];
            valid = sh_valid[k] + sh_off[k];
            low = LOW && sh_valid[k] <= a.low_rows;
            r += sh_off[k];
        }
        const int slot = row0 + r;
        uint4* row = reinterpret_cast<uint4*>(a.Z + static_cast<long long>(r) * a.ld);
        uint4* low_row = LOW ? row + a.low_rows * (a.ld >> 3) : nullptr;
        if (r >= valid) {                                      // no token: zeros, whatever lies there
#pragma unroll
            for (int u = 0; u < kGradVecs; ++u) {
                const int c0 = c_first + u * 2048;
                if (c0 >= a.cols) continue;
                row[c0 >> 3] = make_uint4(0, 0, 0, 0);
                if (LOW && low) low_row[c0 >> 3] = make_uint4(0, 0, 0, 0);
            }
            continue;
        }
        const float* tm = a.tile_max + static_cast<long long>(r) * a.n_tiles;
        uint4 raw[kGradVecs];
        float shift[kGradVecs];
#pragma unroll
        for (int u = 0; u < kGradVecs; ++u) {
            const int c0 = c_first + u * 2048;
            raw[u] = make_uint4(0, 0, 0, 0);
            if (c0 < a.cols) { raw[u] = row[c0 >> 3]; shift[u] = tm[c0 / kTileN]; }
        }
        // the last step (p = 0) is looked for in all of the thread's 32 entries at once: 12 instructions, 28 vector by vector
        unsigned last = 0u;
#pragma unroll
        for (int u = 0; u < kGradVecs; ++u) last = __vimax3_u16x2(__vimax3_u16x2(last, raw[u].x, raw[u].y), raw[u].z, raw[u].w);
        const bool far = last >= 0xffff0000u || (last & 0xffffu) == 0xffffu;
        const float base = kRefRoom - a.row_lse[slot] * 1.4426950408889634f;
        const float cp = a.coef_p[slot], cu = a.coef_g[slot] * a.uniform, gt = a.target_g[slot];
        const int tgt = a.target_p[slot];
#pragma unroll
        for (int u = 0; u < kGradVecs; ++u) {
            const int c0 = c_first + u * 2048;
            if (c0 >= a.cols) continue;
            const float sh = fmaf(shift[u], a.c2, base);
            unsigned* w = reinterpret_cast<unsigned*>(&raw[u]);
            unsigned lw[4], gone = 0u;
            if (far) {
#pragma unroll
                for (int j = 0; j < 4; ++j) gone |= (((w[j] & 0xffffu) == 0xffffu ? 1u : 0u) | (w[j] >= 0xffff0000u ? 2u : 0u)) << (2 * j);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float u0 = __uint_as_float(__byte_perm(w[j], 0x4b000000u, 0x7610)) - 8388608.f;
                const float u1 = __uint_as_float(__byte_perm(w[j], 0x4b000000u, 0x7632)) - 8388608.f;
                const float g0 = fmaf(cp, ptx::ex2(fmaf(u0, -1.f / kStashSteps, sh)), -cu);
                const float g1 = fmaf(cp, ptx::ex2(fmaf(u1, -1.f / kStashSteps, sh)), -cu);
                const __nv_bfloat162 h = __floats2bfloat162_rn(g0, g1);
                w[j] = *reinterpret_cast<const unsigned*>(&h);
                if (LOW) {
                    const float2 f = __bfloat1622float2(h);
                    const __nv_bfloat162 l = __floats2bfloat162_rn(g0 - f.x, g1 - f.y);
                    lw[j] = *reinterpret_cast<const unsigned*>(&l);
                }
            }
            if (gone != 0u) {                                  // entries beyond the steps' range: p = 0 (or NaN, as the whole row)
                const float g = fmaf(0.f, base, -cu);
                const __nv_bfloat16 hi = __float2bfloat16_rn(g);
                const unsigned bits = __bfloat16_as_ushort(hi) * 0x10001u;
                const unsigned low = LOW ? __bfloat16_as_ushort(__float2bfloat16_rn(g - __bfloat162float(hi))) * 0x10001u : 0u;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const unsigned m = ((gone >> (2 * j) & 1u) ? 0xffffu : 0u) | ((gone >> (2 * j) & 2u) ? 0xffff0000u : 0u);
                    w[j] = (w[j] & ~m) | (bits & m);
                    if (LOW) lw[j] = (lw[j] & ~m) | (low & m);
                }
            }
            if (static_cast<unsigned>(tgt - c0) < 8u) {        // the target is among this thread's eight
                const __nv_bfloat16 hi = __float2bfloat16_rn(gt);
                const unsigned bits = __bfloat16_as_ushort(hi);
                const unsigned low = LOW ? __bfloat16_as_ushort(__float2bfloat16_rn(gt - __bfloat162float(hi))) : 0u;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (tgt - c0 == 2 * j) { w[j] = (w[j] & 0xffff0000u) | bits; if (LOW) lw[j] = (lw[j] & 0xffff0000u) | low; }
                    if (tgt - c0 == 2 * j + 1) { w[j] = (w[j] & 0x0000ffffu) | (bits << 16); if (LOW) lw[j] = (lw[j] & 0x0000ffffu) | (low << 16); }
                }
            }
            row[c0 >> 3] = raw[u];
            if (LOW && low) low_row[c0 >> 3] = make_uint4(lw[0], lw[1], lw[2], lw[3]);
        }
        if (a.n_top > 0) {                                     // the row's listed entries among this block's columns
            __syncthreads();
            const long long at = static_cast<long long>(slot) * a.n_top;
            const int cnt = a.cnt_p[slot];
            for (int j = threadIdx.x; j < cnt; j += 256) {
                const int c = a.ids_p[at + j] - c_lo;
                if (c < 0 || c >= kGradCols) continue;
                const float g = a.top_g[at + j];
                const __nv_bfloat16 hi = __float2bfloat16_rn(g);
                reinterpret_cast<__nv_bfloat16*>(row)[c_lo + c] = hi;
                if (LOW && low) reinterpret_cast<__nv_bfloat16*>(low_row)[c_lo + c] = __float2bfloat16_rn(g - __bfloat162float(hi));
            }
        }
    }
}

__device__ __forceinline__ float4 sum_parts(const float* src, int splits, long long stride) {
    float4 v = *reinterpret_cast<const float4*>(src);
    int s = 1;
    for (; s + 4 <= splits; s += 4) {                          // four loads in flight
        float4 o[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) o[u] = *reinterpret_cast<const float4*>(src + (s + u) * stride);
#pragma unroll
        for (int u = 0; u < 4; ++u) { v.x += o[u].x; v.y += o[u].y; v.z += o[u].z; v.w += o[u].w; }
    }
    for (; s < splits; ++s) {
        const float4 o = *reinterpret_cast<const float4*>(src + s * stride);
        v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
    }
    return v;
}
__device__ __forceinline__ uint2 pack4(float4 v) {
    const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
    return make_uint2(*reinterpret_cast<const unsigned*>(&lo), *reinterpret_cast<const unsigned*>(&hi));
}

// Four columns per thread: the parts added in their order, one rounding to bf16.
__global__ void __launch_bounds__(256) k_store_parts(StoreArgs a) {
    begin();
    const int per_row = a.H >> 2;
    const long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
    int r = static_cast<int>(i / per_row), model = a.span.model;
    const int c = static_cast<int>(i - static_cast<long long>(r) * per_row) * 4;
    int slot0 = 0, rows;
    const float* parts = a.parts;
    if (model < 0) {
        if (r >= a.span.plan->off[a.K]) return;
        model = 0;
        while (r >= a.span.plan->off[model + 1]) ++model;
        slot0 = a.span.plan->off[model];
        rows = min(a.span.plan->off[model + 1] - slot0, a.span.row_cap);
        r -= slot0;
        parts += model * a.part_stride;
    } else {
        span_resolve(a.span, slot0, rows);
    }
    if (r >= rows) return;
    const int tok = a.slot_tok[slot0 + r];
    const int splits = a.shapes ? a.shapes->dh[model][rows == a.span.row_cap ? 0 : 1].splits : a.parts_n;
    if (tok < 0) return;
    float4 v = sum_parts(parts + static_cast<long long>(r) * a.H + c, splits, static_cast<long long>(rows) * a.H);
    if (a.low_rows > 0 && a.span.plan->counts[model] <= a.low_rows) {
        const float4 l = sum_parts(parts + static_cast<long long>(r + a.low_rows) * a.H + c, splits, static_cast<long long>(rows) * a.H);
        v.x += l.x; v.y += l.y; v.z += l.z; v.w += l.w;
    }
    const float f = a.alpha[model];
    v.x *= f; v.y *= f; v.z *= f; v.w *= f;
    *reinterpret_cast<uint2*>(a.dHidden + static_cast<long long>(tok) * a.H + c) = pack4(v);
}

// The same for dW, four values per thread, plus the old value where it accumulates; zeros where the span has no token.
__global__ void __launch_bounds__(256) k_sum_dw(SumDwArgs a) {
    begin();
    const long long i = (static_cast<long long>(blockIdx.x) * 256 + threadIdx.x) * 4;
    if (i >= a.n) return;
    int slot0, rows;
    span_resolve(a.span, slot0, rows);
    if (rows <= 0 && a.add) return;
    const SplitShape& plan = a.shapes->dw[a.span.model][rows == a.span.row_cap ? 0 : 1];
    const int splits = rows > 0 ? parts_in_use(plan.splits, plan.per_split, span_slab_rows(a.span, rows) / kTileK) : 0;
    float4 v = rows > 0 ? sum_parts(a.parts + i, splits, a.n) : make_float4(0.f, 0.f, 0.f, 0.f);
    const float f = a.alpha ? a.alpha[a.span.model] : 1.f;
    v.x *= f; v.y *= f; v.z *= f; v.w *= f;
    if (a.out16 != nullptr) {
        uint2* out = reinterpret_cast<uint2*>(a.out16 + i);
        if (a.add) {
            const uint2 old = *out;
            v.x += __uint_as_float(old.x << 16); v.y += __uint_as_float(old.x & 0xffff0000u);
            v.z += __uint_as_float(old.y << 16); v.w += __uint_as_float(old.y & 0xffff0000u);
        }
        *out = pack4(v);
    } else {
        float4* out = reinterpret_cast<float4*>(a.out + i);
        if (a.add) { const float4 old = *out; v.x += old.x; v.y += old.y; v.z += old.z; v.w += old.w; }
        *out = v;
    }
}

// dst = bf16(*alpha * src (+ dst)): one rounding of the fp32 sum over all row blocks.  Eight values per thread and step.
__global__ void __launch_bounds__(256) k_cast_dw(const float4* __restrict__ src, uint4* __restrict__ dst, long long n8, const float* alpha, int add) {
    begin();
    const float f = *alpha;
    const long long stride = static_cast<long long>(gridDim.x) * blockDim.x;
    for (long long i = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x; i < n8; i += stride) {
        const float4 a = src[2 * i], b = src[2 * i + 1];
        float v[8] = {f * a.x, f * a.y, f * a.z, f * a.w, f * b.x, f * b.y, f * b.z, f * b.w};
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

cudaError_t launch_loss_pack(const LossRouteArgs& a, const LossGatherArgs& g, cudaStream_t stream, int* n_launches) {
    const long long work = (g.max_slots > g.n_tok ? g.max_slots : g.n_tok) * (g.n_top > 0 ? 2 : 1);
    const unsigned blocks = static_cast<unsigned>((work + 7) / 8);
    *n_launches += 1;
    if (g.n_tok <= kLossPackTokens) return launch(k_loss_pack, dim3(blocks + 1), 256, stream, a, g);
    cudaError_t e;
    if (g.n_tok <= kLossRouteTokens) {
        e = launch(k_loss_route, dim3(1), 1024, stream, a);
    } else {
        const size_t n = static_cast<size_t>(g.n_tok);
        if (a.tok_loss && (e = cudaMemsetAsync(a.tok_loss, 0, sizeof(float) * n, stream)) != cudaSuccess) return e;
        if (a.lse && (e = cudaMemsetAsync(a.lse, 0, sizeof(float) * n, stream)) != cudaSuccess) return e;
        if ((e = cudaMemsetAsync(a.route.slot_tok, 0xff, sizeof(int) * a.max_slots, stream)) != cudaSuccess) return e;
        if ((e = cudaMemsetAsync(a.counters, 0, sizeof(unsigned) * a.n_counters, stream)) != cudaSuccess) return e;
        RouteArgs r = a.route;                                 // (its statistics bases are written again below: the cheapest plan)
        r.fwd.gmax = 1;
        if ((e = launch_route(r, stream, n_launches)) != cudaSuccess) return e;
        e = launch(k_loss_shapes, dim3(1), 1024, stream, a);
    }
    if (e != cudaSuccess) return e;
    *n_launches += 1;
    return launch(k_loss_gather, dim3(blocks), 256, stream, g);
}

cudaError_t launch_loss_rows(const LossRowArgs& a, cudaStream_t stream) {
    const long long n = a.block.model >= 0 ? a.block.row_cap : a.max_slots;
    if (n <= 0) return cudaSuccess;
    return launch(k_loss_rows, dim3(static_cast<unsigned>((n + 7) / 8)), 256, stream, a);
}

cudaError_t launch_teacher_scatter(const TeacherScatterArgs& a, cudaStream_t stream) {
    return launch(k_teacher_scatter, dim3(static_cast<unsigned>((a.span.row_cap + 7) / 8)), 256, stream, a);
}

cudaError_t launch_loss_grad_inplace(const LossGradArgs& a, int sm_count, cudaStream_t stream) {
    const long long items = static_cast<long long>(a.span.row_cap) * ((a.cols + kGradCols - 1) / kGradCols);
    const long long blocks = 8ll * sm_count;                  // as many as are resident
    return launch(a.low_rows > 0 ? k_loss_grad_inplace<true> : k_loss_grad_inplace<false>, dim3(static_cast<unsigned>(items < blocks ? items : blocks)), 256, stream, a);
}

cudaError_t launch_store_parts(const StoreArgs& a, cudaStream_t stream) {
    return launch(k_store_parts, dim3(static_cast<unsigned>((a.bound * (a.H >> 2) + 255) / 256)), 256, stream, a);
}

cudaError_t launch_sum_dw(const SumDwArgs& a, cudaStream_t stream) {
    return launch(k_sum_dw, dim3(static_cast<unsigned>((a.n / 4 + 255) / 256)), 256, stream, a);
}

cudaError_t launch_cast_dw(const float* src, __nv_bfloat16* dst, long long n, const float* alpha, bool add, cudaStream_t stream) {
    return launch(k_cast_dw, dim3(1184), 256, stream, reinterpret_cast<const float4*>(src), reinterpret_cast<uint4*>(dst), n >> 3, alpha, add ? 1 : 0);
}

}  // namespace unity
